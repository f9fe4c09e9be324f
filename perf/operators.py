"""Operators of microscaled 4-bit weights (MX4) and of products grouped by expert: the calls by
which their speed is judged, beside the same in plain torch.

A block of 32 consecutive elements of a row holds 4-bit E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and
their negatives) and one E8M0 scale, a power of two. A blob of n x k is the codes of the rows, two a
byte, the even one in the low bits, then one byte of scale a block. Y = X W'^T of fp16 rows X, or of
rows rounded to the same format; grouped by expert, rows offsets[e] .. offsets[e + 1] - 1 of X are
multiplied with the matrix of expert e.

A case is a dict:
  op       quantize | gemm | gemm_a4 | grouped | grouped_a4
  n, k, m  output features, reduction length, rows of activations
  experts  matrices of a grouped product (else 0)
  weights  mx4, or for `grouped` uniform codes (u3g64, u4g128, ..) or codebooks (c3g128, c4g64, ..)
"""
import math
import random

import torch

own = False

DEV = "cuda"
GROUPED = ["mx4", "mx4", "mx4", "u4g128", "u4g64", "u4g32", "u3g64", "u3g128", "c4g64", "c4g128", "c3g128"]


def _case(op, n, k, m, experts=0, weights="mx4"):
    return {"op": op, "n": n, "k": k, "m": m, "experts": experts, "weights": weights}


def listed():
    return [
        # activations of 16 sequences rounded to 4 bits and back: the smallest call, launches count
        dict(_case("quantize", 0, 4096, 16), name="quantize_m16"),
        # the gate|up matrix of a 7B decoder (hidden 4096, MLP 11008) rounded where it lies
        dict(_case("quantize", 0, 4096, 22016), name="quantize_gate_up"),
        # one projection of one token
        dict(_case("gemm", 4096, 4096, 1), name="gemv_4096"),
        # gate|up for 8 sequences decoded together
        dict(_case("gemm", 22016, 4096, 8), name="decode_m8"),
        # one MLP matrix for prompts of 2001 tokens together, fp16 activations
        dict(_case("gemm", 11008, 4096, 2001), name="prefill_m2001"),
        # the down projection of 16 sequences, weights and activations in 4 bits
        dict(_case("gemm_a4", 4096, 11008, 16), name="a4_decode_m16"),
        # gate|up for 4096 prompt tokens, both in 4 bits: the largest product
        dict(_case("gemm_a4", 22016, 4096, 4096), name="a4_prefill_m4096"),
        # a decode step of 8 sequences, 4 of 32 experts each: experts with a few rows, and none
        dict(_case("grouped", 2816, 4096, 32, 32), name="experts_decode"),
        # down projections of the experts for 1000 prompt tokens, 4 experts each, a ragged last one
        dict(_case("grouped", 4096, 1408, 4001, 32), name="experts_prefill"),
        # 8 experts as the framework's 4-bit uniform weights, one of 8 shards of an MLP
        dict(_case("grouped", 1376, 4096, 999, 8, "u4g128"), name="experts_u4_shard"),
        # decoding with many small experts, both sides in 4 bits
        dict(_case("grouped_a4", 2816, 2048, 48, 64), name="experts_a4_decode"),
        # the prompts of several users through the experts, both sides in 4 bits
        dict(_case("grouped_a4", 2816, 4096, 8192, 32), name="experts_a4_prefill"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = work(listed()[6])["flops"]
    while True:
        op = rng.choice(["quantize", "gemm", "gemm", "gemm_a4", "gemm_a4", "grouped", "grouped", "grouped_a4"])
        k = 128 * _log_int(rng, 4, 88)
        if op == "quantize":
            c = _case(op, 0, k, _log_int(rng, 1, 22016))
        else:
            n = _log_int(rng, 256, 22016)
            if rng.random() < 0.5:  # sizes of layers are mostly multiples of 16
                n = (n + 15) // 16 * 16
            grouped = op.startswith("grouped")
            m = _log_int(rng, 4 if grouped else 1, 8192 if grouped else 4096)
            c = _case(op, n, k, m, _log_int(rng, 4, 64) if grouped else 0,
                      rng.choice(GROUPED) if op == "grouped" else "mx4")
        if c["k"] * max(c["m"], c["n"] * max(1, c["experts"])) <= 370_000_000 and work(c)["flops"] <= most:
            return c


# ------------------------------------------------------------------ weights, rows and routes
def _gen(seed, at):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + at + 1) % (1 << 62))
    return g


def _counts(case):
    """Rows of every expert: as a router shares them, some experts three times as often as others."""
    r = random.Random(case["experts"] * 1000003 + case["m"])
    share = [math.exp(0.7 * r.gauss(0, 1)) for _ in range(case["experts"])]
    count = [0] * case["experts"]
    for e in r.choices(range(case["experts"]), share, k=case["m"]):
        count[e] += 1
    return count


def _offsets(case, seed):
    """Where the rows of every expert begin: the counts in an order that the seed gives."""
    count = _counts(case)
    random.Random(seed).shuffle(count)
    at = [0]
    for c in count:
        at.append(at[-1] + c)
    return at


def _rows(case, seed):
    """Activations N(0, 1) with 1 % outlier channels of twenty times the size; for `quantize` of a
    whole matrix, and of its rows, the same."""
    g = _gen(seed, 0)
    x = torch.randn(case["m"], case["k"], generator=g, device=DEV)
    x[:, torch.randperm(case["k"], generator=g, device=DEV)[: round(0.01 * case["k"])]] *= 20
    return x.half()


def _groups(seed, e, n, k, size):
    """Weights of expert e, N(0, 0.02) with rows of different size, in groups."""
    g = _gen(seed, 1 + e)
    w = torch.randn(n, k // size, size, generator=g, device=DEV)
    return w * (0.01 + 0.02 * torch.rand(n, 1, 1, generator=g, device=DEV))


def _mx4(seed, e, n, k):
    """Codes [n][k / 32][32] and scale codes [n][k / 32] of one matrix."""
    w = _groups(seed, e, n, k, 32)
    s = torch.frexp(w.abs().amax(-1)).exponent - 3  # floor(log2) - 2
    v = torch.ldexp(w, -s.unsqueeze(-1))
    a = v.abs()
    code = ((a > 0.25).byte() + (a > 0.75) + (a > 1.25) + (a > 1.75) + (a > 2.5) + (a > 3.5) + (a > 5))
    return code + 8 * (v < 0).byte(), (s + 127).byte()


def _table(seed, e, n, k, fmt):
    """Codes [n][groups][size] and the tables of one matrix in a format of uniform codes or codebooks."""
    bits, size = int(fmt[1]), int(fmt[3:])
    w = _groups(seed, e, n, k, size)
    last = (1 << bits) - 1
    if fmt[0] == "u":
        lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
        s = ((hi - lo) / last).half()
        z = (-lo / s).round().clamp(0, last)
        code = ((w / s.float().unsqueeze(-1)).round() + z.unsqueeze(-1)).clamp(0, last).byte()
        return code, torch.stack([s, z.half()], -1)
    t = torch.linspace(-1, 1, last + 1, device=DEV)
    jit = 0.9 + 0.2 * torch.rand(n, k // size, 1, generator=_gen(seed, 1000 + e), device=DEV)
    book = (t.sign() * t.abs() ** 1.4 * jit * w.abs().amax(-1, keepdim=True)).half()
    code = torch.zeros(w.shape, dtype=torch.uint8, device=DEV)
    for i in range(last):
        code += w > ((book[..., i].float() + book[..., i + 1].float()) / 2).unsqueeze(-1)
    return code, book


def _planes(code, bits):
    """The codes region of the framework's 3- and 4-bit layout: chunks of 128 codes in slices of 16
    bytes, slice s of all chunks of a row together."""
    n = code.shape[0]
    c = code.reshape(n, -1, 128)
    if bits == 4:
        chunk = c[..., 0::2] | (c[..., 1::2] << 4)
    else:
        chunk = c[..., :48] | (c[..., 48:96] << 3)
        spare = c[..., 96:]
        chunk[..., :32] |= (spare & 3) << 6
        chunk[..., 32:] |= ((spare[..., :16] >> 2) << 6) | ((spare[..., 16:] >> 2) << 7)
    return chunk.view(n, -1, bits, 16).transpose(1, 2).reshape(-1)


def _blob(case, seed, e):
    """One matrix as the framework keeps it, and for formats that plain torch does not read there its
    codes and tables."""
    n, k, fmt = case["n"], case["k"], case["weights"]
    if fmt == "mx4":
        code, scale = _mx4(seed, e, n, k)
        return torch.cat([(code[..., 0::2] | (code[..., 1::2] << 4)).reshape(-1), scale.view(-1)]), None
    code, table = _table(seed, e, n, k, fmt)
    return torch.cat([_planes(code, int(fmt[1])), table.reshape(-1).view(torch.uint8)]), (code, table)


def prepare(case, seed):
    state = dict(case, x=_rows(case, seed))
    if case["op"] == "quantize":
        return state
    if not case["experts"]:
        state["blob"] = _blob(case, seed, 0)[0]
        return state
    first, raw = _blob(case, seed, 0)
    # one row of the tensor an expert, each starting at a multiple of 16 bytes
    state["blob"] = torch.zeros(case["experts"], (first.numel() + 15) // 16 * 16, dtype=torch.uint8, device=DEV)
    raws = []
    for e in range(case["experts"]):
        blob, raw = _blob(case, seed, e)
        state["blob"][e, : blob.numel()] = blob
        raws.append(raw)
    if raws[0] is not None:
        state["codes"] = torch.stack([c for c, _ in raws])
        state["tables"] = torch.stack([t for _, t in raws])
    at = _offsets(case, seed)
    state["offsets"] = torch.tensor(at, dtype=torch.int32, device=DEV)
    state["most"] = max(b - a for a, b in zip(at, at[1:]))
    return state


# ------------------------------------------------------------------ one pass
def _own(state):
    import paper_2505_07531_amd as qx

    op, x, fmt = state["op"], state["x"], state["weights"]
    if op == "quantize":
        return qx.quantize_mx4(x).dequant()
    kind = {"m": qx.QX_MX4, "u": qx.QX_UNIFORM, "c": qx.QX_CODEBOOK}[fmt[0]]
    bits, size = (4, 32) if fmt == "mx4" else (int(fmt[1]), int(fmt[3:]))
    d = qx.desc(state["n"], state["k"], bits, size, kind)
    if state["experts"]:
        w = qx.PackedExperts(d, state["blob"])
        return w.gemm(x, state["offsets"]) if op == "grouped" else w.gemm_a4(qx.quantize_mx4(x), state["offsets"])
    w = qx.PackedWeight.from_blob(d, state["blob"])
    if op == "gemm_a4":
        return w.gemm_a4(qx.quantize_mx4(x))
    return w.gemm(x) if state["m"] > 1 else w.gemv(x[0])


def _rounded(x):
    """The rows' MX4 values, in 32 bits."""
    b = x.float().view(x.shape[0], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    scale = torch.ldexp(torch.ones_like(top), torch.frexp(top).exponent - 3)
    a = b.abs() / scale
    # steps between neighbouring values; a tie goes to the even code
    v = 0.5 * (a > 0.25) + 0.5 * (a >= 0.75) + 0.5 * (a > 1.25) + 0.5 * (a >= 1.75) + (a > 2.5) + 1.0 * (a >= 3.5) + 2.0 * (a > 5)
    return (torch.sign(b) * v * scale).view(x.shape)


def _weights(state):
    """W' in 32 bits, [n][k] or [experts][n][k]."""
    n, k, fmt = state["n"], state["k"], state["weights"]
    if fmt == "mx4":
        blob = state["blob"]
        lead = list(blob.shape[:-1]) + [n]
        code = blob[..., : n * k // 2].reshape(*lead, k // 32, 16)
        scale = blob[..., n * k // 2 : n * k // 2 + n * k // 32].reshape(*lead, k // 32, 1)
        code = torch.stack([code & 15, code >> 4], -1).flatten(-2)
        low = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=blob.device)
        values = torch.cat([low, -low])
        return (values[code.int()] * torch.exp2(scale.float() - 127)).view(*lead, k)
    if fmt[0] == "u":
        t = state["tables"].float()
        w = (state["codes"].float() - t[..., 1:]) * t[..., :1]
    else:
        w = state["tables"].float().gather(-1, state["codes"].long())
    return w.view(-1, n, k)


def run(state):
    if own:
        return _own(state)
    op, x = state["op"], state["x"]
    if op == "quantize":
        return _rounded(x).half()
    w = _weights(state)
    x = _rounded(x) if op.endswith("a4") else x.float()
    if not state["experts"]:
        return (x @ w.t()).half() if state["m"] > 1 or op == "gemm_a4" else (w @ x[0]).half()
    # every expert's rows at the head of a slot of `most` rows
    at = torch.arange(state["m"], device=x.device)
    expert = torch.searchsorted(state["offsets"][1:].long(), at, right=True)
    row = at - state["offsets"].long()[expert]
    slots = x.new_zeros(state["experts"], state["most"], state["k"])
    slots[expert, row] = x
    return torch.bmm(slots, w.transpose(1, 2))[expert, row].half()


def _blob_bytes(n, k, fmt):
    if fmt == "mx4":
        return n * k // 2 + n * k // 32
    bits, size = int(fmt[1]), int(fmt[3:])
    return n * k * bits // 8 + n * (k // size) * (4 if fmt[0] == "u" else 2 << bits)


def work(case):
    n, k, m = case["n"], case["k"], case["m"]
    if case["op"] == "quantize":
        return {"bytes": 4 * m * k, "flops": 4 * m * k}
    used = sum(c > 0 for c in _counts(case)) if case["experts"] else 1  # experts without rows are not read
    return {"bytes": used * _blob_bytes(n, k, case["weights"]) + 2 * m * k + 2 * m * n, "flops": 2 * m * n * k}


# ------------------------------------------------------------------ the same in 64 bits
def _nearest(x):
    """Every element of the 64-bit rows to the nearest of the 15 values times its block's scale: the
    largest power of two not above the block's largest, by 4."""
    b = x.view(x.shape[0], -1, 32)
    # (fp16 has no value so near below a power of two that the factor matters)
    top = b.abs().amax(-1, keepdim=True).clamp(min=2.0**-24)
    unit = torch.exp2(torch.floor(torch.log2(top * (1 + 1e-9))) - 2)
    a = (b.abs() / unit).clamp(max=6)
    # steps of 0.5 below 2, of 1 below 4, of 2 above; round() takes ties to the even multiple
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    return (torch.round(a / step) * step * unit * b.sign()).view(x.shape)


def _levels(case, seed, e):
    n, k, fmt = case["n"], case["k"], case["weights"]
    if fmt == "mx4":
        code, scale = _mx4(seed, e, n, k)
        mag = (code & 7).double()
        mag = torch.where(mag < 2, mag / 2, (1 + (mag % 2) / 2) * 2 ** (torch.floor(mag / 2) - 1))
        w = mag * (1 - 2 * (code >> 3).double()) * 2 ** (scale.double().unsqueeze(-1) - 127)
    else:
        code, table = _table(seed, e, n, k, fmt)
        table = table.double()
        w = (code.double() - table[..., 1:]) * table[..., :1] if fmt[0] == "u" else table.gather(-1, code.long())
    return w.view(n, k)


def exact(case, seed):
    x = _rows(case, seed).double()
    if case["op"] == "quantize" or case["op"].endswith("a4"):
        x = _nearest(x)
    if case["op"] == "quantize":
        return x
    if not case["experts"]:
        y = x @ _levels(case, seed, 0).t()
        return y[0] if case["op"] == "gemm" and case["m"] == 1 else y
    at = _offsets(case, seed)
    return torch.cat([x[at[e] : at[e + 1]] @ _levels(case, seed, e).t() for e in range(case["experts"]) if at[e] < at[e + 1]])
