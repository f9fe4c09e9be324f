"""Loads from memory straight into LDS in the built library: on every path of every kernel each of them is
waited for before the next barrier, since the block's other waves read what it brings behind that barrier.
Reads the disassembly of libqx.so's own kernels. CPU only."""
import glob
import os
import re
import shutil
import subprocess

import pytest

import paper_2505_07531_amd as qx

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
LINE = re.compile(r"\t(\w+)(.*?)\s*// ([0-9A-F]+):")
MEMORY = re.compile(r"(global|buffer|flat|scratch)_(load|store|atomic)")


def kernels(text):
    """(name, [(address, instruction, operands)])"""
    name, body = None, []
    for line in text.splitlines():
        head = re.match(r"<(\w+)>:", line)
        m = LINE.match(line)
        if head:
            if body:
                yield name, body
            name, body = head.group(1), []
        elif m and name:
            where = re.search(r"\+0x([0-9a-f]+)>$", line)  # of a branch: its target, from the kernel's start
            body.append((int(m.group(3), 16), m.group(1), m.group(2).strip(), int(where.group(1), 16) if where else 0))
    if body:
        yield name, body


def early_barriers(body):
    """Places of barriers that a wave can reach with a load to LDS still under way. Followed is how many
    accesses to memory there are since the newest such load, at least, on any path: s_waitcnt vmcnt(N)
    waits for all but the last N of them."""
    done = 1 << 30  # no load to LDS under way
    at = {a: i for i, (a, *_) in enumerate(body)}
    start, seen, early, todo = body[0][0], {}, set(), [(0, done)]
    while todo:
        i, since = todo.pop()
        while seen.get(i, done + 1) > since:
            seen[i] = since
            _, op, args, target = body[i]
            if op.startswith("global_load_lds"):
                since = 0
            elif MEMORY.match(op):
                since = min(since + 1, done)
            elif op == "s_waitcnt":
                m = re.search(r"vmcnt\((\d+)\)", args)
                if m and int(m.group(1)) <= since:
                    since = done
            elif op == "s_barrier" and since != done:
                early.add(i)
            if op.startswith(("s_cbranch", "s_branch")):
                todo.append((at[start + target], since))
            if op in ("s_branch", "s_endpgm"):
                break
            i += 1
    return sorted(early)


def body_of(*ops):
    """Instructions of 4 bytes each, from address 0; (op, args, target) or op."""
    ops = [o if isinstance(o, tuple) else (o, "", 0) for o in ops]
    return [(4 * i, *o) for i, o in enumerate(ops)]


def test_the_check_itself():
    load, bar, end = "global_load_lds_dwordx4", "s_barrier", "s_endpgm"
    wait = lambda n: ("s_waitcnt", f"vmcnt({n})", 0)  # noqa: E731
    assert early_barriers(body_of(load, wait(0), bar, end)) == []
    assert early_barriers(body_of(load, bar, end)) == [1]
    assert early_barriers(body_of(load, ("s_waitcnt", "lgkmcnt(0)", 0), bar, end)) == [2]
    assert early_barriers(body_of(load, "global_load_dword", wait(1), bar, end)) == []
    assert early_barriers(body_of(load, "global_load_dword", wait(2), bar, end)) == [3]
    # a branch past the wait, and a loop whose load is not waited for on the way back
    assert early_barriers(body_of(load, ("s_cbranch_scc0", "", 12), wait(0), bar, end)) == [3]
    assert early_barriers(body_of(bar, load, ("s_cbranch_scc0", "", 0), end)) == [0]
    assert early_barriers(body_of(bar, load, wait(0), ("s_cbranch_scc0", "", 0), end)) == []


def test_loads_to_lds_are_waited_for_before_barriers(tmp_path):
    if shutil.which(OBJDUMP) is None:
        pytest.skip("llvm-objdump not available")
    qx.load()
    lib = shutil.copy(qx.LIB_PATH, tmp_path)  # the code objects are written beside it
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, timeout=120)
    found = 0
    for obj in glob.glob(os.path.join(str(tmp_path), "*gfx950")):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", obj], check=True,
                              capture_output=True, text=True, timeout=120).stdout
        if "global_load_lds" not in text:
            continue
        for name, body in kernels(text):
            if any(op.startswith("global_load_lds") for _, op, _, _ in body):
                found += 1
                assert early_barriers(body) == [], name
    assert found >= 100  # 65 of grouped.hip, 39 of mx4_tile.h
