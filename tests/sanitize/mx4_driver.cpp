// Drives the C entry points of the MX4 format and of products grouped by expert (qx_api_mx4.cpp) under the
// sanitizers: packs the cases of the command line (n k seed) into buffers of exactly their size, writes the
// blobs to <out_dir>/<index>.bin, and makes every refused call. Stand-ins for the launchers report QX_E_HIP,
// so that a call that passes its checks is told from one that does nothing.
#include <cstdio>
#include <cstdlib>
#include <string>
#include <vector>

#include "../../paper_2505_07531_amd/csrc/qx_internal.h"

namespace qx {
int launch_quantize_mx4(int, int, const uint16_t*, void*, hipStream_t) { return QX_E_HIP; }
int launch_gemm_a4(const qx_desc*, const void*, int, const void*, uint16_t*, hipStream_t) { return QX_E_HIP; }
int launch_gemm_mx4_grouped(const qx_desc*, const void*, const Experts&, int, const uint16_t*, uint16_t*, hipStream_t) {
  return QX_E_HIP;
}
int launch_gemm_a4_grouped(const qx_desc*, const void*, const Experts&, int, const void*, uint16_t*, hipStream_t) {
  return QX_E_HIP;
}
int launch_gemm_grouped(const qx_desc*, const void*, const Experts&, int, const uint16_t*, uint16_t*, hipStream_t) {
  return QX_E_HIP;
}
}  // namespace qx

static uint32_t lcg(uint64_t& s) {
  s = s * 6364136223846793005ull + 1442695040888963407ull;
  return (uint32_t)(s >> 33);
}

static int bad = 0;
static void expect(int got, int want, const char* what) {
  if (got != want) ++bad, fprintf(stderr, "%s: %d, expected %d\n", what, got, want);
}

int main(int argc, char** argv) {
  if (argc < 2) return 2;
  const std::string out = argv[1];
  for (int i = 2; i + 2 < argc; i += 3) {
    const int n = atoi(argv[i]), k = atoi(argv[i + 1]);
    uint64_t s = strtoull(argv[i + 2], nullptr, 10);
    const qx_desc d = {n, k, 4, 32, QX_MX4, 0};
    std::vector<uint8_t> codes((size_t)n * k), scales((size_t)n * k / 32);
    for (auto& c : codes) c = (uint8_t)(lcg(s) & 15);
    for (auto& c : scales) c = (uint8_t)lcg(s);
    size_t size = 0;
    expect(qx_pack_mx4(&d, nullptr, nullptr, nullptr, 0, &size), QX_OK, "size");
    std::vector<uint8_t> blob(size, 0xCD);
    expect(qx_pack_mx4(&d, codes.data(), scales.data(), blob.data(), blob.size(), &size), QX_OK, "pack");
    FILE* f = fopen((out + "/" + std::to_string(i / 3) + ".bin").c_str(), "wb");
    if (!f) return 3;
    if (!blob.empty()) fwrite(blob.data(), 1, blob.size(), f);
    fclose(f);
    if (n == 0) continue;
    std::vector<uint8_t> small(size - 1, 0xCD);
    expect(qx_pack_mx4(&d, codes.data(), scales.data(), small.data(), small.size(), &size), QX_E_SIZE, "a byte short");
    for (uint8_t c : small) expect(c, 0xCD, "written though short");
    codes.back() = 16;
    expect(qx_pack_mx4(&d, codes.data(), scales.data(), blob.data(), blob.size(), &size), QX_E_ARG, "code of 16");
    expect(qx_pack_mx4(&d, nullptr, scales.data(), blob.data(), blob.size(), &size), QX_E_ARG, "no codes");
    expect(qx_pack_mx4(&d, codes.data(), nullptr, blob.data(), blob.size(), &size), QX_E_ARG, "no scales");
  }
  size_t size;
  const qx_desc d = {4, 128, 4, 32, QX_MX4, 0}, u = {4, 128, 4, 32, QX_UNIFORM, 0}, none = {0, 128, 4, 32, QX_MX4, 0};
  expect(qx_pack_mx4(nullptr, nullptr, nullptr, nullptr, 0, &size), QX_E_ARG, "no descriptor");
  expect(qx_pack_mx4(&d, nullptr, nullptr, nullptr, 0, nullptr), QX_E_ARG, "no size");
  expect(qx_pack_mx4(&u, nullptr, nullptr, nullptr, 0, &size), QX_E_ARG, "another kind");
  for (qx_desc w : {qx_desc{-1, 128, 4, 32, QX_MX4, 0}, qx_desc{4, 100, 4, 32, QX_MX4, 0}, qx_desc{4, 0, 4, 32, QX_MX4, 0},
                    qx_desc{4, (1 << 20) + 128, 4, 32, QX_MX4, 0}, qx_desc{4, 128, 3, 32, QX_MX4, 0},
                    qx_desc{4, 128, 4, 64, QX_MX4, 0}, qx_desc{4, 128, 4, 32, 4, 0}, qx_desc{4, 128, 4, 32, QX_MX4, 1}})
    expect(qx_pack_mx4(&w, nullptr, nullptr, nullptr, 0, &size), QX_E_ARG, "a malformed descriptor");
  // the largest there is: sizes in 64 bits
  const qx_desc most = {2147483647, 1 << 20, 4, 32, QX_MX4, 0};
  expect(qx_pack_mx4(&most, nullptr, nullptr, nullptr, 0, &size), QX_OK, "the largest");
  if (size != (size_t)2147483647 * ((1 << 20) / 32 * 17)) ++bad;

  alignas(16) static uint16_t buf[64];
  alignas(16) static int32_t off[4];
  expect(qx_quantize_mx4(1, 128, buf, buf, nullptr), QX_E_HIP, "quantize");
  expect(qx_quantize_mx4(0, 128, nullptr, nullptr, nullptr), QX_OK, "no rows");
  expect(qx_quantize_mx4(1, 64, buf, buf, nullptr), QX_E_ARG, "k");
  expect(qx_quantize_mx4(1, 128, buf + 4, buf, nullptr), QX_E_ARG, "alignment");
  expect(qx_gemm_a4(&d, buf, 65536, buf, buf + 1, nullptr), QX_E_HIP, "a4");
  expect(qx_gemm_a4(&d, buf, 65537, buf, buf, nullptr), QX_E_ARG, "rows");
  expect(qx_gemm_a4(&u, buf, 1, buf, buf, nullptr), QX_E_UNSUPPORTED, "kind");
  expect(qx_gemm_a4(&none, nullptr, 1, nullptr, nullptr, nullptr), QX_OK, "no columns");
  expect(qx_gemm_grouped(&d, buf, 272, 1024, 65536, buf, off, buf, nullptr), QX_E_HIP, "grouped");
  expect(qx_gemm_grouped(&u, buf, 320, 3, 1, buf, off, buf, nullptr), QX_E_HIP, "grouped uniform");
  expect(qx_gemm_grouped(&d, buf, 256, 2, 1, buf, off, buf, nullptr), QX_E_ARG, "stride");
  expect(qx_gemm_grouped(&d, buf, 280, 2, 1, buf, off, buf, nullptr), QX_E_ARG, "stride's alignment");
  expect(qx_gemm_grouped(&d, buf, 272, 1025, 1, buf, off, buf, nullptr), QX_E_ARG, "experts");
  expect(qx_gemm_grouped(&d, buf, 272, -1, 1, buf, off, buf, nullptr), QX_E_ARG, "experts below none");
  expect(qx_gemm_grouped(&d, buf, 272, 2, 65537, buf, off, buf, nullptr), QX_E_ARG, "rows");
  expect(qx_gemm_grouped(&d, buf, 272, 2, 1, buf, nullptr, buf, nullptr), QX_E_ARG, "no offsets");
  expect(qx_gemm_grouped(&d, nullptr, 272, 0, 1, nullptr, nullptr, nullptr, nullptr), QX_OK, "no experts");
  expect(qx_gemm_a4_grouped(&d, buf, 272, 2, 1, buf, off, buf, nullptr), QX_E_HIP, "a4 grouped");
  expect(qx_gemm_a4_grouped(&u, buf, 320, 2, 1, buf, off, buf, nullptr), QX_E_UNSUPPORTED, "a4 grouped, kind");
  printf("sanitized MX4 front end: %d unexpected statuses\n", bad);
  return bad ? 4 : 0;
}
