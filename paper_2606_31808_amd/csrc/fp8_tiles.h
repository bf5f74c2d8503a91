// The block-scaled FP8 product's kernels and the rule that picks one; plain
// C++, so that the host can check which call takes which.
#pragma once
#include <algorithm>
#include <cstdint>

namespace lmop {

// A tile of 16*mt*wm tokens x 16*nt*wn columns by wm x wn waves, occ
// workgroups a CU; us per group of 128 features with one workgroup on a CU and
// with occ of them (same card, weights from memory), on the 8-bit instruction and
// with whole products (0: not offered).  few: 16*mt tokens x 16 columns by 8 waves
// that share K.
struct Fp8Tile {
  int mt, nt, wm, wn, occ;
  float one[2], all[2];
  constexpr int bm() const { return 16 * mt * wm; }
  constexpr int bn() const { return 16 * nt * wn; }
};
constexpr Fp8Tile kFp8Tiles[] = {
    {8, 4, 2, 4, 1, {1.75f, 0.f}, {1.85f, 0.f}},  // 256 x 256
    {4, 4, 2, 4, 1, {1.08f, 1.78f}, {1.10f, 1.78f}},  // 128 x 256
    {2, 4, 2, 2, 2, {0.55f, 0.77f}, {0.80f, 1.20f}},  // 64 x 128
    {2, 2, 2, 2, 2, {0.38f, 0.49f}, {0.65f, 0.78f}},  // 64 x 64
    {2, 1, 1, 4, 2, {0.29f, 0.45f}, {0.45f, 0.64f}},  // 32 x 64
};
constexpr int kNumFp8Tiles = sizeof(kFp8Tiles) / sizeof(kFp8Tiles[0]);
// the picks after the tiles: up to 16 tokens, parts of 32 tokens
constexpr int kFp8Few16 = kNumFp8Tiles, kFp8Few32 = kNumFp8Tiles + 1;
constexpr int kNumFp8Kernels = kNumFp8Tiles + 2;

// tokens, columns and threads of a kernel's workgroup
struct Fp8Group {
  int bm, bn, threads;
};
constexpr Fp8Group fp8_group(int kernel) {
  if (kernel >= kNumFp8Tiles) return {kernel == kFp8Few32 ? 32 : 16, 16, 512};
  const Fp8Tile& t = kFp8Tiles[kernel];
  return {t.bm(), t.bn(), 64 * t.wm * t.wn};
}

// The most tokens of one launch, whole tiles of them: HIP launches fewer than
// 2^32 threads at a time.  Zero where one row of tiles is too many: the kernel
// is then not picked (one of 128 columns and 256 threads serves 2^30 columns).
inline int fp8_rows(int kernel, int m, int n) {
  const Fp8Group g = fp8_group(kernel);
  const int64_t most = ((int64_t(1) << 32) - 1) / g.threads, across = (n + g.bn - 1) / g.bn;
  return (int)std::min<int64_t>(m, most / across * g.bm);
}

// Estimated us.  Tiles: rounds over the 256 CUs, at least the time in which
// the weight comes from memory (4.4 TB/s), and 3 us around them.  Few tokens:
// 4 us and a time per group, a fixed one or one per tile that grows with the
// tokens (their codes are read again for every 16 columns).  Measured, us, few
// against the best tile (whole products in brackets):
//   1 token:   n 6144 k 4096 8.5 / 12.4, n 4096 k 14336 12.9 / 33, n 28672 k 4096 22.7 / 26.8
//   16 tokens: 11.7 / 11.8, 18.6 / 32.3, 35.6 / 26.6
//   24 tokens: 14.6 / 12.1, 23.8 / 32.6, 44.2 / 27.9; n 2048 k 2048 5.1 / 7.1
//   48 tokens: n 4096 k 4096 14.3 / 11.6 (14.6 / 16.8), n 1536 k 14336 23.3 / 32.2
//   64 tokens: n 6144 k 4096 22.3 / 12.3, n 4096 k 14336 46.6 / 32.8, n 768 k 6272 11.8 / 15.2
//              (12.3 / 22.9), n 2048 k 4096 8.4 / 10.9 (8.8 / 16.2)
//   128:       n 768 k 4096 8.3 / 10.9 (8.7 / 16.2), n 2048 k 2048 8.3 / 7.0
// and of the tiles:
//   256 x 4096, k 4096: 32 x 64 17.1 (24.0), 64 x 64 14.5 (18.4), 64 x 128 19.2 (26.6)
//   512 x 4096, k 4096: 32 x 64 31.7 (43.9), 64 x 64 20.8 (27.3), 64 x 128 19.6 (27.4),
//     128 x 256 35.4 (54.2), 256 x 256 60.0
//   2047 x 4096, k 4096: 64 x 64 71.9 (95.8), 64 x 128 57.0 (81.0), 128 x 256 40.8 (62.5),
//     256 x 256 62.3
//   16384 x 4096, k 14336: 64 x 128 1266 (1926), 128 x 256 902 (1526), 256 x 256 772
//   16384 x 28672, k 4096: 128 x 256 1868, 256 x 256 1645
inline float fp8_cost(int kernel, bool whole, int m, int n, int k) {
  const float groups = (k + 127) / 128;
  if (n >= 1 << 26 && fp8_rows(kernel, m, n) == 0) return 1e30f;
  if (kernel >= kNumFp8Tiles) {
    const bool wide = kernel == kFp8Few32;
    if (!wide && m > 16) return 1e30f;
    const int parts = wide ? (m + 31) / 32 : 1, tokens = (m + parts - 1) / parts;
    const float per = wide ? 0.62e-3f + 0.014e-3f * std::max(tokens - 16, 0)
                           : 0.32e-3f + 0.02e-3f * (tokens - 1);
    const float tiles = (float)parts * (float)((n + 15) / 16);
    return 4.f + groups * std::max(wide ? 0.17f : 0.08f, per * tiles);
  }
  const Fp8Tile& t = kFp8Tiles[kernel];
  if (t.all[whole] == 0.f) return 1e30f;
  const long tiles = (long)((m + t.bm() - 1) / t.bm()) * ((n + t.bn() - 1) / t.bn());
  const long round = 256L * t.occ, full = tiles / round, rem = tiles % round;
  const float rounds =
      full * t.all[whole] + (rem == 0 ? 0.f : rem <= 256 ? t.one[whole] : t.all[whole]);
  return 3.f + std::max(groups * rounds, (float)n * (float)k / 4.4e6f);
}

// The kernel with the least estimated time, the smaller tile of two that wait
// for the same memory.  Every kernel gives the same bits.
inline int pick_fp8_kernel(bool whole, int m, int n, int k) {
  int best = kNumFp8Kernels - 1;
  for (int i = best - 1; i >= 0; --i)
    if (fp8_cost(i, whole, m, n, k) < fp8_cost(best, whole, m, n, k)) best = i;
  return best;
}

}  // namespace lmop
