// C = A B^T (+ add) of E4M3 codes: one fp32 scale per row and 128 features of
// A (tokens), one per 128 x 128 block of B (a weight).
//
// The weight's rows are the MFMA's A operand and the tokens its B operand, so
// a lane of the result holds 4 columns of one token and one scale,
// a_scale[token][group] * b_scale[block][group], serves all of them.  The sum
// over a group of 128 features starts from zero and is added to the running
// sum with one fma per value, groups in order.  Every kernel here does the
// same steps on the same lanes, so which one computes a value never changes
// its bits.
//
// The sum over a group (`dot`), by the result:
//   fp16, bf16, `fast` fp32: one MFMA 16x16x128 on the codes, at twice the fp16 rate.  It
//     cuts products at 2^-13 of the leading bit of the largest of eight neighbours (see
//     mfma16x16x128_e4m3): a sum of eight is off by less than 7 * 2^-13 of its largest
//     product.  On unit-normal tokens and weights that is 1.5e-5 of the result's norm (2.0e-5
//     to 2.5e-5 with a feature in a hundred ten times as large), against 2.1e-4 (fp16) and
//     1.7e-3 (bf16) of the rounding to the type; fp16 results are off by 2.09e-4 then,
//     by 2.07e-4 with whole products, whose groups take a tile 1.3 to 1.7 times as long.
//   fp32 otherwise: the codes converted to fp16, exactly, and four MFMAs 16x16x32,
//     which keep every product whole and add in fp32.
#include "common.h"
#include "fp8_tiles.h"
#include "kernels.h"
#include "lds_dma.h"
#include "lds_dma4.h"

#include <atomic>
#include <type_traits>

namespace lmop {

namespace {

constexpr int GROUP = LMOP_FP8_GROUP;

// The type of C, and whether the inner sums keep their products whole.
template <typename T, bool W>
struct Result {
  using Type = T;
  static constexpr bool WHOLE = W;
};

// The 4 codes of a word (byte 0 first) as fp16, exactly: every E4M3 value is an
// fp16 value, so a unit scale changes nothing.
LMOP_DEVICE f16x4 halves_of(uint32_t d) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(d, 1.0f, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(d, 1.0f, true);
  return f16x4{a.x, a.y, b.x, b.y};
}

// A lane's 32 codes of one row and group: lane 16g + c holds features
// 16g .. 16g+15 and 64+16g .. 64+16g+15 of row c.
struct Codes {
  uint4 w[2];
};
struct Halves {
  f16x8 h[4];
};

// What is left of a lane's codes where `valid` features are left from its first
// one on: the bytes from there on become zero (+0.0).
struct Left {
  uint4 w[2];
};
LMOP_DEVICE Left left_of(int valid) {
  Left l;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = valid - 64 * h - 4 * i;
      w[i] = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
    }
    l.w[h] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return l;
}
LMOP_DEVICE void keep(Codes& c, const Left& l) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    c.w[h] = make_uint4(c.w[h].x & l.w[h].x, c.w[h].y & l.w[h].y, c.w[h].z & l.w[h].z,
                        c.w[h].w & l.w[h].w);
}

// 8 of a lane's 32 codes as fp16
LMOP_DEVICE f16x8 quarter(const Codes& c, int i) {
  const uint4 w = c.w[i >> 1];
  const f16x4 lo = halves_of(i & 1 ? w.z : w.x), hi = halves_of(i & 1 ? w.w : w.y);
  return f16x8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
}

// the operand of `dot`: the codes themselves, or their fp16 values
template <bool WHOLE>
using Operand = std::conditional_t<WHOLE, Halves, Codes>;
template <bool WHOLE>
LMOP_DEVICE Operand<WHOLE> operand(const Codes& c) {
  if constexpr (WHOLE) {
    Halves r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.h[i] = quarter(c, i);
    return r;
  } else {
    return c;
  }
}

LMOP_DEVICE i32x8 words(const Codes& c) {
  return i32x8{(int)c.w[0].x, (int)c.w[0].y, (int)c.w[0].z, (int)c.w[0].w,
               (int)c.w[1].x, (int)c.w[1].y, (int)c.w[1].z, (int)c.w[1].w};
}
// 16 columns x 16 tokens over one group
LMOP_DEVICE f32x4 dot(const Codes& b, const Codes& a) {
  return mfma16x16x128_e4m3(words(b), words(a));
}
LMOP_DEVICE f32x4 dot(const Halves& b, const Halves& a) {
  f32x4 d = mfma16x16x32(b.h[0], a.h[0], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
  for (int i = 1; i < 4; ++i) d = mfma16x16x32(b.h[i], a.h[i], d);
  return d;
}

LMOP_DEVICE void add_scaled(f32x4& acc, f32x4 d, float s) {
#pragma unroll
  for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(d[r], s, acc[r]);
}

// ---------------------------------------------------------------- results to memory
// 16 tokens x NT * 16 columns of a wave from token m, column n on go through
// its LDS at `mine`, so that the lanes of a store hold whole rows; a lane's
// accesses to memory need the alignment of one value only.  With one workgroup
// on a CU nothing hides the stores.  16384 x 28672 of fp16, k 4096: 1824 us with the
// 4 columns that a lane has (32 bytes a row), 1720 with rows of 128 bytes, 1645 streamed
// (STREAM: past the caches), 1535 without any stores; fp32, 16384 x 4096, k 4096:
// 468 (64 bytes a row), 467 (256), 457, 427.
template <int NT>
struct Rows {
  static constexpr int COLS = 16 * NT;
  static constexpr int PITCH = 4 * COLS + 16;  // bytes of a row of fp32; 16 apart in the banks
  static constexpr int LDS = 16 * PITCH;       // of a wave
};

// What a lane stores of 16 rows where every column is in the matrix: Q chunks of
// 16 bytes, chunk q of row at(q) / CHUNKS.
template <typename T, int NT>
struct Chunks {
  static constexpr int W = 16 / sizeof(T), CHUNKS = Rows<NT>::COLS / W, Q = (16 * CHUNKS + 63) / 64;
  typedef T Chunk __attribute__((ext_vector_type(W)));
  typedef Chunk Any __attribute__((aligned(sizeof(T))));
  static LMOP_DEVICE int at(int q) { return q * 64 + (threadIdx.x & 63); }
};

// the chunks of `add` (fp32); rows past the matrix repeat its last one, so that
// the loads of 16 rows are in flight together
template <int NT>
LMOP_DEVICE void load_add(const lmop_matmul_args& p, int m, int n,
                          typename Chunks<float, NT>::Chunk (&v)[Chunks<float, NT>::Q]) {
  using R = Chunks<float, NT>;
#pragma unroll
  for (int q = 0; q < R::Q; ++q) {
    const int r = m + R::at(q) / R::CHUNKS, x = R::at(q) % R::CHUNKS;
    v[q] = *(const typename R::Any*)(p.add + (size_t)(r < p.m ? r : p.m - 1) * p.ldadd + n +
                                     R::W * x);
  }
}

// every column is in the matrix, and 16-bit results have no `add`
template <typename T, int NT, bool STREAM>
LMOP_DEVICE void store_rows(const lmop_matmul_args& p, char* mine, int m, int n,
                            const f32x4 (&v)[NT],
                            const typename Chunks<T, NT>::Chunk (&add)[Chunks<T, NT>::Q]) {
  using R = Chunks<T, NT>;
  constexpr int PITCH = Rows<NT>::COLS * (int)sizeof(T) + 16;
  typedef T T4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  // the wave's earlier reads of these bytes are done
  wait_vmcnt_lgkm0<63>();
#pragma unroll
  for (int j = 0; j < NT; ++j)
    *(T4*)(mine + c * PITCH + (16 * j + 4 * g) * (int)sizeof(T)) =
        T4{(T)v[j][0], (T)v[j][1], (T)v[j][2], (T)v[j][3]};
  wait_vmcnt_lgkm0<63>();
#pragma unroll
  for (int q = 0; q < R::Q; ++q) {
    const int r = R::at(q) / R::CHUNKS, x = R::at(q) % R::CHUNKS;
    if (r < 16 && m + r < p.m) {
      typename R::Chunk w = *(const typename R::Chunk*)(mine + r * PITCH + 16 * x);
      if constexpr (std::is_same_v<T, float>)
        if (p.add) w = add[q] + w;
      T* to = (T*)p.c + (size_t)(m + r) * p.ldc + n + R::W * x;
      if constexpr (STREAM)
        __builtin_nontemporal_store(w, (typename R::Any*)to);
      else
        *(typename R::Any*)to = w;
    }
  }
}

// any columns: a value a lane, the loads of 8 rounds in flight together
template <typename T, int NT>
LMOP_DEVICE void store_values(const lmop_matmul_args& p, char* mine, int m, int n,
                              const f32x4 (&v)[NT]) {
  using R = Rows<NT>;
  constexpr int ROUNDS = 16 * R::COLS / 64, U = ROUNDS < 8 ? ROUNDS : 8;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  wait_vmcnt_lgkm0<63>();
#pragma unroll
  for (int j = 0; j < NT; ++j) *(f32x4*)(mine + c * R::PITCH + (16 * j + 4 * g) * 4) = v[j];
  wait_vmcnt_lgkm0<63>();
#pragma unroll
  for (int q0 = 0; q0 < ROUNDS; q0 += U) {
    float add[U];
    if (p.add)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = (q0 + u) * 64 + lane, r = m + at / R::COLS, x = n + at % R::COLS;
        add[u] = p.add[(size_t)(r < p.m ? r : p.m - 1) * p.ldadd + (x < p.n ? x : p.n - 1)];
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = (q0 + u) * 64 + lane, r = at / R::COLS, x = at % R::COLS;
      float w = *(const float*)(mine + r * R::PITCH + 4 * x);
      if (p.add) w = add[u] + w;
      if (m + r < p.m && n + x < p.n) ((T*)p.c)[(size_t)(m + r) * p.ldc + n + x] = (T)w;
    }
  }
}

// ---------------------------------------------------------------- tiles through LDS
// Bound by the matrix cores, LDS and the vector units together: a group of 256 x 256
// takes the matrix cores 2048 cycles, LDS 2048 (192 KB read, 64 KB filled, 128 B a cycle) and
// each SIMD some 1800 cycles of issue, and they overlap in part: 16384 x 28672, k 4096
// runs at 2340 TFLOP/s (fp16 results; the matrix cores busy 57% of the cycles, 2508 without
// its stores), 16384 x 4096, k 14336 at 2490; with whole products, whose codes become
// fp16, at 1260.
// A workgroup of WM x WN waves computes 16*MT*WM tokens x 16*NT*WN columns; a
// wave MT x NT tiles of 16 x 16.  One ring stage is one group of the tile's
// rows: 128 bytes a row, 16-byte chunks XOR-swizzled by row, and the tokens'
// scales, filled by direct global->LDS loads.
template <int MT, int NT, int WM, int WN, int OCC>
struct Tile {
  static constexpr int BM = 16 * MT * WM, BN = 16 * NT * WN, NW = WM * WN;
  static constexpr int STAGE = (BM + BN) * 128;
  // the tokens' scales of the groups 4q .. 4q+3, for SBUF q in turn
  static constexpr int SCALES = BM * 16;
  static constexpr int NS_FIT = (160 * 1024 / OCC - 3 * SCALES) / STAGE;
  static constexpr int NS = NS_FIT < 8 ? NS_FIT : 8;
  static constexpr int SBUF = (NS + 2) / 4 + 1;  // from the stage in use to the last in flight
  static_assert(NS >= 2, "a stage in use and one in flight");
  static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole loads");
  static_assert(GROUP % (16 * NT) == 0, "a wave's columns lie in one block of B");
  // a wave's loads per stage, 8 rows each
  static constexpr int A_LOADS = BM / 8 / NW, B_LOADS = BN / 8 / NW;
  static constexpr int LOADS = A_LOADS + B_LOADS;
  static constexpr int LDS = NS * STAGE + SBUF * SCALES;
  static_assert((NS - 2) * LOADS < 63, "the loads waited for fit the counter");
};

constexpr int GM = 4;  // token tiles per L2 group

template <typename R, int MT, int NT, int WM, int WN, int OCC, bool STREAM>
__global__ __launch_bounds__((64 * WM * WN), ((OCC * WM * WN + 3) / 4)) void matmul_tile_kernel(
    const lmop_matmul_args p) {
  using C = Tile<MT, NT, WM, WN, OCC>;
  using T = typename R::Type;
  constexpr bool WHOLE = R::WHOLE;
  constexpr int BM = C::BM, BN = C::BN, NW = C::NW, NS = C::NS;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // the XCDs take one contiguous range of tiles each, ordered in groups of GM
  // token tiles that share their L2's weight rows
  const int ntm = (p.m + BM - 1) / BM, ntn = (p.n + BN - 1) / BN;
  const int total = ntm * ntn, xcd = blockIdx.x & 7, per = total >> 3, rem = total & 7;
  const int logical = xcd * per + (xcd < rem ? xcd : rem) + (blockIdx.x >> 3);
  const int grp = logical / (GM * ntn), within = logical - grp * GM * ntn;
  const int gsz = ntm - grp * GM < GM ? ntm - grp * GM : GM;
  const int m0 = (grp * GM + within % gsz) * BM, n0 = within / gsz * BN;

  const int kr = (p.k + 15) / 16 * 16, kb_n = (p.k + GROUP - 1) / GROUP;

  // A wave's loads take rows 8 * (wave + NW * n) .. +7 of the tile's tokens,
  // then of its columns.  Rows past the matrix repeat its last one; chunks past
  // a row's end repeat its last one and are cleared after they are read.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  const uint8_t* abase = p.a + (size_t)m0 * p.lda;
  const uint8_t* bbase = p.b + (size_t)n0 * p.ldb;
  const uint32_t lda = (uint32_t)p.lda, ldb = (uint32_t)p.ldb;
  const uint32_t row0 = (uint32_t)(wave * 8 + (lane >> 3));
  const uint32_t a_first = row0 * lda, b_first = row0 * ldb;
  const uint32_t a_last = (uint32_t)(p.m - 1 - m0 < BM ? p.m - 1 - m0 : BM) * lda;
  const uint32_t b_last = (uint32_t)(p.n - 1 - n0 < BN ? p.n - 1 - n0 : BN) * ldb;
  const uint32_t chunk = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u;
  // A wave loads the scales of SROWS tokens, 16 at a time: lane 4r + q the
  // scale of token r and group 4 * (kb / 4) + q ([token][4] in LDS).
  constexpr int SROWS = BM / NW, SLOADS = (SROWS + 15) / 16;
  const uint32_t scl0 = lds0 + NS * C::STAGE + (uint32_t)(wave * SROWS) * 16u;
  const float* sbase = p.a_scale + (size_t)m0 * p.ldas;
  uint32_t srow[SLOADS];
#pragma unroll
  for (int i = 0; i < SLOADS; ++i) {
    const int r = wave * SROWS + 16 * i + (lane >> 2);
    srow[i] = (uint32_t)(r < p.m - 1 - m0 ? r : p.m - 1 - m0) * (uint32_t)p.ldas;
  }
  auto issue_scales = [&](int kb) {
    const int q = kb + (lane & 3) < kb_n ? kb + (lane & 3) : kb_n - 1;
    const uint32_t to = scl0 + (uint32_t)((kb >> 2) % C::SBUF * C::SCALES);
    const uint64_t on = SROWS >= 16 ? ~0ull : (1ull << (4 * (SROWS % 16))) - 1;
#pragma unroll
    for (int i = 0; i < SLOADS; ++i)
      g2l4_m0_mask(sbase, (srow[i] + (uint32_t)q) * 4u, to + 256u * i, kb % 4 == 0 ? on : 0ull);
  };
  // Instruction n of the loads of stage kb, into its slot; past the last stage
  // the loads repeat that one, so that every stage is as many loads.
  auto issue_one = [&](int n, int kb) {
    const uint32_t st = lds0 + (uint32_t)(kb % NS * C::STAGE);
    kb = kb < kb_n ? kb : kb_n - 1;
    const uint32_t end = (uint32_t)(kr - 16 - kb * GROUP), at = chunk < end ? chunk : end;
    if (n < C::A_LOADS) {
      const uint32_t r = a_first + (uint32_t)(NW * 8 * n) * lda;
      g2l16_m0(abase + (size_t)kb * GROUP, (r < a_last ? r : a_last) + at,
               st + (uint32_t)(wave + NW * n) * 1024u);
    } else {
      const int i = n - C::A_LOADS;
      const uint32_t r = b_first + (uint32_t)(NW * 8 * i) * ldb;
      g2l16_m0(bbase + (size_t)kb * GROUP, (r < b_last ? r : b_last) + at,
               st + (uint32_t)(BM * 128 + (wave + NW * i) * 1024));
    }
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int nblk = n0 + wn * NT * 16 < p.n ? (n0 + wn * NT * 16) / GROUP : (p.n - 1) / GROUP;
  const float* sb = p.b_scale + (size_t)nblk * p.ldbs;

  // this lane's chunks of its rows within a stage: 16 bytes at g and g + 4, so
  // that no two of the 16 lanes that LDS serves at once share a bank (chunks 2g
  // and 2g + 1 conflict in pairs)
  const int off0 = (g ^ (c & 7)) * 16, off1 = ((g + 4) ^ (c & 7)) * 16;
  const int arow = (wm * MT * 16 + c) * 128, brow = (BM + wn * NT * 16 + c) * 128;
  auto codes = [&](int kb, int row, int i) {
    const char* st = smem + kb % NS * C::STAGE + row;
    Codes x;
    x.w[0] = *(const uint4*)(st + off0 + i * 2048);
    x.w[1] = *(const uint4*)(st + off1 + i * 2048);
    return x;
  };
  auto frag = [&](int kb, int row, int i) { return operand<WHOLE>(codes(kb, row, i)); };
  auto scale = [&](int kb, int i) {
    return *(const float*)(smem + NS * C::STAGE + (kb >> 2) % C::SBUF * C::SCALES + kb % 4 * 4 +
                           (wm * MT * 16 + c) * 16 + i * 256);
  };

  // 64 groups at a time: their scales of the wave's columns, one a lane
  const int full = p.k / GROUP;
  auto groups = [&](auto& stage) {
    for (int k0 = 0; k0 < full; k0 += 64) {
      float sb_64 = sb[k0 + lane < kb_n ? k0 + lane : kb_n - 1];
      // waited for here: in the loop the wait would be for the stages in flight too
      asm volatile("" : "+v"(sb_64));
      const int end = full < k0 + 64 ? full : k0 + 64;
      for (int kb = k0; kb < end; ++kb)
        stage(kb, __uint_as_float(
                      __builtin_amdgcn_readlane(__float_as_uint(sb_64), kb - k0)));
    }
  };
  if constexpr (WHOLE) {
    // Whole products: the codes' conversions take the vector units as long as the products
    // take the matrix cores, so each has to run beside the other.  In phase i the
    // tile row i is multiplied, a quarter of the group at a time, while row i - 1
    // is added to the sums and row i + 1 is read and converted; the last phase
    // begins with the barrier, reads the next group's first row and columns, and
    // puts a converted quarter of the columns in the place of the one just used
    // up.  16384 x 4096, k 14336: 1592 us, 1642 with the columns converted at a
    // group's start; 512 x 4096, k 4096 on a workgroup a CU: 54.4, 60.9.
    static_assert(MT % 2 == 0, "rows alternate between two buffers across groups");
    constexpr int PER = (C::LOADS + MT - 1) / MT;
    Halves b[NT], a[2];
    f32x4 d[2][NT];
    float s[2], sc = 0.f;
#pragma unroll
    for (int j = 0; j < NT; ++j) d[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto stage = [&](int kb, float sbk) {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const bool last = i == MT - 1;
        __builtin_amdgcn_sched_barrier(0);
        if (last) {
          // the next stage has landed for every wave, and every wave has read
          // this one, whose slot the loads below refill (the later stages'
          // scales are not counted: a smaller count waits for more)
          wait_vmcnt_lgkm0<(NS - 2) * C::LOADS>();
          barrier();
          issue_scales(kb + NS);
        }
        const int share = (i + 1) % MT;
#pragma unroll
        for (int n = share * PER; n < (share + 1) * PER && n < C::LOADS; ++n)
          issue_one(n, last ? kb + NS : kb + NS - 1);
        __builtin_amdgcn_sched_barrier(0);
        const float sc_before = sc;
        sc = s[i & 1] * sbk;
        const int next = last ? kb + 1 : kb, row = last ? 0 : i + 1;
        const Codes ac = codes(next, arow, row);
        s[(i + 1) & 1] = scale(next, row);
        Codes bc[NT];
        if (last)
#pragma unroll
          for (int j = 0; j < NT; ++j) bc[j] = codes(next, brow, j);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
#pragma unroll
          for (int j = 0; j < NT; ++j)
            d[i & 1][j] = mfma16x16x32(b[j].h[h], a[i & 1].h[h],
                                       h ? d[i & 1][j] : f32x4{0.f, 0.f, 0.f, 0.f});
          a[(i + 1) & 1].h[h] = quarter(ac, h);
#pragma unroll
          for (int j = 0; j < NT; ++j)
            if (j % 4 == h) add_scaled(acc[(i + MT - 1) % MT][j], d[(i + 1) & 1][j], sc_before);
          if (last)
#pragma unroll
            for (int j = 0; j < NT; ++j) b[j].h[h] = quarter(bc[j], h);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int kb = 0; kb < NS; ++kb) {
      issue_scales(kb);
#pragma unroll
      for (int n = 0; n < (kb < NS - 1 ? C::LOADS : PER); ++n) issue_one(n, kb);
    }
    wait_vmcnt_lgkm0<(NS - 2) * C::LOADS>();
    barrier();
#pragma unroll
    for (int j = 0; j < NT; ++j) b[j] = frag(0, brow, j);
    a[0] = frag(0, arow, 0);
    s[0] = scale(0, 0);
    groups(stage);
    if (full > 0)
#pragma unroll
      for (int j = 0; j < NT; ++j) add_scaled(acc[MT - 1][j], d[(MT - 1) & 1][j], sc);
  } else {
    // The 8-bit instruction, one whole group.  In phase i the tile row i is multiplied while row i - 1
    // is added to the sums, row i + 1 is read, and a share of a later stage's
    // loads is issued (waves that issue all of theirs at once hold each other up
    // while the matrix cores run dry).  No branch: one would let the compiler
    // move the additions behind it.
    constexpr int PER = (C::LOADS + MT - 1) / MT < 2 ? 2 : (C::LOADS + MT - 1) / MT;
    auto stage = [&](int kb, float sbk) {
      // the stage has landed for every wave, and every wave is done with the one
      // before it, which the loads below refill (the later stages' scales are not
      // counted: a smaller count waits for more)
      wait_vmcnt_lgkm0<(NS - 2) * C::LOADS>();
      barrier();
      Codes b[NT], a[2];
      f32x4 d[2][NT];
      float s[2], sc = 0.f;
#pragma unroll
      for (int j = 0; j < NT; ++j) b[j] = codes(kb, brow, j);
      a[0] = codes(kb, arow, 0);
      s[0] = scale(kb, 0);
#pragma unroll
      for (int i = 0; i <= MT; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        if (i == 0) issue_scales(kb + NS - 1);
#pragma unroll
        for (int n = i * PER; n < (i + 1) * PER && n < C::LOADS; ++n) issue_one(n, kb + NS - 1);
        __builtin_amdgcn_sched_barrier(0);
        const float sc_before = sc;
        if (i < MT) sc = s[i & 1] * sbk;
        if (i + 1 < MT) {
          a[(i + 1) & 1] = codes(kb, arow, i + 1);
          s[(i + 1) & 1] = scale(kb, i + 1);
        }
        if (i < MT)
#pragma unroll
          for (int j = 0; j < NT; ++j) d[i & 1][j] = dot(b[j], a[i & 1]);
        if (i > 0)
#pragma unroll
          for (int j = 0; j < NT; ++j) add_scaled(acc[i - 1][j], d[(i - 1) & 1][j], sc_before);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
          __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);  // VALU
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };


#pragma unroll
    for (int kb = 0; kb < NS - 1; ++kb) {
      issue_scales(kb);
#pragma unroll
      for (int n = 0; n < C::LOADS; ++n) issue_one(n, kb);
    }
    groups(stage);
  }
  // the loads end before the workgroup does
  wait_vmcnt_lgkm0<0>();
  if (full < kb_n) {
    // the last features, less than a group: their stage is the last one loaded
    barrier();
    const Left left = left_of(p.k - full * GROUP - 16 * g);
    const float sb_last = sb[full];
    auto masked = [&](int row, int i) {
      Codes x = codes(full, row, i);
      keep(x, left);
      return operand<WHOLE>(x);
    };
    Operand<WHOLE> b[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) b[j] = masked(brow, j);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const Operand<WHOLE> a = masked(arow, i);
      const float sc = scale(full, i) * sb_last;
#pragma unroll
      for (int j = 0; j < NT; ++j) add_scaled(acc[i][j], dot(b[j], a), sc);
    }
  }
  static_assert(NW * Rows<NT>::LDS <= C::LDS, "the ring's LDS serves again");
  barrier();  // every wave has read the last stage
  char* mine = smem + wave * Rows<NT>::LDS;
  const int n = n0 + wn * NT * 16;
  if (n + NT * 16 <= p.n && (std::is_same_v<T, float> || !p.add)) {
    // the next 16 rows of `add` are on their way while these are stored
    typename Chunks<T, NT>::Chunk add[2][Chunks<T, NT>::Q];
    const int m = m0 + wm * MT * 16;
    if constexpr (std::is_same_v<T, float>)
      if (p.add) load_add<NT>(p, m, n, add[0]);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if constexpr (std::is_same_v<T, float>)
        if (p.add && i + 1 < MT) load_add<NT>(p, m + (i + 1) * 16, n, add[(i + 1) & 1]);
      store_rows<T, NT, STREAM>(p, mine, m + i * 16, n, acc[i], add[i & 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < MT; ++i) store_values<T, NT>(p, mine, m0 + (wm * MT + i) * 16, n, acc[i]);
  }
}

// ---------------------------------------------------------------- few tokens
// 16*MT tokens x 16 columns by 8 waves, each with its own groups: wave w
// multiplies groups w, w + 8, ... straight from memory, U of them a round, and
// leaves the products in LDS, where the threads (one or more outputs each)
// add them in the order of the groups.  A weight of few rows is then spread
// over the chip along K.  The operands of two rounds are in flight or in
// registers (4 * U * (1 + MT) KB a wave).  Bound by memory for one token (n 28672, k 4096: 117 MB
// in 22.6 us, 5.2 TB/s; n 4096, k 14336: 13.9, 4.2).  What bounds more tokens, whose codes every
// 16 columns read again, is not established (16 tokens 19.0, 24 tokens 24.2 with weights from
// memory, 21.0 with weights in the last cache); twice the loads in flight, or 16 waves, take as
// long.
template <typename R, int MT, int U>
__global__ __launch_bounds__(512, 2) void matmul_few_kernel(const lmop_matmul_args p) {
  using T = typename R::Type;
  constexpr bool WHOLE = R::WHOLE;
  constexpr int NW = 8, CH = NW * U;       // groups of a round
  constexpr int OUT = 256 * MT;            // outputs of the workgroup
  constexpr int PER = (OUT + 511) / 512;   // of a thread
  __shared__ __attribute__((aligned(16))) float prod[2][CH][OUT];
  __shared__ float scl[2][CH][16 * MT + 1];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tn = (p.n + 15) / 16;
  const int m0 = (int)(blockIdx.x / tn) * 16 * MT, n0 = (int)(blockIdx.x % tn) * 16;
  const int kr = (p.k + 15) / 16 * 16, kb_n = (p.k + GROUP - 1) / GROUP;
  const uint8_t* brow = p.b + (size_t)(n0 + c < p.n ? n0 + c : p.n - 1) * p.ldb;
  const uint8_t* arow[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
    arow[i] = p.a + (size_t)(m0 + 16 * i + c < p.m ? m0 + 16 * i + c : p.m - 1) * p.lda;
  // a round's scales: thread t brings group t % CH of token t / CH
  const int st = (int)threadIdx.x / CH, sq = (int)threadIdx.x % CH;
  static_assert(16 * MT * CH <= 512, "a thread brings one scale of a round");
  const float* sa = p.a_scale + (size_t)(m0 + st < p.m ? m0 + st : p.m - 1) * p.ldas;
  const float* sb = p.b_scale + (size_t)(n0 / GROUP) * p.ldbs;
  Codes b[2][U], a[2][U][MT];
  float sak[2], sbk[2];
  auto load = [&](int round, auto set) {
    constexpr int S = decltype(set)::value;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // groups past the last repeat it; their products are not used
      int kb = round * CH + u * NW + wave;
      if (kb >= kb_n) kb = kb_n - 1;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int o = kb * GROUP + 16 * g + 64 * h;
        if (o > kr - 16) o = kr - 16;
        b[S][u].w[h] = *(const uint4*)(brow + o);
#pragma unroll
        for (int i = 0; i < MT; ++i) a[S][u][i].w[h] = *(const uint4*)(arow[i] + o);
      }
    }
    const int kb = round * CH + sq < kb_n ? round * CH + sq : kb_n - 1;
    sak[S] = sa[kb];
    sbk[S] = sb[kb];
  };
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  const int rounds = (kb_n + CH - 1) / CH;
  auto round = [&](int rd, auto set) {
    constexpr int S = decltype(set)::value;
    auto& pr = prod[S];
    auto& sc = scl[S];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = u * NW + wave, kb = rd * CH + q;
      if (kb == kb_n - 1) {
        const Left left = left_of(p.k - kb * GROUP - 16 * g);
        keep(b[S][u], left);
#pragma unroll
        for (int i = 0; i < MT; ++i) keep(a[S][u][i], left);
      }
      const Operand<WHOLE> bo = operand<WHOLE>(b[S][u]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        *(f32x4*)&pr[q][256 * i + 4 * lane] = dot(bo, operand<WHOLE>(a[S][u][i]));
      }
    }
    if (st < 16 * MT) sc[sq][st] = sak[S] * sbk[S];
    if (rd + 2 < rounds) load(rd + 2, set);
    // a round's products are added between this barrier and the next, while
    // the next round's go to the other buffer
    wait_vmcnt_lgkm0<63>();
    barrier();
    const int live = kb_n - rd * CH < CH ? kb_n - rd * CH : CH;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int o = (int)threadIdx.x + 512 * i;
      if (o < OUT) {
        if (live == CH) {
#pragma unroll 8
          for (int q = 0; q < CH; ++q)
            acc[i] = __builtin_fmaf(pr[q][o], sc[q][(o >> 8) * 16 + ((o >> 2) & 15)], acc[i]);
        } else {
          for (int q = 0; q < live; ++q)
            acc[i] = __builtin_fmaf(pr[q][o], sc[q][(o >> 8) * 16 + ((o >> 2) & 15)], acc[i]);
        }
      }
    }
  };
  load(0, std::integral_constant<int, 0>{});
  if (rounds > 1) load(1, std::integral_constant<int, 1>{});
  for (int rd = 0; rd < rounds; rd += 2) {
    round(rd, std::integral_constant<int, 0>{});
    if (rd + 1 < rounds) round(rd + 1, std::integral_constant<int, 1>{});
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    // output o: tile o / 256, lane o / 4 % 64 of its result, register o % 4
    const int o = (int)threadIdx.x + 512 * i;
    const int m = m0 + (o >> 8) * 16 + ((o >> 2) & 15), n = n0 + 4 * ((o >> 6) & 3) + (o & 3);
    if (o < OUT && m < p.m && n < p.n) {
      const float v = acc[i];
      ((T*)p.c)[(size_t)m * p.ldc + n] = (T)(p.add ? p.add[(size_t)m * p.ldadd + n] + v : v);
    }
  }
}

// no features: C = add, or zero
template <typename T>
__global__ __launch_bounds__(256) void matmul_empty_kernel(const lmop_matmul_args p) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)p.m * p.n) return;
  const size_t m = i / p.n, n = i % p.n;
  ((T*)p.c)[m * p.ldc + n] = (T)(p.add ? p.add[m * p.ldadd + n] : 0.f);
}

// Results that the caches (256 MB at last) cannot keep until they are read are
// streamed past them.  fp16 [m][28672], k 4096, and the quantisation that
// reads it, us, streamed against not: 59 MB 131 / 129, 117 MB 257 / 260, 235 MB 484 /
// 490, 940 MB 1910 / 1976.  Rows have to start at 64 bytes: two waves' stores
// share the memory's words otherwise (16282 x 5533, k 359: 116 / 76; 16282 x 5536 of fp32: 125 /
// 140).
constexpr double kStreamBytes = 1e8;

template <typename R, int TILE, bool STREAM>
hipError_t launch_tile_kernel(hipStream_t s, const lmop_matmul_args& a) {
  constexpr Fp8Tile t = kFp8Tiles[TILE];
  using C = Tile<t.mt, t.nt, t.wm, t.wn, t.occ>;
  const size_t tiles = (size_t)((a.m + C::BM - 1) / C::BM) * ((a.n + C::BN - 1) / C::BN);
  auto* k = matmul_tile_kernel<R, t.mt, t.nt, t.wm, t.wn, t.occ, STREAM>;
  // more than 64 KB of LDS: asked for once on each device
  static std::atomic<uint64_t> raised{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (e == hipSuccess && !(raised.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    if (e == hipSuccess) raised.fetch_or(bit, std::memory_order_release);
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)tiles), dim3(64 * C::NW), C::LDS, s, a);
  return hipGetLastError();
}

template <typename R, int TILE>
hipError_t launch_tile(hipStream_t s, const lmop_matmul_args& a) {
  constexpr Fp8Tile t = kFp8Tiles[TILE];
  if constexpr (t.occ == 1) {  // the large tiles, which such results take
    constexpr size_t size = sizeof(typename R::Type);
    if ((double)a.m * a.n * size > kStreamBytes && (uintptr_t)a.c % 64 == 0 &&
        a.ldc * size % 64 == 0)
      return launch_tile_kernel<R, TILE, true>(s, a);
  }
  return launch_tile_kernel<R, TILE, false>(s, a);
}

template <typename R, int MT, int U>
hipError_t launch_few(hipStream_t s, const lmop_matmul_args& a) {
  const size_t tiles = (size_t)((a.m + 16 * MT - 1) / (16 * MT)) * ((a.n + 15) / 16);
  hipLaunchKernelGGL((matmul_few_kernel<R, MT, U>), dim3((unsigned)tiles), dim3(512), 0, s, a);
  return hipGetLastError();
}

template <typename R>
hipError_t launch_part(hipStream_t s, int kernel, const lmop_matmul_args& a) {
  switch (kernel) {
    case 0:
      if constexpr (!R::WHOLE) return launch_tile<R, 0>(s, a);
      return hipErrorInvalidValue;  // not offered
    case 1: return launch_tile<R, 1>(s, a);
    case 2: return launch_tile<R, 2>(s, a);
    case 3: return launch_tile<R, 3>(s, a);
    case 4: return launch_tile<R, 4>(s, a);
    case kFp8Few16: return launch_few<R, 1, 2>(s, a);
    default: return launch_few<R, 2, 1>(s, a);
  }
}

template <typename R>
hipError_t launch_empty(hipStream_t s, const lmop_matmul_args& a) {
  const size_t blocks = ((size_t)a.m * a.n + 255) / 256;
  hipLaunchKernelGGL(matmul_empty_kernel<typename R::Type>, dim3((unsigned)blocks), dim3(256), 0,
                     s, a);
  return hipGetLastError();
}

template <typename R>
hipError_t launch(hipStream_t s, const lmop_matmul_args& a) {
  using T = typename R::Type;
  const int kernel = a.k > 0 ? pick_fp8_kernel(R::WHOLE, a.m, a.n, a.k) : -1;
  const int most = kernel < 0
                       ? (int)std::min<size_t>(a.m, kMaxLaunchThreads / 256 * 256 / a.n)
                       : fp8_rows(kernel, a.m, a.n);
  if (most == 0) return hipErrorInvalidValue;
  for (int done = 0; done < a.m; done += most) {
    lmop_matmul_args p = a;
    p.m = std::min(most, a.m - done);
    p.c = (T*)a.c + (size_t)done * a.ldc;
    if (a.add) p.add = a.add + (size_t)done * a.ldadd;
    if (a.k > 0) {
      p.a = a.a + (size_t)done * a.lda;
      p.a_scale = a.a_scale + (size_t)done * a.ldas;
    }
    const hipError_t e = kernel < 0 ? launch_empty<R>(s, p) : launch_part<R>(s, kernel, p);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_matmul_fp8(hipStream_t s, const lmop_matmul_args& a) {
  if (a.dtype == LMOP_F16) return launch<Result<f16, false>>(s, a);
  if (a.dtype == LMOP_BF16) return launch<Result<bf16, false>>(s, a);
  return a.fast ? launch<Result<float, false>>(s, a) : launch<Result<float, true>>(s, a);
}

}  // namespace lmop
