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
// The sum over a group (`dot`), by the type of the result:
//   fp16, bf16: one MFMA 16x16x128 on the codes, at twice the fp16 rate.  It
//     cuts off the bits of a product below 2^-13 of the largest of its eight
//     neighbours (see mfma16x16x128_e4m3): 1.5e-5 to 2.2e-5 of the result's
//     norm on unit-normal tokens and weights (with a feature in a hundred ten
//     times as large: the larger figure), against 2e-4 (fp16) and 1.7e-3
//     (bf16) of the rounding to the type.
//   fp32: the codes converted to fp16, exactly, and four MFMAs 16x16x32,
//     which keep every product whole and add in fp32.
#include "common.h"
#include "kernels.h"
#include "lds_dma.h"

#include <type_traits>

namespace lmop {

namespace {

constexpr int GROUP = LMOP_FP8_GROUP;

// bytes of a 16-byte chunk from `valid` on become zero (+0.0)
LMOP_DEVICE uint4 keep_bytes(uint4 v, int valid) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = valid - 4 * i;
    w[i] = n >= 4 ? w[i] : n <= 0 ? 0u : w[i] & ((1u << (8 * n)) - 1);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A lane's 32 codes of one row and group: lane 16g + c holds features
// 32g .. 32g+31 of row c.
struct Codes {
  uint4 w[2];
};
struct Halves {
  f16x8 h[4];
};

LMOP_DEVICE void keep_valid(Codes& c, int valid) {
  c.w[0] = keep_bytes(c.w[0], valid);
  c.w[1] = keep_bytes(c.w[1], valid - 16);
}

// the operand of `dot`: the codes themselves, or their fp16 values
template <bool F32>
using Operand = std::conditional_t<F32, Halves, Codes>;
template <bool F32>
LMOP_DEVICE Operand<F32> operand(const Codes& c) {
  if constexpr (F32) {
    Halves r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 w = c.w[i >> 1];
      const f16x4 lo = fp8x4(i & 1 ? w.z : w.x), hi = fp8x4(i & 1 ? w.w : w.y);
      r.h[i] = f16x8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    }
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

// Whether rows of C (and add) take the 4-column accesses of store4.
template <typename T>
bool aligned4(const lmop_matmul_args& p) {
  return (uintptr_t)p.c % (4 * sizeof(T)) == 0 && p.ldc % 4 == 0 &&
         (!p.add || ((uintptr_t)p.add % 16 == 0 && p.ldadd % 4 == 0));
}

// columns n .. n+3 of token m
template <typename T>
LMOP_DEVICE void store4(const lmop_matmul_args& p, bool vec, int m, int n, f32x4 v) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  if (m >= p.m) return;
  T* c = (T*)p.c + (size_t)m * p.ldc + n;
  const float* add = p.add ? p.add + (size_t)m * p.ldadd + n : nullptr;
  if (vec && n + 4 <= p.n) {
    if (add) v = *(const f32x4*)add + v;
    *(T4*)c = T4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < p.n) c[r] = (T)(add ? add[r] + v[r] : v[r]);
  }
}

// ---------------------------------------------------------------- tiles through LDS
// A workgroup of WM x WN waves computes 16*MT*WM tokens x 16*NT*WN columns; a
// wave MT x NT tiles of 16 x 16.  One ring stage is one group of the tile's
// rows: 128 bytes a row, 16-byte chunks XOR-swizzled by row, and the tokens'
// scales, filled by direct global->LDS loads.
template <int MT, int NT, int WM, int WN, int OCC>
struct Tile {
  static constexpr int BM = 16 * MT * WM, BN = 16 * NT * WN, NW = WM * WN;
  static constexpr int STAGE = (BM + BN) * 128 + BM * 4;
  static constexpr int NS_FIT = 160 * 1024 / OCC / STAGE;
  static constexpr int NS = NS_FIT < 4 ? NS_FIT : 4;
  static_assert(NS >= 2, "a stage in use and one in flight");
  static_assert(BM % 64 == 0 && (BM + BN) % (8 * NW) == 0, "whole loads");
  static_assert(GROUP % (16 * NT) == 0, "a wave's columns lie in one block of B");
  static constexpr int CODE_LOADS = (BM + BN) / 8 / NW;  // of a wave and stage
  static constexpr int LOADS = CODE_LOADS + 1;           // and the scales
  static constexpr int LDS = NS * STAGE;
};

constexpr int GM = 4;  // token tiles per L2 group

template <typename T, int MT, int NT, int WM, int WN, int OCC>
__global__ __launch_bounds__((64 * WM * WN), ((OCC * WM * WN + 3) / 4)) void matmul_tile_kernel(
    const lmop_matmul_args p, bool vec) {
  using C = Tile<MT, NT, WM, WN, OCC>;
  constexpr bool F32 = std::is_same_v<T, float>;
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
  const bool ragged = p.k % GROUP != 0;

  // Load i of a wave: 8 rows of the stage (tokens first).  Rows past the
  // matrix repeat its last one; chunks past a row's end repeat its last one
  // and are cleared after they are read.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  const uint8_t* abase = p.a + (size_t)m0 * p.lda;
  const uint8_t* bbase = p.b + (size_t)n0 * p.ldb;
  uint32_t rowoff[C::CODE_LOADS];
  const int chunk = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
  for (int i = 0; i < C::CODE_LOADS; ++i) {
    const int r = (wave + NW * i) * 8 + (lane >> 3);
    const int ra = m0 + r < p.m ? r : p.m - 1 - m0;
    const int rb = n0 + r - BM < p.n ? r - BM : p.n - 1 - n0;
    rowoff[i] = (wave + NW * i) * 8 < BM ? (uint32_t)ra * (uint32_t)p.lda
                                         : (uint32_t)rb * (uint32_t)p.ldb;
  }
  const int srow = (wave * 64) % BM + lane;
  const float* sa = p.a_scale + (size_t)(m0 + srow < p.m ? m0 + srow : p.m - 1) * p.ldas;
  auto issue = [&](int kb) {
    const uint32_t st = lds0 + (uint32_t)(kb % NS * C::STAGE);
    const bool last = ragged && kb == kb_n - 1;
    const int o = last && kb * GROUP + chunk > kr - 16 ? kr - 16 - kb * GROUP : chunk;
#pragma unroll
    for (int i = 0; i < C::CODE_LOADS; ++i) {
      const int q = wave + NW * i;
      g2l16_m0((q * 8 < BM ? abase : bbase) + (size_t)kb * GROUP, rowoff[i] + (uint32_t)o,
               st + (uint32_t)q * 1024u);
    }
    g2l4(sa + kb, st + (uint32_t)((BM + BN) * 128 + (wave * 64) % BM * 4));
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int nblk = n0 + wn * NT * 16 < p.n ? (n0 + wn * NT * 16) / GROUP : (p.n - 1) / GROUP;
  const float* sb = p.b_scale + (size_t)nblk * p.ldbs;

  auto step = [&](int kb, auto tail) {
    const char* st = smem + kb % NS * C::STAGE;
    const int valid = p.k - kb * GROUP - 32 * g;
    auto frag = [&](int row) {
      Codes x;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        x.w[i] = *(const uint4*)(st + row * 128 + (((2 * g + i) ^ (c & 7)) * 16));
      if constexpr (decltype(tail)::value) keep_valid(x, valid);
      return operand<F32>(x);
    };
    const float sbk = sb[kb];
    Operand<F32> b[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) b[j] = frag(BM + (wn * NT + j) * 16 + c);
    f32x4 d[2][NT];
    float s[2];
#pragma unroll
    for (int i = 0; i <= MT; ++i) {
      // the tile before is added while this one is multiplied
      if (i < MT) {
        const int row = (wm * MT + i) * 16 + c;
        const Operand<F32> a = frag(row);
        s[i & 1] = *(const float*)(st + (BM + BN) * 128 + row * 4) * sbk;
#pragma unroll
        for (int j = 0; j < NT; ++j) d[i & 1][j] = dot(b[j], a);
      }
      if (i > 0)
#pragma unroll
        for (int j = 0; j < NT; ++j) add_scaled(acc[i - 1][j], d[(i - 1) & 1][j], s[(i - 1) & 1]);
    }
  };

  for (int kb = 0; kb < NS - 1 && kb < kb_n; ++kb) issue(kb);
  for (int kb = 0; kb < kb_n; ++kb) {
    // stage kb has landed for every wave, and every wave is done with the
    // stage before it, which the next loads refill
    if (kb + NS - 2 < kb_n)
      wait_vmcnt_lgkm0<(NS - 2) * C::LOADS>();
    else
      wait_vmcnt_lgkm0<0>();
    barrier();
    if (kb + NS - 1 < kb_n) issue(kb + NS - 1);
    if (ragged && kb == kb_n - 1)
      step(kb, std::true_type{});
    else
      step(kb, std::false_type{});
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
      store4<T>(p, vec, m0 + (wm * MT + i) * 16 + c, n0 + (wn * NT + j) * 16 + 4 * g, acc[i][j]);
}

// ---------------------------------------------------------------- few tokens
// 16*MT tokens x 16 columns by 8 waves, each with its own groups: wave w
// multiplies groups w, w + 8, ... straight from memory, U at a time, and
// leaves the products in LDS, where the threads (one or more outputs each)
// add them in the order of the groups.  A weight of few rows is then spread
// over the chip along K, with U * 2 KB of it in flight per wave.
template <typename T, int MT, int U>
__global__ __launch_bounds__(512, 2) void matmul_few_kernel(const lmop_matmul_args p, bool vec) {
  constexpr bool F32 = std::is_same_v<T, float>;
  constexpr int NW = 8, CH = NW * U;       // groups of a round
  constexpr int OUT = 256 * MT;            // outputs of the workgroup
  constexpr int PER = (OUT + 511) / 512;   // of a thread
  __shared__ __attribute__((aligned(16))) float prod[2][CH][OUT];
  __shared__ float scl[2][CH][16 * MT];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tn = (p.n + 15) / 16;
  const int m0 = (int)(blockIdx.x / tn) * 16 * MT, n0 = (int)(blockIdx.x % tn) * 16;
  const int kr = (p.k + 15) / 16 * 16, kb_n = (p.k + GROUP - 1) / GROUP;
  const uint8_t* brow = p.b + (size_t)(n0 + c < p.n ? n0 + c : p.n - 1) * p.ldb;
  const float* sb = p.b_scale + (size_t)(n0 / GROUP) * p.ldbs;
  const uint8_t* arow[MT];
  const float* sarow[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = m0 + 16 * i + c < p.m ? m0 + 16 * i + c : p.m - 1;
    arow[i] = p.a + (size_t)m * p.lda;
    sarow[i] = p.a_scale + (size_t)m * p.ldas;
  }
  Codes b[U], a[U][MT];
  float s[U][MT];
  auto load = [&](int round) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // groups past the last repeat it; their products are not used
      int kb = round * CH + u * NW + wave;
      if (kb >= kb_n) kb = kb_n - 1;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int o = kb * GROUP + 32 * g + 16 * h;
        if (o > kr - 16) o = kr - 16;
        b[u].w[h] = *(const uint4*)(brow + o);
#pragma unroll
        for (int i = 0; i < MT; ++i) a[u][i].w[h] = *(const uint4*)(arow[i] + o);
      }
      const float sbk = sb[kb];
#pragma unroll
      for (int i = 0; i < MT; ++i) s[u][i] = sarow[i][kb] * sbk;
    }
  };
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  const int rounds = (kb_n + CH - 1) / CH;
  load(0);
  for (int rd = 0; rd < rounds; ++rd) {
    auto& pr = prod[rd & 1];
    auto& sc = scl[rd & 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = u * NW + wave, kb = rd * CH + q;
      const int valid = p.k - kb * GROUP - 32 * g;
      if (kb == kb_n - 1) {
        keep_valid(b[u], valid);
#pragma unroll
        for (int i = 0; i < MT; ++i) keep_valid(a[u][i], valid);
      }
      const Operand<F32> bo = operand<F32>(b[u]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        *(f32x4*)&pr[q][256 * i + 4 * lane] = dot(bo, operand<F32>(a[u][i]));
        if (g == 0) sc[q][16 * i + c] = s[u][i];
      }
    }
    if (rd + 1 < rounds) load(rd + 1);
    // a round's products are added between this barrier and the next, while
    // the next round's go to the other buffer
    __syncthreads();
    const int live = kb_n - rd * CH < CH ? kb_n - rd * CH : CH;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int o = (int)threadIdx.x + 512 * i;
      if (o < OUT)
        for (int q = 0; q < live; ++q)
          acc[i] = __builtin_fmaf(pr[q][o], sc[q][(o >> 8) * 16 + ((o >> 2) & 15)], acc[i]);
    }
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

template <typename T, int MT, int NT, int WM, int WN, int OCC>
hipError_t launch_tile(hipStream_t s, const lmop_matmul_args& a) {
  using C = Tile<MT, NT, WM, WN, OCC>;
  const size_t tiles = (size_t)((a.m + C::BM - 1) / C::BM) * ((a.n + C::BN - 1) / C::BN);
  if (tiles > 0x3fffffffu) return hipErrorInvalidValue;
  auto* k = matmul_tile_kernel<T, MT, NT, WM, WN, OCC>;
  static const hipError_t raised = hipFuncSetAttribute(
      (const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
  if (raised != hipSuccess) return raised;
  hipLaunchKernelGGL(k, dim3((unsigned)tiles), dim3(64 * C::NW), C::LDS, s, a, aligned4<T>(a));
  return hipGetLastError();
}

template <typename T, int MT, int U>
hipError_t launch_few(hipStream_t s, const lmop_matmul_args& a) {
  const size_t tiles = (size_t)((a.m + 16 * MT - 1) / (16 * MT)) * ((a.n + 15) / 16);
  if (tiles > 0x7fffffffu) return hipErrorInvalidValue;
  hipLaunchKernelGGL((matmul_few_kernel<T, MT, U>), dim3((unsigned)tiles), dim3(512), 0, s, a,
                     aligned4<T>(a));
  return hipGetLastError();
}

template <typename T>
hipError_t launch(hipStream_t s, const lmop_matmul_args& a) {
  if (a.k == 0) {
    const size_t blocks = ((size_t)a.m * a.n + 255) / 256;
    if (blocks > 0x7fffffffu) return hipErrorInvalidValue;
    hipLaunchKernelGGL(matmul_empty_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if (a.m <= 16) return launch_few<T, 1, 4>(s, a);
  if (a.m <= 128) return launch_few<T, 2, 2>(s, a);
  return launch_tile<T, 4, 4, 2, 2, 2>(s, a);
}

}  // namespace

hipError_t launch_matmul_fp8(hipStream_t s, const lmop_matmul_args& a) {
  if (a.dtype == LMOP_F16) return launch<f16>(s, a);
  if (a.dtype == LMOP_BF16) return launch<bf16>(s, a);
  return launch<float>(s, a);
}

}  // namespace lmop
