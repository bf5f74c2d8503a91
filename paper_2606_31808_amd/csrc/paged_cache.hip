// Keys and values of a batch of tokens into the pages of a cache, with the
// rotation on the way, the codes of 8-bit pages, and the mean key of every page that fills.
//
// Bound by memory: each element is read and written once (16,346 tokens of 32 + 8 heads of 128 into 8-bit
// pages: 377 MB in 81 to 86 us, 4.4 to 4.7 TB/s; 8448 of heads of 64, with means, 106 MB in 24 to 28).  A workgroup takes a
// page that the call touches, for one or all kv heads; a head of a token is held by hd / 16
// lanes, lane j with dimensions 8j .. 8j+7 and the same of the upper half, so
// that rotation pairs are in one lane, and a head's largest magnitude takes two or
// three exchanges between lanes.  Pages rather than tokens, because then the workgroup that
// writes a page's last key has all of them in its registers or its page, and the
// mean needs no atomics and no second pass.  Queries are other workgroups of the
// same launch.
#include "kernels.h"
#include "paged.h"

namespace lmop {

namespace {

constexpr int kWaves = 4;

template <typename T>
using Run = T __attribute__((ext_vector_type(8), aligned(sizeof(T))));  // at any alignment

constexpr float kMostF16 = 61440.f;  // 15 * 2^12

// dimensions of one lane: 8 of the lower half of a head, 8 of the upper
struct Dims {
  float lo[8], hi[8];
};

template <typename T>
LMOP_DEVICE Dims load_dims(const T* p, int half) {
  const Run<T> a = *(const Run<T>*)p, b = *(const Run<T>*)(p + half);
  Dims x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x.lo[i] = (float)a[i], x.hi[i] = (float)b[i];
  return x;
}

template <typename T>
LMOP_DEVICE void store_dims(T* p, int half, const Dims& x) {
  Run<T> a, b;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (T)x.lo[i], b[i] = (T)x.hi[i];
  *(Run<T>*)p = a;
  *(Run<T>*)(p + half) = b;
}

// (cos, sin) of this lane's dimensions at a position
struct Angles {
  float cs[8], sn[8];
};
LMOP_DEVICE Angles load_angles(const AppendArgs& a, int64_t pos, int half, int d) {
  Angles w;
  if (pos >= 0 && pos < a.max_seq) {
    const float4* r = (const float4*)(a.rope + (size_t)pos * half + d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = r[i];
      w.cs[2 * i] = v.x, w.sn[2 * i] = v.y, w.cs[2 * i + 1] = v.z, w.sn[2 * i + 1] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w.cs[i] = w.sn[i] = NAN;
  }
  return w;
}

LMOP_DEVICE void turn(Dims& x, const Angles& w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = x.lo[i], b = x.hi[i];
    x.lo[i] = a * w.cs[i] - b * w.sn[i];
    x.hi[i] = a * w.sn[i] + b * w.cs[i];
  }
}

// The codes of a head held by LPH lanes (all lanes of the wave active), and its exponent byte
struct Codes {
  uint2 lo, hi;
  uint32_t exp;
};
LMOP_DEVICE uint2 encode8(const float* y, float scale) {
  uint2 r;
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * scale, y[1] * scale, 0, false);
  r.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * scale, y[3] * scale, w, true);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * scale, y[5] * scale, 0, false);
  r.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * scale, y[7] * scale, w, true);
  return r;
}
template <typename T, int LPH>
LMOP_DEVICE Codes encode(Dims x) {
  // magnitudes as whole numbers: a NaN is the largest
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(x.lo[i]) & 0x7FFFFFFFu, b = __float_as_uint(x.hi[i]) & 0x7FFFFFFFu;
    const uint32_t m = a > b ? a : b;
    top = top > m ? top : m;
  }
  auto most = [&](uint32_t o) { top = top > o ? top : o; };
  most(dpp<0xB1>(top));
  most(dpp<0x4E>(top));
  if constexpr (LPH == 8) most(dpp<0x141>(top));
  if (top >= 0x7F800000u) {
    const uint2 nan = uint2{0x7F7F7F7Fu, 0x7F7F7F7Fu};
    return Codes{nan, nan, 127u};
  }
  if constexpr (sizeof(T) == 2 && __is_same(T, f16)) {
    const uint32_t cap = __float_as_uint(kMostF16);
    top = top < cap ? top : cap;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x.lo[i] = fminf(fmaxf(x.lo[i], -kMostF16), kMostF16);
      x.hi[i] = fminf(fmaxf(x.hi[i], -kMostF16), kMostF16);
    }
  }
  // top = 1.m * 2^E with E = (top >> 23) - 127; 448 = 1.75 * 2^8: e = E - 8, one more
  // where 1.m is above 1.75
  int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = e < -126 ? -126 : e;
  const float scale = exp_scale((uint32_t)(127 - e));
  return Codes{encode8(x.lo, scale), encode8(x.hi, scale), (uint32_t)(e + 127)};
}

LMOP_DEVICE void decode_codes(const uint2& w, float scale, float* y) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t v = i ? w.y : w.x;
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, true);
    y[4 * i] = a[0] * scale, y[4 * i + 1] = a[1] * scale;
    y[4 * i + 2] = b[0] * scale, y[4 * i + 3] = b[1] * scale;
  }
}

// Blocks below kv_blocks: (touched page, group of `heads` kv heads).  The others: a wave takes a token's
// query heads, whose angles are the same, and goes on with every `waves`-th token (272 rows of 60
// tokens of 32 heads of 128 81 us; a wave for every four heads 108).
template <typename T, bool E8, int HD>
__global__ __launch_bounds__(64 * kWaves) void append_kernel(const AppendArgs a, int kv_blocks, int heads) {
  constexpr int LPH = HD / 16, HPW = 64 / LPH;
  constexpr int KEYS = kWaves * HPW;  // of a pass
  const lmop_append_args& p = a.t;
  const lmop_batch& bt = p.batch;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = lane % LPH * 8;

  if ((int)blockIdx.x >= kv_blocks) {
    const int waves = (int)(gridDim.x - kv_blocks) * kWaves;
    for (int t = ((int)blockIdx.x - kv_blocks) * kWaves + wave; t < bt.n_tokens; t += waves) {
      int s = t;
      if (bt.start) {
        if (t < bt.start[0] || t >= bt.start[bt.n_seqs]) continue;
        s = find_seq(bt.n_seqs, t, [&](int i) { return bt.start[i]; });
      }
      const int2 tok = seq_tokens(bt, s);
      if (t < tok.x || t >= tok.y) continue;  // (starts that do not ascend)
      const int64_t index = (int64_t)bt.length[s] - (tok.y - t);
      Angles w;
      if (p.rotate) w = load_angles(a, p.first + index, HD / 2, d);
      for (int h = lane / LPH; h < a.n.nq; h += HPW) {
        Dims x = load_dims((const T*)p.q + t * p.ldq + h * HD + d, HD / 2);
        if (p.rotate) turn(x, w);
        store_dims((T*)p.q_out + t * p.ldqo + h * HD + d, HD / 2, x);
      }
    }
    return;
  }

  const int ps = p.cache.page_size, lps = __builtin_ctz(ps);
  const int groups = (a.n.nkv + heads - 1) / heads;
  const int item = (int)blockIdx.x / groups, h0 = (int)blockIdx.x % groups * heads;
  const int h1 = h0 + heads < a.n.nkv ? h0 + heads : a.n.nkv;
  // the item: page number `nth` of those that sequence s touches
  int s = item, nth = 0;
  if (bt.start) {
    auto base = [&](int i) { return (seq_tokens(bt, i).x >> lps) + 2 * i; };
    s = find_seq(bt.n_seqs, item, base);
    nth = item - base(s);
    if (nth < 0) return;
  }
  const int2 tok = seq_tokens(bt, s);
  const int64_t len = bt.length[s], i0 = len - (tok.y - tok.x);
  const int64_t block = (i0 >> lps) + nth;
  if (tok.y == tok.x || block << lps >= len || block < 0 || block >= bt.max_pages) return;
  const int page = page_of(bt, p.cache.n_pages, s, (int)block);
  if (page < 0) return;
  // slots [lo, hi) of the page are the call's tokens t0 + slot
  const int64_t page0 = block << lps;
  const int lo = (int)(i0 > page0 ? i0 - page0 : 0), hi = (int)(len - page0 < ps ? len - page0 : ps);
  const int64_t t0 = tok.x - (i0 - page0);
  const bool mean = p.cache.k_mean && hi == ps;

  __shared__ double part[kWaves][HD];
  // a pass takes KEYS slots of every head, whose angles stay; where a mean is made, a head's passes
  // follow one another instead
  for (int slot0 = mean ? 0 : lo / KEYS * KEYS; slot0 < hi; slot0 += KEYS) {
    Angles w;
    const int slot = slot0 + threadIdx.x / LPH;
    const bool fresh = slot >= lo && slot < hi;
    if (p.rotate && fresh) w = load_angles(a, p.first + page0 + slot, HD / 2, d);
    for (int h = h0; h < h1; ++h) {
      double sum_lo[8], sum_hi[8];
      if (mean) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_lo[i] = sum_hi[i] = 0;
      }
      for (int sl0 = slot0; sl0 < hi; sl0 += KEYS) {
        const int sl = sl0 + threadIdx.x / LPH;
        const bool now = sl >= lo && sl < hi;
        Dims k = {}, v = {};
        if (now) {
          const int64_t t = t0 + sl;
          k = load_dims((const T*)p.k + t * p.ldk + h * HD + d, HD / 2);
          v = load_dims((const T*)p.v + t * p.ldv + h * HD + d, HD / 2);
          if (p.rotate) {
            if (sl0 != slot0) {
              turn(k, load_angles(a, p.first + page0 + sl, HD / 2, d));
            } else {
              turn(k, w);
            }
          }
        }
        const size_t row = (size_t)h * ps + sl;
        if constexpr (E8) {
          const Codes ck = encode<T, LPH>(k), cv = encode<T, LPH>(v);
          uint8_t* pk = (uint8_t*)p.cache.k + page * p.cache.page_stride + row * HD + d;
          uint8_t* pv = (uint8_t*)p.cache.v + page * p.cache.page_stride + row * HD + d;
          const size_t er = (size_t)page * a.n.nkv * ps + row;
          uint2 wl = ck.lo, wh = ck.hi;
          uint32_t e = ck.exp;
          if (now) {
            *(uint2*)pk = ck.lo, *(uint2*)(pk + HD / 2) = ck.hi;
            *(uint2*)pv = cv.lo, *(uint2*)(pv + HD / 2) = cv.hi;
            if (d == 0) p.cache.k_exp[er] = (uint8_t)ck.exp, p.cache.v_exp[er] = (uint8_t)cv.exp;
          } else if (mean && sl < lo) {
            wl = *(const uint2*)pk, wh = *(const uint2*)(pk + HD / 2);
            e = p.cache.k_exp[er];
          }
          if (mean && sl < hi) {
            decode_codes(wl, exp_scale(e), k.lo);
            decode_codes(wh, exp_scale(e), k.hi);
          }
        } else {
          T* pk = (T*)p.cache.k + page * p.cache.page_stride + row * HD + d;
          T* pv = (T*)p.cache.v + page * p.cache.page_stride + row * HD + d;
          if (now) {
            store_dims(pk, HD / 2, k);
            store_dims(pv, HD / 2, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) k.lo[i] = (float)(T)k.lo[i], k.hi[i] = (float)(T)k.hi[i];
          } else if (mean && sl < lo) {
            k = load_dims((const T*)pk, HD / 2);
          }
        }
        if (!mean) break;
        if (sl < hi) {
#pragma unroll
          for (int i = 0; i < 8; ++i) sum_lo[i] += k.lo[i], sum_hi[i] += k.hi[i];
        }
      }
      if (mean) {
        // over the wave's keys, then over the waves
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
          for (int m = LPH; m < 64; m *= 2) {
            sum_lo[i] += __shfl_xor(sum_lo[i], m, 64);
            sum_hi[i] += __shfl_xor(sum_hi[i], m, 64);
          }
        }
        __syncthreads();
        if (lane < LPH) {
#pragma unroll
          for (int i = 0; i < 8; ++i) part[wave][d + i] = sum_lo[i], part[wave][HD / 2 + d + i] = sum_hi[i];
        }
        __syncthreads();
        if (threadIdx.x < HD) {
          double m = 0;
#pragma unroll
          for (int i = 0; i < kWaves; ++i) m += part[i][threadIdx.x];
          // one rounding: the sum of ordinary keys is exact, and a page a power of two
          const double y = m * (1.0 / ps);
          ((T*)p.cache.k_mean)[((size_t)page * a.n.nkv + h) * HD + threadIdx.x] = (T)y;
        }
      }
    }
    if (mean) break;
  }
}

template <typename T, bool E8, int HD>
hipError_t launch(hipStream_t s, const AppendArgs& a) {
  const lmop_append_args& p = a.t;
  const int64_t items = p.batch.start ? p.batch.n_tokens / p.cache.page_size + 2ll * p.batch.n_seqs
                                      : p.batch.n_seqs;
  // All kv heads in a workgroup take a page's angles once; one each spreads few pages over the chip, and does not
  // make means one after the other.  us, all against one (8 + 32 heads, pages of 64): 1000 tokens 15.5 / 11.4,
  // 4000 23.8 / 20.3, 8448 35.0 / 38.1, 16,384 79.9 / 82.1 (pages of 16 78 / 91); with means, heads of 64, 8448
  // 30.5 / 23.6, 16,384 35.0 / 39.9.
  const int heads = p.batch.n_tokens >= (p.cache.k_mean ? 16384 : 8192) ? a.n.nkv : 1;
  const int64_t kv_blocks = items * ((a.n.nkv + heads - 1) / heads);
  const int64_t want = ((int64_t)p.batch.n_tokens + kWaves - 1) / kWaves;
  const int64_t q_blocks = !p.q ? 0 : want < 65536 ? want : 65536;
  if ((size_t)(kv_blocks + q_blocks) * 64 * kWaves > kMaxLaunchThreads) return hipErrorInvalidValue;
  hipLaunchKernelGGL((append_kernel<T, E8, HD>), dim3((unsigned)(kv_blocks + q_blocks)), dim3(64 * kWaves), 0, s,
                     a, (int)kv_blocks, heads);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(hipStream_t s, const AppendArgs& a) {
  const bool e8 = a.t.cache.dtype == LMOP_E4M3;
  if (a.n.hd == 128) return e8 ? launch<T, true, 128>(s, a) : launch<T, false, 128>(s, a);
  if (a.n.hd == 64) return e8 ? launch<T, true, 64>(s, a) : launch<T, false, 64>(s, a);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_cache_append(hipStream_t s, const AppendArgs& a) {
  return a.t.dtype == LMOP_F16 ? launch_t<f16>(s, a) : launch_t<bf16>(s, a);
}

}  // namespace lmop
