// E4M3 quantisation with one scale per row and group of 128 features, of x or
// of silu(gate) * x (the operand of the block-scaled FP8 products).
//
// Bound by memory: every input is read once, held in registers between the
// maximum and the codes, and every code written once (16384 x 4096 of fp16: 203 MB in 36.4
// us, 5.6 TB/s; 4099 x 14336 of bf16 with a gate: 296 MB in 62.5, 4.7 TB/s, the vector
// units beside it; a copy does 4.8, or 7.2 from the last cache).  Eight lanes hold a
// group, two runs of 8 features each (64 features apart, so that the lanes'
// 16-byte loads lie side by side); the maximum takes three exchanges between
// lanes, without LDS.
#include "common.h"
#include "kernels.h"

#include <algorithm>

namespace lmop {

namespace {

constexpr float kE4m3Max = 448.0f;
constexpr float kAmaxMin = 0x1p-40f;

// 8 features in accesses of 16 bytes, at the alignment of one
template <typename T>
using Run = T __attribute__((ext_vector_type(8), aligned(sizeof(T))));

// features f .. f+7 of a row, zero from cols on
template <typename T>
LMOP_DEVICE void load_run(const T* row, int f, int cols, float (&y)[8]) {
  if (f + 8 <= cols) {
    const Run<T> v = *(const Run<T>*)(row + f);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (float)v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = f + i < cols ? (float)row[f + i] : 0.f;
  }
}

// x * silu(z) = x * z / (1 + exp(-z)), off by a few roundings at every z down
// to -87 (and zero from where exp(-z) leaves fp32).  The rounding of the
// exponent, which grows with |z|, goes into the sum to first order (log2 e is
// held in two parts).  The bounds keep the exponent finite; past them the sum
// is one or infinite already.  Infinite and NaN gates give infinity or NaN.
LMOP_DEVICE float times_silu(float x, float z) {
  constexpr float kLog2e = 0x1.715476p+0f, kLog2eLow = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;
  const float a = __builtin_amdgcn_fmed3f(z, -1000.f, 100.f), t = a * -kLog2e;
  const float rest = __builtin_fmaf(a, -kLog2eLow, __builtin_fmaf(a, -kLog2e, -t));
  const float d = __builtin_fmaf(__builtin_amdgcn_exp2f(t), __builtin_fmaf(rest, kLn2, 1.f), 1.f);
  return z * __builtin_amdgcn_rcpf(d) * x;
}

LMOP_DEVICE uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }

template <typename T, bool GATE>
__global__ __launch_bounds__(256) void quantize_kernel(const lmop_quantize_args p, uint32_t groups,
                                                       uint32_t tasks) {
  const uint32_t task = blockIdx.x * 32u + (threadIdx.x >> 3);
  // lanes past the last task repeat it up to the stores: every lane takes part
  // in the exchanges
  const uint32_t at = task < tasks ? task : tasks - 1;
  const uint32_t row = at / groups, g = at - row * groups;
  const int lane = threadIdx.x & 7, f0 = (int)g * LMOP_FP8_GROUP + lane * 8;
  float y[2][8];
  const T* x = (const T*)p.x + (size_t)row * p.ldx;
#pragma unroll
  for (int h = 0; h < 2; ++h) load_run<T>(x, f0 + 64 * h, p.cols, y[h]);
  if constexpr (GATE) {
    const T* gt = (const T*)p.gate + (size_t)row * p.ldg;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float z[8];
      load_run<T>(gt, f0 + 64 * h, p.cols, z);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[h][i] = times_silu(y[h][i], z[i]);
    }
  }
  // the magnitudes' bits order like the magnitudes, with infinity and then
  // NaN above every finite one
  uint32_t top = __float_as_uint(kAmaxMin);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_u32(top, __float_as_uint(y[h][i]) & 0x7FFFFFFFu);
  top = max_u32(top, dpp<0xB1>(top));
  top = max_u32(top, dpp<0x4E>(top));
  top = max_u32(top, dpp<0x141>(top));
  const float amax = top < 0x7F800000u ? __uint_as_float(top) : NAN;
  const float inv = kE4m3Max / amax;
  if (task >= tasks) return;
  uint8_t* q = p.q + (size_t)row * p.ldq;
  const int up = (p.cols + 15) / 16 * 16;  // codes of features from cols on are zero
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int f = f0 + 64 * h;
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float* v = &y[h][4 * i];
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, c, true);
      w[i] = (uint32_t)c;
      const int n = p.cols - f - 4 * i;  // a NaN group's codes end there too
      if (n < 4) w[i] = n > 0 ? w[i] & ((1u << (8 * n)) - 1) : 0u;
    }
    if (f < up) *(uint2*)(q + f) = make_uint2(w[0], w[1]);
  }
  if (lane == 0) p.scale[(size_t)row * p.lds + g] = amax / kE4m3Max;
}

template <typename T>
hipError_t launch(hipStream_t s, const lmop_quantize_args& a) {
  const size_t groups = ((size_t)a.cols + LMOP_FP8_GROUP - 1) / LMOP_FP8_GROUP;
  auto* k = a.gate ? quantize_kernel<T, true> : quantize_kernel<T, false>;
  const int most = (int)std::min<size_t>(kMaxLaunchThreads / 256 * 32 / groups, a.rows);
  if (most == 0) return hipErrorInvalidValue;
  for (int done = 0, rows; done < a.rows; done += rows) {
    rows = std::min(most, a.rows - done);
    lmop_quantize_args p = a;
    p.x = (const T*)a.x + (size_t)done * a.ldx;
    if (a.gate) p.gate = (const T*)a.gate + (size_t)done * a.ldg;
    p.q = a.q + (size_t)done * a.ldq;
    p.scale = a.scale + (size_t)done * a.lds;
    const size_t tasks = rows * groups;
    hipLaunchKernelGGL(k, dim3((unsigned)((tasks + 31) / 32)), dim3(256), 0, s, p, (uint32_t)groups,
                       (uint32_t)tasks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_quantize(hipStream_t s, const lmop_quantize_args& a) {
  if (a.dtype == LMOP_F16) return launch<f16>(s, a);
  if (a.dtype == LMOP_BF16) return launch<bf16>(s, a);
  return launch<float>(s, a);
}

}  // namespace lmop
