// E4M3 quantisation with one scale per row and group of 128 features, of x or
// of silu(gate) * x (the operand of the block-scaled FP8 products).
#include "common.h"
#include "kernels.h"

namespace lmop {

namespace {

constexpr float kE4m3Max = 448.0f;
constexpr float kAmaxMin = 0x1p-40f;

// One half-wave of 32 lanes per group, four features a lane.
template <typename T>
__global__ __launch_bounds__(256) void quantize_kernel(const lmop_quantize_args p, int groups) {
  const size_t task = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (task >= (size_t)p.rows * groups) return;
  const size_t row = task / groups;
  const int g = (int)(task % groups), lane = threadIdx.x & 31;
  const T* x = (const T*)p.x + row * p.ldx;
  const T* gt = p.gate ? (const T*)p.gate + row * p.ldg : nullptr;
  float y[4], amax = kAmaxMin;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int f = g * LMOP_FP8_GROUP + lane * 4 + i;
    y[i] = f < p.cols ? (float)x[f] : 0.f;
    if (gt && f < p.cols) {
      const float z = (float)gt[f];
      y[i] *= z / (1.0f + expf(-z));
    }
    amax = fmaxf(amax, fabsf(y[i]));
    bad |= !(fabsf(y[i]) < INFINITY);
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    amax = fmaxf(amax, shfl_xor(amax, o));
    bad |= shfl_xor((int)bad, o) != 0;
  }
  if (bad) amax = NAN;
  const float inv = kE4m3Max / amax;
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, w, true);
  const int f = g * LMOP_FP8_GROUP + lane * 4;
  uint32_t code = (uint32_t)w;
  if (f + 4 > p.cols) code = f < p.cols ? code & ((1u << (8 * (p.cols - f))) - 1) : 0u;
  if (f < (p.cols + 15) / 16 * 16) *(uint32_t*)(p.q + row * p.ldq + f) = code;
  if (lane == 0) p.scale[row * p.lds + g] = amax / kE4m3Max;
}

}  // namespace

hipError_t launch_quantize(hipStream_t s, const lmop_quantize_args& a) {
  const int groups = (a.cols + LMOP_FP8_GROUP - 1) / LMOP_FP8_GROUP;
  const size_t blocks = ((size_t)a.rows * groups + 7) / 8;
  if (blocks > 0x7fffffffu) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  if (a.dtype == LMOP_F16)
    hipLaunchKernelGGL(quantize_kernel<f16>, grid, dim3(256), 0, s, a, groups);
  else if (a.dtype == LMOP_BF16)
    hipLaunchKernelGGL(quantize_kernel<bf16>, grid, dim3(256), 0, s, a, groups);
  else
    hipLaunchKernelGGL(quantize_kernel<float>, grid, dim3(256), 0, s, a, groups);
  return hipGetLastError();
}

}  // namespace lmop
