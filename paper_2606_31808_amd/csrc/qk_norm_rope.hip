// RMSNorm of every query and key head, rotate-half RoPE and the write of keys
// and values into a cache, in one pass over a batch of tokens.
#include "common.h"
#include "kernels.h"

namespace lmop {

namespace {

// One wave per (token, head): the pair (i, i + hd/2) in lane i.  Heads are
// numbered queries, keys, values.
template <typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const QkArgs a) {
  const lmop_qk_norm_rope_args& p = a.t;
  const int lane = threadIdx.x & 63, half = a.hd / 2;
  const int heads = a.nq + 2 * a.nkv;
  const size_t task = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (task >= (size_t)p.n_tokens * heads) return;
  const size_t t = task / heads;
  int h = (int)(task % heads);
  const int sec = h < a.nq ? 0 : h < a.nq + a.nkv ? 1 : 2;
  h -= sec == 0 ? 0 : sec == 1 ? a.nq : a.nq + a.nkv;
  const T* in = sec == 0 ? (const T*)p.q : sec == 1 ? (const T*)p.k : (const T*)p.v;
  if (in == nullptr) return;
  in += t * (sec == 0 ? p.ldq : sec == 1 ? p.ldk : p.ldv) + h * a.hd;
  const int slot = sec == 0 ? 0 : p.slot ? p.slot[t] : (int)t;
  if (sec > 0 && (slot < 0 || slot >= p.n_slots)) return;
  const bool on = lane < half;
  const T r1 = on ? in[lane] : (T)0.f, r2 = on ? in[lane + half] : (T)0.f;
  if (sec == 2) {
    if (!on) return;
    T* o = (T*)p.v_out;
    if (p.v_layout == LMOP_V_ROWS) {
      o += (size_t)slot * p.ldvo + h * a.hd;
      o[lane] = r1;
      o[lane + half] = r2;
    } else {
      o += (size_t)(h * a.hd + lane) * p.ldvo + slot;
      o[0] = r1;
      o[(size_t)half * p.ldvo] = r2;
    }
    return;
  }
  float x1 = (float)r1, x2 = (float)r2;
  const float* gain = sec == 0 ? p.q_gain : p.k_gain;
  if (gain) {
    float ss = x1 * x1 + x2 * x2;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) ss += shfl_xor(ss, o);
    const float r = 1.0f / sqrtf(ss / (float)a.hd + a.eps);
    if (on) {
      x1 = x1 * r * gain[lane];
      x2 = x2 * r * gain[lane + half];
    }
  }
  if (!on) return;
  const int pos = p.pos[t];
  float2 cs = make_float2(NAN, NAN);
  if (pos >= 0 && pos < a.max_seq) cs = a.rope[(size_t)pos * half + lane];
  T* o = sec == 0 ? (T*)p.q_out + t * p.ldqo : (T*)p.k_out + (size_t)slot * p.ldko;
  o += h * a.hd;
  o[lane] = (T)(x1 * cs.x - x2 * cs.y);
  o[lane + half] = (T)(x1 * cs.y + x2 * cs.x);
}

}  // namespace

hipError_t launch_qk_norm_rope(hipStream_t s, const QkArgs& a) {
  const size_t blocks = ((size_t)a.t.n_tokens * (a.nq + 2 * a.nkv) + 3) / 4;
  if (blocks > 0x7fffffffu) return hipErrorInvalidValue;
  if (a.t.dtype == LMOP_F16)
    hipLaunchKernelGGL(qk_norm_rope_kernel<f16>, dim3((unsigned)blocks), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(qk_norm_rope_kernel<bf16>, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace lmop
