// RMSNorm of every query and key head, rotate-half RoPE and the write of keys
// and values into a cache, in one pass over a batch of tokens.
//
// Bound by memory: each element is read and written once (16,384 tokens of 32 + 8
// heads of 128 and their values: 411 MB in 80 us where row evaluation wrote them
// just before, 92 from memory, 4.5 to 5.1 TB/s; 9 tokens: 3 us).  A head is held by
// hd / 16 lanes, lane j with dimensions 8j .. 8j+7 and the same of the upper
// half, so that both members of every rotation pair are in one lane and the
// sum of squares takes two or three exchanges between lanes, without LDS.  A
// wave takes 64 / (hd / 16) heads of a token at a time.
#include "common.h"
#include "kernels.h"

namespace lmop {

namespace {

constexpr int kWaves = 4;       // of a workgroup
constexpr int kValueTokens = 64;  // of a workgroup that transposes values
constexpr int kValueDims = 64;

// 16 bytes, at the alignment of one value
template <typename T>
using Run = T __attribute__((ext_vector_type(8), aligned(sizeof(T))));
typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));

// One workgroup: kValueTokens tokens x kValueDims dimensions of one value
// head, transposed through LDS.  Tokens in consecutive slots (a prompt's) are
// written 16 bytes of a dimension's row at a time where the slots reach a
// multiple of 8; other tokens one value each, the lanes along the slots.
template <typename T, int HD>
LMOP_DEVICE void value_columns(const QkArgs& a, int block, uint16_t (*tile)[kValueDims + 2]) {
  const lmop_qk_norm_rope_args& p = a.t;
  constexpr int DT = HD / kValueDims;
  const int per_tile = a.nkv * DT;
  const int t0 = block / per_tile * kValueTokens, d0 = block % per_tile * kValueDims;
  const int tid = threadIdx.x, lane = tid & 63;
  const int n = p.n_tokens - t0 < kValueTokens ? p.n_tokens - t0 : kValueTokens;
  const T* v = (const T*)p.v + d0;
#pragma unroll
  for (int i = 0; i < kValueTokens * kValueDims / 8 / (64 * kWaves); ++i) {
    const int t = (tid >> 3) + i * 8 * kWaves, d = (tid & 7) * 8;
    if (t < n) {
      const T* src = v + (size_t)(t0 + t) * p.ldv + d;
      const Run<T> r = *(const Run<T>*)src;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const T x = r[j];  // of the vector's element itself the cast takes element 0
        tile[t][d + j] = __builtin_bit_cast(uint16_t, x);
      }
    }
  }
  const int tl = lane < n ? t0 + lane : t0 + n - 1;
  const int slot = p.slot ? p.slot[tl] : tl;
  const int s0 = __shfl(slot, 0, 64);
  const bool here = slot >= 0 && slot < p.n_slots;
  const bool run = __all(here && (lane >= n || slot == s0 + lane));
  __syncthreads();
  uint16_t* out = (uint16_t*)p.v_out + (size_t)d0 * p.ldvo;
  if (run) {
    // chunk j: slots first + 8j .. +7
    const int first = s0 & ~7, chunks = (s0 - first + n + 7) / 8;
    for (int i = tid; i < chunks * kValueDims; i += 64 * kWaves) {
      const int d = i / chunks, j = i - d * chunks;
      const int t = first + 8 * j - s0;
      uint16_t* o = out + (size_t)d * p.ldvo + first + 8 * j;
      if (t >= 0 && t + 8 <= n) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          w[q] = tile[t + 2 * q][d] | (uint32_t)tile[t + 2 * q + 1][d] << 16;
        *(Words*)o = Words{w[0], w[1], w[2], w[3]};
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (t + q >= 0 && t + q < n) o[q] = tile[t + q][d];
      }
    }
  } else if (lane < n && here) {
    for (int d = tid >> 6; d < kValueDims; d += kWaves) out[(size_t)d * p.ldvo + slot] = tile[lane][d];
  }
}

// Blocks below value_blocks transpose values; a wave of the others takes
// `chunks` head chunks of a token, from chunk task % splits * chunks on, and
// goes on with every `waves`-th (token, chunk range).  Heads are numbered
// queries, keys, and (LMOP_V_ROWS) values.
template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves) void qk_norm_rope_kernel(const QkArgs a, int value_blocks,
                                                                   int chunks, int splits) {
  constexpr int LPH = HD / 16;   // lanes of a head
  constexpr int HPW = 64 / LPH;  // heads of a chunk
  const lmop_qk_norm_rope_args& p = a.t;
  if ((int)blockIdx.x < value_blocks) {
    __shared__ uint16_t tile[kValueTokens][kValueDims + 2];
    value_columns<T, HD>(a, blockIdx.x, tile);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int wave =
      __builtin_amdgcn_readfirstlane((blockIdx.x - value_blocks) * kWaves + (threadIdx.x >> 6));
  const int waves = (int)(gridDim.x - value_blocks) * kWaves;
  const int d = lane % LPH * 8;
  const int heads = a.nq + a.nkv + (p.v && p.v_layout == LMOP_V_ROWS ? a.nkv : 0);
  const long tasks = (long)p.n_tokens * splits;
  for (long task = wave; task < tasks; task += waves) {
    const int t = (int)(task / splits), c0 = (int)(task % splits) * chunks;
    const int pos = p.pos ? p.pos[t] : 0;
    const int slot = p.slot ? p.slot[t] : t;
    const bool here = slot >= 0 && slot < p.n_slots;
    // the angles of this lane's dimensions, for all the heads
    float cs[8], sn[8];
    if (pos >= 0 && pos < a.max_seq) {
      const float4* r = (const float4*)(a.rope + (size_t)pos * (HD / 2) + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 w = r[i];
        cs[2 * i] = w.x, sn[2 * i] = w.y, cs[2 * i + 1] = w.z, sn[2 * i + 1] = w.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i] = sn[i] = NAN;
    }
    for (int c = c0; c < c0 + chunks; ++c) {
      const int h = c * HPW + lane / LPH;
      const int sec = h < a.nq ? 0 : h < a.nq + a.nkv ? 1 : 2;
      const int hs = h - (sec == 0 ? 0 : sec == 1 ? a.nq : a.nq + a.nkv);
      const T* in = sec == 0 ? (const T*)p.q + t * p.ldq
                    : sec == 1 ? (const T*)p.k + (a.k_in_slots ? slot : t) * p.ldk
                               : (const T*)p.v + t * p.ldv;
      T* out = sec == 0 ? (T*)p.q_out + t * p.ldqo
               : sec == 1 ? (T*)p.k_out + slot * p.ldko
                          : (T*)p.v_out + slot * p.ldvo;
      const bool on = h < heads && (sec == 0 ? p.q != nullptr
                                             : here && (sec == 2 || p.k != nullptr));
      in += hs * HD + d;
      out += hs * HD + d;
      Run<T> r1 = {}, r2 = {};
      if (on) {
        r1 = *(const Run<T>*)in;
        r2 = *(const Run<T>*)(in + HD / 2);
      }
      if (sec < 2) {
        float x1[8], x2[8], ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x1[i] = (float)r1[i], x2[i] = (float)r2[i];
          ss = __builtin_fmaf(x1[i], x1[i], ss);
          ss = __builtin_fmaf(x2[i], x2[i], ss);
        }
        ss += dpp<0xB1>(ss);
        ss += dpp<0x4E>(ss);
        if constexpr (LPH == 8) ss += dpp<0x141>(ss);
        const float* gain = sec == 0 ? p.q_gain : p.k_gain;
        if (gain) {
          const float rn = __builtin_amdgcn_rsqf(ss * (1.0f / HD) + a.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x1[i] = x1[i] * rn * gain[d + i];
            x2[i] = x2[i] * rn * gain[HD / 2 + d + i];
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          r1[i] = (T)(x1[i] * cs[i] - x2[i] * sn[i]);
          r2[i] = (T)(x1[i] * sn[i] + x2[i] * cs[i]);
        }
      }
      if (on) {
        *(Run<T>*)out = r1;
        *(Run<T>*)(out + HD / 2) = r2;
      }
    }
  }
}

template <typename T, int HD>
hipError_t launch(hipStream_t s, const QkArgs& a) {
  const lmop_qk_norm_rope_args& p = a.t;
  const bool columns = p.v && p.v_layout == LMOP_V_COLUMNS;
  const long value_blocks = columns ? (long)((p.n_tokens + kValueTokens - 1) / kValueTokens) *
                                          a.nkv * (HD / kValueDims)
                                    : 0;
  const int heads = a.nq + a.nkv + (p.v && !columns ? a.nkv : 0);
  const int all = (heads + 64 / (HD / 16) - 1) / (64 / (HD / 16));
  // few tokens: a wave per chunk of heads, to spread them over the chip; many: a
  // wave keeps a token's angles for all its heads.  us, the first against the
  // second: 32 + 8 heads of 128, 9 tokens 3.0 / 5.2, 512 4.9 / 7.4, 2048 10.8 / 13.1, 4096 17.7 /
  // 17.9, 16384 78.2 / 76.6; of 64, 9 tokens 2.9 / 4.0, 2048 7.4 / 7.8, 4096 11.8 / 11.3, 16384
  // 33.6 / 32.2.
  const int chunks = (long)p.n_tokens * all <= 10240 ? 1 : all, splits = all / chunks;
  const long want = ((long)p.n_tokens * splits + kWaves - 1) / kWaves;
  const long blocks = (!p.q && !p.k && (columns || !p.v)) ? 0 : want < 65536 ? want : 65536;
  if ((size_t)(value_blocks + blocks) * 64 * kWaves > kMaxLaunchThreads) return hipErrorInvalidValue;
  hipLaunchKernelGGL((qk_norm_rope_kernel<T, HD>), dim3((unsigned)(value_blocks + blocks)),
                     dim3(64 * kWaves), 0, s, a, (int)value_blocks, chunks, splits);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(hipStream_t s, const QkArgs& a) {
  const bool wide = a.hd == 128;
  if (!wide && a.hd != 64) return hipErrorInvalidValue;
  if (a.t.dtype == LMOP_F16) return wide ? launch<f16, 128>(s, a) : launch<f16, 64>(s, a);
  return wide ? launch<bf16, 128>(s, a) : launch<bf16, 64>(s, a);
}

}  // namespace lmop
