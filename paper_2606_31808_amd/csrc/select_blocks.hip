// The blocks (pages) that a token's attention reads: scores by the pages' mean
// keys, and the largest of them.
//
//   score(b) = (sum of the queries of a kv head's group) . mean[page of b]
//
// in fp64: products of 16-bit values and sums of a few hundred of them fit its 53 bits for ordinary
// values, so scores are exact, and which blocks are chosen depends neither on the order
// of a sum nor on what else is in the call.  A score becomes a 64-bit whole number with the
// same order; the least one of the chosen is found eight bits at a time from the
// counts of the values that remain, and one pass in order writes the chosen ones.
#include "kernels.h"
#include "paged.h"

namespace lmop {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// whole numbers in the order of the scores; NaN below all
LMOP_DEVICE uint64_t order_of(double x) {
  if (x != x) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);  // (-0 is 0)
  return (u >> 63) ? ~u : u | (1ull << 63);
}

// One workgroup: a token and a kv head.  LDS: the group's query, then the blocks' scores.
template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void select_kernel(const lmop_select_args p, const Heads n) {
  constexpr int LANES = HD / 8;             // of a mean
  constexpr int PAGES = kThreads / LANES;   // of a pass
  __shared__ double s_q[HD];
  __shared__ int s_count[256];
  __shared__ int s_pick[2];
  extern __shared__ __attribute__((aligned(16))) uint64_t s_key[];
  const lmop_batch& bt = p.batch;
  const int tid = threadIdx.x, lane = tid & 63;
  const int t = blockIdx.x / n.nkv, h = blockIdx.x % n.nkv;
  const int G = n.nq / n.nkv;
  int s = t;
  if (bt.start) {
    if (t < bt.start[0] || t >= bt.start[bt.n_seqs]) return;
    s = find_seq(bt.n_seqs, t, [&](int i) { return bt.start[i]; });
  }
  const int len = bt.length[s];
  const int64_t index = (int64_t)len - (seq_tokens(bt, s).y - t);
  const int lps = __builtin_ctz(p.cache.page_size);
  const int64_t mine64 = index >> lps;
  int32_t* out = p.blocks + ((size_t)t * n.nkv + h) * p.n_blocks;
  if (index < 0 || len > p.max_length || mine64 >= bt.max_pages) {
    for (int i = tid; i < p.n_blocks; i += kThreads) out[i] = -1;
    return;
  }
  const int mine = (int)mine64;  // blocks before the token's own
  const int need = p.n_blocks - 1 < mine ? p.n_blocks - 1 : mine;
  if (need == mine) {
    for (int i = tid; i < p.n_blocks; i += kThreads) out[i] = i <= mine ? i : -1;
    return;
  }
  if (need == 0) {
    if (tid == 0) out[0] = mine;
    return;
  }
  if (tid < HD) {
    const T* q = (const T*)p.q + t * p.ldq + h * G * HD + tid;
    double sum = 0;
    for (int i = 0; i < G; ++i) sum += (double)(float)q[i * HD];
    s_q[tid] = sum;
  }
  __syncthreads();
  const int d = tid % LANES * 8;
  double q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = s_q[d + i];
  for (int b0 = 0; b0 < mine; b0 += PAGES) {
    const int b = b0 + tid / LANES;
    const int page = b < mine ? page_of(bt, p.cache.n_pages, s, b) : -1;
    double z = 0;
    if (page >= 0) {
      const typename Half<T>::x8 x = *(const typename Half<T>::x8*)((const T*)p.cache.k_mean + ((size_t)page * n.nkv + h) * HD + d);
#pragma unroll
      for (int i = 0; i < 8; ++i) z = __builtin_fma(q[i], (double)(float)x[i], z);
    }
#pragma unroll
    for (int m = 1; m < LANES; m *= 2) z += __shfl_xor(z, m, 64);
    if (tid % LANES == 0 && b < mine) s_key[b] = page >= 0 ? order_of(z) : 0;
  }

  // the need-th largest: `at` holds its leading bits so far, `want` how many are taken among those
  // that share them
  uint64_t at = 0, mask = 0;
  int want = need;
  for (int shift = 56; shift >= 0; shift -= 8) {
    s_count[tid] = 0;
    __syncthreads();
    for (int b = tid; b < mine; b += kThreads)
      if ((s_key[b] & mask) == at) atomicAdd(&s_count[(s_key[b] >> shift) & 255], 1);
    __syncthreads();
    if (tid < 64) {
      // lane i: bins 255 - 4 i and the three below
      int c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = s_count[255 - 4 * lane - i], sum += c[i];
      int before = sum;
#pragma unroll
      for (int m = 1; m < 64; m *= 2) {
        const int o = __shfl_up(before, m, 64);
        if (lane >= m) before += o;
      }
      before -= sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < want && before + c[i] >= want) s_pick[0] = 255 - 4 * lane - i, s_pick[1] = want - before;
        before += c[i];
      }
    }
    __syncthreads();
    at |= (uint64_t)s_pick[0] << shift;
    mask |= 255ull << shift;
    want = s_pick[1];
  }
  // above `at`: taken; equal to it: the first `want`
  if (tid < 64) {
    int placed = 0, equal = 0;
    for (int b0 = 0; b0 < mine; b0 += 64) {
      const int b = b0 + lane;
      const uint64_t k = b < mine ? s_key[b] : 0;
      const bool eq = b < mine && k == at;
      const uint64_t eqs = __ballot(eq), below = (1ull << lane) - 1;
      const bool take = b < mine && (k > at || (eq && equal + __builtin_popcountll(eqs & below) < want));
      const uint64_t takes = __ballot(take);
      if (take) out[placed + __builtin_popcountll(takes & below)] = b;
      placed += __builtin_popcountll(takes);
      equal += __builtin_popcountll(eqs);
    }
    if (lane == 0) out[need] = mine;
  }
}

template <typename T, int HD>
hipError_t launch(hipStream_t s, const lmop_select_args& a, const Heads& n) {
  const int64_t pages = (a.max_length + (int64_t)a.cache.page_size - 1) / a.cache.page_size;
  const int lds = (int)((pages > 1 ? pages : 1) * 8);
  if (lds > 65536 - 4096) {
    const hipError_t e = hipFuncSetAttribute((const void*)select_kernel<T, HD>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((select_kernel<T, HD>), dim3((unsigned)((int64_t)a.batch.n_tokens * n.nkv)), dim3(kThreads),
                     lds, s, a, n);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_select_blocks(hipStream_t s, const lmop_select_args& a, const Heads& n) {
  if (n.hd == 128) return a.dtype == LMOP_F16 ? launch<f16, 128>(s, a, n) : launch<bf16, 128>(s, a, n);
  if (n.hd == 64) return a.dtype == LMOP_F16 ? launch<f16, 64>(s, a, n) : launch<bf16, 64>(s, a, n);
  return hipErrorInvalidValue;
}

}  // namespace lmop
