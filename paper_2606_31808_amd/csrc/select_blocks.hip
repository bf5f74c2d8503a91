// The blocks (pages) that a token's attention reads: scores by the pages' mean
// keys, and the largest of them.
//
//   score(b) = (sum of the queries of a kv head's group) . mean[page of b]
//
// in fp64: products of 16-bit values and sums of a few hundred of them fit its 53 bits for ordinary
// values, so scores are exact, and which blocks are chosen depends neither on the order
// of a sum nor on what else is in the call.  A score becomes a 64-bit whole number with the
// same order and stays in LDS; a wave finds the least one of the chosen eight bits at a time from
// the counts of the values that remain, until those are as many as are wanted, and one pass in order
// writes the chosen ones.
//
// Single tokens read each mean once, 16 bytes a lane, and are bound by that; tokens of one sequence are
// taken 16 at a time, with the fp64 matrix instruction, and share the means.
#include "kernels.h"
#include "paged.h"

namespace lmop {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kTileTokens = 16;
constexpr int kScores = 16384;  // a workgroup holds at most (128 KB)

typedef double f64x4 __attribute__((ext_vector_type(4)));

// whole numbers in the order of the scores; NaN below all
LMOP_DEVICE uint64_t order_of(double x) {
  if (x != x) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);  // (-0 is 0)
  return (u >> 63) ? ~u : u | (1ull << 63);
}

// a wave's own LDS accesses happen in order; the compiler has to keep them so
LMOP_DEVICE void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// By a whole wave: writes to out the `need` largest of key[0 .. n), 0 < need < n, of equal ones
// the first, in ascending order of their index.  count: 256 words of LDS of the wave.
LMOP_DEVICE void pick(const uint64_t* key, int n, int need, int* count, int32_t* out) {
  const int lane = threadIdx.x & 63;
  // `at`: the leading bits (mask) that the least of the chosen has; `want`: how many are chosen of those that
  // share them
  uint64_t at = 0, mask = 0;
  int want = need;
  for (int shift = 56; shift >= 0; shift -= 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) count[64 * i + lane] = 0;
    wave_order();
    for (int b = lane; b < n; b += 64) {
      const uint64_t k = key[b];
      if ((k & mask) == at) atomicAdd(&count[(k >> shift) & 255], 1);
    }
    wave_order();
    // lane i: values 255 - 4 i and the three below
    int c[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = count[255 - 4 * lane - i], sum += c[i];
    int before = sum;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const int o = __shfl_up(before, m, 64);
      if (lane >= m) before += o;
    }
    before -= sum;
    // the value where the counts from above reach `want`: in one lane
    int value = -1, above = 0, share = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (value < 0 && before < want && before + c[i] >= want) value = 255 - 4 * lane - i, above = before, share = c[i];
      before += c[i];
    }
    const int who = __builtin_ctzll(__ballot(value >= 0));
    at |= (uint64_t)(uint32_t)__shfl(value, who, 64) << shift;
    mask |= 255ull << shift;
    want -= __shfl(above, who, 64);
    if (__shfl(share, who, 64) == want) break;  // all that share the leading bits
  }
  // above `at`: chosen; sharing its bits: the first `want`
  int placed = 0, equal = 0;
  for (int b0 = 0; b0 < n && placed < need; b0 += 64) {
    const int b = b0 + lane;
    const uint64_t k = b < n ? key[b] & mask : 0;
    const bool eq = b < n && k == at;
    const uint64_t eqs = __ballot(eq), below = (1ull << lane) - 1;
    const bool take = b < n && (k > at || (eq && equal + __builtin_popcountll(eqs & below) < want));
    const uint64_t takes = __ballot(take);
    if (take) out[placed + __builtin_popcountll(takes & below)] = b;
    placed += __builtin_popcountll(takes);
    equal += __builtin_popcountll(eqs);
  }
}

// What is chosen without scores: *done, or `mine` blocks before the token's own of which `need` are
// chosen.  By a whole wave.
struct Choice {
  int mine, need;
  bool done;
};
LMOP_DEVICE Choice settle(const lmop_select_args& p, int64_t index, int len, int32_t* out) {
  const int lane = threadIdx.x & 63;
  const int64_t mine = index >> __builtin_ctz(p.cache.page_size);
  if (index < 0 || len > p.max_length || mine >= p.batch.max_pages) {
    for (int i = lane; i < p.n_blocks; i += 64) out[i] = -1;
    return Choice{0, 0, true};
  }
  const int need = p.n_blocks - 1 < mine ? p.n_blocks - 1 : (int)mine;
  if (need == mine) {
    for (int i = lane; i < p.n_blocks; i += 64) out[i] = i <= mine ? i : -1;
    return Choice{0, 0, true};
  }
  if (lane == 0) out[need] = (int)mine;
  return Choice{(int)mine, need, need == 0};
}

// One workgroup: a token and a kv head.
template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void select_one_kernel(const lmop_select_args p, const Heads n) {
  constexpr int LANES = HD / 8;             // of a mean
  constexpr int PAGES = kThreads / LANES;   // of a pass
  constexpr int UNROLL = 8;                 // passes whose loads are under way together
  __shared__ double s_q[HD];
  __shared__ int s_count[256];
  extern __shared__ __attribute__((aligned(16))) uint64_t s_key[];
  const lmop_batch& bt = p.batch;
  const int tid = threadIdx.x;
  const int t = blockIdx.x / n.nkv, h = blockIdx.x % n.nkv;
  const int G = n.nq / n.nkv;
  int s = t;
  if (bt.start) {
    if (t < bt.start[0] || t >= bt.start[bt.n_seqs]) return;
    s = find_seq(bt.n_seqs, t, [&](int i) { return bt.start[i]; });
  }
  const int len = bt.length[s];
  int32_t* out = p.blocks + ((size_t)t * n.nkv + h) * p.n_blocks;
  const Choice c = settle(p, (int64_t)len - (seq_tokens(bt, s).y - t), len, out);
  if (c.done) return;
  if (tid < HD) {
    const T* q = (const T*)p.q + t * p.ldq + h * G * HD + tid;
    double sum = 0;
    for (int i = 0; i < G; ++i) sum += (double)(float)q[i * HD];
    s_q[tid] = sum;
  }
  // the pages, in place of the scores that they become
  for (int b = tid; b < c.mine; b += kThreads) s_key[b] = (uint64_t)(int64_t)page_of(bt, p.cache.n_pages, s, b);
  __syncthreads();
  const int d = tid % LANES * 8;
  double q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = s_q[d + i];
  const T* mean = (const T*)p.cache.k_mean + h * HD + d;
  for (int b0 = tid / LANES; b0 < c.mine; b0 += PAGES * UNROLL) {
    typename Half<T>::x8 x[UNROLL];
    int page[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int b = b0 + u * PAGES;
      page[u] = b < c.mine ? (int)s_key[b] : -1;
      x[u] = *(const typename Half<T>::x8*)(mean + (size_t)(page[u] < 0 ? 0 : page[u]) * n.nkv * HD);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      double z = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) z = __builtin_fma(q[i], (double)(float)x[u][i], z);
#pragma unroll
      for (int m = 1; m < LANES; m *= 2) z += __shfl_xor(z, m, 64);
      const int b = b0 + u * PAGES;
      if (d == 0 && b < c.mine) s_key[b] = page[u] >= 0 ? order_of(z) : 0;
    }
  }
  __syncthreads();
  if (tid < 64) pick(s_key, c.mine, c.need, s_count, out);
}

// One workgroup: up to 16 tokens of a sequence (a.tile) and a kv head.  Scores are a product of the
// tokens' queries and 16 means at a time: lane 16 g + c has token c's dimensions g * HD / 4 .. as the
// one operand and page c's as the other, and gets tokens 4 r + g of page c.
template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void select_tile_kernel(const lmop_select_args p, const Heads n, int tile,
                                                               int pages) {
  constexpr int DIMS = HD / 4;
  __shared__ int s_count[kWaves][256];
  extern __shared__ __attribute__((aligned(16))) uint64_t s_key[];  // [tile][pages]
  const lmop_batch& bt = p.batch;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int item = blockIdx.x / n.nkv, h = blockIdx.x % n.nkv;
  const int G = n.nq / n.nkv;
  auto base = [&](int i) { return seq_tokens(bt, i).x / tile + i; };
  const int s = find_seq(bt.n_seqs, item, base);
  const int2 tok = seq_tokens(bt, s);
  const int nth = item - base(s);
  const int t0 = tok.x + nth * tile;
  if (nth < 0 || t0 >= tok.y) return;
  const int nt = tok.y - t0 < tile ? tok.y - t0 : tile;
  const int len = bt.length[s];
  const int64_t index0 = (int64_t)len - (tok.y - t0);
  // the blocks before the last token's own, if it has one
  int64_t most = (index0 + nt - 1) >> __builtin_ctz(p.cache.page_size);
  if (len > p.max_length || most > bt.max_pages) most = len > p.max_length ? 0 : bt.max_pages;

  double q[DIMS];
  {
    double sum[DIMS];
#pragma unroll
    for (int i = 0; i < DIMS; ++i) sum[i] = 0;
    if (c < nt) {
      typedef T xu __attribute__((ext_vector_type(8), aligned(2)));
      const T* src = (const T*)p.q + (t0 + c) * p.ldq + h * G * HD + g * DIMS;
      for (int j = 0; j < G; ++j)
#pragma unroll
        for (int i = 0; i < DIMS; i += 8) {
          const xu x = *(const xu*)(src + j * HD + i);
#pragma unroll
          for (int k = 0; k < 8; ++k) sum[i + k] += (double)(float)x[k];
        }
    }
#pragma unroll
    for (int i = 0; i < DIMS; ++i) q[i] = sum[i];
  }
  const T* mean = (const T*)p.cache.k_mean + h * HD + g * DIMS;
  for (int b0 = wave * 16; b0 < most; b0 += 16 * kWaves) {
    const int b = b0 + c;
    const int page = b < most ? page_of(bt, p.cache.n_pages, s, b) : -1;
    const T* src = mean + (size_t)(page < 0 ? 0 : page) * n.nkv * HD;
    typename Half<T>::x8 x[DIMS / 8];
#pragma unroll
    for (int i = 0; i < DIMS / 8; ++i) x[i] = *(const typename Half<T>::x8*)(src + 8 * i);
    f64x4 z = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < DIMS; ++i)
      z = __builtin_amdgcn_mfma_f64_16x16x4f64(q[i], (double)(float)x[i >> 3][i & 7], z, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = 4 * r + g;
      if (t < nt && b < most) s_key[(size_t)t * pages + b] = page >= 0 ? order_of(z[r]) : 0;
    }
  }
  __syncthreads();
  for (int t = wave; t < nt; t += kWaves) {
    int32_t* out = p.blocks + ((size_t)(t0 + t) * n.nkv + h) * p.n_blocks;
    const Choice ch = settle(p, index0 + t, len, out);
    if (!ch.done) pick(s_key + (size_t)t * pages, ch.mine, ch.need, s_count[wave], out);
  }
}

template <typename K>
hipError_t allow_lds(K kernel, int lds) {
  if (lds <= 32768) return hipSuccess;
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

template <typename T, int HD>
hipError_t launch(hipStream_t s, const lmop_select_args& a, const Heads& n) {
  const lmop_batch& b = a.batch;
  int64_t pages = (a.max_length + (int64_t)a.cache.page_size - 1) / a.cache.page_size;
  if (pages < 1) pages = 1;
  // Sequences of four tokens or more share their means, as long as four tokens' scores fit.
  const int tile = (int)(kScores / pages < kTileTokens ? kScores / pages : kTileTokens);
  if (b.start && b.n_tokens / 4 >= b.n_seqs && tile >= 4) {
    const int64_t items = b.n_tokens / tile + b.n_seqs;
    const int lds = (int)(tile * pages * 8);
    const hipError_t e = allow_lds(select_tile_kernel<T, HD>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((select_tile_kernel<T, HD>), dim3((unsigned)(items * n.nkv)), dim3(kThreads), lds, s, a, n,
                       tile, (int)pages);
  } else {
    const int lds = (int)(pages * 8);
    const hipError_t e = allow_lds(select_one_kernel<T, HD>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((select_one_kernel<T, HD>), dim3((unsigned)((int64_t)b.n_tokens * n.nkv)), dim3(kThreads),
                       lds, s, a, n);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_select_blocks(hipStream_t s, const lmop_select_args& a, const Heads& n) {
  if (n.hd == 128) return a.dtype == LMOP_F16 ? launch<f16, 128>(s, a, n) : launch<bf16, 128>(s, a, n);
  if (n.hd == 64) return a.dtype == LMOP_F16 ? launch<f16, 64>(s, a, n) : launch<bf16, 64>(s, a, n);
  return hipErrorInvalidValue;
}

}  // namespace lmop
