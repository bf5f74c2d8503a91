// The blocks (pages) that a token's attention reads: scores by the pages' mean
// keys, and the largest of them.
//
//   score(b) = (sum of the queries of a kv head's group) . mean[page of b]
//
// in fp64: products of 16-bit values and sums of a few hundred of them fit its 53 bits for ordinary
// values, so scores are exact, and which blocks are chosen depends neither on the order
// of a sum nor on what else is in the call.  Scores stay in LDS, and a wave picks the largest.
//
// Single tokens read each mean once, 16 bytes a lane, and are bound by that; tokens of one sequence are
// taken 16 at a time, with the fp64 matrix instruction, and share the means.  32 contexts of 500 pages (8 kv
// heads of 128: 31 MB): 12 us, of which some 8 are the launch and a workgroup's chain of page look-up,
// means, choice; 2048 tokens of such a context: 73 us, of which 25 are the fp64 matrix instructions.
#include "kernels.h"
#include "paged.h"
#include "select_plan.h"

namespace lmop {

namespace {

constexpr int kTileWaves = kSelectTileWaves;

typedef double f64x4 __attribute__((ext_vector_type(4)));

// a score as it is ranked: NaN, and that of a page that does not exist, as the least
LMOP_DEVICE double ranked(double x, int page) { return page < 0 || x != x ? -INFINITY : x; }

// The sum over a lane and those below it; the largest of all lanes.  (Lanes that a step does not reach add
// `old`, or keep their own.)
template <int CTRL, int ROWS>
LMOP_DEVICE int dpp_rows(int old, int x) {
  return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWS, 0xF, false);
}
LMOP_DEVICE int scan(int x) {
  x += dpp_rows<0x111, 0xF>(0, x);
  x += dpp_rows<0x112, 0xF>(0, x);
  x += dpp_rows<0x114, 0xF>(0, x);
  x += dpp_rows<0x118, 0xF>(0, x);
  x += dpp_rows<0x142, 0xA>(0, x);
  x += dpp_rows<0x143, 0xC>(0, x);
  return x;
}
LMOP_DEVICE float wave_max(float x) {
  auto step = [&](int y) { x = fmaxf(x, __int_as_float(y)); };
  step(dpp_rows<0x111, 0xF>(__float_as_int(x), __float_as_int(x)));
  step(dpp_rows<0x112, 0xF>(__float_as_int(x), __float_as_int(x)));
  step(dpp_rows<0x114, 0xF>(__float_as_int(x), __float_as_int(x)));
  step(dpp_rows<0x118, 0xF>(__float_as_int(x), __float_as_int(x)));
  step(dpp_rows<0x142, 0xA>(__float_as_int(x), __float_as_int(x)));
  step(dpp_rows<0x143, 0xC>(__float_as_int(x), __float_as_int(x)));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Of 256 counts, the value where those from above reach `want`, by the whole wave: the value, how many
// are above it, its own count
struct Cut {
  int value, above, share;
};
LMOP_DEVICE Cut cut_at(const int* count, int want) {
  const int lane = threadIdx.x & 63;
  // lane i: values 255 - 4 i and the three below
  const int4 c4 = *(const int4*)(count + 252 - 4 * lane);
  const int c[4] = {c4.w, c4.z, c4.y, c4.x};
  int before = scan(c[0] + c[1] + c[2] + c[3]) - (c[0] + c[1] + c[2] + c[3]);
  Cut r{-1, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (r.value < 0 && before < want && before + c[i] >= want) r = Cut{255 - 4 * lane - i, before, c[i]};
    before += c[i];
  }
  const int who = __builtin_ctzll(__ballot(r.value >= 0));
  return Cut{__builtin_amdgcn_readlane(r.value, who), __builtin_amdgcn_readlane(r.above, who),
             __builtin_amdgcn_readlane(r.share, who)};
}

// whole numbers in the order of the scores
LMOP_DEVICE uint64_t order_of(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);  // (-0 is 0)
  return (u >> 63) ? ~u : u | (1ull << 63);
}

// By a whole wave: writes to out the `need` largest of score[0 .. n) (no NaN), 0 < need < n, of equal ones
// the first, in ascending order of their index.  count: 256 words of LDS of the wave, 16-byte aligned.
//
// Scores are counted in 256 intervals between the least and the largest.  All above the one where the count
// reaches `need` are chosen, and of those in it, if 64 or fewer, the ones with the lowest rank.  Else the
// least of the chosen is found eight bits at a time.
LMOP_DEVICE void pick(const double* score, int n, int need, int* count, int32_t* out) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = (1ull << lane) - 1;
  // f(first index of 64, this lane's score, whether it is one) in ascending order; eight reads at a time
  auto each = [&](auto&& f) {
    for (int b0 = 0; b0 < n; b0 += 512) {
      double x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int b = b0 + 64 * i + lane;
        x[i] = score[b < n ? b : n - 1];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (b0 + 64 * i < n) f(b0 + 64 * i, x[i], b0 + 64 * i + lane < n);
    }
  };
  auto clear = [&]() {
    wave_order();
    *(int4*)(count + 4 * lane) = int4{0, 0, 0, 0};
    wave_order();
  };
  // classes of scores: above the cut, in it (of which the first `want` are chosen, or those in `marked`), below
  int placed = 0, in_cut = 0;
  auto write = [&](int b0, bool above, bool cut, int want, uint64_t marked) {
    const uint64_t cuts = __ballot(cut);
    const int nth = in_cut + __builtin_popcountll(cuts & below);
    const bool take = above || (cut && nth < want && (nth >= 64 || (marked >> nth & 1)));
    const uint64_t takes = __ballot(take);
    if (take) out[placed + __builtin_popcountll(takes & below)] = b0 + lane;
    placed += __builtin_popcountll(takes);
    in_cut += __builtin_popcountll(cuts);
  };

  float hi = -INFINITY, lo = -INFINITY;  // lo: of the negated scores
  each([&](int, double x, bool) { hi = fmaxf(hi, (float)x), lo = fmaxf(lo, -(float)x); });
  hi = wave_max(hi), lo = -wave_max(lo);
  const float per = 255.0f / (hi - lo);
  if (hi - lo > 0.f && hi - lo < INFINITY && per < INFINITY) {
    auto interval = [&](double x) {  // ascends with x
      const int i = (int)(((float)x - lo) * per);
      return i < 255 ? i : 255;
    };
    clear();
    each([&](int, double x, bool is) {
      if (is) atomicAdd(&count[interval(x)], 1);
    });
    wave_order();
    const Cut cut = cut_at(count, need);
    const int want = need - cut.above;
    if (cut.share <= 64) {
      uint64_t marked = ~0ull;
      if (cut.share > want) {
        // ranks of those in the interval, in the place of the counts
        wave_order();
        double* s = (double*)count;
        int found = 0;
        each([&](int, double x, bool is) {
          const bool in = is && interval(x) == cut.value;
          const uint64_t ins = __ballot(in);
          if (in) s[found + __builtin_popcountll(ins & below)] = x;
          found += __builtin_popcountll(ins);
        });
        wave_order();
        const double mine = s[lane < cut.share ? lane : 0];
        int rank = 0;
        for (int i = 0; i < cut.share; ++i) rank += s[i] > mine || (s[i] == mine && i < lane);
        marked = __ballot(lane < cut.share && rank < want);
      }
      each([&](int b0, double x, bool is) {
        const int i = is ? interval(x) : -1;
        write(b0, i > cut.value, i == cut.value, 64, marked);
      });
      return;
    }
  }
  // `at`: the leading bits (mask) that the least of the chosen has; `want`: how many are chosen of those that
  // share them
  uint64_t at = 0, mask = 0;
  int want = need;
  for (int shift = 56; shift >= 0; shift -= 8) {
    clear();
    each([&](int, double x, bool is) {
      const uint64_t k = order_of(x);
      if (is && (k & mask) == at) atomicAdd(&count[(k >> shift) & 255], 1);
    });
    wave_order();
    const Cut cut = cut_at(count, want);
    at |= (uint64_t)(uint32_t)cut.value << shift;
    mask |= 255ull << shift;
    want -= cut.above;
    if (cut.share == want) break;  // all that share the leading bits
  }
  each([&](int b0, double x, bool is) {
    const uint64_t k = is ? order_of(x) & mask : 0;
    write(b0, is && k > at, is && k == at, want, ~0ull);
  });
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

// One workgroup: a token (from `first` on) and a kv head.
template <typename T, int HD, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void select_one_kernel(const lmop_select_args p, const Heads n, int first) {
  constexpr int kThreads = 64 * WAVES;
  constexpr int LANES = HD / 8;             // of a mean
  constexpr int PAGES = kThreads / LANES;   // of a pass
  constexpr int UNROLL = 8;                 // passes whose loads are under way together
  __shared__ double s_q[HD];
  __shared__ __attribute__((aligned(16))) int s_count[256];
  extern __shared__ __attribute__((aligned(16))) double s_score[];
  const lmop_batch& bt = p.batch;
  const int tid = threadIdx.x;
  const int t = first + blockIdx.x / n.nkv, h = blockIdx.x % n.nkv;
  const int G = n.nq / n.nkv;
  int s = t;
  if (bt.start) {
    if (t < bt.start[0] || t >= bt.start[bt.n_seqs]) return;
    s = find_seq(bt.n_seqs, t, [&](int i) { return bt.start[i]; });
  }
  const int2 tok = seq_tokens(bt, s);
  if (t < tok.x || t >= tok.y) return;  // (starts that do not ascend)
  const int len = bt.length[s];
  int32_t* out = p.blocks + ((size_t)t * n.nkv + h) * p.n_blocks;
  const Choice c = settle(p, (int64_t)len - (tok.y - t), len, out);
  if (c.done) return;
  if (tid < HD) {
    const T* q = (const T*)p.q + t * p.ldq + h * G * HD + tid;
    double sum = 0;
    for (int i = 0; i < G; ++i) sum += (double)(float)q[i * HD];
    s_q[tid] = sum;
  }
  // the pages, in place of the scores that they become
  for (int b = tid; b < c.mine; b += kThreads) s_score[b] = page_of(bt, p.cache.n_pages, s, b);
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
      page[u] = b < c.mine ? (int)s_score[b] : -1;
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
      if (d == 0 && b < c.mine) s_score[b] = ranked(z, page[u]);
    }
  }
  __syncthreads();
  if (tid < 64) pick(s_score, c.mine, c.need, s_count, out);
}

// One workgroup: up to 16 tokens of a sequence (tile number `first` and on) and a kv head.  Scores are a product of the
// tokens' queries and 16 means at a time: lane 16 g + c has token c's dimensions g * HD / 4 .. as the
// one operand and page c's as the other, and gets tokens 4 r + g of page c.
template <typename T, int HD>
__global__ __launch_bounds__(64 * kTileWaves) void select_tile_kernel(const lmop_select_args p, const Heads n, int first,
                                                               int tile, int pages) {
  constexpr int DIMS = HD / 4;
  __shared__ __attribute__((aligned(16))) int s_count[kTileWaves][256];
  extern __shared__ __attribute__((aligned(16))) double s_score[];  // [tile][pages]
  const lmop_batch& bt = p.batch;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int item = first + blockIdx.x / n.nkv, h = blockIdx.x % n.nkv;
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
  typedef typename Half<T>::x8 x8;
  // the next 16 means are on their way while these are multiplied, and their pages before that
  auto look_up = [&](int b0) { return b0 + c < most ? page_of(bt, p.cache.n_pages, s, b0 + c) : -1; };
  auto load = [&](int page, x8 (&x)[DIMS / 8]) {
    const T* src = mean + (size_t)(page < 0 ? 0 : page) * n.nkv * HD;
#pragma unroll
    for (int i = 0; i < DIMS / 8; ++i) x[i] = *(const x8*)(src + 8 * i);
  };
  constexpr int STEP = 16 * kTileWaves;
  x8 next[DIMS / 8];
  int page = look_up(wave * 16), next_page = look_up(wave * 16 + STEP);
  load(page, next);
  for (int b0 = wave * 16; b0 < most; b0 += STEP) {
    x8 x[DIMS / 8];
#pragma unroll
    for (int i = 0; i < DIMS / 8; ++i) x[i] = next[i];
    load(next_page, next);
    const int after = look_up(b0 + 2 * STEP);
    f64x4 z = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < DIMS; ++i)
      z = __builtin_amdgcn_mfma_f64_16x16x4f64(q[i], (double)(float)x[i >> 3][i & 7], z, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = 4 * r + g;
      if (t < nt && b0 + c < most) s_score[(size_t)t * pages + b0 + c] = ranked(z[r], page);
    }
    page = next_page, next_page = after;
  }
  __syncthreads();
  for (int t = wave; t < nt; t += kTileWaves) {
    int32_t* out = p.blocks + ((size_t)(t0 + t) * n.nkv + h) * p.n_blocks;
    const Choice ch = settle(p, index0 + t, len, out);
    if (!ch.done) pick(s_score + (size_t)t * pages, ch.mine, ch.need, s_count[wave], out);
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
  const SelectPlan plan =
      plan_select(SelectSizes{b.n_seqs, b.n_tokens, a.max_length, a.cache.page_size, n.nkv, n.hd, b.start != nullptr});
  const int lds = (plan.tile ? plan.tile : 1) * plan.pages * 8;
  const dim3 threads(64 * plan.waves);
  auto queue = [&](auto kernel, auto... more) {
    const hipError_t e = allow_lds(kernel, lds);
    if (e != hipSuccess) return e;
    for (int64_t first = 0; first < plan.items; first += plan.each) {
      const int64_t items = plan.items - first < plan.each ? plan.items - first : plan.each;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(items * n.nkv)), threads, lds, s, a, n, (int)first, more...);
      const hipError_t l = hipGetLastError();
      if (l != hipSuccess) return l;
    }
    return hipSuccess;
  };
  if (plan.tile) return queue(select_tile_kernel<T, HD>, plan.tile, plan.pages);
  return plan.waves == 16 ? queue(select_one_kernel<T, HD, 16>) : queue(select_one_kernel<T, HD, 4>);
}

}  // namespace

hipError_t launch_select_blocks(hipStream_t s, const lmop_select_args& a, const Heads& n) {
  if (n.hd == 128) return a.dtype == LMOP_F16 ? launch<f16, 128>(s, a, n) : launch<bf16, 128>(s, a, n);
  if (n.hd == 64) return a.dtype == LMOP_F16 ? launch<f16, 64>(s, a, n) : launch<bf16, 64>(s, a, n);
  return hipErrorInvalidValue;
}

}  // namespace lmop
