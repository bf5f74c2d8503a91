// Attention of a batch's tokens over a paged cache, and over a prefix that the
// batch shares.
//
// Per query vector (a token and a head; the G heads of a kv head lie side by side)
//   out = sum_i exp(z_i - m) v_i / sum_i exp(z_i - m),   z_i = scale * q . k_i,
// in one pass over the keys: m is a reference that follows the largest score, and
// when it moves, the sums so far are multiplied by exp(m_old - m_new).  Sums over
// disjoint sets of keys join the same way, so a long axis is split among
// workgroups and the prefix is walked once for all sequences' tokens;
// combine_kernel joins the parts.
//
// Kernels:
//  * few vectors (a decode step: G vectors against a sequence's keys).  Bound by
//    reading the cache once.  Keys and values go from memory straight to the registers of
//    the wave that uses them: nothing is shared between waves, so a stage in LDS would only
//    add a copy and a barrier.  32 contexts of 1000 to 32,000 keys, 8-bit, 8 kv heads of 128: 1.16 GB in 227 us,
//    5.1 TB/s; 4 of 32,000, fp16: 524 MB in 99 us.
//  * tiles (prompts, rows, the shared prefix): 128 vectors against blocks of 64 keys
//    in LDS.  Bound by the matrix and vector units: a prompt of 8448 tokens, 32 + 8 heads of 128, 784 to 810 us,
//    740 TFLOP/s and half as much again for the weights' second terms, matrix instructions 50% of the time.
//  * both at once: single tokens behind a long prefix, whose keys tiles of all sequences' tokens read once
//    (256 tokens behind 8192 keys 79 us and 9 to join).
//  * a walk over the blocks that a sequence's tokens chose (2000 tokens, 16 of 500 blocks: 324 us).  Bound by the
//    latency of loads at two waves a SIMD.
//
// All compute S^T = K Q^T and O^T = V^T P^T with the 16x16x32 instruction, so
// that scores, maxima and outputs of a query vector stay in one column of lanes
// (lane 16 g + c: vector c) and P^T leaves the first product in the layout that
// the second one reads, if key rows are taken in score_key's order.  P is held in two terms of the type
// (Weights), each with a product of its own: to 16 bits and more, as the fp32 around it.  Row sums of
// P come from the same instruction, with ones for V^T: they are then the sums of the weights as multiplied,
// and cost the vector units nothing.
#include <math.h>

#include "attend_plan.h"
#include "kernels.h"
#include "lds_dma.h"
#include "paged.h"

namespace lmop {

namespace {

// The tile of 32 keys: score tile hf (0, 1) row m holds key 8 (m / 4) + 4 hf + m % 4, so
// lane group g has scores of keys 8g + 4 hf + r, r = 0..3: 8g .. 8g+7 in order
LMOP_DEVICE int score_key(int hf, int m) { return 8 * (m >> 2) + 4 * hf + (m & 3); }

// (of fmaxf the compiler makes an instruction more for every operand, against signalling NaN)
LMOP_DEVICE float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
LMOP_DEVICE float max3(float a, float b, float c) { return max2(max2(a, b), c); }

// over the lanes 16 and 32 apart: the four lanes of a query vector
LMOP_DEVICE float max4(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

struct Args {
  lmop_attend_args t;
  Heads n;
  AttendLaunch l;
  float c;      // scale * log2(e): weights are 2^(c z' - c m) of the unscaled scores z'
  int flat;     // the launch over the prefix: vectors of all tokens
  int fused;    // own launch that walks the prefix first
  int parts;    // 0: writes the output
  int part0;    // the launch's first part
};

// partial results in the workspace: o [part][token][head][hd], then (m, l) [part][token][head]
LMOP_DEVICE float* part_o(const Args& a, int part, int t, int h) {
  return (float*)a.t.workspace + (((size_t)part * a.t.batch.n_tokens + t) * a.n.nq + h) * a.n.hd;
}
LMOP_DEVICE float2* part_ml(const Args& a, int part, int t, int h) {
  return (float2*)((float*)a.t.workspace + (size_t)a.parts * a.t.batch.n_tokens * a.n.nq * a.n.hd) +
         ((size_t)part * a.t.batch.n_tokens + t) * a.n.nq + h;
}

// The running state of a vector: reference m of the unscaled scores (-inf: none seen yet).  It moves
// only where a score exceeds it by more than 2^8 in weight, so that the sums are seldom rescaled.
LMOP_DEVICE float ref_of(float m) { return m == -INFINITY ? 0.f : m; }

// Weights are 2^(c z - c m) in one multiply-add of c m, rounded: off by half a step of c m, one factor for all of a
// vector's weights, which its division takes away.  From 2^20 on, where that factor leaves 2^(1/32) (at 2^30 it is up to
// 2^64, past either end of the weights' types), scores are taken from the reference before the scale: exact next to it.
// Vectors apart, so that one's large scores leave another's bits.
template <int N>
LMOP_DEVICE float from_reference(f32x4 (&st)[N], float m, float c, float lift) {
  const float ref = ref_of(m), nmc = -ref * c;
  const bool far = fabsf(nmc) > 0x1p20f;
  if (!__any(far)) return nmc + lift;
  const float off = far ? ref : 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) st[i][r] -= off;
  return far ? lift : nmc + lift;
}

// exp2 of a difference of references, 0 where there was none
LMOP_DEVICE float rescale(float m_old, float m_new, float c) {
  return m_old == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_old - m_new) * c);
}

// What a workgroup works on: vectors v0 .. of tokens [tok.x, tok.y); a vector is token
// tok.x + v / G, head kv * G + v % G
struct Tile {
  int2 tok;
  int v0;
  int seq;
  int len;   // keys of the sequence
  bool bad;  // the sequence gets NaN
};

LMOP_DEVICE Tile find_tile(const Args& a, int tile, int vectors) {
  const lmop_batch& b = a.t.batch;
  Tile w{};
  if (a.flat) {
    w.tok = int2{0, b.n_tokens};
    w.v0 = tile * vectors;
    return w;
  }
  const int G = a.n.nq / a.n.nkv;
  if (a.l.per_seq) {
    w.seq = tile / a.l.per_seq;
    w.tok = seq_tokens(b, w.seq);
    w.v0 = tile % a.l.per_seq * vectors;
  } else {
    // sequence s has the tiles from base(s) on, at least as many as it needs
    auto base = [&](int i) { return (int)((int64_t)seq_tokens(b, i).x * G / vectors) + i; };
    w.seq = find_seq(b.n_seqs, tile, base);
    w.tok = seq_tokens(b, w.seq);
    const int nth = tile - base(w.seq);
    w.v0 = nth < 0 ? (w.tok.y - w.tok.x) * G : nth * vectors;
  }
  w.len = b.length[w.seq];
  w.bad = w.len < 0 || w.len > a.t.max_length || w.tok.y - w.tok.x > a.t.max_tokens;
  return w;
}

template <typename T>
LMOP_DEVICE void write_bad(const Args& a, int t, int h, int part, int lane, int lanes) {
  if (a.parts) {
    if (lane == 0) *part_ml(a, part, t, h) = float2{0.f, NAN};
    return;
  }
  for (int d = lane; d < a.n.hd; d += lanes) ((T*)a.t.out)[t * a.t.ldo + h * a.n.hd + d] = (T)NAN;
  if (lane == 0 && a.t.lse) a.t.lse[(size_t)t * a.n.nq + h] = NAN;
}

template <typename T>
LMOP_DEVICE float lse_of(const Args& a, float m, float l) {
  // l > 0 means that some score was finite (the lift taken off before the logarithm, where that is exact)
  constexpr float kLift = Weights<T>::kLift, kDown = kLift > 0 ? 1.f / (1 << (int)kLift) : (float)(1 << (int)-kLift);
  return l == 0.f ? -INFINITY : (m * a.c + __log2f(l * kDown)) * 0.6931471805599453f;
}

// A value that one vector of a workgroup sees and another does not must not reach the second one, but
// 0 * inf and 0 * NaN in its column would.  So where vectors see different keys, infinities and
// NaN among the values become zeros in the product, and are added to the vectors that see
// them: the weight, being positive, does not matter.  Where all vectors see all keys they go through the product, in
// which a second term of zero makes NaN of them; a result that is not finite is what settled() says, for which its keys
// are gone over once more (a prompt of 8448 tokens with an infinity on every page 11 ms instead of 0.8).
template <typename T>
LMOP_DEVICE uint32_t unbounded(uint32_t w) {  // a mask of those of two values that are
  constexpr uint32_t E = __is_same(T, f16) ? 0x7C00u : 0x7F80u;
  return ((w & E) == E ? 0xFFFFu : 0) | ((w >> 16 & E) == E ? 0xFFFF0000u : 0);
}

// four values of the cache, as the product would read them
template <typename T, bool E8>
LMOP_DEVICE f32x4 value4(const lmop_cache& k, const Heads& n, int page, int h, int slot, int d) {
  const size_t row = (size_t)h * k.page_size + slot, at = page * k.page_stride + row * n.hd + d;
  f32x4 r;
  if constexpr (E8) {
    const uint32_t w = *(const uint32_t*)((const uint8_t*)k.v + at);
    const float s = exp_scale(k.v_exp[(size_t)page * n.nkv * k.page_size + row]);
    const auto x = Half<T>::template decode<false>(w, s), y = Half<T>::template decode<true>(w, s);
    r = f32x4{(float)x[0], (float)x[1], (float)y[0], (float)y[1]};
  } else {
    const typename Half<T>::x4 x = *(const typename Half<T>::x4*)((const T*)k.v + at);
    r = f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
  }
  return r;
}

// Four results x of a vector whose weights' sum is l.  Those that are not finite, because their vector saw infinite values or
// NaN in their dimensions, become the sum of these; each(f) calls f with every four values that it saw.  (Where it saw none
// x is what it is, and where l is NaN all are NaN.)
template <typename F>
LMOP_DEVICE f32x4 settled(const f32x4& x, float l, F&& each) {
  bool finite = true;
#pragma unroll
  for (int r = 0; r < 4; ++r) finite = finite && fabsf(x[r]) < INFINITY;
  if (!__any(!finite && l == l)) return x;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f}, y;
  each([&](const f32x4& v) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!(fabsf(v[r]) < INFINITY)) sum[r] += v[r];
  });
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = fabsf(x[r]) < INFINITY || sum[r] == 0.f ? x[r] : sum[r];
  return y;
}

// ---------------------------------------------------------------- few vectors
constexpr int kFewWaves = 4;

// A wave that takes 16 QS vectors against 32 keys at a time, which come from memory to its
// registers, the next chunk's while this one is worked on.  Lanes side by side read a row:
// the caches take four lanes' 64 bytes at a time if they adjoin (a row to each lane, as the first product
// has them, took four times the accesses, and bound the walk over chosen blocks: 403 us, 350 with this).  So
// keys change lanes, through LDS of the wave's own, without a barrier.  Of the values a lane has
// 8 rows (its group's keys), 16 lanes side by side along hd; the second product needs 8 keys of a
// dimension in a lane, so the rows are transposed in registers, half a v_perm an element.
template <typename T, bool E8, int HD, int QS>
struct WaveCore {
  typedef typename Half<T>::x8 x8;
  typedef typename Half<T>::x2 x2;
  static constexpr int NS = HD / 32;  // k-steps of the score product
  static constexpr int NT = HD / 16;  // output tiles; lane column c has dimensions NT c .. of a value row

  const lmop_cache& cache;
  const Heads& n;
  int lane, g, c, h, ps, lps;
  x8 qf[QS][NS];
  f32x4 o[QS][NT], l4[QS];
  float m[QS];
  static constexpr int ROW = HD * (E8 ? 1 : 2);  // bytes of a row
  static constexpr int CH = ROW / 16;            // its 16-byte chunks
  static constexpr int KL = 32 * ROW / 1024;     // loads of a chunk's keys
  char* lds;                                     // 32 rows of keys
  uint4 kr[KL];
  uint2 kx;                                      // the exponents of keys 8 (c / 4) .. +7
  uint32_t vw[8][E8 ? NT / 4 : NT / 2];  // 8 value rows, as they are in the page
  uint2 vx;

  LMOP_DEVICE WaveCore(const Args& a, int h_, char* lds_) : cache(a.t.cache), n(a.n), h(h_), lds(lds_) {
    lane = threadIdx.x & 63;
    g = lane >> 4, c = lane & 15;
    ps = cache.page_size, lps = __builtin_ctz(ps);
    clear();
  }
  LMOP_DEVICE void clear() {
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      m[qs] = -INFINITY;
      l4[qs] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NT; ++i) o[qs][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // q: the vector's first element, NULL past the end
  LMOP_DEVICE void load_query(int qs, const T* q) {
    typedef T xu __attribute__((ext_vector_type(8), aligned(2)));
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      // dimensions of step s: 32 s + 8 g; of 8-bit rows, read 16 at a time, 64 (s / 2) + 16 g + 8 (s % 2)
      const int d = E8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
      const xu x = q ? *(const xu*)(q + d) : xu{};
#pragma unroll
      for (int i = 0; i < 8; ++i) qf[qs][s][i] = x[i];
    }
  }

  // chunk ch of key row r in LDS: the rows that a fragment takes meet every bank
  static LMOP_DEVICE int key_at(int r, int ch) {
    const int m = ((r >> 1) & 12) | (r & 3);  // row r is row m of a score tile
    return r * ROW + (ch ^ (m & (CH - 1))) * 16;
  }
  // A chunk's two halves of 16 keys lie in one page each (at least 0); page and slot are the same for the
  // whole wave
  LMOP_DEVICE void load_keys(const int (&page)[2], const int (&slot)[2]) {
    constexpr int RPL = 64 / CH;  // rows of a load
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const int half = i * RPL / 16;
      const char* base = (const char*)cache.k + (page[half] * cache.page_stride + ((int64_t)h * ps + slot[half]) * HD) * (E8 ? 1 : 2);
      kr[i] = *(const uint4*)(base + (i * RPL % 16 + lane / CH) * ROW + lane % CH * 16);
    }
    if constexpr (E8) {
      const int half = c >> 3;
      kx = *(const uint2*)(cache.k_exp + ((int64_t)(half ? page[1] : page[0]) * n.nkv + h) * ps +
                           (half ? slot[1] : slot[0]) + 8 * ((c >> 2) & 1));
    }
  }
  uint32_t key_exp[2];
  // (other lanes' rows are read in scores(): of the chunk before until here, of this one from here on)
  LMOP_DEVICE void stash_keys() {
    constexpr int RPL = 64 / CH;
    wave_order();
#pragma unroll
    for (int i = 0; i < KL; ++i) *(uint4*)(lds + key_at(i * RPL + lane / CH, lane % CH)) = kr[i];
    wave_order();
    if constexpr (E8) {
      key_exp[0] = (kx.x >> (8 * (c & 3))) & 255u;
      key_exp[1] = (kx.y >> (8 * (c & 3))) & 255u;
    }
  }
  // values of half g / 2 are this lane's
  LMOP_DEVICE int value_half() const { return g >> 1; }
  LMOP_DEVICE void load_values(int64_t page, int slot) {
    const size_t row = (size_t)h * ps + slot + 8 * (g & 1);
    constexpr int W = E8 ? NT / 4 : NT / 2;  // words of a lane's part of a row
    typedef uint32_t words __attribute__((ext_vector_type(W)));
    const char* v = (const char*)cache.v + (page * cache.page_stride + row * HD) * (E8 ? 1 : 2) + 4 * W * c;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (W == 1) {
        vw[j][0] = *(const uint32_t*)(v + j * HD);
      } else {
        const words x = *(const words*)(v + j * HD * (E8 ? 1 : 2));
#pragma unroll
        for (int i = 0; i < W; ++i) vw[j][i] = x[i];
      }
    }
    if constexpr (E8) vx = *(const uint2*)(cache.v_exp + page * n.nkv * ps + row);
  }

  // st[qs][hf]: register r of lane group g is the score of key 8 g + 4 hf + r
  LMOP_DEVICE void scores(f32x4 (&st)[QS][2]) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      x8 k[NS];
      const int row = score_key(hf, c);
      if constexpr (E8) {
        const float sc = exp_scale(key_exp[hf]);
#pragma unroll
        for (int u = 0; u < NS / 2; ++u) {
          const uint4 w = *(const uint4*)(lds + key_at(row, 4 * u + g));
          k[2 * u] = decode8<T>(w.x, w.y, sc);
          k[2 * u + 1] = decode8<T>(w.z, w.w, sc);
        }
      } else {
#pragma unroll
        for (int s = 0; s < NS; ++s) k[s] = *(const x8*)(lds + key_at(row, 4 * s + g));
      }
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) {
        st[qs][hf] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) st[qs][hf] = Half<T>::mfma(k[s], qf[qs][s], st[qs][hf]);
      }
    }
  }

  // the vectors' weights of the chunk and their sums; the states move to a new reference where needed
  LMOP_DEVICE Weights<T> weights(int qs, f32x4 (&st)[2], float cs, float thr) {
    const x8 ones = {(T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f};
    float mb = max3(st[0][0], st[0][1], st[0][2]);
    mb = max3(mb, st[0][3], st[1][0]);
    mb = max3(mb, st[1][1], st[1][2]);
    mb = max4(max2(mb, st[1][3]));
    if (__any(mb > m[qs] + thr)) {
      const float m_new = mb > m[qs] + thr ? mb : m[qs];
      const float alpha = rescale(m[qs], m_new, cs);
      l4[qs] *= alpha;
#pragma unroll
      for (int i = 0; i < NT; ++i) o[qs][i] *= alpha;
      m[qs] = m_new;
    }
    const float nmc = from_reference(st, m[qs], cs, Weights<T>::kLift);
    Weights<T> pb;
    auto weight = [&](float z) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z, cs, nmc)); };
    pb.template set<0>(weight(st[0][0]), weight(st[0][1]));
    pb.template set<2>(weight(st[0][2]), weight(st[0][3]));
    pb.template set<4>(weight(st[1][0]), weight(st[1][1]));
    pb.template set<6>(weight(st[1][2]), weight(st[1][3]));
    l4[qs] = Half<T>::mfma(ones, pb.hi, l4[qs]);
    l4[qs] = Half<T>::mfma(ones, pb.lo, l4[qs]);
    return pb;
  }

  // The lane's value rows as 16-bit words.  Those from `any` on, which no vector sees, become zeros: they
  // may hold anything.  With `bounded` infinities and NaN in the others do too; returns the rows that have some.
  LMOP_DEVICE uint32_t values(uint32_t (&w)[8][NT / 2], bool mend, int any, bool bounded) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (E8) {
        const float sc = exp_scale(((j < 4 ? vx.x : vx.y) >> (8 * (j & 3))) & 255u);
#pragma unroll
        for (int i = 0; i < NT / 4; ++i) {
          w[j][2 * i] = __builtin_bit_cast(uint32_t, Half<T>::template decode<false>(vw[j][i], sc));
          w[j][2 * i + 1] = __builtin_bit_cast(uint32_t, Half<T>::template decode<true>(vw[j][i], sc));
        }
      } else {
#pragma unroll
        for (int i = 0; i < NT / 2; ++i) w[j][i] = vw[j][i];
      }
    }
    uint32_t odd = 0;
    if (mend) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < NT / 2; ++i) {
          if (j >= any) w[j][i] = 0;
          if (!bounded) continue;
          const uint32_t out = unbounded<T>(w[j][i]);
          if (out) odd |= 1u << j, w[j][i] &= ~out;
        }
    }
    return odd;
  }

  // O^T += V^T P^T.  Tile i: dimension NT c + i of the lane group's 8 keys
  LMOP_DEVICE void product(const uint32_t (&w)[8][NT / 2], const Weights<T> (&pb)[QS]) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
      uint32_t x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = __builtin_amdgcn_perm(w[2 * q + 1][i >> 1], w[2 * q][i >> 1], sel);
      const x8 v = __builtin_bit_cast(x8, uint4{x[0], x[1], x[2], x[3]});
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) o[qs][i] = Half<T>::mfma(v, pb[qs].hi, o[qs][i]);
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) o[qs][i] = Half<T>::mfma(v, pb[qs].lo, o[qs][i]);
    }
  }

  LMOP_DEVICE bool finite() const {
    float sum = 0.f;  // of zeros, and NaN where one is infinite or NaN
#pragma unroll
    for (int qs = 0; qs < QS; ++qs)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum = __builtin_fmaf(o[qs][i][r], 0.f, sum);
    return sum == 0.f;
  }

  // the infinities and NaN of a value row that were left out, for the vectors that see it
  LMOP_DEVICE void add_unbounded(int page, int slot, const bool (&sees)[QS]) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NT; i += 4) {
        const f32x4 x = value4<T, E8>(cache, n, page, h, slot, NT * (4 * g + r) + i);
#pragma unroll
        for (int qs = 0; qs < QS; ++qs)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (sees[qs] && !(fabsf(x[q]) < INFINITY)) o[qs][i + q][r] += x[q];
      }
  }
};

// One workgroup: 16 vectors x a kv head x a split.  Its pages are looked up once, into LDS; wave
// w takes the 32-key chunks w, w + WAVES, ...; the waves' states are joined through LDS at the
// end.
template <typename T, bool E8, int HD, int WAVES>
struct FewLds {
  typedef WaveCore<T, E8, HD, 1> Core;
  static constexpr int ORow = HD + 4;  // of the joined outputs
  static constexpr int KEYS = 32 * Core::ROW, OUTS = 16 * ORow * 4;
  union {  // the waves' keys, and in their place at the end their outputs
    char keys[WAVES][KEYS];
    float o[WAVES][16][ORow];
  };
  float ml[WAVES][2][16];
  int page[kMaxEntries + 4], first[kMaxEntries + 4], cap[kMaxEntries + 4];
};

template <typename T, bool E8, int HD, bool BLOCKS, int WAVES>
LMOP_DEVICE void few_vectors(const Args& a, int block, int split, FewLds<T, E8, HD, WAVES>& lds) {
  typedef WaveCore<T, E8, HD, 1> Core;
  typedef typename Core::x8 x8;
  constexpr int NT = Core::NT;
  auto& s_o = lds.o;
  auto& s_ml = lds.ml;
  int *e_page = lds.page, *e_first = lds.first, *e_cap = lds.cap;
  const lmop_attend_args& p = a.t;
  const int lane = threadIdx.x & 63, tid = WAVES == 1 ? lane : threadIdx.x;
  const int wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  // what the waves have written is there for all of them
  auto meet = [&]() {
    if constexpr (WAVES == 1)
      wave_order();
    else
      __syncthreads();
  };
  const int tile = block / a.n.nkv, h = block % a.n.nkv;
  const int G = a.n.nq / a.n.nkv;
  const int part = a.part0 + split;

  Tile w;
  if constexpr (BLOCKS) {
    const int t = tile / a.l.per_seq;
    w = Tile{};
    w.seq = t;
    if (p.batch.start) {
      if (t < p.batch.start[0] || t >= p.batch.start[p.batch.n_seqs]) return;
      w.seq = find_seq(p.batch.n_seqs, t, [&](int i) { return p.batch.start[i]; });
    }
    const int2 all = seq_tokens(p.batch, w.seq);
    if (t < all.x || t >= all.y) return;  // (starts that do not ascend)
    // the sequence as it was at this token
    w.tok = int2{t, t + 1};
    const int len = p.batch.length[w.seq];
    w.bad = len < 0 || len > p.max_length || all.y - all.x > p.max_tokens;
    w.len = w.bad ? 0 : len - (all.y - t) + 1;
    w.v0 = tile % a.l.per_seq * kFewVectors;
  } else {
    w = find_tile(a, tile, kFewVectors);
  }
  const int nv = (w.tok.y - w.tok.x) * G;  // vectors
  if (w.bad) {
    // a workgroup of the sequence's first tile does all of its tokens: there may be more than max_tokens
    if (w.v0 == 0)
      for (int v = wave; v < nv; v += WAVES)
        write_bad<T>(a, w.tok.x + v / G, h * G + v % G, part, lane, 64);
    return;
  }
  if (w.v0 >= nv) return;

  // the keys that the tile's vectors see, and the pages that hold them
  Core k(a, h, lds.keys[wave]);
  const int ps = k.ps, lps = k.lps;
  const int n_tok = w.tok.y - w.tok.x;
  const int t_first = w.v0 / G;
  const int t_last = (w.v0 + kFewVectors - 1) / G < n_tok ? (w.v0 + kFewVectors - 1) / G : n_tok - 1;
  // index of the last key that a token of the sequence sees
  const int lim_max = w.len - n_tok + t_last;
  const bool shared = a.flat || a.fused;
  const int n_pre = shared ? (int)((p.prefix_length + (int64_t)ps - 1) >> lps) : 0;
  const int n_own = a.flat ? 0 : BLOCKS ? p.n_blocks : lim_max < 0 ? 0 : (lim_max >> lps) + 1;
  const int64_t from = (int64_t)split * a.l.chunk;
  const int64_t left = (int64_t)n_pre + n_own - from;
  const int ne = (int)(left < 0 ? 0 : left < a.l.chunk ? left : a.l.chunk);
  const int32_t* list = BLOCKS ? p.blocks + ((size_t)w.tok.x * a.n.nkv + h) * p.n_blocks : nullptr;
  bool ascending = true;
  if constexpr (BLOCKS) {
    for (int i = tid + 1; i < p.n_blocks; i += 64 * WAVES)
      ascending = ascending && (list[i] < 0 || (list[i - 1] >= 0 && list[i] > list[i - 1]));
    if constexpr (WAVES == 1)
      ascending = __all(ascending);
    else
      ascending = !__syncthreads_or(!ascending);
  }
  // (one entry more: of 16-token pages, an odd number of them ends inside a chunk)
  for (int i = tid; i <= ne; i += 64 * WAVES) {
    int page = 0, first = 0, cap = 0;
    if (i < ne) {
      const int e = (int)from + i;
      if (e < n_pre) {
        const int q = p.prefix[e];
        page = q >= 0 && q < p.cache.n_pages ? q : -1;
        first = -(1 << 28);  // every token sees it: indexes are above -2^24 and below 2^30
        cap = p.prefix_length - (e << lps) < ps ? p.prefix_length - (e << lps) : ps;
      } else {
        int b = e - n_pre;
        if constexpr (BLOCKS) {
          // one listed twice counts once; lists of select_blocks ascend, which rules that out at a glance
          const int at = b;
          b = list[at];
          bool twice = false;
          for (int j = ascending ? at : 0; j < at; ++j) twice = twice || list[j] == b;
          if (twice) b = -1;
        }
        // (a block past what the token sees is left out here, so its page does not matter)
        if (b >= 0 && b < p.batch.max_pages && b <= (lim_max >> lps)) {
          page = page_of(p.batch, p.cache.n_pages, w.seq, b);
          first = b << lps;
          cap = ps;
        }
      }
    }
    e_page[i] = page, e_first[i] = first, e_cap[i] = cap;
  }

  // this lane's query vector
  const int v = w.v0 + k.c;
  const int tok = v < nv ? v / G : t_last;
  const int lim = a.flat ? 0 : w.len - n_tok + tok, lim_any = a.flat ? 0 : lim_max;
  const bool one = t_first == t_last || a.flat;  // all vectors see the same keys
  k.load_query(0, v < nv ? (const T*)p.q + (int64_t)(w.tok.x + tok) * p.ldq + (h * G + v - tok * G) * HD : nullptr);
  meet();

  const float thr = 8.0f / a.c;
  const int n_keys = ne << lps;
  auto load_keys = [&](int kb) {
    int page[2], slot[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = kb + 16 * i, q = __builtin_amdgcn_readfirstlane(e_page[at >> lps]);
      page[i] = q < 0 ? 0 : q, slot[i] = at & (ps - 1);
    }
    k.load_keys(page, slot);
  };
  auto load_values = [&](int kb) {
    const int at = kb + 16 * k.value_half(), page = e_page[at >> lps];
    k.load_values(page < 0 ? 0 : page, at & (ps - 1));
  };
  constexpr int STEP = 32 * WAVES;
  if (wave * 32 < n_keys) {
    load_keys(wave * 32);
    load_values(wave * 32);
  }
  for (int kb = wave * 32; kb < n_keys; kb += STEP) {
    f32x4 st[1][2];
    k.stash_keys();
    if (kb + STEP < n_keys) load_keys(kb + STEP);
    k.scores(st);
    // of the lane's 8 keys (4 hf + r), its vector sees the first `seen`; any vector the first `any`
    const int at = kb + 16 * k.value_half(), e = at >> lps, slot = (at & (ps - 1)) + 8 * (k.g & 1);
    const bool gone = e_page[e] < 0;
    const int room = e_cap[e] - slot, first = e_first[e] + slot;
    const int seen = room < lim - first + 1 ? room : lim - first + 1;
    const int any = gone ? 0 : room < lim_any - first + 1 ? room : lim_any - first + 1;
    const bool whole = __all(seen >= 8 && !gone);
    if (!whole) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          st[0][hf][r] = 4 * hf + r < seen ? (gone ? NAN : st[0][hf][r]) : -INFINITY;
    }
    const Weights<T> pb[1] = {k.weights(0, st[0], a.c, thr)};
    uint32_t vals[8][NT / 2];
    const uint32_t odd = k.values(vals, !whole, any, !one);
    k.product(vals, pb);
    if (kb + STEP < n_keys) load_values(kb + STEP);
    if (__any(odd != 0)) {
      for (int j = 0; j < 32; ++j) {
        // key j of the chunk, its rows held by the lanes of group j / 8
        if (!((__ballot((odd >> (j & 7)) & 1) >> (16 * (j >> 3))) & 0xFFFF)) continue;
        const int key = kb + j;
        const bool sees[1] = {e_first[key >> lps] + (key & (ps - 1)) <= lim};
        k.add_unbounded(e_page[key >> lps], key & (ps - 1), sees);
      }
    }
  }

  if (__any(!k.finite())) {  // seldom
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NT; i += 4) {
        const f32x4 x = settled(f32x4{k.o[0][i][r], k.o[0][i + 1][r], k.o[0][i + 2][r], k.o[0][i + 3][r]}, k.l4[0][0], [&](auto&& f) {
          for (int kb = wave * 32; kb < n_keys; kb += STEP)
#pragma unroll 4
            for (int key = kb; key < kb + 32 && key < n_keys; ++key) {
              const int e = key >> lps, slot = key & (ps - 1);
              if (e_page[e] >= 0 && slot < e_cap[e] && e_first[e] + slot <= lim)
                f(value4<T, E8>(p.cache, a.n, e_page[e], h, slot, NT * (4 * k.g + r) + i));
            }
        });
#pragma unroll
        for (int q = 0; q < 4; ++q) k.o[0][i + q][r] = x[q];
      }
  }

  // join the waves
  const int g = k.g, c = k.c;
  if (g == 0) s_ml[wave][0][c] = k.m[0], s_ml[wave][1][c] = k.l4[0][0];
  meet();
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) top = fmaxf(top, s_ml[i][0][c]);
  const float f = rescale(k.m[0], top, a.c);
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < NT; i += 4) {
      const f32x4 y = {k.o[0][i][r] * f, k.o[0][i + 1][r] * f, k.o[0][i + 2][r] * f, k.o[0][i + 3][r] * f};
      *(f32x4*)&s_o[wave][c][NT * (4 * g + r) + i] = y;
    }
  meet();
  // 16 lanes a vector, NT dimensions each
  for (int vo = tid >> 4; vo < kFewVectors && w.v0 + vo < nv; vo += 4 * WAVES) {
    const int d = (tid & 15) * NT;
    const int t = w.tok.x + (w.v0 + vo) / G, ho = h * G + (w.v0 + vo) % G;
    float mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mt = fmaxf(mt, s_ml[i][0][vo]);
    float y[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) y[i] = 0.f;
#pragma unroll
    for (int q = 0; q < WAVES; ++q) {
      const float lq = s_ml[q][1][vo];
      lt += lq != lq ? lq : lq * rescale(s_ml[q][0][vo], mt, a.c);
#pragma unroll
      for (int i = 0; i < NT; i += 4) {
        const f32x4 x = *(const f32x4*)&s_o[q][vo][d + i];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[i + r] += x[r];
      }
    }
    if (a.parts) {
      float* dst = part_o(a, part, t, ho) + d;
#pragma unroll
      for (int i = 0; i < NT; i += 4) *(f32x4*)(dst + i) = f32x4{y[i], y[i + 1], y[i + 2], y[i + 3]};
      if (d == 0) *part_ml(a, part, t, ho) = float2{mt, lt};
      continue;
    }
    const float inv = lt == 0.f ? 0.f : 1.0f / lt;
    typedef T xo __attribute__((ext_vector_type(NT), aligned(2)));
    xo r;
#pragma unroll
    for (int i = 0; i < NT; ++i) r[i] = (T)(lt == 0.f ? 0.f : y[i] * inv);
    *(xo*)((T*)p.out + t * p.ldo + ho * HD + d) = r;
    if (p.lse && d == 0) p.lse[(size_t)t * a.n.nq + ho] = lse_of<T>(a, mt, lt);
  }
}

// Chosen blocks of neighbouring tokens: a wave, alone, takes 32 vectors (8 tokens of 4 heads) and walks
// the blocks that any of its tokens chose, in ascending order, a window of kWindow
// at a time.  Neighbours choose many blocks in common, and waves that walk the same way
// find them in their L2, if the waves of a kv head are on one XCD (consecutive workgroups are dealt
// to the eight XCDs in turn).
constexpr int kWindow = kWalkWindow;
constexpr int kWalkTokens = kWalkVectors;  // at most, with one head a group

template <typename T, bool E8, int HD>
__global__ __launch_bounds__(64, 2) void walk_kernel(const Args a) {
  constexpr int QS = kWalkVectors / 16;
  typedef WaveCore<T, E8, HD, QS> Core;
  typedef typename Core::x8 x8;
  constexpr int NT = Core::NT;
  static_assert(kWalkTokens <= 32, "a word of tokens");
  __shared__ uint32_t s_mask[kWindow];                           // the window's blocks: which tokens chose them
  __shared__ int s_id[kWindow + 2], s_page[kWindow + 2];         // the chosen ones
  __shared__ uint32_t s_who[kWindow + 2];
  __shared__ __attribute__((aligned(16))) char s_keys[32 * Core::ROW];

  const lmop_attend_args& p = a.t;
  const int lane = threadIdx.x;
  const int h = blockIdx.x % a.n.nkv, split = blockIdx.y, part = a.part0 + split;
  const int G = a.n.nq / a.n.nkv;
  const Tile w = find_tile(a, (int)blockIdx.x / a.n.nkv, kWalkVectors);
  const int n_tok = w.tok.y - w.tok.x, nv = n_tok * G;
  if (w.v0 >= nv) return;
  if (w.bad) {
    const int end = a.l.per_seq && w.v0 + kWalkVectors >= a.l.per_seq * kWalkVectors ? nv : w.v0 + kWalkVectors;
    for (int v = w.v0; v < end && v < nv; ++v) write_bad<T>(a, w.tok.x + v / G, h * G + v % G, part, lane, 64);
    return;
  }
  const int t_first = w.v0 / G;
  const int t_last = (w.v0 + kWalkVectors - 1) / G < n_tok ? (w.v0 + kWalkVectors - 1) / G : n_tok - 1;
  const int lim0 = w.len - n_tok, lim_max = lim0 + t_last;

  Core k(a, h, s_keys);
  const int ps = k.ps, lps = k.lps;
  int lim[QS];
  uint32_t bit[QS];
#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    const int v = w.v0 + 16 * qs + k.c;
    const int tok = v < nv ? v / G : t_last;
    lim[qs] = v < nv ? lim0 + tok : -1;
    bit[qs] = 1u << (tok - t_first);
    k.load_query(qs, v < nv ? (const T*)p.q + (int64_t)(w.tok.x + tok) * p.ldq + (h * G + v - tok * G) * HD : nullptr);
  }
  const float thr = 8.0f / a.c;
  const int32_t* lists = p.blocks + ((size_t)(w.tok.x + t_first) * a.n.nkv + h) * p.n_blocks;
  const int n_list = (t_last - t_first + 1) * p.n_blocks;
  const int blocks = lim_max < 0 ? 0 : (lim_max >> lps) + 1;
  const int64_t w_from = (int64_t)split * a.l.chunk * kWindow;
  const int first_block = w_from < blocks ? (int)w_from : blocks;
  const int last_block =
      blocks - first_block < (int64_t)a.l.chunk * kWindow ? blocks : first_block + a.l.chunk * kWindow;

  // Infinities and NaN among the values reach vectors that do not see them (0 * inf).  They are rare, so the
  // walk looks for them only when it has to go again: careful.
  for (int careful = 0; careful < 2; ++careful) {
    for (int wb = first_block; wb < last_block; wb += kWindow) {
      const int wn = last_block - wb < kWindow ? last_block - wb : kWindow;
      __syncthreads();
      for (int i = lane; i < kWindow; i += 64) s_mask[i] = 0;
      __syncthreads();
      for (int i = lane; i < n_list; i += 64) {
        const int t = i / p.n_blocks, b = lists[(size_t)t * a.n.nkv * p.n_blocks + (i - t * p.n_blocks)];
        if (b >= wb && b - wb < wn && b <= ((lim0 + t_first + t) >> lps)) atomicOr(&s_mask[b - wb], 1u << t);
      }
      __syncthreads();
      int ne = 0;
      for (int i = 0; i < kWindow; i += 64) {
        const uint32_t who = s_mask[i + lane];
        const uint64_t set = __ballot(who != 0);
        if (who) {
          const int at = ne + __builtin_popcountll(set & ((1ull << lane) - 1));
          s_id[at] = wb + i + lane;
          s_who[at] = who;
          s_page[at] = page_of(p.batch, p.cache.n_pages, w.seq, wb + i + lane);
        }
        ne += __builtin_popcountll(set);
      }
      // (of 16-token pages, an odd number of them ends inside a chunk)
      if (lane == 0) s_id[ne] = 0, s_page[ne] = 0, s_who[ne] = 0;
      __syncthreads();

      const int n_keys = ne << lps;
      auto load_keys = [&](int kb) {
        int page[2], slot[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = kb + 16 * i, q = __builtin_amdgcn_readfirstlane(s_page[at >> lps]);
          page[i] = q < 0 ? 0 : q, slot[i] = at & (ps - 1);
        }
        k.load_keys(page, slot);
      };
      auto load_values = [&](int kb) {
        const int at = kb + 16 * k.value_half(), page = s_page[at >> lps];
        k.load_values(page < 0 ? 0 : page, at & (ps - 1));
      };
      if (n_keys > 0) {
        load_keys(0);
        load_values(0);
      }
      for (int kb = 0; kb < n_keys; kb += 32) {
        f32x4 st[QS][2];
        k.stash_keys();
        if (kb + 32 < n_keys) load_keys(kb + 32);
        k.scores(st);
        const int at = kb + 16 * k.value_half(), e = at >> lps, slot = (at & (ps - 1)) + 8 * (k.g & 1);
        const bool gone = s_page[e] < 0;
        const uint32_t who = s_who[e];
        const int index = (s_id[e] << lps) + slot;
        Weights<T> pb[QS];
#pragma unroll
        for (int qs = 0; qs < QS; ++qs) {
          // of the lane's 8 keys, its vector sees the first `seen`
          const int seen = who & bit[qs] ? lim[qs] + 1 - index : 0;
          if (!__any(seen > 0)) {  // a block that only the other 16 vectors chose
            pb[qs] = Weights<T>{};
            continue;
          }
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              st[qs][hf][r] = 4 * hf + r < seen ? (gone ? NAN : st[qs][hf][r]) : -INFINITY;
          pb[qs] = k.weights(qs, st[qs], a.c, thr);
        }
        const int any = gone || who == 0 ? 0 : lim_max + 1 - index;
        uint32_t vals[8][NT / 2];
        const uint32_t odd = k.values(vals, careful || !__all(any >= 8), any, careful);
        k.product(vals, pb);
        if (kb + 32 < n_keys) load_values(kb + 32);
        if (careful && __any(odd != 0)) {
          for (int j = 0; j < 32; ++j) {
            if (!((__ballot((odd >> (j & 7)) & 1) >> (16 * (j >> 3))) & 0xFFFF)) continue;
            const int key = kb + j, en = key >> lps;
            bool sees[QS];
#pragma unroll
            for (int qs = 0; qs < QS; ++qs)
              sees[qs] = (s_who[en] & bit[qs]) && (s_id[en] << lps) + (key & (ps - 1)) <= lim[qs];
            k.add_unbounded(s_page[en], key & (ps - 1), sees);
          }
        }
      }
    }
    if (careful || __all(k.finite())) break;
    k.clear();
  }

#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    const int v = w.v0 + 16 * qs + k.c;
    if (v >= nv) continue;
    const int t = w.tok.x + v / G, hq = h * G + v % G;
    const float l = k.l4[qs][0];
    if (a.parts) {
      float* dst = part_o(a, part, t, hq);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < NT; i += 4)
          *(f32x4*)(dst + NT * (4 * k.g + r) + i) =
              f32x4{k.o[qs][i][r], k.o[qs][i + 1][r], k.o[qs][i + 2][r], k.o[qs][i + 3][r]};
      if (k.g == 0) *part_ml(a, part, t, hq) = float2{k.m[qs], l};
      continue;
    }
    const float inv = 1.0f / l;
    T* dst = (T*)p.out + t * p.ldo + hq * HD;
    typedef T xo __attribute__((ext_vector_type(NT), aligned(2)));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      xo y;
#pragma unroll
      for (int i = 0; i < NT; ++i) y[i] = (T)(l == 0.f ? 0.f : k.o[qs][i][r] * inv);
      *(xo*)(dst + NT * (4 * k.g + r)) = y;
    }
    if (p.lse && k.g == 0) p.lse[(size_t)t * a.n.nq + hq] = lse_of<T>(a, k.m[qs], l);
  }
}

// ---------------------------------------------------------------- tiles
constexpr int kTileWaves = 4;
constexpr int KB = kTileKeys;

// 16-byte chunk c of LDS row `key` lies at chunk c ^ kswz: score fragments (score_key's rows, one
// chunk column) then meet every bank
template <int HD>
LMOP_DEVICE int kswz(int key) {
  const int s = ((key >> 1) & 12) | (key & 3);  // = m of score_key within a tile
  return HD == 128 ? s : (s & 7);
}
// values: 32-byte units, by the keys that one transposing read takes together (4 of one lane
// group, and the next group's)
template <int HD>
LMOP_DEVICE int vswz(int key) {
  return HD == 128 ? (key & 3) | (key >> 1 & 4) : (key >> 1 & 1) | (key >> 2 & 2);
}

// 4 keys of a dimension: within 16 lanes, lane 4 j + i gives the address of 4 dimensions (i) of key
// j, and lane n gets dimension n of keys 0..3
template <typename T>
LMOP_DEVICE typename Half<T>::x4 read_transposed(const char* lds) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const s16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)lds);
  return __builtin_bit_cast(typename Half<T>::x4, r);
}

// A block's four groups of 16 keys, which lie in one page each
struct Groups {
  int page[4];   // 0 for a page that does not exist, or keys past the end
  int slot;      // of the block's first key; group i's is (slot + 16 i) % page_size
  uint32_t bad;  // groups whose page does not exist
};

// A workgroup: 128 vectors x a kv head, 32 vectors a wave.  Blocks of 64
// keys come into one of two LDS stages while the block before them is worked on:
// 16-bit pages by direct loads (a row's chunks permuted on the way), 8-bit ones through
// registers, where they become 16 bits.
template <typename T, bool E8, int HD>
struct TileCore {
  typedef typename Half<T>::x8 x8;
  typedef typename Half<T>::x4 x4;
  typedef typename Half<T>::x2 x2;
  static constexpr int NS = HD / 32, NT = HD / 16, QS = 2;
  static constexpr int ROW = HD * 2;                    // bytes of an LDS row
  static constexpr int STAGE = 2 * KB * ROW;            // K, then V
  static constexpr int RPL = 1024 / ROW;                // rows of a wave's direct load
  static constexpr int DMA = KB / RPL / kTileWaves;     // direct loads of a wave, of K or V
  static constexpr int LANES = HD / 16;                 // 16-byte loads of an 8-bit row
  static constexpr int ROWS = 64 * kTileWaves / LANES;  // 8-bit rows of a pass
  static constexpr int LOADS = E8 ? KB / ROWS : 1;
  static_assert(E8 || DMA == 4 || DMA == 2, "which group a direct load belongs to");

  const lmop_cache& cache;
  const Heads& n;
  char* smem;
  int tid, lane, wave, g, c, h, ps;
  uint32_t lds0, koff[DMA], voff;
  uint4 kr[LOADS], vr[LOADS];
  uint32_t kx[LOADS], vx[LOADS];
  x8 qf[QS][NS];
  f32x4 o[QS][NT], l4[QS];
  float m[QS];

  LMOP_DEVICE TileCore(const Args& a, char* smem_, int h_) : cache(a.t.cache), n(a.n), smem(smem_), h(h_) {
    tid = threadIdx.x, lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    g = lane >> 4, c = lane & 15;
    ps = cache.page_size;
    lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem + (uint32_t)wave * 1024u;
    // this lane's share of a direct load: row `lrow` of a group, its chunk permuted
    const int lrow = ((wave * RPL) & 15) + lane / (HD / 8), ch = lane % (HD / 8);
#pragma unroll
    for (int i = 0; i < DMA; ++i) {
      const int r = (wave + kTileWaves * i) * RPL + lane / (HD / 8);
      koff[i] = (uint32_t)((h * ps + lrow) * HD + (ch ^ kswz<HD>(r)) * 8) * 2u;
    }
    voff = (uint32_t)((h * ps + lrow) * HD + ((((ch >> 1) ^ vswz<HD>(lrow)) << 1) | (ch & 1)) * 8) * 2u;
    clear();
  }

  LMOP_DEVICE void clear() {
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      m[qs] = -INFINITY;
      l4[qs] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NT; ++i) o[qs][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // q: the vector's first element, NULL past the end
  LMOP_DEVICE void load_query(int qs, const T* q) {
    typedef T xu __attribute__((ext_vector_type(8), aligned(2)));
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const xu x = q ? *(const xu*)(q + 32 * s + 8 * g) : xu{};
#pragma unroll
      for (int i = 0; i < 8; ++i) qf[qs][s][i] = x[i];
    }
  }

  // A block on its way: 16-bit pages to the stage, 8-bit ones to registers (store() follows)
  LMOP_DEVICE void load(const Groups& b, int st) {
    if constexpr (!E8) {
      // (scalar instructions: those of four pages' addresses a block are worth a branch)
      const int64_t whole = (b.page[0] * cache.page_stride + b.slot * HD) * 2;
#pragma unroll
      for (int i = 0; i < DMA; ++i) {
        const int grp = DMA == 4 ? i : 2 * i + (wave >> 1);
        int64_t at = whole + grp * (16 * HD * 2);
        if (ps < KB) {
          const int page = DMA == 4 ? b.page[i] : (wave >> 1) ? b.page[2 * i + 1] : b.page[2 * i];
          at = (page * cache.page_stride + ((b.slot + 16 * grp) & (ps - 1)) * HD) * 2;
        }
        const uint32_t dst = lds0 + (uint32_t)(st * STAGE + kTileWaves * 1024 * i);
        g2l16_m0((const char*)cache.k + at, koff[i], dst);
        g2l16_m0((const char*)cache.v + at, voff, dst + KB * ROW);
      }
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int r = tid / LANES + i * ROWS;
        const int grp = __builtin_amdgcn_readfirstlane(r >> 4);
        const int page = grp == 0 ? b.page[0] : grp == 1 ? b.page[1] : grp == 2 ? b.page[2] : b.page[3];
        const size_t row = (size_t)h * ps + ((b.slot + r) & (ps - 1));
        const size_t at = page * cache.page_stride + row * HD + tid % LANES * 16;
        kr[i] = *(const uint4*)((const char*)cache.k + at);
        vr[i] = *(const uint4*)((const char*)cache.v + at);
        kx[i] = cache.k_exp[(size_t)page * n.nkv * ps + row];
        vx[i] = cache.v_exp[(size_t)page * n.nkv * ps + row];
      }
    }
  }
  // 16-byte chunk ch of a value row
  static LMOP_DEVICE int vchunk(int r, int ch) { return r * ROW + (((ch >> 1) ^ vswz<HD>(r)) * 32) + (ch & 1) * 16; }
  LMOP_DEVICE void store(int st) {
    char* sk = smem + st * STAGE;
    char* sv = sk + KB * ROW;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = tid / LANES + i * ROWS, ch = tid % LANES * 2;
      const float ks = exp_scale(kx[i]), vs = exp_scale(vx[i]);
      *(x8*)(sk + r * ROW + ((ch ^ kswz<HD>(r)) * 16)) = decode8<T>(kr[i].x, kr[i].y, ks);
      *(x8*)(sk + r * ROW + (((ch + 1) ^ kswz<HD>(r)) * 16)) = decode8<T>(kr[i].z, kr[i].w, ks);
      *(x8*)(sv + vchunk(r, ch)) = decode8<T>(vr[i].x, vr[i].y, vs);
      *(x8*)(sv + vchunk(r, ch + 1)) = decode8<T>(vr[i].z, vr[i].w, vs);
    }
  }

  // Value rows that no vector sees (gone(row)) become zeros: they may hold anything.  With `bounded`
  // infinities and NaN in the others do too, and their rows are marked in odd[2].
  template <typename F>
  LMOP_DEVICE void mend(int st, F&& gone, bool bounded, uint32_t* odd) {
    char* sv = smem + st * STAGE + KB * ROW;
#pragma unroll
    for (int i = 0; i < KB * HD / 8 / (64 * kTileWaves); ++i) {
      const int at = tid + i * 64 * kTileWaves, r = at / (HD / 8);
      uint4* x = (uint4*)(sv + vchunk(r, at % (HD / 8)));
      if (gone(r)) {
        *x = uint4{0, 0, 0, 0};
      } else if (bounded) {
        uint4 y = *x;
        bool any = false;
        uint32_t* ys = (uint32_t*)&y;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t out = unbounded<T>(ys[q]);
          ys[q] &= ~out;
          any = any || out != 0;
        }
        if (any) {
          *x = y;
          atomicOr(&odd[r >> 5], 1u << (r & 31));
        }
      }
    }
  }

  // st[qs][kt]: register r of lane group g is the score of key 32 (kt / 2) + 8 g + 4 (kt % 2) + r
  LMOP_DEVICE void scores(int stage, f32x4 (&st)[QS][4]) {
    const char* sk = smem + stage * STAGE;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      const int key = 32 * (kt >> 1) + score_key(kt & 1, c);
      x8 kf[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) kf[s] = *(const x8*)(sk + key * ROW + (((4 * s + g) ^ kswz<HD>(key)) * 16));
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) {
        st[qs][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) st[qs][kt] = Half<T>::mfma(kf[s], qf[qs][s], st[qs][kt]);
      }
    }
  }

  // The vectors' weights of the block and their sums; the states move to a new reference where needed
  LMOP_DEVICE void weights(int qs, f32x4 (&st)[4], float cs, float thr, Weights<T> (&pb)[2]) {
    const x8 ones = {(T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f, (T)1.f};
    float mb = max3(st[0][0], st[0][1], st[0][2]);
    mb = max3(mb, st[0][3], st[1][0]);
    mb = max3(mb, st[1][1], st[1][2]);
    mb = max3(mb, st[1][3], st[2][0]);
    mb = max3(mb, st[2][1], st[2][2]);
    mb = max3(mb, st[2][3], st[3][0]);
    mb = max3(mb, st[3][1], st[3][2]);
    mb = max4(max2(mb, st[3][3]));
    if (__any(mb > m[qs] + thr)) {
      const float m_new = mb > m[qs] + thr ? mb : m[qs];
      const float alpha = rescale(m[qs], m_new, cs);
      l4[qs] *= alpha;
#pragma unroll
      for (int i = 0; i < NT; ++i) o[qs][i] *= alpha;
      m[qs] = m_new;
    }
    const float nmc = from_reference(st, m[qs], cs, Weights<T>::kLift);
    auto weight = [&](float z) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z, cs, nmc)); };
#pragma unroll
    for (int kc = 0; kc < 2; ++kc) {
      const f32x4 &x = st[2 * kc], &y = st[2 * kc + 1];
      pb[kc].template set<0>(weight(x[0]), weight(x[1]));
      pb[kc].template set<2>(weight(x[2]), weight(x[3]));
      pb[kc].template set<4>(weight(y[0]), weight(y[1]));
      pb[kc].template set<6>(weight(y[2]), weight(y[3]));
    }
#pragma unroll
    for (int kc = 0; kc < 2; ++kc) {
      l4[qs] = Half<T>::mfma(ones, pb[kc].hi, l4[qs]);
      l4[qs] = Half<T>::mfma(ones, pb[kc].lo, l4[qs]);
    }
  }

  // O^T += V^T P^T.  Tile i: dimensions 16 i .. +15; lane (g, c) gets dimension 16 i + c of keys
  // 32 kc + 8 g .. +7
  LMOP_DEVICE void product(int stage, const Weights<T> (&pb)[QS][2]) {
    const char* sv = smem + stage * STAGE + KB * ROW;
#pragma unroll
    for (int kc = 0; kc < 2; ++kc)
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int key = 32 * kc + 8 * g + (c >> 2);
        const x4 lo = read_transposed<T>(sv + key * ROW + ((i ^ vswz<HD>(key)) * 32) + (c & 3) * 8);
        const x4 hi = read_transposed<T>(sv + (key + 4) * ROW + ((i ^ vswz<HD>(key + 4)) * 32) + (c & 3) * 8);
        const x8 x = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
        for (int qs = 0; qs < QS; ++qs) o[qs][i] = Half<T>::mfma(x, pb[qs][kc].hi, o[qs][i]);
#pragma unroll
        for (int qs = 0; qs < QS; ++qs) o[qs][i] = Half<T>::mfma(x, pb[qs][kc].lo, o[qs][i]);
      }
  }

  LMOP_DEVICE bool finite() const {
    float sum = 0.f;  // of zeros, and NaN where one is infinite or NaN
#pragma unroll
    for (int qs = 0; qs < QS; ++qs)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum = __builtin_fmaf(o[qs][i][r], 0.f, sum);
    return sum == 0.f;
  }

  // The infinities and NaN of a value row that were left out, for the vectors that see it
  LMOP_DEVICE void add_unbounded(int page, int slot, const bool* sees) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const f32x4 x = value4<T, E8>(cache, n, page, h, slot, 16 * i + 4 * g);
#pragma unroll
      for (int qs = 0; qs < QS; ++qs)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (sees[qs] && !(fabsf(x[r]) < INFINITY)) o[qs][i][r] += x[r];
    }
  }

  // The wave's results: vector qs of lane column c is (token t, head hq)
  LMOP_DEVICE void write(const Args& a, int qs, int t, int hq, int part) {
    const float l = l4[qs][0];
    if (a.parts) {
      float* dst = part_o(a, part, t, hq);
#pragma unroll
      for (int i = 0; i < NT; ++i) *(f32x4*)(dst + 16 * i + 4 * g) = o[qs][i];
      if (g == 0) *part_ml(a, part, t, hq) = float2{m[qs], l};
      return;
    }
    const float inv = 1.0f / l;
    T* dst = (T*)a.t.out + t * a.t.ldo + hq * HD;
    typedef T xo __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      xo y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = (T)(l == 0.f ? 0.f : o[qs][i][r] * inv);
      *(xo*)(dst + 16 * i + 4 * g) = y;
    }
    if (a.t.lse && g == 0) a.t.lse[(size_t)t * a.n.nq + hq] = lse_of<T>(a, m[qs], l);
  }
};

// What a tile's vectors see of their sequence
struct Span {
  int n_tok, nv, t_first, t_last;
  LMOP_DEVICE Span(const Tile& w, int G) {
    n_tok = w.tok.y - w.tok.x, nv = n_tok * G;
    t_first = w.v0 / G;
    t_last = (w.v0 + kTileVectors - 1) / G < n_tok ? (w.v0 + kTileVectors - 1) / G : n_tok - 1;
  }
};

template <typename T>
LMOP_DEVICE void write_bad_tile(const Args& a, const Tile& w, int nv, int h, int part) {
  // its tiles cover all of its tokens, but where per_seq was reckoned from max_tokens
  const int end = a.l.per_seq && w.v0 + kTileVectors >= a.l.per_seq * kTileVectors ? nv : w.v0 + kTileVectors;
  const int G = a.n.nq / a.n.nkv;
  for (int v = w.v0 + (threadIdx.x >> 6); v < end && v < nv; v += kTileWaves)
    write_bad<T>(a, w.tok.x + v / G, h * G + v % G, part, threadIdx.x & 63, 64);
}

// A split of the keys: the prefix's, then the sequence's own up to the tile's last token
template <typename T, bool E8, int HD>
LMOP_DEVICE void tile_vectors(const Args& a, int block, int split, char* smem) {
  typedef TileCore<T, E8, HD> Core;
  __shared__ uint32_t s_odd[2][2];  // by block parity: keys with infinities or NaN among their values

  const lmop_attend_args& p = a.t;
  const int h = block % a.n.nkv;
  const int G = a.n.nq / a.n.nkv;
  const int ps = p.cache.page_size, lps = __builtin_ctz(ps);
  const int part = a.part0 + split;
  // later tiles of a prompt see more keys: they go first
  const Tile w = find_tile(a, a.l.tiles - 1 - block / a.n.nkv, kTileVectors);
  const Span sp(w, G);
  if (w.v0 >= sp.nv) return;
  if (w.bad) return write_bad_tile<T>(a, w, sp.nv, h, part);

  const int lim_max = a.flat ? -1 : w.len - sp.n_tok + sp.t_last, lim_min = a.flat ? -1 : w.len - sp.n_tok + sp.t_first;
  const int n_pre = a.flat || a.fused ? p.prefix_length : 0;
  const int n_own = lim_max + 1 > 0 ? lim_max + 1 : 0;
  const int nb_pre = (n_pre + KB - 1) / KB;
  const int nb = nb_pre + (n_own + KB - 1) / KB;
  const int64_t b_from = (int64_t)split * a.l.chunk;
  const int b0 = b_from < nb ? (int)b_from : nb;
  const int b1 = nb - b0 < a.l.chunk ? nb : b0 + a.l.chunk;

  // Pages are looked up a block before they are loaded: lane i fetches group i's, and the wave takes them when
  // the block before has come, for which it waits anyway (a wait at the look-up would be one for the
  // loads before it, too).
  const int32_t* own_table = p.batch.table + (int64_t)w.seq * p.batch.ld_table;
  auto fetch = [&](int b) {
    const bool pre = b < nb_pre;
    const int key = (pre ? b : b - nb_pre) * KB + 16 * (threadIdx.x & 3);
    return b < b1 && key < (pre ? n_pre : n_own) ? (pre ? p.prefix : own_table)[key >> lps] : 0;
  };
  auto resolve = [&](int b, int fetched) {
    Groups r;
    r.bad = 0;
    r.slot = (b < nb_pre ? b : b - nb_pre) * KB & (ps - 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.page[i] = __builtin_amdgcn_readlane(fetched, i);
      if (r.page[i] < 0 || r.page[i] >= p.cache.n_pages) r.page[i] = 0, r.bad |= 1u << i;
    }
    return r;
  };

  Core k(a, smem, h);
  int lim[Core::QS];
#pragma unroll
  for (int qs = 0; qs < Core::QS; ++qs) {
    const int v = w.v0 + k.wave * 16 * Core::QS + 16 * qs + k.c;
    const int tok = v < sp.nv ? v / G : sp.t_last;
    lim[qs] = a.flat ? -1 : w.len - sp.n_tok + tok;
    k.load_query(qs, v < sp.nv ? (const T*)p.q + (int64_t)(w.tok.x + tok) * p.ldq + (h * G + v - tok * G) * HD : nullptr);
  }
  // a wave whose vectors all lie past the end only helps to load
  const bool active = w.v0 + k.wave * 16 * Core::QS < sp.nv;
  const float thr = 8.0f / a.c;

  if (k.tid < 4) s_odd[k.tid >> 1][k.tid & 1] = 0;
  uint32_t bad = 0;
  int fetched = 0;
  if (b0 < b1) {
    const Groups first = resolve(b0, fetch(b0));
    k.load(first, b0 & 1);
    bad = first.bad;
    fetched = fetch(b0 + 1);
    if constexpr (E8) k.store(b0 & 1);
  }
  for (int b = b0; b < b1; ++b) {
    // the block is in LDS for every wave, and every wave is done with the one before it, whose
    // stage the next one takes
    if constexpr (!E8) wait_vmcnt<0>();
    __syncthreads();
    uint32_t next_bad = 0;
    if (b + 1 < b1) {
      const Groups next = resolve(b + 1, fetched);
      next_bad = next.bad;
      k.load(next, (b + 1) & 1);
      fetched = fetch(b + 2);
    }
    const bool pre = b < nb_pre;
    const int kb = (pre ? b : b - nb_pre) * KB, n = pre ? n_pre : n_own;
    const bool mixed = !pre && kb + KB - 1 > lim_min;  // not every vector sees every key
    uint64_t odd = 0;
    if (mixed || kb + KB > n) {
      if (k.tid < 2) s_odd[(b + 1) & 1][k.tid] = 0;
      k.mend(b & 1, [&](int r) { return kb + r >= n; }, mixed, s_odd[b & 1]);
      __syncthreads();
      odd = s_odd[b & 1][0] | (uint64_t)s_odd[b & 1][1] << 32;
    }
    if (active) {
      f32x4 st[Core::QS][4];
      k.scores(b & 1, st);
      if (mixed || kb + KB > n || bad != 0) {
#pragma unroll
        for (int qs = 0; qs < Core::QS; ++qs) {
          // key kb + 32 (kt / 2) + 8 g + 4 (kt % 2) + r is seen if below `end`
          const int end = pre ? n : n < lim[qs] + 1 ? n : lim[qs] + 1;
          const int dl = end - kb - 8 * k.g;
#pragma unroll
          for (int kt = 0; kt < 4; ++kt) {
            const bool gone = (bad >> (2 * (kt >> 1) + (k.g >> 1))) & 1;
#pragma unroll
            for (int r = 0; r < 4; ++r)
              st[qs][kt][r] = 32 * (kt >> 1) + 4 * (kt & 1) + r < dl ? (gone ? NAN : st[qs][kt][r]) : -INFINITY;
          }
        }
      }
      Weights<T> pb[Core::QS][2];
#pragma unroll
      for (int qs = 0; qs < Core::QS; ++qs) k.weights(qs, st[qs], a.c, thr, pb[qs]);
      k.product(b & 1, pb);
      while (odd) {
        const int key = kb + __builtin_ctzll(odd);
        odd &= odd - 1;
        const int page = own_table[key >> lps];
        const bool sees[2] = {key <= lim[0], key <= lim[1]};
        if (page >= 0 && page < p.cache.n_pages) k.add_unbounded(page, key & (ps - 1), sees);
      }
    }
    bad = next_bad;
    if constexpr (E8) {
      if (b + 1 < b1) k.store((b + 1) & 1);
    }
  }

  if (!active) return;
  if (__any(!k.finite())) {  // seldom
#pragma unroll
    for (int qs = 0; qs < Core::QS; ++qs)
#pragma unroll
      for (int i = 0; i < Core::NT; ++i)
        k.o[qs][i] = settled(k.o[qs][i], k.l4[qs][0], [&](auto&& f) {
          for (int b = b0; b < b1; ++b) {
            const bool pre = b < nb_pre;
            const int kb = (pre ? b : b - nb_pre) * KB, n = pre ? n_pre : n_own;
#pragma unroll 4
            for (int key = kb; key < kb + KB && key < n; ++key) {
              const int page = (pre ? p.prefix : own_table)[key >> lps];
              if (page >= 0 && page < p.cache.n_pages && (pre || key <= lim[qs]))
                f(value4<T, E8>(p.cache, a.n, page, h, key & (ps - 1), 16 * i + 4 * k.g));
            }
          }
        });
  }
#pragma unroll
  for (int qs = 0; qs < Core::QS; ++qs) {
    const int v = w.v0 + k.wave * 16 * Core::QS + 16 * qs + k.c;
    if (v < sp.nv) k.write(a, qs, w.tok.x + v / G, h * G + v % G, part);
  }
}

// ---------------------------------------------------------------- joining the parts
// out = sum_i f_i o_i / sum_i f_i l_i with f_i = 2^(c (m_i - max m)), in a fixed order.  A group of hd / 4 lanes
// takes a (token, head), or, of at most 4096 of them, a workgroup, whose groups share the parts: each part
// costs a group two dependent loads.  us, groups against workgroups: 32 of 62 parts 63 / 31, 128 of 7 21.2 / 18.8, 2048 of
// a prefix of 4096 keys 30.9 / 24.5, but 8192 54.0 / 58.7 and 32,000 95.6 / 113.9.
struct Sum {
  f32x4 o;
  float m, l;
};
LMOP_DEVICE void add_part(Sum& s, float m, float l, const f32x4& o, float c) {
  if (l != l) {
    s.l = l;
    return;
  }
  if (l == 0.f) return;  // it saw nothing, and may not have written its outputs
  const float m_new = m > s.m ? m : s.m, f = rescale(m, m_new, c), g = rescale(s.m, m_new, c);
#pragma unroll
  for (int r = 0; r < 4; ++r) s.o[r] = s.o[r] * g + o[r] * f;
  s.l = s.l * g + l * f;
  s.m = m_new;
}

template <typename T, int HD, bool WIDE>
__global__ __launch_bounds__(256) void combine_kernel(const Args a) {
  constexpr int LANES = HD / 4, GROUPS = 256 / LANES;
  const lmop_attend_args& p = a.t;
  const int group = threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
  const int64_t i = WIDE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * GROUPS + group;
  if (i >= (int64_t)p.batch.n_tokens * a.n.nq) return;
  const int t = (int)(i / a.n.nq), h = (int)(i % a.n.nq);
  if (p.batch.start && (t < p.batch.start[0] || t >= p.batch.start[p.batch.n_seqs])) return;
  Sum s{f32x4{0.f, 0.f, 0.f, 0.f}, -INFINITY, 0.f};
  for (int q = WIDE ? group : 0; q < a.parts; q += WIDE ? GROUPS : 1) {
    const float2 ml = *part_ml(a, q, t, h);
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    if (ml.y > 0.f) o = *(const f32x4*)(part_o(a, q, t, h) + d);
    add_part(s, ml.x, ml.y, o, a.c);
  }
  if constexpr (WIDE) {
    __shared__ f32x4 s_o[GROUPS][LANES];
    __shared__ float s_m[GROUPS], s_l[GROUPS];
    s_o[group][threadIdx.x % LANES] = s.o;
    if (d == 0) s_m[group] = s.m, s_l[group] = s.l;
    __syncthreads();
    if (group > 0) return;
    for (int q = 1; q < GROUPS; ++q) add_part(s, s_m[q], s_l[q], s_o[q][threadIdx.x % LANES], a.c);
  }
  const float inv = 1.0f / s.l;
  typedef T xo __attribute__((ext_vector_type(4), aligned(2)));
  xo r;
#pragma unroll
  for (int k = 0; k < 4; ++k) r[k] = (T)(s.l == 0.f ? 0.f : s.o[k] * inv);
  *(xo*)((T*)p.out + t * p.ldo + h * HD + d) = r;
  if (p.lse && d == 0) p.lse[(size_t)t * a.n.nq + h] = lse_of<T>(a, s.m, s.l);
}

// ---------------------------------------------------------------- kernels
// (with 8-bit pages three waves fit a SIMD, which reads faster: 32 contexts of up to 32,000 tokens 227 us,
// of two 268)
template <typename T, bool E8, int HD, bool BLOCKS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, E8 && WAVES == 4 ? 3 : 2) void few_kernel(const Args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  few_vectors<T, E8, HD, BLOCKS, WAVES>(a, blockIdx.x, blockIdx.y, *(FewLds<T, E8, HD, WAVES>*)smem);
}

template <typename T, bool E8, int HD>
__global__ __launch_bounds__(64 * kTileWaves, 2) void tile_kernel(const Args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  tile_vectors<T, E8, HD>(a, blockIdx.x, blockIdx.y, smem);
}

// Both launches of a batch behind a prefix at once: the prefix's workgroups, which take longer, first.  With
// SINGLE the own part's waves have sequences of their own.
template <typename T, bool E8, int HD, bool FEW, bool SINGLE>
__global__ __launch_bounds__(64 * kTileWaves, 2) void pair_kernel(const Args prefix, const Args own) {
  static_assert(kTileWaves == kFewWaves, "one size of workgroup");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int each = prefix.l.tiles * prefix.n.nkv, first = each * prefix.l.splits;
  const int block = blockIdx.x;
  if (block < first) {
    if constexpr (FEW)
      few_vectors<T, E8, HD, false, kFewWaves>(prefix, block % each, block / each,
                                               *(FewLds<T, E8, HD, kFewWaves>*)smem);
    else
      tile_vectors<T, E8, HD>(prefix, block % each, block / each, smem);
  } else {
    const int per = own.l.tiles * own.n.nkv;
    if constexpr (SINGLE) {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      const int b = (block - first) * kFewWaves + wave;
      if (b < per * own.l.splits)
        few_vectors<T, E8, HD, false, 1>(own, b % per, b / per, ((FewLds<T, E8, HD, 1>*)smem)[wave]);
    } else {
      few_vectors<T, E8, HD, false, kFewWaves>(own, (block - first) % per, (block - first) / per,
                                               *(FewLds<T, E8, HD, kFewWaves>*)smem);
    }
  }
}

template <typename K>
hipError_t allow_lds(K kernel, int lds) {
  if (lds <= 32768) return hipSuccess;  // else more than HIP allows unasked, with what a kernel has of its own
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

template <typename T, bool E8, int HD>
hipError_t launch(hipStream_t s, const lmop_attend_args& t, const Heads& n, const AttendPlan& plan) {
  constexpr int tile_lds = 2 * TileCore<T, E8, HD>::STAGE;
  constexpr auto few_lds = [](int waves) {
    return (int)(waves == 1   ? sizeof(FewLds<T, E8, HD, 1>)
                 : waves == 4 ? sizeof(FewLds<T, E8, HD, 4>)
                              : sizeof(FewLds<T, E8, HD, 8>));
  };
  Args a{};
  a.t = t;
  a.n = n;
  a.c = (t.scale == 0.f ? 1.0f / sqrtf((float)HD) : t.scale) * 1.4426950408889634f;
  a.parts = plan.parts;
  a.l = plan.own;
  a.fused = plan.prefix.tiles == 0 && t.prefix_length > 0;
  const dim3 grid(n.nkv * a.l.tiles, a.l.splits);
  auto queue = [&](auto kernel, int threads, int lds) {
    const hipError_t e = allow_lds(kernel, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, s, a);
    return hipGetLastError();
  };
  hipError_t e;
  if (plan.prefix.tiles > 0) {
    Args q = a;
    q.l = plan.prefix;
    q.flat = 1;
    q.part0 = plan.own.splits;
    const bool single = a.l.waves == 1;
    const auto kernel = q.l.few ? (single ? pair_kernel<T, E8, HD, true, true> : pair_kernel<T, E8, HD, true, false>)
                                : (single ? pair_kernel<T, E8, HD, false, true> : pair_kernel<T, E8, HD, false, false>);
    int lds = single ? kFewWaves * few_lds(1) : few_lds(kFewWaves);
    const int other = q.l.few ? few_lds(kFewWaves) : tile_lds;
    lds = lds > other ? lds : other;
    e = allow_lds(kernel, lds);
    if (e != hipSuccess) return e;
    const unsigned own = (unsigned)n.nkv * a.l.tiles * a.l.splits;
    const unsigned blocks = (unsigned)n.nkv * q.l.tiles * q.l.splits + (single ? (own + kFewWaves - 1) / kFewWaves : own);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * kTileWaves), lds, s, q, a);
    e = hipGetLastError();
  } else if (t.blocks && !a.l.few) {
    e = queue(walk_kernel<T, E8, HD>, 64, 0);
  } else if (!a.l.few) {
    e = queue(tile_kernel<T, E8, HD>, 64 * kTileWaves, tile_lds);
  } else if (a.l.waves == 1) {
    e = t.blocks ? queue(few_kernel<T, E8, HD, true, 1>, 64, few_lds(1))
                 : queue(few_kernel<T, E8, HD, false, 1>, 64, few_lds(1));
  } else if (a.l.waves == 4) {
    e = t.blocks ? queue(few_kernel<T, E8, HD, true, 4>, 256, few_lds(4))
                 : queue(few_kernel<T, E8, HD, false, 4>, 256, few_lds(4));
  } else {
    e = t.blocks ? queue(few_kernel<T, E8, HD, true, 8>, 512, few_lds(8))
                 : queue(few_kernel<T, E8, HD, false, 8>, 512, few_lds(8));
  }
  if (e != hipSuccess || plan.parts == 0) return e;
  const int64_t groups = (int64_t)t.batch.n_tokens * n.nq, per = 256 / (HD / 4);
  if (groups <= 4096)
    hipLaunchKernelGGL((combine_kernel<T, HD, true>), dim3((unsigned)groups), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((combine_kernel<T, HD, false>), dim3((unsigned)((groups + per - 1) / per)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(hipStream_t s, const lmop_attend_args& t, const Heads& n, const AttendPlan& plan) {
  const bool e8 = t.cache.dtype == LMOP_E4M3;
  if (n.hd == 128) return e8 ? launch<T, true, 128>(s, t, n, plan) : launch<T, false, 128>(s, t, n, plan);
  if (n.hd == 64) return e8 ? launch<T, true, 64>(s, t, n, plan) : launch<T, false, 64>(s, t, n, plan);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_attend(hipStream_t s, const lmop_attend_args& a, const Heads& n, const AttendPlan& plan) {
  return a.dtype == LMOP_F16 ? launch_t<f16>(s, a, n, plan) : launch_t<bf16>(s, a, n, plan);
}

}  // namespace lmop
