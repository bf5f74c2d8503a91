// Device side of a paged cache: batches, pages, and the types that pages hold.
#pragma once
#include "common.h"
#include "lmop.h"

namespace lmop {

typedef f16 f16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 16-bit types: vectors, the matrix instruction (operands as mfma16x16x32's), E4M3 codes times a
// power of two (two codes of a word; exact, but for what lies past the type's range)
template <typename T>
struct Half;
template <>
struct Half<f16> {
  typedef f16x2 x2;
  typedef f16x4 x4;
  typedef f16x8 x8;
  static LMOP_DEVICE f32x4 mfma(x8 a, x8 b, f32x4 c) { return mfma16x16x32(a, b, c); }
  template <bool HI>
  static LMOP_DEVICE x2 decode(uint32_t w, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HI);
  }
};
template <>
struct Half<bf16> {
  typedef bf16x2 x2;
  typedef bf16x4 x4;
  typedef bf16x8 x8;
  static LMOP_DEVICE f32x4 mfma(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  template <bool HI>
  static LMOP_DEVICE x2 decode(uint32_t w, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI);
  }
};

// Positive weights in two terms: the nearest of the type, and the nearest of what is left.  Together off by 2^-16 of a
// bf16 weight, 2^-22 of an fp16 one of 2^-3 and more, and 2^-25 of a smaller one.  All are taken times 2^kLift, of which
// the division rids them: the largest of a softmax may pass its reference by 2^8.  fp16 ones are then 2^7 to 2^15 at the
// top, and what is lost is 2^-32 of that; bf16 ones 2^-8 to 1, so that values up to the type's end stay within fp32.
//
// In one term results were 1.25 to 1.3 times as far from the formula as their own rounding takes them, and fp16 weights
// below 2^-25 were lost however many.  The second term is a second product with the values, half as much again for the
// matrix units: a prompt of 8448 tokens 583 -> 790 us (1.1 PFLOP/s with it, what a large library product reaches), 272 rows
// behind 512 keys 280 -> 345, 256 tokens behind 8192 keys 76 -> 88, the walk over chosen blocks 285 -> 325; long single
// tokens, whose matrix units wait for memory, 1 to 2%, one over 573 keys 8.3 -> 8.8.
template <typename T>
struct Weights {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef typename Half<T>::x2 x2;
  typename Half<T>::x8 hi, lo;
  static constexpr float kLift = __is_same(T, f16) ? 7.f : -8.f;
  template <int I>
  LMOP_DEVICE void set(float x, float y) {  // weights I and I + 1
    const x2 h = __builtin_convertvector((f32x2{x, y}), x2);
    x2 l;  // what is left, exact in fp32
    if constexpr (__is_same(T, f16)) {
      // (a -1 that the compiler does not see through: a multiply-add of both types, with the rounding, is one instruction,
      // the subtraction would be three)
      float minus = -1.f;
      asm("" : "+s"(minus));
      l = x2{(T)__builtin_fmaf((float)h[0], minus, x), (T)__builtin_fmaf((float)h[1], minus, y)};
    } else {
      // (the instruction that multiplies two of the type and adds would save the unpacking: prompt 777 -> 800 us)
      l = __builtin_convertvector((f32x2{x - (float)h[0], y - (float)h[1]}), x2);
    }
    hi[I] = h[0], hi[I + 1] = h[1];
    lo[I] = l[0], lo[I + 1] = l[1];
  }
};

// 2^(e - 127) of an exponent byte 1 .. 254
LMOP_DEVICE float exp_scale(uint32_t e) { return __uint_as_float(e << 23); }

// eight codes of two words
template <typename T>
LMOP_DEVICE typename Half<T>::x8 decode8(uint32_t lo, uint32_t hi, float scale) {
  const auto a = Half<T>::template decode<false>(lo, scale), b = Half<T>::template decode<true>(lo, scale);
  const auto c = Half<T>::template decode<false>(hi, scale), d = Half<T>::template decode<true>(hi, scale);
  return typename Half<T>::x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The tokens of sequence s: [x, y)
LMOP_DEVICE int2 seq_tokens(const lmop_batch& b, int s) {
  if (!b.start) return int2{s, s + 1};
  int x = b.start[s], y = b.start[s + 1];
  x = x < 0 ? 0 : x > b.n_tokens ? b.n_tokens : x;
  y = y < x ? x : y > b.n_tokens ? b.n_tokens : y;
  return int2{x, y};
}

// The last s in [0, n) with base(s) <= i (base ascending, base(0) <= i), by a whole
// wave: 64 probes a step, so two dependent loads for up to 4096 sequences.
template <typename F>
LMOP_DEVICE int find_seq(int n, int i, F&& base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int at = lo + (lane + 1) * step;
    const bool below = at < hi && base(at) <= i;
    const int count = __builtin_popcountll(__ballot(below));
    lo += count * step;
    hi = hi < lo + step ? hi : lo + step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Between LDS accesses of a wave's lanes to the same place: the hardware does them in order, the compiler has
// to keep them so.
LMOP_DEVICE void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The page of a sequence's keys b * page_size and on, or -1
LMOP_DEVICE int page_of(const lmop_batch& b, int n_pages, int s, int block) {
  if (block < 0 || block >= b.max_pages) return -1;
  const int p = b.table[(int64_t)s * b.ld_table + block];
  return p >= 0 && p < n_pages ? p : -1;
}

}  // namespace lmop
