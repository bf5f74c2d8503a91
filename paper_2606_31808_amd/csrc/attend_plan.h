// How an attention call over a paged cache is divided among workgroups: plain
// C++, from the sizes in the call's arguments alone.
#pragma once
#include <stdint.h>

namespace lmop {

constexpr int kFewVectors = 16;    // query vectors (token, head of the group) of a few-vector workgroup
constexpr int kTileVectors = 128;  // of a tile workgroup
constexpr int kTileKeys = 64;      // keys of a tile workgroup's step
constexpr int kWalkVectors = 32;   // of a wave that walks the blocks its tokens chose
constexpr int kWalkWindow = 128;   // blocks that it gathers at a time
constexpr int kMaxEntries = 512;   // pages a few-vector workgroup walks at most

struct AttendSizes {
  int n_seqs, n_tokens, max_tokens, max_length, prefix_length;
  int n_blocks;  // 0: all of a sequence's keys
  int page_size, nq, nkv, hd;
  bool starts;   // ragged: sequences of other than one token
};

// One launch: `tiles` x kv heads x `splits` workgroups; split z walks `chunk`
// steps (few-vector kernel: pages; tile kernel: kTileKeys keys) from z * chunk on.
struct AttendLaunch {
  bool few = false;
  int waves = 4;      // few-vector kernel: 1, 4 or 8 of a workgroup
  int tiles = 0, splits = 1, chunk = 1;
  int per_seq = 0;  // tiles of a sequence, or 0: as many as it needs, found from the starts
};

struct AttendPlan {
  AttendLaunch own;     // each sequence's tokens over its keys (and the prefix, if not separate)
  AttendLaunch prefix;  // all tokens over the prefix; tiles = 0: own walks it
  int parts = 0;        // partial results for every token and head; 0: the own launch writes the output
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Divides `steps` among at most `want` splits of at least `least` steps and at most `most`; up to `whole`
// steps stay together if `most` allows it.
inline void split_steps(AttendLaunch& l, int64_t steps, int64_t want, int64_t least, int64_t most, int64_t whole = 0) {
  if (steps < 1) steps = 1;
  int64_t n = steps <= whole ? 1 : steps / least;
  if (n > want) n = want;
  if (n < 1) n = 1;
  int64_t chunk = ceil_div(steps, n);
  if (chunk > most) chunk = most;
  l.chunk = (int)chunk;
  l.splits = (int)ceil_div(steps, chunk);
}

// workgroups that fill the chip
constexpr int kFewFill = 1024, kTileFill = 512, kWalkFill = 2048;

// Waves of a few-vector workgroup.  Where there are workgroups for less than half the CUs, eight: more of
// their keys are on their way at once (573 keys of one row 8.8 -> 7.9 us).  Where there are two waves for
// every SIMD without a second one in a workgroup, and few keys each, one: nothing is joined (256 rows
// of up to 112 keys 22 -> 9 us).  The other part of a launch has four.
inline void pick_waves(AttendLaunch& l, const AttendSizes& s, bool pair) {
  const int64_t workgroups = (int64_t)l.tiles * s.nkv * l.splits, keys = (int64_t)l.chunk * s.page_size;
  l.waves = workgroups >= 2048 && keys <= 512 ? 1 : workgroups <= 128 && !pair ? 8 : 4;
}

// chosen blocks: vectors of a sequence from which waves walk the blocks of several tokens
constexpr int kWalkLeast = 64;

inline AttendPlan plan_attend(const AttendSizes& s) {
  AttendPlan p;
  const int group = s.nq / s.nkv;
  const int64_t vectors = (int64_t)s.max_tokens * group;
  const int64_t pages = ceil_div(s.max_length, s.page_size);
  const int64_t prefix_pages = ceil_div(s.prefix_length, s.page_size);
  // Joining parts takes a second launch and some 4 us, in which a few-vector workgroup walks 512 keys (1024
  // keys for each of 256 workgroups: 42 us whole, 50 in two parts, with the choice of blocks before it)
  const int64_t few_least = ceil_div(512, s.page_size), few_whole = ceil_div(1024, s.page_size);
  // tiles of `of` vectors: as many as the sequences need, found from the starts, or max_tokens' for each
  auto tiles = [&](AttendLaunch& l, int of) {
    const int64_t each = ceil_div(vectors, of);
    const int64_t ragged = (int64_t)s.n_tokens * group / of + s.n_seqs;
    l.per_seq = s.n_seqs * each <= ragged ? (int)each : 0;
    l.tiles = (int)(l.per_seq ? s.n_seqs * each : ragged);
  };
  if (s.n_blocks > 0 && s.starts && (int64_t)s.n_tokens * group >= (int64_t)kWalkLeast * s.n_seqs) {
    tiles(p.own, kWalkVectors);
    split_steps(p.own, ceil_div(pages, kWalkWindow), kWalkFill / ((int64_t)p.own.tiles * s.nkv), 1, 1 << 20);
    p.parts = p.own.splits > 1 ? p.own.splits : 0;
    return p;
  }
  if (s.n_blocks > 0) {
    p.own.few = true;
    p.own.per_seq = (int)ceil_div(group, kFewVectors);  // of a token here
    p.own.tiles = s.n_tokens * p.own.per_seq;
    split_steps(p.own, s.n_blocks, kFewFill / ((int64_t)p.own.tiles * s.nkv), few_least, kMaxEntries, few_whole);
    pick_waves(p.own, s, false);
    p.parts = p.own.splits > 1 ? p.own.splits : 0;
    return p;
  }
  p.own.few = vectors <= kFewVectors || !s.starts;
  const bool separate = s.prefix_length > 0 && p.own.few && s.n_seqs > 1;
  if (p.own.few) {
    p.own.per_seq = (int)ceil_div(vectors, kFewVectors);
    p.own.tiles = s.n_seqs * p.own.per_seq;
    split_steps(p.own, pages + (separate ? 0 : prefix_pages),
                kFewFill / ((int64_t)p.own.tiles * s.nkv), few_least, kMaxEntries, few_whole);
    pick_waves(p.own, s, separate);
  } else {
    tiles(p.own, kTileVectors);
    split_steps(p.own, ceil_div(s.max_length, kTileKeys) + ceil_div(s.prefix_length, kTileKeys),
                kTileFill / ((int64_t)p.own.tiles * s.nkv), 8, 1 << 30);
  }
  if (separate) {
    const int64_t all = (int64_t)s.n_tokens * group;
    p.prefix.few = all <= 2 * kFewVectors;
    p.prefix.tiles = (int)ceil_div(all, p.prefix.few ? kFewVectors : kTileVectors);
    if (p.prefix.few)
      split_steps(p.prefix, prefix_pages, kFewFill / ((int64_t)p.prefix.tiles * s.nkv), few_least, kMaxEntries, few_whole);
    else
      split_steps(p.prefix, ceil_div(s.prefix_length, kTileKeys), kTileFill / ((int64_t)p.prefix.tiles * s.nkv),
                  4, 1 << 30);
  }
  p.parts = p.own.splits + (separate ? p.prefix.splits : 0);
  if (p.parts == 1) p.parts = 0;
  return p;
}

// A call's partial results: for each part, token and head an fp32 output (not
// divided), and the reference score and sum that go with it.
inline uint64_t attend_workspace(const AttendPlan& p, const AttendSizes& s) {
  return (uint64_t)p.parts * s.n_tokens * s.nq * (s.hd + 2) * sizeof(float);
}

}  // namespace lmop
