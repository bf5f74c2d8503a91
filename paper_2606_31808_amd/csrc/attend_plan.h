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

// Divides `steps` into n splits of equal chunks, of at most `most` steps
inline void split_steps(AttendLaunch& l, int64_t steps, int64_t n, int64_t most) {
  if (steps < 1) steps = 1;
  if (n < 1) n = 1;
  int64_t chunk = ceil_div(steps, n);
  if (chunk > most) chunk = most;
  l.chunk = (int)chunk;
  l.splits = (int)ceil_div(steps, chunk);
}
inline int64_t least_of(int64_t a, int64_t b) { return a < b ? a : b; }

// Splits of a few-vector launch of `workgroups` before it is split, over `keys` keys at most.  Joining parts takes a
// second launch and some 4 us, in which a workgroup walks 512 keys, so up to 1024 stay together (16 blocks
// of 64 for each of 256 workgroups: 25 us whole, 32 in four parts).  Two workgroups fit a CU: where the sequences
// are alike, 512 of them are the fastest (us, with 1024 of them in brackets; 32 + 8 heads of 128: 16 sequences of
// 8000 keys 98.3 (100.0), 64 of 2000 95.5 (100.5), 8-bit 4 of 32,000 47.9 (56.4) and 16 of 8000 46.7
// (54.6)).  Where they are not, only some have keys in each split, and up to 1024 of long chunks balance
// better: 32 of 1000 to 32,000, 8-bit, 228 us, of 512 workgroups 312.  Parts of at least 512 keys: one sequence of 4000
// takes 12.3 us, in parts of 2048 26.9 (of 32,000 keys 30.9 and 27.7).
inline int64_t few_splits(int64_t workgroups, int64_t keys) {
  if (keys <= 1024) return 1;
  const int64_t even = least_of(512 / workgroups, keys / 512), ragged = least_of(1024 / workgroups, keys / 4096);
  return even > ragged ? even : ragged;
}
// Splits of a tile launch of `workgroups` over `blocks` steps, with `outputs` = tokens x heads.  Up to two
// workgroups a CU (up to four: 64 tokens over 32,000 keys 70 -> 93 us; one: 256 tokens 209 -> 271).  A step takes
// some 1.2 us; each part more costs outputs / 2048 * 0.5 us, written and read once more, so that their sum is
// least at sqrt(4800 blocks / outputs) parts.  us, at that many, at twice and at half of them: 64 tokens over
// 1000 keys 19.0, 20.1, 22.9; prefixes of 8192 keys, 16 tokens 21.6, 26.0, 26.7, of 4096, 32 tokens 23.2, 22.0, 29.0, of
// 8192, 64 tokens 33.0, 37.1, 46.3, of 2048, 256 tokens 33.9, 45.6, 46.6.
inline int64_t tile_splits(int64_t workgroups, int64_t blocks, int64_t outputs) {
  int64_t n = least_of(512 / workgroups, blocks / 2);
  while (n > 1 && n * n * outputs > 4800 * blocks) --n;
  return n;
}
// Waves of a walk that fill the chip
constexpr int kWalkFill = 2048;

// Waves of a few-vector workgroup.  Where there are workgroups for less than half the CUs, eight: more of
// their keys are on their way at once (573 keys of one row 9.7 -> 8.6 us).  Where there are two waves for
// every SIMD without a second one in a workgroup, and few keys each, one: nothing is joined (256 rows of
// up to 112 keys behind a prefix of 3900: 59 -> 52 us).  Beside a prefix's workgroups never eight.
inline void pick_waves(AttendLaunch& l, const AttendSizes& s, bool pair) {
  const int64_t workgroups = (int64_t)l.tiles * s.nkv * l.splits, keys = (int64_t)l.chunk * s.page_size;
  l.waves = workgroups >= 2048 && keys <= 512 ? 1 : workgroups <= 128 && !pair ? 8 : 4;
}

// Chosen blocks: from so many waves on, and vectors of a sequence, waves walk the blocks of several tokens.
// us, walked against a workgroup a token (32 + 8 heads of 128, 16 of 500 blocks): one sequence of 256
// tokens 100 / 74, 512 (512 waves) 124 / 137, 1000 197 / 265, 2000 324 / 518; eight of 64 (512 waves) 182 / 131, of 128
// 200 / 258; heads of 64: 256 tokens 76 / 37, 1000 145 / 129.  So the best border depends on the sequences and the heads
// too: at 512 waves either side wins, and with heads of 64 the walk loses up to 1000 tokens.
constexpr int kWalkWaves = 640, kWalkLeast = 128;

// Keys of the prefix that the sequences' workgroups would read, from which it is walked on its own, for
// all sequences together: that takes another launch.  us, alone against with each (32 + 8 heads of 128):
// 512 keys and 64 sequences (262144) 16.7 / 13.4, 128 of them 22.7 / 25.0, 256 24.3 / 44.1; 1024 and 32 16.8 / 15.7, 64
// (524288) 20.1 / 18.3; 4096 and 8 (262144) 13.6 / 16.1, 16 18.6 / 21.7: a long prefix gains somewhat earlier, a short one later.
constexpr int64_t kSharedKeys = 400000;

inline AttendPlan plan_attend(const AttendSizes& s) {
  AttendPlan p;
  const int group = s.nq / s.nkv;
  const int64_t vectors = (int64_t)s.max_tokens * group;
  const int64_t pages = ceil_div(s.max_length, s.page_size);
  const int64_t prefix_pages = ceil_div(s.prefix_length, s.page_size);
  // tiles of `of` vectors: as many as the sequences need, found from the starts, or max_tokens' for each
  auto tiles = [&](AttendLaunch& l, int of) {
    const int64_t each = ceil_div(vectors, of);
    const int64_t ragged = (int64_t)s.n_tokens * group / of + s.n_seqs;
    l.per_seq = s.n_seqs * each <= ragged ? (int)each : 0;
    l.tiles = (int)(l.per_seq ? s.n_seqs * each : ragged);
  };
  if (s.n_blocks > 0 && s.starts && (int64_t)s.n_tokens * group >= (int64_t)kWalkLeast * s.n_seqs &&
      (int64_t)s.n_tokens * group / kWalkVectors * s.nkv >= kWalkWaves) {
    tiles(p.own, kWalkVectors);
    const int64_t windows = ceil_div(pages, kWalkWindow);
    split_steps(p.own, windows, least_of(kWalkFill / ((int64_t)p.own.tiles * s.nkv), windows), 1 << 20);
    p.parts = p.own.splits > 1 ? p.own.splits : 0;
    return p;
  }
  if (s.n_blocks > 0) {
    p.own.few = true;
    p.own.per_seq = (int)ceil_div(group, kFewVectors);  // of a token here
    p.own.tiles = s.n_tokens * p.own.per_seq;
    split_steps(p.own, s.n_blocks, few_splits((int64_t)p.own.tiles * s.nkv, (int64_t)s.n_blocks * s.page_size), kMaxEntries);
    pick_waves(p.own, s, false);
    p.parts = p.own.splits > 1 ? p.own.splits : 0;
    return p;
  }
  // (us, of sequences of up to 64 vectors with few-vector workgroups in brackets: 4 of 8 tokens of 4 heads over 2000 keys
  // 18.6 (15.9), but 64 of 16 tokens 111 (158), whose keys a tile reads once.  All sequences go by the longest: a call
  // that mixes prompts and single tokens gives each of these a tile, most of it empty, and walks its keys in
  // a few workgroups, and its prefix once a sequence.)
  p.own.few = vectors <= kFewVectors || !s.starts;
  const bool separate = p.own.few && (int64_t)s.n_seqs * s.nkv * s.prefix_length >= kSharedKeys;
  if (p.own.few) {
    p.own.per_seq = (int)ceil_div(vectors, kFewVectors);
    p.own.tiles = s.n_seqs * p.own.per_seq;
    const int64_t walked = pages + (separate ? 0 : prefix_pages);
    split_steps(p.own, walked, few_splits((int64_t)p.own.tiles * s.nkv, walked * s.page_size), kMaxEntries);
    pick_waves(p.own, s, separate);
  } else {
    tiles(p.own, kTileVectors);
    const int64_t blocks = ceil_div(s.max_length, kTileKeys) + ceil_div(s.prefix_length, kTileKeys);
    split_steps(p.own, blocks, tile_splits((int64_t)p.own.tiles * s.nkv, blocks, (int64_t)s.n_tokens * s.nq), 1 << 30);
  }
  if (separate) {
    const int64_t all = (int64_t)s.n_tokens * group;
    // (us, as tiles in brackets: 16 vectors over 8192 keys 16.3 (22.1), 32 of them 17.2 (20.5), but 64
    // 23.6 (22.5))
    p.prefix.few = all <= 2 * kFewVectors;
    p.prefix.tiles = (int)ceil_div(all, p.prefix.few ? kFewVectors : kTileVectors);
    const int64_t workgroups = (int64_t)p.prefix.tiles * s.nkv, blocks = ceil_div(s.prefix_length, kTileKeys);
    if (p.prefix.few)
      split_steps(p.prefix, prefix_pages, few_splits(workgroups, s.prefix_length), kMaxEntries);
    else
      split_steps(p.prefix, blocks, tile_splits(workgroups, blocks, (int64_t)s.n_tokens * s.nq), 1 << 30);
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
