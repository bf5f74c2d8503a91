// How a choice of blocks is divided among workgroups and launches: plain C++, from the sizes in the
// call's arguments alone.
#pragma once
#include <stdint.h>

namespace lmop {

constexpr int kSelectTokens = 16;    // of a sequence that share a workgroup, at most
constexpr int kSelectScores = 16384; // a workgroup holds at most (128 KB)
constexpr int kSelectTileWaves = 8;

struct SelectSizes {
  int n_seqs, n_tokens, max_length, page_size, nkv, hd;
  bool starts;
};

struct SelectPlan {
  int pages;      // scores of a token
  int tile;       // tokens of a sequence in a workgroup; 0: a workgroup a token and kv head
  int waves;      // of a workgroup
  int64_t items;  // tiles, or tokens; times kv heads: workgroups
  int64_t each;   // items of a launch: of more than 2^32 - 1 threads HIP makes none, and a call is several
};

inline SelectPlan plan_select(const SelectSizes& s) {
  SelectPlan p;
  const int64_t pages = (s.max_length + (int64_t)s.page_size - 1) / s.page_size;
  p.pages = (int)(pages < 1 ? 1 : pages);
  // Sequences of four tokens or more share their means, as long as four tokens' scores fit.  A workgroup of 16 tokens
  // takes longer than one of a single token, so only where those would be more than run at once.  us, shared against
  // single (8 kv heads of 128): 16 tokens of 469 pages 24.5 / 10.9, 64 20.3 / 18.1, 200 25.3 / 48.6; 256 of 63 or
  // 125 pages 13.6 / 14.6, 14.9 / 15.9; 32 of 469 pages in sequences of two 22.1 / 11.4.
  const int fit = kSelectScores / p.pages < kSelectTokens ? kSelectScores / p.pages : kSelectTokens;
  const bool shared = s.starts && s.n_tokens / 4 >= s.n_seqs && fit >= 4 && (int64_t)s.n_tokens * s.nkv >= 1024;
  p.tile = shared ? fit : 0;
  // a token's: enough waves for all means to be on their way at once (32 contexts of 500 pages: 11 us, with four
  // waves 16)
  p.waves = shared ? kSelectTileWaves : p.pages > 4 * 64 / (s.hd / 8) * 8 ? 16 : 4;
  p.items = shared ? (int64_t)s.n_tokens / p.tile + s.n_seqs : s.n_tokens;
  p.each = ((int64_t(1) << 32) - 1) / (64 * p.waves) / s.nkv;
  if (p.each > p.items) p.each = p.items;
  return p;
}

}  // namespace lmop
