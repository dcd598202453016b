// Records and argument blocks of causal attention with grouped heads (packed prompts), shared by the
// planner (causal_plan.cpp), the C ABI (sra_text_api.cpp) and the kernels (sra_causal_fwd.hip, sra_causal_bwd.hip).
//
// The G = heads / kv_heads query heads of one K/V head are taken together: "rows" of a sequence are its
// (token, head of the group) pairs, row = token G + g, so a tile of 256 rows spans 256 / G tokens, reads a key
// tile once for all of them and has fewer tiles on the diagonal than 256 tokens of one head would.
#pragma once
#include <stdint.h>

#include <vector>

#include "sra_config.h"

namespace sra {

// One work item of a launch.
//   kForward, kDq: rows [start, start + len) of a sequence's (token, g) rows, against the keys [lo, hi);
//     lo is a multiple of 64, and so is hi unless it ends at the last key that a row of the item sees.
//   kDkv: keys [start, start + len), against the query tiles [lo, hi) of the item's list (causal_tile).
enum CausalKind : int32_t { kForward = 0, kDq = 1, kDkv = 2 };
struct CausalItem {
  int32_t kind;
  int32_t kvh;     // K/V head
  int32_t start;
  int32_t len;     // <= 256 (forward: <= CausalTables::fwd_tile)
  int32_t q0, nq;  // packed row of the sequence's first token, tokens
  int32_t k0, nk;  // packed row of its first key, keys
  int32_t lo, hi;
  int32_t slot;    // 0: results are final; k > 0: partial results go to slot k - 1 of the kind
  int32_t seq;
};
// A split item: pieces' partial results of slots [lo, lo + hi), added up in that order by the combine kernels.

// The causal rule: token i of a sequence sees the keys j <= i + nk - nq.
//
// The query tiles of a dK/dV item: 64 tokens of one head each, from the first token t0 that sees key `start` on;
// n a head, the first d of them on the diagonal (their first token does not see all of the item's keys). The list
// holds those off the diagonal, head by head, then those on it, so that the kernel runs one loop for each kind.
struct CausalTiles {
  int32_t t0, n, d;
};
struct CausalTile {
  int32_t hg, tok;  // head of the group, first token
};
#ifndef SRA_HD
#ifdef __HIPCC__
#define SRA_HD __host__ __device__
#else
#define SRA_HD
#endif
#endif
SRA_HD inline CausalTiles causal_tiles(const CausalItem& it) {
  const int32_t off = it.nk - it.nq;
  const int32_t t0 = it.start > off ? it.start - off : 0;
  const int32_t n = it.nq > t0 ? (it.nq - t0 + 63) / 64 : 0;
  const int32_t hidden = it.start + it.len - 1 - off - t0;  // tokens from t0 on that do not see all keys
  const int32_t d = hidden > 0 ? (hidden + 63) / 64 : 0;
  return {t0, n, d < n ? d : n};
}
// Tile i of the G n of the list, which must not be empty.
SRA_HD inline CausalTile causal_tile(const CausalTiles& t, int32_t G, int32_t i) {
  const int32_t full = t.n - t.d, diagonal = i - G * full;
  if (diagonal < 0) return {i / full, t.t0 + 64 * (t.d + i % full)};
  return {diagonal / t.d, t.t0 + 64 * (diagonal % t.d)};
}

constexpr int kCausalTile = 256;  // rows or keys per item

struct CausalTables {
  int32_t batch = 0, heads = 0, kv_heads = 0, head_dim = 0;
  bool backward = false;
  std::vector<int32_t> nq, nk;
  int64_t q_rows = 0, k_rows = 0;  // packed tokens, packed keys
  std::vector<CausalItem> fwd, fwd_combine, grad, grad_combine;
  int32_t fwd_tile = kCausalTile;  // rows per forward item
  int32_t fwd_slots = 0, q_slots = 0, kv_slots = 0;
};

// Fills t's item lists from its sizes (host only).
void build_causal_tables(CausalTables* t);

}  // namespace sra
