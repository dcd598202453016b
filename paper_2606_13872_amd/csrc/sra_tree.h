// Argument blocks and launchers of the attention of drafted tokens over a paged cache, and of appending to it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sra {

constexpr int kTreeMaxBatch = 2048;  // sequences: their bounds sit in LDS
constexpr int kTreeChunk = 32;       // keys a wave takes at a time
constexpr int kTreeGroups = 256;     // workgroups of a launch: one per compute unit, whose LDS it takes
// What beginning a group of rows costs a workgroup, in chunks: its bounds, queries, first loads and the merge of the
// waves are a chain of latencies (about 5 us, the time of as many chunks of four waves when the cache bounds them).
constexpr int kTreeStart = 8;
constexpr int kTreeMinRun = kTreeStart + 8;  // a workgroup takes at least so much: two chunks per wave
// The same of the shared kernel, where a 64-key chunk costs 3 with up to 128 rows (1.9 us) and 4 with
// more (2.5 us in long launches). Trees of up to 48 tokens over 16 contexts take 70 us for 67 with a start of 16 or 33; 16
// requests of 1,000 positions and 10 tokens 29 us for 26 with a least run of 48.
constexpr int kSharedStart = 24, kSharedMinRun = 36, kSharedNarrow = 3, kSharedWide = 4;
// Launches whose runs of wide groups (256 rows) would cost less than this are dealt as narrow ones (128): more groups, so
// fewer are split, for reading the keys of sequences with more rows again. 16 requests of 64 tokens x 4 heads: over 1,000
// positions 39 us for 54, over 8,000 184 for 167; trees of up to 48 tokens over 16 contexts, near the limit, 81 for 84.
constexpr int kSharedShortRun = 70;
constexpr int kTreeMaxGroup = 1024;          // query heads of a K/V head

#ifndef SRA_HD
#ifdef __HIPCC__
#define SRA_HD __host__ __device__
#else
#define SRA_HD
#endif
#endif

// What each workgroup takes of a launch that costs `total` in all (up to 2^31 - 1, so rounded up without adding to it), at
// least `least`.
SRA_HD inline int32_t tree_run(int32_t total, int32_t least) {
  const int32_t run = total / kTreeGroups + (total % kTreeGroups != 0);
  return run > least ? run : least;
}

// A group of rows whose keys were split over workgroups, written by the one (w) that has its first keys. That piece is
// in slot 2 w + 1, the others, with which their workgroups begin, in slots 2 (w + i).
struct TreeSplit {
  int32_t pieces;  // 0: none
  int32_t tok0;    // packed token of the sequence's first
  int32_t row0;    // first (token, head of the group) row of the sequence
  int32_t rows;
  int32_t kvh;
};

struct PagedCache {
  __bf16 *k, *v;
  int64_t k_page, v_page, k_token, v_token;  // strides in elements
  const int32_t* table;                      // [batch] rows of table_stride page ids
  int64_t table_stride;
  const int32_t* context_lens;               // [batch]
  const int32_t* cu_tokens;                  // [batch + 1]
  int32_t batch, tokens, pages, page_shift, max_pages, kv_heads;
};

// Cached positions of sequence b.
SRA_HD inline int32_t cache_context(const PagedCache& c, int32_t b) {
  const int64_t room = int64_t(c.max_pages) << c.page_shift, n = c.context_lens[b];
  return int32_t(n < 0 ? 0 : n < room ? n : room);
}
// Page of position pos of sequence b, or -1. pos >= 0.
SRA_HD inline int32_t cache_page(const PagedCache& c, int32_t b, int64_t pos) {
  const int64_t i = pos >> c.page_shift;
  if (i >= c.max_pages) return -1;
  const int32_t id = c.table[int64_t(b) * c.table_stride + i];
  return id >= 0 && id < c.pages ? id : -1;
}
// Position that token i of sequence b is appended at, or -1 where it is not b's.
SRA_HD inline int64_t append_position(const PagedCache& c, int32_t b, int32_t i) {
  const int64_t pos = int64_t(c.context_lens[b] > 0 ? c.context_lens[b] : 0) + i;
  const int32_t first = c.cu_tokens[b] > 0 ? c.cu_tokens[b] : 0;
  return i < first ? -1 : pos - first;
}

// 8-element (16-byte) strides in 32 bits, for the scalar address arithmetic of the tree kernels' loads: a page holds less
// than 2^35 elements.
struct PageSteps {
  uint32_t page, token;
};

struct TreeArgs {
  PagedCache c;
  const __bf16 *q, *k, *v;  // [tokens, heads, D], [tokens, kv_heads, D]
  int64_t qs, ks, vs;
  const uint64_t* tree;     // [tokens] or null: a chain
  __bf16* o;                // dense
  float* lse;               // [heads, tokens]
  int32_t heads;
  uint32_t group_magic;     // ceil(2^32 / G), for exact divisions of small numbers by G = heads / kv_heads > 1
  PageSteps k_step, v_step;
  float scale_log2;
  float* part;              // [2 kTreeGroups] slots: O [rows, D], then (m, l) per row (rows per group of rows)
  TreeSplit* split;         // [kTreeGroups]
};

struct AppendArgs {
  PagedCache c;
  const __bf16 *k, *v;      // [rows, kv_heads, D]
  int64_t ks, vs;
  const int32_t* rows;      // [tokens] or null: row of each token
  int32_t n_rows;
  int32_t row_elems;        // kv_heads * D
};

// rows per group of rows: 16 or 32 (each wave takes its own keys) or kTreeShared (each wave its own rows)
constexpr int kTreeShared = 256;
hipError_t launch_tree(const TreeArgs& a, int rows, int head_dim, hipStream_t stream);
hipError_t launch_append(const AppendArgs& a, hipStream_t stream);

}  // namespace sra
