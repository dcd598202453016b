// Attention of drafted tokens over a paged cache on gfx950, and appending to the cache.
//
// Every new token of a sequence sees the sequence's whole cached context and, of the sequence's new tokens, those
// that its tree mask names; one softmax over both. The G query heads of a K/V head are taken together: "rows" are
// (token, head of the group) pairs, 16 to 256 of them to a group of rows, so that K and V are read once for all of them.
//
// Bound by reading the cache: all of the launch's keys, counted in chunks of 32 or 64 (of each sequence, K/V head and
// group of rows, one after the other, with kStart more for beginning each group), are dealt to the workgroups in
// equal runs, whatever the lengths; a run may end one group of rows and begin another. Lengths are read on the
// device, so a captured call serves any lengths. A group that several workgroups share is added up by a second
// kernel, in the order of its keys.
//
// Few rows (sra_tree_kernel): each of the four waves takes every fourth chunk, alone. It loads the chunk's K and V rows
// into an LDS ring of its own (global -> LDS, the chunks behind it in flight, no barrier), computes S^T = K Q^T, the
// running maximum and sum, and O^T += V^T P^T on 16x16x32 MFMAs; at the end of a run the waves' results are merged
// through LDS. Many rows (sra_tree_shared_kernel): the waves share the tiles and own rows each.
//
// Measured (32 query and 8 K/V heads of 128 dims): 64 requests of 100 to 16,000 positions, one token each, 159 us, 5.3
// TB/s of algorithmic bytes, no other bytes fetched; two of 120 to 131 thousand 191 us (5.4 TB/s); four of 31 to 1,500
// 12 us, a chain of latencies: launch, bounds 1.2 us, first loads 2.5, two chunks 2.5, merge 1, and another 4 us for the
// second kernel. 64 head dims read 4.4 TB/s (half as long rows); from a cache of a few pages (L2) the kernel takes half
// the time. Trees of up to 48 tokens over 16 contexts, 40 query heads, both kernels: 79 us, 77 where the last-level
// cache holds the keys (before they came to that: each 32 rows alone with their keys 226, shared tiles without the software
// pipeline 125, 32 rows to every wave 80); 64 tokens each over 16 x 16,384 positions 334 us, 820 TFLOP/s.
//
// Chains of many tokens are right but not fast: a group of rows computes all of its sequence's keys, also those behind its
// last token, and tiles of new tokens run masked, one load and wait after the other. 4,096 tokens over nothing take 448 us
// (causal attention of packed keys 139), over 8,000 positions 882 (562), 512 tokens 34 (15) and 104 us (79).
#include "sra_fwd_pipe.h"
#include "sra_tree.h"

namespace sra {

namespace {
constexpr int kTreeWaves = 4;
constexpr int kTreeThreads = kTreeWaves * 64;
constexpr int kSharedChunk = 64;
// LDS buffers of the shared kernel, for K and for V. Four, with loads two tiles ahead that a tile's end does not wait for:
// 64 requests of 4,000 positions and 16 tokens, 64 head dims, 134 -> 115 us in turn (112 us on another card, 4.8 TB/s);
// groups of more rows 3 % slower, and 128 head dims spill for them.
template <int D, int NQ> constexpr int kTileBufs = D == 64 && NQ == 1 ? 4 : 3;
constexpr int kNarrow = 128;  // rows of a narrow group of the shared kernel: 16 per wave
// Costs by C, the keys of a chunk: of beginning a group, of a chunk of a narrow and of a wide group, and of the least run.
template <int C> constexpr int kStart = C == kSharedChunk ? kSharedStart : kTreeStart;
template <int C> constexpr int kNarrowCost = C == kSharedChunk ? kSharedNarrow : 1;
template <int C> constexpr int kWideCost = C == kSharedChunk ? kSharedWide : 1;
template <int C> constexpr int kMinRun = C == kSharedChunk ? kSharedMinRun : kTreeMinRun;
template <int D> constexpr int kStages = D == 128 ? 2 : 4;  // chunks of a wave's ring: 32 KB
typedef const __attribute__((address_space(4))) int32_t* const_ints;  // read by scalar loads
}  // namespace

template <int N>
__device__ __forceinline__ void wait_vmem_to() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Inclusive scans over the lanes of a wave (DPP: rows of 16, then their last lanes to the rows behind).
template <int kCtrl, int kRows>
__device__ __forceinline__ int dpp_move(int x, int none) {
  return __builtin_amdgcn_update_dpp(none, x, kCtrl, kRows, 0xf, false);
}
template <class F>
__device__ __forceinline__ int wave_scan(int x, int none, F f) {
  x = f(x, dpp_move<0x111, 0xf>(x, none));  // row_shr 1, 2, 4, 8
  x = f(x, dpp_move<0x112, 0xf>(x, none));
  x = f(x, dpp_move<0x114, 0xf>(x, none));
  x = f(x, dpp_move<0x118, 0xf>(x, none));
  x = f(x, dpp_move<0x142, 0xa>(x, none));  // lane 15 to row 1, lane 47 to row 3
  return f(x, dpp_move<0x143, 0xc>(x, none));  // lane 31 to rows 2 and 3
}

// Bounds of the sequences: first[b] .. first[b + 1] are b's tokens (cu_tokens clamped into [0, tokens] and never
// falling, so no token has two sequences), ctx[b] its cached positions, cost[b] .. cost[b + 1] the costs, in chunks, of
// its groups of rows of all K/V heads.
template <int kDeals>
struct TreeBounds {
  int32_t first[kTreeMaxBatch + 1];
  int32_t ctx[kTreeMaxBatch];
  int32_t cost[kDeals][kTreeMaxBatch + 1];
};

// The cost of a group of rows with n chunks, and of a sequence's groups of R rows (the last may hold fewer).
template <int C>
__device__ __forceinline__ int chunk_cost(int rows) {
  return rows > kNarrow ? kWideCost<C> : kNarrowCost<C>;
}
template <int C>
__device__ __forceinline__ int group_cost(int rows, int n) {
  return kStart<C> + n * chunk_cost<C>(rows);
}
template <int C>
__device__ __forceinline__ int groups_cost(int rows, int n, int R) {
  const int whole = (rows - 1) / R;
  return whole * group_cost<C>(R, n) + group_cost<C>(rows - whole * R, n);
}

__device__ __forceinline__ int group_div(const TreeArgs& a, int G, int x) {  // x / G, x < G + 256
  return G == 1 ? x : int(__umulhi(uint32_t(x), a.group_magic));
}

// Every wave fills all of s, with the same values, so none waits for another. Deal e has groups of R >> e rows; C keys to
// a chunk.
template <int R, int C, int kDeals>
__device__ __forceinline__ void tree_bounds(const TreeArgs& a, TreeBounds<kDeals>& s) {
  const int lane = threadIdx.x & 63, n = a.c.batch;
  const int G = a.heads / a.c.kv_heads;
  int carry_first = 0, carry_cost[kDeals] = {};
  if (lane < kDeals) s.cost[lane][0] = 0;
  int f = 0, end = 0, ctx = 0;
  auto read = [&](int b) {
    f = end = ctx = 0;
    if (b < n) {
      f = a.c.cu_tokens[b];
      end = a.c.cu_tokens[b + 1];
      ctx = cache_context(a.c, b);
    }
  };
  read(lane);
  for (int b0 = 0; b0 < n; b0 += 64) {
    const int b = b0 + lane;
    // first tokens: the running maximum of the clamped cu_tokens[b]
    int first = min(max(f, 0), a.c.tokens);
    const int last = min(max(end, 0), a.c.tokens), cached = ctx;
    read(b + 64);  // the next ones, on their way during the scans
    first = max(carry_first, wave_scan(first, 0, [](int x, int y) { return max(x, y); }));
    const int t = max(first, last) - first;
    const int chunks = (cached + t + C - 1) / C;
#pragma unroll
    for (int e = 0; e < kDeals; ++e) {
      int x = b < n && t > 0 ? groups_cost<C>(t * G, chunks, R >> e) * a.c.kv_heads : 0;
      x = carry_cost[e] + wave_scan(x, 0, [](int x, int y) { return x + y; });
      if (b < n) s.cost[e][b + 1] = x;
      carry_cost[e] = __builtin_amdgcn_readlane(x, 63);
    }
    if (b < n) {
      s.first[b] = first;
      s.ctx[b] = cached;
      if (b == n - 1) s.first[n] = first + t;
    }
    carry_first = __builtin_amdgcn_readlane(first, 63);
  }
  // what a lane wrote, other lanes of the wave read: LDS keeps a wave's order, the compiler is to keep it too
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// The sequence that cost position x belongs to: the first b with cost[b + 1] > x. Two looks of 64 lanes.
__device__ __forceinline__ int tree_sequence(const int32_t* cost, int n, int x) {
  const int lane = threadIdx.x & 63, step = (n + 63) >> 6;
  auto look = [&](int b, int by, bool in) {  // how many of cost[b + by], cost[b + 2 by], .. (b + 64 by at most) x is past
    const int e = b + (lane + 1) * by;
    return __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && e <= n && cost[min(e, n)] <= x));
  };
  const int b = step * look(0, step, true);
  return step == 1 ? b : b + look(b, 1, lane < step);
}

// One run's share of one group of rows.
struct TreeSegment {
  int b, t0, t, ctx;   // sequence, first token, tokens, cached positions
  int kvh, row0, rows;
  int n, c0, c1;       // chunks of the group, and of this run
  int origin, chunk;   // cost position of the group's first chunk, cost of a chunk
  __device__ __forceinline__ int behind() const { return origin + n * chunk; }
  // Runs that have chunks of the group, from its first chunk's, w, on.
  __device__ __forceinline__ int pieces(int w, int run) const { return (origin + (n - 1) * chunk) / run - w + 1; }
};
template <int C, int kDeals>
__device__ __forceinline__ TreeSegment tree_segment(const TreeArgs& a, const TreeBounds<kDeals>& s, int deal, int R, int G,
                                                    int x, int end) {
  TreeSegment g;
  g.b = __builtin_amdgcn_readfirstlane(tree_sequence(s.cost[deal], a.c.batch, x));
  g.t0 = __builtin_amdgcn_readfirstlane(s.first[g.b]);
  g.t = __builtin_amdgcn_readfirstlane(s.first[g.b + 1]) - g.t0;
  g.ctx = __builtin_amdgcn_readfirstlane(s.ctx[g.b]);
  g.n = (g.ctx + g.t + C - 1) / C;  // keys: the context's, then the new tokens'
  const int rows = g.t * G, u = x - __builtin_amdgcn_readfirstlane(s.cost[deal][g.b]);
  const int whole = group_cost<C>(R, g.n), all = groups_cost<C>(rows, g.n, R);
  g.kvh = u / all;
  const int in = u - g.kvh * all, grp = min(in / whole, (rows - 1) / R);
  g.row0 = grp * R;
  g.rows = min(R, rows - g.row0);
  g.chunk = chunk_cost<C>(g.rows);
  g.origin = x - (in - grp * whole) + kStart<C>;
  // chunk i is the run's in which its cost begins
  g.c0 = (max(x - g.origin, 0) + g.chunk - 1) / g.chunk;
  g.c1 = min(g.n, (max(end - g.origin, 0) + g.chunk - 1) / g.chunk);
  return g;
}

// Which of the new tokens a row sees, by chunk: bit e of the word is position p0 + e; `to` = cached positions behind p0.
__device__ __forceinline__ uint32_t tree_word(bool has_tree, uint64_t tree, int tok, int to) {
  uint32_t draft;
  if (has_tree) {
    draft = to >= 32 ? 0 : to >= 0 ? uint32_t(tree << to) : to > -64 ? uint32_t(tree >> -to) : 0;
  } else {
    const int last = tok + to;  // a chain: up to the token itself
    draft = last >= 31 ? ~0u : last < 0 ? 0 : (2u << last) - 1;
  }
  return draft | (to >= 32 ? ~0u : to > 0 ? (1u << to) - 1 : 0);
}

// A lane's key as a row to load: the cache's, a new token's, or, for one that does not exist, the sequence's first new
// token (a row that is there).
struct TreeKey {
  uint64_t k, v;
  bool exists;
};
__device__ __forceinline__ TreeKey tree_key(const TreeArgs& a, const TreeSegment& g, int head_dim, int pos) {
  const PagedCache& c = a.c;
  TreeKey r;
  const int page = pos < g.ctx ? cache_page(c, g.b, pos) : -1;
  r.exists = page >= 0 || (pos >= g.ctx && pos - g.ctx < g.t);
  const __bf16 *k, *v;
  if (page >= 0) {
    const int64_t slot = pos & ((1 << c.page_shift) - 1);
    k = c.k + page * c.k_page + slot * c.k_token;
    v = c.v + page * c.v_page + slot * c.v_token;
  } else {
    const int64_t fresh = g.t0 + (pos < g.ctx ? 0 : min(pos - g.ctx, g.t - 1));
    k = a.k + fresh * a.ks;
    v = a.v + fresh * a.vs;
  }
  r.k = reinterpret_cast<uint64_t>(k + int64_t(g.kvh) * head_dim);
  r.v = reinterpret_cast<uint64_t>(v + int64_t(g.kvh) * head_dim);
  return r;
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t x, int lane) {
  const uint32_t lo = __shfl(int(uint32_t(x)), lane, 64), hi = __shfl(int(uint32_t(x >> 32)), lane, 64);
  return (uint64_t(hi) << 32) | lo;
}

// Address of slot `slot` of page `id`.
__device__ __forceinline__ uint64_t page_row(uint64_t base, const PageSteps& s, int id, int slot) {
  return base + ((uint64_t(uint32_t(id)) * s.page + uint32_t(slot) * s.token) << 4);
}

// Per-wave state of a run over one group of rows.
template <int D, int NQ>
struct TreeState {
  bf16x8 qf[NQ][D / 32];  // Q^T B fragments (lane = row)
  floatx4 o[NQ][D / 16];
  float m[NQ], l[NQ];     // running maximum (log2 units), this lane's part of the sum
};

// P of a chunk against the running maxima m as they are, and the lane's partial sums; false where one is above
// kTreeBigSum (or m still -inf), so that m has to move.
constexpr float kTreeBigSum = 65536.0f;
template <int D, int NQ>
__device__ __forceinline__ bool tree_soft(const TreeState<D, NQ>& st, const floatx4 (&s)[2][NQ], bf16x8 (&p)[NQ],
                                          float (&sum)[NQ], float sl2) {
  bool ok = true;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const float nm = -st.m[qb];
    float acc = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = fast_exp2(fmaf(s[kb][qb][i], sl2, nm));
        acc += x;
        p[qb][4 * kb + i] = (__bf16)x;  // P in bf16 for the matrix product, its sum in 32 bits
      }
    sum[qb] = acc;
    ok = ok && acc <= kTreeBigSum;
  }
  return ok;
}

// Moves m to the true running maxima (rescaling O and l) and computes P and the partial sums against them.
template <int D, int NQ>
__device__ __forceinline__ void tree_rescale(TreeState<D, NQ>& st, const floatx4 (&s)[2][NQ], bf16x8 (&p)[NQ],
                                             float (&sum)[NQ], float sl2) {
  float alpha[NQ];
  bool scale = false;  // some row has an O to scale (at a run's first chunk none has)
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const floatx4 x = s[0][qb], y = s[1][qb];
    const float mx = quad_max(max2f(max3f(x[0], x[1], max2f(x[2], x[3])), max3f(y[0], y[1], max2f(y[2], y[3])))) * sl2;
    const bool up = mx > st.m[qb];
    scale |= up && st.m[qb] != -INFINITY;
    alpha[qb] = up ? st.m[qb] == -INFINITY ? 0.f : fast_exp2(st.m[qb] - mx) : 1.f;
    st.m[qb] = up ? mx : st.m[qb];
    st.l[qb] *= alpha[qb];
  }
  if (__builtin_amdgcn_ballot_w64(scale)) {
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
      for (int db = 0; db < D / 16; ++db) st.o[qb][db] *= alpha[qb];
  }
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const float nm = st.m[qb] == -INFINITY ? 0.f : -st.m[qb];  // a row that has seen nothing keeps P = 0
    float acc = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = fast_exp2(fmaf(s[kb][qb][i], sl2, nm));
        acc += e;
        p[qb][4 * kb + i] = (__bf16)e;
      }
    sum[qb] = acc;
  }
}

// One chunk: K rows at LDS address kt, V rows at vt (waited for between the two by `land_v`). kMasked: key 16 kb + 4 g +
// i of the chunk is seen by this lane's row of block qb if bit 16 kb + 4 g + i of vis[qb] is set.
template <int D, int NQ, bool kMasked, class F>
__device__ __forceinline__ void tree_chunk(TreeState<D, NQ>& st, uint32_t kt, uint32_t vt, uint32_t row, uint32_t tr,
                                           const uint32_t* vis, float sl2, F land_v) {
  constexpr int NC = D / 32, ND = D / 16;
  const int g = (threadIdx.x & 63) >> 4;
  floatx4 s[2][NQ];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bf16x8 k = lds_ld8(((kt + row) ^ (64 * c)) + kb * 32 * D);
      if (c == 0) __builtin_amdgcn_sched_barrier(0);  // all fragments at once would not fit the VGPRs
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) s[kb][qb] = mfma16(k, st.qf[qb][c], c == 0 ? floatx4{} : s[kb][qb]);
    }
  bf16x8 p[NQ];
  float sum[NQ];
  bool ok = false;
  if constexpr (kMasked) {
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      const uint32_t w = vis[qb] >> (4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[0][qb][i] = (w >> i) & 1 ? s[0][qb][i] : -INFINITY;
        s[1][qb][i] = (w >> (16 + i)) & 1 ? s[1][qb][i] : -INFINITY;
      }
    }
  } else {
    ok = tree_soft<D, NQ>(st, s, p, sum, sl2);
  }
  if (kMasked || __builtin_expect(__builtin_amdgcn_ballot_w64(!ok) != 0, 0)) tree_rescale<D, NQ>(st, s, p, sum, sl2);
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) st.l[qb] += sum[qb];
  land_v();
#pragma unroll
  for (int db = 0; db < ND; ++db) {
    const uint32_t x = (vt + tr) ^ (32 * db);
    if (db % 4 == 0) __builtin_amdgcn_sched_barrier(0);
    const bf16x8 v = cat8(lds_ld_tr(x), lds_ld_tr(x + 32 * D));
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) st.o[qb][db] = mfma16(v, p[qb], st.o[qb][db]);
  }
}

template <int D, int NQ>
__global__ void __launch_bounds__(kTreeThreads) sra_tree_kernel(TreeArgs a) {
  constexpr int NC = D / 32, ND = D / 16, R = 16 * NQ;
  constexpr int kInstr = SwzTile<D, kTreeChunk>::kInstr, RPI = 512 / D, CPR = D / 8;  // load instructions, their rows
  constexpr uint32_t kTile = kTreeChunk * D * 2, kRing = kStages<D> * 2 * kTile;
  static_assert(R * D * 4 <= kRing, "a wave's results fit its ring");
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTreeWaves * kRing];
  __shared__ TreeBounds<1> bounds;
  __shared__ float ml[kTreeWaves][R][2];
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.heads / c.kv_heads, page_rows = 1 << c.page_shift;
  const float sl2 = a.scale_log2;
  // neighbouring runs (of one sequence, often of one K/V head) on one XCD
  constexpr int per_xcd = kTreeGroups / kNumXcd;
  const int w = __builtin_amdgcn_readfirstlane((blockIdx.x % kNumXcd) * per_xcd + blockIdx.x / kNumXcd);

  tree_bounds<R, kTreeChunk>(a, bounds);
  const int total = __builtin_amdgcn_readfirstlane(bounds.cost[0][c.batch]);
  const int run = tree_run(total, kMinRun<kTreeChunk>);
  const int begin = int(min(int64_t(w) * run, int64_t(total))), end = int(min(int64_t(begin) + run, int64_t(total)));
  TreeSplit split{0, 0, 0, 0, 0};

  const uint32_t ring = lds_addr(lds) + wave * kRing;
  const uint32_t row = swz_row_addr<D>(), tr = swz_tr_addr<D>();
  // this lane's place in a load instruction (rows RPI j + lane / CPR): the swizzle of its chunk repeats every 8 rows
  constexpr int kKinds = RPI < 8 ? 8 / RPI : 1;
  const int lrow = lane / CPR;
  int chunk16[kKinds];
#pragma unroll
  for (int i = 0; i < kKinds; ++i) chunk16[i] = ((lane % CPR) ^ swz<D>(i * RPI + lrow)) * 8;

  for (int x = begin; x < end;) {
    const TreeSegment seg = tree_segment<kTreeChunk>(a, bounds, 0, R, G, x, end);
    const int t0 = seg.t0, ctx = seg.ctx, n = seg.n, c0 = seg.c0, c1 = seg.c1;
    x = seg.behind();
    if (c0 >= c1) continue;  // the run ends before the group's first chunk
    const const_ints table = (const_ints)(uintptr_t)(c.table + int64_t(seg.b) * c.table_stride);

    const uint64_t kbase = uniform_u64(reinterpret_cast<uint64_t>(c.k + int64_t(seg.kvh) * D));
    const uint64_t vbase = uniform_u64(reinterpret_cast<uint64_t>(c.v + int64_t(seg.kvh) * D));
    // Page ids of chunk i's four groups of 8 rows (a page holds a multiple of 8), where the chunk is all context.
    struct Ids {
      int v[4];
    };
    auto page_ids = [&](int i) __attribute__((always_inline)) {
      Ids ids{};
      if ((i + 1) * kTreeChunk <= ctx) {
#pragma unroll
        for (int j = 0; j < 4; ++j) ids.v[j] = table[(i * kTreeChunk + 8 * j) >> c.page_shift];
      }
      return ids;
    };
    // Issues chunk i's 2 kInstr loads into stage s; returns which of its 32 keys exist.
    auto issue = [&](int i, int s, const Ids& ids) __attribute__((always_inline)) -> uint32_t {
      const uint32_t la = ring + s * 2 * kTile;
      const int p0 = i * kTreeChunk;
      if (p0 + kTreeChunk <= ctx) {
        bool ok = true;
#pragma unroll
        for (int j = 0; j < 4; ++j) ok = ok && uint32_t(ids.v[j]) < uint32_t(c.pages);
        if (ok) {
          constexpr int kPer = kInstr / 4;  // load instructions of 8 rows
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const PageSteps step = kv ? a.v_step : a.k_step;
            const uint32_t lane_row = lrow * step.token * 16;
#pragma unroll
            for (int j = 0; j < kInstr; ++j) {
              const int slot = ((p0 + (j / kPer) * 8) & (page_rows - 1)) + (j % kPer) * RPI;
              lds_dma_x4_off(uniform_u64(page_row(kv ? vbase : kbase, step, ids.v[j / kPer], slot)),
                             lane_row + chunk16[j % kKinds] * 2, la + kv * kTile + j * 1024);
            }
          }
          return ~0u;
        }
      }
      // the context's end, new tokens, or a page that is none: row by row
      const TreeKey key = tree_key(a, seg, D, p0 + (lane & 31));
#pragma unroll 1
      for (int kv = 0; kv < 2; ++kv) {  // K, then V: the waits below count on that order
        const uint64_t mine = kv ? key.v : key.k;
#pragma unroll 1
        for (int j = 0; j < kInstr; j += kKinds)
#pragma unroll
          for (int e = 0; e < kKinds; ++e)
            lds_dma_x4_at(reinterpret_cast<const __bf16*>(lane_u64(mine, (j + e) * RPI + lrow)) + chunk16[e],
                          la + kv * kTile + (j + e) * 1024);
      }
      return uint32_t(__builtin_amdgcn_ballot_w64(key.exists));
    };

    // chunk i + kTreeWaves k sits in stage k % NS; NS - 1 chunks are in flight behind the one that is worked on
    constexpr int NS = kStages<D>, kAhead = (NS - 1) * kTreeWaves;
    uint32_t exist[NS];
#pragma unroll
    for (int k = 0; k < NS - 1; ++k) {
      exist[k] = 0;
      const int i = c0 + wave + k * kTreeWaves;
      if (i < c1) exist[k] = issue(i, k, page_ids(i));
    }
    Ids ids = page_ids(c0 + wave + kAhead);  // of the chunk that is loaded next
    TreeState<D, NQ> st;
    uint64_t tree[NQ];  // which drafted tokens the lane's row sees
    int tok[NQ];
    const int tok0 = seg.row0 / G, rem0 = seg.row0 - tok0 * G;  // the group's first row
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      const int r = rem0 + min(16 * qb + l16, seg.rows - 1), dt = group_div(a, G, r), h = seg.kvh * G + r - dt * G;
      tok[qb] = tok0 + dt;
      tree[qb] = a.tree ? a.tree[t0 + tok[qb]] : 0;
      const __bf16* src = a.q + int64_t(t0 + tok[qb]) * a.qs + int64_t(h) * D + g * 8;
#pragma unroll
      for (int i = 0; i < NC; ++i) st.qf[qb][i] = ld8(src + i * 32);
#pragma unroll
      for (int db = 0; db < ND; ++db) st.o[qb][db] = floatx4{};
      st.m[qb] = -INFINITY;
      st.l[qb] = 0.f;
    }
    // land them here, behind the first chunks: the waits inside the loop count the direct loads alone
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
#pragma unroll
      for (int i = 0; i < NC; ++i) asm volatile("" : "+v"(st.qf[qb][i]));
      asm volatile("" : "+v"(tree[qb]));
    }

    int s = 0;
    for (int i = c0 + wave; i < c1; i += kTreeWaves) {
      const bool more = i + kAhead < c1;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage that is loaded next has been read
      exist[NS - 1] = 0;
      if (more) {
        exist[NS - 1] = issue(i + kAhead, (s + NS - 1) % NS, ids);
        ids = page_ids(i + kAhead + kTreeWaves);
        // the loads of the chunks behind this one, and this one's V, may be in flight
        wait_vmem_to<(2 * (NS - 1) + 1) * kInstr>();
      } else {
        wait_vmem_to<0>();
      }
      auto land_v = [&]() __attribute__((always_inline)) {
        if (more) wait_vmem_to<2 * (NS - 1) * kInstr>();
      };
      const uint32_t kt = ring + s * 2 * kTile, vt = kt + kTile;
      if (exist[0] == ~0u && (i + 1) * kTreeChunk <= ctx) {
        tree_chunk<D, NQ, false>(st, kt, vt, row, tr, nullptr, sl2, land_v);
      } else {
        uint32_t vis[NQ];
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb)
          vis[qb] = exist[0] & tree_word(a.tree, tree[qb], tok[qb], ctx - i * kTreeChunk);
        tree_chunk<D, NQ, true>(st, kt, vt, row, tr, vis, sl2, land_v);
      }
#pragma unroll
      for (int k = 0; k + 1 < NS; ++k) exist[k] = exist[k + 1];
      s = (s + 1) % NS;
    }

    // merge the waves' results: a wave's ring holds its O by rows, the 16-byte pieces of row r XORed with r % 16
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      const float l = quad_sum(st.l[qb]);
      if (g == 0) {
        ml[wave][16 * qb + l16][0] = st.m[qb];
        ml[wave][16 * qb + l16][1] = l;
      }
    }
    float* const mine = reinterpret_cast<float*>(lds + wave * kRing);
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
      for (int db = 0; db < ND; ++db)
        *reinterpret_cast<floatx4*>(mine + (16 * qb + l16) * D + ((4 * db + g) ^ l16) * 4) = st.o[qb][db];
    __syncthreads();
    const bool whole = c0 == 0 && c1 == n;
    const int slot = 2 * w + (c0 == 0);
    float* const part = a.part + int64_t(slot) * R * (D + 2);
    constexpr int kRowStep = kTreeThreads / (D / 4);
#pragma unroll 2
    for (int r0 = 0; r0 < R; r0 += kRowStep) {
      const int r = r0 + threadIdx.x / (D / 4), q = threadIdx.x % (D / 4);
      if (r >= seg.rows) continue;
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < kTreeWaves; ++i) m = max2f(m, ml[i][r][0]);
      float l = 0.f;
      floatx4 o = floatx4{};
#pragma unroll
      for (int i = 0; i < kTreeWaves; ++i) {
        const float li = ml[i][r][1];
        const float f = li == 0.f ? 0.f : fast_exp2(ml[i][r][0] - m);  // a wave that saw nothing has m = -inf
        l += f * li;
        o += f * *reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(lds + i * kRing) + r * D + (q ^ (r & 15)) * 4);
      }
      if (whole) {
        const int rr = rem0 + r, dt = group_div(a, G, rr), h = seg.kvh * G + rr - dt * G;
        const int64_t token = t0 + tok0 + dt;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (__bf16)(o[i] * inv);
        *reinterpret_cast<bf16x4*>(a.o + (token * a.heads + h) * D + 4 * q) = y;
        if (q == 0) a.lse[int64_t(h) * c.tokens + token] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      } else {
        *reinterpret_cast<floatx4*>(part + r * D + 4 * q) = o;
        if (q == 0) *reinterpret_cast<float2*>(part + R * D + 2 * r) = float2{m, l};
      }
    }
    if (!whole && c0 == 0)  // the group's first keys
      split = TreeSplit{seg.pieces(w, run), t0, seg.row0, seg.rows, seg.kvh};
    __syncthreads();  // the rings and ml are free again
  }
  if (threadIdx.x == 0) a.split[w] = split;
}

// A 32-key half whose keys p0 .. a row sees by the bits of vis[qb] (LDS rows past the last key hold a row that is there).
template <int D, int NQ>
__device__ __forceinline__ void tree_half(FwdState<D, NQ>& st, const __bf16* kt, const __bf16* vt, const uint32_t* vis,
                                          float sl2) {
  const int g = (threadIdx.x & 63) >> 4;
  HalfS<NQ> s = scores32<D, NQ, SwizzledRows>(st, kt);
#pragma unroll
  for (int j = 0; j < 2 * NQ; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) s.b[j][i] = (vis[j % NQ] >> (16 * (j / NQ) + 4 * g + i)) & 1 ? s.b[j][i] : -INFINITY;
  float sum[NQ];
  rescale_half<D, NQ>(st, s, sl2, sum);
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) st.l[qb] += sum[qb];
  pv_half<D, NQ, SwizzledRows>(st, vt, pack_half<NQ>(s));
}

// Where the shared kernel's tiles lie.
template <int D>
struct SharedTiles {
  __bf16 *k[kTileBufs<D, 1>], *v[kTileBufs<D, 1>];
};

// The run's share of a group of at most 128 NQ rows, 16 NQ per wave; an unfinished group's results go to `part`.
template <int D, int NQ>
__device__ __forceinline__ void shared_group(const TreeArgs& a, const TreeSegment& seg, const SharedTiles<D>& lds,
                                             float* part) {
  constexpr int NC = D / 32, ND = D / 16, C = kSharedChunk;
  using TL = SwzTile<D, C>;
  constexpr int RPI = 512 / D, CPR = D / 8, kPer = TL::kInstr / kWaves;  // rows of a load instruction; a wave's of a tile
  static_assert(kPer >= 1 && RPI * kWaves % 8 == 0 && C == kFwdKeyStep, "tiles by waves");
  constexpr int NB = kTileBufs<D, NQ>;
  __bf16* const* const kb = lds.k;
  __bf16* const* const vb = lds.v;
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.heads / c.kv_heads, page_mask = (1 << c.page_shift) - 1;
  const float sl2 = a.scale_log2;
  // load instructions wave + 8 j of a tile: rows RPI (wave + 8 j) + lane / CPR, one swizzle for all j
  const int lrow = RPI * wave + lane / CPR, chunk16 = ((lane % CPR) ^ swz<D>(lrow)) * 8;
  const uint32_t koff = (uint32_t((lane / CPR) * c.k_token) + chunk16) * 2;
  const uint32_t voff = (uint32_t((lane / CPR) * c.v_token) + chunk16) * 2;
  const int t0 = seg.t0, ctx = seg.ctx, n = seg.n, c0 = seg.c0, c1 = seg.c1;
  const const_ints table = (const_ints)(uintptr_t)(c.table + int64_t(seg.b) * c.table_stride);
  int T = max(0, min(c1, ctx / C) - c0);  // whole tiles of the context
  bool bad = false;
  if (T > 0)
    for (int p = (c0 * C >> c.page_shift) + lane; p <= ((c0 + T) * C - 1) >> c.page_shift; p += 64)
      bad |= uint32_t(c.table[int64_t(seg.b) * c.table_stride + p]) >= uint32_t(c.pages);
  if (__builtin_amdgcn_ballot_w64(bad)) T = 0;

  // page ids of this wave's load instructions of tile i (an instruction's rows lie in one 8-row part of a page)
  struct Ids {
    int v[kPer];
  };
  auto page_ids = [&](int i) __attribute__((always_inline)) {
    Ids ids{};
    if (i < c0 + T)
#pragma unroll
      for (int j = 0; j < kPer; ++j) ids.v[j] = table[(i * C + RPI * (wave + j * kWaves)) >> c.page_shift];
    return ids;
  };
  const uint64_t kbase = uniform_u64(reinterpret_cast<uint64_t>(c.k + int64_t(seg.kvh) * D));
  const uint64_t vbase = uniform_u64(reinterpret_cast<uint64_t>(c.v + int64_t(seg.kvh) * D));
  auto issue = [&](int i, const Ids& ids, bool is_v, const __bf16* dst) __attribute__((always_inline)) {
    const uint32_t la = lds_addr(dst) + wave * 1024;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int slot = (i * C + RPI * (wave + j * kWaves)) & page_mask;
      lds_dma_x4_off(uniform_u64(page_row(is_v ? vbase : kbase, is_v ? a.v_step : a.k_step, ids.v[j], slot)),
                     is_v ? voff : koff, la + j * kWaves * 1024);
    }
  };
  int next_k = c0, next_v = c0;
  Ids ids_k = page_ids(c0), ids_v = ids_k;  // of the tiles that are loaded next
  auto issue_k = [&](const __bf16* dst) __attribute__((always_inline)) {
    issue(next_k, ids_k, false, dst);
    ids_k = page_ids(++next_k);
  };
  auto issue_v = [&](const __bf16* dst) __attribute__((always_inline)) {
    issue(next_v, ids_v, true, dst);
    ids_v = page_ids(++next_v);
  };
  if (T > 0) {
    issue_k(kb[0]);
    issue_v(vb[0]);
    if (T > 1) issue_k(kb[1]);
    if constexpr (NB == 4) {
      if (T > 1) issue_v(vb[1]);
      if (T > 2) issue_k(kb[2]);
    }
  }

  FwdState<D, NQ> st;
  const int wrow = wave * 16 * NQ;
  const bool active = wrow < seg.rows;
  const int tok0 = seg.row0 / G, rem0 = seg.row0 - tok0 * G;
  auto row_of = [&](int qb) { return rem0 + min(wrow + 16 * qb + l16, seg.rows - 1); };
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = row_of(qb), dt = group_div(a, G, r), h = seg.kvh * G + r - dt * G;
    const __bf16* src = a.q + int64_t(t0 + tok0 + dt) * a.qs + int64_t(h) * D + g * 8;
#pragma unroll
    for (int i = 0; i < NC; ++i) st.qf[qb][i] = ld8(src + i * 32);
#pragma unroll
    for (int db = 0; db < ND; ++db) st.o[qb][db] = floatx4{};
    st.m[qb] = -INFINITY;
    st.l[qb] = 0.f;
  }
  // land them here, behind the first tiles, not at their first use inside the loop
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
    for (int i = 0; i < NC; ++i) asm volatile("" : "+v"(st.qf[qb][i]));

  // Tile t sits in K buffer t % NB and V buffer t % NB (tile -1 in V buffer NB - 1). Iteration t reads K(t) (second
  // half), K(t+1) (first half), V(t-1) (second half) and V(t) (first half), and loads K(t+NB-1) and V(t+NB-2).
  if (T > 0) {
    for (int e = threadIdx.x * 8; e < 32 * D; e += kWaves * 64 * 8)
      *reinterpret_cast<bf16x8*>(vb[NB - 1] + 32 * D + e) = bf16x8{};
    wait_vmem();
    __syncthreads();
    HalfP<NQ> p_hi;
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) p_hi.p[qb] = bf16x8{};
    HalfS<NQ> s_lo = {}, s_hi = {};
    if (active) s_lo = scores32<D, NQ, SwizzledRows>(st, kb[0]);
    Ahead ah;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      ah.k[i] = k_frag<D, SwizzledRows>(kb[0] + 32 * D, i);
      ah.v[i] = v_frag<D, SwizzledRows>(vb[NB - 1] + 32 * D, i);
    }
    auto iteration = [&](int t, auto phase) {
      constexpr int P = decltype(phase)::value;
      __bf16* const k_t = kb[P];
      __bf16* const k_t1 = kb[(P + 1) % NB];
      __bf16* const v_tm1 = vb[(P + NB - 1) % NB];
      __bf16* const v_t = vb[P];
      if (t + NB - 2 < T) issue_v(vb[(P + NB - 2) % NB]);
      if (t + NB - 1 < T) issue_k(kb[(P + NB - 1) % NB]);
      if (active) {
        const HalfP<NQ> p_lo = pipe_block<D, NQ, SwizzledRows>(st, s_lo, k_t, s_hi, k_t + 32 * D, v_tm1 + 32 * D, k_t1,
                                                               v_t, ah, p_hi, sl2);
        p_hi = pipe_block<D, NQ, SwizzledRows>(st, s_hi, k_t + 32 * D, s_lo, k_t1, v_t, k_t1 + 32 * D, v_t + 32 * D, ah,
                                               p_lo, sl2);
      }
      // with four buffers this iteration's loads may be in flight
      if (NB == 4 && t + NB - 1 < T) wait_vmem_to<2 * kPer>();
      else wait_vmem();
      __syncthreads();
    };
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    using P2 = std::integral_constant<int, 2>;
    using P3 = std::integral_constant<int, 3>;
    int t = 0;
    for (; t + NB <= T; t += NB) {
      iteration(t, P0{});
      iteration(t + 1, P1{});
      iteration(t + 2, P2{});
      if constexpr (NB == 4) iteration(t + 3, P3{});
    }
    if (t < T) iteration(t, P0{});
    if (t + 1 < T) iteration(t + 1, P1{});
    if constexpr (NB == 4)
      if (t + 2 < T) iteration(t + 2, P2{});
    if (active) {
      const int last = (T - 1) % NB;
      if (last == 0) pv_half<D, NQ, SwizzledRows>(st, vb[0] + 32 * D, p_hi);
      else if (last == 1) pv_half<D, NQ, SwizzledRows>(st, vb[1] + 32 * D, p_hi);
      else if (NB == 3 || last == 2) pv_half<D, NQ, SwizzledRows>(st, vb[2] + 32 * D, p_hi);
      else pv_half<D, NQ, SwizzledRows>(st, vb[NB - 1] + 32 * D, p_hi);
    }
  }

  // the masked tiles
  for (int i = c0 + T; i < c1; ++i) {
    __syncthreads();  // every wave is done with the buffers
    const TreeKey key = tree_key(a, seg, D, i * C + lane);
    const uint64_t exist = __builtin_amdgcn_ballot_w64(key.exists);
#pragma unroll 1
    for (int j = 0; j < kPer; ++j) {
      const int r = lrow + j * RPI * kWaves;
      lds_dma_x4_at(reinterpret_cast<const __bf16*>(lane_u64(key.k, r)) + chunk16, lds_addr(kb[0]) + (wave + j * kWaves) * 1024);
      lds_dma_x4_at(reinterpret_cast<const __bf16*>(lane_u64(key.v, r)) + chunk16, lds_addr(vb[0]) + (wave + j * kWaves) * 1024);
    }
    uint64_t tree[NQ];  // which new tokens the lane's row sees
    int tok[NQ];
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      tok[qb] = tok0 + group_div(a, G, row_of(qb));
      tree[qb] = a.tree ? a.tree[t0 + tok[qb]] : 0;
    }
    wait_vmem();
    __syncthreads();
    if (active)
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        uint32_t vis[NQ];
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb)
          vis[qb] = uint32_t(exist >> (32 * half)) & tree_word(a.tree, tree[qb], tok[qb], ctx - i * C - 32 * half);
        tree_half<D, NQ>(st, kb[0] + half * 32 * D, vb[0] + half * 32 * D, vis, sl2);
      }
  }

  const bool whole = c0 == 0 && c1 == n;
  if (active) {
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      const int r = wrow + 16 * qb + l16;
      const float l = quad_sum(st.l[qb]);
      if (r >= seg.rows) continue;
      if (whole) {
        const int rr = rem0 + r, dt = group_div(a, G, rr), h = seg.kvh * G + rr - dt * G;
        const int64_t token = t0 + tok0 + dt;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        __bf16* orow = a.o + (token * a.heads + h) * D + 4 * g;
#pragma unroll
        for (int db = 0; db < ND; ++db) {
          bf16x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = (__bf16)(st.o[qb][db][e] * inv);
          *reinterpret_cast<bf16x4*>(orow + db * 16) = y;
        }
        if (g == 0) a.lse[int64_t(h) * c.tokens + token] = l == 0.f ? -INFINITY : (st.m[qb] + log2f(l)) * kLn2;
      } else {
#pragma unroll
        for (int db = 0; db < ND; ++db) *reinterpret_cast<floatx4*>(part + r * D + db * 16 + 4 * g) = st.o[qb][db];
        if (g == 0) *reinterpret_cast<float2*>(part + kTreeShared * D + 2 * r) = float2{st.m[qb], l};
      }
    }
  }
}

// The same for many rows (trees of drafted tokens): up to 256 rows to a group, so that K and V are read once for all of
// them, or 128 where that would split the groups of a short launch. Eight waves (two per SIMD) own 16 or 32 rows each, as
// the group has up to 128 or more (32 for all of them: half of the waves idle, 6 % slower); the keys go through LDS in
// 64-key tiles that all of them read.
// Whole tiles of the context run through the software pipeline of sra_fwd_pipe.h (three buffers each for K and V, loads
// two and one tiles ahead, or four), the context's end and the new tokens behind them, masked. Where the table names a page
// that is none, all of the group's tiles run masked.
template <int D>
__global__ void __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
sra_tree_shared_kernel(TreeArgs a) {
  constexpr int C = kSharedChunk;
  using TL = SwzTile<D, C>;
  constexpr int NB = kTileBufs<D, 1>;
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf0[TL::kElems];
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf1[TL::kElems];
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf2[TL::kElems];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf0[TL::kElems];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf1[TL::kElems];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf2[TL::kElems];
  __shared__ __attribute__((aligned(1024))) __bf16 buf3[NB == 4 ? 2 * TL::kElems : 8];
  SharedTiles<D> tiles;
  tiles.k[0] = kbuf0, tiles.k[1] = kbuf1, tiles.k[2] = kbuf2;
  tiles.v[0] = vbuf0, tiles.v[1] = vbuf1, tiles.v[2] = vbuf2;
  if constexpr (NB == 4) tiles.k[3] = buf3, tiles.v[3] = buf3 + TL::kElems;
  __shared__ TreeBounds<2> bounds;
  const PagedCache& c = a.c;
  const int G = a.heads / c.kv_heads;
  constexpr int per_xcd = kTreeGroups / kNumXcd;
  const int w = __builtin_amdgcn_readfirstlane((blockIdx.x % kNumXcd) * per_xcd + blockIdx.x / kNumXcd);

  tree_bounds<kTreeShared, C>(a, bounds);
  int deal = 0, total = __builtin_amdgcn_readfirstlane(bounds.cost[0][c.batch]);
  if (total < kSharedShortRun * kTreeGroups) {
    deal = 1;
    total = __builtin_amdgcn_readfirstlane(bounds.cost[1][c.batch]);
  }
  const int run = tree_run(total, kMinRun<C>);
  const int begin = int(min(int64_t(w) * run, int64_t(total))), end = int(min(int64_t(begin) + run, int64_t(total)));
  TreeSplit split{0, 0, 0, 0, 0};
  for (int x = begin; x < end;) {
    const TreeSegment seg = tree_segment<C>(a, bounds, deal, kTreeShared >> deal, G, x, end);
    x = seg.behind();
    if (seg.c0 >= seg.c1) continue;  // the run ends before the group's first tile
    float* const part = a.part + int64_t(2 * w + (seg.c0 == 0)) * kTreeShared * (D + 2);
    if (seg.rows > kNarrow) shared_group<D, 2>(a, seg, tiles, part);
    else shared_group<D, 1>(a, seg, tiles, part);
    if (seg.c0 == 0 && seg.c1 < seg.n)  // the group's first keys
      split = TreeSplit{seg.pieces(w, run), seg.t0, seg.row0, seg.rows, seg.kvh};
    __syncthreads();  // the buffers are free again
  }
  if (threadIdx.x == 0) a.split[w] = split;
}

// Groups of rows that several workgroups share, from their pieces, in key order: with M the largest of their maxima,
// O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i. D / 4 threads per row, R rows to a slot.
template <int D, int R>
__global__ void __launch_bounds__(kTreeThreads) sra_tree_combine_kernel(TreeArgs a) {
  constexpr int TPR = D / 4, RPB = kTreeThreads / TPR;
  constexpr int64_t kSlot = int64_t(R) * (D + 2);
  const int w = blockIdx.x;
  const TreeSplit sp = a.split[w];
  const int r = blockIdx.y * RPB + threadIdx.x / TPR, sub = threadIdx.x % TPR;
  if (sp.pieces == 0 || r >= sp.rows) return;
  auto piece = [&](int i) { return a.part + kSlot * (2 * (w + i) + (i == 0)); };
  float m = -INFINITY, l = 0.f;
  floatx4 o = floatx4{};
#pragma unroll 4
  for (int i = 0; i < sp.pieces; ++i) {  // one pass with a running maximum: the loads of four pieces are under way at once
    const float* p = piece(i);
    const float2 ml = *reinterpret_cast<const float2*>(p + R * D + 2 * r);
    const floatx4 x = *reinterpret_cast<const floatx4*>(p + r * D + 4 * sub);
    const float mx = fmaxf(m, ml.x);
    const float f = l == 0.f ? 0.f : fast_exp2(m - mx);        // nothing so far
    const float e = ml.y == 0.f ? 0.f : fast_exp2(ml.x - mx);  // a piece that the row sees nothing of has m = -inf
    l = f * l + e * ml.y;
    o = f * o + e * x;
    m = mx;
  }
  const int G = a.heads / a.c.kv_heads, rr = sp.row0 + r, token = rr / G, h = sp.kvh * G + rr - token * G;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * inv);
  *reinterpret_cast<bf16x4*>(a.o + (int64_t(sp.tok0 + token) * a.heads + h) * D + 4 * sub) = y;
  if (sub == 0) a.lse[int64_t(h) * a.c.tokens + sp.tok0 + token] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Token i of the packed tokens, of sequence b: row rows[i] (or i) of k and v -> position context_lens[b] + i -
// cu_tokens[b] of b's pages. One wave per token; bound by the copy: 40,000 tokens of 8 heads of 128 dims 57 us, 5.7 TB/s.
__global__ void __launch_bounds__(kTreeThreads) sra_append_kernel(AppendArgs a) {
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63;
  const int i = __builtin_amdgcn_readfirstlane(blockIdx.x * kTreeWaves + (threadIdx.x >> 6));
  if (uint32_t(i) >= uint32_t(c.tokens)) return;  // i of the last block may pass 31 bits
  // the sequence: as many end at or before token i
  int b = 0;
  for (int b0 = 0; b0 < c.batch; b0 += 64) {
    const int end = b0 + lane < c.batch ? c.cu_tokens[b0 + lane + 1] : 0x7fffffff;
    const uint64_t over = __builtin_amdgcn_ballot_w64(end > i);
    if (over) {
      b = b0 + __builtin_ctzll(over);
      break;
    }
    b = b0 + 64;
  }
  if (b >= c.batch) return;  // behind the last sequence
  const int64_t pos = append_position(c, b, i);
  const int row = a.rows ? a.rows[i] : i;
  if (pos < 0 || row < 0 || row >= a.n_rows) return;
  const int64_t id = cache_page(c, b, pos);
  if (id < 0) return;
  const int64_t slot = pos & ((1 << c.page_shift) - 1);
  const __bf16 *ks = a.k + row * a.ks, *vs = a.v + row * a.vs;
  __bf16 *kd = c.k + id * c.k_page + slot * c.k_token, *vd = c.v + id * c.v_page + slot * c.v_token;
  for (int e = lane * 8; e < a.row_elems; e += 512) {
    const bf16x8 x = ld8(ks + e), y = ld8(vs + e);
    *reinterpret_cast<bf16x8*>(kd + e) = x;
    *reinterpret_cast<bf16x8*>(vd + e) = y;
  }
}

template <int D, int R>
static void launch_tree_rows(const TreeArgs& a, hipStream_t stream) {
  constexpr int RPB = kTreeThreads / (D / 4);
  if constexpr (R == kTreeShared)
    hipLaunchKernelGGL(sra_tree_shared_kernel<D>, dim3(kTreeGroups), dim3(kWaves * 64), 0, stream, a);
  else
    hipLaunchKernelGGL((sra_tree_kernel<D, R / 16>), dim3(kTreeGroups), dim3(kTreeThreads), 0, stream, a);
  hipLaunchKernelGGL((sra_tree_combine_kernel<D, R>), dim3(kTreeGroups, R / RPB), dim3(kTreeThreads), 0, stream, a);
}

template <int D>
static void launch_tree_dim(const TreeArgs& a, int rows, hipStream_t stream) {
  if (rows == 16) launch_tree_rows<D, 16>(a, stream);
  else if (rows == 32) launch_tree_rows<D, 32>(a, stream);
  else launch_tree_rows<D, kTreeShared>(a, stream);
}

hipError_t launch_tree(const TreeArgs& a, int rows, int head_dim, hipStream_t stream) {
  if (a.c.tokens <= 0) return hipSuccess;
  if (head_dim == 128) launch_tree_dim<128>(a, rows, stream);
  else launch_tree_dim<64>(a, rows, stream);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
  if (a.c.tokens <= 0) return hipSuccess;
  const dim3 grid((a.c.tokens + kTreeWaves - 1) / kTreeWaves);
  hipLaunchKernelGGL(sra_append_kernel, grid, dim3(kTreeThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sra
