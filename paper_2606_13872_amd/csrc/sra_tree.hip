// Attention of drafted tokens over a paged cache on gfx950, and appending to the cache.
//
// Every new token of a sequence sees the sequence's whole cached context and, of the sequence's new tokens, those
// that its tree mask names; one softmax over both. The G query heads of a K/V head are taken together: "rows" are
// (token, head of the group) pairs, 16 NQ of them to a group of rows, so that K and V are read once for all of them.
//
// Bound by reading the cache: all of the launch's keys, counted in 32-key chunks (of each sequence, K/V head and
// group of rows, one after the other, with kTreeStart more for beginning each group), are dealt to the workgroups in
// equal runs, whatever the lengths; a run may end one group of rows and begin another. Lengths are read on the
// device, so a captured call serves any lengths. A group that several workgroups share is added up by a second
// kernel, in the order of its keys.
//
// In a workgroup each of the four waves takes every fourth chunk, alone: it loads the chunk's K and V rows into an
// LDS ring of its own (global -> LDS, the chunks behind it in flight, no barrier), computes S^T = K Q^T, the running maximum and
// sum, and O^T += V^T P^T on 16x16x32 MFMAs; at the end of a run the waves' results are merged through LDS.
#include "sra_tiles.h"
#include "sra_tree.h"

namespace sra {

namespace {
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kTreeWaves = 4;
constexpr int kTreeThreads = kTreeWaves * 64;
template <int D> constexpr int kStages = D == 128 ? 2 : 4;  // chunks of a wave's ring: 32 KB
typedef const __attribute__((address_space(4))) int32_t* const_ints;  // read by scalar loads
}  // namespace

template <int N>
__device__ __forceinline__ void wait_vmem_to() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Bounds of the sequences: first[b] .. first[b + 1] are b's tokens (cu_tokens clamped into [0, tokens] and never
// falling, so no token has two sequences), chunk[b] .. chunk[b + 1] the costs, in chunks, of its groups of rows of all
// K/V heads.
struct TreeBounds {
  int32_t first[kTreeMaxBatch + 1];
  int32_t chunk[kTreeMaxBatch + 1];
  int32_t wave[2][kTreeWaves];
};

template <int NQ>
__device__ __forceinline__ void tree_bounds(const TreeArgs& a, TreeBounds& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.c.batch;
  const int G = a.heads / a.c.kv_heads;
  int carry_first = 0, carry_chunk = 0;
  if (threadIdx.x == 0) s.chunk[0] = 0;
  for (int b0 = 0; b0 < n; b0 += kTreeThreads) {
    const int b = b0 + threadIdx.x;
    const bool in = b < n;
    // first tokens: the running maximum of the clamped cu_tokens[b]
    int f = in ? min(max(a.c.cu_tokens[b], 0), a.c.tokens) : 0;
    const int end_raw = in ? min(max(a.c.cu_tokens[b + 1], 0), a.c.tokens) : 0;
    const int ctx = in ? cache_context(a.c, b) : 0;
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) {
      const int y = __shfl_up(f, w, 64);
      if (lane >= w) f = max(f, y);
    }
    if (lane == 63) s.wave[0][wave] = f;
    __syncthreads();
    f = max(f, carry_first);
    for (int w = 0; w < wave; ++w) f = max(f, s.wave[0][w]);
    const int end = max(f, end_raw), t = end - f;
    const int chunks = kTreeStart + (ctx + t + kTreeChunk - 1) / kTreeChunk;
    int x = t > 0 ? chunks * ((t * G + 16 * NQ - 1) / (16 * NQ)) * a.c.kv_heads : 0;
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) {
      const int y = __shfl_up(x, w, 64);
      if (lane >= w) x += y;
    }
    if (lane == 63) s.wave[1][wave] = x;
    __syncthreads();
    x += carry_chunk;
    for (int w = 0; w < wave; ++w) x += s.wave[1][w];
    if (in) {
      s.first[b] = f;
      s.chunk[b + 1] = x;
      if (b == n - 1) s.first[n] = end;
    }
    for (int w = 0; w < kTreeWaves; ++w) {
      carry_first = max(carry_first, s.wave[0][w]);
      carry_chunk += s.wave[1][w];
    }
    __syncthreads();
  }
  __syncthreads();
}

// Per-wave state of a run over one group of rows.
template <int D, int NQ>
struct TreeState {
  static constexpr bool kAgpr = NQ == 4;  // O in AGPRs (inline-assembly MFMAs): with it the VGPRs would not do
  bf16x8 qf[NQ][D / 32];  // Q^T B fragments (lane = row)
  floatx4 o[NQ][D / 16];
  float m[NQ], l[NQ];     // running maximum (log2 units), this lane's part of the sum
  // O may be read and written by vector instructions from here on
  __device__ __forceinline__ void settle() {
    if constexpr (kAgpr) {
      mfma_drain();
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
        for (int db = 0; db < D / 16; ++db) asm volatile("" : "+a"(o[qb][db]));
    }
  }
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
  st.settle();
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const floatx4 x = s[0][qb], y = s[1][qb];
    const float mx = quad_max(max2f(max3f(x[0], x[1], max2f(x[2], x[3])), max3f(y[0], y[1], max2f(y[2], y[3])))) * sl2;
    if (mx > st.m[qb]) {
      const float alpha = fast_exp2(st.m[qb] - mx);  // 0 when m was -inf
      st.m[qb] = mx;
      st.l[qb] *= alpha;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) st.o[qb][db] *= alpha;
    }
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
    const bf16x8 v = cat8(lds_ld_tr(x), lds_ld_tr(x + 32 * D));
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      if constexpr (TreeState<D, NQ>::kAgpr) mfma16_agpr(st.o[qb][db], v, p[qb]);
      else st.o[qb][db] = mfma16(v, p[qb], st.o[qb][db]);
    }
  }
}

template <int D, int NQ>
__global__ void __launch_bounds__(kTreeThreads) sra_tree_kernel(TreeArgs a) {
  constexpr int NC = D / 32, ND = D / 16, R = 16 * NQ;
  constexpr int kInstr = SwzTile<D, kTreeChunk>::kInstr, RPI = 512 / D, CPR = D / 8;  // load instructions, their rows
  constexpr uint32_t kTile = kTreeChunk * D * 2, kRing = kStages<D> * 2 * kTile;
  static_assert(R * D * 4 <= kRing, "a wave's results fit its ring");
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTreeWaves * kRing];
  __shared__ TreeBounds bounds;
  __shared__ float ml[kTreeWaves][R][2];
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.heads / c.kv_heads, page_rows = 1 << c.page_shift;
  const float sl2 = a.scale_log2;
  // neighbouring runs (of one sequence, often of one K/V head) on one XCD
  constexpr int per_xcd = kTreeGroups / kNumXcd;
  const int w = __builtin_amdgcn_readfirstlane((blockIdx.x % kNumXcd) * per_xcd + blockIdx.x / kNumXcd);

  tree_bounds<NQ>(a, bounds);
  const int total = __builtin_amdgcn_readfirstlane(bounds.chunk[c.batch]);
  const int run = max(kTreeMinRun, (total + kTreeGroups - 1) / kTreeGroups);
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
    // the sequence that chunk x belongs to
    int b = 0;
    for (int lo = 0, hi = c.batch; lo < hi;) {  // the last b with chunk[b] <= x and chunks of its own
      b = (lo + hi) >> 1;
      if (__builtin_amdgcn_readfirstlane(bounds.chunk[b + 1]) <= x) lo = ++b;
      else hi = b;
    }
    const int t0 = __builtin_amdgcn_readfirstlane(bounds.first[b]);
    const int t = __builtin_amdgcn_readfirstlane(bounds.first[b + 1]) - t0;
    const int ctx = __builtin_amdgcn_readfirstlane(cache_context(c, b));
    const int n = (ctx + t + kTreeChunk - 1) / kTreeChunk;  // keys: the context's, then the new tokens'
    const int blocks = (t * G + R - 1) / R;
    const int u = x - __builtin_amdgcn_readfirstlane(bounds.chunk[b]), cost = kTreeStart + n, grp = u / cost;
    // chunk i of the group is at origin + i
    const int origin = x - (u - grp * cost) + kTreeStart, c0 = max(x - origin, 0), c1 = min(n, end - origin);
    x = origin + n;
    if (c0 >= c1) continue;  // the run ends before its first chunk
    const int kvh = grp / blocks, row0 = (grp - kvh * blocks) * R, rows = min(R, t * G - row0);
    const const_ints table = (const_ints)(uintptr_t)(c.table + int64_t(b) * c.table_stride);

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
            const __bf16* base = (kv ? c.v : c.k) + int64_t(kvh) * D;
            const int64_t ps = kv ? c.v_page : c.k_page, ts = kv ? c.v_token : c.k_token;
            const uint32_t lane_row = uint32_t(lrow * ts);
#pragma unroll
            for (int j = 0; j < kInstr; ++j) {
              const int slot = (p0 + (j / kPer) * 8) & (page_rows - 1);
              const __bf16* src = base + ids.v[j / kPer] * ps + slot * ts + (j % kPer) * (RPI * ts);
              lds_dma_x4_off(uniform_u64(reinterpret_cast<uint64_t>(src)), (lane_row + chunk16[j % kKinds]) * 2,
                             la + kv * kTile + j * 1024);
            }
          }
          return ~0u;
        }
      }
      // the context's end, new tokens, or a page that is none: row by row. Keys that do not exist read a new token of
      // the sequence instead, a row that is there
      const int pos = p0 + (lane & 31);
      const int page = pos < ctx ? cache_page(c, b, pos) : -1;
      const uint32_t exist = uint32_t(__builtin_amdgcn_ballot_w64(page >= 0 || (pos >= ctx && pos - ctx < t)));
#pragma unroll 1
      for (int e = 0; e < 2 * kInstr; ++e) {  // K, then V: the waits below count on that order
        const int j = e % kInstr, r = j * RPI + lrow, p = p0 + r;
        const bool is_v = e >= kInstr;
        const int64_t id = __shfl(page, r, 64), slot = p & (page_rows - 1);
        const int64_t fresh = t0 + (p < ctx ? 0 : min(p - ctx, t - 1));
        const __bf16* src = id >= 0 ? (is_v ? c.v : c.k) + id * (is_v ? c.v_page : c.k_page) + slot * (is_v ? c.v_token : c.k_token)
                                    : (is_v ? a.v : a.k) + fresh * (is_v ? a.vs : a.ks);
        lds_dma_x4_at(src + kvh * D + ((lane % CPR) ^ swz<D>(r)) * 8, la + is_v * kTile + j * 1024);
      }
      return exist;
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
    uint64_t tree[NQ];  // which drafted tokens the lane's row sees (a chain: all up to itself; see below)
    int tok[NQ];
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      const int r = row0 + min(16 * qb + l16, rows - 1), token = r / G, h = kvh * G + r - token * G;
      tok[qb] = token;
      tree[qb] = a.tree ? a.tree[t0 + token] : 0;
      const __bf16* src = a.q + int64_t(t0 + token) * a.qs + int64_t(h) * D + g * 8;
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
        for (int qb = 0; qb < NQ; ++qb) {
          // bit e is position 32 i + e, new token e - to
          const int to = ctx - i * kTreeChunk;
          uint32_t draft;
          if (a.tree) {
            draft = to >= 32 ? 0 : to >= 0 ? uint32_t(tree[qb] << to) : to > -64 ? uint32_t(tree[qb] >> -to) : 0;
          } else {
            const int last = tok[qb] + to;
            draft = last >= 31 ? ~0u : last < 0 ? 0 : (2u << last) - 1;
          }
          const uint32_t cached = to >= 32 ? ~0u : to > 0 ? (1u << to) - 1 : 0;
          vis[qb] = exist[0] & (cached | draft);
        }
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
    st.settle();
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
    for (int e = threadIdx.x; e < rows * (D / 4); e += kTreeThreads) {
      const int r = e / (D / 4), q = e % (D / 4);
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
        const int rr = row0 + r, token = rr / G, h = kvh * G + rr - token * G;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (__bf16)(o[i] * inv);
        *reinterpret_cast<bf16x4*>(a.o + (int64_t(t0 + token) * a.heads + h) * D + 4 * q) = y;
        if (q == 0) a.lse[int64_t(h) * c.tokens + t0 + token] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      } else {
        *reinterpret_cast<floatx4*>(part + r * D + 4 * q) = o;
        if (q == 0) *reinterpret_cast<float2*>(part + R * D + 2 * r) = float2{m, l};
      }
    }
    if (!whole && c0 == 0)  // the group's first keys
      split = TreeSplit{(origin + n - 1) / run - w + 1, t0, row0, rows, kvh};
    __syncthreads();  // the rings and ml are free again
  }
  if (threadIdx.x == 0) a.split[w] = split;
}

// Groups of rows that several workgroups share, from their pieces, in key order: with M the largest of their maxima,
// O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i. D / 4 threads per row.
template <int D, int NQ>
__global__ void __launch_bounds__(kTreeThreads) sra_tree_combine_kernel(TreeArgs a) {
  constexpr int TPR = D / 4, RPB = kTreeThreads / TPR, R = 16 * NQ;
  constexpr int64_t kSlot = int64_t(R) * (D + 2);
  const int w = blockIdx.x;
  const TreeSplit sp = a.split[w];
  const int r = blockIdx.y * RPB + threadIdx.x / TPR, sub = threadIdx.x % TPR;
  if (sp.pieces == 0 || r >= sp.rows) return;
  auto piece = [&](int i) { return a.part + kSlot * (2 * (w + i) + (i == 0)); };
  float m = -INFINITY;
  for (int i = 0; i < sp.pieces; ++i) m = fmaxf(m, piece(i)[R * D + 2 * r]);
  floatx4 o = floatx4{};
  float l = 0.f;
  for (int i = 0; i < sp.pieces; ++i) {
    const float* p = piece(i);
    const float2 x = *reinterpret_cast<const float2*>(p + R * D + 2 * r);
    const float f = x.y == 0.f ? 0.f : fast_exp2(x.x - m);
    l += f * x.y;
    o += f * *reinterpret_cast<const floatx4*>(p + r * D + 4 * sub);
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
// cu_tokens[b] of b's pages. One wave per token; bound by the copy.
__global__ void __launch_bounds__(kTreeThreads) sra_append_kernel(AppendArgs a) {
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63;
  const int i = __builtin_amdgcn_readfirstlane(blockIdx.x * kTreeWaves + (threadIdx.x >> 6));
  if (i >= c.tokens) return;
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

template <int D, int NQ>
static void launch_tree_nq(const TreeArgs& a, hipStream_t stream) {
  constexpr int RPB = kTreeThreads / (D / 4);
  hipLaunchKernelGGL((sra_tree_kernel<D, NQ>), dim3(kTreeGroups), dim3(kTreeThreads), 0, stream, a);
  hipLaunchKernelGGL((sra_tree_combine_kernel<D, NQ>), dim3(kTreeGroups, (16 * NQ + RPB - 1) / RPB), dim3(kTreeThreads), 0,
                     stream, a);
}

hipError_t launch_tree(const TreeArgs& a, int nq, int head_dim, hipStream_t stream) {
  if (a.c.tokens <= 0) return hipSuccess;
  if (head_dim == 128) {
    if (nq == 1) launch_tree_nq<128, 1>(a, stream);
    else if (nq == 2) launch_tree_nq<128, 2>(a, stream);
    else launch_tree_nq<128, 4>(a, stream);
  } else {
    if (nq == 1) launch_tree_nq<64, 1>(a, stream);
    else if (nq == 2) launch_tree_nq<64, 2>(a, stream);
    else launch_tree_nq<64, 4>(a, stream);
  }
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
  if (a.c.tokens <= 0) return hipSuccess;
  const dim3 grid((a.c.tokens + kTreeWaves - 1) / kTreeWaves);
  hipLaunchKernelGGL(sra_append_kernel, grid, dim3(kTreeThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sra
