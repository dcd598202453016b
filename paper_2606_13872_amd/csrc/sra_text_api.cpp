// C ABI of causal attention over packed prompts and of the paged cache (include/sra.h): validation, plans, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <memory>
#include <new>
#include <string>

#include "sra.h"
#include "sra_causal_kernels.h"
#include "sra_internal.h"
#include "sra_tree.h"

struct sra_causal_plan {
  sra::CausalTables t;
  // tables in the device buffer: fwd | fwd_combine | grad | grad_combine
  size_t offset[4] = {0, 0, 0, 0};
  size_t table_bytes = 0, forward_workspace = 0, backward_workspace = 0, stat_bytes = 0, part_q_bytes = 0;
};

namespace {

using namespace sra;

constexpr size_t kAlign = 256;
constexpr int64_t kMaxInt = 2147483647;
constexpr int64_t kMaxStride = kMaxInt / 64;  // offsets inside a tile are 32-bit
// A launch has less than 2^32 threads: the delta kernel takes up to 16 for a (token, head) pair, the items 256 or 512
// each, the append 64 a token.
constexpr int64_t kMaxPairs = (int64_t(1) << 28) - 1;
constexpr int64_t kMaxItems = int64_t(1) << 22;
constexpr int32_t kMaxTokens = 1 << 25;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
sra_status fail(sra_status s, const std::string& msg) { return set_error(s, msg.c_str()); }
sra_status hip_fail(hipError_t e, const char* what) { return fail(SRA_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e)); }
bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

const std::vector<CausalItem>* lists(const CausalTables& t, int i) {
  const std::vector<CausalItem>* l[4] = {&t.fwd, &t.fwd_combine, &t.grad, &t.grad_combine};
  return l[i];
}

// Heads and head_dim of every call here.
sra_status check_heads(int32_t heads, int32_t kv_heads, int32_t head_dim) {
  if (heads < 1 || kv_heads < 1 || heads % kv_heads)
    return fail(SRA_ERR_INVALID_ARGUMENT, "num_heads must be a positive multiple of num_kv_heads");
  if (head_dim < 1) return fail(SRA_ERR_INVALID_ARGUMENT, "head_dim must be positive");
  if (head_dim != 64 && head_dim != 128) return fail(SRA_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  return SRA_OK;
}

// A token stride: 0 selects the dense one.
sra_status check_stride(int64_t* stride, int32_t heads, int32_t head_dim, const char* name) {
  const int64_t dense = int64_t(heads) * head_dim;
  if (*stride == 0) *stride = dense;
  if (*stride < dense || *stride % 8)
    return fail(SRA_ERR_INVALID_ARGUMENT, std::string(name) + " stride must be a multiple of 8 and at least heads * head_dim");
  if (*stride > kMaxStride) return fail(SRA_ERR_UNSUPPORTED, std::string(name) + " stride is too large");
  return SRA_OK;
}

sra_status check_pointers(std::initializer_list<const void*> ps) {
  for (const void* p : ps) {
    if (!p) return fail(SRA_ERR_INVALID_ARGUMENT, "a tensor pointer is NULL");
    if (misaligned(p, 16)) return fail(SRA_ERR_INVALID_ARGUMENT, "tensor pointers must be 16-byte aligned");
  }
  return SRA_OK;
}

sra_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (bytes < need) return fail(SRA_ERR_WORKSPACE_TOO_SMALL, "the call needs " + std::to_string(need) + " workspace bytes");
  if (need && (!ws || misaligned(ws, kAlign)))
    return fail(SRA_ERR_INVALID_ARGUMENT, "workspace must be non-NULL and 256-byte aligned");
  return SRA_OK;
}

float scale_of(float scale, int32_t head_dim) {
  return scale > 0 ? scale : float(1.0 / __builtin_sqrt(double(head_dim)));
}

// Checks of a causal call before anything is enqueued, and the arguments both directions share.
sra_status causal_args(const sra_causal_plan* plan, const void* tables, const void* q, const void* k, const void* v,
                       int64_t q_stride, int64_t k_stride, int64_t v_stride, float scale, CausalArgs* a) {
  if (!plan) return fail(SRA_ERR_INVALID_ARGUMENT, "plan is NULL");
  const CausalTables& t = plan->t;
  sra_status st = check_stride(&q_stride, t.heads, t.head_dim, "q");
  if (st == SRA_OK) st = check_stride(&k_stride, t.kv_heads, t.head_dim, "k");
  if (st == SRA_OK) st = check_stride(&v_stride, t.kv_heads, t.head_dim, "v");
  if (st != SRA_OK) return st;
  if (!(scale == scale) || scale > 3.0e38f) return fail(SRA_ERR_INVALID_ARGUMENT, "softmax_scale must be finite");
  if (t.q_rows && (st = check_pointers({q})) != SRA_OK) return st;
  if (t.k_rows && (st = check_pointers({k, v})) != SRA_OK) return st;
  if (plan->table_bytes && (!tables || misaligned(tables, 16)))
    return fail(SRA_ERR_INVALID_ARGUMENT, "tables must be non-NULL and 16-byte aligned");
  a->q = static_cast<const __bf16*>(q);
  a->k = static_cast<const __bf16*>(k);
  a->v = static_cast<const __bf16*>(v);
  a->qs = q_stride;
  a->ks = k_stride;
  a->vs = v_stride;
  a->q_rows = int32_t(t.q_rows);
  a->heads = t.heads;
  a->kv_heads = t.kv_heads;
  a->scale = scale_of(scale, t.head_dim);
  a->scale_log2 = float(double(a->scale) * 1.4426950408889634);
  return SRA_OK;
}

const CausalItem* table(const sra_causal_plan* p, const void* tables, int i) {
  return reinterpret_cast<const CausalItem*>(static_cast<const char*>(tables) + p->offset[i]);
}

// Checks of a paged cache (pointers == false: of its sizes alone) and the kernels' view of it.
sra_status check_cache(const sra_paged_cache* c, bool pointers, bool tensors, PagedCache* out) {
  if (!c) return fail(SRA_ERR_INVALID_ARGUMENT, "cache is NULL");
  sra_status st = check_heads(c->num_kv_heads, c->num_kv_heads, c->head_dim);
  if (st != SRA_OK) return st;
  if (c->batch < 1 || c->tokens < 0 || c->num_pages < 1 || c->max_pages < 1)
    return fail(SRA_ERR_INVALID_ARGUMENT, "batch, num_pages and max_pages must be positive, tokens not negative");
  if (c->batch > kTreeMaxBatch) return fail(SRA_ERR_UNSUPPORTED, "batch must be at most " + std::to_string(kTreeMaxBatch));
  if (c->page_size < 8 || (c->page_size & (c->page_size - 1)))
    return fail(SRA_ERR_INVALID_ARGUMENT, "page_size must be a power of two of at least 8");
  if (int64_t(c->max_pages) * c->page_size > (int64_t(1) << 30))
    return fail(SRA_ERR_UNSUPPORTED, "max_pages * page_size must be at most 2^30");
  if (c->tokens > kMaxTokens) return fail(SRA_ERR_UNSUPPORTED, "tokens must be at most " + std::to_string(kMaxTokens));
  if (int64_t(c->tokens) * c->num_kv_heads > kMaxInt) return fail(SRA_ERR_UNSUPPORTED, "heads * tokens must be below 2^31");
  out->k = static_cast<__bf16*>(c->k);
  out->v = static_cast<__bf16*>(c->v);
  out->k_token = c->k_token_stride;
  out->v_token = c->v_token_stride;
  if ((st = check_stride(&out->k_token, c->num_kv_heads, c->head_dim, "k token")) != SRA_OK) return st;
  if ((st = check_stride(&out->v_token, c->num_kv_heads, c->head_dim, "v token")) != SRA_OK) return st;
  out->k_page = c->k_page_stride ? c->k_page_stride : out->k_token * c->page_size;
  out->v_page = c->v_page_stride ? c->v_page_stride : out->v_token * c->page_size;
  const int64_t row = int64_t(c->num_kv_heads) * c->head_dim;
  if (out->k_page < out->k_token * (c->page_size - 1) + row || out->v_page < out->v_token * (c->page_size - 1) + row ||
      out->k_page % 8 || out->v_page % 8)
    return fail(SRA_ERR_INVALID_ARGUMENT, "page strides must be multiples of 8 and hold a page");
  if (out->k_page >= (int64_t(1) << 35) || out->v_page >= (int64_t(1) << 35))
    return fail(SRA_ERR_UNSUPPORTED, "a page stride is too large");
  out->table_stride = c->table_stride ? c->table_stride : c->max_pages;
  if (out->table_stride < c->max_pages) return fail(SRA_ERR_INVALID_ARGUMENT, "table_stride must be at least max_pages");
  out->table = c->page_table;
  out->context_lens = c->context_lens;
  out->cu_tokens = c->cu_tokens;
  if (pointers && (!c->page_table || !c->context_lens || !c->cu_tokens || misaligned(c->page_table, 4) ||
                   misaligned(c->context_lens, 4) || misaligned(c->cu_tokens, 4)))
    return fail(SRA_ERR_INVALID_ARGUMENT, "page_table, context_lens and cu_tokens must be given, 4-byte aligned");
  if (tensors && (st = check_pointers({c->k, c->v})) != SRA_OK) return st;
  out->batch = c->batch;
  out->tokens = c->tokens;
  out->pages = c->num_pages;
  out->page_shift = __builtin_ctz(uint32_t(c->page_size));
  out->max_pages = c->max_pages;
  out->kv_heads = c->num_kv_heads;
  return SRA_OK;
}

// Rows per group of rows: as many as a sequence's (token, head of the group) rows fill on average (the host knows no more).
// More would leave the matrix instructions' columns empty, fewer read K and V once for each of several groups. 16 rows a
// sequence in groups of 16 take 16.5 us (16 requests of 300 positions), in groups of 32 19.7, shared 19.7; 32 rows in
// groups of 32 366 us (64 of 8,000), shared 380; 40 rows, 16 of 8,000: 119 us shared.
// Uneven steps pay for going by the average: 128 single tokens (500 to 8,000 positions) with a chain of 256 tokens over
// 8,000 take 421 us, by themselves 311 and 61; 64 with a chain of 512 238 us, by themselves 160 and 104. Padding rows count
// as rows: 64 single tokens 162 us, among 448 padding rows 158 (shared), among 960 172.
int tree_rows(const sra_paged_cache& c, int32_t heads) {
  const int64_t rows = (int64_t(c.tokens) + c.batch - 1) / c.batch * (heads / c.num_kv_heads);
  return rows <= 16 ? 16 : rows <= 32 ? 32 : kTreeShared;
}

size_t tree_slots_bytes(int rows, int32_t head_dim) {
  return align_up(size_t(2) * kTreeGroups * rows * (head_dim + 2) * 4);
}

sra_status check_tree(const sra_paged_cache* c, int32_t num_heads, bool pointers, PagedCache* out, size_t* bytes) {
  sra_status st = check_cache(c, pointers, pointers, out);
  if (st != SRA_OK) return st;
  if ((st = check_heads(num_heads, c->num_kv_heads, c->head_dim)) != SRA_OK) return st;
  if (int64_t(c->tokens) * num_heads > kMaxInt) return fail(SRA_ERR_UNSUPPORTED, "heads * tokens must be below 2^31");
  if (num_heads / c->num_kv_heads > kTreeMaxGroup)
    return fail(SRA_ERR_UNSUPPORTED, "at most " + std::to_string(kTreeMaxGroup) + " query heads per K/V head");
  const int rows = tree_rows(*c, num_heads);
  // the launch's cost is counted in 32 bits
  const int64_t chunks = int64_t(c->max_pages) * c->page_size / kTreeChunk + c->tokens / kTreeChunk + 2;
  const int64_t cost = rows < kTreeShared ? kTreeStart + chunks : kSharedStart + kSharedWide * (chunks / 2 + 1);
  const int64_t groups = c->batch + int64_t(c->tokens) * (num_heads / c->num_kv_heads) / std::min(rows, kTreeShared / 2);
  if (double(cost) * double(groups) * c->num_kv_heads > double(kMaxInt))
    return fail(SRA_ERR_UNSUPPORTED, "the tokens times the cache's reach are too many for one call");
  *bytes = tree_slots_bytes(rows, c->head_dim) + align_up(kTreeGroups * sizeof(TreeSplit));
  return SRA_OK;
}

}  // namespace

extern "C" {

sra_status sra_causal_plan_create(const sra_causal_problem* p, int backward, sra_causal_plan** plan) {
  set_error(SRA_OK, "");
  if (!p || !plan) return fail(SRA_ERR_INVALID_ARGUMENT, "problem or plan is NULL");
  *plan = nullptr;
  sra_status st = check_heads(p->num_heads, p->num_kv_heads, p->head_dim);
  if (st != SRA_OK) return st;
  if (p->batch < 1 || !p->q_lens) return fail(SRA_ERR_INVALID_ARGUMENT, "batch must be positive and q_lens given");
  try {
    std::unique_ptr<sra_causal_plan> c(new sra_causal_plan);
    CausalTables& t = c->t;
    t.batch = p->batch;
    t.heads = p->num_heads;
    t.kv_heads = p->num_kv_heads;
    t.head_dim = p->head_dim;
    t.backward = backward != 0;
    if (int64_t(t.heads) * t.head_dim > kMaxStride) return fail(SRA_ERR_UNSUPPORTED, "too many heads");
    const int32_t* k_lens = p->k_lens ? p->k_lens : p->q_lens;
    for (int32_t b = 0; b < p->batch; ++b)
      if (p->q_lens[b] < 0 || k_lens[b] < 0) return fail(SRA_ERR_INVALID_ARGUMENT, "lengths must not be negative");
    const int64_t G = t.heads / t.kv_heads;
    int64_t q_items = 0, k_items = 0;
    for (int32_t b = 0; b < p->batch; ++b) {
      t.nq.push_back(p->q_lens[b]);
      t.nk.push_back(k_lens[b]);
      t.q_rows += p->q_lens[b];
      t.k_rows += k_lens[b];
      if (t.q_rows * t.heads > kMaxPairs || t.k_rows * t.kv_heads > kMaxPairs)
        return fail(SRA_ERR_UNSUPPORTED, "heads * packed tokens must be below 2^28");
      q_items += (p->q_lens[b] * G + kCausalTile - 1) / kCausalTile * t.kv_heads;
      k_items += (int64_t(k_lens[b]) + kCausalTile - 1) / kCausalTile * t.kv_heads;
      if (q_items > kMaxItems || k_items > kMaxItems) return fail(SRA_ERR_UNSUPPORTED, "too many sequences times K/V heads");
    }
    build_causal_tables(&t);
    size_t at = 0;
    for (int i = 0; i < 4; ++i) {
      c->offset[i] = at;
      at += align_up(lists(t, i)->size() * sizeof(CausalItem));
    }
    c->table_bytes = at;
    c->forward_workspace = align_up(size_t(t.fwd_slots) * kCausalTile * (t.head_dim + 2) * 4);
    if (t.backward) {
      c->stat_bytes = align_up(size_t(t.heads) * t.q_rows * 4);
      c->part_q_bytes = align_up(size_t(t.q_slots) * kCausalTile * t.head_dim * 4);
      c->backward_workspace = 2 * c->stat_bytes + c->part_q_bytes +
                              align_up(size_t(t.kv_slots) * 2 * kCausalTile * t.head_dim * 4);
    }
    *plan = c.release();
  } catch (const std::bad_alloc&) {
    return fail(SRA_ERR_INTERNAL, "out of host memory");
  } catch (...) {
    return fail(SRA_ERR_INTERNAL, "planning failed");
  }
  return SRA_OK;
}

sra_status sra_causal_plan_destroy(sra_causal_plan* plan) {
  set_error(SRA_OK, "");
  delete plan;
  return SRA_OK;
}

sra_status sra_causal_plan_sizes(const sra_causal_plan* plan, size_t* table_bytes, size_t* forward_workspace,
                                 size_t* backward_workspace) {
  set_error(SRA_OK, "");
  if (!plan) return fail(SRA_ERR_INVALID_ARGUMENT, "plan is NULL");
  if (table_bytes) *table_bytes = plan->table_bytes;
  if (forward_workspace) *forward_workspace = plan->forward_workspace;
  if (backward_workspace) *backward_workspace = plan->backward_workspace;
  return SRA_OK;
}

sra_status sra_causal_plan_tables(const sra_causal_plan* plan, void* host, size_t bytes) {
  set_error(SRA_OK, "");
  if (!plan || (!host && plan->table_bytes)) return fail(SRA_ERR_INVALID_ARGUMENT, "plan or host buffer is NULL");
  if (bytes < plan->table_bytes) return fail(SRA_ERR_INVALID_ARGUMENT, "the host buffer is smaller than the tables");
  if (plan->table_bytes) std::memset(host, 0, plan->table_bytes);
  for (int i = 0; i < 4; ++i) {
    const std::vector<CausalItem>& l = *lists(plan->t, i);
    if (!l.empty()) std::memcpy(static_cast<char*>(host) + plan->offset[i], l.data(), l.size() * sizeof(CausalItem));
  }
  return SRA_OK;
}

sra_status sra_causal_plan_mask(const sra_causal_plan* plan, int which, int32_t sequence, int32_t head, uint8_t* out) {
  set_error(SRA_OK, "");
  if (!plan || !out) return fail(SRA_ERR_INVALID_ARGUMENT, "plan or out is NULL");
  const CausalTables& t = plan->t;
  if (which != SRA_SCHED_FORWARD && which != SRA_SCHED_BWD_DQ && which != SRA_SCHED_BWD_DKDV)
    return fail(SRA_ERR_INVALID_ARGUMENT, "unknown schedule");
  if (sequence < 0 || sequence >= t.batch || head < 0 || head >= t.heads)
    return fail(SRA_ERR_INVALID_ARGUMENT, "sequence or head out of range");
  if (which != SRA_SCHED_FORWARD && !t.backward) return fail(SRA_ERR_INVALID_ARGUMENT, "the plan has no backward");
  const int32_t G = t.heads / t.kv_heads, kvh = head / G, hg = head % G, nq = t.nq[sequence], nk = t.nk[sequence];
  const CausalKind kind = which == SRA_SCHED_FORWARD ? kForward : which == SRA_SCHED_BWD_DQ ? kDq : kDkv;
  std::memset(out, 0, size_t(nq) * nk);
  for (const CausalItem& it : which == SRA_SCHED_FORWARD ? t.fwd : t.grad) {
    if (it.kind != kind || it.seq != sequence || it.kvh != kvh) continue;
    if (kind != kDkv) {
      for (int32_t r = it.start; r < it.start + it.len; ++r) {
        if (r % G != hg) continue;
        const int32_t i = r / G;
        for (int32_t j = it.lo; j < it.hi && j <= i + nk - nq; ++j) out[size_t(i) * nk + j]++;
      }
    } else {
      const CausalTiles tiles = causal_tiles(it);
      for (int32_t x = it.lo; x < it.hi; ++x) {
        const CausalTile c = causal_tile(tiles, G, x);
        if (c.hg != hg) continue;
        const int32_t first = c.tok;
        const bool masked = first + nk - nq < it.start + it.len - 1;
        if (masked != (x >= G * (tiles.n - tiles.d))) return fail(SRA_ERR_INTERNAL, "a tile of the wrong kind");
        for (int32_t i = first; i < std::min(first + 64, nq); ++i)
          for (int32_t j = it.start; j < it.start + it.len && j <= i + nk - nq; ++j) out[size_t(i) * nk + j]++;
      }
    }
  }
  return SRA_OK;
}

sra_status sra_causal_forward(const sra_causal_plan* plan, const void* tables, const void* q, const void* k,
                              const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride, void* o,
                              float* lse, float softmax_scale, void* workspace, size_t workspace_bytes,
                              void* stream) {
  set_error(SRA_OK, "");
  CausalArgs a{};
  sra_status st = causal_args(plan, tables, q, k, v, q_stride, k_stride, v_stride, softmax_scale, &a);
  if (st != SRA_OK) return st;
  const CausalTables& t = plan->t;
  if (t.q_rows && (st = check_pointers({o, lse})) != SRA_OK) return st;
  st = check_workspace(workspace, workspace_bytes, plan->forward_workspace);
  if (st != SRA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  a.items = table(plan, tables, 0);
  a.o = static_cast<__bf16*>(o);
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  const hipError_t e = timed_launch(SRA_KERNEL_CAUSAL_FORWARD, s, [&] {
    const hipError_t x = launch_causal_forward(a, int(t.fwd.size()), t.head_dim, t.fwd_tile, s);
    if (x != hipSuccess) return x;
    return launch_causal_forward_combine(a, table(plan, tables, 1), int(t.fwd_combine.size()), t.head_dim, s);
  });
  return e == hipSuccess ? SRA_OK : hip_fail(e, "causal forward launch");
}

sra_status sra_causal_backward(const sra_causal_plan* plan, const void* tables, const void* q, const void* k,
                               const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                               const void* o, const float* lse, const void* dout, void* dq, void* dk, void* dv,
                               float softmax_scale, void* workspace, size_t workspace_bytes, void* stream) {
  set_error(SRA_OK, "");
  CausalArgs a{};
  sra_status st = causal_args(plan, tables, q, k, v, q_stride, k_stride, v_stride, softmax_scale, &a);
  if (st != SRA_OK) return st;
  const CausalTables& t = plan->t;
  if (!t.backward) return fail(SRA_ERR_INVALID_ARGUMENT, "the plan was made without the backward");
  if (t.q_rows && (st = check_pointers({o, lse, dout, dq})) != SRA_OK) return st;
  if (t.k_rows && (st = check_pointers({dk, dv})) != SRA_OK) return st;
  st = check_workspace(workspace, workspace_bytes, plan->backward_workspace);
  if (st != SRA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  CausalDeltaArgs d{};
  d.o = static_cast<const __bf16*>(o);
  d.dout = static_cast<const __bf16*>(dout);
  d.lse = lse;
  d.lse2 = reinterpret_cast<float*>(ws);
  d.ndelta = reinterpret_cast<float*>(ws + plan->stat_bytes);
  d.q_rows = a.q_rows;
  d.heads = a.heads;
  hipError_t e = timed_launch(SRA_KERNEL_CAUSAL_DELTA, s, [&] { return launch_causal_delta(d, t.head_dim, s); });
  if (e != hipSuccess) return hip_fail(e, "causal delta launch");
  a.items = table(plan, tables, 2);
  a.dout = d.dout;
  a.lse2 = d.lse2;
  a.ndelta = d.ndelta;
  a.dq = static_cast<__bf16*>(dq);
  a.dk = static_cast<__bf16*>(dk);
  a.dv = static_cast<__bf16*>(dv);
  a.part_q = reinterpret_cast<float*>(ws + 2 * plan->stat_bytes);
  a.part_kv = reinterpret_cast<float*>(ws + 2 * plan->stat_bytes + plan->part_q_bytes);
  e = timed_launch(SRA_KERNEL_CAUSAL_GRAD, s, [&] {
    const hipError_t x = launch_causal_grad(a, int(t.grad.size()), t.head_dim, s);
    if (x != hipSuccess) return x;
    return launch_causal_grad_combine(a, table(plan, tables, 3), int(t.grad_combine.size()), t.head_dim, s);
  });
  return e == hipSuccess ? SRA_OK : hip_fail(e, "causal gradient launch");
}

sra_status sra_tree_workspace_size(const sra_paged_cache* c, int32_t num_heads, size_t* bytes) {
  set_error(SRA_OK, "");
  if (!bytes) return fail(SRA_ERR_INVALID_ARGUMENT, "bytes is NULL");
  PagedCache view{};
  return check_tree(c, num_heads, false, &view, bytes);
}

sra_status sra_tree_attention(const sra_paged_cache* c, int32_t num_heads, const void* q, const void* k,
                              const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                              const uint64_t* tree, void* o, float* lse, float softmax_scale, void* workspace,
                              size_t workspace_bytes, void* stream) {
  set_error(SRA_OK, "");
  TreeArgs a{};
  size_t need = 0;
  sra_status st = check_tree(c, num_heads, true, &a.c, &need);
  if (st != SRA_OK) return st;
  if ((st = check_stride(&q_stride, num_heads, c->head_dim, "q")) != SRA_OK) return st;
  if ((st = check_stride(&k_stride, c->num_kv_heads, c->head_dim, "k")) != SRA_OK) return st;
  if ((st = check_stride(&v_stride, c->num_kv_heads, c->head_dim, "v")) != SRA_OK) return st;
  if (!(softmax_scale == softmax_scale) || softmax_scale > 3.0e38f)
    return fail(SRA_ERR_INVALID_ARGUMENT, "softmax_scale must be finite");
  if (c->tokens == 0) return SRA_OK;
  if ((st = check_pointers({q, k, v, o, lse})) != SRA_OK) return st;
  if (misaligned(tree, 8)) return fail(SRA_ERR_INVALID_ARGUMENT, "tree must be 8-byte aligned");
  if ((st = check_workspace(workspace, workspace_bytes, need)) != SRA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int rows = tree_rows(*c, num_heads);
  a.q = static_cast<const __bf16*>(q);
  a.k = static_cast<const __bf16*>(k);
  a.v = static_cast<const __bf16*>(v);
  a.qs = q_stride;
  a.ks = k_stride;
  a.vs = v_stride;
  a.tree = tree;
  a.o = static_cast<__bf16*>(o);
  a.lse = lse;
  a.heads = num_heads;
  const uint32_t G = uint32_t(num_heads / c->num_kv_heads);
  a.group_magic = G > 1 ? uint32_t((uint64_t(1) << 32) / G + 1) : 0;
  a.k_step = {uint32_t(a.c.k_page / 8), uint32_t(a.c.k_token / 8)};
  a.v_step = {uint32_t(a.c.v_page / 8), uint32_t(a.c.v_token / 8)};
  a.scale_log2 = float(double(scale_of(softmax_scale, c->head_dim)) * 1.4426950408889634);
  a.part = static_cast<float*>(workspace);
  a.split = reinterpret_cast<TreeSplit*>(static_cast<char*>(workspace) + tree_slots_bytes(rows, c->head_dim));
  const hipError_t e = timed_launch(SRA_KERNEL_TREE, s, [&] { return launch_tree(a, rows, c->head_dim, s); });
  return e == hipSuccess ? SRA_OK : hip_fail(e, "tree attention launch");
}

sra_status sra_cache_append(const sra_paged_cache* c, const void* k, const void* v, int64_t k_stride,
                            int64_t v_stride, const int32_t* rows, int32_t n_rows, void* stream) {
  set_error(SRA_OK, "");
  AppendArgs a{};
  sra_status st = check_cache(c, true, true, &a.c);
  if (st != SRA_OK) return st;
  if ((st = check_stride(&k_stride, c->num_kv_heads, c->head_dim, "k")) != SRA_OK) return st;
  if ((st = check_stride(&v_stride, c->num_kv_heads, c->head_dim, "v")) != SRA_OK) return st;
  if (n_rows < 0 || (!rows && n_rows != c->tokens))
    return fail(SRA_ERR_INVALID_ARGUMENT, "without rows, k and v must have one row per token");
  if (misaligned(rows, 4)) return fail(SRA_ERR_INVALID_ARGUMENT, "rows must be 4-byte aligned");
  if (c->tokens == 0 || n_rows == 0) return SRA_OK;
  if ((st = check_pointers({k, v})) != SRA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  a.k = static_cast<const __bf16*>(k);
  a.v = static_cast<const __bf16*>(v);
  a.ks = k_stride;
  a.vs = v_stride;
  a.rows = rows;
  a.n_rows = n_rows;
  a.row_elems = c->num_kv_heads * c->head_dim;
  const hipError_t e = timed_launch(SRA_KERNEL_APPEND, s, [&] { return launch_append(a, s); });
  return e == hipSuccess ? SRA_OK : hip_fail(e, "cache append launch");
}

sra_status sra_cache_rows(const sra_paged_cache* c, int64_t* append_rows, int32_t sequence, int64_t* context_rows) {
  set_error(SRA_OK, "");
  PagedCache p{};
  sra_status st = check_cache(c, true, false, &p);
  if (st != SRA_OK) return st;
  if (context_rows && (sequence < 0 || sequence >= p.batch)) return fail(SRA_ERR_INVALID_ARGUMENT, "sequence out of range");
  auto cache_row = [&](int32_t b, int64_t pos) -> int64_t {
    const int64_t id = pos < 0 ? -1 : cache_page(p, b, pos);
    return id < 0 ? -1 : (id << p.page_shift) + (pos & (c->page_size - 1));
  };
  if (append_rows)
    for (int32_t i = 0; i < p.tokens; ++i) {
      int32_t b = 0;
      while (b < p.batch && p.cu_tokens[b + 1] <= i) ++b;
      append_rows[i] = b < p.batch ? cache_row(b, append_position(p, b, i)) : -1;
    }
  if (context_rows)
    for (int64_t pos = 0; pos < int64_t(p.max_pages) << p.page_shift; ++pos)
      context_rows[pos] = pos < cache_context(p, sequence) ? cache_row(sequence, pos) : -1;
  return SRA_OK;
}

}  // extern "C"
