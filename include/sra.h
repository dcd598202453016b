/*
 * sra.h — C ABI of libsra: Sparse Reference Attention (SRA) on AMD Instinct MI355X (gfx950).
 *
 * SRA is the asymmetric attention of Avatar V (§1 contributions; §2.1 "Sparse Reference
 * Attention"; §4.3 reference KV caching and invalid-token skipping; §8 related work):
 *   - every generation (gen) query attends to all gen keys of its sample and to every valid
 *     reference (ref) key of its sample, through ONE softmax over the concatenated key set
 *     (§4.3 concatenates the cached reference K/V with the generation K/V);
 *   - every ref query attends only to the ref keys of its own self-attention group, never to
 *     gen keys (§1, §8.2: the reference side attends only within itself). A group is `group_frames`
 *     consecutive reference latent frames; group_frames = 1 keeps the cost linear in the
 *     reference length (§1, §2.1);
 *   - tokens of invalid reference frames (§4.3, e.g. frames where the face is not visible),
 *     and single reference tokens marked invalid, are neither keys nor queries: their
 *     outputs are 0, their log-sum-exp is -inf and their gradients are 0.
 * Samples of a packed (varlen) batch never see each other.
 *
 * Conventions shared by every entry point
 *   Tensors   bf16 tensors are [tokens, heads, head_dim] with head stride head_dim and element
 *             stride 1. Tokens of all samples are packed back to back in sample order, and
 *             frame-major (frame, row, column) inside a sample. q/k/v of a stream use that
 *             stream's token stride (elements between consecutive tokens, >= heads*head_dim,
 *             so q/k/v packed into one buffer work); o, do, dq, dk, dv are dense
 *             (token stride heads*head_dim). lse tensors are fp32 [heads, tokens], natural log.
 *   Memory    every data pointer and the workspace are DEVICE pointers owned by the caller.
 *             The library allocates no device memory. It owns pinned host staging buffers for
 *             its cached schedules (reused across plans, freed by sra_release_caches or at
 *             process exit); a geometry not seen before costs one host planning pass and, when
 *             no staging buffer is free, one hipHostMalloc (the cache holds 256 plans).
 *   Streams   `stream` is a hipStream_t (NULL = the default stream). Calls only enqueue work
 *             on it and never synchronise the device.
 *   Errors    every argument is validated before anything is enqueued, so a call that
 *             returns an error has written nothing. sra_last_error() gives a per-thread
 *             message. No C++ exception crosses this boundary. All functions are thread safe.
 *   Supported head_dim in {64, 128}; heads >= 1; batch >= 1; every sample has >= 1 gen token.
 *   Limits    packed tokens of each stream <= 2^31 - 1 (beyond: SRA_ERR_INVALID_ARGUMENT);
 *             num_heads * packed tokens of each stream <= 2^31 - 1 (beyond: SRA_ERR_UNSUPPORTED;
 *             per-row statistics are indexed in 32 bits); token strides <= (2^31 - 1) / 64
 *             elements (beyond: SRA_ERR_UNSUPPORTED; offsets inside a tile are 32-bit). Tensors
 *             themselves may exceed 2^31 elements: token offsets are 64-bit.
 */
#ifndef SRA_H_
#define SRA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum sra_status {
  SRA_OK = 0,
  SRA_ERR_INVALID_ARGUMENT = 1,     /* bad geometry, null pointer, stride, flag, ...           */
  SRA_ERR_UNSUPPORTED = 2,          /* valid request the library does not implement (head_dim) */
  SRA_ERR_WORKSPACE_TOO_SMALL = 3,  /* workspace_bytes below sra_workspace_size()              */
  SRA_ERR_HIP = 4,                  /* the HIP runtime reported an error while enqueuing       */
  SRA_ERR_INTERNAL = 5              /* host allocation failure or internal inconsistency       */
} sra_status;

/* Geometry of one sample (host memory). Gen tokens G = gen_frames*gen_h*gen_w (>= 1);
 * ref tokens R = ref_frames*ref_h*ref_w (>= 0); F = ref_h*ref_w tokens per ref frame. */
typedef struct sra_sample_geom {
  int32_t gen_frames, gen_h, gen_w;
  int32_t ref_frames, ref_h, ref_w;
  int32_t group_frames;              /* >= 1: ref frames per ref self-attention group          */
  int32_t gen_window;                /* with SRA_FLAG_GEN_WINDOW: >= 0, see below; else ignored */
  const uint8_t* ref_frame_valid;    /* host, ref_frames bytes (0 = invalid); NULL = all valid */
  const uint8_t* ref_token_valid;    /* host, R bytes, frame-major (0 = invalid token); NULL =
                                        every token of a valid frame. A ref token takes part iff
                                        its frame and its own entry are valid (§4.3 invalid
                                        tokens); invalid tokens are treated like tokens of
                                        invalid frames. */
} sra_sample_geom;

typedef struct sra_problem {
  int32_t batch;                     /* samples in the packed batch, >= 1                      */
  int32_t num_heads;                 /* H >= 1 (same for Q, K and V)                           */
  int32_t head_dim;                  /* d in {64, 128}                                         */
  float softmax_scale;               /* <= 0 selects 1/sqrt(head_dim)                          */
  const sra_sample_geom* samples;    /* host array [batch]                                     */
  int64_t gen_token_stride;          /* elements between gen q/k/v tokens; 0 selects H*d       */
  int64_t ref_token_stride;          /* elements between ref q/k/v tokens; 0 selects H*d       */
  uint32_t flags;                    /* 0 or SRA_FLAG_* bits                                   */
} sra_problem;

/* Problem flags.
 * SRA_FLAG_GEN_QUERIES_ONLY: reference tokens are context only, not queries. This is the
 *   inference path of cached reference K/V (§4.3): across denoising steps the reference
 *   tokens' own outputs do not change, so only the generation rows are computed. The
 *   forward writes o_gen and lse_gen only; q_ref, o_ref and lse_ref are not read or written
 *   and may be NULL. The backward is that of the gen rows alone (equivalently: do_ref = 0):
 *   it writes dq_gen, dk_gen, dv_gen, dk_ref and dv_ref; q_ref, o_ref, lse_ref, do_ref and
 *   dq_ref are not touched and may be NULL. Pair counts and schedules omit the ref queries.
 * SRA_FLAG_GEN_WINDOW: temporal window on generation-to-generation attention, the sparse
 *   temporal attention of the super-resolution refiner (§2.4, which restricts each frame's
 *   receptive field to a local neighbourhood of frames and gives no width): a gen query in
 *   gen latent frame t sees the gen keys of frames t' with |t - t'| <= gen_window of its
 *   sample, and still every valid reference key. Reference queries are unchanged. */
enum { SRA_FLAG_GEN_QUERIES_ONLY = 1u, SRA_FLAG_GEN_WINDOW = 2u };

/* Which schedule an inspection hook looks at. */
enum {
  SRA_SCHED_FORWARD = 0,   /* query tiles -> key spans (forward pass)                 */
  SRA_SCHED_BWD_DQ = 1,    /* query tiles -> key spans (dQ kernel of the backward)    */
  SRA_SCHED_BWD_DKDV = 2   /* key tiles -> query spans (dK/dV kernel of the backward) */
};

/* Bytes of device workspace sra_forward (backward = 0) or sra_backward (backward = 1) needs
 * for problem `p`. Writes *bytes; host only, enqueues nothing. */
sra_status sra_workspace_size(const sra_problem* p, int backward, size_t* bytes);

/* Forward pass of SRA (the definition at the top of this file).
 * In : q_gen, k_gen, v_gen  bf16 [sumG, H, d] (gen token stride);
 *      q_ref, k_ref, v_ref  bf16 [sumR, H, d] (ref token stride); may be NULL when sumR = 0.
 * Out: o_gen bf16 [sumG, H, d], o_ref bf16 [sumR, H, d] (dense);
 *      lse_gen fp32 [H, sumG], lse_ref fp32 [H, sumR]: natural-log log-sum-exp of the scaled
 *      logits of each query row (-inf for rows of invalid frames).
 * Results are deterministic: every sum's order is fixed by the problem. It follows the launch, and so
 * the whole batch and all heads: a sample or head computed in another batch may differ by rounding.
 * workspace: device buffer of at least sra_workspace_size(p, 0) bytes, 256-byte aligned; its
 * contents are scratch and need no initialisation. Every output element is written. */
sra_status sra_forward(const sra_problem* p,
                       const void* q_gen, const void* k_gen, const void* v_gen,
                       const void* q_ref, const void* k_ref, const void* v_ref,
                       void* o_gen, void* o_ref, float* lse_gen, float* lse_ref,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Backward pass (§3.3: personality SFT trains the model with Sparse Reference Attention in the
 * loop, so the method needs the gradient of the attention of the top of this file; it is the
 * gradient of masked softmax attention, which the paper does not spell out).
 * Gradients of the forward outputs o_gen/o_ref with respect to every input,
 * given the upstream gradients do_gen/do_ref (bf16, dense, same shapes as o) and the forward's
 * o and lse (as sra_forward wrote them). Writes dq/dk/dv for both streams (bf16, dense,
 * same shapes as q/k/v); it overwrites them and does not accumulate. Gradients of tokens of
 * invalid frames are 0. Internally: D = rowsum(dO * O) in fp32, then the dK/dV and dQ
 * products of the softmax gradient with fp32 accumulation.
 * workspace: at least sra_workspace_size(p, 1) bytes, 256-byte aligned, no initialisation. */
sra_status sra_backward(const sra_problem* p,
                        const void* q_gen, const void* k_gen, const void* v_gen,
                        const void* q_ref, const void* k_ref, const void* v_ref,
                        const void* o_gen, const void* o_ref,
                        const float* lse_gen, const float* lse_ref,
                        const void* do_gen, const void* do_ref,
                        void* dq_gen, void* dk_gen, void* dv_gen,
                        void* dq_ref, void* dk_ref, void* dv_ref,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---- allocation-free forward ------------------------------------------------------------ */

/* Size in bytes of the library's static device scratch array, the workspace of
 * sra_forward_noalloc (one array per device, held from the first such call on that device until
 * the process ends). */
#define SRA_NOALLOC_WORKSPACE_MAX (32u << 20)

/* For callers that cannot allocate device memory (code under stream capture, tight serving
 * loops, harnesses that forbid hipMalloc): sra_forward with the workspace taken from the
 * library's static scratch array on the current device instead of a caller buffer. Same
 * kernels, so results are bitwise those of sra_forward.
 * In/out tensors, stream and validation as sra_forward; `stream` must belong to the current
 * device (else SRA_ERR_INVALID_ARGUMENT). A problem whose workspace (sra_workspace_size with
 * backward = 0) exceeds SRA_NOALLOC_WORKSPACE_MAX is rejected with SRA_ERR_WORKSPACE_TOO_SMALL
 * before anything is enqueued: in practice every problem whose token masks do not force the
 * compacted reference stream fits (the 720p layer needs 0.5 MB).
 * Allocates no device memory and no pinned host memory (no hipMalloc, hipHostMalloc or
 * hipFree): the schedule tables are copied from the plan's host image, and not at all when the
 * previous sra_forward_noalloc call on this device used the same geometry and stream (the
 * array keeps the last call's tables). A geometry not seen before is planned in host heap
 * memory, as for every entry point.
 * All calls on one device share one array: calls that overlap on a device (different streams
 * or threads without ordering between them) race and may read each other's tables. The first
 * call on a device loads the array there (a one-time cost of milliseconds). */
sra_status sra_forward_noalloc(const sra_problem* p,
                               const void* q_gen, const void* k_gen, const void* v_gen,
                               const void* q_ref, const void* k_ref, const void* v_ref,
                               void* o_gen, void* o_ref, float* lse_gen, float* lse_ref,
                               void* stream);

/* ---- host-only inspection hooks (no device needed; used to test the schedules) ---------- */

/* Visible (query, key) pairs per head summed over samples: the work of the attention, which
 * §1 and §2.1 state grows (almost) linearly with the reference length; from the closed form
 * G*(G + R_valid) for gen queries (G*R_valid plus the window's gen pairs with
 * SRA_FLAG_GEN_WINDOW) and sum over groups of (valid tokens of the group)^2 for ref queries.
 * Either output pointer may be NULL. */
sra_status sra_pair_counts(const sra_problem* p, int64_t* gen_pairs, int64_t* ref_pairs);

/* The visibility rule of the top of this file (§1, §2.1, §4.3; the window of §2.4 with
 * SRA_FLAG_GEN_WINDOW) written out for `sample` as a (G+R) x (G+R) byte matrix, rows = queries
 * and columns = keys in [gen ; ref] order of that sample: out[q*(G+R)+k] = 1 when query q sees
 * key k, else 0. Computed from the geometry alone (not from a schedule; sra_schedule_mask
 * gives what a schedule covers). Other flags do not change it. out must hold (G+R)^2 bytes
 * (host memory owned by the caller); host only. */
sra_status sra_dense_mask(const sra_problem* p, int32_t sample, uint8_t* out);

/* Sizes of schedule `which` (SRA_SCHED_*), the tile schedules that realise the visibility rule
 * of §1, §2.1 and §4.3 without a dense mask: work items (all heads) and span entries, and the
 * (query, key) pairs the schedule covers per head (must equal the pair count). */
sra_status sra_schedule_info(const sra_problem* p, int which, int64_t* n_items,
                             int64_t* n_spans, int64_t* covered_pairs);

/* Expands schedule `which` (the visibility rule of §1, §2.1 and §4.3 as tiles) for head 0 of
 * `sample` into a (G+R) x (G+R) byte matrix, rows =
 * queries and columns = keys in [gen ; ref] order of that sample: out[q*(G+R)+k] = number of
 * work items that compute the pair (q, k), so a correct schedule gives exactly the 0/1
 * visibility mask. out must hold (G+R)^2 bytes (host). */
sra_status sra_schedule_mask(const sra_problem* p, int which, int32_t sample, uint8_t* out);

/* What a call launches for schedule `which`. The hooks above report whole work items of 256 rows;
 * a call may take larger tiles, and splits items along their spans (their partial results are
 * combined by a kernel of their own) where too few, too long items would leave compute units
 * idle. n_items: work items and pieces, tile: rows per work item, split_items: items that are
 * split; any may be NULL. Host only. */
sra_status sra_launch_info(const sra_problem* p, int which, int64_t* n_items, int64_t* tile,
                           int64_t* split_items);

/* sra_schedule_mask of what a call launches, for head `head`: the pieces of a split item cover
 * its pairs once between them, so the matrix is again exactly the 0/1 visibility mask. Fails with
 * SRA_ERR_INTERNAL where pieces and the slots of their partial results do not match. */
sra_status sra_launch_mask(const sra_problem* p, int which, int32_t sample, int32_t head,
                           uint8_t* out);

/* Copies schedule `which` (the tiles realising §1, §2.1 and §4.3) into host buffers:
 * items[8*i + 0..7] = {stream, head, start, length,
 * span_offset, span_count, sample, reserved} per work item, spans[4*j + 0..3] = {stream,
 * start, length, keys} per span (stream 0 = gen, 1 = ref; start = packed token row; keys, in
 * the dK/dV schedule only: the item's keys [lo, hi), counted from its first key, that the
 * span's queries see, packed lo | hi << 16, or 0 for all of them).
 * items/spans may be NULL to query only; capacities count int32 elements.
 * Items are whole (256 rows) and listed in launch order (item i runs on XCD i % 8). When the head count is a
 * multiple of 8, an item whose first span is its sample's gen rows may start that span part
 * way in and wrap around (the span then appears as two entries, its tail first), so that the
 * items resident on one XCD stream the same rows at the same time; the rows covered are the
 * same either way.
 * When token masks split reference frames into more runs of valid tokens than there are
 * groups with a valid token, the library runs on the compacted reference stream (the valid
 * reference tokens of the batch back to back, in sample, group and token order: gathered
 * before the kernels, outputs scattered back after); ref rows of the schedule are then rows
 * of that stream. */
sra_status sra_schedule_export(const sra_problem* p, int which, int32_t* items,
                               int64_t items_capacity, int32_t* spans, int64_t spans_capacity);

/* sra_schedule_export of what a call launches for schedule `which` (the tiles realising §1, §2.1 and
 * §4.3, larger or cut as sra_launch_info says). items[8*i + 7] is 0, or k for the piece whose partial
 * results go to slot k - 1. Where a backward runs as one launch, the dQ and dK/dV schedules list
 * their items of it and share its span table. n_items and n_spans (either may be NULL) receive the
 * tables' sizes, padding items included. Host only. */
sra_status sra_launch_export(const sra_problem* p, int which, int32_t* items, int64_t items_capacity,
                             int32_t* spans, int64_t spans_capacity, int64_t* n_items, int64_t* n_spans);

/* ---- language-model attention: packed prompts, and serving over a paged cache -------------
 *
 * The audio engine (§2.3) is a language model over discrete audio tokens. Its attention is causal, several query
 * heads may share a K/V head, and it serves from a cache. Conventions as above, with these differences:
 *   Tensors   q, o, do, dq are [tokens, num_heads, head_dim], k, v, dk, dv [keys, num_kv_heads, head_dim], bf16;
 *             lse fp32 [num_heads, tokens]. num_heads = G num_kv_heads, query head h reads K/V head h / G. Inputs
 *             q, k and v have a token stride of their own each (0 selects the dense one; q, k and v may be views
 *             of one buffer); o, do and the gradients are dense.
 *   Errors    as above. Device-resident sizes (sra_tree_attention, sra_cache_append) cannot be refused on the
 *             host: what a call does for bad ones is stated there, and no such value makes it read or write
 *             outside the tensors it was given.
 *   Roundings sums, maxima, o and the gradients' sums are held in 32 bits; P and dS are rounded to bf16 as inputs of
 *             the matrix products, and D = rowsum(do o) takes the stored o.
 *   Rows that see no key have o = 0, lse = -inf and no part in any gradient. So have rows whose scores are all
 *             -inf. An infinity or NaN in v (the gradients: in any input) reaches, as in a product with zeros,
 *             also rows and keys of its sequence that the mask keeps apart from it, never another sequence's.
 *   Devices   a call launches on the current device, which must be the stream's.                             */

/* Lengths of packed sequences (host memory, read by sra_causal_plan_create only). */
typedef struct sra_causal_problem {
  int32_t batch;             /* sequences, >= 1                                              */
  int32_t num_heads;         /* a multiple of num_kv_heads                                   */
  int32_t num_kv_heads;      /* >= 1                                                         */
  int32_t head_dim;          /* 64 or 128                                                    */
  const int32_t* q_lens;     /* [batch] query tokens, >= 0                                   */
  const int32_t* k_lens;     /* [batch] keys, >= 0; NULL = q_lens                            */
} sra_causal_problem;

/* The tile schedule of causal attention for one set of lengths: made once, used for every layer and
 * call with these lengths, from any thread (immutable). It holds host memory only; its tables go into
 * a device buffer of the caller's. */
typedef struct sra_causal_plan sra_causal_plan;

/* Plans causal attention (§2.3) of packed sequences: token i of a sequence with nq tokens and nk keys sees the keys
 * j <= i + nk - nq, so the last token sees the last key (nk > nq: the sequence continues earlier keys; with
 * nq > nk the first nq - nk tokens see nothing). backward != 0 plans the gradients too.
 * Host only. num_heads * tokens and num_kv_heads * keys are below 2^28, and there are at most 2^22 / num_kv_heads
 * blocks of 256 keys, and of 256 (token, query head of a K/V head) pairs, of a sequence each (beyond:
 * SRA_ERR_UNSUPPORTED). */
sra_status sra_causal_plan_create(const sra_causal_problem* p, int backward, sra_causal_plan** plan);

/* Library infrastructure: frees a plan (NULL is allowed). Calls that were enqueued with it do not need it any more, only
 * the device copy of its tables. */
sra_status sra_causal_plan_destroy(sra_causal_plan* plan);

/* Library infrastructure: bytes of the plan's tables and of the workspaces of sra_causal_forward and
 * sra_causal_backward (0: none is needed). Any pointer may be NULL. */
sra_status sra_causal_plan_sizes(const sra_causal_plan* plan, size_t* table_bytes, size_t* forward_workspace,
                                 size_t* backward_workspace);

/* Library infrastructure: writes the plan's tables to host memory, for the caller to copy to the device. */
sra_status sra_causal_plan_tables(const sra_causal_plan* plan, void* host, size_t bytes);

/* Host-only inspection hook: what the launches of `which` (SRA_SCHED_*) cover of the rule of
 * sra_causal_plan_create (§2.3), for query head `head` of sequence `sequence`: out[i * nk + j] = how many items and
 * pieces compute the pair (token i, key j) without masking it, so a correct plan gives the 0/1 mask. */
sra_status sra_causal_plan_mask(const sra_causal_plan* plan, int which, int32_t sequence, int32_t head, uint8_t* out);

/* Causal attention of packed prompts (§2.3), forward: o and lse of every query row.
 * tables: device copy of the plan's tables, 16-byte aligned. softmax_scale <= 0 selects 1/sqrt(head_dim).
 * Strides in elements, multiples of 8. workspace: as sra_causal_plan_sizes says, 256-byte aligned.
 * Deterministic; enqueues kernels only, so it can be captured into a graph. */
sra_status sra_causal_forward(const sra_causal_plan* plan, const void* tables, const void* q, const void* k,
                              const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride, void* o,
                              float* lse, float softmax_scale, void* workspace, size_t workspace_bytes,
                              void* stream);

/* Gradients of sra_causal_forward (§2.3; the gradient of masked softmax attention), given its o and lse and the
 * upstream gradient dout (dense): dq, dk, dv are overwritten; dk and dv hold the sums over the query heads
 * that share a K/V head. The plan must have been made with backward != 0. Deterministic, no atomics. */
sra_status sra_causal_backward(const sra_causal_plan* plan, const void* tables, const void* q, const void* k,
                               const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                               const void* o, const float* lse, const void* dout, void* dq, void* dk, void* dv,
                               float softmax_scale, void* workspace, size_t workspace_bytes, void* stream);

/* A paged K/V cache and the sequences of one serving step (§2.3: the audio engine's language model answers token by
 * token). Pages hold page_size positions of all K/V heads: k and v are bf16 [num_pages, page_size, num_kv_heads,
 * head_dim] with heads contiguous and a page and a token stride each (0 selects the dense ones). Position p of
 * sequence b is slot p % page_size of page page_table[b * table_stride + p / page_size].
 * page_table, context_lens and cu_tokens are DEVICE arrays, read when the call runs: a captured call serves any
 * values. Sequence b holds context_lens[b] cached positions (taken as 0 below 0, and as max_pages * page_size
 * above that) and the new tokens cu_tokens[b] .. cu_tokens[b + 1] - 1 of the packed ones (clamped to [0, tokens];
 * sra_tree_attention also takes a falling entry as equal to the one before). Tokens before the first sequence's and
 * behind the last one's are padding: their outputs are left as they were. */
typedef struct sra_paged_cache {
  int32_t batch;              /* sequences, 1 .. 2048                                       */
  int32_t tokens;             /* rows of the packed new tokens, 0 .. 2^25                   */
  int32_t num_kv_heads;
  int32_t head_dim;           /* 64 or 128                                                  */
  int32_t num_pages;          /* >= 1                                                       */
  int32_t page_size;          /* a power of two, >= 8                                       */
  int32_t max_pages;          /* entries of a page_table row, >= 1; max_pages * page_size <= 2^30 */
  void* k;
  void* v;
  int64_t k_page_stride, v_page_stride;    /* elements, < 2^35; 0 selects page_size * token stride */
  int64_t k_token_stride, v_token_stride;  /* elements; 0 selects num_kv_heads * head_dim   */
  const int32_t* page_table;
  int64_t table_stride;       /* entries between rows, >= max_pages; 0 selects max_pages    */
  const int32_t* context_lens;  /* [batch]     */
  const int32_t* cu_tokens;     /* [batch + 1] */
} sra_paged_cache;

/* Bytes of device workspace of sra_tree_attention (library infrastructure). Host only; the pointers of `c` are not
 * looked at. */
sra_status sra_tree_workspace_size(const sra_paged_cache* c, int32_t num_heads, size_t* bytes);

/* Attention of each sequence's new tokens (§2.3; one token, or a tree of drafted ones that are checked in one pass): a
 * token sees its sequence's whole cached context and, of the sequence's new tokens, those that its mask names, through
 * one softmax (as §4.3 joins cached K/V with the current tokens'). Nothing is written to the cache.
 * q, o: bf16 [tokens, num_heads, head_dim], k, v: the new tokens' bf16 [tokens, num_kv_heads, head_dim].
 * Lengths may be mixed in any way; the kernel is chosen by the average rows of a sequence (tokens / batch x num_heads /
 * num_kv_heads, padding included), and long chains are computed with the keys behind each token, masked.
 * tree: device [tokens], bit j of token i's mask = it sees new token j (< 64) of its sequence; itself only if that bit
 *   is set, and later tokens of a longer sequence are seen by none. NULL: a chain of any length, each token sees the
 *   new tokens of its sequence up to itself.
 * Positions of pages whose id is not in [0, num_pages) are seen by no token.
 * At most 1024 query heads per K/V head. Deterministic; enqueues kernels only. The order of sums follows all lengths of
 * the call. workspace: 256-byte aligned, as sra_tree_workspace_size says, no initialisation; calls that may overlap
 * need one each. */
sra_status sra_tree_attention(const sra_paged_cache* c, int32_t num_heads, const void* q, const void* k,
                              const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                              const uint64_t* tree, void* o, float* lse, float softmax_scale, void* workspace,
                              size_t workspace_bytes, void* stream);

/* Writes K and V of new tokens (§2.3; a prompt's, or the accepted ones of a drafted tree) behind their sequences'
 * context: token i of sequence b goes to position context_lens[b] + i - cu_tokens[b]. k, v: bf16 [n_rows,
 * num_kv_heads, head_dim]; rows: device [tokens], the row of k and v that each token is (NULL: token i is row i, and
 * n_rows = tokens). context_lens is not changed: the caller adds the tokens' number when it wants them seen.
 * Tokens whose position lies behind the page_table row or in a page whose id is not in [0, num_pages), or whose row
 * is not in [0, n_rows), are skipped. Two tokens of a call never share a position of a sequence; where page_table
 * names a page twice, which of its writers' rows a slot ends up with is not defined. No row of the k pages shares memory
 * with one of the v pages, nor with k or v. */
sra_status sra_cache_append(const sra_paged_cache* c, const void* k, const void* v, int64_t k_stride,
                            int64_t v_stride, const int32_t* rows, int32_t n_rows, void* stream);

/* Host-only inspection hook of the two calls above (§2.3), with the arrays of `c` in HOST memory (k and v are not looked
 * at): append_rows[i] = the cache row (page * page_size + slot) that token i is written to, or -1 (rows are taken as
 * valid), and context_rows[p] = the cache row of position p of sequence `sequence`, or -1 where no token sees it;
 * either may be NULL. context_rows holds max_pages * page_size entries. */
sra_status sra_cache_rows(const sra_paged_cache* c, int64_t* append_rows, int32_t sequence, int64_t* context_rows);

/* ---- per-kernel timing (tracing hook; library infrastructure, no passage of the paper) --- */

/* Kernels of the library, for sra_kernel_timing. */
enum {
  SRA_KERNEL_FORWARD = 0,   /* forward pass                              */
  SRA_KERNEL_DELTA = 1,     /* backward: D = rowsum(dO * O)              */
  SRA_KERNEL_DKDV = 2,      /* backward: dK and dV (key-major); with dQ where few items of both
                             * kinds run as one launch                   */
  SRA_KERNEL_DQ = 3,        /* backward: dQ (query-major)                */
  SRA_KERNEL_FILL = 4,      /* rows of invalid reference frames          */
  SRA_KERNEL_GATHER = 5,    /* reference rows into the compacted stream  */
  SRA_KERNEL_SCATTER = 6,   /* compacted rows back to the reference rows */
  SRA_KERNEL_CAUSAL_FORWARD = 7,  /* sra_causal_forward                  */
  SRA_KERNEL_CAUSAL_DELTA = 8,    /* sra_causal_backward: D              */
  SRA_KERNEL_CAUSAL_GRAD = 9,     /* sra_causal_backward: dQ, dK and dV  */
  SRA_KERNEL_TREE = 10,           /* sra_tree_attention                  */
  SRA_KERNEL_APPEND = 11,         /* sra_cache_append                    */
  SRA_KERNEL_COUNT = 12
};

/* enable != 0: from now on every kernel launch is bracketed by two hipEvents recorded on the
 * caller's stream, and the accumulated totals are reset. enable == 0 stops recording. */
sra_status sra_kernel_timing_enable(int enable);

/* Waits for the recorded events and returns the summed duration (ms) and launch count of
 * kernel `kernel` (SRA_KERNEL_*) since timing was enabled. */
sra_status sra_kernel_timing(int kernel, double* total_ms, int64_t* launches);

/* Library infrastructure (no passage of the paper). Frees cached schedules and their pinned
 * host staging buffers, after waiting for the copies that read them (the only entry point that
 * waits on the device). Evicting a plan from the cache neither waits nor frees: its staging
 * buffer is reused for a later plan once the copies out of it have completed. Safe to call at
 * any time; later calls rebuild what they need. */
sra_status sra_release_caches(void);

/* Library infrastructure (no passage of the paper): status names, the per-thread detail of
 * the last failing call ("" if none), and the version as major*10000 + minor*100 + patch. */
const char* sra_status_string(sra_status s);
const char* sra_last_error(void);
int32_t sra_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SRA_H_ */
