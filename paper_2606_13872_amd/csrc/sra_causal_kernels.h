// Argument blocks and launchers of the causal attention kernels.
#pragma once
#include <hip/hip_runtime.h>

#include "sra_causal.h"

namespace sra {

struct CausalArgs {
  const CausalItem* items;
  const __bf16* q;  // [q_rows, heads, D], token strides in elements
  const __bf16* k;  // [k_rows, kv_heads, D]
  const __bf16* v;
  int64_t qs, ks, vs;
  int32_t q_rows, heads, kv_heads;
  float scale, scale_log2;
  // forward
  __bf16* o;        // dense, as every tensor below
  float* lse;       // [heads, q_rows], natural log
  float* part;      // slots of split items: O [256, D] unscaled, then (m, l) per row
  // backward
  const __bf16* dout;
  const float* lse2;    // [heads, q_rows], log2 units, +inf on rows that see nothing
  const float* ndelta;  // [heads, q_rows], -rowsum(dO * O)
  __bf16 *dq, *dk, *dv;
  float* part_q;        // slots: dQ unscaled [256, D]
  float* part_kv;       // slots: dK unscaled and dV [256, D]
};

struct CausalDeltaArgs {
  const __bf16 *o, *dout;
  const float* lse;
  float *lse2, *ndelta;
  int32_t q_rows, heads;
};

// tile: rows per item
hipError_t launch_causal_forward(const CausalArgs& a, int n_items, int head_dim, int tile, hipStream_t stream);
hipError_t launch_causal_forward_combine(const CausalArgs& a, const CausalItem* items, int n, int head_dim,
                                         hipStream_t stream);
hipError_t launch_causal_delta(const CausalDeltaArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_causal_grad(const CausalArgs& a, int n_items, int head_dim, hipStream_t stream);
hipError_t launch_causal_grad_combine(const CausalArgs& a, const CausalItem* items, int n, int head_dim,
                                      hipStream_t stream);

}  // namespace sra
