// Forward pass of Sparse Reference Attention on gfx950.
//
// One workgroup (8 wave64s, two per SIMD) takes one work item: a tile of up to 128 NQ (256, 384 or
// 512) query rows of one stream and head, plus the list of key spans those rows see (Avatar V §1,
// §2.1, §4.3: gen rows see the gen keys and the valid ref frames of their sample; ref rows
// see the valid frames of their own group). Every wave owns 16 NQ query rows, as NQ MFMA column
// blocks, and keeps Q^T and O^T in VGPRs; keys stream through LDS in 64-row tiles (direct
// global->LDS loads, three buffers each for K and V):
//
//   S^T (keys x queries) = K Q^T          bf16 MFMA 16x16x32, K row fragments from LDS
//   online softmax over keys in base 2, lanes = queries (row sums are lane-local plus two
//   permlane swaps)
//   O^T (d x queries) += V^T P^T          V^T fragments via the LDS transpose read
//
// 16x16x32 MFMAs: at the board's power limit they sustain 2,050 TFLOP/s from registers on
// random data, 32x32x16 ones 1,840 (one wave per SIMD) or 1,350 (two). Launches that end before that
// limit sets in run on 32x32x16 ones (sra_fwd32.hip).
//
// Bound by the clock that the board's power allows (720p: 1.94 of 2.4 GHz) and by issue: the MFMA pipes
// are busy 65 % of the cycles, with 1.9 vector instructions per MFMA; waves wait for an issue slot in
// 31 % of their cycles, for data or a barrier in 29 %, for LDS in 2 %.
//
// What one 16-row block costs in LDS reads falls with the rows per wave: 32 rows (d = 128, 256-row
// items) feed two MFMAs per fragment, 48 (d = 128) three, 64 (d = 64) four. 480p layer, 40 heads:
// 26.2 ms with 32x32x16 MFMAs, 25.5 with these, 23.8 (1,340 TFLOP/s) with 48 rows.
//
// The key loop is software-pipelined in 32-key halves and each wave's instruction stream is
// laid out by hand: one block issues the P V product of the previous half and the S^T product
// of the next half, slot by slot, each MFMA followed by its share of the softmax of the current
// half; LDS fragments are read one slot pair ahead, across blocks too. A wave's MFMAs then run
// while the same wave issues its softmax arithmetic, instead of the two alternating in phases.
//
// The running max m is not tracked per half. P is computed against the current m, and its
// partial row sum doubles as the overflow check: if some lane's 8 values of a row sum to more
// than kBigSum (some P > kBigSum, or an inf from m = -inf at the start), the wave takes the rare
// slow path: recompute that half's S, set m to the true running max, rescale O and l,
// recompute P. So m always lies within log2(kBigSum) of the true row max.
//
// Full 64-key tiles of all spans run through the pipeline first; the ragged tail of each
// span runs afterwards in a masked, unpipelined step (the accumulation is order-independent).
#include <type_traits>

#include "sra_fwd_pipe.h"

namespace sra {

template <int D, int NQ, int NS>
__global__ void __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
sra_fwd_kernel(FwdArgs a) {
  constexpr int NC = D / 32, ND = D / 16, BK = kFwdKeyStep, RK = kPadRS<D>, RV = kPadRS<D>;
  constexpr int KE = KTile<D>::kElems, VE = VTile<D>::kElems;
  // Three buffers each for K and V, as separate arrays addressed only with compile-time
  // choices (the loop is unrolled by three): the compiler can then tell a buffer being filled
  // by direct loads from the ones being read, and does not stall the reads on those loads.
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf0[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf1[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf2[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf0[VE];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf1[VE];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf2[VE];
  __bf16* const kb[3] = {kbuf0, kbuf1, kbuf2};
  __bf16* const vb[3] = {vbuf0, vbuf1, vbuf2};

  const WorkItem it = a.items[blockIdx.x];
  if (it.stream < 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int h = it.head, s = it.stream;
  const int wrow0 = wave * 16 * NQ;
  const bool active = wrow0 < it.len;
  const float sl2 = a.scale_log2;

  FwdState<D, NQ> st;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = wrow0 + 16 * qb + l16;
    const __bf16* src = a.q[s] + int64_t(it.start + min(r, it.len - 1)) * a.in_stride[s] + h * D + g * 8;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bf16x8 x = *reinterpret_cast<const bf16x8*>(src + c * 32);
      st.qf[qb][c] = (r < it.len) ? x : bf16x8{};
    }
#pragma unroll
    for (int db = 0; db < ND; ++db) st.o[qb][db] = floatx4{};
    st.m[qb] = -INFINITY;
    st.l[qb] = 0.f;
  }

  const Span* sp = a.spans + it.span_off;
  int T = 0;  // full tiles over all spans
  for (int i = 0; i < it.span_cnt; ++i) T += __builtin_amdgcn_readfirstlane(sp[i].len) / BK;

  // byte offsets of this wave's direct loads from the tile's first row (K and V tiles are laid
  // out alike; the streams differ in their token stride)
  using TL = PaddedTile<D, BK, RK>;
  constexpr int kSlots = (TL::kInstr + kWaves - 1) / kWaves, kFull = TL::kInstr / kWaves;
  uint32_t voff[NS][kSlots];
#pragma unroll
  for (int ss = 0; ss < NS; ++ss) {
    TileLoader<D, BK, RK, kWaves> tl;
    tl.init(a.in_stride[ss], h, wave);
#pragma unroll
    for (int j = 0; j < kSlots; ++j) voff[ss][j] = uint32_t(tl.voff[j]) * 2;
  }
  FullTileCursor<BK> kc, vc;  // next full tile to load for K, for V
  kc.init(sp, it.span_cnt);
  vc.init(sp, it.span_cnt);
  // per-stream bases as uniform scalars and this wave's LDS slots as byte addresses, so a
  // tile's loads need no argument reads and no address arithmetic per lane
  const uint64_t kb0 = uniform_u64(reinterpret_cast<uint64_t>(a.k[0]));
  const uint64_t kb1 = uniform_u64(reinterpret_cast<uint64_t>(a.k[1]));
  const uint64_t vb0 = uniform_u64(reinterpret_cast<uint64_t>(a.v[0]));
  const uint64_t vb1 = uniform_u64(reinterpret_cast<uint64_t>(a.v[1]));
  const int64_t st0 = a.in_stride[0] * 2, st1 = a.in_stride[1] * 2;  // bytes
  const bool extra = wave + kFull * kWaves < TL::kInstr;
  auto issue = [&](const FullTileCursor<BK>& c, uint64_t b0, uint64_t b1, const __bf16* dst) __attribute__((always_inline)) {
    const int ss = c.cur_stream;
    const uint64_t g = (ss ? b1 : b0) + uint64_t(int64_t(c.cur_start + c.off) * (ss ? st1 : st0));
    const uint32_t la = lds_addr(dst) + wave * 1024;
#pragma unroll
    for (int j = 0; j < kSlots; ++j)
      if (j < kFull || extra)
        lds_dma_x4_off(g, NS == 1 || !ss ? voff[0][j] : voff[NS - 1][j], la + j * kWaves * 1024);
  };
  auto issue_k = [&](const __bf16* dst) __attribute__((always_inline)) {
    issue(kc, kb0, kb1, dst);
    kc.advance();
  };
  auto issue_v = [&](const __bf16* dst) __attribute__((always_inline)) {
    issue(vc, vb0, vb1, dst);
    vc.advance();
  };

  // Pipelined full tiles. Tile t sits in K buffer t % 3 and V buffer t % 3 (tile -1 in V
  // buffer 2). Iteration t reads K(t) (second half), K(t+1) (first half), V(t-1) (second
  // half) and V(t) (first half), and loads K(t+2) and V(t+1).
  if (T > 0) {
    // V buffer 2 stands for tile -1: zero its second half so the first P V (P = 0) adds 0.
    for (int e = threadIdx.x * 8; e < 32 * RV; e += kWaves * 64 * 8)
      *reinterpret_cast<bf16x8*>(vbuf2 + 32 * RV + e) = bf16x8{};
    issue_k(kbuf0);
    issue_v(vbuf0);
    if (T > 1) issue_k(kbuf1);
    wait_vmem();
    __syncthreads();
    HalfP<NQ> p_hi;  // P of the previous tile's second half (zero before the first tile)
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) p_hi.p[qb] = bf16x8{};
    HalfS<NQ> s_lo = {}, s_hi = {};
    if (active) s_lo = scores32<D, NQ>(st, kbuf0);
    Ahead ah;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      ah.k[i] = k_frag<D>(kbuf0 + 32 * RK, i);
      ah.v[i] = v_frag<D>(vbuf2 + 32 * RV, i);
    }
    auto iteration = [&](int t, auto phase) {
      constexpr int P = decltype(phase)::value;
      __bf16* const k_t = kb[P];
      __bf16* const k_t1 = kb[(P + 1) % 3];
      __bf16* const v_tm1 = vb[(P + 2) % 3];
      __bf16* const v_t = vb[P];
      if (t + 1 < T) issue_v(vb[(P + 1) % 3]);
      if (t + 2 < T) issue_k(kb[(P + 2) % 3]);
      if (active) {
        // block 1: S^T of this tile's second half and P V of the previous tile's second
        // half, under the softmax of this tile's first half
        const HalfP<NQ> p_lo = pipe_block<D, NQ>(st, s_lo, k_t, s_hi, k_t + 32 * RK, v_tm1 + 32 * RV, k_t1, v_t, ah, p_hi, sl2);
        // block 2: S^T of the next tile's first half and P V of this tile's first half,
        // under the softmax of this tile's second half (the last iteration's S^T is unused)
        p_hi = pipe_block<D, NQ>(st, s_hi, k_t + 32 * RK, s_lo, k_t1, v_t, k_t1 + 32 * RK, v_t + 32 * RV, ah, p_lo, sl2);
      }
      wait_vmem();
      __syncthreads();
    };
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    using P2 = std::integral_constant<int, 2>;
    int t = 0;
    for (; t + 3 <= T; t += 3) {
      iteration(t, P0{});
      iteration(t + 1, P1{});
      iteration(t + 2, P2{});
    }
    if (t < T) iteration(t, P0{});
    if (t + 1 < T) iteration(t + 1, P1{});
    // the last tile's second half: V(T-1) sits in buffer (T-1) % 3
    if (active) {
      const int last = (T - 1) % 3;
      if (last == 0) pv_half<D, NQ>(st, vbuf0 + 32 * RV, p_hi);
      else if (last == 1) pv_half<D, NQ>(st, vbuf1 + 32 * RV, p_hi);
      else pv_half<D, NQ>(st, vbuf2 + 32 * RV, p_hi);
    }
  }

  // Ragged span tails (masked, not pipelined).
  for (int i = 0; i < it.span_cnt; ++i) {
    const Span sp_i = sp[i];
    const int len = __builtin_amdgcn_readfirstlane(sp_i.len);
    const int rem = len % BK;
    if (rem == 0) continue;
    __syncthreads();  // every wave is done with the buffers
    const int ss = __builtin_amdgcn_readfirstlane(sp_i.stream);
    const int st0 = __builtin_amdgcn_readfirstlane(sp_i.start);
    tile_load_lds<D, BK, RK, kWaves>(kbuf0, a.k[ss], a.in_stride[ss], h, st0, len, len - rem, wave);
    tile_load_lds<D, BK, RV, kWaves>(vbuf0, a.v[ss], a.in_stride[ss], h, st0, len, len - rem, wave);
    wait_vmem();
    __syncthreads();
    if (active) {
      masked_half<D, NQ>(st, kbuf0, vbuf0, rem, sl2);
      if (rem > 32) masked_half<D, NQ>(st, kbuf0 + 32 * RK, vbuf0 + 32 * RV, rem - 32, sl2);
    }
  }

  if (!active) return;
  const int64_t ostride = int64_t(a.heads) * D;
  float* part = it.slot ? a.part + int64_t(it.slot - 1) * (kWaves * 16 * NQ) * (D + 2) : nullptr;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = wrow0 + 16 * qb + l16;
    const float lt = quad_sum(st.l[qb]);
    if (part) {  // a piece of a split item
      if (r >= it.len) continue;
#pragma unroll
      for (int db = 0; db < ND; ++db) *reinterpret_cast<floatx4*>(part + r * D + db * 16 + 4 * g) = st.o[qb][db];
      if (g == 0) *reinterpret_cast<float2*>(part + kWaves * 16 * NQ * D + 2 * r) = float2{st.m[qb], lt};
      continue;
    }
    const float inv = 1.f / lt;
    if (r >= it.len) continue;
    __bf16* orow = a.o[s] + int64_t(it.start + r) * ostride + h * D;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (__bf16)(st.o[qb][db][e] * inv);
      *reinterpret_cast<bf16x4*>(orow + db * 16 + 4 * g) = w;
    }
    if (g == 0) a.lse[s][int64_t(h) * a.rows[s] + it.start + r] = (st.m[qb] + log2f(lt)) * kLn2;
  }
}

// Rows of the split items from their pieces: with M the largest of the pieces' running maxima,
// O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i, in piece order. D / 4 threads per row. A piece whose
// scores of a row are all -inf has weight 0; a row of which all are so ends as in a whole item (LSE -inf).
// Bound by reading the partial results (28 MB at most): 3 heads of 800 + 429 tokens 38.5 -> 25.3 us.
template <int D>
__global__ void __launch_bounds__(kThreads) sra_fwd_combine_kernel(FwdArgs a, const CombineItem* items) {
  constexpr int TPR = D / 4, RPB = kThreads / TPR;
  const CombineItem it = items[blockIdx.x];
  const int r = blockIdx.y * RPB + threadIdx.x / TPR, sub = threadIdx.x % TPR, tile = a.tile;
  if (r >= it.len) return;
  const int64_t slot = int64_t(tile) * (D + 2);
  const float* p = a.part + it.slot0 * slot;
  float m = -INFINITY;
  for (int i = 0; i < it.n; ++i) m = fmaxf(m, p[i * slot + int64_t(tile) * D + 2 * r]);
  floatx4 o = floatx4{};
  float l = 0.f;
  for (int i = 0; i < it.n; ++i) {
    const float2 ml = *reinterpret_cast<const float2*>(p + i * slot + int64_t(tile) * D + 2 * r);
    const float w = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m);
    l += w * ml.y;
    o += w * *reinterpret_cast<const floatx4*>(p + i * slot + r * D + 4 * sub);
  }
  const float inv = 1.f / l;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * inv);
  *reinterpret_cast<bf16x4*>(a.o[it.stream] + (int64_t(it.start + r) * a.heads + it.head) * D + 4 * sub) = y;
  if (sub == 0) a.lse[it.stream][int64_t(it.head) * a.rows[it.stream] + it.start + r] = (m + log2f(l)) * kLn2;
}

template <int D, int NQ>
static void launch_tile(const FwdArgs& a, int n_items, hipStream_t stream) {
  const dim3 grid(n_items), block(kWaves * 64);
  if (a.in_stride[0] == a.in_stride[1])
    hipLaunchKernelGGL((sra_fwd_kernel<D, NQ, 1>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((sra_fwd_kernel<D, NQ, 2>), grid, block, 0, stream, a);
}

hipError_t launch_forward(const FwdArgs& a, int n_items, int head_dim, bool mfma32, hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  if (mfma32) return launch_forward32(a, n_items, head_dim, stream);
  if (head_dim == 64) launch_tile<64, fwd_large_tile(64) / 128>(a, n_items, stream);
  else if (a.tile == kFwdQueryTile) launch_tile<128, kFwdQueryTile / 128>(a, n_items, stream);
  else launch_tile<128, fwd_large_tile(128) / 128>(a, n_items, stream);
  return hipGetLastError();
}

hipError_t launch_forward_combine(const FwdArgs& a, const CombineItem* items, int n, int head_dim, hipStream_t stream) {
  if (n <= 0) return hipSuccess;
  const int rows = kThreads / (head_dim / 4);
  const dim3 grid(n, (a.tile + rows - 1) / rows);
  if (head_dim == 128)
    hipLaunchKernelGGL(sra_fwd_combine_kernel<128>, grid, dim3(kThreads), 0, stream, a, items);
  else
    hipLaunchKernelGGL(sra_fwd_combine_kernel<64>, grid, dim3(kThreads), 0, stream, a, items);
  return hipGetLastError();
}

}  // namespace sra
