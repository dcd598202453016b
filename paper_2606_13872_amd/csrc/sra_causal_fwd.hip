// Forward pass of causal attention over packed sequences with grouped heads on gfx950.
//
//   S = scale Q K^T on the keys j <= i + nk - nq of token i, LSE = ln sum exp S, O = exp(S - LSE) V,
//
// one pass over the keys with a running maximum and sum. One workgroup (8 wave64s, two per SIMD) takes one work
// item (sra_causal.h): up to 256 (token, head of the group) rows, 32 per wave (short launches: 128, for more and shorter
// items; long ones: 384, or 512 of 64 head dims, which read and load the keys less often), against the keys up to the
// last that its rows see. The key tiles that every row sees run through the software pipeline of sra_fwd_pipe.h; those
// on the diagonal (256 / G tokens wide) run behind it, three at a time, masked by each row's last key. Rows that see
// nothing (nq > nk) end with l = 0: O = 0, LSE = -inf. P is rounded to bf16 for the matrix product; its sum, the maxima
// and O stay in 32 bits.
//
// Long launches are bound by the clock that the board's power allows (1.88 of 2.4 GHz, MFMA pipes busy 65 % of the
// cycles): 32,768 tokens, 32 query and 8 K/V heads of 128 dims 6.75 -> 6.28 ms (1,400 TFLOP/s; timed in turn)
// with 384 rows for 256. Short ones by the chain of an item: 6 us (128 rows) to 8 us (256) for its loads, diagonal and
// epilogue, and 0.9 or 1.4 us a step of 64 keys: 512, 700 and 129 tokens of 16 heads of 64 dims 19.3 -> 12.5 us with 128
// rows for 256, 512 tokens of 8 heads of 128 dims 23.6 -> 14.0. Loading the first diagonal tile within the pipeline gained
// nothing (1.5 % slower: more code). Running the diagonal through the pipeline too, with masked blocks, was 1 to 2 %
// slower on every size (more vector work per MFMA, twice the code), and one loop body with its buffers chosen at run time,
// instead of three, 3 % on long ones. 64 head dims: 32,768 tokens of as many heads 4.08 ms, 1,080 TFLOP/s (512 rows an item):
// the softmax's vector work is per score, so twice as much of it goes with a product (3.9 VALU instructions an MFMA for
// 2.0), and the MFMA pipes are busy 47 % of the cycles at 2.15 GHz.
#include <type_traits>

#include "sra_causal_kernels.h"
#include "sra_fwd_pipe.h"

namespace sra {

// A 32-key half whose first key is key0: row block qb sees the keys up to lim[qb]. P of hidden keys is 0.
template <int D, int NQ>
__device__ __forceinline__ void causal_half(FwdState<D, NQ>& st, const __bf16* kt, const __bf16* vt, int key0,
                                            const int* lim, float sl2) {
  const int g = (threadIdx.x & 63) >> 4;
  HalfS<NQ> s = scores32<D, NQ>(st, kt);
#pragma unroll
  for (int j = 0; j < 2 * NQ; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) s.b[j][i] = key0 + 16 * (j / NQ) + 4 * g + i <= lim[j % NQ] ? s.b[j][i] : -INFINITY;
  float sum[NQ];
  rescale_half<D, NQ>(st, s, sl2, sum);
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) st.l[qb] += sum[qb];
  pv_half<D, NQ>(st, vt, pack_half<NQ>(s));
}

// kOneStride: k and v share one token stride, so one set of load offsets serves both.
template <int D, int NQ, bool kOneStride>
__global__ void __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
sra_causal_fwd_kernel(CausalArgs a) {
  constexpr int kRowsPerWave = 16 * NQ, NC = D / 32, ND = D / 16, BK = kFwdKeyStep, RK = kPadRS<D>;
  constexpr int KE = KTile<D>::kElems;
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf0[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf1[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 kbuf2[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf0[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf1[KE];
  __shared__ __attribute__((aligned(1024))) __bf16 vbuf2[KE];
  __bf16* const kb[3] = {kbuf0, kbuf1, kbuf2};
  __bf16* const vb[3] = {vbuf0, vbuf1, vbuf2};

  const CausalItem it = a.items[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.heads / a.kv_heads, off = it.nk - it.nq;
  const int wrow0 = wave * kRowsPerWave;
  const bool active = wrow0 < it.len;
  const float sl2 = a.scale_log2;

  FwdState<D, NQ> st;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = wrow0 + 16 * qb + l16, row = it.start + min(r, it.len - 1);
    const int token = row / G, hg = row - token * G;
    const __bf16* src = a.q + int64_t(it.q0 + token) * a.qs + int64_t(it.kvh * G + hg) * D + g * 8;
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

  // full tiles: those that end at or before the last key of the item's first row
  const int first_lim = __builtin_amdgcn_readfirstlane(it.start / G + off);
  const int T = max(0, (min(it.hi, first_lim + 1) - it.lo) >> 6);

  // direct loads of a whole tile: K and V bases as uniform scalars, this lane's byte offsets from the first row
  using TL = PaddedTile<D, BK, RK>;
  constexpr int kSlots = (TL::kInstr + kWaves - 1) / kWaves, kFull = TL::kInstr / kWaves;
  uint32_t offs[kOneStride ? 1 : 2][kSlots];
#pragma unroll
  for (int s = 0; s < (kOneStride ? 1 : 2); ++s) {
    TileLoader<D, BK, RK, kWaves> tl;
    tl.init(s ? a.vs : a.ks, 0, wave);
#pragma unroll
    for (int j = 0; j < kSlots; ++j) offs[s][j] = uint32_t(tl.voff[j]) * 2;
  }
  const __bf16* const k0 = a.k + int64_t(it.k0) * a.ks + int64_t(it.kvh) * D;
  const __bf16* const v0 = a.v + int64_t(it.k0) * a.vs + int64_t(it.kvh) * D;
  uint64_t kp = uniform_u64(reinterpret_cast<uint64_t>(k0 + int64_t(it.lo) * a.ks));
  uint64_t vp = uniform_u64(reinterpret_cast<uint64_t>(v0 + int64_t(it.lo) * a.vs));
  const uint64_t kstep = uint64_t(a.ks) * (2 * BK), vstep = uint64_t(a.vs) * (2 * BK);
  const bool extra = wave + kFull * kWaves < TL::kInstr;
  auto issue = [&](uint64_t base, const uint32_t* off16, const __bf16* dst) __attribute__((always_inline)) {
    const uint32_t la = lds_addr(dst) + wave * 1024;
#pragma unroll
    for (int j = 0; j < kSlots; ++j)
      if (j < kFull || extra) lds_dma_x4_off(base, off16[j], la + j * kWaves * 1024);
  };
  auto issue_k = [&](const __bf16* dst) __attribute__((always_inline)) {
    issue(kp, offs[0], dst);
    kp += kstep;
  };
  auto issue_v = [&](const __bf16* dst) __attribute__((always_inline)) {
    issue(vp, offs[kOneStride ? 0 : 1], dst);
    vp += vstep;
  };

  // Pipelined full tiles. Tile t sits in K buffer t % 3 and V buffer t % 3 (tile -1 in V buffer 2). Iteration t
  // reads K(t) (second half), K(t+1) (first half), V(t-1) (second half) and V(t) (first half), and loads K(t+2)
  // and V(t+1).
  if (T > 0) {
    for (int e = threadIdx.x * 8; e < 32 * RK; e += kWaves * 64 * 8)
      *reinterpret_cast<bf16x8*>(vbuf2 + 32 * RK + e) = bf16x8{};
    issue_k(kbuf0);
    issue_v(vbuf0);
    if (T > 1) issue_k(kbuf1);
    wait_vmem();
    __syncthreads();
    HalfP<NQ> p_hi;
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) p_hi.p[qb] = bf16x8{};
    HalfS<NQ> s_lo = {}, s_hi = {};
    if (active) s_lo = scores32<D, NQ>(st, kbuf0);
    Ahead ah;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      ah.k[i] = k_frag<D>(kbuf0 + 32 * RK, i);
      ah.v[i] = v_frag<D>(vbuf2 + 32 * RK, i);
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
        const HalfP<NQ> p_lo = pipe_block<D, NQ>(st, s_lo, k_t, s_hi, k_t + 32 * RK, v_tm1 + 32 * RK, k_t1, v_t, ah, p_hi, sl2);
        p_hi = pipe_block<D, NQ>(st, s_hi, k_t + 32 * RK, s_lo, k_t1, v_t, k_t1 + 32 * RK, v_t + 32 * RK, ah, p_lo, sl2);
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
    if (active) {
      const int last = (T - 1) % 3;
      if (last == 0) pv_half<D, NQ>(st, vbuf0 + 32 * RK, p_hi);
      else if (last == 1) pv_half<D, NQ>(st, vbuf1 + 32 * RK, p_hi);
      else pv_half<D, NQ>(st, vbuf2 + 32 * RK, p_hi);
    }
  }

  // The other tiles: on the diagonal, or ragged. Rows past hi are clamped to the last key before it; no row sees
  // them (hi is behind the last key of the item's last row, or a multiple of 64 away from lo).
  const int wlast = __builtin_amdgcn_readfirstlane((it.start + min(wrow0 + kRowsPerWave, it.len) - 1) / G + off);
  int lim[NQ];  // the last key that this lane's row sees (-1 and below: none)
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) lim[qb] = (it.start + min(wrow0 + 16 * qb + l16, it.len - 1)) / G + off;
  for (int key0 = it.lo + BK * T; key0 < it.hi; key0 += 3 * BK) {
    __syncthreads();  // every wave is done with the buffers
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (key0 + j * BK < it.hi) {
        tile_load_lds<D, BK, RK, kWaves>(kb[j], k0, a.ks, 0, 0, it.hi, key0 + j * BK, wave);
        tile_load_lds<D, BK, RK, kWaves>(vb[j], v0, a.vs, 0, 0, it.hi, key0 + j * BK, wave);
      }
    wait_vmem();
    __syncthreads();
    if (active)
#pragma unroll 1
      for (int o = 0; o < 6; ++o) {  // one body for the halves: short calls wait for instructions
        const int key = key0 + 32 * o, j = o >> 1;
        if (key >= it.hi || key > wlast) break;
        const __bf16* const kt = j == 0 ? kbuf0 : j == 1 ? kbuf1 : kbuf2;
        const __bf16* const vt = j == 0 ? vbuf0 : j == 1 ? vbuf1 : vbuf2;
        causal_half<D, NQ>(st, kt + (o & 1) * 32 * RK, vt + (o & 1) * 32 * RK, key, lim, sl2);
      }
  }

  if (!active) return;
  float* part = it.slot ? a.part + int64_t(it.slot - 1) * kCausalTile * (D + 2) : nullptr;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = wrow0 + 16 * qb + l16;
    const float lt = quad_sum(st.l[qb]);
    if (r >= it.len) continue;
    if (part) {  // a piece of a split item
#pragma unroll
      for (int db = 0; db < ND; ++db) *reinterpret_cast<floatx4*>(part + r * D + db * 16 + 4 * g) = st.o[qb][db];
      if (g == 0) *reinterpret_cast<float2*>(part + kCausalTile * D + 2 * r) = float2{st.m[qb], lt};
      continue;
    }
    const int row = it.start + r, token = row / G, h = it.kvh * G + row - token * G;
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    __bf16* orow = a.o + (int64_t(it.q0 + token) * a.heads + h) * D;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (__bf16)(st.o[qb][db][e] * inv);
      *reinterpret_cast<bf16x4*>(orow + db * 16 + 4 * g) = w;
    }
    if (g == 0) a.lse[int64_t(h) * a.q_rows + it.q0 + token] = lt == 0.f ? -INFINITY : (st.m[qb] + log2f(lt)) * kLn2;
  }
}

// Rows of the split items from their pieces, in piece order: with M the largest of the pieces' running maxima,
// O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i. D / 4 threads per row. Bound by reading the partial results (25 MB:
// 8.5 us; with the maxima in a pass of their own 15 us).
template <int D>
__global__ void __launch_bounds__(kThreads) sra_causal_fwd_combine_kernel(CausalArgs a, const CausalItem* items) {
  constexpr int TPR = D / 4, RPB = kThreads / TPR;
  const CausalItem it = items[blockIdx.x];
  const int r = blockIdx.y * RPB + threadIdx.x / TPR, sub = threadIdx.x % TPR;
  if (r >= it.len) return;
  constexpr int64_t slot = int64_t(kCausalTile) * (D + 2);
  const float* p = a.part + it.lo * slot;
  float m = -INFINITY, l = 0.f;
  floatx4 o = floatx4{};
#pragma unroll 4
  for (int i = 0; i < it.hi; ++i) {  // one pass with a running maximum: the loads of four pieces are under way at once
    const float2 ml = *reinterpret_cast<const float2*>(p + i * slot + int64_t(kCausalTile) * D + 2 * r);
    const floatx4 x = *reinterpret_cast<const floatx4*>(p + i * slot + r * D + 4 * sub);
    const float mx = fmaxf(m, ml.x);
    const float f = l == 0.f ? 0.f : fast_exp2(m - mx);  // nothing so far
    const float w = ml.y == 0.f ? 0.f : fast_exp2(ml.x - mx);  // a piece that the row sees nothing of has m = -inf
    l = f * l + w * ml.y;
    o = f * o + w * x;
    m = mx;
  }
  const int G = a.heads / a.kv_heads, row = it.start + r, token = row / G, h = it.kvh * G + row - token * G;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * inv);
  *reinterpret_cast<bf16x4*>(a.o + (int64_t(it.q0 + token) * a.heads + h) * D + 4 * sub) = y;
  if (sub == 0) a.lse[int64_t(h) * a.q_rows + it.q0 + token] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int D, int NQ>
static void launch_tile(const CausalArgs& a, int n_items, hipStream_t stream) {
  const dim3 grid(n_items), block(kWaves * 64);
  if (a.ks == a.vs) hipLaunchKernelGGL((sra_causal_fwd_kernel<D, NQ, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((sra_causal_fwd_kernel<D, NQ, false>), grid, block, 0, stream, a);
}

hipError_t launch_causal_forward(const CausalArgs& a, int n_items, int head_dim, int tile, hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  constexpr int kRows = 16 * kWaves;
  if (head_dim == 128) {
    if (tile < kCausalTile) launch_tile<128, 1>(a, n_items, stream);
    else if (tile == kCausalTile) launch_tile<128, kCausalTile / kRows>(a, n_items, stream);
    else launch_tile<128, fwd_large_tile(128) / kRows>(a, n_items, stream);
  } else {
    if (tile < kCausalTile) launch_tile<64, 1>(a, n_items, stream);
    else if (tile == kCausalTile) launch_tile<64, kCausalTile / kRows>(a, n_items, stream);
    else launch_tile<64, fwd_large_tile(64) / kRows>(a, n_items, stream);
  }
  return hipGetLastError();
}

hipError_t launch_causal_forward_combine(const CausalArgs& a, const CausalItem* items, int n, int head_dim,
                                         hipStream_t stream) {
  if (n <= 0) return hipSuccess;
  const dim3 grid(n, kCausalTile * (head_dim / 4) / kThreads);
  if (head_dim == 128)
    hipLaunchKernelGGL(sra_causal_fwd_combine_kernel<128>, grid, dim3(kThreads), 0, stream, a, items);
  else
    hipLaunchKernelGGL(sra_causal_fwd_combine_kernel<64>, grid, dim3(kThreads), 0, stream, a, items);
  return hipGetLastError();
}

}  // namespace sra
