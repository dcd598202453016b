// Backward pass of causal attention over packed sequences with grouped heads on gfx950.
//
// With P = exp(S - LSE) on the visible pairs, D = rowsum(dO * O) and head h reading K/V head h / G:
//     dV = sum_g P^T dO,  dS = P (dO V^T - D),  dQ = scale dS K,  dK = scale sum_g dS^T Q.
// Deterministic, no atomics: a delta kernel (-D and the LSE in log2 units; +inf where a row sees nothing, so that
// its P is 0), then one launch of dK/dV items (256 keys, in short launches 128; the query tiles of all G heads of the
// group run through one item, which so holds the heads' sum) and of dQ items (256 or 128 (token, head of the group)
// rows). The halves are those of sra_dkv.h and sra_dq.h; tiles on the diagonal take their masked forms.
//
// P and dS are rounded to bf16 for their matrix products, the sums stay in 32 bits; D takes the O that the forward stored
// (bf16). Against 64 bits dQ and dK are 2.7e-3 of their norm off, of which storing them is 1.7e-3, dS 1.7e-3 and
// D 1.1e-3.
//
// Bound by the clock that the board's power allows and by issue (2.04 of 2.4 GHz, MFMA pipes busy 58 % of the cycles,
// waves wait for an issue slot in 29 % of theirs): 2.3 us a dQ step of 64 keys x 256 rows (1,400 TFLOP/s executed),
// 3.2 us a dK/dV step of 64 tokens x 256 keys (1,340); an item costs 9 us (dQ) and 15 to 23 us (dK/dV) besides. 16,384
// and 9,001 tokens, 40 query and 8 K/V heads 10.0 ms. XCDs end up to 6 % apart (their clocks differ); a persistent
// launch that lets the fast ones take the others' items spilled registers around the accumulators and was not kept.
// Short launches are bound by the chain of an item: 512 tokens of 8 heads 43 -> 30 us, both kernels, with items of 128.
// 64 head dims: the same 16,384 and 9,001 tokens 5.8 ms, MFMA pipes busy 49 % of the cycles at 2.2 GHz (2.4 VALU
// instructions an MFMA for 1.4).
#include "sra_causal_kernels.h"
#include "sra_dkv.h"
#include "sra_dq.h"

namespace sra {

namespace {
constexpr float kLog2e = 1.44269504088896340736f;
}

// --------------------------------------------------------------------------- delta
// Bound by reading O and dO: 5.6 TB/s (8,192 tokens x 32 heads of 128 dims: 24 us).
template <int D>
__global__ void __launch_bounds__(kThreads) sra_causal_delta_kernel(CausalDeltaArgs a) {
  constexpr int TPR = D / 8, RPB = kThreads / TPR;  // threads per (row, head), pairs per block
  const int64_t pair = int64_t(blockIdx.x) * RPB + threadIdx.x / TPR;
  const int64_t total = int64_t(a.q_rows) * a.heads;
  const int sub = threadIdx.x % TPR;
  float acc = 0.f;
  if (pair < total) {
    const bf16x8 x = ld8(a.o + pair * D + sub * 8);
    const bf16x8 y = ld8(a.dout + pair * D + sub * 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc = fmaf(float(x[j]), float(y[j]), acc);
  }
#pragma unroll
  for (int w = 1; w < TPR; w <<= 1) acc += __shfl_xor(acc, w, TPR);
  if (pair < total && sub == 0) {
    const int64_t row = pair / a.heads;
    const int64_t i = (pair - row * a.heads) * a.q_rows + row;
    const float lse = a.lse[i];
    a.ndelta[i] = -acc;
    a.lse2[i] = lse == -INFINITY ? INFINITY : lse * kLog2e;
  }
}

// --------------------------------------------------------------------------- dK, dV
// The query tiles [lo, hi) of the item's list, all on the diagonal (kDiagonal) or all off it, through the pipeline.
template <int D, bool kDiagonal>
__device__ __forceinline__ void causal_dkv_tiles(const CausalArgs& a, const CausalItem& it, DkvState<D>& st,
                                                 const DkvAddr& ad, const CausalTiles& tiles, int G, int lo, int hi,
                                                 uint32_t lds0, uint32_t qoff, uint32_t doff, int wave, bool active) {
  using L = DkvLds<D>;
  using TL = SwzTile<D, kDkvTile>;
  constexpr int NB = kDkvBufs, NW = kDkvWaves, kLoads = TL::kInstr / NW, kEvery = 4 * (D / 16) / kLoads;
  const int T = hi - lo;
  if (T <= 0) return;
  const int lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
  const int off = it.nk - it.nq;
  const float sl2 = a.scale_log2;
  const int64_t dstride = int64_t(a.heads) * D;
  // a head's tiles of this kind: tokens [first, end)
  const int first_tok = kDiagonal ? tiles.t0 : tiles.t0 + kDkvTile * tiles.d;
  const int end_tok = kDiagonal ? tiles.t0 + kDkvTile * tiles.d : it.nq;
  CausalTile ld = causal_tile(tiles, G, lo), cu = ld;
  auto next = [&](CausalTile& c) __attribute__((always_inline)) {
    c.tok += kDkvTile;
    if (c.tok >= end_tok) {
      c.tok = first_tok;
      ++c.hg;
    }
  };
  const uint64_t qb = uniform_u64(reinterpret_cast<uint64_t>(a.q + int64_t(it.q0) * a.qs + int64_t(it.kvh) * G * D));
  const uint64_t db = uniform_u64(reinterpret_cast<uint64_t>(a.dout + int64_t(it.q0) * dstride + int64_t(it.kvh) * G * D));
  const uint64_t sb = uniform_u64(reinterpret_cast<uint64_t>((wave == 0 ? a.lse2 : a.ndelta) + int64_t(it.kvh) * G * a.q_rows + it.q0));

  // the pending tile load
  uint64_t lq = 0, ldo = 0, lstat = 0;
  const uint64_t qstep = uint64_t(a.qs) * (2 * NW * TL::kRowsPerInstr);
  const uint64_t dstep = uint64_t(dstride) * (2 * NW * TL::kRowsPerInstr);
  uint32_t lbuf = 0;
  bool lfull = false;
  auto prepare = [&](int b) __attribute__((always_inline)) {  // the next tile -> buffer b
    const uint64_t q = qb + uint64_t(ld.hg) * (2 * D), d = db + uint64_t(ld.hg) * (2 * D);
    const uint64_t s = sb + uint64_t(int64_t(ld.hg) * a.q_rows) * 4;
    lbuf = lds0 + b * L::kBuf;
    lfull = ld.tok + kDkvTile <= it.nq;
    if (lfull) {
      lq = q + uint64_t(int64_t(ld.tok) * a.qs) * 2;
      ldo = d + uint64_t(int64_t(ld.tok) * dstride) * 2;
      lstat = s + uint64_t(ld.tok) * 4;
    } else {
      swz_load_clamped<D, kDkvTile, NW>(lbuf, q, a.qs, 0, 0, it.nq, ld.tok, wave);
      swz_load_clamped<D, kDkvTile, NW>(lbuf + L::kTile, d, dstride, 0, 0, it.nq, ld.tok, wave);
      if (wave < 2) {  // rows past the sequence: LSE = +inf (P = 0), -D = 0
        const bool in = ld.tok + lane < it.nq;
        const float x = reinterpret_cast<const float*>(s)[min(ld.tok + lane, it.nq - 1)];
        lds_st_f(lbuf + 2 * L::kTile + wave * 256 + lane * 4, in ? x : wave == 0 ? INFINITY : 0.f);
      }
    }
    next(ld);
  };
  auto load = [&](int j) __attribute__((always_inline)) {  // load j of 2 kLoads + 1 of the pending tile
    if (!lfull) return;
    if (j < kLoads) lds_dma_x4_off(lq + j * qstep, qoff, lbuf + (wave + j * NW) * 1024);
    else if (j < 2 * kLoads) lds_dma_x4_off(ldo + (j - kLoads) * dstep, doff, lbuf + L::kTile + (wave + (j - kLoads) * NW) * 1024);
    else if (wave < 2) lds_dma_x1_off(lstat, lane * 4, lbuf + 2 * L::kTile + wave * 256);
  };
  __syncthreads();  // every wave is done with the buffers
  prepare(0);
#pragma unroll
  for (int j = 0; j <= 2 * kLoads; ++j) load(j);
  wait_vmem();
  __syncthreads();
#pragma unroll
  for (int kb = 0; kb < 4; ++kb) st.ds[kb] = bf16x8{};  // the half before the first adds 0

  // Tile t sits in buffer t % NB; iteration t loads tile t + 1 into buffer (t + 1) % NB, last read (as the half
  // before tile t - 1's first) in iteration t - 1, before the barrier that ended it.
  uint32_t qtp = lds0;
  int b = 0;
  for (int t = 0; t < T; ++t) {
    const uint32_t qt = lds0 + b * L::kBuf;
    const int rows = it.nq - cu.tok;
    int kv = 0;
    if constexpr (kDiagonal) kv = cu.tok + off + 4 * g - (it.start + wave * 64 + l16);
    next(cu);
    b = b + 1 == NB ? 0 : b + 1;
    lfull = false;
    if (t + 1 < T) prepare(b);
    if (active) {
      // the loads are spread over the groups of MFMAs
      dkv_half<D, kDiagonal ? 2 : 0>(st, ad, qt, qt + L::kTile, qt + 2 * L::kTile, qtp, sl2, kv,
                                     [&](int u) __attribute__((always_inline)) {
                                       if (u % kEvery == 0) load(u / kEvery);
                                       if (u == 2) load(2 * kLoads);
                                     });
      qtp = qt;
    }
    if (active && rows > 32) {
      dkv_half<D, kDiagonal ? 2 : 0>(st, ad, qt + 64 * D, qt + L::kTile + 64 * D, qt + 2 * L::kTile + 128, qtp, sl2,
                                     kv + 32, [&](int u) __attribute__((always_inline)) {
                                       if (u % kEvery == 0) load(kLoads + u / kEvery);
                                     });
      qtp = qt + 64 * D;
    } else {
#pragma unroll
      for (int j = 0; j <= 2 * kLoads; ++j)
        if (!active || (j >= kLoads && j < 2 * kLoads)) load(j);
    }
    wait_vmem();
    __syncthreads();
  }
  if (active) {  // dK of the last half
#pragma unroll
    for (int f = 0; f < D / 16; ++f) {
      const uint32_t x = (qtp + ad.tr) ^ (32 * f);
      const bf16x8 tf = cat8(lds_ld_tr(x), lds_ld_tr(x + 32 * D));
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) mfma16_agpr(st.dk[kb][f], tf, st.ds[kb]);
    }
  }
}

template <int D>
__device__ __forceinline__ void causal_dkv_item(const CausalArgs& a, const CausalItem& it, const unsigned char* lds) {
  constexpr int NC = D / 32, ND = D / 16;
  using L = DkvLds<D>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.heads / a.kv_heads;
  const bool active = wave * 64 < it.len;
  const uint32_t lds0 = lds_addr(lds), kl0 = lds0 + kDkvBufs * L::kBuf;

  // the item's keys: V and K fragments into VGPRs, K's upper head dims into LDS (as in dkv_item)
  const __bf16* const kp = a.k + int64_t(it.k0) * a.ks + int64_t(it.kvh) * D;
  const __bf16* const vp = a.v + int64_t(it.k0) * a.vs + int64_t(it.kvh) * D;
  if constexpr (D > 64)
    swz_load_clamped<64, kDkvKeyTile, kDkvWaves>(kl0, reinterpret_cast<uint64_t>(kp + 64), a.ks, 0, it.start, it.len, 0, wave);
  DkvState<D> st;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb) {
    const int r = wave * 64 + 16 * kb + l16;
    const int64_t row = it.start + min(r, it.len - 1);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bf16x8 y = ld8(vp + row * a.vs + g * 8 + c * 32);
      st.vf[kb][c] = (r < it.len) ? y : bf16x8{};
      if (c < kRegChunks) st.kf[kb][c] = ld8(kp + row * a.ks + g * 8 + c * 32);
    }
#pragma unroll
    for (int db = 0; db < ND; ++db) st.dk[kb][db] = st.dv[kb][db] = floatx4{};
  }
  // land them here, not at their first use inside the loop
#pragma unroll
  for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(st.vf[kb][c]));
#pragma unroll
    for (int c = 0; c < kRegChunks; ++c) asm volatile("" : "+v"(st.kf[kb][c]));
  }
  const DkvAddr ad{swz_row_addr<D>(), swz_tr_addr<D>(), kl0 + uint32_t(wave) * 64 * 128 + swz_row_addr<64>()};
  const uint32_t qoff = swz_load_off<D>(a.qs, 0, wave), doff = swz_load_off<D>(int64_t(a.heads) * D, 0, wave);

  const CausalTiles tiles = causal_tiles(it);
  const int full = G * (tiles.n - tiles.d);
  causal_dkv_tiles<D, false>(a, it, st, ad, tiles, G, it.lo, min(it.hi, full), lds0, qoff, doff, wave, active);
  causal_dkv_tiles<D, true>(a, it, st, ad, tiles, G, max(it.lo, full), it.hi, lds0, qoff, doff, wave, active);
  wait_vmem();  // of an item without tiles: no direct load outlives the workgroup
  mfma_drain();
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int db = 0; db < ND; ++db) asm volatile("" : "+a"(st.dk[kb][db]), "+a"(st.dv[kb][db]));

  if (!active) return;
  float* part = it.slot ? a.part_kv + int64_t(it.slot - 1) * 2 * kDkvKeyTile * D : nullptr;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb) {
    const int r = wave * 64 + 16 * kb + l16;
    if (r >= it.len) continue;
    if (part) {  // a piece of a split item
      float* p = part + r * D + 4 * g;
#pragma unroll
      for (int db = 0; db < ND; ++db) {
        *reinterpret_cast<floatx4*>(p + db * 16) = st.dk[kb][db];
        *reinterpret_cast<floatx4*>(p + kDkvKeyTile * D + db * 16) = st.dv[kb][db];
      }
      continue;
    }
    const int64_t out = (int64_t(it.k0 + it.start + r) * a.kv_heads + it.kvh) * D;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      bf16x4 wk, wv;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        wk[e] = (__bf16)(st.dk[kb][db][e] * a.scale);
        wv[e] = (__bf16)(st.dv[kb][db][e]);
      }
      *reinterpret_cast<bf16x4*>(a.dk + out + db * 16 + 4 * g) = wk;
      *reinterpret_cast<bf16x4*>(a.dv + out + db * 16 + 4 * g) = wv;
    }
  }
}

// --------------------------------------------------------------------------- dQ
// One 32-key half, plain, whose first key is key0: row block qb sees the keys up to lim[qb].
template <int D>
__device__ __forceinline__ void causal_dq_half(DqState<D>& st, const DqAddr& ad, uint32_t kt, uint32_t vt, int key0,
                                               const int* lim, float sl2) {
  constexpr int NC = D / 32;
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    floatx4 s[4], dp[4];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bf16x8 ka = lds_ld8(((kt + ad.row) ^ (64 * c)) + kb * 32 * D);
      const bf16x8 va = lds_ld8(((vt + ad.row) ^ (64 * c)) + kb * 32 * D);
#pragma unroll
      for (int qb = 0; qb < 4; ++qb) {
        s[qb] = mfma16(ka, st.qf[qb][c], c == 0 ? floatx4{} : s[qb]);
        dp[qb] = mfma16(va, st.df[qb][c], c == 0 ? st.nd[qb] : dp[qb]);
      }
    }
#pragma unroll
    for (int qb = 0; qb < 4; ++qb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = fast_exp2(fmaf(s[qb][i], sl2, -st.lse2[qb]));
        s[qb][i] = key0 + 16 * kb + 4 * g + i <= lim[qb] ? p : 0.f;
      }
    if (kb == 0) {
#pragma unroll
      for (int e = 0; e < 16; ++e) dq_ds(s, dp, st.ds, 0, e);
    } else {
#pragma unroll
      for (int qb = 0; qb < 4; ++qb) {
        st.p1[qb] = s[qb];
        st.dp1[qb] = dp[qb];
      }
    }
  }
  dq_flush<D>(st, ad, kt);
}

template <int D>
__device__ __forceinline__ void causal_dq_item(const CausalArgs& a, const CausalItem& it, const unsigned char* lds) {
  constexpr int NC = D / 32, ND = D / 16, BK = kDqTile, NB = kDqBufs;
  using TL = SwzTile<D, BK>;
  constexpr uint32_t kTileBytes = TL::kElems * 2;
  constexpr int kLoads = TL::kInstr / kDqWaves;  // of K, and of V, per wave and tile
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.heads / a.kv_heads, off = it.nk - it.nq;
  const bool active = wave * 64 < it.len;
  const float sl2 = a.scale_log2;
  const int64_t dstride = int64_t(a.heads) * D;
  const uint32_t lds0 = lds_addr(lds);

  // full tiles: those that end at or before the last key of the item's first row
  const int first_lim = __builtin_amdgcn_readfirstlane(it.start / G + off);
  const int T = max(0, (min(it.hi, first_lim + 1) - it.lo) >> 6);

  const __bf16* const k0 = a.k + int64_t(it.k0) * a.ks + int64_t(it.kvh) * D;
  const __bf16* const v0 = a.v + int64_t(it.k0) * a.vs + int64_t(it.kvh) * D;
  uint64_t kp = uniform_u64(reinterpret_cast<uint64_t>(k0 + int64_t(it.lo) * a.ks));
  uint64_t vp = uniform_u64(reinterpret_cast<uint64_t>(v0 + int64_t(it.lo) * a.vs));
  const uint64_t kline = uint64_t(a.ks) * 2, vline = uint64_t(a.vs) * 2;
  const uint32_t koff = swz_load_off<D>(a.ks, 0, wave), voff = swz_load_off<D>(a.vs, 0, wave);
  // the pending tile load: bases and LDS address of this wave's instructions
  uint64_t lk = 0, lv = 0;
  uint32_t lla = 0;
  const uint64_t kstep = kline * (kDqWaves * TL::kRowsPerInstr), vstep = vline * (kDqWaves * TL::kRowsPerInstr);
  auto prepare = [&](int b) __attribute__((always_inline)) {  // the next full tile -> buffer b
    lla = lds0 + b * 2 * kTileBytes + wave * 1024;
    lk = kp;
    lv = vp;
    kp += kline * BK;
    vp += vline * BK;
  };
  auto load = [&](int j) __attribute__((always_inline)) {  // load j of 2 kLoads of the pending tile
    if (j < kLoads) lds_dma_x4_off(lk + j * kstep, koff, lla + j * kDqWaves * 1024);
    else lds_dma_x4_off(lv + (j - kLoads) * vstep, voff, lla + kTileBytes + (j - kLoads) * kDqWaves * 1024);
  };
  for (int b = 0; b < 2 && b < T; ++b) {
    prepare(b);
#pragma unroll
    for (int j = 0; j < 2 * kLoads; ++j) load(j);
  }

  DqState<D> st;
#pragma unroll
  for (int qb = 0; qb < 4; ++qb) {
    const int r = wave * 64 + 16 * qb + l16, row = it.start + min(r, it.len - 1);
    const int token = row / G, h = it.kvh * G + row - token * G;
    const int64_t tok = it.q0 + token;
    const __bf16* qp = a.q + tok * a.qs + int64_t(h) * D + g * 8;
    const __bf16* dp = a.dout + tok * dstride + int64_t(h) * D + g * 8;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bf16x8 x = ld8(qp + c * 32);
      const bf16x8 y = ld8(dp + c * 32);
      st.qf[qb][c] = (r < it.len) ? x : bf16x8{};
      st.df[qb][c] = (r < it.len) ? y : bf16x8{};
    }
#pragma unroll
    for (int db = 0; db < ND; ++db) st.dq[qb][db] = floatx4{};
    st.lse2[qb] = a.lse2[int64_t(h) * a.q_rows + tok];
    const float x = a.ndelta[int64_t(h) * a.q_rows + tok];
    st.nd[qb] = floatx4{x, x, x, x};
    st.p1[qb] = st.dp1[qb] = floatx4{};  // the half before the first adds 0
    st.ds[qb] = bf16x8{};
  }
  // land the rows' loads here, not at their first use inside the loop
#pragma unroll
  for (int qb = 0; qb < 4; ++qb) {
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(st.qf[qb][c]), "+v"(st.df[qb][c]));
    asm volatile("" : "+v"(st.lse2[qb]), "+v"(st.nd[qb]));
  }
  const DqAddr ad{swz_row_addr<D>(), swz_tr_addr<D>()};
  wait_vmem();
  __syncthreads();

  // Tile t sits in buffer t % NB; iteration t loads tile t + 2 into buffer (t + 2) % NB (the last two iterations
  // the last tile again, into buffers that nothing reads by then).
  if (T > 0) {
    uint32_t ktp = lds0;
    int b = 0, bl = T > 1 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < kDqLook; ++i) st.ah[i] = lds_ld8(((lds0 + ad.row) ^ (64 * (i % NC))) + (i / NC) * 32 * D);
    for (int t = 0; t < T; ++t) {
      const uint32_t kt = lds0 + b * 2 * kTileBytes, vt = kt + kTileBytes;
      b = (b + 1) % NB;
      const uint32_t ktn = lds0 + b * 2 * kTileBytes;
      if (t + 2 < T) prepare(bl);
      else lla = lds0 + bl * 2 * kTileBytes + wave * 1024;
      bl = (bl + 1) % NB;
      if (active) {
        constexpr int kEvery = 3 * (D / 16) / (2 * kLoads);
        dq_half<D>(st, ad, kt, vt, ktp, kt + 64 * D, sl2, [&](int u) __attribute__((always_inline)) {
          if (u % kEvery == 0 && u / kEvery < 2 * kLoads) load(u / kEvery);
        });
        dq_half<D>(st, ad, kt + 64 * D, vt + 64 * D, kt, ktn, sl2, [](int) {});
        ktp = kt + 64 * D;
      } else {
#pragma unroll
        for (int j = 0; j < 2 * kLoads; ++j) load(j);
      }
      wait_vmem();
      block_barrier();
    }
    if (active) dq_flush<D>(st, ad, ktp);
  }
  int lim[4];  // the last key that this lane's row of each block sees
#pragma unroll
  for (int qb = 0; qb < 4; ++qb) lim[qb] = (it.start + min(wave * 64 + 16 * qb + l16, it.len - 1)) / G + off;
  // the other tiles, on the diagonal or ragged: rows past hi clamped to the last key before it, which no row sees
  // but those that see all of them
  const int wlast = __builtin_amdgcn_readfirstlane((it.start + min(wave * 64 + 64, it.len) - 1) / G + off);
  for (int key0 = it.lo + BK * T; key0 < it.hi; key0 += NB * BK) {
    __syncthreads();  // every wave is done with the buffers
    for (int j = 0; j < NB && key0 + j * BK < it.hi; ++j) {
      const uint32_t la = lds0 + j * 2 * kTileBytes;
      swz_load_clamped<D, BK, kDqWaves>(la, reinterpret_cast<uint64_t>(k0), a.ks, 0, 0, it.hi, key0 + j * BK, wave);
      swz_load_clamped<D, BK, kDqWaves>(la + kTileBytes, reinterpret_cast<uint64_t>(v0), a.vs, 0, 0, it.hi, key0 + j * BK, wave);
    }
    wait_vmem();
    __syncthreads();
    if (active)
      for (int o = 0; o < NB * BK && key0 + o < it.hi && key0 + o <= wlast; o += 32) {
        const uint32_t kt = lds0 + (o / BK) * 2 * kTileBytes + (o % BK) * 2 * D;
        causal_dq_half<D>(st, ad, kt, kt + kTileBytes, key0 + o, lim, sl2);
      }
  }
  mfma_drain();
#pragma unroll
  for (int qb = 0; qb < 4; ++qb)
#pragma unroll
    for (int db = 0; db < ND; ++db) asm volatile("" : "+a"(st.dq[qb][db]));

  if (!active) return;
  float* part = it.slot ? a.part_q + int64_t(it.slot - 1) * kDqQueryTile * D : nullptr;
#pragma unroll
  for (int qb = 0; qb < 4; ++qb) {
    const int r = wave * 64 + 16 * qb + l16;
    if (r >= it.len) continue;
    if (part) {  // a piece of a split item
#pragma unroll
      for (int db = 0; db < ND; ++db) *reinterpret_cast<floatx4*>(part + r * D + db * 16 + 4 * g) = st.dq[qb][db];
      continue;
    }
    const int row = it.start + r, token = row / G, h = it.kvh * G + row - token * G;
    __bf16* orow = a.dq + (int64_t(it.q0 + token) * a.heads + h) * D;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (__bf16)(st.dq[qb][db][e] * a.scale);
      *reinterpret_cast<bf16x4*>(orow + db * 16 + 4 * g) = w;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kDkvWaves * 64) __attribute__((amdgpu_waves_per_eu(1, 1)))
sra_causal_grad_kernel(CausalArgs a) {
  static_assert(kDkvWaves == kDqWaves && kDkvKeyTile == kCausalTile && kDqQueryTile == kCausalTile, "one block size");
  constexpr uint32_t kBytes = DkvLds<D>::kBytes > kDqLdsBytes<D> ? DkvLds<D>::kBytes : kDqLdsBytes<D>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kBytes];
  const CausalItem it = a.items[blockIdx.x];
  if (it.kind == kDkv) causal_dkv_item<D>(a, it, lds);
  else causal_dq_item<D>(a, it, lds);
}

// Sums of the split items' pieces, in piece order. D / 4 threads per row. Bound by reading the partial sums (23 MB:
// 6 us).
template <int D>
__global__ void __launch_bounds__(kThreads) sra_causal_grad_combine_kernel(CausalArgs a, const CausalItem* items) {
  constexpr int TPR = D / 4, RPB = kThreads / TPR;
  const CausalItem it = items[blockIdx.x];
  const int r = blockIdx.y * RPB + threadIdx.x / TPR, sub = threadIdx.x % TPR;
  if (r >= it.len) return;
  auto sum = [&](const float* p, int64_t slot, float scale, __bf16* dst) {
    floatx4 x = *reinterpret_cast<const floatx4*>(p);
#pragma unroll 4
    for (int i = 1; i < it.hi; ++i) x += *reinterpret_cast<const floatx4*>(p + i * slot);
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(x[e] * scale);
    *reinterpret_cast<bf16x4*>(dst) = y;
  };
  if (it.kind == kDkv) {
    constexpr int64_t slot = int64_t(2) * kCausalTile * D;
    const int64_t out = (int64_t(it.k0 + it.start + r) * a.kv_heads + it.kvh) * D + 4 * sub;
    const float* p = a.part_kv + it.lo * slot + r * D + 4 * sub;
    sum(p, slot, a.scale, a.dk + out);
    sum(p + kCausalTile * D, slot, 1.f, a.dv + out);
  } else {
    constexpr int64_t slot = int64_t(kCausalTile) * D;
    const int G = a.heads / a.kv_heads, row = it.start + r, token = row / G, h = it.kvh * G + row - token * G;
    sum(a.part_q + it.lo * slot + r * D + 4 * sub, slot, a.scale, a.dq + (int64_t(it.q0 + token) * a.heads + h) * D + 4 * sub);
  }
}

hipError_t launch_causal_delta(const CausalDeltaArgs& a, int head_dim, hipStream_t stream) {
  const int rpb = kThreads / (head_dim / 8);
  const int64_t blocks = (int64_t(a.q_rows) * a.heads + rpb - 1) / rpb;
  if (blocks == 0) return hipSuccess;
  if (head_dim == 128)
    hipLaunchKernelGGL(sra_causal_delta_kernel<128>, dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(sra_causal_delta_kernel<64>, dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_causal_grad(const CausalArgs& a, int n_items, int head_dim, hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  const dim3 grid(n_items), block(kDkvWaves * 64);
  if (head_dim == 128) hipLaunchKernelGGL(sra_causal_grad_kernel<128>, grid, block, 0, stream, a);
  else hipLaunchKernelGGL(sra_causal_grad_kernel<64>, grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_causal_grad_combine(const CausalArgs& a, const CausalItem* items, int n, int head_dim,
                                      hipStream_t stream) {
  if (n <= 0) return hipSuccess;
  const dim3 grid(n, kCausalTile * (head_dim / 4) / kThreads);
  if (head_dim == 128)
    hipLaunchKernelGGL(sra_causal_grad_combine_kernel<128>, grid, dim3(kThreads), 0, stream, a, items);
  else
    hipLaunchKernelGGL(sra_causal_grad_combine_kernel<64>, grid, dim3(kThreads), 0, stream, a, items);
  return hipGetLastError();
}

}  // namespace sra
