// Software-pipelined softmax attention over 64-key LDS tiles on 16x16x32 MFMAs: the per-wave state and
// steps of the forward kernels (what they do and why stands in sra_fwd.hip).
#pragma once
#include "sra_kernels.h"
#include "sra_tiles.h"

namespace sra {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kBigSum = 65536.0f;  // a lane's half-step sum of P above this forces a rescale
constexpr int kLook = 1;             // LDS fragments are read this many slot pairs ahead
constexpr int kWaves = 8;
template <int D> using KTile = PaddedTile<D, kFwdKeyStep, kPadRS<D>>;  // row-fragment reads
template <int D> using VTile = PaddedTile<D, kFwdKeyStep, kPadRS<D>>;  // transpose reads

template <int D, int NQ>
struct FwdState {
  bf16x8 qf[NQ][D / 32];  // Q^T MFMA B fragments of the 16-row blocks: lane = query, 8 head dims
  floatx4 o[NQ][D / 16];  // O^T accumulators, 16 head dims each
  float m[NQ];            // running max (log2 units)
  float l[NQ];            // per-lane partial row sum (fp32)
};

// Scores of a 32-key half for the wave's 16 NQ query rows: b[NQ * kb + qb] holds keys 16 kb .. + 15
// of row block qb. Element e of the flat order is register e % 4 of block e / 4.
template <int NQ>
struct HalfS {
  floatx4 b[2 * NQ];
};

// P of one 32-key half as the B fragments of the P V product, one per row block: elements 0..3
// are keys 4 g + i and elements 4..7 keys 16 + 4 g + i (g = lane / 16), the MFMA output's order.
template <int NQ>
struct HalfP {
  bf16x8 p[NQ];
};

// The first kLook K and V fragments of the next pipelined block, read during the last slots of
// the block before it (their tiles have landed by then, also across the barrier between tiles).
struct Ahead {
  bf16x8 k[kLook], v[kLook];
};

// How a 64-key LDS tile is laid out: padded rows (PaddedTile) or swizzled ones (SwzTile), whose load instructions hold
// whole rows. Both read their fragments without bank conflicts at compile-time offsets from a few per-lane addresses.
// k_frag: K row fragment i of the 32 keys at kt (A operand of S^T = K Q^T): keys 16 kb .. + 15 and head dims
//   32 c .. + 31, i = (D / 32) kb + c.
// v_frag: V^T fragment db of the 32 keys at vt (A operand of O^T += V^T P^T): head dims 16 db .. + 15. The transpose
//   read gives lane (head dim) the 8 keys whose P values the B fragment holds.
struct PaddedRows {
  template <int D>
  static __device__ __forceinline__ bf16x8 k_frag(const __bf16* kt, int i) {
    const int lane = threadIdx.x & 63, kb = i / (D / 32), c = i % (D / 32);
    return *reinterpret_cast<const bf16x8*>(kt + ((lane & 15) + 16 * kb) * kPadRS<D> + c * 32 + (lane >> 4) * 8);
  }
  template <int D>
  static __device__ __forceinline__ bf16x8 v_frag(const __bf16* vt, int db) {
    const int lane = threadIdx.x & 63;
    const int r0 = 4 * (lane >> 4) + ((lane & 15) >> 2), col = db * 16 + 4 * (lane & 3);
    return cat8(lds_read_tr(vt + r0 * kPadRS<D> + col), lds_read_tr(vt + (r0 + 16) * kPadRS<D> + col));
  }
};
struct SwizzledRows {
  template <int D>
  static __device__ __forceinline__ bf16x8 k_frag(const __bf16* kt, int i) {
    const int kb = i / (D / 32), c = i % (D / 32);
    return *reinterpret_cast<const bf16x8*>(kt + kb * 16 * D + (swz_row_addr<D>() ^ (64 * c)) / 2);
  }
  template <int D>
  static __device__ __forceinline__ bf16x8 v_frag(const __bf16* vt, int db) {
    const uint32_t x = (swz_tr_addr<D>() ^ (32 * db)) / 2;
    return cat8(lds_read_tr(vt + x), lds_read_tr(vt + 16 * D + x));
  }
};
template <int D, class L = PaddedRows>
__device__ __forceinline__ bf16x8 k_frag(const __bf16* kt, int i) {
  return L::template k_frag<D>(kt, i);
}
template <int D, class L = PaddedRows>
__device__ __forceinline__ bf16x8 v_frag(const __bf16* vt, int db) {
  return L::template v_frag<D>(vt, db);
}

// S^T of 32 keys, plain (used outside the pipeline).
template <int D, int NQ, class L = PaddedRows>
__device__ __forceinline__ HalfS<NQ> scores32(const FwdState<D, NQ>& st, const __bf16* kt) {
  HalfS<NQ> s;
#pragma unroll
  for (int j = 0; j < 2 * NQ; ++j) s.b[j] = floatx4{};
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const int kb = i / (D / 32), c = i % (D / 32);
    const bf16x8 k = k_frag<D, L>(kt, i);
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) s.b[NQ * kb + qb] = mfma16(k, st.qf[qb][c], s.b[NQ * kb + qb]);
  }
  return s;
}

template <int NQ>
__device__ __forceinline__ HalfP<NQ> pack_half(const HalfS<NQ>& s) {
  HalfP<NQ> h;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h.p[qb][i] = (__bf16)s.b[qb][i];
      h.p[qb][4 + i] = (__bf16)s.b[NQ + qb][i];
    }
  return h;
}

// Rare path: s holds S^T of a half (recomputed); move m to the true running max, rescale O
// and l, and leave P of the half in s and the lane's partial sums in sum.
template <int D, int NQ>
__device__ __forceinline__ void rescale_half(FwdState<D, NQ>& st, HalfS<NQ>& s, float sl2, float sum[NQ]) {
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    floatx4& a = s.b[qb];
    floatx4& b = s.b[NQ + qb];
    const float mx = quad_max(max2f(max3f(a[0], a[1], max2f(a[2], a[3])), max3f(b[0], b[1], max2f(b[2], b[3])))) * sl2;
    if (mx > st.m[qb]) {
      const float alpha = fast_exp2(st.m[qb] - mx);  // 0 when m was -inf
      st.m[qb] = mx;
      st.l[qb] *= alpha;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) st.o[qb][db] *= alpha;
    }
    // A row whose scores so far are all -inf (keys masked by an infinite head dim) keeps P = 0, wherever
    // its work item or piece begins.
    const float nm = st.m[qb] == -INFINITY ? 0.f : -st.m[qb];
    float acc = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = fast_exp2(fmaf(a[i], sl2, nm));
      b[i] = fast_exp2(fmaf(b[i], sl2, nm));
      acc += a[i] + b[i];
    }
    sum[qb] = acc;
  }
}

// The softmax work issued behind MFMA U of a block's 16 NQ (two per element of the half),
// software-pipelined so that instructions issued together never depend on each other: behind an
// even MFMA the exp2 of the element one ahead, behind an odd one the scale-and-shift FMA of the
// element two ahead and the row-sum add (with the bf16 pack of every second one) of element U / 2.
template <int E, int NQ>
__device__ __forceinline__ void soft_fma(HalfS<NQ>& s, const float* nm, float sl2) {
  if constexpr (E < 8 * NQ) s.b[E / 4][E % 4] = fmaf(s.b[E / 4][E % 4], sl2, nm[(E / 4) % NQ]);
}
template <int E, int NQ>
__device__ __forceinline__ void soft_exp(HalfS<NQ>& s) {
  if constexpr (E < 8 * NQ) s.b[E / 4][E % 4] = fast_exp2(s.b[E / 4][E % 4]);
}
template <int U, int NQ>
__device__ __forceinline__ void soft_step(HalfS<NQ>& s, const float* nm, float sl2, float* acc, HalfP<NQ>& out) {
  constexpr int e = U / 2, blk = e / 4, qb = blk % NQ, kb = blk / NQ, i = e % 4;
  if constexpr (U % 2 == 0) {
    soft_exp<e + 1>(s);
  } else {
    soft_fma<e + 2>(s, nm, sl2);
    acc[qb] += s.b[blk][i];
    if constexpr (i & 1) {
      const bf16x2 pr = {(__bf16)s.b[blk][i - 1], (__bf16)s.b[blk][i]};
      out.p[qb][4 * kb + i - 1] = pr[0];
      out.p[qb][4 * kb + i] = pr[1];
    }
  }
}

// MFMA U of a pipelined block (recursion over U): slots of NQ MFMAs sharing one LDS fragment
// alternate S^T of K fragment U / 2 NQ of the next half and P V of V fragment U / 2 NQ of a
// finished half. Each MFMA is followed by its softmax step (a 16x16x32 MFMA of 16 cycles hides
// about 8 cycles of vector work). Fragments LOOK slot pairs ahead are read from LDS. Scheduling
// barriers keep the order.
template <int U, int D, int NQ, int LOOK, class L>
__device__ __forceinline__ void pipe_slots(FwdState<D, NQ>& st, HalfS<NQ>& s_cur, HalfS<NQ>& sn, bf16x8* kf, bf16x8* vf,
                                           const __bf16* kq, const __bf16* vp, const __bf16* kn, const __bf16* vn,
                                           const HalfP<NQ>& pv, const float* nm, float sl2, float* acc,
                                           HalfP<NQ>& out) {
  constexpr int NC = D / 16;
  if constexpr (U < 2 * NC * NQ) {
    constexpr int I = U / (2 * NQ), qb = U % NQ;
    if constexpr (U % (2 * NQ) < NQ) {
      constexpr int kb = I / (D / 32), c = I % (D / 32);
      if constexpr (qb == 0) kf[I + LOOK] = I + LOOK < NC ? k_frag<D, L>(kq, I + LOOK) : k_frag<D, L>(kn, I + LOOK - NC);
      sn.b[NQ * kb + qb] = mfma16(kf[I], st.qf[qb][c], c == 0 ? floatx4{} : sn.b[NQ * kb + qb]);
    } else {
      if constexpr (qb == 0) vf[I + LOOK] = I + LOOK < NC ? v_frag<D, L>(vp, I + LOOK) : v_frag<D, L>(vn, I + LOOK - NC);
      st.o[qb][I] = mfma16(vf[I], pv.p[qb], st.o[qb][I]);
    }
    __builtin_amdgcn_sched_barrier(0);
    // D = 64 has one MFMA per element: both of an element's steps follow it
    if constexpr (D == 128) {
      soft_step<U>(s_cur, nm, sl2, acc, out);
    } else {
      soft_step<2 * U>(s_cur, nm, sl2, acc, out);
      soft_step<2 * U + 1>(s_cur, nm, sl2, acc, out);
    }
    __builtin_amdgcn_sched_barrier(0);
    pipe_slots<U + 1, D, NQ, LOOK, L>(st, s_cur, sn, kf, vf, kq, vp, kn, vn, pv, nm, sl2, acc, out);
  }
}

// One pipelined block. MFMA slots alternate S^T = K Q^T of the next half (K rows at kq, into
// s_next) and O^T += V^T P^T of a finished half (V rows at vp, P in pv); after each group of
// MFMAs one slice of the softmax of the current half (s_cur, whose K rows are at kc) is issued.
// Returns P of the current half. Slot order is fixed with scheduling barriers.
template <int D, int NQ, class L = PaddedRows>
__device__ __forceinline__ HalfP<NQ> pipe_block(FwdState<D, NQ>& st, HalfS<NQ>& s_cur, const __bf16* kc,
                                                HalfS<NQ>& s_next, const __bf16* kq, const __bf16* vp,
                                                const __bf16* kn, const __bf16* vn, Ahead& ah, const HalfP<NQ>& pv,
                                                float sl2) {
  constexpr int NC = D / 16;  // K fragments of a half (2 x D/32), V fragments of a half (D/16)
  float nm[NQ], acc[NQ];
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    nm[qb] = -st.m[qb];
    acc[qb] = 0.f;
  }
  HalfP<NQ> out;
  bf16x8 kf[NC + kLook], vf[NC + kLook];
#pragma unroll
  for (int i = 0; i < kLook; ++i) {
    kf[i] = ah.k[i];
    vf[i] = ah.v[i];
  }
  HalfS<NQ> sn;
  // prologue of the softmax pipeline: FMA of elements 0 and 1, exp2 of element 0
  soft_fma<0>(s_cur, nm, sl2);
  soft_fma<1>(s_cur, nm, sl2);
  soft_exp<0>(s_cur);
  pipe_slots<0, D, NQ, kLook, L>(st, s_cur, sn, kf, vf, kq, vp, kn, vn, pv, nm, sl2, acc, out);
  s_next = sn;
#pragma unroll
  for (int i = 0; i < kLook; ++i) {
    ah.k[i] = kf[NC + i];
    ah.v[i] = vf[NC + i];
  }
  // keep the bf16 packs in the slots above (not sunk past the rare-path branch)
  bool ok = true;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    asm volatile("" : "+v"(out.p[qb]));
    ok = ok && acc[qb] <= kBigSum;
  }
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(!ok) != 0, 0)) {
    s_cur = scores32<D, NQ, L>(st, kc);
    rescale_half<D, NQ>(st, s_cur, sl2, acc);
    out = pack_half<NQ>(s_cur);
  }
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) st.l[qb] += acc[qb];
  return out;
}

// O^T += V^T P^T for one half, plain.
template <int D, int NQ, class L = PaddedRows>
__device__ __forceinline__ void pv_half(FwdState<D, NQ>& st, const __bf16* vt, const HalfP<NQ>& h) {
#pragma unroll
  for (int db = 0; db < D / 16; ++db) {
    const bf16x8 v = v_frag<D, L>(vt, db);
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) st.o[qb][db] = mfma16(v, h.p[qb], st.o[qb][db]);
  }
}

// Masked half for the ragged tails (keys >= nvalid are outside the span); always takes the
// exact path (row max, rescale when it grew), since tails are rare.
template <int D, int NQ>
__device__ __forceinline__ void masked_half(FwdState<D, NQ>& st, const __bf16* kt, const __bf16* vt, int nvalid,
                                            float sl2) {
  const int g = (threadIdx.x & 63) >> 4;
  HalfS<NQ> s = scores32<D, NQ>(st, kt);
#pragma unroll
  for (int j = 0; j < 2 * NQ; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) s.b[j][i] = (16 * (j / NQ) + 4 * g + i) < nvalid ? s.b[j][i] : -INFINITY;
  float sum[NQ];
  rescale_half<D, NQ>(st, s, sl2, sum);
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) st.l[qb] += sum[qb];
  pv_half<D, NQ>(st, vt, pack_half<NQ>(s));
}

}  // namespace sra
