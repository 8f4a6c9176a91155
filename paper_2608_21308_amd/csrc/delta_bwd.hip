// Gated delta rule, backward chain over the chunks in reverse (mathematics and
// layouts: delta_common.h).  With dW the adjoint of the state at the chunk
// end, per chunk
//   dU = P^T dO + e^{b_C - b} K dW^T
//   Y  = T^T dU                       (dR = eta Y = dV)
//   dW_0 = G_C dW + sum_i s G_i dO_i q_i^T - sum_i eta_i G_i Y_i k_i^T.
// As in the forward, a wave owns 16 columns of dW^T and carries them in its
// accumulators; dW at every chunk end and Y are left for the gradients that
// sum over the value dimension (delta_grads.hip).  Long chains of few units run
// as segments (delta_fwd.hip): a segment with the transition F takes the
// adjoint at its end to dW F^T + B at its start.  256 units of 64, 64 chunks: 295
// us, 5.2 TB/s of the 93 KB that a chunk moves; 128 units 237 us, 3.7 us a chunk.
#include "delta_grads.h"

namespace e2ttt {
namespace {

// LDS of a workgroup (offsets in bytes).
template <bool BF, int DK, int NW, bool STATE>
struct BwdLds {
  static constexpr int e = (int)sizeof(typename DOp<BF>::E), ks = kDC * DK * e;
  static constexpr int qs = ks, vs = qs + (ks), ts = vs + kDC * 16 * NW * e;
  static constexpr int gl = ts + 2 * tri_bytes(BF), bytes = gl + kGateChain * 4;
};

// STATE: only the adjoint at every segment's start, from zero at its end.
template <bool BF, int DK, int NW, bool STATE>
__device__ __forceinline__ void bwd_chain(const DeltaArgs& a, int nsl, long blk, char* lds) {
  using O = DOp<BF>;
  using E = typename O::E;
  using L = LTile<BF, DK>;
  using LV = LTile<BF, 16 * NW>;
  constexpr unsigned ES = sizeof(E);
  constexpr int NTH = 64 * NW, KT = DK / 32, MT = DK / 16;
  constexpr int PK = kDC * L::NP / NTH, PV = kDC * LV::NP / NTH;
  constexpr int NF = 2 * tri_bytes(BF) / 16;   // pieces of T and P
  constexpr int PF = (NF + NTH - 1) / NTH;
  static_assert(kDC * L::NP % NTH == 0 && NTH % L::NP == 0 && NTH % LV::NP == 0,
                "whole rounds of pieces");
  using M = BwdLds<BF, DK, NW, STATE>;
  E* ks = reinterpret_cast<E*>(lds);
  E* qs = reinterpret_cast<E*>(lds + M::qs);
  E* vs = reinterpret_cast<E*>(lds + M::vs);             // dO rows
  char* ts = lds + M::ts;                                // T, then P
  float* gl = reinterpret_cast<float*>(lds + M::gl);

  const char* ps = ts + tri_bytes(BF);
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = wave_id();
  const long U = (long)a.B * a.H;
  const long us = (blk / (8 * nsl)) * 8 + blk % 8;       // (unit, segment)
  if (us >= U * a.nseg) return;
  const int u = __builtin_amdgcn_readfirstlane((int)(us / a.nseg));
  const int seg = __builtin_amdgcn_readfirstlane((int)(us % a.nseg));
  if (STATE && seg == 0) return;
  const int sl = (int)((blk / 8) % nsl);
  const int b = u / a.H, h = u % a.H, hk = h / (a.H / a.HK);
  const int nlive = live_tokens(a, b);
  const int r0 = a.r0 + seg * a.seglen;                  // (up to the sequence's last chunk)
  const int r1 = min(min(a.r1, r0 + a.seglen), (nlive + kDC - 1) / kDC);
  const int sc0 = sl * NW * 16, col = sc0 + 16 * w + c, tile = sl * NW + w;
  const unsigned sat = tile < a.dvp / 16 ? 0 : kNowhere;   // (no stores behind the value channels)
  const int krow = tid / L::NP, kcol = (tid % L::NP) * L::PE;
  const int vrow = tid / LV::NP, vcol = (tid % LV::NP) * LV::PE;
  const bool kok = kcol < a.dk, vok = sc0 + vcol < a.dv;
  const int kst = (int)a.k.t, qst = (int)a.q.t, vst = (int)a.d_out.t;

  f32x4 st[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int kc = lab(m, 4 * g);
    st[m] = zero4();
    if constexpr (STATE) continue;
    if (a.nseg > 1) {
      if (col < a.dvp)
        st[m] = *reinterpret_cast<const f32x4*>(a.segs + us * a.dvp * DK +
                                                lane_at(tile, m / 2, KT, lane) + 256 * (m & 1));
    } else if (a.d_w_out && col < a.dv && kc < a.dk) {
      st[m] = *reinterpret_cast<const f32x4*>(a.d_w_out + ((long)u * a.dv + col) * a.dk + kc);
    }
  }

  u32x4 rk[PK], rq[PK], rv[PV];
  u32x4 rf[PF], rg;
  // byte offsets within a chunk
  const unsigned kat = (unsigned)(krow * kst + kcol) * ES, qat = (unsigned)(krow * qst + kcol) * ES;
  const unsigned vat = (unsigned)(vrow * vst + vcol) * ES;
  auto fetch = [&](int r) {
    const int t0 = r * kDC, nt = nlive - t0;
    const long cu = (long)u * a.nc_buf + (r - a.r_base);
    const Buf kb = buf_of(row_of<E>(a.k, b, hk, t0)), qb = buf_of(row_of<E>(a.q, b, hk, t0));
    const Buf vb = buf_of(row_of<E>(a.d_out, b, h, t0) + sc0);
#pragma unroll
    for (int x = 0; x < PK; ++x) {
      const int row = krow + x * (NTH / L::NP);
      const unsigned no = kok && row < nt ? 0 : kNowhere;
      rk[x] = buf_ld(kb, (kat + (unsigned)(x * (NTH / L::NP) * kst) * ES) | no);
      rq[x] = buf_ld(qb, (qat + (unsigned)(x * (NTH / L::NP) * qst) * ES) | no);
    }
#pragma unroll
    for (int x = 0; x < PV; ++x) {
      const unsigned no = vok && vrow + x * (NTH / LV::NP) < nt ? 0 : kNowhere;
      rv[x] = buf_ld(vb, (vat + (unsigned)(x * (NTH / LV::NP) * vst) * ES) | no);
    }
    const Buf fb = buf_of(a.frag + cu * 2 * tri_bytes(BF));
#pragma unroll
    for (int x = 0; x < PF; ++x) rf[x] = buf_ld(fb, 16 * min(tid + x * NTH, NF - 1));   // (the last piece by several)
    rg = buf_ld(buf_of(a.gate + cu * kGateFloats), 16 * min(tid, kGateChain / 4 - 1));
  };
  auto stage = [&]() {
#pragma unroll
    for (int x = 0; x < PK; ++x) {
      const int at = L::at(krow + x * (NTH / L::NP), tid % L::NP);
      *reinterpret_cast<u32x4*>(ks + at) = rk[x];
      *reinterpret_cast<u32x4*>(qs + at) = rq[x];
    }
#pragma unroll
    for (int x = 0; x < PV; ++x)
      *reinterpret_cast<u32x4*>(vs + LV::at(vrow + x * (NTH / LV::NP), tid % LV::NP)) = rv[x];
#pragma unroll
    for (int x = 0; x < PF; ++x)
      reinterpret_cast<u32x4*>(ts)[min(tid + x * NTH, NF - 1)] = rf[x];
    if (tid < kGateChain / 4) *reinterpret_cast<u32x4*>(gl + 4 * tid) = rg;
  };
  if (r0 < r1) {
    fetch(r1 - 1);
    stage();
  }

  for (int r = r1 - 1; r >= r0; --r) {
    const long cu = (long)u * a.nc_buf + (r - a.r_base);
    __syncthreads();
    if (r > r0) fetch(r - 1);

    const Buf wb = buf_of(a.dwst + cu * a.dvp * DK), yb = buf_of(a.yst + cu * a.dvp * kDC);
    typename O::S sb[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      sb[kt] = O::split(st[2 * kt], st[2 * kt + 1]);
      if constexpr (!STATE) {
        const unsigned at = sat + 4 * (unsigned)lane_at(tile, kt, KT, lane);
        buf_st(wb, at, st[2 * kt]);
        buf_st(wb, at + 1024, st[2 * kt + 1]);
      }
    }
    f32x4 xa[4];
#pragma unroll
    for (int m = 0; m < 4; m += 2) {
      xa[m] = xa[m + 1] = zero4();
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
        O::xs2(xa[m], L::frag(ks, lab(m, c), kt, g), sb[kt], xa[m + 1],
               L::frag(ks, lab(m + 1, c), kt, g), sb[kt]);
      xa[m] = xa[m] * *reinterpret_cast<const f32x4*>(gl + kGEnd + lab(m, 4 * g));
      xa[m + 1] = xa[m + 1] * *reinterpret_cast<const f32x4*>(gl + kGEnd + lab(m + 1, 4 * g));
    }
    typename O::X dob[2];           // dO as an operand
    typename O::S gb[2];            // s G dO
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      dob[x] = LV::template frag_t<true>(vs, w, x, g, c);
      f32x4 d0, d1;
      O::values(dob[x], d0, d1);
      gb[x] = O::split(
          d0 * *reinterpret_cast<const f32x4*>(gl + kGsG + 32 * x + 8 * g),
          d1 * *reinterpret_cast<const f32x4*>(gl + kGsG + 32 * x + 8 * g + 4));
    }
#pragma unroll
    for (int m = 0; m < 4; m += 2)
#pragma unroll
      for (int x = m / 2; x < 2; ++x)
        O::sx2(xa[m], ld_frag_t<BF>(ps, m, x, g, c), dob[x], xa[m + 1],
               ld_frag_t<BF>(ps, m + 1, x, g, c), dob[x]);
    typename O::S rb[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) rb[x] = O::split(xa[2 * x], xa[2 * x + 1]);
    const float gC = gl[kGC];
#pragma unroll
    for (int m = 0; m < MT; m += 2) {  // (needs nothing of Y: fills the waits of its products)
      st[m] = st[m] * gC;
      st[m + 1] = st[m + 1] * gC;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        O::xs2(st[m], L::template frag_t<false>(qs, m, x, g, c), gb[x], st[m + 1],
               L::template frag_t<false>(qs, m + 1, x, g, c), gb[x]);
    }
#pragma unroll
    for (int m = 0; m < 4; m += 2) {
      xa[m] = xa[m + 1] = zero4();
#pragma unroll
      for (int x = m / 2; x < 2; ++x)
        O::ss2(xa[m], ld_frag_t<BF>(ts, m, x, g, c), rb[x], xa[m + 1],
               ld_frag_t<BF>(ts, m + 1, x, g, c), rb[x]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if constexpr (!STATE) {
        const unsigned at = sat + 4 * (unsigned)lane_at(tile, x, 2, lane);
        buf_st(yb, at, xa[2 * x]);
        buf_st(yb, at + 1024, xa[2 * x + 1]);
      }
      const float* gp = gl + kGEtaG + 32 * x + 8 * g;
      rb[x] = O::split(xa[2 * x] * -*reinterpret_cast<const f32x4*>(gp),
                       xa[2 * x + 1] * -*reinterpret_cast<const f32x4*>(gp + 4));
    }
#pragma unroll
    for (int m = 0; m < MT; m += 2)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        O::xs2(st[m], L::template frag_t<false>(ks, m, x, g, c), rb[x], st[m + 1],
               L::template frag_t<false>(ks, m + 1, x, g, c), rb[x]);
    if (r > r0) {
      __syncthreads();                       // (the chunk in LDS is done with)
      stage();
    }
  }

  if constexpr (STATE) {
    if (col < a.dvp) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
        st_lane(a.segb + us * a.dvp * DK + lane_at(tile, kt, KT, lane), st[2 * kt], st[2 * kt + 1]);
    }
    return;
  }
  if (a.d_w_in && seg == 0) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int kc = lab(m, 4 * g);
      if (col < a.dv && kc < a.dk)
        *reinterpret_cast<f32x4*>(a.d_w_in + ((long)u * a.dv + col) * a.dk + kc) = st[m];
    }
  }
}

// (f32 io: one wave a SIMD, as in the forward: a step of 256 units of 64, 16
// chunks, 592 us against 693.)
template <bool BF, int DK, int NW, bool STATE>
__global__ void __launch_bounds__(64 * NW, BF && (NW == 8 || DK <= 64) ? 2 : 1)
delta_bwd_kernel(DeltaArgs a, int nsl) {
  __shared__ __align__(16) char lds[BwdLds<BF, DK, NW, STATE>::bytes];
  bwd_chain<BF, DK, NW, STATE>(a, nsl, blockIdx.x, lds);
}

template <bool BF, int DK, int NW>
hipError_t go(const DeltaArgs& a, bool state, hipStream_t s) {
  const int nsl = (a.dvp + 16 * NW - 1) / (16 * NW);
  const long u8 = ((long)a.B * a.H * a.nseg + 7) / 8 * 8;
  const dim3 grid((unsigned)(u8 * nsl)), blk(64 * NW);
  if (state)
    hipLaunchKernelGGL((delta_bwd_kernel<BF, DK, NW, true>), grid, blk, 0, s, a, nsl);
  else
    hipLaunchKernelGGL((delta_bwd_kernel<BF, DK, NW, false>), grid, blk, 0, s, a, nsl);
  return hipGetLastError();
}

// The first `nchain` workgroups run the chain, those behind them form the
// gradients of the ng chunks from g0 on, which the launch before has passed.
template <bool ONE>
__global__ void __launch_bounds__(256, 2)
delta_bwd_grads_kernel(DeltaArgs a, int nsl, int nchain, int g0, int ng) {
  constexpr int kChain = BwdLds<true, 64, 4, false>::bytes, kGrads = GradsLds<true, 64, 4>::bytes;
  __shared__ __align__(16) char lds[kChain > kGrads ? kChain : kGrads];
  if ((int)blockIdx.x < nchain)
    bwd_chain<true, 64, 4, false>(a, nsl, blockIdx.x, lds);
  else
    grads_chunk<true, 64, 4, ONE>(a, g0, ng, blockIdx.x - nchain, lds);
}

}  // namespace

hipError_t launch_delta_chain_bwd_grads(const DeltaArgs& a, int g0, int ng, hipStream_t s) {
  const int nsl = (a.dvp + 63) / 64;
  const long nchain = ((long)a.B * a.H + 7) / 8 * 8 * nsl;
  const dim3 grid((unsigned)(nchain + (long)a.B * a.HK * ng)), blk(256);
  if (a.H == a.HK)
    hipLaunchKernelGGL((delta_bwd_grads_kernel<true>), grid, blk, 0, s, a, nsl, (int)nchain, g0, ng);
  else
    hipLaunchKernelGGL((delta_bwd_grads_kernel<false>), grid, blk, 0, s, a, nsl, (int)nchain, g0, ng);
  return hipGetLastError();
}

hipError_t launch_delta_chain_bwd(const DeltaArgs& a, bool bf, bool state, hipStream_t s) {
  const int dkp = delta_dkp(a.dk);
  if (bf) {
    if (dkp == 32) return go<true, 32, 2>(a, state, s);
    if (dkp == 64) return go<true, 64, 4>(a, state, s);
    // (as in the forward; a step of 256 units of 128, 16 chunks, takes 870 us with either)
    if ((long)a.B * a.H * a.nseg * ((a.dvp / 16 + 7) / 8) <= 128) return go<true, 128, 4>(a, state, s);
    return go<true, 128, 8>(a, state, s);
  }
  if (dkp == 32) return go<false, 32, 2>(a, state, s);
  if (dkp == 64) return go<false, 64, 4>(a, state, s);
  return go<false, 128, 4>(a, state, s);
}

}  // namespace e2ttt
