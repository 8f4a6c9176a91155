// Gated delta rule, forward chain over the chunks (the mathematics and the
// layouts: delta_common.h).
//
// A wave owns 16 columns of W^T (rows of the state: value channels), which
// depend on each other in nothing, and keeps them in fp32 accumulators for the
// whole sequence; a workgroup is NW waves of one unit that share the staged
// chunk (K, Q, V rows and the T, P fragments).  Per chunk a wave takes
//   X = K W^T,  U = T (eta V - eta G X)
//   O = s G Q W^T + P U              -> out
//   W^T = G_C W^T + K^T (e^{b_C - b} U)
// with every accumulator turned into the next product's operand in place.  O
// is formed transposed (operands exchanged), so that a lane holds four
// neighbouring channels of a token and stores them at once.  The next chunk's
// global loads are issued before the current one's products.
//
// With 256 units of 64 and more it is bound by HBM (saving: 101 KB a chunk, 64
// chunks in 443 us, 3.8 TB/s; matrix units busy for 16 %, vector units for 18 %);
// with fewer by one chunk's chain of dependent products and conversions, with 128
// units of dk = 64 3.9 us saving and 3.7 us without, of 128 and two waves a SIMD 7.5.
//
// A chain is as long as its sequence, and few units leave most of the card
// idle.  The chunks then run as segments: what a segment makes of a state is
// W -> W F + B, so a first pass takes B (the columns above from zero) and F
// (dk more columns, from the unit matrix, with V = 0) of every segment at
// once, delta_join.hip forms the states that the segments start from, and
// this pass runs them all at once.  Some more units leave CUs idle whose own
// chains segments would not shorten: there the launch takes a part of the chain
// beside the preparation of the next (delta_api.hip holds the rules of both).
#include "delta_prep.h"

namespace e2ttt {
namespace {

enum { kPlain = 0, kSave = 1, kState = 2 };

// LDS of a workgroup (offsets in bytes).
template <bool BF, int DK, int NW, int MODE>
struct FwdLds {
  static constexpr int e = (int)sizeof(typename DOp<BF>::E), ks = kDC * DK * e;
  static constexpr int qs = ks, vs = qs + (MODE != kState ? ks : 0), ts = vs + kDC * 16 * NW * e;
  static constexpr int gl = ts + (MODE != kState ? 2 : 1) * tri_bytes(BF), bytes = gl + kGateChain * 4;
};

template <bool BF, int DK, int NW, int MODE>
__device__ __forceinline__ void fwd_chain(const DeltaArgs& a, int nsl, long blk, char* lds) {
  constexpr bool SAVE = MODE == kSave, OUT = MODE != kState;
  using O = DOp<BF>;
  using E = typename O::E;
  using L = LTile<BF, DK>;
  using LV = LTile<BF, 16 * NW>;
  constexpr unsigned ES = sizeof(E);
  constexpr int NTH = 64 * NW, KT = DK / 32, MT = DK / 16;
  constexpr int PK = kDC * L::NP / NTH;                 // a thread's pieces of K (Q) rows
  constexpr int PV = kDC * LV::NP / NTH;                // and of V rows
  constexpr int NF = (OUT ? 2 : 1) * tri_bytes(BF) / 16;   // pieces of T and P
  constexpr int PF = (NF + NTH - 1) / NTH;
  static_assert(kDC * L::NP % NTH == 0 && NTH % L::NP == 0 && NTH % LV::NP == 0,
                "whole rounds of pieces");
  using M = FwdLds<BF, DK, NW, MODE>;
  E* ks = reinterpret_cast<E*>(lds);
  E* qs = reinterpret_cast<E*>(lds + M::qs);
  E* vs = reinterpret_cast<E*>(lds + M::vs);
  char* ts = lds + M::ts;                                // T, then P
  float* gl = reinterpret_cast<float*>(lds + M::gl);

  const char* ps = ts + tri_bytes(BF);
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = wave_id();
  // the slices of a unit go to one XCD (workgroups are dealt to the eight in turn)
  const long U = (long)a.B * a.H;
  const long us = (blk / (8 * nsl)) * 8 + blk % 8;       // (unit, segment)
  if (us >= U * a.nseg) return;
  const int u = __builtin_amdgcn_readfirstlane((int)(us / a.nseg));
  const int seg = __builtin_amdgcn_readfirstlane((int)(us % a.nseg));
  const int r0 = a.r0 + seg * a.seglen, r1 = min(a.r1, r0 + a.seglen);
  const int sl = (int)((blk / 8) % nsl);
  // (nothing starts behind the last segment; the backward wants its transition)
  if (MODE == kState && seg == a.nseg - 1 && (!a.save || (sl + 1) * NW <= a.dvp / 16)) return;
  const int b = u / a.H, h = u % a.H, hk = h / (a.H / a.HK);
  const int nlive = live_tokens(a, b);
  const int rl = min(r1, (nlive + kDC - 1) / kDC);       // chunks up to the sequence's end (zeros behind)
  const int sc0 = sl * NW * 16;                          // the workgroup's first column
  const int col = sc0 + 16 * w + c;                      // the lane's
  const int tile = sl * NW + w, nvt = a.dvp / 16;        // the wave's tile: of B, or behind them of F
  const unsigned sat = tile < a.dvp / 16 ? 0 : kNowhere;   // (no stores behind the value channels)
  // thread offsets within a chunk (32 bits: rows are at most 2^23 elements apart)
  const int krow = tid / L::NP, kcol = (tid % L::NP) * L::PE;
  const int vrow = tid / LV::NP, vcol = (tid % LV::NP) * LV::PE;
  const bool kok = kcol < a.dk, vok = sc0 + vcol < a.dv;
  const int kst = (int)a.k.t, qst = (int)a.q.t, vst = (int)a.v.t, ost = (int)a.out.t;

  f32x4 st[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int kc = lab(m, 4 * g);
    st[m] = zero4();
    if constexpr (MODE == kState) {
#pragma unroll
      for (int e = 0; e < 4; ++e) st[m][e] = 16 * (tile - nvt) + c == kc + e ? 1.0f : 0.0f;
    } else if (a.nseg > 1) {
      if (col < a.dvp)
        st[m] = *reinterpret_cast<const f32x4*>(a.segs + us * a.dvp * DK +
                                                lane_at(tile, m / 2, KT, lane) + 256 * (m & 1));
    } else if (a.w_in && col < a.dv && kc < a.dk) {
      st[m] = *reinterpret_cast<const f32x4*>(a.w_in + ((long)u * a.dv + col) * a.dk + kc);
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
    const Buf vb = buf_of(row_of<E>(a.v, b, h, t0) + sc0);
#pragma unroll
    for (int x = 0; x < PK; ++x) {
      const int row = krow + x * (NTH / L::NP);
      const unsigned no = kok && row < nt ? 0 : kNowhere;
      rk[x] = buf_ld(kb, (kat + (unsigned)(x * (NTH / L::NP) * kst) * ES) | no);
      if constexpr (OUT) rq[x] = buf_ld(qb, (qat + (unsigned)(x * (NTH / L::NP) * qst) * ES) | no);
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
      if constexpr (OUT) *reinterpret_cast<u32x4*>(qs + at) = rq[x];
    }
#pragma unroll
    for (int x = 0; x < PV; ++x)
      *reinterpret_cast<u32x4*>(vs + LV::at(vrow + x * (NTH / LV::NP), tid % LV::NP)) = rv[x];
#pragma unroll
    for (int x = 0; x < PF; ++x)
      reinterpret_cast<u32x4*>(ts)[min(tid + x * NTH, NF - 1)] = rf[x];
    if (tid < kGateChain / 4) *reinterpret_cast<u32x4*>(gl + 4 * tid) = rg;
  };
  if (r0 < rl) {
    fetch(r0);
    stage();
  }

  for (int r = r0; r < rl; ++r) {
    const int t0 = r * kDC;
    const long cu = (long)u * a.nc_buf + (r - a.r_base);
    __syncthreads();
    if (r + 1 < rl) fetch(r + 1);

    const Buf wb = buf_of(a.wst + cu * a.dvp * DK), ub_ = buf_of(a.ust + cu * a.dvp * kDC);
    // X, per 32 columns of the state
    typename O::S sb[KT];
    f32x4 xa[4], oa[4], ua[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) xa[m] = oa[m] = ua[m] = zero4();
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      sb[kt] = O::split(st[2 * kt], st[2 * kt + 1]);
      if constexpr (SAVE) {
        const unsigned at = sat + 4 * (unsigned)lane_at(tile, kt, KT, lane);
        buf_st(wb, at, st[2 * kt]);
        buf_st(wb, at + 1024, st[2 * kt + 1]);
      }
#pragma unroll
      for (int m = 0; m < 4; m += 2)
        O::xs2(xa[m], L::frag(ks, lab(m, c), kt, g), sb[kt], xa[m + 1],
               L::frag(ks, lab(m + 1, c), kt, g), sb[kt]);
    }
    // R, and while it is formed the state's part of O
    typename O::S rb[2], ub[2], ue[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      f32x4 v0, v1;
      O::values(LV::template frag_t<true>(vs, w, x, g, c), v0, v1);
      const float* gp = gl + 32 * x + 8 * g;
      const f32x4 e0 = *reinterpret_cast<const f32x4*>(gp + kGEta);
      const f32x4 e1 = *reinterpret_cast<const f32x4*>(gp + kGEta + 4);
      const f32x4 h0 = *reinterpret_cast<const f32x4*>(gp + kGEtaG);
      const f32x4 h1 = *reinterpret_cast<const f32x4*>(gp + kGEtaG + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        xa[2 * x][e] = fmaf(-h0[e], xa[2 * x][e], e0[e] * v0[e]);
        xa[2 * x + 1][e] = fmaf(-h1[e], xa[2 * x + 1][e], e1[e] * v1[e]);
      }
      rb[x] = O::split(xa[2 * x], xa[2 * x + 1]);
      if constexpr (OUT) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
          O::sx2(oa[2 * x], sb[kt], L::frag(qs, lab(2 * x, c), kt, g), oa[2 * x + 1],
                 sb[kt], L::frag(qs, lab(2 * x + 1, c), kt, g));
        oa[2 * x] = oa[2 * x] * gl[kGsG + lab(2 * x, c)];
        oa[2 * x + 1] = oa[2 * x + 1] * gl[kGsG + lab(2 * x + 1, c)];
      }
    }
    // U, half by half; the first half's use overlaps the second's products
    const float gC = gl[kGC];
#pragma unroll
    for (int m = 0; m < MT; ++m) st[m] = st[m] * gC;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int y = 0; y <= x; ++y)
        O::ss2(ua[2 * x], ld_frag<BF>(ts, fidx(2 * x, y), lane), rb[y], ua[2 * x + 1],
               ld_frag<BF>(ts, fidx(2 * x + 1, y), lane), rb[y]);
      if constexpr (SAVE) {
        const unsigned at = sat + 4 * (unsigned)lane_at(tile, x, 2, lane);
        buf_st(ub_, at, ua[2 * x]);
        buf_st(ub_, at + 1024, ua[2 * x + 1]);
      }
      const f32x4 n0 = *reinterpret_cast<const f32x4*>(gl + kGEnd + 32 * x + 8 * g);
      const f32x4 n1 = *reinterpret_cast<const f32x4*>(gl + kGEnd + 32 * x + 8 * g + 4);
      ue[x] = O::split(ua[2 * x] * n0, ua[2 * x + 1] * n1);
      if constexpr (OUT) ub[x] = O::split(ua[2 * x], ua[2 * x + 1]);
#pragma unroll
      for (int m = 0; m < MT; m += 2)
        O::xs2(st[m], L::template frag_t<false>(ks, m, x, g, c), ue[x], st[m + 1],
               L::template frag_t<false>(ks, m + 1, x, g, c), ue[x]);
    }
    if constexpr (OUT) {
    const Buf ob = buf_of(row_of<E>(a.out, b, h, t0) + sc0);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      if (m % 2 == 0) {
#pragma unroll
        for (int x = 0; x <= m / 2; ++x)
          O::ss2(oa[m], ub[x], ld_frag<BF>(ps, fidx(m, x), lane), oa[m + 1], ub[x],
                 ld_frag<BF>(ps, fidx(m + 1, x), lane));
      }
      const unsigned no = sc0 + 16 * w + 4 * g < a.dv && t0 + lab(m, c) < nlive ? 0 : kNowhere;
      buf_st_io<BF>(ob, (unsigned)(lab(m, c) * ost + 16 * w + 4 * g) * ES | no, oa[m]);
    }
    }
    if (r + 1 < rl) {
      __syncthreads();                       // (the chunk in LDS is done with)
      stage();
    }
  }

  if constexpr (OUT) {
    const int t1 = (int)min((long)r1 * kDC, (long)a.T);
    for (int t = max(r0 * kDC, nlive) + vrow; t < t1; t += NTH / LV::NP)
      if (vok)
        *reinterpret_cast<u32x4*>(row_of_w<E>(a.out, b, h, t) + sc0 + vcol) = u32x4{0, 0, 0, 0};
  }
  if constexpr (MODE == kState) {
    if (tile < nvt) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
        st_lane(a.segb + us * a.dvp * DK + lane_at(tile, kt, KT, lane), st[2 * kt], st[2 * kt + 1]);
    } else if (tile < nvt + MT) {
      float* f = a.segf + us * 2 * DK * DK;
      const int row = 16 * (tile - nvt) + c;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
        st_lane(f + lane_at(tile - nvt, kt, KT, lane), st[2 * kt], st[2 * kt + 1]);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) f[DK * DK + operand_at(lab(m, 4 * g) + e, row, KT)] = st[m][e];
    }
    return;
  }
  if (a.w_out && seg == a.nseg - 1) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int kc = lab(m, 4 * g);
      if (col < a.dv && kc < a.dk)
        *reinterpret_cast<f32x4*>(a.w_out + ((long)u * a.dv + col) * a.dk + kc) = st[m];
    }
  }
}

// (f32 io: one wave a SIMD, as 256 registers would spill some 40: 256 units of 64,
// 16 chunks, 187 us against 262)
template <bool BF, int DK, int NW, int MODE>
__global__ void __launch_bounds__(64 * NW, BF && (NW == 8 || DK <= 64) ? 2 : 1)
delta_fwd_kernel(DeltaArgs a, int nsl) {
  __shared__ __align__(16) char lds[FwdLds<BF, DK, NW, MODE>::bytes];
  fwd_chain<BF, DK, NW, MODE>(a, nsl, blockIdx.x, lds);
}

template <bool BF, int DK, int NW>
hipError_t go(const DeltaArgs& a, bool save, bool state, hipStream_t s) {
  const int tiles = a.dvp / 16 + (state ? DK / 16 : 0), nsl = (tiles + NW - 1) / NW;
  const long u8 = ((long)a.B * a.H * a.nseg + 7) / 8 * 8;
  const dim3 grid((unsigned)(u8 * nsl)), blk(64 * NW);
  if (state)
    hipLaunchKernelGGL((delta_fwd_kernel<BF, DK, NW, kState>), grid, blk, 0, s, a, nsl);
  else if (save)
    hipLaunchKernelGGL((delta_fwd_kernel<BF, DK, NW, kSave>), grid, blk, 0, s, a, nsl);
  else
    hipLaunchKernelGGL((delta_fwd_kernel<BF, DK, NW, kPlain>), grid, blk, 0, s, a, nsl);
  return hipGetLastError();
}

// The first `nchain` workgroups run the chain, those behind them prepare the np
// chunks from p0 on, which the next launch takes.
template <int MODE>
__global__ void __launch_bounds__(256, 2)
delta_fwd_prep_kernel(DeltaArgs a, int nsl, int nchain, int p0, int np) {
  constexpr int kChain = FwdLds<true, 64, 4, MODE>::bytes;
  __shared__ __align__(16) char lds[kChain > kPrepLds ? kChain : kPrepLds];
  if ((int)blockIdx.x < nchain)
    fwd_chain<true, 64, 4, MODE>(a, nsl, blockIdx.x, lds);
  else
    prep_chunk<true, 64>(a, p0, np, blockIdx.x - nchain, lds);
}

}  // namespace

hipError_t launch_delta_chain_prep(const DeltaArgs& a, bool save, int p0, int np, hipStream_t s) {
  const int nsl = (a.dvp + 63) / 64;
  const long units = (long)a.B * a.H, nchain = (units + 7) / 8 * 8 * nsl;
  const dim3 grid((unsigned)(nchain + units * np)), blk(256);
  if (save)
    hipLaunchKernelGGL((delta_fwd_prep_kernel<kSave>), grid, blk, 0, s, a, nsl, (int)nchain, p0, np);
  else
    hipLaunchKernelGGL((delta_fwd_prep_kernel<kPlain>), grid, blk, 0, s, a, nsl, (int)nchain, p0, np);
  return hipGetLastError();
}

hipError_t launch_delta_chain(const DeltaArgs& a, bool bf, bool save, bool state, hipStream_t s) {
  const int dkp = delta_dkp(a.dk);
  if (bf) {
    if (dkp == 32) return go<true, 32, 2>(a, save, state, s);
    if (dkp == 64) return go<true, 64, 4>(a, save, state, s);
    // eight waves share a staged chunk (256 units of 128, 16 chunks: 165 us, with
    // four 224); four where eight would leave half of the 256 CUs idle (128 units,
    // 32 chunks: 209 us, with eight 240; saving, a step 914 and 997)
    const long tiles = a.dvp / 16 + (state ? 8 : 0);
    if ((long)a.B * a.H * a.nseg * ((tiles + 7) / 8) <= 128) return go<true, 128, 4>(a, save, state, s);
    return go<true, 128, 8>(a, save, state, s);
  }
  if (dkp == 32) return go<false, 32, 2>(a, save, state, s);
  if (dkp == 64) return go<false, 64, 4>(a, save, state, s);
  return go<false, 128, 4>(a, save, state, s);
}

}  // namespace e2ttt
