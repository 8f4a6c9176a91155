// Gated delta rule, the gradients of a chunk that sum over the value
// dimension, every chunk at once: one workgroup per chunk of 64 tokens and key
// head, over the value heads that share it in turn.  With W_0,
// U from the forward and dW (chunk end), Y from the backward chain:
//   A_ij = s D_ij (dO_i . U_j)   (j <= i),   N_ij = -eta_i D_ij (Y_i . U_j)  (j < i)
//   dQ = s G dO W_0 + A K
//   dK = A^T Q + (N + N^T) K - eta G Y W_0 + e^{b_C - b} U dW
//   d eta_i = Y_i . e_i = (Y_i . U_i) / eta_i, as U = eta e; where eta is too
//     small to divide by: e_i = v_i - G_i W_0 k_i - sum_j D_ij (k_i . k_j) u_j
//   d g_l = sum_{j < l <= i} (A_ij q_i . k_j + N_ij k_i . k_j)
//           + sum_{i >= l} s G_i (dO W_0)_i . q_i - eta_i G_i (Y W_0)_i . k_i
//           + sum_{j < l} e^{b_C - b_j} (U dW)_j . k_j + G_C <W_0, dW>
// (g_l multiplies exactly the paths that cross token l.  The pair sums are
// differences of row and column sums of the same fp32 numbers, so what cancels
// cancels to fp32 rounding.)
//
// The value dimension is taken in blocks of 32 through LDS, the next block's
// loads under way meanwhile.  For the 64 x DK products wave w holds column tile
// w mod (DK / 16) and its share of the four row tiles; for the 64 x 64 ones rows
// lab(w mod 4, .), with eight waves one of the two 32-column blocks.  Four
// waves up to DK = 64, so that two workgroups share a CU and one computes while
// the other waits; eight, and one workgroup a CU, at 128.
//
// 16384 chunks of dk = dv = 64 (112 KB each) take 559 us, 3.3 TB/s: a wave waits
// for 30 % of it, for the next block and for the others, and the two of a SIMD issue
// vector instructions for 60 % of it (registers and 77 KB of LDS leave two
// workgroups a CU).  8192 of 128: 800 us.
#pragma once

#include "delta_common.h"

namespace e2ttt {
namespace {

constexpr float kMinEta = 8.6736174e-19f;   // 2^-60

// Sum over the 16 lanes of a group for each of four row registers.
__device__ __forceinline__ f32x4 sum16(f32x4 x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = group16_sum(x[e]);
  return x;
}
// The same for eight: lane c returns the sum of value 4 (c / 8) + 2 (c / 4 mod 2)
// + c / 2 mod 2, of x's four and then y's.
__device__ __forceinline__ float sum16x8(f32x4 x, f32x4 y, int c) {
  const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  return row16_reduce_scatter8(v, c);
}

// LDS of a workgroup (offsets in bytes).
template <bool BF, int DK, int NWV>
struct GradsLds {
  using E = typename DOp<BF>::E;
  static constexpr int kStage =
      (2 * DOp<BF>::NT * 32 * (DK + kDC) + kDC * 32) * (int)sizeof(E);
  static constexpr int qs = kDC * DK * (int)sizeof(E), buf = 2 * qs;
  static constexpr int gl = buf + (kStage > 2 * tri_bytes(BF) ? kStage : 2 * tri_bytes(BF));
  static constexpr int srow = gl + kGateFloats * 4, srr = srow + 2 * (DK / 16) * kDC * 4;
  static constexpr int sx = srr + (DK / 16) * kDC * 4, scol = sx + 4 * kDC * 4;
  static constexpr int syu = scol + 4 * kDC * 4, bytes = syu + (kDC + NWV) * 4;
};

// ONE: a value head to a key head, whose sums then need no registers ahead.
// Workgroup `blk` of the chunks c0 .. c0 + nr - 1 of every key head.
template <bool BF, int DK, int NWV, bool ONE>
__device__ __forceinline__ void grads_chunk(const DeltaArgs& a, int c0, int nr, long blk, char* lds) {
  using O = DOp<BF>;
  using E = typename O::E;
  using L = LTile<BF, DK>;      // K, Q rows; states
  using LV = LTile<BF, 32>;     // dO rows of a value block
  constexpr int NT = O::NT, KT = DK / 32, NTH = 64 * NWV;
  constexpr int CTS = DK / 16;                          // column tiles
  constexpr int MG = NWV / CTS, MR = 4 / MG;            // row groups, row tiles of a wave
  constexpr int NB = 8 / NWV;                           // blocks of a wave in the 64x64 products
  constexpr int WP = 32 * DK, UP = 32 * kDC;            // elements of a term's block
  constexpr int PK = kDC * L::NP / NTH;                 // a thread's pieces of K (Q)
  constexpr int PW = (WP / 8 + NTH - 1) / NTH;          // of the states' block, eight values each
  constexpr int PU = 2 * UP / 8 / NTH;                  // of U and Y
  constexpr int PO = (kDC * LV::NP + NTH - 1) / NTH;    // of dO
  static_assert(kDC * L::NP % NTH == 0 && 2 * UP / 8 % NTH == 0 && NTH % 64 == 0, "whole rounds");
  using M = GradsLds<BF, DK, NWV>;
  E* ks = reinterpret_cast<E*>(lds);
  E* qs = reinterpret_cast<E*>(lds + M::qs);
  char* buf = lds + M::buf;                             // value blocks, then A and N
  float* gl = reinterpret_cast<float*>(lds + M::gl);
  float(*srow)[CTS][kDC] = reinterpret_cast<float(*)[CTS][kDC]>(lds + M::srow);   // row dots by column tile: O + R, S terms
  float(*srr)[kDC] = reinterpret_cast<float(*)[kDC]>(lds + M::srr);   // (Y W_0)_i . k_i, where eta is too small
  float(*sx)[2][kDC] = reinterpret_cast<float(*)[2][kDC]>(lds + M::sx);   // row sums by block: pairs, (Y U^T) o M
  float(*scol)[kDC] = reinterpret_cast<float(*)[kDC]>(lds + M::scol);   // column sums of the pairs by row tile
  float* syu = reinterpret_cast<float*>(lds + M::syu);  // Y_i . U_i
  float* sdot = syu + kDC;                              // <W_0, dW> by wave

  E* w0s = reinterpret_cast<E*>(buf);
  E* dws = w0s + NT * WP;
  E* us = dws + NT * WP;
  E* ys = us + NT * UP;
  E* dos = ys + NT * UP;
  char* as = buf;
  char* ns = buf + tri_bytes(BF);

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = wave_id();
  const int rep = ONE ? 1 : a.H / a.HK;
  const int bh = __builtin_amdgcn_readfirstlane((int)(blk / nr));
  const int r = __builtin_amdgcn_readfirstlane(c0 + (int)(blk % nr));
  const int b = bh / a.HK, hk = bh % a.HK;
  const int t0 = r * kDC, nt = min(kDC, max(0, live_tokens(a, b) - t0));
  const int kst = (int)a.k.t, qst = (int)a.q.t, gst = (int)a.d_out.t, ost = (int)a.dv_.t;

  if (nt < kDC) {                            // behind the sequence: zeros
    const int rows = min(kDC, a.T - t0);
    auto clear = [&](const View& v, int h, int d) {
      const int np = d / L::PE;
      for (int p = tid; p < (rows - nt) * np; p += NTH)
        *reinterpret_cast<u32x4*>(row_of_w<E>(v, b, h, t0 + nt + p / np) + p % np * L::PE) =
            u32x4{0, 0, 0, 0};
    };
    clear(a.dq, hk, a.dk);
    clear(a.dkk, hk, a.dk);
    for (int h = hk * rep; h < (hk + 1) * rep; ++h) {
      clear(a.dv_, h, a.dv);
      if (tid >= nt && tid < rows) {
        *row_of_w<float>(a.deta, b, h, t0 + tid) = 0.0f;
        if (a.dgam.p) *row_of_w<float>(a.dgam, b, h, t0 + tid) = 0.0f;
      }
    }
    if (nt == 0) return;
  }

  // the next value block on its way: v0 of value head h (chunk unit cu)
  u32x4 rw[PW][4], ru[PU][2], ro[PO];
  auto fetch = [&](int h, long cu, int v0) {
    const Buf w0b = buf_of(a.wst + (cu * a.dvp + v0) * DK), dwb = buf_of(a.dwst + (cu * a.dvp + v0) * DK);
    const Buf ub = buf_of(a.ust + (cu * a.dvp + v0) * kDC), yb = buf_of(a.yst + (cu * a.dvp + v0) * kDC);
#pragma unroll
    for (int x = 0; x < PW; ++x) {           // a wave takes 16 rows x 32 columns
      const int p = tid + x * NTH;
      const unsigned no = WP / 8 % NTH == 0 || p < WP / 8 ? 0 : kNowhere;
      const unsigned at = 4 * (unsigned)lane_at(p / (64 * KT), (p >> 6) % KT, KT, lane) | no;
      rw[x][0] = buf_ld(w0b, at);
      rw[x][1] = buf_ld(w0b, at + 1024);
      rw[x][2] = buf_ld(dwb, at);
      rw[x][3] = buf_ld(dwb, at + 1024);
    }
#pragma unroll
    for (int x = 0; x < PU; ++x) {           // (256 pieces of U, then of Y: a wave's are of one)
      const int p = tid + x * NTH;
      const unsigned at = 4 * (unsigned)lane_at((p >> 7) & 1, (p >> 6) & 1, 2, lane);
      const bool y = 4 * x * NWV >= 16 || (NWV > 4 && w >= 4);
      ru[x][0] = buf_ld(y ? yb : ub, at);
      ru[x][1] = buf_ld(y ? yb : ub, at + 1024);
    }
    const Buf ob = buf_of(row_of<E>(a.d_out, b, h, t0) + v0);
#pragma unroll
    for (int x = 0; x < PO; ++x) {
      const int p = tid + x * NTH, row = p / LV::NP, col = (p % LV::NP) * LV::PE;
      const unsigned no = row < nt && v0 + col < a.dv ? 0 : kNowhere;
      ro[x] = buf_ld(ob, (unsigned)(row * gst + col) * (unsigned)sizeof(E) | no);
    }
  };
  {
    const Buf kb = buf_of(row_of<E>(a.k, b, hk, t0)), qb = buf_of(row_of<E>(a.q, b, hk, t0));
    u32x4 rk[PK], rq[PK];
#pragma unroll
    for (int x = 0; x < PK; ++x) {
      const int p = tid + x * NTH, row = p / L::NP, col = (p % L::NP) * L::PE;
      const unsigned no = row < nt && col < a.dk ? 0 : kNowhere;
      rk[x] = buf_ld(kb, (unsigned)(row * kst + col) * (unsigned)sizeof(E) | no);
      rq[x] = buf_ld(qb, (unsigned)(row * qst + col) * (unsigned)sizeof(E) | no);
    }
    fetch(hk * rep, ((long)b * a.H + hk * rep) * a.nc_buf + (r - a.r_base), 0);
#pragma unroll
    for (int x = 0; x < PK; ++x) {
      const int p = tid + x * NTH, at = L::at(p / L::NP, p % L::NP);
      *reinterpret_cast<u32x4*>(ks + at) = rk[x];
      *reinterpret_cast<u32x4*>(qs + at) = rq[x];
    }
  }
  __syncthreads();

  const int rt = w & 3, xb0 = NB == 1 ? w >> 2 : 0;    // row tile, (first) block of the 64x64 products
  const int ct = w % CTS, m0 = MG == 1 ? 0 : (w / CTS) * MR;   // column tile, first row tile of the 64xDK ones
  f32x4 dq[MR], dk[MR];
#pragma unroll
  for (int m = 0; m < MR; ++m) dq[m] = dk[m] = zero4();

  for (int hv = 0; hv < rep; ++hv) {
    const int h = hk * rep + hv;
    const long cu = ((long)b * a.H + h) * a.nc_buf + (r - a.r_base);
    __syncthreads();                         // gl, buf and the sums are free
    for (int x = tid; x < kGateFloats / 4; x += NTH)
      *reinterpret_cast<f32x4*>(gl + 4 * x) =
          *reinterpret_cast<const f32x4*>(a.gate + cu * kGateFloats + 4 * x);

    f32x4 ow[MR], yw[MR], uw[MR], du[NB][2], yu[NB][2];
    float wdot = 0.0f;
#pragma unroll
    for (int n = 0; n < NB; ++n) du[n][0] = du[n][1] = yu[n][0] = yu[n][1] = zero4();
#pragma unroll
    for (int m = 0; m < MR; ++m) ow[m] = yw[m] = uw[m] = zero4();
    auto stage = [&]() {
#pragma unroll
      for (int x = 0; x < PW; ++x) {
        const int p = tid + x * NTH, row = 16 * (p / (64 * KT)) + c, p8 = 4 * ((p >> 6) % KT) + g;
        if (WP / 8 % NTH == 0 || p < WP / 8) {
          f32x4 v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = __builtin_bit_cast(f32x4, rw[x][k]);
          put_terms<BF, DK>(w0s, WP, row, p8, v[0], v[1]);
          put_terms<BF, DK>(dws, WP, row, p8, v[2], v[3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) wdot = fmaf(v[0][e], v[2][e], fmaf(v[1][e], v[3][e], wdot));
        }
      }
#pragma unroll
      for (int x = 0; x < PU; ++x) {
        const int p = tid + x * NTH;
        put_terms<BF, kDC>(p >> 8 ? ys : us, UP, 16 * ((p >> 7) & 1) + c, 4 * ((p >> 6) & 1) + g,
                           __builtin_bit_cast(f32x4, ru[x][0]), __builtin_bit_cast(f32x4, ru[x][1]));
      }
#pragma unroll
      for (int x = 0; x < PO; ++x) {
        const int p = tid + x * NTH;
        if (kDC * LV::NP % NTH == 0 || p < kDC * LV::NP)
          *reinterpret_cast<u32x4*>(dos + LV::at(p / LV::NP, p % LV::NP)) = ro[x];
      }
    };
    stage();
    for (int v0 = 0; v0 < a.dvp; v0 += 32) {
      E2TTT_LANE_IDS;                        // (addresses formed here, not kept in registers)
      const int i = lab(rt, c);
      __syncthreads();
      if (v0 + 32 < a.dvp)
        fetch(h, cu, v0 + 32);
      else if (!ONE && hv + 1 < rep)
        fetch(h + 1, cu + a.nc_buf, 0);
      auto products = [&](int m, const auto& wf, const auto& df, const auto& um) {
        ow[m] = O::xs(ow[m], LV::frag(dos, lab(m0 + m, c), 0, g), wf);
        yw[m] = O::ss(yw[m], terms_t<BF, kDC, false>(ys, UP, m0 + m, g, c), wf);
        uw[m] = O::ss(uw[m], um, df);
      };
      if constexpr (MR < 4) {
        const auto wf = terms_t<BF, DK, true>(w0s, WP, ct, g, c);
        const auto df = terms_t<BF, DK, true>(dws, WP, ct, g, c);
#pragma unroll
        for (int m = 0; m < MR; ++m) products(m, wf, df, terms_t<BF, kDC, false>(us, UP, m0 + m, g, c));
      }
      const auto doi = LV::frag(dos, i, 0, g);
      const auto yi = terms_t<BF, kDC, false>(ys, UP, rt, g, c);
      if (xb0 == 0) {                        // dV = eta Y, eight channels a lane
        f32x4 y0, y1;
        O::sum(yi, y0, y1);
        const Buf vb = buf_of(row_of<E>(a.dv_, b, h, t0) + v0);
        const unsigned no = i < nt && v0 + 8 * g < a.dv ? 0 : kNowhere;
        const unsigned at = (unsigned)(i * ost + 8 * g) * (unsigned)sizeof(E) | no;
        buf_st_io<BF>(vb, at, y0 * gl[kGEta + i]);
        buf_st_io<BF>(vb, at + 4 * (unsigned)sizeof(E), y1 * gl[kGEta + i]);
      }
      auto pairs = [&](int n, int y, const auto& uj) {
        du[n][y] = O::sx(du[n][y], uj, doi);
        yu[n][y] = O::ss(yu[n][y], uj, yi);
      };
      if constexpr (MR < 4) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
          if (xb0 + n <= rt / 2) {
            pairs(n, 0, terms_t<BF, kDC, false>(us, UP, 2 * (xb0 + n), g, c));
            pairs(n, 1, terms_t<BF, kDC, false>(us, UP, 2 * (xb0 + n) + 1, g, c));
          }
      } else {                               // (both take every row tile of U: read once)
        const auto wf = terms_t<BF, DK, true>(w0s, WP, ct, g, c);
        const auto df = terms_t<BF, DK, true>(dws, WP, ct, g, c);
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          const auto um = terms_t<BF, kDC, false>(us, UP, m, g, c);
          products(m, wf, df, um);
          if (m / 2 <= rt / 2 && (NB == 2 || m / 2 == xb0)) pairs(NB == 2 ? m / 2 : 0, m % 2, um);
        }
      }
      if (v0 + 32 < a.dvp) {
        __syncthreads();                     // (the block in LDS is done with)
        stage();
      }
    }
    __syncthreads();                         // the value blocks are done: buf holds A and N
    if (ONE) {
#pragma unroll
      for (int m = 0; m < MR; ++m) dq[m] = dk[m] = zero4();
    }

    // 64x64 terms of row i, columns j = 32 xb + 8 g + 4 y + e
    {
    E2TTT_LANE_IDS;
    const int i = lab(rt, c);
    const float eta_i = gl[kGEta + i];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int xb = xb0 + n;
      float rx = 0.0f, rm = 0.0f;
      f32x4 kk[2], qk[2];                    // k_i . k_j, q_i . k_j
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        kk[y] = qk[y] = zero4();
        if (xb <= rt / 2) {                  // (the block reaches below the diagonal)
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            const auto kj = L::frag(ks, lab(2 * xb + y, c), kt, g);
            kk[y] = O::xx(kk[y], kj, L::frag(ks, i, kt, g));
            qk[y] = O::xx(qk[y], kj, L::frag(qs, i, kt, g));
          }
        }
      }
      const float bhi = gl[kGBh + i], bli = gl[kGBl + i];
      f32x4 pa[2], pn[2], pair[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int j0 = 32 * xb + 8 * g + 4 * y;
        const f32x4 bhj = *reinterpret_cast<const f32x4*>(gl + kGBh + j0);
        const f32x4 blj = *reinterpret_cast<const f32x4*>(gl + kGBl + j0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = j0 + e;
          const float d = j <= i ? exp_finite((bhi - bhj[e]) + (bli - blj[e])) : 0.0f;
          const float dy = j < i ? d * yu[n][y][e] : 0.0f;
          pa[y][e] = a.scale * (d * du[n][y][e]);
          pn[y][e] = -eta_i * dy;
          rm = fmaf(dy, kk[y][e], rm);
          pair[y][e] = j < i ? fmaf(pa[y][e], qk[y][e], pn[y][e] * kk[y][e]) : 0.0f;
          rx += pair[y][e];
          if (j == i) syu[i] = yu[n][y][e];
        }
      }
      if (xb <= rt / 2) {
        put_frag<BF>(as, fidx(rt, xb), lane, pa[0], pa[1]);
        put_frag<BF>(ns, fidx(rt, xb), lane, pn[0], pn[1]);
      }
      const float cs = sum16x8(pair[0], pair[1], c);     // of column 8 g + c / 2 of the block
      if (!(c & 1)) scol[rt][32 * xb + 8 * g + (c >> 1)] = cs;
      rx += __shfl_xor(rx, 16);
      rx += __shfl_xor(rx, 32);
      rm += __shfl_xor(rm, 16);
      rm += __shfl_xor(rm, 32);
      if (g == 0) {
        sx[0][xb][i] = rx;
        sx[1][xb][i] = rm;
      }
    }
    }
    wdot = wave_sum(wdot);
    E2TTT_LANE_IDS;
    if (lane == 0) sdot[w] = wdot;
    // row dots with q and k, and the state terms of dQ and dK
    const bool tiny = __any(!(fabsf(gl[kGEta + lane]) >= kMinEta) && lane < nt);
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      const int tr = lab(m0 + m, 4 * g);
      const f32x4 sg = *reinterpret_cast<const f32x4*>(gl + kGsG + tr);
      const f32x4 eg = *reinterpret_cast<const f32x4*>(gl + kGEtaG + tr);
      const f32x4 en = *reinterpret_cast<const f32x4*>(gl + kGEnd + tr);
      const int col = ct * 16 + c;
      f32x4 d0, d1, d2;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = L::at(tr + e, col / L::PE) + col % L::PE;
        const float kv = (float)ks[at], qv = (float)qs[at];
        const float os = sg[e] * ow[m][e];
        d1[e] = yw[m][e] * kv;
        d0[e] = fmaf(os, qv, -(eg[e] * d1[e]));
        const float us_ = en[e] * uw[m][e];
        d2[e] = us_ * kv;
        dq[m][e] += os;
        dk[m][e] += us_ - eg[e] * yw[m][e];
      }
      const float ds = sum16x8(d0, d2, c);               // of row c / 2 mod 4, d0 then d2
      if (!(c & 1)) srow[c >> 3][ct][tr + ((c >> 1) & 3)] = ds;
      if (tiny) {
        d1 = sum16(d1);
        if (c == 0) *reinterpret_cast<f32x4*>(&srr[ct][tr]) = d1;
      }
    }
    __syncthreads();

#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const auto kf = L::template frag_t<true>(ks, ct, x, g, c);
      const auto qf = L::template frag_t<true>(qs, ct, x, g, c);
#pragma unroll
      for (int mm = 0; mm < MR; ++mm) {
        const int m = m0 + mm;
        if (x <= m / 2) {
          dq[mm] = O::sx(dq[mm], ld_frag<BF>(as, fidx(m, x), lane), kf);
          dk[mm] = O::sx(dk[mm], ld_frag<BF>(ns, fidx(m, x), lane), kf);
        }
        if (x >= m / 2) {
          dk[mm] = O::sx(dk[mm], ld_frag_t<BF>(as, m, x, g, c), qf);
          dk[mm] = O::sx(dk[mm], ld_frag_t<BF>(ns, m, x, g, c), kf);
        }
      }
    }
    if (w == NWV - 1) {                            // gate gradients, one token a lane
      const int t = lane;
      const bool live = t < nt;
      const float eta = gl[kGEta + t];
      float so = 0.0f, sr = 0.0f, ss = 0.0f, sc = 0.0f, dot = 0.0f;
#pragma unroll
      for (int x = 0; x < CTS; ++x) {
        so += srow[0][x][t];
        ss += srow[1][x][t];
        if (tiny) sr += srr[x][t];
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) sc += scol[x][t];
#pragma unroll
      for (int x = 0; x < NWV; ++x) dot += sdot[x];
      float de = syu[t] / eta;
      if (live && !(fabsf(eta) >= kMinEta)) {
        // eta (near) zero: Y_i . e_i by its definition
        const float* yp = a.yst + cu * a.dvp * kDC + (t & 4) * 64 + (t & 3);
        const E* vp = row_of<E>(a.v, b, h, t0 + t);
        float yv = 0.0f;
        for (int n = 0; n < a.dv; ++n)
          yv = fmaf(yp[lane_at(n >> 4, t >> 5, 2, 16 * ((t >> 3) & 3) + (n & 15))], (float)vp[n], yv);
        de = yv - expf(gl[kGBh + t]) * sr - (sx[1][0][t] + sx[1][1][t]);
      }
      // sums over tokens at and after t, and before t
      const double after = (double)sx[0][0][t] + sx[0][1][t] - sc + so, upto = ss;
      double p = upto, q = after;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(p, o), z = __shfl_down(q, o);
        if (lane >= o) p += y;
        if (lane + o < 64) q += z;
      }
      if (live) {
        *row_of_w<float>(a.deta, b, h, t0 + t) = de;
        if (a.dgam.p)
          *row_of_w<float>(a.dgam, b, h, t0 + t) =
              (float)(q + (p - upto) + (double)gl[kGC] * dot);
      }
    }
  }

  const int dqst = (int)a.dq.t, dkst = (int)a.dkk.t;
  E* dqp = row_of_w<E>(a.dq, b, hk, t0);
  E* dkp = row_of_w<E>(a.dkk, b, hk, t0);
  const int col = ct * 16 + c;
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = lab(m0 + m, 4 * g) + e;
      if (t < nt && col < a.dk) {
        dqp[t * dqst + col] = (E)dq[m][e];
        dkp[t * dkst + col] = (E)dk[m][e];
      }
    }
}

}  // namespace
}  // namespace e2ttt
