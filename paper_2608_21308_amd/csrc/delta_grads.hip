// Gated delta rule, the gradients of a chunk that sum over the value
// dimension, every chunk at once: one workgroup of eight waves per chunk of 64
// tokens and key head, over the value heads that share it in turn.  With W_0,
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
// The value dimension is taken in blocks of 32 through LDS.  For the 64 x DK
// products wave w holds column tile w mod (DK / 16) and as many of the four row
// tiles as make eight waves; for the 64 x 64 ones rows lab(w mod 4, .) and the
// 32-column block w / 4.
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

template <bool BF, int DK>
__global__ void __launch_bounds__(512) delta_grads_kernel(DeltaArgs a) {
  using O = DOp<BF>;
  using E = typename O::E;
  using L = LTile<BF, DK>;      // K, Q rows; states
  using LV = LTile<BF, 32>;     // dO rows of a value block
  using LU = LTile<BF, kDC>;    // U^T, Y^T
  constexpr int NT = O::NT, KT = DK / 32, NTH = 512;
  constexpr int CTS = DK / 16;                          // column tiles
  constexpr int MG = 8 / CTS, MR = 4 / MG;              // row groups, row tiles of a wave
  constexpr int WP = 32 * DK, UP = 32 * kDC;            // elements of a term's block
  constexpr int kStage = (2 * NT * WP + 2 * NT * UP + kDC * 32) * (int)sizeof(E);
  constexpr int kBuf = kStage > 2 * tri_bytes(BF, 2) ? kStage : 2 * tri_bytes(BF, 2);
  __shared__ __align__(16) E ks[kDC * DK];
  __shared__ __align__(16) E qs[kDC * DK];
  __shared__ __align__(16) char buf[kBuf];              // value blocks, then A and N
  __shared__ __align__(16) float gl[kGateFloats];
  __shared__ float srow[3][CTS][kDC];                   // row dots by column tile: O, R, S terms
  __shared__ float sx[2][2][kDC];                       // row sums by block: pairs, (Y U^T) o M
  __shared__ float scol[4][kDC];                        // column sums of the pairs by row tile
  __shared__ float syu[kDC];                            // Y_i . U_i
  __shared__ float sdot[8];                             // <W_0, dW> by wave

  E* w0s = reinterpret_cast<E*>(buf);
  E* dws = w0s + NT * WP;
  E* us = dws + NT * WP;
  E* ys = us + NT * UP;
  E* dos = ys + NT * UP;
  char* as = buf;
  char* ns = buf + tri_bytes(BF, 2);

  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
  const int nr = a.r1 - a.r0, rep = a.H / a.HK;
  const long bh = blockIdx.x / nr;
  const int r = a.r0 + (int)(blockIdx.x % nr);
  const int b = (int)(bh / a.HK), hk = (int)(bh % a.HK);
  const int t0 = r * kDC, nt = min(kDC, max(0, live_tokens(a, b) - t0));
  const E* kp = row_of<E>(a.k, b, hk, t0);
  const E* qp = row_of<E>(a.q, b, hk, t0);
  for (int p = tid; p < kDC * L::NP; p += NTH) {
    const int row = p / L::NP, col = (p % L::NP) * L::PE;
    uint4 x = make_uint4(0, 0, 0, 0), y = x;
    if (row < nt && col < a.dk) {
      x = *reinterpret_cast<const uint4*>(kp + (long)row * a.k.t + col);
      y = *reinterpret_cast<const uint4*>(qp + (long)row * a.q.t + col);
    }
    *reinterpret_cast<uint4*>(ks + L::at(row, p % L::NP)) = x;
    *reinterpret_cast<uint4*>(qs + L::at(row, p % L::NP)) = y;
  }
  __syncthreads();

  const int rt = w & 3, xb = w >> 2;         // row tile and block of the 64x64 products
  const int i = lab(rt, c);
  const bool low = xb <= rt / 2;             // the block reaches below the diagonal
  f32x4 kk[2], qk[2];                        // k_i . k_j, q_i . k_j at j = 32 xb + 8 g + 4 y + e
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    kk[y] = qk[y] = zero4();
    if (low) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const auto kj = L::frag(ks, lab(2 * xb + y, c), kt, g);
        kk[y] = O::xx(kk[y], kj, L::frag(ks, i, kt, g));
        qk[y] = O::xx(qk[y], kj, L::frag(qs, i, kt, g));
      }
    }
  }
  const int ct = w % CTS, m0 = (w / CTS) * MR;   // column tile, first row tile of the 64xDK ones
  f32x4 dq[MR], dk[MR];
#pragma unroll
  for (int m = 0; m < MR; ++m) dq[m] = dk[m] = zero4();

  for (int hv = 0; hv < rep; ++hv) {
    const int h = hk * rep + hv;
    const long cu = ((long)b * a.H + h) * a.nc_buf + (r - a.r_base);
    const E* dop = row_of<E>(a.d_out, b, h, t0);
    __syncthreads();                         // gl, buf and the sums are free
    for (int x = tid; x < kGateFloats; x += NTH) gl[x] = a.gate[cu * kGateFloats + x];

    f32x4 ow[MR], yw[MR], uw[MR], du[2], yu[2];
    float wdot = 0.0f;
    du[0] = du[1] = yu[0] = yu[1] = zero4();
#pragma unroll
    for (int m = 0; m < MR; ++m) ow[m] = yw[m] = uw[m] = zero4();
    for (int v0 = 0; v0 < a.dvp; v0 += 32) {
      __syncthreads();
      constexpr int PW = WP / 8, PU = UP / 8, PO = kDC * LV::NP;
      const float* w0g = a.wst + (cu * a.dvp + v0) * DK;
      const float* dwg = a.dwst + (cu * a.dvp + v0) * DK;
      const float* ug = a.ust + (cu * a.dvp + v0) * kDC;
      const float* yg = a.yst + (cu * a.dvp + v0) * kDC;
      for (int p = tid; p < PW; p += NTH) {  // a wave takes 16 rows x 32 columns
        const int tile = p / (64 * KT), kt = (p >> 6) % KT;
        const long at = lane_at(tile, kt, KT, lane);
        const f32x4 x0 = *reinterpret_cast<const f32x4*>(w0g + at);
        const f32x4 x1 = *reinterpret_cast<const f32x4*>(w0g + at + 256);
        const f32x4 y0 = *reinterpret_cast<const f32x4*>(dwg + at);
        const f32x4 y1 = *reinterpret_cast<const f32x4*>(dwg + at + 256);
        put_terms<BF, DK>(w0s, WP, 16 * tile + c, 4 * kt + g, x0, x1);
        put_terms<BF, DK>(dws, WP, 16 * tile + c, 4 * kt + g, y0, y1);
#pragma unroll
        for (int e = 0; e < 4; ++e) wdot = fmaf(x0[e], y0[e], fmaf(x1[e], y1[e], wdot));
      }
      for (int p = tid; p < 2 * PU; p += NTH) {
        const int s = p >= PU, tile = (p >> 7) & 1, x = (p >> 6) & 1;
        const float* src = (s ? yg : ug) + lane_at(tile, x, 2, lane);
        put_terms<BF, kDC>(s ? ys : us, UP, 16 * tile + c, 4 * x + g,
                           *reinterpret_cast<const f32x4*>(src),
                           *reinterpret_cast<const f32x4*>(src + 256));
      }
      for (int p = tid; p < PO; p += NTH) {
        const int row = p / LV::NP, col = v0 + (p % LV::NP) * LV::PE;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (row < nt && col < a.dv)
          x = *reinterpret_cast<const uint4*>(dop + (long)row * a.d_out.t + col);
        *reinterpret_cast<uint4*>(dos + LV::at(row, p % LV::NP)) = x;
      }
      __syncthreads();
      {
        const auto wf = terms_t<BF, DK, true>(w0s, WP, ct, g, c);
        const auto df = terms_t<BF, DK, true>(dws, WP, ct, g, c);
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          ow[m] = O::template xs<3>(ow[m], LV::frag(dos, lab(m0 + m, c), 0, g), wf);
          yw[m] = O::template ss<3>(yw[m], terms_t<BF, kDC, false>(ys, UP, m0 + m, g, c), wf);
          uw[m] = O::template ss<3>(uw[m], terms_t<BF, kDC, false>(us, UP, m0 + m, g, c), df);
        }
      }
      if (low) {
        const auto doi = LV::frag(dos, i, 0, g);
        const auto yi = terms_t<BF, kDC, false>(ys, UP, rt, g, c);
        if (xb == 0 && t0 + i < a.T && v0 + 8 * g < a.dv) {   // dV = eta Y, eight channels a lane
          f32x4 y0, y1;
          O::sum(yi, y0, y1);
          E* p = row_of_w<E>(a.dv_, b, h, t0 + i) + v0 + 8 * g;
          IoT<BF>::st4(p, y0 * gl[kGEta + i]);
          IoT<BF>::st4(p + 4, y1 * gl[kGEta + i]);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const auto uj = terms_t<BF, kDC, false>(us, UP, 2 * xb + y, g, c);
          du[y] = O::template sx<3>(du[y], uj, doi);
          yu[y] = O::template ss<3>(yu[y], uj, yi);
        }
      }
    }
    __syncthreads();                         // the value blocks are done: buf holds A and N

    // 64x64 terms of row i, columns j = 32 xb + 8 g + 4 y + e
    {
      float rx = 0.0f, rm = 0.0f;
      const float bhi = gl[kGBh + i], bli = gl[kGBl + i], eta = gl[kGEta + i];
      f32x4 pa[2], pn[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        f32x4 pair;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = 32 * xb + 8 * g + 4 * y + e;
          pa[y][e] = pn[y][e] = pair[e] = 0.0f;
          if (j <= i) {
            const float d = expf((bhi - gl[kGBh + j]) + (bli - gl[kGBl + j]));
            pa[y][e] = a.scale * (d * du[y][e]);
            if (j < i) {
              const float dy = d * yu[y][e];
              pn[y][e] = -eta * dy;
              rm = fmaf(dy, kk[y][e], rm);
              pair[e] = fmaf(pa[y][e], qk[y][e], pn[y][e] * kk[y][e]);
              rx += pair[e];
            } else {
              syu[i] = yu[y][e];
            }
          }
        }
        pair = sum16(pair);
        if (c == 0) *reinterpret_cast<f32x4*>(&scol[rt][32 * xb + 8 * g + 4 * y]) = pair;
      }
      if (low) {
        put_frag<BF, 2>(as, fidx(rt, xb), lane, pa[0], pa[1]);
        put_frag<BF, 2>(ns, fidx(rt, xb), lane, pn[0], pn[1]);
      }
      rx += __shfl_xor(rx, 16);
      rx += __shfl_xor(rx, 32);
      rm += __shfl_xor(rm, 16);
      rm += __shfl_xor(rm, 32);
      if (g == 0) {
        sx[0][xb][i] = rx;
        sx[1][xb][i] = rm;
      }
    }
    wdot = wave_sum(wdot);
    if (lane == 0) sdot[w] = wdot;
    // row dots with q and k, and the state terms of dQ and dK
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
        d0[e] = ow[m][e] * qv;
        d1[e] = yw[m][e] * kv;
        d2[e] = uw[m][e] * kv;
      }
      dq[m] += sg * ow[m];
      dk[m] += en * uw[m] - eg * yw[m];
      d0 = sum16(d0);
      d1 = sum16(d1);
      d2 = sum16(d2);
      if (c == 0) {
        *reinterpret_cast<f32x4*>(&srow[0][ct][tr]) = d0;
        *reinterpret_cast<f32x4*>(&srow[1][ct][tr]) = d1;
        *reinterpret_cast<f32x4*>(&srow[2][ct][tr]) = d2;
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
          dq[mm] = O::template sx<2>(dq[mm], ld_frag<BF, 2>(as, fidx(m, x), lane), kf);
          dk[mm] = O::template sx<2>(dk[mm], ld_frag<BF, 2>(ns, fidx(m, x), lane), kf);
        }
        if (x >= m / 2) {
          dk[mm] = O::template sx<2>(dk[mm], ld_frag_t<BF, 2>(as, m, x, g, c), qf);
          dk[mm] = O::template sx<2>(dk[mm], ld_frag_t<BF, 2>(ns, m, x, g, c), kf);
        }
      }
    }
    if (w == 7) {                            // gate gradients, one token a lane
      const int t = lane;
      const bool live = t < nt;
      const float eta = gl[kGEta + t];
      float so = 0.0f, sr = 0.0f, ss = 0.0f, sc = 0.0f, dot = 0.0f;
#pragma unroll
      for (int x = 0; x < CTS; ++x) {
        so += srow[0][x][t];
        sr += srow[1][x][t];
        ss += srow[2][x][t];
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) sc += scol[x][t];
#pragma unroll
      for (int x = 0; x < 8; ++x) dot += sdot[x];
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
      const double after = (double)sx[0][0][t] + sx[0][1][t] - sc + (double)gl[kGsG + t] * so -
                           (double)gl[kGEtaG + t] * sr;
      const double upto = (double)gl[kGEnd + t] * ss;
      double p = upto, q = after;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(p, o), z = __shfl_down(q, o);
        if (lane >= o) p += y;
        if (lane + o < 64) q += z;
      }
      if (t0 + t < a.T) {
        *row_of_w<float>(a.deta, b, h, t0 + t) = live ? de : 0.0f;
        if (a.dgam.p)
          *row_of_w<float>(a.dgam, b, h, t0 + t) =
              live ? (float)(q + (p - upto) + (double)gl[kGC] * dot) : 0.0f;
      }
    }
  }

  E* dqp = row_of_w<E>(a.dq, b, hk, t0);
  E* dkp = row_of_w<E>(a.dkk, b, hk, t0);
  const int col = ct * 16 + c;
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = lab(m0 + m, 4 * g) + e;
      if (t0 + t < a.T && col < a.dk) {
        dqp[(long)t * a.dq.t + col] = (E)dq[m][e];
        dkp[(long)t * a.dkk.t + col] = (E)dk[m][e];
      }
    }
}

template <bool BF>
hipError_t go(const DeltaArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.B * a.HK * (a.r1 - a.r0))), blk(512);
  switch (delta_dkp(a.dk)) {
    case 32: hipLaunchKernelGGL((delta_grads_kernel<BF, 32>), grid, blk, 0, s, a); break;
    case 64: hipLaunchKernelGGL((delta_grads_kernel<BF, 64>), grid, blk, 0, s, a); break;
    default: hipLaunchKernelGGL((delta_grads_kernel<BF, 128>), grid, blk, 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_grads(const DeltaArgs& a, bool bf, hipStream_t stream) {
  return bf ? go<true>(a, stream) : go<false>(a, stream);
}

}  // namespace e2ttt
