// Gated delta rule, backward chain over the chunks in reverse (mathematics and
// layouts: delta_common.h).  With dW the adjoint of the state at the chunk
// end, per chunk
//   dU = P^T dO + e^{b_C - b} K dW^T
//   Y  = T^T dU,  dR = eta Y = dV
//   dW_0 = G_C dW + sum_i s G_i dO_i q_i^T - sum_i eta_i G_i Y_i k_i^T.
// As in the forward, a wave owns 16 columns of dW^T and carries them in its
// accumulators; dW at every chunk end and Y are left for the gradients that
// sum over the value dimension (delta_grads.hip).
#include "delta_common.h"

namespace e2ttt {
namespace {

template <bool BF, int DK, int NT, int NW>
__global__ void __launch_bounds__(64 * NW) delta_bwd_kernel(DeltaArgs a, int nsl) {
  using O = DOp<BF>;
  using E = typename O::E;
  using L = LTile<BF, DK>;
  constexpr int NTH = 64 * NW, KT = DK / 32, MT = DK / 16;
  constexpr int NP = kDC * L::NP, PK = NP / NTH;
  constexpr int NF = 2 * kDeltaFrags * 64, PF = NF / NTH;  // lanes' parts of the T and P fragments
  static_assert(NP % NTH == 0 && NF % NTH == 0, "whole rounds of pieces");
  __shared__ __align__(16) E ks[kDC * DK];
  __shared__ __align__(16) E qs[kDC * DK];
  __shared__ __align__(16) char ts[tri_lds<BF>(O::NT)];
  __shared__ __align__(16) char ps[tri_lds<BF>(O::NT)];
  __shared__ __align__(16) float gl[4 * kDC];

  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
  const long U = (long)a.B * a.H;
  const long blk = blockIdx.x;
  const long u = (blk / (8 * nsl)) * 8 + blk % 8;
  if (u >= U) return;
  const int sl = (int)((blk / 8) % nsl);
  const int b = (int)(u / a.H), h = (int)(u % a.H), hk = h / (a.H / a.HK);
  const int nlive = live_tokens(a, b);
  const int col0 = (sl * NW + w) * 16 * NT + NT * c;
  const E* kp = row_of<E>(a.k, b, hk, 0);
  const E* qp = row_of<E>(a.q, b, hk, 0);
  const E* dop = row_of<E>(a.d_out, b, h, 0);
  E* dvp = row_of_w<E>(a.dv_, b, h, 0);

  f32x4 st[MT][NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int kcol = lab(m, 4 * g);
      st[m][n] = zero4();
      if (a.d_w_out && col0 + n < a.dv && kcol < a.dk)
        st[m][n] = *reinterpret_cast<const f32x4*>(a.d_w_out + (u * a.dv + col0 + n) * a.dk + kcol);
    }

  uint4 rk[PK], rq[PK];
  f32x4 rf[PF][2];
  float rg[2];
  E rv[16 * NT];
  auto fetch = [&](int r) {
    const int t0 = r * kDC, nt = nlive - t0;
    const long cu = u * a.nc_buf + (r - a.r_base);
#pragma unroll
    for (int x = 0; x < PK; ++x) {
      const int p = tid + x * NTH, row = p / L::NP, col = (p % L::NP) * L::PE;
      rk[x] = rq[x] = make_uint4(0, 0, 0, 0);
      if (row < nt && col < a.dk) {
        rk[x] = *reinterpret_cast<const uint4*>(kp + (long)(t0 + row) * a.k.t + col);
        rq[x] = *reinterpret_cast<const uint4*>(qp + (long)(t0 + row) * a.q.t + col);
      }
    }
    const char* f = a.frag + cu * 2 * kTriBytes;
#pragma unroll
    for (int x = 0; x < PF; ++x) {
      const int p = tid + x * NTH;
      const char* fp = f + (p >> 6) * kFragBytes + (p & 63) * 16;
      rf[x][0] = *reinterpret_cast<const f32x4*>(fp);
      rf[x][1] = *reinterpret_cast<const f32x4*>(fp + 1024);
    }
    const float* gp = a.gate + cu * kGateFloats;
#pragma unroll
    for (int x = 0; x < 2; ++x)
      if (tid + x * NTH < 4 * kDC) rg[x] = gp[tid + x * NTH];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = lab(m, 4 * g) + e;
#pragma unroll
        for (int n = 0; n < NT; ++n) rv[(4 * m + e) * NT + n] = (E)0.0f;
        if (t < nt && col0 < a.dv) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
            rv[(4 * m + e) * NT + n] = dop[(long)(t0 + t) * a.d_out.t + col0 + n];
        }
      }
  };
  if (a.r0 < a.r1) fetch(a.r1 - 1);

  for (int r = a.r1 - 1; r >= a.r0; --r) {
    const int t0 = r * kDC;
    const long cu = u * a.nc_buf + (r - a.r_base);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PK; ++x) {
      const int p = tid + x * NTH;
      *reinterpret_cast<uint4*>(ks + L::at(p / L::NP, p % L::NP)) = rk[x];
      *reinterpret_cast<uint4*>(qs + L::at(p / L::NP, p % L::NP)) = rq[x];
    }
#pragma unroll
    for (int x = 0; x < PF; ++x) {
      const int p = tid + x * NTH;
      if (p < NF / 2)
        put_frag<BF, O::NT>(ts, p, rf[x][0], rf[x][1]);
      else
        put_frag<BF, O::NT>(ps, p - NF / 2, rf[x][0], rf[x][1]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
      if (tid + x * NTH < 4 * kDC) gl[tid + x * NTH] = rg[x];
    float vv[16 * NT];
#pragma unroll
    for (int x = 0; x < 16 * NT; ++x) vv[x] = (float)rv[x];
    const float gC = a.gate[cu * kGateFloats + kGC];
    __syncthreads();
    if (r > a.r0) fetch(r - 1);

    typename O::S sb[KT][NT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        sb[kt][n] = O::template split<3>(st[2 * kt][n], st[2 * kt + 1][n]);
        if (col0 + n < a.dvp) {
          float* p = a.dwst + (cu * a.dvp + col0 + n) * DK + 32 * kt + 8 * g;
          *reinterpret_cast<f32x4*>(p) = st[2 * kt][n];
          *reinterpret_cast<f32x4*>(p + 4) = st[2 * kt + 1][n];
        }
      }
    f32x4 xa[4][NT];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f32x4 en = *reinterpret_cast<const f32x4*>(gl + kGEnd + lab(m, 4 * g));
#pragma unroll
      for (int n = 0; n < NT; ++n) xa[m][n] = zero4();
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const auto kf = L::frag(ks, lab(m, c), kt, g);
#pragma unroll
        for (int n = 0; n < NT; ++n) xa[m][n] = O::template xs<3>(xa[m][n], kf, sb[kt][n]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) xa[m][n] = xa[m][n] * en;
    }
    // dO as an operand, and s G dO
    typename O::X dob[2][NT];
    typename O::S gb[2][NT];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const f32x4 s0 = *reinterpret_cast<const f32x4*>(gl + kGsG + lab(2 * x, 4 * g));
      const f32x4 s1 = *reinterpret_cast<const f32x4*>(gl + kGsG + lab(2 * x + 1, 4 * g));
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        f32x4 d0, d1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          d0[e] = vv[(8 * x + e) * NT + n];
          d1[e] = vv[(8 * x + 4 + e) * NT + n];
        }
        dob[x][n] = O::exact(d0, d1);
        gb[x][n] = O::template split<3>(d0 * s0, d1 * s1);
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int x = m / 2; x < 2; ++x) {
        const auto pf = ld_frag_t<BF, 3>(ps, m, x, g, c);
#pragma unroll
        for (int n = 0; n < NT; ++n) xa[m][n] = O::template sx<3>(xa[m][n], pf, dob[x][n]);
      }
    typename O::S rb[2][NT];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int n = 0; n < NT; ++n) rb[x][n] = O::template split<3>(xa[2 * x][n], xa[2 * x + 1][n]);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
#pragma unroll
      for (int n = 0; n < NT; ++n) xa[m][n] = zero4();
#pragma unroll
      for (int x = m / 2; x < 2; ++x) {
        const auto tf = ld_frag_t<BF, 3>(ts, m, x, g, c);
#pragma unroll
        for (int n = 0; n < NT; ++n) xa[m][n] = O::template ss<3>(xa[m][n], tf, rb[x][n]);
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (col0 + n < a.dvp) {
          float* p = a.yst + (cu * a.dvp + col0 + n) * kDC + 32 * x + 8 * g;
          *reinterpret_cast<f32x4*>(p) = xa[2 * x][n];
          *reinterpret_cast<f32x4*>(p + 4) = xa[2 * x + 1][n];
        }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f32x4 eta = *reinterpret_cast<const f32x4*>(gl + kGEta + lab(m, 4 * g));
      const f32x4 eg = *reinterpret_cast<const f32x4*>(gl + kGEtaG + lab(m, 4 * g));
      if (col0 < a.dv) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = t0 + lab(m, 4 * g) + e;
          if (t < a.T) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
              dvp[(long)t * a.dv_.t + col0 + n] = (E)(eta[e] * xa[m][n][e]);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) xa[m][n] = xa[m][n] * -eg;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int n = 0; n < NT; ++n) rb[x][n] = O::template split<3>(xa[2 * x][n], xa[2 * x + 1][n]);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int n = 0; n < NT; ++n) st[m][n] = st[m][n] * gC;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const auto qf = L::template frag_t<false>(qs, m, x, g, c);
        const auto kf = L::template frag_t<false>(ks, m, x, g, c);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          st[m][n] = O::template xs<3>(st[m][n], qf, gb[x][n]);
          st[m][n] = O::template xs<3>(st[m][n], kf, rb[x][n]);
        }
      }
    }
  }

  if (a.d_w_in) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int kcol = lab(m, 4 * g);
        if (col0 + n < a.dv && kcol < a.dk)
          *reinterpret_cast<f32x4*>(a.d_w_in + (u * a.dv + col0 + n) * a.dk + kcol) = st[m][n];
      }
  }
}

template <bool BF, int DK, int NT, int NW>
hipError_t go(const DeltaArgs& a, hipStream_t s) {
  const int nsl = (a.dvp + 16 * NT * NW - 1) / (16 * NT * NW);
  const long u8 = ((long)a.B * a.H + 7) / 8 * 8;
  hipLaunchKernelGGL((delta_bwd_kernel<BF, DK, NT, NW>), dim3((unsigned)(u8 * nsl)), dim3(64 * NW),
                     0, s, a, nsl);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_chain_bwd(const DeltaArgs& a, bool bf, hipStream_t s) {
  const int dkp = delta_dkp(a.dk);
  if (bf) {
    if (dkp == 32) return go<true, 32, 1, 2>(a, s);
    if (dkp == 64) return go<true, 64, 1, 4>(a, s);
    return go<true, 128, 1, 4>(a, s);
  }
  if (dkp == 32) return go<false, 32, 1, 2>(a, s);
  if (dkp == 64) return go<false, 64, 1, 4>(a, s);
  return go<false, 128, 1, 4>(a, s);
}

}  // namespace e2ttt
