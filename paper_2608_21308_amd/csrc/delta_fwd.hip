// Gated delta rule, forward chain over the chunks (the mathematics and the
// layouts: delta_common.h).
//
// A wave owns 16 NT columns of W^T (rows of the state: value channels), which
// depend on each other in nothing, and keeps them in fp32 accumulators for the
// whole sequence; a workgroup is NW waves of one unit that share the staged
// chunk (K, Q rows and the T, P fragments).  Per chunk a wave takes
//   X = K W^T,  Y = Q W^T            (W in bf16 terms, K and Q exact)
//   U = T (eta V - eta G X)          (both operands in terms)
//   O = s G Y + P U                  -> out
//   W^T = G_C W^T + K^T (e^{b_C - b} U)
// with every accumulator turned into the next product's operand in place.
// The next chunk's global loads are issued before the current one's products.
#include "delta_common.h"

namespace e2ttt {
namespace {

template <bool BF, int DK, int NT, int NW, bool SAVE>
__global__ void __launch_bounds__(64 * NW) delta_fwd_kernel(DeltaArgs a, int nsl) {
  using O = DOp<BF>;
  using E = typename O::E;
  using L = LTile<BF, DK>;
  constexpr int NTH = 64 * NW, KT = DK / 32, MT = DK / 16;
  constexpr int NP = kDC * L::NP;                       // pieces of a token tile
  constexpr int PK = (NP + NTH - 1) / NTH;
  constexpr int NF = 2 * kDeltaFrags * 64, PF = NF / NTH;  // lanes' parts of the T and P fragments
  static_assert(NP % NTH == 0 && NF % NTH == 0, "whole rounds of pieces");
  __shared__ __align__(16) E ks[kDC * DK];
  __shared__ __align__(16) E qs[kDC * DK];
  __shared__ __align__(16) char ts[tri_lds<BF>(O::NT)];
  __shared__ __align__(16) char ps[tri_lds<BF>(2)];
  __shared__ __align__(16) float gl[kGateFloats];

  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
  // the slices of a unit go to one XCD (workgroups are dealt to the eight in turn)
  const long U = (long)a.B * a.H;
  const long blk = blockIdx.x;
  const long u = (blk / (8 * nsl)) * 8 + blk % 8;
  if (u >= U) return;
  const int sl = (int)((blk / 8) % nsl);
  const int b = (int)(u / a.H), h = (int)(u % a.H), hk = h / (a.H / a.HK);
  const int nlive = live_tokens(a, b);
  const int col0 = (sl * NW + w) * 16 * NT + NT * c;     // the lane's columns: col0 + n
  const E* kp = row_of<E>(a.k, b, hk, 0);
  const E* qp = row_of<E>(a.q, b, hk, 0);
  const E* vp = row_of<E>(a.v, b, h, 0);
  E* op = row_of_w<E>(a.out, b, h, 0);

  f32x4 st[MT][NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int kcol = lab(m, 4 * g);
      st[m][n] = zero4();
      if (a.w_in && col0 + n < a.dv && kcol < a.dk)
        st[m][n] = *reinterpret_cast<const f32x4*>(a.w_in + (u * a.dv + col0 + n) * a.dk + kcol);
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
    for (int x = 0; x < 2; ++x)      // the first four arrays and G_C
      if (tid + x * NTH < 4 * kDC) rg[x] = gp[tid + x * NTH];
  };
  auto fetch_v = [&](int r) {
    const int t0 = r * kDC, nt = nlive - t0;
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
            rv[(4 * m + e) * NT + n] = vp[(long)(t0 + t) * a.v.t + col0 + n];
        }
      }
  };
  if (a.r0 < a.r1) {
    fetch(a.r0);
    fetch_v(a.r0);
  }

  for (int r = a.r0; r < a.r1; ++r) {
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
        put_frag<BF, 2>(ps, p - NF / 2, rf[x][0], rf[x][1]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
      if (tid + x * NTH < 4 * kDC) gl[tid + x * NTH] = rg[x];
    float vv[16 * NT];
#pragma unroll
    for (int x = 0; x < 16 * NT; ++x) vv[x] = (float)rv[x];
    const float gC = a.gate[cu * kGateFloats + kGC];
    __syncthreads();
    if (r + 1 < a.r1) {
      fetch(r + 1);
      fetch_v(r + 1);
    }

    typename O::S sb[KT][NT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        sb[kt][n] = O::template split<3>(st[2 * kt][n], st[2 * kt + 1][n]);
        if constexpr (SAVE) {
          const int row = col0 + n;
          if (row < a.dvp) {
            float* p = a.wst + (cu * a.dvp + row) * DK + 32 * kt + 8 * g;
            *reinterpret_cast<f32x4*>(p) = st[2 * kt][n];
            *reinterpret_cast<f32x4*>(p + 4) = st[2 * kt + 1][n];
          }
        }
      }
    f32x4 xa[4][NT], oa[4][NT];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
#pragma unroll
      for (int n = 0; n < NT; ++n) xa[m][n] = oa[m][n] = zero4();
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const auto kf = L::frag(ks, lab(m, c), kt, g);
#pragma unroll
        for (int n = 0; n < NT; ++n) xa[m][n] = O::template xs<3>(xa[m][n], kf, sb[kt][n]);
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const auto qf = L::frag(qs, lab(m, c), kt, g);
#pragma unroll
        for (int n = 0; n < NT; ++n) oa[m][n] = O::template xs<2>(oa[m][n], qf, sb[kt][n]);
      }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f32x4 eta = *reinterpret_cast<const f32x4*>(gl + kGEta + lab(m, 4 * g));
      const f32x4 eg = *reinterpret_cast<const f32x4*>(gl + kGEtaG + lab(m, 4 * g));
      const f32x4 sg = *reinterpret_cast<const f32x4*>(gl + kGsG + lab(m, 4 * g));
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          xa[m][n][e] = eta[e] * vv[(4 * m + e) * NT + n] - eg[e] * xa[m][n][e];
          oa[m][n][e] *= sg[e];
        }
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
      for (int x = 0; x <= m / 2; ++x) {
        const auto tf = ld_frag<BF, 3>(ts, fidx(m, x), lane);
#pragma unroll
        for (int n = 0; n < NT; ++n) xa[m][n] = O::template ss<3>(xa[m][n], tf, rb[x][n]);
      }
    }
    typename O::S ub[2][NT];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        ub[x][n] = O::template split<3>(xa[2 * x][n], xa[2 * x + 1][n]);
        if constexpr (SAVE) {
          const int row = col0 + n;
          if (row < a.dvp) {
            float* p = a.ust + (cu * a.dvp + row) * kDC + 32 * x + 8 * g;
            *reinterpret_cast<f32x4*>(p) = xa[2 * x][n];
            *reinterpret_cast<f32x4*>(p + 4) = xa[2 * x + 1][n];
          }
        }
      }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
#pragma unroll
      for (int x = 0; x <= m / 2; ++x) {
        const auto pf = ld_frag<BF, 2>(ps, fidx(m, x), lane);
#pragma unroll
        for (int n = 0; n < NT; ++n) oa[m][n] = O::template ss<2>(oa[m][n], pf, ub[x][n]);
      }
      if (col0 < a.dv) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = t0 + lab(m, 4 * g) + e;
          if (t < a.T) {
#pragma unroll
            for (int n = 0; n < NT; ++n) op[(long)t * a.out.t + col0 + n] = (E)oa[m][n][e];
          }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f32x4 en = *reinterpret_cast<const f32x4*>(gl + kGEnd + lab(m, 4 * g));
#pragma unroll
      for (int n = 0; n < NT; ++n) xa[m][n] = xa[m][n] * en;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int n = 0; n < NT; ++n) ub[x][n] = O::template split<3>(xa[2 * x][n], xa[2 * x + 1][n]);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int n = 0; n < NT; ++n) st[m][n] = st[m][n] * gC;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const auto kf = L::template frag_t<false>(ks, m, x, g, c);
#pragma unroll
        for (int n = 0; n < NT; ++n) st[m][n] = O::template xs<3>(st[m][n], kf, ub[x][n]);
      }
    }
  }

  if (a.w_out) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int kcol = lab(m, 4 * g);
        if (col0 + n < a.dv && kcol < a.dk)
          *reinterpret_cast<f32x4*>(a.w_out + (u * a.dv + col0 + n) * a.dk + kcol) = st[m][n];
      }
  }
}

template <bool BF, int DK, int NT, int NW>
hipError_t go(const DeltaArgs& a, bool save, hipStream_t s) {
  const int nsl = (delta_dvp(a.dv) + 16 * NT * NW - 1) / (16 * NT * NW);
  const long u8 = ((long)a.B * a.H + 7) / 8 * 8;
  const dim3 grid((unsigned)(u8 * nsl)), blk(64 * NW);
  if (save)
    hipLaunchKernelGGL((delta_fwd_kernel<BF, DK, NT, NW, true>), grid, blk, 0, s, a, nsl);
  else
    hipLaunchKernelGGL((delta_fwd_kernel<BF, DK, NT, NW, false>), grid, blk, 0, s, a, nsl);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_chain(const DeltaArgs& a, bool bf, bool save, hipStream_t s) {
  const int dkp = delta_dkp(a.dk);
  if (bf) {
    if (dkp == 32) return go<true, 32, 1, 2>(a, save, s);
    if (dkp == 64) return go<true, 64, 1, 4>(a, save, s);
    return go<true, 128, 1, 4>(a, save, s);
  }
  if (dkp == 32) return go<false, 32, 1, 2>(a, save, s);
  if (dkp == 64) return go<false, 64, 1, 4>(a, save, s);
  return go<false, 128, 1, 4>(a, save, s);
}

}  // namespace e2ttt
