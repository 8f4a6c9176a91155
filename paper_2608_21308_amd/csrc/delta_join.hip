// Gated delta rule in segments: the states that the segments start from (see
// delta_fwd.hip),   W_{p+1} = W_p F_p + B_p   from w_in, or in the backward
// those that they end with,   dW_{p-1} = dW_p F_p^T + B_p   from d_w_out.
//
// One workgroup per unit and 16 rows of W (columns of W^T), a wave per 16 rows
// of W^T, so that a step is dk / 32 products of the state's precision a wave; the state
// goes round through LDS, and the next two F are on their way meanwhile.  Bound
// by that round: 1 us a segment at dk = 64, 2 us at 128 (backward 3).
#include "delta_common.h"

namespace e2ttt {
namespace {

template <bool BF, int DK, bool BWD>
__global__ void __launch_bounds__(4 * DK) delta_join_kernel(DeltaArgs a) {
  using O = DOp<BF>;
  using E = typename O::E;
  constexpr int KT = DK / 32, LD = DK + 8;
  __shared__ __align__(16) E ws[2][O::NT][16 * LD];       // the state's rows, in terms
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int w = wave_id();
  const int nvt = a.dvp / 16;
  // the tiles of a unit, which read the same F, go to one XCD
  const long u = (blockIdx.x / (8 * nvt)) * 8 + blockIdx.x % 8;
  if (u >= (long)a.B * a.H) return;
  const int tile = (int)(blockIdx.x / 8 % nvt);
  const int row = 16 * tile + c, kc = lab(w, 4 * g);     // the lane's row of W, its columns kc ..
  const int live = live_tokens(a, (int)(u / a.H));       // (segments behind it leave the state)
  const int first = BWD ? a.nseg - 1 : 0, step = BWD ? -1 : 1;
  const float* from = BWD ? a.d_w_out : a.w_in;
  f32x4 st = zero4();
  if (from && row < a.dv && kc < a.dk)
    st = *reinterpret_cast<const f32x4*>(from + (u * a.dv + row) * a.dk + kc);
  f32x4 f[2][KT][2], bb[2];                              // two steps' operands under way
  auto fetch = [&](int p, f32x4 (&f)[KT][2], f32x4& bb) {
    const float* fp = a.segf + (u * a.nseg + p) * 2 * DK * DK;
    const int r = lab(w, c);                             // row of the operand
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      // row r, columns 32 kt + 8 g .. of F^T (forward), F (backward)
      const float* q = BWD ? fp + lane_at(r >> 4, kt, KT, 16 * g + (r & 15))
                           : fp + DK * DK + lane_at(w, kt, KT, lane);
      f[kt][0] = *reinterpret_cast<const f32x4*>(q);
      f[kt][1] = *reinterpret_cast<const f32x4*>(q + 256);
    }
    bb = *reinterpret_cast<const f32x4*>(a.segb + (u * a.nseg + p) * a.dvp * DK +
                                         lane_at(tile, w >> 1, KT, lane) + 256 * (w & 1));
  };
  auto one = [&](int i, f32x4 (&f)[KT][2], f32x4& bb) {
    const int p = first + step * i;
    if constexpr (BF) {
      const auto own = O::split(st, zero4());
#pragma unroll
      for (int t = 0; t < O::NT; ++t)
        *reinterpret_cast<bf16x4*>(&ws[i & 1][t][c * LD + kc]) =
            __builtin_shufflevector(own.t[t], own.t[t], 0, 1, 2, 3);
    } else {
      *reinterpret_cast<f32x4*>(&ws[i & 1][0][c * LD + kc]) = st;
    }
    __syncthreads();                                     // (the other buffer is read until the next)
    const f32x4 was = st;
    st = bb;
    typename O::S fa[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) fa[kt] = O::split(f[kt][0], f[kt][1]);
    if (i + 3 < a.nseg) fetch(p + 2 * step, f, bb);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      typename O::S sb;
      const E* row = &ws[i & 1][0][c * LD + 32 * kt + 8 * g];
      if constexpr (BF) {
#pragma unroll
        for (int t = 0; t < O::NT; ++t) sb.t[t] = *reinterpret_cast<const bf16x8*>(row + t * 16 * LD);
      } else {
        sb.a = *reinterpret_cast<const f32x4*>(row);
        sb.b = *reinterpret_cast<const f32x4*>(row + 4);
      }
      st = O::ss(st, fa[kt], sb);
    }
    if ((long)(a.r0 + p * a.seglen) * kDC >= live) st = was;
    *reinterpret_cast<f32x4*>(a.segs + (u * a.nseg + p + step) * a.dvp * DK +
                              lane_at(tile, w >> 1, KT, lane) + 256 * (w & 1)) = st;
  };
  // (the first state too, from where every segment then reads: the launch that
  // reads them writes the last one's result, which may lie where `from` does)
  *reinterpret_cast<f32x4*>(a.segs + (u * a.nseg + first) * a.dvp * DK +
                            lane_at(tile, w >> 1, KT, lane) + 256 * (w & 1)) = st;
  fetch(first, f[0], bb[0]);
  if (a.nseg > 2) fetch(first + step, f[1], bb[1]);
  for (int i = 0; i + 1 < a.nseg; i += 2) {
    one(i, f[0], bb[0]);
    if (i + 2 < a.nseg) one(i + 1, f[1], bb[1]);
  }
}

template <bool BF, bool BWD>
hipError_t go(const DeltaArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(((long)a.B * a.H + 7) / 8 * 8 * (a.dvp / 16)));
  switch (delta_dkp(a.dk)) {
    case 32: hipLaunchKernelGGL((delta_join_kernel<BF, 32, BWD>), grid, dim3(128), 0, s, a); break;
    case 64: hipLaunchKernelGGL((delta_join_kernel<BF, 64, BWD>), grid, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((delta_join_kernel<BF, 128, BWD>), grid, dim3(512), 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_join(const DeltaArgs& a, bool bf, bool bwd, hipStream_t stream) {
  if (bf) return bwd ? go<true, true>(a, stream) : go<true, false>(a, stream);
  return bwd ? go<false, true>(a, stream) : go<false, false>(a, stream);
}

}  // namespace e2ttt
