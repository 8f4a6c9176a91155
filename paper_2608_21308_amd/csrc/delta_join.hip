// Gated delta rule in segments: the states that the segments start from (see
// delta_fwd.hip),   W_{p+1} = W_p F_p + B_p   from w_in, or in the backward
// those that they end with,   dW_{p-1} = dW_p F_p^T + B_p   from d_w_out.
//
// One workgroup per unit and 16 rows of W (columns of W^T), a wave per 16 rows
// of W^T, so that a step is dk / 32 products of fp32 accuracy a wave; the state
// goes round through LDS, and the next F is on its way meanwhile.  A step takes
// about a microsecond, a few for a call.
#include "delta_common.h"

namespace e2ttt {
namespace {

template <int DK, bool BWD>
__global__ void __launch_bounds__(4 * DK) delta_join_kernel(DeltaArgs a) {
  using O = DOp<true>;     // (fp32 products by bf16 terms, whatever the io type)
  constexpr int KT = DK / 32, LD = DK + 4;
  __shared__ __align__(16) float ws[2][16 * LD];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int w = wave_id();
  const int nvt = a.dvp / 16;
  const long u = blockIdx.x / nvt;
  const int tile = (int)(blockIdx.x % nvt);
  const int row = 16 * tile + c, kc = lab(w, 4 * g);     // the lane's row of W, its columns kc ..
  const int first = BWD ? a.nseg - 1 : 0, step = BWD ? -1 : 1;
  const float* from = BWD ? a.d_w_out : a.w_in;
  f32x4 st = zero4();
  if (from && row < a.dv && kc < a.dk)
    st = *reinterpret_cast<const f32x4*>(from + (u * a.dv + row) * a.dk + kc);
  f32x4 f[KT][2], bb;
  auto fetch = [&](int p) {
    const float* fp = a.segf + (u * a.nseg + p) * 2 * DK * DK;
    const int r = lab(w, c);                             // row of the operand
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      // F^T (forward): row r, columns 32 kt + 8 g ..; F (backward) in lane order
      const float* q = BWD ? fp + lane_at(r >> 4, kt, KT, 16 * g + (r & 15))
                           : fp + DK * DK + r * DK + 32 * kt + 8 * g;
      f[kt][0] = *reinterpret_cast<const f32x4*>(q);
      f[kt][1] = *reinterpret_cast<const f32x4*>(q + (BWD ? 256 : 4));
    }
    bb = *reinterpret_cast<const f32x4*>(a.segb + (u * a.nseg + p) * a.dvp * DK +
                                         lane_at(tile, w >> 1, KT, lane) + 256 * (w & 1));
  };
  fetch(first);
  for (int i = 0; i + 1 < a.nseg; ++i) {
    const int p = first + step * i;
    float* s = ws[i & 1];
    *reinterpret_cast<f32x4*>(s + c * LD + kc) = st;
    __syncthreads();                                     // (the other buffer is read until the next)
    st = bb;
    O::S fa[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) fa[kt] = O::split<3>(f[kt][0], f[kt][1]);
    if (i + 2 < a.nseg) fetch(p + step);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const float* q = s + c * LD + 32 * kt + 8 * g;
      st = O::ss<3>(st, fa[kt], O::split<3>(*reinterpret_cast<const f32x4*>(q),
                                            *reinterpret_cast<const f32x4*>(q + 4)));
    }
    *reinterpret_cast<f32x4*>(a.segs + (u * a.nseg + p + step) * a.dvp * DK +
                              lane_at(tile, w >> 1, KT, lane) + 256 * (w & 1)) = st;
  }
}

template <bool BWD>
hipError_t go(const DeltaArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.B * a.H * (a.dvp / 16)));
  switch (delta_dkp(a.dk)) {
    case 32: hipLaunchKernelGGL((delta_join_kernel<32, BWD>), grid, dim3(128), 0, s, a); break;
    case 64: hipLaunchKernelGGL((delta_join_kernel<64, BWD>), grid, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((delta_join_kernel<128, BWD>), grid, dim3(512), 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_join(const DeltaArgs& a, bool bwd, hipStream_t stream) {
  return bwd ? go<true>(a, stream) : go<false>(a, stream);
}

}  // namespace e2ttt
