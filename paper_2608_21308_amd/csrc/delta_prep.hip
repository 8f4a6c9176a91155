// Gated delta rule, the chunks' preparation as a launch of its own (delta_prep.h).
#include "delta_prep.h"

namespace e2ttt {
namespace {

template <bool BF, int DK>
__global__ void __launch_bounds__(256, 4) delta_prep_kernel(DeltaArgs a) {
  __shared__ __align__(16) char lds[kPrepLds];
  prep_chunk<BF, DK>(a, a.r0, a.r1 - a.r0, blockIdx.x, lds);
}

template <bool BF>
hipError_t go(const DeltaArgs& a, hipStream_t s) {
  const long n = (long)a.B * a.H * (a.r1 - a.r0);
  const dim3 grid((unsigned)n), blk(256);
  switch (delta_dkp(a.dk)) {
    case 32: hipLaunchKernelGGL((delta_prep_kernel<BF, 32>), grid, blk, 0, s, a); break;
    case 64: hipLaunchKernelGGL((delta_prep_kernel<BF, 64>), grid, blk, 0, s, a); break;
    default: hipLaunchKernelGGL((delta_prep_kernel<BF, 128>), grid, blk, 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_prep(const DeltaArgs& a, bool bf, hipStream_t stream) {
  return bf ? go<true>(a, stream) : go<false>(a, stream);
}

}  // namespace e2ttt
