// Gated delta rule, the chunks' gradients as a launch of their own (delta_grads.h).
#include "delta_grads.h"

namespace e2ttt {
namespace {

template <bool BF, int DK, int NWV, bool ONE>
__global__ void __launch_bounds__(64 * NWV, 2) delta_grads_kernel(DeltaArgs a) {
  __shared__ __align__(16) char lds[GradsLds<BF, DK, NWV>::bytes];
  grads_chunk<BF, DK, NWV, ONE>(a, a.r0, a.r1 - a.r0, blockIdx.x, lds);
}

template <bool BF, int DK, int NWV>
hipError_t go(const DeltaArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.B * a.HK * (a.r1 - a.r0))), blk(64 * NWV);
  if (a.H == a.HK)
    hipLaunchKernelGGL((delta_grads_kernel<BF, DK, NWV, true>), grid, blk, 0, s, a);
  else
    hipLaunchKernelGGL((delta_grads_kernel<BF, DK, NWV, false>), grid, blk, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_grads(const DeltaArgs& a, bool bf, hipStream_t s) {
  const int dkp = delta_dkp(a.dk);
  if (bf) {
    if (dkp == 32) return go<true, 32, 4>(a, s);
    if (dkp == 64) return go<true, 64, 4>(a, s);
    return go<true, 128, 8>(a, s);
  }
  if (dkp == 32) return go<false, 32, 4>(a, s);
  if (dkp == 64) return go<false, 64, 4>(a, s);
  return go<false, 128, 8>(a, s);
}

}  // namespace e2ttt
