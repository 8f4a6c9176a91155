// Division by numbers that a launch fixes.
#pragma once

#include <hip/hip_runtime.h>

namespace e2ttt {

// Division by a fixed number in five scalar instructions (Granlund and Montgomery 1994):
// with l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1, n / d is (t + (n - t) / 2) /
// 2^(l - 1), t the upper half of m n, for every n (d = 1: l - 1 counts as 0 and t is 0).
struct Div {
  unsigned d, m, s1, s2;
  __device__ __forceinline__ unsigned of(unsigned n) const {
    const unsigned t = __umulhi(m, n);
    return (t + ((n - t) >> s1)) >> s2;
  }
};
inline Div div_by(unsigned d) {
  unsigned l = 0;
  while (l < 32 && (1ull << l) < d) ++l;
  const unsigned m = (unsigned)((((1ull << l) - d) << 32) / d + 1);
  return Div{d, m, l > 1 ? 1 : l, l > 0 ? l - 1 : 0};
}

}  // namespace e2ttt
