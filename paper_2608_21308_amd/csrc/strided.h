// Host-side checks of token tensors given by their strides.
#pragma once

#include "delta_common.h"
#include "e2ttt.h"

namespace e2ttt {

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// The strides of a [B][H][T][inner] tensor: `given`, or C order.
inline e2ttt_strides strides_of(const e2ttt_strides* given, long H, long T, long inner) {
  if (given) return *given;
  return e2ttt_strides{H * T * inner, T * inner, inner};
}
// Strides in range (the rows of a 64-token chunk are addressed in 32 bits);
// with `vec` every row starts on 16 bytes (as its tensor does).
inline bool rows_ok(const e2ttt_strides& s, long elt, bool vec) {
  const int64_t lim = (int64_t)1 << 46;
  for (int64_t x : {s.b, s.h, s.t}) {
    if (x < 0 || x > lim) return false;
    if (vec && (x * elt) % 16) return false;
  }
  return s.t <= ((int64_t)1 << 23);
}
// No two elements of a written tensor share memory: taken by rising stride,
// each dimension (of more than one) starts behind all that the ones before span.
inline bool disjoint(const e2ttt_strides& s, long B, long H, long T, long inner) {
  int64_t st[3] = {s.b, s.h, s.t};
  long n[3] = {B, H, T};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (st[j] > st[j + 1]) {
        const int64_t x = st[j];
        st[j] = st[j + 1];
        st[j + 1] = x;
        const long y = n[j];
        n[j] = n[j + 1];
        n[j + 1] = y;
      }
  double span = (double)inner;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if ((double)st[i] < span) return false;
    span += (double)st[i] * (n[i] - 1);
  }
  return true;
}
inline View view(const void* p, const e2ttt_strides& s) {
  return View{p, (long)s.b, (long)s.h, (long)s.t};
}

// Token tensors [B][H][T][d] of the io type: checked, and as a View.
struct RowSpec {
  long B, T, d;
  int io;
  bool read(const e2ttt_strides* s, const void* p, long H, View* o) const {
    const e2ttt_strides x = strides_of(s, H, T, d);
    *o = view(p, x);
    return rows_ok(x, io == E2TTT_DT_BF16 ? 2 : 4, true) && !misaligned(p);
  }
  bool write(const e2ttt_strides* s, const void* p, long H, View* o) const {
    return read(s, p, H, o) && disjoint(strides_of(s, H, T, d), B, H, T, d);
  }
};

}  // namespace e2ttt
