// Preparation of queries and keys (e2ttt_qk_forward / e2ttt_qk_backward): per
// row x of d elements, each step optional,
//   s = SiLU(x),   y = s / sqrt(sum s^2 + eps),
//   z = y with its first `rot` elements turned: for pair p of channels (a, b),
//       z_a = m (y_a cos - y_b sin),  z_b = m (y_b cos + y_a sin),
//       angle = position * inv_freq[p],  m = rot_scale.
// The backward turns dz back (the transposed map), then with r = 1 / sqrt(..)
//   ds = r (dy - s r^2 (s . dy)),  dx = ds sigma(x) (1 + x (1 - sigma(x))).
//
// Bound by HBM: each element is read once (twice in the backward, with its
// gradient) and written once.  An item is the two pieces of V elements that hold V whole
// pairs (p and p + rot / 2 of a half layout, neighbours otherwise), so a pair
// never leaves its lane; V is the widest that divides rot / 2 (16 bytes for
// the usual head; an odd rot / 2 goes element by element, tail included: 8 x 4096
// tokens of 16 + 16 heads of 128 take 204 and 303 us with rot = 34, 143 and 199 with
// 32).  The lanes of a row sum by shuffles.  A group of lanes
// keeps its angles' sines and cosines over several heads of a token.  Angles
// are reduced in 64 bits: a far position times a frequency loses its fraction
// of a turn in 32.  8 x 4096 tokens of 16 + 16 heads of 64: 55 us forward, 76
// backward, 4.9 and 5.3 TB/s, the rate of a large copy.
#include <math.h>

#include "delta_common.h"
#include "e2ttt.h"
#include "strided.h"

namespace e2ttt {
namespace {

struct QkArgs {
  View x[2], y[2], g[2];      // queries, keys: input, output (gradient of x), gradient of z
  const float* inv_freq;
  const int64_t* pos;         // nullable: 0 .. T - 1
  int B, T, d, half;          // half: pairs that turn (rot / 2)
  int nh[2];                  // heads of queries and keys
  int hpg, nhg;               // heads of a group of lanes, groups of heads
  int lanes, llanes;          // lanes of a row (a power of two), its logarithm
  int tfast;                  // neighbouring groups: tokens (else heads)
  float eps, m;
};

template <class E, int V> struct Piece { typedef __attribute__((ext_vector_type(V))) E T; };
template <class E> struct Piece<E, 1> { typedef E T; };

template <class E, int V>
__device__ __forceinline__ void widen(float (&o)[V], const typename Piece<E, V>::T& x) {
  if constexpr (V == 1) {
    o[0] = (float)x;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = (float)x[i];
  }
}
template <class E, int V>
__device__ __forceinline__ void st_piece(E* p, const float (&v)[V]) {
  typename Piece<E, V>::T x;
  if constexpr (V == 1) {
    x = (E)v[0];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (E)v[i];
  }
  __builtin_nontemporal_store(x, reinterpret_cast<typename Piece<E, V>::T*>(p));
}

// Sum over the lanes of a row (a power of two, neighbours).
__device__ __forceinline__ float row_sum(float v, int lanes) {
  if (lanes > 1) v += dpp_f<0xB1>(v);    // quad_perm [1,0,3,2]
  if (lanes > 2) v += dpp_f<0x4E>(v);    // quad_perm [2,3,0,1]
  if (lanes > 4) v += dpp_f<0x141>(v);   // row_half_mirror
  if (lanes > 8) v += dpp_f<0x140>(v);   // row_mirror
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
}

// sigma(x), to a few 2^-24 of its value however small (below 2^-126 it is zero), by
// the hardware's exponential and reciprocal, an ulp each.  e^-x is 2^h (1 + d), h = -x
// times the upper 16 bits of log2 e and d = -x times the rest of ln 2 log2 e: a bf16
// x gives h without rounding, a float's rounding is put into d.  (e^-104 is zero; d > 0
// where 2^h overflows.)
template <bool BF>
__device__ __forceinline__ float sigma(float x) {
  const float y = fmaxf(-x, -104.0f), h = y * 1.44268799f;
  float d = y * 4.8885e-6f;
  if constexpr (!BF) d = fmaf(fmaf(y, 1.44268799f, -h), 0.693147181f, d);
  const float p = __builtin_amdgcn_exp2f(h);
  return rcp_f(1.0f + fmaf(p, d, p));
}

// m times cosine and sine of 2 pi t, |t| <= 1/2: Taylor's series to x^10 around
// the nearest quarter turn, which is taken off in 64 bits (|x| <= pi / 4; the
// remainders, x^11 / 11! and x^12 / 12!, are below 2^-29).
__device__ __forceinline__ void turn(double t, float m, float& co, float& si) {
  const double q = rint(4.0 * t);
  const float x = (float)(fma(-0.25, q, t) * 6.283185307179586), x2 = x * x;
  float s = fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(x2, s, 8.3333333e-3f);
  s = fmaf(x2, s, -1.6666667e-1f);
  s = m * fmaf(x * x2, s, x);
  float c = fmaf(x2, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(x2, c, -1.3888889e-3f);
  c = fmaf(x2, c, 4.1666667e-2f);
  c = fmaf(x2, c, -0.5f);
  c = m * fmaf(x2, c, 1.0f);
  const int n = (int)q;                     // -2 .. 2 quarter turns
  const float a = n & 1 ? s : c, b = n & 1 ? c : s;
  co = (n + 1) & 2 ? -a : a;
  si = n & 2 ? -b : b;
}

// The pair (a, b) of index i in an item's two pieces.
template <bool INTER, int V>
__device__ __forceinline__ float& first_of(float (&u)[2][V], int i) {
  return INTER ? u[(2 * i) / V][(2 * i) % V] : u[0][i];
}
template <bool INTER, int V>
__device__ __forceinline__ float& second_of(float (&u)[2][V], int i) {
  return INTER ? u[(2 * i + 1) / V][(2 * i + 1) % V] : u[1][i];
}

// IPL: items of a lane.
template <bool BF, int V, int IPL, bool BWD, bool INTER>
__global__ void __launch_bounds__(256) qk_kernel(QkArgs a, unsigned flags) {
  using E = typename DOp<BF>::E;
  using P = typename Piece<E, V>::T;
  // (at most 10^9 rows: 32 bits)
  const unsigned gid = blockIdx.x * (256u >> a.llanes) + (threadIdx.x >> a.llanes);
  const int l = threadIdx.x & (a.lanes - 1);
  const unsigned ntok = (unsigned)a.B * a.T;
  if (gid >= ntok * a.nhg) return;          // whole rows of lanes leave together
  const unsigned tok = a.tfast ? gid % ntok : gid / a.nhg;
  const int hg = (int)(a.tfast ? gid / ntok : gid % a.nhg);
  const int b = (int)(tok / (unsigned)a.T), t = (int)(tok - (unsigned)b * a.T);
  const bool silu = flags & E2TTT_QK_SILU, unit = flags & E2TTT_QK_UNIT;
  const int np = a.half / V;                // items that turn
  const int ntail = (a.d - 2 * a.half) / V; // pieces that do not

  int c0[IPL], c1[IPL];                     // first elements of an item's pieces (-1: none)
  float co[IPL][V], si[IPL][V];
#pragma unroll
  for (int x = 0; x < IPL; ++x) {
    const int it = l + x * a.lanes;
    c0[x] = c1[x] = -1;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      co[x][i] = 1.0f;
      si[x][i] = 0.0f;
    }
    if (it < np) {
      c0[x] = INTER ? 2 * it * V : it * V;
      c1[x] = INTER ? c0[x] + V : c0[x] + a.half;
      const double p = a.pos ? (double)a.pos[tok] : (double)t;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        double turns = p * (double)a.inv_freq[it * V + i] * 0.15915494309189535;
        turns -= rint(turns);
        turn(turns, a.m, co[x][i], si[x][i]);
      }
    } else {
      const int q = 2 * (it - np);
      if (q < ntail) c0[x] = 2 * a.half + q * V;
      if (q + 1 < ntail) c1[x] = 2 * a.half + (q + 1) * V;
    }
  }

  // rows of this token: queries, then keys
  const E* xb[2] = {row_of<E>(a.x[0], b, 0, t), row_of<E>(a.x[1], b, 0, t)};
  const E* gb[2] = {row_of<E>(a.g[0], b, 0, t), row_of<E>(a.g[1], b, 0, t)};
  E* yb[2] = {row_of_w<E>(a.y[0], b, 0, t), row_of_w<E>(a.y[1], b, 0, t)};
  const bool need = !BWD || silu || unit;
  P rx[IPL][2], rg[IPL][2];                 // the next row, as it lies in memory
  auto load = [&](int hh) {
    const bool s = hh >= a.nh[0];
    const long h = s ? hh - a.nh[0] : hh;
    const E* xp = (s ? xb[1] : xb[0]) + h * (s ? a.x[1].h : a.x[0].h);
    const E* gp = (s ? gb[1] : gb[0]) + h * (s ? a.g[1].h : a.g[0].h);
#pragma unroll
    for (int x = 0; x < IPL; ++x)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int at = k ? c1[x] : c0[x];
        rx[x][k] = rg[x][k] = P{};
        if (at >= 0) {
          if (need) rx[x][k] = *reinterpret_cast<const P*>(xp + at);
          if (BWD) rg[x][k] = *reinterpret_cast<const P*>(gp + at);
        }
      }
  };
  const int h1 = min(a.nh[0] + a.nh[1], (hg + 1) * a.hpg);
  load(hg * a.hpg);
  for (int hh = hg * a.hpg; hh < h1; ++hh) {
    float u[IPL][2][V], z[IPL][2][V], raw[IPL][2][V];
#pragma unroll
    for (int x = 0; x < IPL; ++x)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        widen<E, V>(u[x][k], rx[x][k]);
        if (BWD) widen<E, V>(z[x][k], rg[x][k]);
      }
    if (hh + 1 < h1) load(hh + 1);
    if (BWD) {                              // back through the turn
#pragma unroll
      for (int x = 0; x < IPL; ++x)
        if (l + x * a.lanes < np) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float &p = first_of<INTER, V>(z[x], i), &q = second_of<INTER, V>(z[x], i);
            const float za = p, zb = q;
            p = za * co[x][i] + zb * si[x][i];
            q = zb * co[x][i] - za * si[x][i];
          }
        }
    }
    if (silu) {
#pragma unroll
      for (int x = 0; x < IPL; ++x)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float sg = sigma<BF>(u[x][k][i]);
            if (BWD) raw[x][k][i] = sg * fmaf(u[x][k][i], 1.0f - sg, 1.0f);   // the derivative
            u[x][k][i] *= sg;
          }
    }
    float r = 1.0f, f = 0.0f;
    if (unit) {
      float ss = 0.0f, sd = 0.0f;
#pragma unroll
      for (int x = 0; x < IPL; ++x)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            ss = fmaf(u[x][k][i], u[x][k][i], ss);
            if (BWD) sd = fmaf(u[x][k][i], z[x][k][i], sd);
          }
      r = rsq_f(row_sum(ss, a.lanes) + a.eps);
      if (BWD) f = row_sum(sd, a.lanes) * r * r;
    }
#pragma unroll
    for (int x = 0; x < IPL; ++x)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) u[x][k][i] = BWD ? r * fmaf(-f, u[x][k][i], z[x][k][i]) : r * u[x][k][i];
    if (BWD && silu) {
#pragma unroll
      for (int x = 0; x < IPL; ++x)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < V; ++i) u[x][k][i] *= raw[x][k][i];
    }
    const bool s = hh >= a.nh[0];
    const long h = s ? hh - a.nh[0] : hh;
    E* yp = (s ? yb[1] : yb[0]) + h * (s ? a.y[1].h : a.y[0].h);
#pragma unroll
    for (int x = 0; x < IPL; ++x) {
      if (!BWD && l + x * a.lanes < np) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float &p = first_of<INTER, V>(u[x], i), &q = second_of<INTER, V>(u[x], i);
          const float ya = p, yb_ = q;
          p = ya * co[x][i] - yb_ * si[x][i];
          q = yb_ * co[x][i] + ya * si[x][i];
        }
      }
      if (c0[x] >= 0) st_piece<E, V>(yp + c0[x], u[x][0]);
      if (c1[x] >= 0) st_piece<E, V>(yp + c1[x], u[x][1]);
    }
  }
}

// The widest pieces of a head, the lanes of a row, and how many heads a group
// of lanes takes.
struct Shape {
  int v, items, llanes, hpg, nhg;
  long blocks;
};
Shape shape_of(const e2ttt_qk_desc* d) {
  Shape s;
  const int h = d->rot / 2;
  s.v = d->io == E2TTT_DT_BF16 && h % 8 == 0 ? 8 : h % 4 == 0 ? 4 : h % 2 == 0 ? 2 : 1;
  s.items = h / s.v + ((d->d - 2 * h) / s.v + 1) / 2;
  s.llanes = 0;
  while ((1 << s.llanes) < s.items && s.llanes < 6) ++s.llanes;
  // Several heads to a group (their angles are the same) as long as the card
  // stays full: 256 CUs of 2048 lanes.
  const long tokens = (long)d->B * d->T, heads = (long)d->H + d->HK;
  s.hpg = 1;
  while (s.hpg < 8 && ((tokens * heads / (2 * s.hpg)) << s.llanes) >= 256L * 2048) s.hpg *= 2;
  s.nhg = (int)((heads + s.hpg - 1) / s.hpg);
  s.blocks = (((tokens * s.nhg) << s.llanes) + 255) / 256;
  return s;
}

template <bool BF, int V, bool BWD>
hipError_t go(const QkArgs& a, const Shape& sh, unsigned flags, hipStream_t s) {
  // (d <= 256: only single pairs to a piece can make more than 64 items)
  constexpr int kMost = V == 1 ? 2 : 1;
  const dim3 grid((unsigned)sh.blocks), blk(256);
  const bool inter = flags & E2TTT_QK_INTERLEAVED;
  if (sh.items > 64) {
    if (inter) hipLaunchKernelGGL((qk_kernel<BF, V, kMost, BWD, true>), grid, blk, 0, s, a, flags);
    else hipLaunchKernelGGL((qk_kernel<BF, V, kMost, BWD, false>), grid, blk, 0, s, a, flags);
  } else {
    if (inter) hipLaunchKernelGGL((qk_kernel<BF, V, 1, BWD, true>), grid, blk, 0, s, a, flags);
    else hipLaunchKernelGGL((qk_kernel<BF, V, 1, BWD, false>), grid, blk, 0, s, a, flags);
  }
  return hipGetLastError();
}

template <bool BWD>
e2ttt_status launch(const QkArgs& a, const e2ttt_qk_desc* d, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf = d->io == E2TTT_DT_BF16;
  const unsigned f = d->flags;
  const Shape sh = shape_of(d);
  hipError_t e;
  if (sh.v == 8) e = go<true, 8, BWD>(a, sh, f, s);
  else if (sh.v == 4) e = bf ? go<true, 4, BWD>(a, sh, f, s) : go<false, 4, BWD>(a, sh, f, s);
  else if (sh.v == 2) e = bf ? go<true, 2, BWD>(a, sh, f, s) : go<false, 2, BWD>(a, sh, f, s);
  else e = bf ? go<true, 1, BWD>(a, sh, f, s) : go<false, 1, BWD>(a, sh, f, s);
  return e == hipSuccess ? E2TTT_OK : E2TTT_ERR_HIP;
}

constexpr unsigned kFlags = E2TTT_QK_SILU | E2TTT_QK_UNIT | E2TTT_QK_INTERLEAVED;

e2ttt_status check_desc(const e2ttt_qk_desc* d) {
  if (!d) return E2TTT_ERR_NULL_ARG;
  if (d->B <= 0 || d->H <= 0 || d->HK < 0 || d->T <= 0 || d->d <= 0 || d->rot < 0 ||
      d->rot > d->d || d->rot % 2)
    return E2TTT_ERR_BAD_SHAPE;
  // (the reciprocal root of a smaller number is infinite, and a row of zeros times it NaN)
  if (!isfinite(d->rot_scale) ||
      ((d->flags & E2TTT_QK_UNIT) && !(isfinite(d->eps) && d->eps >= 1.17549435e-38f)))
    return E2TTT_ERR_BAD_SHAPE;
  if ((d->io != E2TTT_DT_F32 && d->io != E2TTT_DT_BF16) || (d->flags & ~kFlags) || d->d % 8 ||
      d->d > 256 || (double)d->B * d->T * ((double)d->H + d->HK) > 1e9)
    return E2TTT_ERR_UNSUPPORTED;
  // (a launch numbers its threads in 32 bits)
  return shape_of(d).blocks > 0xffffff ? E2TTT_ERR_UNSUPPORTED : E2TTT_OK;
}

QkArgs args_of(const e2ttt_qk_desc* d, const float* inv_freq, const int64_t* pos) {
  QkArgs a{};
  a.B = d->B; a.T = d->T; a.d = d->d; a.half = d->rot / 2;
  a.nh[0] = d->H; a.nh[1] = d->HK;
  a.inv_freq = inv_freq; a.pos = pos;
  a.eps = d->eps; a.m = d->rot_scale;
  const Shape s = shape_of(d);
  a.llanes = s.llanes; a.lanes = 1 << s.llanes;
  a.hpg = s.hpg; a.nhg = s.nhg;
  return a;
}

}  // namespace
}  // namespace e2ttt

using namespace e2ttt;

extern "C" e2ttt_status e2ttt_qk_forward(const e2ttt_qk_desc* desc, const e2ttt_qk_strides* strides,
                                         const void* q, const void* k, const float* inv_freq,
                                         const int64_t* positions, void* q_out, void* k_out,
                                         void* stream) {
  e2ttt_status st = check_desc(desc);
  if (st != E2TTT_OK) return st;
  const bool ks = desc->HK > 0;
  if (!q || !q_out || (ks && (!k || !k_out)) || (desc->rot && !inv_freq)) return E2TTT_ERR_NULL_ARG;
  QkArgs a = args_of(desc, inv_freq, positions);
  const RowSpec in{desc->B, desc->T, desc->d, desc->io};
  if (!in.read(strides ? &strides->q : nullptr, q, desc->H, &a.x[0]) ||
      !in.write(strides ? &strides->q_out : nullptr, q_out, desc->H, &a.y[0]) ||
      (ks && (!in.read(strides ? &strides->k : nullptr, k, desc->HK, &a.x[1]) ||
              !in.write(strides ? &strides->k_out : nullptr, k_out, desc->HK, &a.y[1]))))
    return E2TTT_ERR_BAD_SHAPE;
  a.tfast = a.x[0].t < a.x[0].h;
  return launch<false>(a, desc, stream);
}

extern "C" e2ttt_status e2ttt_qk_backward(const e2ttt_qk_desc* desc,
                                          const e2ttt_qk_strides* strides, const void* q,
                                          const void* k, const float* inv_freq,
                                          const int64_t* positions, const void* d_q_out,
                                          const void* d_k_out, void* dq, void* dk, void* stream) {
  e2ttt_status st = check_desc(desc);
  if (st != E2TTT_OK) return st;
  const bool ks = desc->HK > 0;
  const bool need = desc->flags & (E2TTT_QK_SILU | E2TTT_QK_UNIT);   // x itself
  if ((need && (!q || (ks && !k))) || !d_q_out || !dq || (ks && (!d_k_out || !dk)) ||
      (desc->rot && !inv_freq))
    return E2TTT_ERR_NULL_ARG;
  QkArgs a = args_of(desc, inv_freq, positions);
  const RowSpec in{desc->B, desc->T, desc->d, desc->io};
  const bool ok =
      (!need || in.read(strides ? &strides->q : nullptr, q, desc->H, &a.x[0])) &&
      in.read(strides ? &strides->d_q_out : nullptr, d_q_out, desc->H, &a.g[0]) &&
      in.write(strides ? &strides->dq : nullptr, dq, desc->H, &a.y[0]) &&
      (!ks || ((!need || in.read(strides ? &strides->k : nullptr, k, desc->HK, &a.x[1])) &&
               in.read(strides ? &strides->d_k_out : nullptr, d_k_out, desc->HK, &a.g[1]) &&
               in.write(strides ? &strides->dk : nullptr, dk, desc->HK, &a.y[1])));
  if (!ok) return E2TTT_ERR_BAD_SHAPE;
  a.tfast = a.g[0].t < a.g[0].h;
  return launch<true>(a, desc, stream);
}
