// Attention, backward: the probabilities are formed again from the scores and lse,
// once by queries for dq and once by keys for dk and dv, so that every sum stays in
// its wave's registers and no order of atomics enters the results (seven products
// where five would do with sums in memory):
//   by queries: S^T = K Q^T, U^T = V do^T, dS^T = P^T o (U^T - D), dq^T += K^T dS^T
//   by keys:    S = Q K^T, U = do V^T, dv^T += do^T P, dk^T += Q^T dS.
// The first also leaves D = sum do o - d_lse and the exponents' part of lse for the
// second.  P and dS are rounded
// to the io type as operands (bf16: half a step each, of either sign); all sums and
// the scores are fp32.
#include <math.h>

#include <type_traits>

#include "attn_common.h"

namespace e2ttt {
namespace {

// -lse log2 e, -inf for a query that sees nothing: its 2^(..) are then all zero.  (Another
// lse whose product passes fp32's range does not look like that.)
__device__ __forceinline__ float exponent_of(float lse) {
  const float x = -lse * kLog2e;
  return lse == kNegInf ? kNegInf : x == kNegInf ? NAN : x;
}

template <bool BF, int D, int BK>
__global__ void __launch_bounds__(256, BF ? 2 : 1) attn_dq_kernel(AttnArgs a, int ntile) {
  using O = MOp<BF>;
  using E = typename O::E;
  using X = typename O::X;
  using A = ATile<BF, D>;
  constexpr int NT = BK / 32, KS = D / 16, NM = D / 32;
  __shared__ __align__(16) E lk0[BK * D], lk1[BK * D], lv0[BK * D], lv1[BK * D];
  const int lane = threadIdx.x & 63, w = wave_id(), h = lane >> 5, c = lane & 31;
  const Place wk = place_of(a.work, blockIdx.x);
  const int tile = ntile - 1 - wk.tile;
  const int b = wk.b, hk = wk.hk, hq = hk * a.rep + wk.head, split = wk.split, u = b * a.H + hq;
  const int off = a.S - a.T, live = live_of(a, b), end = live + off;
  const int t0 = tile * 128, tw = t0 + 32 * w, t = tw + c;
  const bool on = t < live;

  X q[KS], g[KS];
  const E* qrow = on ? row_of<E>(a.q, b, hq, t) : nullptr;
  const E* grow = on ? row_of<E>(a.d_out, b, hq, t) : nullptr;
  const E* orow = on ? row_of<E>(a.out, b, hq, t) : nullptr;
  float dot = 0.0f;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    q[s] = row_frag<BF>(qrow, 16 * s + 8 * h, a.d);
    g[s] = row_frag<BF>(grow, 16 * s + 8 * h, a.d);
    const X o = row_frag<BF>(orow, 16 * s + 8 * h, a.d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (BF) dot = fmaf((float)g[s].v[j], (float)o.v[j], dot);
      else dot = fmaf(j < 4 ? g[s].a[j & 3] : g[s].b[j & 3], j < 4 ? o.a[j & 3] : o.b[j & 3], dot);
    }
  }
  dot = both_sum(dot);
  const long at = (long)u * a.T + t;
  float ex = kNegInf;
  if (on) ex = exponent_of(a.lse[at]);
  f32x16 o[NM], none;         // (-D where the products with do begin)
#pragma unroll
  for (int m = 0; m < NM; ++m) o[m] = zero16();
  float fix = 0.0f;
  const float cs = a.scale * kLog2e;
  const int p0 = t0 + off, p1 = min(t0 + 128, live) + off;
  int lo = a.left < 0 ? 0 : max(0, p0 - a.left);
  int hi = t0 >= live ? lo : a.right < 0 ? end : min(end, p1 + a.right);
  const int pw0 = tw + off, pw1 = min(tw + 32, live) + off, p = pw0 + c;
  const int wlo = a.left < 0 ? 0 : max(0, pw0 - a.left);
  const int whi = tw >= live ? wlo : a.right < 0 ? end : min(end, pw1 + a.right);

  Stage<BF, D, BK, 4> sk, sv;
  sk.init(a.k.t, a.d, w, lane);
  sv.init(a.v.t, a.d, w, lane);
  const E* kb = row_of<E>(a.k, b, hk, 0);
  const E* vb = row_of<E>(a.v, b, hk, 0);
  // first: only sum P (do v^T - D) of every query, which is what sum do o still lacks
  auto step = [&](auto first, int j0, const E* lk, const E* lv, E* nk, E* nv) __attribute__((always_inline)) {
    staged();
    if (j0 + BK < hi) {
      sk.load(nk, kb + (j0 + BK) * a.k.t, end - j0 - BK, w);
      sv.load(nv, vb + (j0 + BK) * a.v.t, end - j0 - BK, w);
    }
    if (j0 + BK <= wlo || j0 >= whi) return;
    f32x16 s[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      s[n] = zero16();
#pragma unroll
      for (int x = 0; x < KS; ++x) s[n] = O::mm(s[n], A::rows(lk, 32 * n + c, x, h), q[x]);
    }
    if (j0 + BK > end || (a.left >= 0 && j0 < pw1 - 1 - a.left) ||
        (a.right >= 0 && j0 + BK - 1 > pw0 + a.right)) {
      const int k0 = a.left < 0 ? 0 : p - a.left;
      const int k1 = a.right < 0 ? end : min(end, p + a.right + 1);
      cut_rows(s, k0 - j0, k1 - j0, h);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      f32x16 v = none;
      X fr[KS];
#pragma unroll
      for (int x = 0; x < KS; ++x) fr[x] = A::rows(lv, 32 * n + c, x, h);
      sched_fence();
#pragma unroll
      for (int x = 0; x < KS; ++x) v = O::mm(v, fr[x], g[x]);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], cs, ex)) * v[i];
      if constexpr (first) {
#pragma unroll
        for (int i = 0; i < 16; ++i) fix += s[n][i];
        continue;
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const X f = O::of(s[n], x);
#pragma unroll
        for (int m = 0; m < NM; ++m)
          o[m] = O::mm(o[m], A::rows_t(lk, 32 * n + 16 * x, m, h, c), f);
      }
    }
  };
  auto pass = [&](auto first) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) none[i] = -dot;
    if (lo < hi) {
      sk.load(lk0, kb + lo * a.k.t, end - lo, w);
      sv.load(lv0, vb + lo * a.v.t, end - lo, w);
    }
    for (int j0 = lo; j0 < hi; j0 += 2 * BK) {
      step(first, j0, lk0, lv0, lk1, lv1);
      if (j0 + BK < hi) step(first, j0 + BK, lk1, lv1, lk0, lv0);
    }
  };
  // sum do o from a bf16 out has the rounding of both, which weighs as much as that of dS
  // where a query sees few keys (two keys: dq and dk off by 2.3 times what their own
  // rounding leaves, 22: 1.5; without it 1.4).  A pass ahead makes it exact where it is
  // short (8 x 16 x 4096 x 64, windows of 32: backward 470 us and 450 without, of 128 440
  // and 440).  Each stretch takes the whole range, so that they agree on D.
  if (BF && hi - lo <= 192) {
    pass(std::true_type{});
    dot += both_sum(fix);
    __syncthreads();
  }
  if (a.d_lse && ex != kNegInf) dot -= a.d_lse[at];
  if (t < a.T && h == 0 && split == 0) {
    a.ex[at] = ex;
    a.delta[at] = -dot;
  }
  if (a.nsplit > 1) stretch_of(lo, hi, BK, split, a.nsplit);
  pass(std::false_type{});
  if (t >= a.T) return;
  if (ex == kNegInf) {            // (zero also where zeros have met an infinity)
#pragma unroll
    for (int m = 0; m < NM; ++m) o[m] = zero16();
  }
  if (a.nsplit > 1) {
    float* row = a.part + ((long)split * a.B * a.H * a.T + at) * a.d;
#pragma unroll
    for (int m = 0; m < NM; ++m) st_part(row, o[m], m, h, a.d);
    return;
  }
  E* drow = row_of_w<E>(a.dq, b, hq, t);
#pragma unroll
  for (int m = 0; m < NM; ++m) st_tile<BF>(drow, o[m], a.scale, m, h, a.d);
}

template <bool BF, int D, int BQ>
__global__ void __launch_bounds__(256, BF && D <= 64 ? 2 : 1) attn_dkv_kernel(AttnArgs a) {
  using O = MOp<BF>;
  using E = typename O::E;
  using X = typename O::X;
  using A = ATile<BF, D>;
  constexpr int NT = BQ / 32, KS = D / 16, NM = D / 32;
  __shared__ __align__(16) E lq0[BQ * D], lq1[BQ * D], lg0[BQ * D], lg1[BQ * D];
  __shared__ __align__(16) float lx0[2][64], lx1[2][64];   // exponents and -D of the queries
  const int lane = threadIdx.x & 63, w = wave_id(), h = lane >> 5, c = lane & 31;
  const Place wk = place_of(a.work, blockIdx.x);
  const int b = wk.b, hk = wk.hk, rep = a.rep, split = wk.split, u = b * a.HK + hk;
  const int off = a.S - a.T, live = live_of(a, b), end = live + off;
  const int j0 = wk.tile * 128, jw = j0 + 32 * w, j = jw + c;

  X k[KS], v[KS];
  const E* krow = j < end ? row_of<E>(a.k, b, hk, j) : nullptr;
  const E* vrow = j < end ? row_of<E>(a.v, b, hk, j) : nullptr;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    k[s] = row_frag<BF>(krow, 16 * s + 8 * h, a.d);
    v[s] = row_frag<BF>(vrow, 16 * s + 8 * h, a.d);
  }
  f32x16 dk[NM], dv[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) {
    dk[m] = zero16();
    dv[m] = zero16();
  }
  const float cs = a.scale * kLog2e;
  // queries that see a key of the workgroup, of this wave, of this lane: p >= j - right,
  // p <= j + left
  const int j1 = min(j0 + 128, end), jw1 = min(jw + 32, end);
  const int lo = a.right < 0 ? 0 : max(0, j0 - a.right - off);
  const int hi = j0 >= end ? lo : a.left < 0 ? live : min(live, j1 + a.left - off);
  const int wlo = a.right < 0 ? 0 : max(0, jw - a.right - off);
  const int whi = jw >= end ? wlo : a.left < 0 ? live : min(live, jw1 + a.left - off);
  const int q0 = a.right < 0 ? 0 : j - a.right - off;
  const int q1 = j >= end ? 0 : a.left < 0 ? live : min(live, j + a.left - off + 1);

  Stage<BF, D, BQ, 4> sq, sg;
  sq.init(a.q.t, a.d, w, lane);
  sg.init(a.d_out.t, a.d, w, lane);
  const int per = hi > lo ? (hi - lo + BQ - 1) / BQ : 0;
  auto fetch = [&](int r, int t, E* nq, E* ng, float (*nx)[64]) __attribute__((always_inline)) {
    const int hq = hk * rep + r;
    sq.load(nq, row_of<E>(a.q, b, hq, t), live - t, w);
    sg.load(ng, row_of<E>(a.d_out, b, hq, t), live - t, w);
    // (queries behind the live ones: q, do and D are zero, and so is what they add)
    const long at = ((long)b * a.H + hq) * a.T + t;
    if (w < 2) stage64(nx[w], (w ? a.delta : a.ex) + at, min(live - t, BQ), lane);
  };
  // the stretch of (head, tile of queries) that this workgroup takes
  const long n0 = (long)per * rep * split / a.nsplit_kv, n1 = (long)per * rep * (split + 1) / a.nsplit_kv;
  int r = per ? (int)(n0 / per) : 0, t0 = per ? lo + (int)(n0 % per) * BQ : lo;
  long left = n1 - n0;
  if (left > 0) fetch(r, t0, lq0, lg0, lx0);
  auto step = [&](const E* lq, const E* lg, const float (*lx)[64], E* nq, E* ng,
                  float (*nx)[64]) __attribute__((always_inline)) {
    staged();
    const int tt = t0;
    t0 += BQ;
    if (t0 >= hi) {
      t0 = lo;
      ++r;
    }
    if (--left > 0) fetch(r, t0, nq, ng, nx);
    if (tt + BQ <= wlo || tt >= whi) return;
    f32x16 s[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      s[n] = zero16();
      X fr[KS];
#pragma unroll
      for (int y = 0; y < KS; ++y) fr[y] = A::rows(lq, 32 * n + c, y, h);
      sched_fence();
#pragma unroll
      for (int y = 0; y < KS; ++y) s[n] = O::mm(s[n], fr[y], k[y]);
    }
    if (jw + 32 > end || (a.right >= 0 && tt + off < jw + 31 - a.right) ||
        (a.left >= 0 && tt + BQ - 1 + off > jw + a.left))
      cut_rows(s, q0 - tt, q1 - tt, h);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      f32x16 x;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const f32x4 d4 = *reinterpret_cast<const f32x4*>(&lx[1][32 * n + 8 * i4 + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * i4 + i] = d4[i];
      }
      X fr[KS];
#pragma unroll
      for (int y = 0; y < KS; ++y) fr[y] = A::rows(lg, 32 * n + c, y, h);
      sched_fence();
#pragma unroll
      for (int y = 0; y < KS; ++y) x = O::mm(x, fr[y], v[y]);
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const f32x4 e4 = *reinterpret_cast<const f32x4*>(&lx[0][32 * n + 8 * i4 + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int y = 4 * i4 + i;
          s[n][y] = __builtin_amdgcn_exp2f(fmaf(s[n][y], cs, e4[i]));
          x[y] *= s[n][y];
        }
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const X pf = O::of(s[n], y), df = O::of(x, y);
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          dv[m] = O::mm(dv[m], A::rows_t(lg, 32 * n + 16 * y, m, h, c), pf);
          dk[m] = O::mm(dk[m], A::rows_t(lq, 32 * n + 16 * y, m, h, c), df);
        }
      }
    }
  };
  while (left > 0) {
    step(lq0, lg0, lx0, lq1, lg1, lx1);
    if (left > 0) step(lq1, lg1, lx1, lq0, lg0, lx0);
  }
  if (j >= a.S) return;
  if (j >= end) {
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      dk[m] = zero16();
      dv[m] = zero16();
    }
  }
  if (a.nsplit_kv > 1) {
    const long rows = (long)a.B * a.HK * a.S, row = split * rows + (long)u * a.S + j;
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      st_part(a.part + row * a.d, dk[m], m, h, a.d);
      st_part(a.part + (a.nsplit_kv * rows + row) * a.d, dv[m], m, h, a.d);
    }
    return;
  }
  E* dkr = row_of_w<E>(a.dk, b, hk, j);
  E* dvr = row_of_w<E>(a.dv, b, hk, j);
#pragma unroll
  for (int m = 0; m < NM; ++m) {
    st_tile<BF>(dkr, dk[m], a.scale, m, h, a.d);
    st_tile<BF>(dvr, dv[m], 1.0f, m, h, a.d);
  }
}

// The stretches of a row [B][H][T] joined: a thread per four channels.
template <bool BF>
__global__ void __launch_bounds__(256) attn_sum_kernel(View out, const float* part, int n, int B, int H,
                                                       int T, int d, float scale) {
  const int nq = d / 4;
  const long id = (long)blockIdx.x * 256 + threadIdx.x, rows = (long)B * H * T;
  if (id >= rows * nq) return;
  const long row = id / nq;
  const int ch = (int)(id % nq) * 4, t = (int)(row % T), u = (int)(row / T);
  f32x4 x = zero4();
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const f32x4 o = *reinterpret_cast<const f32x4*>(part + (s * rows + row) * d + ch);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += o[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] *= scale;
  IoT<BF>::st4(row_of_w<typename MOp<BF>::E>(out, u / H, u % H, t) + ch, x);
}
template <bool BF>
void join(const View& out, const float* part, int n, int B, int H, int T, int d, float scale, hipStream_t s) {
  hipLaunchKernelGGL((attn_sum_kernel<BF>), dim3((unsigned)(((long)B * H * T * (d / 4) + 255) / 256)),
                     dim3(256), 0, s, out, part, n, B, H, T, d, scale);
}

template <bool BF, int D>
hipError_t go(AttnArgs a, hipStream_t s) {
  constexpr int BK = attn_tile_bwd(D);
  const int nq = (a.T + 127) / 128, nk = (a.S + 127) / 128;
  const bool uneven = (a.left < 0) != (a.right < 0);
  a.work = work_of(a.B, a.HK, a.rep, nq, a.nsplit, uneven ? 64 : 0, uneven && (BF || D <= 32));
  hipLaunchKernelGGL((attn_dq_kernel<BF, D, BK>), dim3((unsigned)((long)a.B * a.H * nq * a.nsplit)),
                     dim3(256), 0, s, a, nq);
  if (a.nsplit > 1) join<BF>(a.dq, a.part, a.nsplit, a.B, a.H, a.T, a.d, a.scale, s);
  a.work = work_of(a.B, a.HK, 1, nk, a.nsplit_kv, uneven ? BF && D <= 64 ? 64 : 32 : 0, false);
  hipLaunchKernelGGL((attn_dkv_kernel<BF, D, BK>),
                     dim3((unsigned)((long)a.B * a.HK * nk * a.nsplit_kv)), dim3(256), 0, s, a);
  if (a.nsplit_kv > 1) {
    const long all = (long)a.nsplit_kv * a.B * a.HK * a.S * a.d;
    join<BF>(a.dk, a.part, a.nsplit_kv, a.B, a.HK, a.S, a.d, a.scale, s);
    join<BF>(a.dv, a.part + all, a.nsplit_kv, a.B, a.HK, a.S, a.d, 1.0f, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_backward(const AttnArgs& a, bool bf, hipStream_t s) {
  if (bf) return a.d <= 32 ? go<true, 32>(a, s) : a.d <= 64 ? go<true, 64>(a, s) : go<true, 128>(a, s);
  return a.d <= 32 ? go<false, 32>(a, s) : a.d <= 64 ? go<false, 64>(a, s) : go<false, 128>(a, s);
}

}  // namespace e2ttt
