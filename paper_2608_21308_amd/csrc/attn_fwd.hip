// Attention, forward: a wave holds 32 queries (as columns of the transposed scores)
// and passes once over the keys that they see, with the running maximum m and sum
// l of the softmax per query in a lane:
//   S^T = K Q^T,  P^T = 2^(c (S^T - m)),  O^T <- O^T 2^(c (m_old - m)) + V^T P^T,
// c = scale log2 e.  P is rounded to the io type for the second product (bf16: half
// a step of 2^-8 each, of either sign, averaged over the keys; the sum l is of the
// unrounded ones).
#include <math.h>

#include <algorithm>

#include "attn_common.h"

namespace e2ttt {
namespace {

template <bool BF, int D, int BK>
__global__ void __launch_bounds__(256, BF ? 2 : 1) attn_fwd_kernel(AttnArgs a, int ntile) {
  using O = MOp<BF>;
  using E = typename O::E;
  using X = typename O::X;
  using A = ATile<BF, D>;
  constexpr int NT = BK / 32, KS = D / 16, NM = D / 32;
  // (apart by name: a read of one is then known not to wait for loads into another)
  __shared__ __align__(16) E lk0[BK * D], lk1[BK * D], lv0[BK * D], lv1[BK * D];
  const int lane = threadIdx.x & 63, w = wave_id(), h = lane >> 5, c = lane & 31;
  const Place wk = place_of(a.work, blockIdx.x);
  const int tile = ntile - 1 - wk.tile;               // (long rows of a causal mask first)
  const int b = wk.b, hk = wk.hk, hq = hk * a.rep + wk.head, split = wk.split, u = b * a.H + hq;
  const int off = a.S - a.T, live = live_of(a, b), end = live + off;
  const int t0 = tile * 128, tw = t0 + 32 * w, t = tw + c;

  X q[KS];
  const E* qrow = t < live ? row_of<E>(a.q, b, hq, t) : nullptr;
#pragma unroll
  for (int s = 0; s < KS; ++s) q[s] = row_frag<BF>(qrow, 16 * s + 8 * h, a.d);

  f32x16 o[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) o[m] = zero16();
  // ref stands in for the maximum: it follows once a score passes it by 8 powers of
  // two, so that O is rarely scaled again
  float top = kNegInf, ref = 0.0f, sum = 0.0f;
  const float cs = a.scale * kLog2e, slack = 8.0f / cs;

  // keys that some query of the workgroup, of this wave sees
  const int p0 = t0 + off, p1 = min(t0 + 128, live) + off;
  int lo = a.left < 0 ? 0 : max(0, p0 - a.left);
  int hi = t0 >= live ? lo : a.right < 0 ? end : min(end, p1 + a.right);
  if (a.nsplit > 1) stretch_of(lo, hi, BK, split, a.nsplit);
  const int pw0 = tw + off, pw1 = min(tw + 32, live) + off, p = pw0 + c;
  const int wlo = a.left < 0 ? 0 : max(0, pw0 - a.left);
  const int whi = tw >= live ? wlo : a.right < 0 ? end : min(end, pw1 + a.right);

  Stage<BF, D, BK, 4> sk, sv;
  sk.init(a.k.t, a.d, w, lane);
  sv.init(a.v.t, a.d, w, lane);
  const E* kb = row_of<E>(a.k, b, hk, 0);
  const E* vb = row_of<E>(a.v, b, hk, 0);
  if (lo < hi) {
    sk.load(lk0, kb + lo * a.k.t, end - lo, w);
    sv.load(lv0, vb + lo * a.v.t, end - lo, w);
  }
  auto step = [&](int j0, const E* lk, const E* lv, E* nk, E* nv) __attribute__((always_inline)) {
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
      if constexpr (D > 64) {       // (the loads together: 2 x 8 x 4096 x 128 95 -> 88 us; at 64
        X fr[KS];                   // the registers are those of a SIMD's fourth wave: 173 -> 181)
#pragma unroll
        for (int x = 0; x < KS; ++x) fr[x] = A::rows(lk, 32 * n + c, x, h);
        sched_fence();
#pragma unroll
        for (int x = 0; x < KS; ++x) s[n] = O::mm(s[n], fr[x], q[x]);
      } else {
#pragma unroll
        for (int x = 0; x < KS; ++x) s[n] = O::mm(s[n], A::rows(lk, 32 * n + c, x, h), q[x]);
      }
    }
    if (j0 + BK > end || (a.left >= 0 && j0 < pw1 - 1 - a.left) ||
        (a.right >= 0 && j0 + BK - 1 > pw0 + a.right)) {
      const int k0 = a.left < 0 ? 0 : p - a.left;
      const int k1 = a.right < 0 ? end : min(end, p + a.right + 1);
      cut_rows(s, k0 - j0, k1 - j0, h);
    }
    float most = s[0][0];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, s[n][i]);
    most = both_max(most);
    if (__any(most > top + slack)) {
      const float was = top == kNegInf ? kNegInf : ref;       // (no key before: nothing to keep)
      top = fmaxf(top, most);
      ref = top == kNegInf ? 0.0f : top;
      const float shrink = __builtin_amdgcn_exp2f((was - ref) * cs);
      sum *= shrink;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[m][i] *= shrink;
    }
    const float off2 = -ref * cs;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], cs, off2));
        sum += s[n][i];
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const X pf = O::of(s[n], x);
        if constexpr (D > 64) {
          X fr[NM];
#pragma unroll
          for (int m = 0; m < NM; ++m) fr[m] = A::rows_t(lv, 32 * n + 16 * x, m, h, c);
          sched_fence();
#pragma unroll
          for (int m = 0; m < NM; ++m) o[m] = O::mm(o[m], fr[m], pf);
        } else {
#pragma unroll
          for (int m = 0; m < NM; ++m)
            o[m] = O::mm(o[m], A::rows_t(lv, 32 * n + 16 * x, m, h, c), pf);
        }
      }
    }
  };
  for (int j0 = lo; j0 < hi; j0 += 2 * BK) {
    step(j0, lk0, lv0, lk1, lv1);
    if (j0 + BK < hi) step(j0 + BK, lk1, lv1, lk0, lv0);
  }
  if (t >= a.T) return;
  sum = both_sum(sum);
  const long at = (long)u * a.T + t;
  const bool on = t < live;
  if (!on || sum == 0.0f) {       // (zero also where zeros have met an infinity)
    sum = 0.0f;
#pragma unroll
    for (int m = 0; m < NM; ++m) o[m] = zero16();
  }
  if (a.nsplit > 1) {
    const long row = (long)split * a.B * a.H * a.T + at;
#pragma unroll
    for (int m = 0; m < NM; ++m) st_part(a.part + row * a.d, o[m], m, h, a.d);
    if (h == 0) a.part_ml[row] = make_float2(on && (sum != 0.0f || top != kNegInf) ? ref : kNegInf, sum);
    return;
  }
  const bool some = on && sees_some(a, p, end);
  sum = sum_of(sum);
  const float inv = some ? 1.0f / sum : 0.0f;
  E* orow = row_of_w<E>(a.out, b, hq, t);
#pragma unroll
  for (int m = 0; m < NM; ++m) st_tile<BF>(orow, o[m], inv, m, h, a.d);
  if (a.lse && h == 0)
    a.lse[at] = some ? fmaf(ref, a.scale, logf(sum)) : kNegInf;
}

// The stretches of a query joined: a thread per four channels.
template <bool BF>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs a) {
  using E = typename MOp<BF>::E;
  const int nq = a.d / 4;
  const long id = (long)blockIdx.x * 256 + threadIdx.x, rows = (long)a.B * a.H * a.T;
  if (id >= rows * nq) return;
  const long row = id / nq;
  const int ch = (int)(id % nq) * 4, t = (int)(row % a.T), u = (int)(row / a.T), b = u / a.H;
  const float cs = a.scale * kLog2e;
  float most = kNegInf, sum = 0.0f;
  for (int s = 0; s < a.nsplit; ++s) most = fmaxf(most, a.part_ml[s * rows + row].x);
  const float ref = most == kNegInf ? 0.0f : most;
  f32x4 x = zero4();
#pragma unroll 4
  for (int s = 0; s < a.nsplit; ++s) {
    const float2 ml = a.part_ml[s * rows + row];
    const float f = __builtin_amdgcn_exp2f((ml.x - ref) * cs);
    const f32x4 o = *reinterpret_cast<const f32x4*>(a.part + (s * rows + row) * a.d + ch);
    sum = fmaf(ml.y, f, sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fmaf(o[i], f, x[i]);
  }
  const int live = live_of(a, b), off = a.S - a.T;
  const bool some = t < live && sees_some(a, t + off, live + off);
  sum = sum_of(sum);
  const float inv = some ? 1.0f / sum : 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] *= inv;
  IoT<BF>::st4(row_of_w<E>(a.out, b, u % a.H, t) + ch, x);
  if (a.lse && ch == 0) a.lse[row] = some ? fmaf(ref, a.scale, logf(sum)) : kNegInf;
}

template <bool BF, int D>
hipError_t go(AttnArgs a, hipStream_t s) {
  const int ntile = (a.T + 127) / 128;
  const bool uneven = (a.left < 0) != (a.right < 0);
  a.work = work_of(a.B, a.HK, a.rep, ntile, a.nsplit, uneven ? 64 : 0,
                   uneven && (BF || D <= 32));
  hipLaunchKernelGGL((attn_fwd_kernel<BF, D, attn_tile(BF, D)>),
                     dim3((unsigned)((long)a.B * a.H * ntile * a.nsplit)), dim3(256), 0, s, a, ntile);
  if (a.nsplit > 1)
    hipLaunchKernelGGL((attn_join_kernel<BF>),
                       dim3((unsigned)(((long)a.B * a.H * a.T * (a.d / 4) + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// A workgroup alone on its CU takes a tile of keys in 1 to 2 us, a split costs the
// join, 5 us and more with the head dim.  `places` 512 (two workgroups on a CU) and 256,
// us, forward / backward.  Head dim 64: 64 groups of 128 tiles 32.7 / 79 and 38.1 / 89;
// 16 groups of 140 tiles 30.6 / 64 and 29.4 / 68.  Head dim 128: 64 groups of 32 tiles
// 28.1 / 82 and 22.8 / 63, of 72 tiles 40.1 / 120 and 38.8 / 112, 80 of 32 29.2 / 87 and
// 25.2 / 72, 128 of 32 33.9 / 102 and 30.9 / 89; where 256 leaves a fifth of the CUs
// empty, the forward turns: 96 groups of 64 tiles 39.3 / 124 and 44.9 / 123, 144 of 32
// 35.9 / 111 and 37.9 / 110.  float32, 64 groups of 32 tiles 77 / 242 and 51 / 156.
// Not split: 8 groups of 15 tiles 18.8 (in 3: 14.2), 192 groups of 24 tiles 33 (in 2:
// 37), 16 groups of 9 tiles 15.4 (in 2: 17.6).
// Up to 256 groups have a CU each and the longest row sets the end, `halve`, whole and
// in two: 8 heads of 4096 rows 59.7 / 140 and 45 / 115 (64), 76 / 229 and 63 / 189 (128),
// dk and dv of 32 query and 8 key heads (128) 493 and 403; but 16 of 2048 32.3 / 77 and 31 / 76
// (64), 39 / 124 and 41 / 136 (128).  float32, 64: 8 of 4096 275 / 959 and 169 / 579, 32
// of 1024 74 / 252 and 57 / 220.
// The same for 129 to 160 groups where 256 places give them one stretch each: dk and dv of 128,
// backward of 4 heads of 4608 210 and 167, of 16 query and 4 key heads 697 and 455; float32, 64:
// 4 of 4608 306 / 1062 and 164 / 560, 16 of 1152 82 / 280 and 52 / 162.
int attn_splits(long groups, long tiles, long places, bool halve) {
  const long least = halve && groups > 128 && groups <= 256 ? 2 : 1;
  return (int)(groups > 160 ? least : std::max(least, std::min(places / groups, tiles / 6)));
}

hipError_t launch_attn_forward(const AttnArgs& a, bool bf, hipStream_t s) {
  if (bf) return a.d <= 32 ? go<true, 32>(a, s) : a.d <= 64 ? go<true, 64>(a, s) : go<true, 128>(a, s);
  return a.d <= 32 ? go<false, 32>(a, s) : a.d <= 64 ? go<false, 64>(a, s) : go<false, 128>(a, s);
}

}  // namespace e2ttt
