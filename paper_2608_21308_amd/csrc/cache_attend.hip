// Attention of a few arriving tokens over the 4-bit cache:
//   s_j = scale q . k_j,  o = sum_j softmax_j(s) v_j  over p - left <= j <= p.
// The queries of a key head (its G query heads times T tokens) are the columns of 16
// x 16 x 32 products, so that a page is decoded once for up to 16 of them; a wave takes
// whole pages, with the running maximum and sum per column in its lanes:
//   S^T = K Q^T,  P^T = 2^(c (S^T - m)),  O^T += V^T P^T,  c = scale log2 e.
// Codes become bf16 without loss (two to an instruction, scale included).  Queries and
// probabilities enter as bf16 terms: queries exactly (one term of bf16, three of
// fp32), P as NP: three for fp32 tensors, two for bf16, off by at most 2^-16 of each P
// ahead of the out's rounding of 2^-8.  fp32 queries cost a tenth to a fifth: 64 x 8 key
// heads of 128, 8192 tokens: 118 us and 108, 4 x 4, 64k tokens: 39.1 and 33.3, 8 x 16 of
// 64, 2048 tokens: 12.4 and 11.5.
// Bound by HBM: 17/16 d bytes a token and key head, read once.  Where sequences and
// heads are few, the pages are dealt to several workgroups and their parts joined by
// a second kernel.
#include <math.h>

#include <algorithm>

#include "cache_common.h"

namespace e2ttt {
namespace {

constexpr float kLog2e = 1.44269504088896f;

// What one wave's lane takes of a page.
template <int NB>
struct Raw {
  unsigned k[4][NB];      // row tile a: codes of token 16 a + r, blocks in order
  unsigned ks[NB];
  u32x4 v[NB], vs[NB];
  bool on;
};
// (Without branches, so that the loads of one page are waited for without those of the
// next: of no page the lane asks for nothing.)
template <int NB>
__device__ __forceinline__ void fetch(Raw<NB>& x, const CacheArgs& a, const unsigned char* page,
                                      int g, int r) {
  constexpr int D = 32 * NB;
  x.on = page != nullptr;
  const Buf b = buf_of(x.on ? page : a.cache);
  const unsigned none = x.on ? 0u : kNowhere;
  const unsigned kc = none + r * 16 * NB + g * 4 * NB, ks = none + 32 * D + r * 4;
  const unsigned vc = none + 34 * D + r * 64 + g * 16, vs = none + 66 * D + g * 16;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const unsigned at = kc + 16 * t * 16 * NB;
    if constexpr (NB == 4) {
      const u32x4 w = buf_ld(b, at);
#pragma unroll
      for (int i = 0; i < 4; ++i) x.k[t][i] = w[i];
    } else if constexpr (NB == 2) {
      const auto w = __builtin_amdgcn_raw_buffer_load_b64(b, (int)at, 0, 0);
      x.k[t][0] = w[0];
      x.k[t][1] = w[1];
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) x.k[t][i] = __builtin_amdgcn_raw_buffer_load_b32(b, (int)(at + 4 * i), 0, 0);
    }
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    x.ks[i] = __builtin_amdgcn_raw_buffer_load_b32(b, (int)(ks + i * 64), 0, 0);
    x.v[i] = buf_ld(b, vc + i * 1024);
    x.vs[i] = buf_ld(b, vs + i * 64);
  }
}

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) unsigned u4;
template <int SEL>
__device__ __forceinline__ unsigned pair_of(unsigned w, float s) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL));
}
__device__ __forceinline__ bf16x8 eight_of(unsigned w, float s) {
  return __builtin_bit_cast(bf16x8, u4{pair_of<0>(w, s), pair_of<1>(w, s), pair_of<2>(w, s),
                                       pair_of<3>(w, s)});
}
__device__ __forceinline__ f32x4 mm(const f32x4& c, const bf16x8& a, const bf16x8& b) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Over the four lane groups (lanes r, 16 + r, 32 + r, 48 + r).
__device__ __forceinline__ float groups_max(float x) {
  auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
  u = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(u[0]) + __uint_as_float(u[1]);
  u = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(u[0]) + __uint_as_float(u[1]);
}

// The maximum of a column that sees keys, all of them with scores of -inf (below fp32's
// range): with a sum of zero, and not the -inf of a column that sees none.
constexpr float kNoScore = -3.402823466e38f;
// The sum of a column that sees keys: positive and finite (the largest of its terms is at
// least one) unless a score has left the range of fp32.
__device__ __forceinline__ float sum_of(float x) { return x > 0.0f && x < INFINITY ? x : NAN; }

// Partial results of a stretch, per sequence, key head and tile of 16 columns: [16]
// maxima (of the scores), [16] sums, then the outputs of [16] columns, d each.
__host__ __device__ inline long part_floats(int d) { return 32 + 16L * d; }

template <bool BF, int NB, int NW>
__global__ void __launch_bounds__(64 * NW, 2) cache_attend_kernel(CacheArgs a, int ntile) {
  using E = typename DOp<BF>::E;
  constexpr int NQ = BF ? 1 : 3, NP = BF ? 2 : 3, D = 32 * NB;
  __shared__ __align__(16) float lo_[NW][D * 16];
  __shared__ float lm[NW][16], ll[NW][16];
  const int lane = threadIdx.x & 63, w = wave_id(), g = lane >> 4, r = lane & 15;
  const int u = a.by_split.of(blockIdx.x), split = blockIdx.x - u * a.nsplit;
  const int y = a.by_tile.of(u), tile = u - y * ntile, b = a.by_HK.of(y), hk = y - b * a.HK;
  const int rep = a.by_rep.d, col = 16 * tile + r;
  const int qt = a.by_rep.of(col), hq = hk * rep + col - qt * rep;   // token, head of the lane's column
  const Held h = held_of(a, b);
  const int live = (int)(h.end - h.start);
  const bool on = qt < live && h.start + qt >= 0;

  bf16x8 q[NB][NQ];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if constexpr (BF) {
      q[i][0] = bf16x8{};
      if (on) q[i][0] = *reinterpret_cast<const bf16x8*>(row_of<E>(a.x, b, hq, qt) + 32 * i + 8 * g);
    } else {
      f32x4 x = zero4(), y = zero4();
      if (on) {
        const E* p = row_of<E>(a.x, b, hq, qt) + 32 * i + 8 * g;
        x = *reinterpret_cast<const f32x4*>(p);
        y = *reinterpret_cast<const f32x4*>(p + 4);
      }
      const auto s = DOp<true>::split(x, y);
#pragma unroll
      for (int n = 0; n < NQ; ++n) q[i][n] = s.t[n];
    }
  }
  // what the column sees, and what any of them may (the call's tokens together)
  const long p = h.start + qt;
  const long see0 = on ? max(h.first, a.left < 0 ? 0L : p - a.left) : 0, see1 = on ? p + 1 : 0;
  const long any0 = max(h.first, a.left < 0 ? 0L : max(0L, h.start - a.left));
  const long any1 = live > 0 ? h.end : any0;
  const int pg0 = (int)(any0 / kPage), np = any1 > any0 ? (int)((any1 + kPage - 1) / kPage) - pg0 : 0;
  const int each = a.by_split.of(np + a.nsplit - 1);
  const int s0 = pg0 + min(np, each * split), s1 = pg0 + min(np, each * (split + 1));

  f32x4 o[NB][2];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i][0] = o[i][1] = zero4();
  // (ref stands in for the maximum: it follows once a score passes it by 8 powers of two)
  float top = -INFINITY, ref = 0.0f, sum = 0.0f;
  const float cs = a.scale * kLog2e, slack = 8.0f / cs;

  // the wave's pages w, w + NW, ..: their bytes one turn ahead, their places two
  int entry = s0 + w - (int)a.by_P.of(s0 + w) * a.P;
  auto place = [&](int pg) __attribute__((always_inline)) {
    const unsigned char* x = pg < s1 ? page_at(a, b, hk, entry) : nullptr;
    entry += NW;
    while (entry >= a.P) entry -= a.P;
    return x;
  };
  auto turn = [&](Raw<NB>& cur, int pg) __attribute__((always_inline)) {
    if (!cur.on) return;
    f32x4 s[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      s[x] = zero4();
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const float f = x == 0 ? scale_of<0>(cur.ks[i]) : x == 1 ? scale_of<1>(cur.ks[i]) :
                        x == 2 ? scale_of<2>(cur.ks[i]) : scale_of<3>(cur.ks[i]);
        const bf16x8 k = eight_of(cur.k[x][i], f);
#pragma unroll
        for (int n = NQ - 1; n >= 0; --n) s[x] = mm(s[x], k, q[i][n]);
      }
    }
    const long j0 = (long)pg * kPage;
    const bool cut = j0 < any0 || j0 + kPage > h.start + 1 || (a.left >= 0 && j0 < h.end - 1 - a.left);
    if (cut) {
      // (tokens of the lane counted from 4 g on)
      const int k0 = (int)max(see0 - j0, -1L) - 4 * g, k1 = (int)max(min(see1 - j0, 64L), -1L) - 4 * g;
      const int n0 = (int)max(any0 - j0, -1L) - 4 * g, n1 = (int)min(any1 - j0, 64L) - 4 * g;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        unsigned held = 0;         // (rows that hold nothing: finite values for zeros to meet)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = 16 * x + i;
          s[x][i] = j >= k0 && j < k1 ? s[x][i] : -INFINITY;
          held |= j >= n0 && j < n1 ? 255u << (8 * i) : 0u;
        }
#pragma unroll
        for (int m = 0; m < NB; ++m) cur.vs[m][x] &= held;
        sched_fence();
      }
    }
    float most = s[0][0];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, s[x][i]);
    most = groups_max(most);
    if (__any(most > top + slack)) {
      const float was = top == -INFINITY ? -INFINITY : ref;     // (no key before: nothing to keep)
      top = fmaxf(top, most);
      ref = top == -INFINITY ? 0.0f : top;
      const float shrink = __builtin_amdgcn_exp2f((was - ref) * cs);
      sum *= shrink;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          o[i][0][y] *= shrink;
          o[i][1][y] *= shrink;
        }
    }
    const float off = -ref * cs;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[x][i] = __builtin_amdgcn_exp2f(fmaf(s[x][i], cs, off));
        sum += s[x][i];
      }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const auto pt = DOp<true>::split(s[2 * x], s[2 * x + 1]);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        u4 even, odd;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const unsigned c = cur.v[i][2 * x + y], sc = cur.vs[i][2 * x + y];
          const unsigned t0 = pair_of<0>(c, scale_of<0>(sc)), t1 = pair_of<1>(c, scale_of<1>(sc));
          const unsigned t2 = pair_of<2>(c, scale_of<2>(sc)), t3 = pair_of<3>(c, scale_of<3>(sc));
          even[2 * y] = __builtin_amdgcn_perm(t1, t0, 0x05040100u);
          even[2 * y + 1] = __builtin_amdgcn_perm(t3, t2, 0x05040100u);
          odd[2 * y] = __builtin_amdgcn_perm(t1, t0, 0x07060302u);
          odd[2 * y + 1] = __builtin_amdgcn_perm(t3, t2, 0x07060302u);
        }
#pragma unroll
        for (int n = NP - 1; n >= 0; --n) {
          o[i][0] = mm(o[i][0], __builtin_bit_cast(bf16x8, even), pt.t[n]);
          o[i][1] = mm(o[i][1], __builtin_bit_cast(bf16x8, odd), pt.t[n]);
        }
      }
    }
  };
  Raw<NB> x, z;
  int pg = s0 + w;
  const unsigned char* next = place(pg);
  fetch<NB>(x, a, next, g, r);
  next = place(pg + NW);
  for (; pg < s1; pg += 2 * NW) {
    fetch<NB>(z, a, next, g, r);
    next = place(pg + 2 * NW);
    turn(x, pg);
    fetch<NB>(x, a, next, g, r);
    next = place(pg + 3 * NW);
    turn(z, pg + NW);
  }

  sum = groups_sum(on ? sum : 0.0f);
  if (sum == 0.0f) {          // (a column that sees nothing has gone along with the others)
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i][0] = o[i][1] = zero4();
  }
  // (of the wave's pages a column sees none, or only scores of -inf: its places tell)
  const bool none = on && sum == 0.0f && top == -INFINITY;
  bool seen = false;
  if (__any(none))
    for (int pg = s0 + w; pg < s1; pg += NW) {
      const long j0 = (long)pg * kPage;
      seen = seen || (none && max(see0, j0) < min(see1, j0 + kPage) &&
                      page_at(a, b, hk, pg - (int)a.by_P.of(pg) * a.P));
    }
  // the waves' parts together: lane (g, r) has channels 32 i + 8 g + 2 y + n of column r
  if (g == 0) {
    lm[w][r] = on && (sum != 0.0f || top != -INFINITY) ? ref : seen ? kNoScore : -INFINITY;
    ll[w][r] = sum;
  }
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int y = 0; y < 4; ++y) lo_[w][(32 * i + 8 * g + 2 * y + n) * 16 + r] = o[i][n][y];
  __syncthreads();
  float f[NW], all = -INFINITY, total = 0.0f;
#pragma unroll
  for (int x = 0; x < NW; ++x) all = fmaxf(all, lm[x][r]);
  const float base = all == -INFINITY ? 0.0f : all;
#pragma unroll
  for (int x = 0; x < NW; ++x) {
    f[x] = __builtin_amdgcn_exp2f((lm[x][r] - base) * cs);
    total += ll[x][r] * f[x];
  }
  if (a.nsplit > 1) {
    float* part = a.part + (long)blockIdx.x * part_floats(D);
    if (threadIdx.x < 16) {
      part[r] = all;
      part[16 + r] = total;
    }
    for (int ch = 4 * (threadIdx.x >> 4); ch < D; ch += 16 * NW) {
      f32x4 x = zero4();
#pragma unroll
      for (int n = 0; n < NW; ++n)
#pragma unroll
        for (int y = 0; y < 4; ++y) x[y] = fmaf(lo_[n][(ch + y) * 16 + r], f[n], x[y]);
      *reinterpret_cast<f32x4*>(part + 32 + r * D + ch) = x;
    }
    return;
  }
  if (qt >= a.T) return;
  const bool some = all != -INFINITY;
  total = sum_of(total);
  const float inv = some ? 1.0f / total : 0.0f;
  E* orow = row_of_w<E>(a.y, b, hq, qt);
  for (int ch = 4 * (threadIdx.x >> 4); ch < D; ch += 16 * NW) {
    f32x4 x = zero4();
#pragma unroll
    for (int n = 0; n < NW; ++n)
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = fmaf(lo_[n][(ch + y) * 16 + r], f[n] * inv, x[y]);
    IoT<BF>::st4(orow + ch, x);
  }
  if (a.lse && threadIdx.x < 16)
    a.lse[((long)b * a.H + hq) * a.T + qt] = some ? fmaf(all, a.scale, logf(total)) : -INFINITY;
}

// The stretches' parts joined: a workgroup per sequence, key head, tile of columns and
// 16 channels (16 columns x 4 quads of channels x 4 shares of the stretches).
constexpr int kMostSplits = 256;
template <bool BF>
__global__ void __launch_bounds__(256) cache_join_kernel(CacheArgs a, int ntile) {
  using E = typename DOp<BF>::E;
  __shared__ float wt[kMostSplits * 16];
  __shared__ float red[16][16];
  __shared__ f32x4 acc[4][64];
  const int nc = a.d / 16, u = blockIdx.x / nc, c0 = (int)(blockIdx.x % nc) * 16;
  const int tile = u % ntile, hk = u / ntile % a.HK, b = u / ntile / a.HK;
  const int r = threadIdx.x & 15, y = threadIdx.x >> 4, rep = a.H / a.HK, col = 16 * tile + r;
  const int qt = col / rep, hq = hk * rep + col % rep;
  const long each = part_floats(a.d);
  const float* part = a.part + (long)u * a.nsplit * each;
  const float cs = a.scale * kLog2e;
  float m = -INFINITY, total = 0.0f;
  for (int s = y; s < a.nsplit; s += 16) m = fmaxf(m, part[s * each + r]);
  red[y][r] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, red[i][r]);
  const float ref = m == -INFINITY ? 0.0f : m;
  __syncthreads();
  for (int s = y; s < a.nsplit; s += 16) {
    const float f = __builtin_amdgcn_exp2f((part[s * each + r] - ref) * cs);
    wt[s * 16 + r] = f;
    total += part[s * each + 16 + r] * f;
  }
  red[y][r] = total;
  __syncthreads();
  total = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) total += red[i][r];
  const bool some = m != -INFINITY;
  total = sum_of(total);
  const float inv = some ? 1.0f / total : 0.0f;
  f32x4 x = zero4();
  const float* from = part + 32 + r * a.d + c0 + 4 * (y & 3);
#pragma unroll 4
  for (int s = y >> 2; s < a.nsplit; s += 4) {
    const f32x4 o = *reinterpret_cast<const f32x4*>(from + s * each);
    const float f = wt[s * 16 + r];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fmaf(o[i], f, x[i]);
  }
  acc[y >> 2][(y & 3) * 16 + r] = x;
  __syncthreads();
  if (threadIdx.x >= 64 || qt >= a.T) return;
  f32x4 o = zero4();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int n = 0; n < 4; ++n) o[n] += acc[i][threadIdx.x][n];
#pragma unroll
  for (int n = 0; n < 4; ++n) o[n] *= inv;
  IoT<BF>::st4(row_of_w<E>(a.y, b, hq, qt) + c0 + 4 * y, o);
  if (a.lse && c0 == 0 && y == 0)
    a.lse[((long)b * a.H + hq) * a.T + qt] = some ? fmaf(m, a.scale, logf(total)) : -INFINITY;
}

int tiles_of(const CacheArgs& a) { return (int)(((long)a.H / a.HK * a.T + 15) / 16); }

template <bool BF, int NB>
hipError_t go(CacheArgs a, hipStream_t s) {
  const int nt = tiles_of(a);
  const long units = (long)a.B * a.HK * nt;
  a.by_split = div_by(a.nsplit);
  a.by_tile = div_by(nt);
  a.by_HK = div_by(a.HK);
  a.by_rep = div_by(a.H / a.HK);
  a.by_P = div_by(a.P);
  hipLaunchKernelGGL((cache_attend_kernel<BF, NB, 8>), dim3((unsigned)(units * a.nsplit)),
                     dim3(512), 0, s, a, nt);
  if (a.nsplit > 1)
    hipLaunchKernelGGL((cache_join_kernel<BF>), dim3((unsigned)(units * (a.d / 16))), dim3(256), 0, s, a, nt);
  return hipGetLastError();
}
template <bool BF>
hipError_t pick(const CacheArgs& a, hipStream_t s) {
  switch (a.d / 32) {
    case 1: return go<BF, 1>(a, s);
    case 2: return go<BF, 2>(a, s);
    case 3: return go<BF, 3>(a, s);
    default: return go<BF, 4>(a, s);
  }
}

}  // namespace

// A workgroup's eight waves take a page each at a time, some 1.2 us; a split adds the
// join, 4 us. (128 units of 64, 34 pages: 12.8 us whole, 15.3 in two, 17.5 in three.)  So
// the pages are split from 64 on, into stretches of 16 at least, while the stretches of
// all units find a CU each (16 units of 128, 1030 pages: 34.6 us in 16, 38.6 in 32, 47.7
// in 8).
int cache_splits(const CacheArgs& a) {
  const long units = (long)a.B * a.HK * tiles_of(a);
  long pages = a.P;
  if (a.left >= 0) pages = std::min(pages, ((long)a.left + a.T) / kPage + 2);
  if (pages < 64) return 1;
  return (int)std::max(1L, std::min({256 / units, (pages + 15) / 16, (long)kMostSplits}));
}
size_t cache_part_floats(const CacheArgs& a) {
  const int n = cache_splits(a);
  return n == 1 ? 0 : (size_t)a.B * a.HK * tiles_of(a) * n * part_floats(a.d);
}

hipError_t launch_cache_attend(const CacheArgs& a, bool bf, hipStream_t s) {
  return bf ? pick<true>(a, s) : pick<false>(a, s);
}

}  // namespace e2ttt
