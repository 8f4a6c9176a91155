// Attention of a few arriving tokens over the 4-bit cache:
//   s_j = scale q . k_j,  o = sum_j softmax_j(s) v_j  over p - left <= j <= p.
// The queries of a key head (its G query heads times T tokens) are the columns of 16
// x 16 x 32 products, so that a page is decoded once for up to 16 of them; a wave takes
// whole pages, with the running maximum and sum per column in its lanes:
//   S^T = K Q^T,  P^T = 2^(c (S^T - m)),  O^T += V^T P^T,  c = scale log2 e.
// Codes become bf16 without loss (two to an instruction, scale included).  Queries and
// probabilities enter as bf16 terms: queries exactly (one term of bf16, three of
// fp32), P as NP terms, so that out is an fp32 result rounded once.
// Bound by HBM: 17/16 d bytes a token and key head, read once.  Where sequences and
// heads are few, the pages are dealt to several workgroups and their parts joined by
// a second kernel.
#include <math.h>

#include "cache_common.h"

namespace e2ttt {
namespace {

constexpr float kLog2e = 1.44269504088896f;
constexpr int kWaves = 4;

// What one wave's lane takes of a page.
template <int NB>
struct Raw {
  unsigned k[4][NB];      // row tile a: codes of token 16 a + r, blocks in order
  unsigned ks[NB];
  u32x4 v[NB], vs[NB];
  bool on;
};
template <int NB>
__device__ __forceinline__ void fetch(Raw<NB>& x, const unsigned char* page, int g, int r) {
  x.on = page != nullptr;
  if (!page) return;
  constexpr int D = 32 * NB;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const unsigned char* p = page + (16 * a + r) * 16 * NB + g * 4 * NB;
    if constexpr (NB == 4) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) x.k[a][i] = w[i];
    } else if constexpr (NB == 2) {
      const uint2 w = *reinterpret_cast<const uint2*>(p);
      x.k[a][0] = w.x;
      x.k[a][1] = w.y;
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) x.k[a][i] = *reinterpret_cast<const unsigned*>(p + 4 * i);
    }
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    x.ks[i] = *reinterpret_cast<const unsigned*>(page + 32 * D + i * 64 + r * 4);
    x.v[i] = *reinterpret_cast<const u32x4*>(page + 34 * D + (i * 16 + r) * 64 + g * 16);
    x.vs[i] = *reinterpret_cast<const u32x4*>(page + 66 * D + i * 64 + g * 16);
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

// Partial results of a stretch: per sequence, key head and tile of 16 columns, [16]
// maxima (of the scores), [16] sums, then [d][16] outputs.
__host__ __device__ inline long part_floats(int d) { return 32 + 16L * d; }

template <bool BF, int NB>
__global__ void __launch_bounds__(64 * kWaves, 2) cache_attend_kernel(CacheArgs a, int ntile) {
  using E = typename DOp<BF>::E;
  constexpr int NQ = BF ? 1 : 3, NP = BF ? 2 : 3, D = 32 * NB;
  __shared__ __align__(16) float lo_[kWaves][D * 16];
  __shared__ float lm[kWaves][16], ll[kWaves][16];
  const int lane = threadIdx.x & 63, w = wave_id(), g = lane >> 4, r = lane & 15;
  const int split = (int)(blockIdx.x % a.nsplit);
  const long u = blockIdx.x / a.nsplit;
  const int tile = (int)(u % ntile);
  const int hk = (int)(u / ntile % a.HK), b = (int)(u / ntile / a.HK);
  const int rep = a.H / a.HK, col = 16 * tile + r;
  const int qt = col / rep, hq = hk * rep + col % rep;      // token, head of the lane's column
  const Held h = held_of(a, b);
  const int live = (int)(h.end - h.start);
  const bool on = qt < live && h.start + qt >= 0;

  bf16x8 q[NB][NQ];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if constexpr (BF) {
      q[i][0] = bf16x8{};
      if (on) q[i][0] = *reinterpret_cast<const bf16x8*>(row_of<E>(a.q, b, hq, qt) + 32 * i + 8 * g);
    } else {
      f32x4 x = zero4(), y = zero4();
      if (on) {
        const E* p = row_of<E>(a.q, b, hq, qt) + 32 * i + 8 * g;
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
  const long pg0 = any0 / kPage, np = any1 > any0 ? (any1 + kPage - 1) / kPage - pg0 : 0;
  const long s0 = pg0 + np * split / a.nsplit, s1 = pg0 + np * (split + 1) / a.nsplit;

  f32x4 o[NB][2];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i][0] = o[i][1] = zero4();
  float top = -INFINITY, sum = 0.0f;
  const float cs = a.scale * kLog2e;

  Raw<NB> cur, next;
  long pg = s0 + w;
  next.on = false;
  if (pg < s1) fetch<NB>(next, page_of(a, b, hk, pg), g, r);
  for (; pg < s1; pg += kWaves) {
    cur = next;
    if (pg + kWaves < s1) fetch<NB>(next, page_of(a, b, hk, pg + kWaves), g, r);
    if (!cur.on) continue;
    f32x4 s[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      s[x] = zero4();
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const bf16x8 k = eight_of(cur.k[x][i], pow_of(cur.ks[i] >> (8 * x) & 255u));
#pragma unroll
        for (int n = NQ - 1; n >= 0; --n) s[x] = mm(s[x], k, q[i][n]);
      }
    }
    const long j0 = pg * kPage;
    const bool cut = j0 < any0 || j0 + kPage > h.start + 1 || (a.left >= 0 && j0 < h.end - 1 - a.left);
    if (cut) {
      const int k0 = (int)max(see0 - j0, -1L), k1 = (int)min(see1 - j0, 64L);
      const int n0 = (int)max(any0 - j0, -1L), n1 = (int)min(any1 - j0, 64L);
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = 16 * x + 4 * g + i;
          if (j < k0 || j >= k1) s[x][i] = -INFINITY;
          if (j < n0 || j >= n1) {      // (rows that hold nothing: finite values for zeros to meet)
#pragma unroll
            for (int m = 0; m < NB; ++m) cur.vs[m][x] &= ~(255u << (8 * i));
          }
        }
    }
    float most = s[0][0];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, s[x][i]);
    most = fmaxf(top, groups_max(most));
    const float ref = most == -INFINITY ? 0.0f : most;
    const float shrink = __builtin_amdgcn_exp2f((top - ref) * cs);
    top = most;
    sum *= shrink;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        o[i][0][y] *= shrink;
        o[i][1][y] *= shrink;
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
          const unsigned t0 = pair_of<0>(c, pow_of(sc & 255u)), t1 = pair_of<1>(c, pow_of(sc >> 8 & 255u));
          const unsigned t2 = pair_of<2>(c, pow_of(sc >> 16 & 255u)), t3 = pair_of<3>(c, pow_of(sc >> 24));
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
  }

  if (!on) {                  // (a column of no live query has gone along with the others)
    top = -INFINITY;
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i][0] = o[i][1] = zero4();
  }
  // the waves' parts together: lane (g, r) has channels 32 i + 8 g + 2 y + n of column r
  sum = groups_sum(sum);
  if (g == 0) {
    lm[w][r] = top;
    ll[w][r] = sum;
  }
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int y = 0; y < 4; ++y) lo_[w][(32 * i + 8 * g + 2 * y + n) * 16 + r] = o[i][n][y];
  __syncthreads();
  float f[kWaves], all = -INFINITY, total = 0.0f;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) all = fmaxf(all, lm[x][r]);
  const float ref = all == -INFINITY ? 0.0f : all;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    f[x] = __builtin_amdgcn_exp2f((lm[x][r] - ref) * cs);
    total += ll[x][r] * f[x];
  }
  if (a.nsplit > 1) {
    float* part = a.part + (long)blockIdx.x * part_floats(D);
    if (threadIdx.x < 16) {
      part[r] = all;
      part[16 + r] = total;
    }
    for (int y = threadIdx.x; y < D * 16; y += 64 * kWaves) {     // (column y % 16 = r)
      float x = 0.0f;
#pragma unroll
      for (int n = 0; n < kWaves; ++n) x += lo_[n][y] * f[n];
      part[32 + y] = x;
    }
    return;
  }
  if (qt >= a.T) return;
  const float inv = total > 0.0f ? 1.0f / total : 0.0f;
  E* orow = row_of_w<E>(a.out, b, hq, qt);
  for (int ch = 4 * (threadIdx.x >> 4); ch < D; ch += 4 * 4 * kWaves) {
    f32x4 x = zero4();
#pragma unroll
    for (int n = 0; n < kWaves; ++n)
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = fmaf(lo_[n][(ch + y) * 16 + r], f[n] * inv, x[y]);
    IoT<BF>::st4(orow + ch, x);
  }
  if (a.lse && threadIdx.x < 16)
    a.lse[((long)b * a.H + hq) * a.T + qt] = inv > 0.0f ? fmaf(all, a.scale, logf(total)) : -INFINITY;
}

// The stretches' parts joined: a workgroup per sequence, key head and tile of columns.
template <bool BF>
__global__ void __launch_bounds__(256) cache_join_kernel(CacheArgs a, int ntile) {
  using E = typename DOp<BF>::E;
  const long u = blockIdx.x;
  const int tile = (int)(u % ntile), hk = (int)(u / ntile % a.HK), b = (int)(u / ntile / a.HK);
  const int r = threadIdx.x & 15, rep = a.H / a.HK, col = 16 * tile + r;
  const int qt = col / rep, hq = hk * rep + col % rep;
  if (qt >= a.T) return;
  const long each = part_floats(a.d);
  const float* part = a.part + u * a.nsplit * each;
  const float cs = a.scale * kLog2e;
  float all = -INFINITY, total = 0.0f;
  for (int s = 0; s < a.nsplit; ++s) all = fmaxf(all, part[s * each + r]);
  const float ref = all == -INFINITY ? 0.0f : all;
  for (int s = 0; s < a.nsplit; ++s)
    total += part[s * each + 16 + r] * __builtin_amdgcn_exp2f((part[s * each + r] - ref) * cs);
  const float inv = total > 0.0f ? 1.0f / total : 0.0f;
  E* orow = row_of_w<E>(a.out, b, hq, qt);
  for (int ch = 4 * (threadIdx.x >> 4); ch < a.d; ch += 64) {
    f32x4 x = zero4();
    for (int s = 0; s < a.nsplit; ++s) {
      const float f = __builtin_amdgcn_exp2f((part[s * each + r] - ref) * cs) * inv;
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = fmaf(part[s * each + 32 + (ch + y) * 16 + r], f, x[y]);
    }
    IoT<BF>::st4(orow + ch, x);
  }
  if (a.lse && threadIdx.x < 16)
    a.lse[((long)b * a.H + hq) * a.T + qt] = inv > 0.0f ? fmaf(all, a.scale, logf(total)) : -INFINITY;
}

int tiles_of(const CacheArgs& a) { return (int)(((long)a.H / a.HK * a.T + 15) / 16); }

template <bool BF, int NB>
hipError_t go(const CacheArgs& a, hipStream_t s) {
  const int nt = tiles_of(a);
  const long units = (long)a.B * a.HK * nt;
  hipLaunchKernelGGL((cache_attend_kernel<BF, NB>), dim3((unsigned)(units * a.nsplit)),
                     dim3(64 * kWaves), 0, s, a, nt);
  if (a.nsplit > 1)
    hipLaunchKernelGGL((cache_join_kernel<BF>), dim3((unsigned)units), dim3(256), 0, s, a, nt);
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

int cache_splits(const CacheArgs& a) {
  const long units = (long)a.B * a.HK * tiles_of(a);
  long pages = a.P;
  if (a.left >= 0) pages = pages < ((long)a.left + a.T) / kPage + 2 ? pages : ((long)a.left + a.T) / kPage + 2;
  const long want = (768 + units - 1) / units, most = (pages + 7) / 8;
  const long n = want < most ? want : most;
  return n < 1 ? 1 : (int)n;
}
size_t cache_part_floats(const CacheArgs& a) {
  const int n = cache_splits(a);
  return n == 1 ? 0 : (size_t)a.B * a.HK * tiles_of(a) * n * part_floats(a.d);
}

hipError_t launch_cache_attend(const CacheArgs& a, bool bf, hipStream_t s) {
  return bf ? pick<true>(a, s) : pick<false>(a, s);
}

}  // namespace e2ttt
