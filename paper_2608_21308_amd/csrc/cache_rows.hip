// Rows of keys and values into the 4-bit cache and back.  A thread takes eight
// channels of the four tokens whose positions lie in one aligned group of four (a
// word of V's codes); four neighbouring threads make a block of 32 channels, whose
// largest magnitude they find by DPP.
#include "cache_common.h"

namespace e2ttt {
namespace {

// Thread -> (sequence, key head, group of four tokens, block, eighth of 32 channels).
struct Deal {
  Div blocks, groups, heads;
  unsigned n;                         // sequences x key heads x groups
  bool tokens_first;
};
struct Where {
  int b, hk, grp, blk, g;
};
__device__ __forceinline__ bool where_of(const Deal& d, Where& o) {
  const unsigned id = blockIdx.x * 256u + threadIdx.x, x = id >> 2, y = d.blocks.of(x);
  o.g = id & 3;
  o.blk = x - y * d.blocks.d;
  if (y >= d.n) return false;
  if (d.tokens_first) {               // neighbouring rows of a head
    const unsigned z = d.groups.of(y), b = d.heads.of(z);
    o.grp = y - z * d.groups.d;
    o.hk = z - b * d.heads.d;
    o.b = b;
  } else {                            // neighbouring heads of a token
    const unsigned z = d.heads.of(y), b = d.groups.of(z);
    o.hk = y - z * d.heads.d;
    o.grp = z - b * d.groups.d;
    o.b = b;
  }
  return true;
}

__device__ __forceinline__ unsigned quad_max(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
}

template <bool BF>
__device__ __forceinline__ void ld8(float (&x)[8], const typename DOp<BF>::E* p) {
  if constexpr (BF) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  } else {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p), w = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = v[i];
      x[4 + i] = w[i];
    }
  }
}
template <bool BF>
__device__ __forceinline__ void st8(typename DOp<BF>::E* p, const float (&x)[8]) {
  if constexpr (BF) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
    st_stream(reinterpret_cast<bf16x8*>(p), v);
  } else {
    st_stream(reinterpret_cast<f32x4*>(p), f32x4{x[0], x[1], x[2], x[3]});
    st_stream(reinterpret_cast<f32x4*>(p + 4), f32x4{x[4], x[5], x[6], x[7]});
  }
}

// Eight elements of a block as codes (channel order from the low end), and the
// block's scale byte: with m the largest magnitude, the least e with m <= 7 2^e.
__device__ __forceinline__ unsigned encode(const float (&x)[8], unsigned& exp) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  m = quad_max(m);
  // (the significand of 7 is 1.75: above it the exponent takes one more)
  exp = m >= 0x7f800000u ? (unsigned)kNanExp
                         : (unsigned)max((int)((m + 0x1fffffu) >> 23) - 2, kMinExp);
  const float s = __uint_as_float(exp == kNanExp ? 0x3f800000u : exp << 23);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
}

template <bool BF>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheArgs a, Deal deal) {
  using E = typename DOp<BF>::E;
  Where o;
  if (!where_of(deal, o)) return;      // (whole quads leave together)
  const int nb = a.d / 32;
  const Held h = held_of(a, o.b);
  const long p0 = ((h.start >> 2) + o.grp) * 4;
  if (p0 + 4 <= 0 || p0 + 4 <= h.first || p0 >= h.end) return;
  unsigned char* page = p0 >= 0 ? page_at(a, o.b, o.hk, (int)(p0 / kPage % a.P)) : nullptr;
  if (!page) return;
  const int j0 = (int)(p0 % kPage), ta = j0 >> 4, tg = (j0 >> 2) & 3;
  const int ch = 32 * o.blk + 8 * o.g;
  unsigned kc[4], vc[4], ke[4], ve[4];
  bool on[4], all = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long p = p0 + i;
    on[i] = p >= h.start && p >= h.first && p < h.end;
    all = all && on[i];
    float x[8] = {}, y[8] = {};
    if (on[i]) {
      const int t = (int)(p - h.start);
      ld8<BF>(x, row_of<E>(a.x, o.b, o.hk, t) + ch);
      ld8<BF>(y, row_of<E>(a.y, o.b, o.hk, t) + ch);
    }
    kc[i] = encode(x, ke[i]);
    vc[i] = encode(y, ve[i]);
  }
  unsigned char* kp = page + j0 * 16 * nb + o.g * 4 * nb + o.blk * 4;
  unsigned char* ks = page + 32 * a.d + o.blk * 64 + 16 * tg + ta;
  unsigned char* vp = page + 34 * a.d + (o.blk * 16 + 4 * o.g) * 64 + tg * 16 + ta * 4;
  unsigned char* vs = page + 66 * a.d + o.blk * 64 + tg * 16 + ta * 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (on[i]) {
      *reinterpret_cast<unsigned*>(kp + i * 16 * nb) = kc[i];
      if (o.g == i) ks[4 * i] = (unsigned char)ke[i];
    }
  if (all) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {        // byte j of every token's code, tokens in order
      const unsigned lo = __builtin_amdgcn_perm(vc[1], vc[0], 0x0c0c0400u + 0x0101u * j);
      const unsigned hi = __builtin_amdgcn_perm(vc[3], vc[2], 0x0c0c0400u + 0x0101u * j);
      *reinterpret_cast<unsigned*>(vp + 64 * j) = lo | hi << 16;
    }
    if (o.g == 0)
      *reinterpret_cast<unsigned*>(vs) = ve[0] | ve[1] << 8 | ve[2] << 16 | ve[3] << 24;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (on[i]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) vp[64 * j + i] = (unsigned char)(vc[i] >> (8 * j));
        if (o.g == 0) vs[i] = (unsigned char)ve[i];
      }
  }
}

__device__ __forceinline__ void decode(float (&x)[8], unsigned c, float s) {
  typedef __attribute__((ext_vector_type(2))) float f2;
  const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0);
  const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
  const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2);
  const f2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  x[4] = d[0]; x[5] = d[1]; x[6] = e[0]; x[7] = e[1];
}

template <bool BF>
__global__ void __launch_bounds__(256) cache_read_kernel(CacheArgs a, Deal deal) {
  using E = typename DOp<BF>::E;
  Where o;
  if (!where_of(deal, o)) return;
  const int nb = a.d / 32;
  const Held h = held_of(a, o.b);
  const long p0 = ((h.start >> 2) + o.grp) * 4;
  const unsigned char* page = p0 >= 0 && p0 + 4 > h.first && p0 < h.end
                                  ? page_at(a, o.b, o.hk, (int)(p0 / kPage % a.P)) : nullptr;
  const int j0 = (int)((p0 >= 0 ? p0 : 0) % kPage), ta = j0 >> 4, tg = (j0 >> 2) & 3;
  const int ch = 32 * o.blk + 8 * o.g;
  unsigned kc[4] = {}, vw[4] = {}, ke[4] = {}, ve = 0;
  if (page) {
    const unsigned char* vp = page + 34 * a.d + (o.blk * 16 + 4 * o.g) * 64 + tg * 16 + ta * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kc[i] = *reinterpret_cast<const unsigned*>(page + (j0 + i) * 16 * nb + o.g * 4 * nb + o.blk * 4);
      ke[i] = page[32 * a.d + o.blk * 64 + 16 * tg + 4 * i + ta];
      vw[i] = *reinterpret_cast<const unsigned*>(vp + 64 * i);
    }
    ve = *reinterpret_cast<const unsigned*>(page + 66 * a.d + o.blk * 64 + tg * 16 + ta * 4);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long p = p0 + i;
    if (p < h.start || p >= h.start + a.T) continue;
    float x[8] = {}, y[8] = {};
    if (page && p >= h.first && p < h.end) {
      unsigned c = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c |= (vw[j] >> (8 * i) & 255u) << (8 * j);
      decode(x, kc[i], scale_of<0>(ke[i]));
      decode(y, c, scale_of<0>(ve >> (8 * i)));
    }
    const int t = (int)(p - h.start);
    st8<BF>(row_of_w<E>(a.x, o.b, o.hk, t) + ch, x);
    st8<BF>(row_of_w<E>(a.y, o.b, o.hk, t) + ch, y);
  }
}

Deal deal_of(const CacheArgs& a) {
  const int groups = (a.T + 2) / 4 + 1;
  return Deal{div_by(a.d / 32), div_by(groups), div_by(a.HK), (unsigned)((long)a.B * a.HK * groups),
              a.x.t < a.x.h};
}
dim3 grid_of(const CacheArgs& a, const Deal& d) {
  return dim3((unsigned)(((long)d.n * (a.d / 8) + 255) / 256));
}

}  // namespace

hipError_t launch_cache_write(const CacheArgs& a, bool bf, hipStream_t s) {
  const Deal d = deal_of(a);
  if (bf) hipLaunchKernelGGL(cache_write_kernel<true>, grid_of(a, d), dim3(256), 0, s, a, d);
  else hipLaunchKernelGGL(cache_write_kernel<false>, grid_of(a, d), dim3(256), 0, s, a, d);
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheArgs& a, bool bf, hipStream_t s) {
  const Deal d = deal_of(a);
  if (bf) hipLaunchKernelGGL(cache_read_kernel<true>, grid_of(a, d), dim3(256), 0, s, a, d);
  else hipLaunchKernelGGL(cache_read_kernel<false>, grid_of(a, d), dim3(256), 0, s, a, d);
  return hipGetLastError();
}

}  // namespace e2ttt
