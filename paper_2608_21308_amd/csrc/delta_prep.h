// Gated delta rule, what a chunk needs that does not depend on the state: the
// decay sums, T = (I + diag(eta) M)^-1 and P = s lower(D o Q K^T) as operand
// fragments (delta_common.h), one workgroup of four waves per chunk of 64
// tokens and unit.
//
// Wave w forms rows lab(w, .) of K K^T and Q K^T by MFMA with operands
// straight from global memory (each chunk's rows are read by one workgroup,
// 16 bytes a lane), transposed, so that the accumulators are already in the
// order of the fragments to be written.  The inverse is taken in fp32 by blocks
// of doubling size, each wave a 16x16 diagonal block and then its share of the
// blocks below, with fp32 MFMA.
//
// Near HBM's rate: 16384 chunks of dk = 64 (16 KB read and 38 KB written each)
// take 187 us, 4.8 TB/s where a large copy reaches 5.2.
#pragma once

#include "delta_common.h"

namespace e2ttt {
namespace {

constexpr int LDT = kDC + 4;   // row of the 64x64 fp32 arrays in LDS

// LDS written and read by the same wave completes in order; this only keeps the
// compiler from exchanging the two.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// C += A[ar.., ak..] B[bk.., bc..], 16x16 blocks of a row-major LDS array;
// contraction index of slot (g, i) is 4 g + i.
__device__ __forceinline__ f32x4 blk_a(const float* m, int r0, int k0, int g, int c) {
  return *reinterpret_cast<const f32x4*>(m + (r0 + c) * LDT + k0 + 4 * g);
}
__device__ __forceinline__ f32x4 blk_b(const float* m, int k0, int c0, int g, int c) {
  f32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = m[(k0 + 4 * g + i) * LDT + c0 + c];
  return x;
}
__device__ __forceinline__ f32x4 mm16(f32x4 acc, f32x4 a, f32x4 b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
  return acc;
}

__device__ __forceinline__ void mm16_2(f32x4& x, f32x4 a, f32x4 b, f32x4& y, f32x4 c, f32x4 d) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], x, 0, 0, 0);
    y = __builtin_amdgcn_mfma_f32_16x16x4f32(c[i], d[i], y, 0, 0, 0);
  }
}
// Whether (r, c) lies in the lower left h x h block of a diagonal 2h x 2h block.
__device__ __forceinline__ bool below(int r, int c, int h) {
  return ((r ^ c) & (15 & ~(h - 1))) == h && (r & h);
}

// Eight values (zeros at kNowhere).
template <bool BF>
__device__ __forceinline__ typename DOp<BF>::X ld_row(Buf p, unsigned at) {
  typename DOp<BF>::X x;
  if constexpr (BF) {
    x.v = __builtin_bit_cast(bf16x8, buf_ld(p, at));
  } else {
    x.a = __builtin_bit_cast(f32x4, buf_ld(p, at));
    x.b = __builtin_bit_cast(f32x4, buf_ld(p, at + 16));
  }
  return x;
}

constexpr int kPrepLds = (kGateFloats + kDC * LDT) * 4;

// Workgroup `blk` of the chunks r0 .. r0 + nr - 1 of every unit, with kPrepLds of LDS.
template <bool BF, int DK>
__device__ __forceinline__ void prep_chunk(const DeltaArgs& a, int r0, int nr, long blk, char* lds) {
  using O = DOp<BF>;
  using E = typename O::E;
  float* gl = reinterpret_cast<float*>(lds);
  float* am = gl + kGateFloats;     // diag(eta) M, block by block replaced by the unit lower inverse
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = wave_id();
  const int u = __builtin_amdgcn_readfirstlane((int)(blk / nr));
  const int r = __builtin_amdgcn_readfirstlane(r0 + (int)(blk % nr));
  const int b = u / a.H, h = u % a.H, hk = h / (a.H / a.HK);
  const int t0 = r * kDC, nt = min(kDC, max(0, live_tokens(a, b) - t0));
  const long cu = (long)u * a.nc_buf + (r - a.r_base);
  if (nt == 0) return;              // (no kernel reads anything of such a chunk)

  if (w == 0) {
    const bool ok = lane < nt;
    const float eta = ok ? *row_of<float>(a.eta, b, h, t0 + lane) : 0.0f;
    float gm = ok && a.gam.p ? *row_of<float>(a.gam, b, h, t0 + lane) : 0.0f;
    // -10^4 is as good as -inf (63 gates of at most e^88 each do not lift the sum back to
    // what fp32 holds), and differences of sums stay finite (a NaN stays NaN)
    gm = gm < -1e4f ? -1e4f : gm;
    double s = gm;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(s, o);
      if (lane >= o) s += y;
    }
    const double last = __shfl(s, 63);
    const float bh = (float)s, gi = expf(bh);
    gl[kGEta + lane] = eta;
    gl[kGEtaG + lane] = eta * gi;
    gl[kGsG + lane] = a.scale * gi;
    gl[kGEnd + lane] = expf((float)(last - s));
    gl[kGBh + lane] = bh;
    gl[kGBl + lane] = (float)(s - (double)bh);
    if (lane < 16) gl[kGC + lane] = expf((float)last);
  }

  // rows of the products: i = lab(w, c) (columns of the MFMA tile), columns
  // j = lab(m, .) of tile m (its rows)
  const Buf kp = buf_of(row_of<E>(a.k, b, hk, t0)), qp = buf_of(row_of<E>(a.q, b, hk, t0));
  const int i = lab(w, c), kst = (int)a.k.t, qst = (int)a.q.t;
  auto at = [&](int row, int st, int col) {   // byte offset of 8 elements of a live row
    return (unsigned)(row * st + col) * (unsigned)sizeof(E) | (row < nt && col < a.dk ? 0 : kNowhere);
  };
  typename O::X ki[DK / 32], qi[DK / 32];
#pragma unroll
  for (int kt = 0; kt < DK / 32; ++kt) {
    const int col = 32 * kt + 8 * g;
    ki[kt] = ld_row<BF>(kp, at(i, kst, col));
    qi[kt] = ld_row<BF>(qp, at(i, qst, col));
  }
  const int na = w / 2 + 1;         // 32-column blocks of this wave's rows
  f32x4 kk[4], qk[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    kk[m] = qk[m] = zero4();
    if (m < 2 * na) {
      const int j = lab(m, c);
#pragma unroll
      for (int kt = 0; kt < DK / 32; ++kt) {
        const int col = 32 * kt + 8 * g;
        const auto kj = ld_row<BF>(kp, at(j, kst, col));
        kk[m] = O::xx(kk[m], kj, ki[kt]);
        qk[m] = O::xx(qk[m], kj, qi[kt]);
      }
    }
  }
  __syncthreads();

  char* frag = a.frag + cu * 2 * tri_bytes(BF);
  const float bhi = gl[kGBh + i], bli = gl[kGBl + i], eta = gl[kGEta + i];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (x < na) {
      f32x4 p[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int j0 = 32 * x + 8 * g + 4 * y;
        const f32x4 bhj = *reinterpret_cast<const f32x4*>(gl + kGBh + j0);
        const f32x4 blj = *reinterpret_cast<const f32x4*>(gl + kGBl + j0);
        f32x4 m4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = j0 + e;
          const float d = exp_finite((bhi - bhj[e]) + (bli - blj[e]));
          m4[e] = j < i ? eta * (d * kk[2 * x + y][e]) : 0.0f;
          p[y][e] = j <= i ? a.scale * (d * qk[2 * x + y][e]) : 0.0f;
        }
        *reinterpret_cast<f32x4*>(am + i * LDT + j0) = m4;
      }
      put_frag<BF>(frag + tri_bytes(BF), fidx(w, x), lane, p[0], p[1]);
    }
  }
  if (w == 0) {
    float* go = a.gate + cu * kGateFloats;
#pragma unroll
    for (int x = 0; x < 6; ++x) go[64 * x + lane] = gl[64 * x + lane];
    if (lane < 16) go[6 * 64 + lane] = gl[6 * 64 + lane];
  }
  __syncthreads();

  // diagonal block w: its inverse by blocks of doubling size h (the inverse of
  // [[X, 0], [Z, Y]] has -Y^-1 Z X^-1 below its diagonal blocks).  T and its
  // transpose are kept in accumulator order, in which each is also the other's
  // row operand.
  {
    float* d = am + 16 * w * LDT + 16 * w;
    const f32x4 ar = blk_a(d, 0, 0, g, c), ac = blk_b(d, 0, 0, g, c);   // rows c; columns c
    f32x4 t, u;                         // T, T^T: rows 4 g + e of column c
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * g + e;
      t[e] = r == c ? 1.0f : below(r, c, 1) ? -ac[e] : 0.0f;
      u[e] = r == c ? 1.0f : below(c, r, 1) ? -ar[e] : 0.0f;
    }
#pragma unroll
    for (int h = 2; h < 16; h *= 2) {
      f32x4 mr, mc, z, y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * g + e;
        mr[e] = below(c, r, h) ? -ar[e] : 0.0f;
        mc[e] = below(r, c, h) ? -ac[e] : 0.0f;
      }
      z = y = zero4();
      mm16_2(z, mr, t, y, mc, u);
      const f32x4 t0 = t, u0 = u;
      mm16_2(t, u0, z, u, t0, y);
    }
    wave_lds_order();                   // (the block is read by this wave alone)
#pragma unroll
    for (int e = 0; e < 4; ++e) d[(4 * g + e) * LDT + c] = t[e];
  }
  __syncthreads();
  if (w < 2) {   // 16x16 blocks (1, 0) and (3, 2), each read by its wave alone
    const int o = 32 * w;
    f32x4 z = mm16(zero4(), blk_a(am, o + 16, o, g, c), blk_b(am, o, o, g, c));
    z = mm16(zero4(), blk_a(am, o + 16, o + 16, g, c), z);
    wave_lds_order();
#pragma unroll
    for (int e = 0; e < 4; ++e) am[(o + 16 + 4 * g + e) * LDT + o + c] = -z[e];
  }
  __syncthreads();
  {              // the 32x32 block below: wave w its block (w / 2, w mod 2)
    const int rt = w >> 1, ct = w & 1;
    f32x4 acc = zero4();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (x <= rt) {
        f32x4 z = zero4();
#pragma unroll
        for (int y = 0; y < 2; ++y)
          if (y >= ct)
            z = mm16(z, blk_a(am, 32 + 16 * x, 16 * y, g, c), blk_b(am, 16 * y, 16 * ct, g, c));
        acc = mm16(acc, blk_a(am, 32 + 16 * rt, 32 + 16 * x, g, c), z);
      }
    }
    __syncthreads();                    // every wave has read the block
#pragma unroll
    for (int e = 0; e < 4; ++e) am[(32 + 16 * rt + 4 * g + e) * LDT + 16 * ct + c] = -acc[e];
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (x < na) {
      const float* p = am + i * LDT + 32 * x + 8 * g;
      put_frag<BF>(frag, fidx(w, x), lane, *reinterpret_cast<const f32x4*>(p),
                      *reinterpret_cast<const f32x4*>(p + 4));
    }
  }
}

}  // namespace
}  // namespace e2ttt
