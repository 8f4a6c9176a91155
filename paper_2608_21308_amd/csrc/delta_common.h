// Shared pieces of the gated delta rule kernels (delta_*.hip).
//
// The rule, per unit (sequence, value head) and token, state W [dv][dk]:
//   Wd = exp(g) W,  e = v - Wd k,  u = eta e,  W' = Wd + u k^T,  o = s W' q.
// Over a chunk of 64 tokens with start state W_0, b_i = g_1 + .. + g_i,
// G_i = exp(b_i), D_ij = exp(b_i - b_j) and M = strictly lower(D o K K^T):
//   (I + diag(eta) M) U = diag(eta) R,       R = V - diag(G) K W_0^T
//   O   = s diag(G) Q W_0^T + P U,           P = s lower(D o Q K^T)
//   W_C = G_C W_0 + sum_j exp(b_C - b_j) u_j k_j^T
// (unrolling W_i and collecting u_j; the system is unit lower triangular).
// With T = (I + diag(eta) M)^-1 everything is a matrix product, T and P are
// independent of the state (delta_prep.hip, every chunk at once), and the
// columns of W^T (the value dimension) never meet: one wave carries 16 of
// them through all chunks in its registers (delta_fwd.hip).
//
// Layouts.  MFMA tiles are 16x16; the accumulator of a tile holds, in lane
// (g, c), rows 4 g + i (i = 0..3) of column c.  Token and key rows of tile m
// are labelled
//   lab(m, r) = 32 (m / 2) + 8 (r / 4) + 4 (m mod 2) + r mod 4,
// so that the registers of tiles 2 a and 2 a + 1, joined, are eight
// consecutive rows 32 a + 8 g .. + 7 of column c: the B operand of a product
// that contracts over those rows.  A chain of products (K W^T -> T R -> P U ->
// K^T U) then goes from accumulator to operand without leaving the lane.
#pragma once

#include <hip/hip_runtime.h>

#include "e2ttt.h"
#include "e2ttt_device.h"

namespace e2ttt {

constexpr int kDC = 64;           // tokens per chunk
constexpr int kDeltaFrags = 6;    // 16x32 fragments of a lower triangular 64x64 matrix
// Per chunk and unit: eta, eta G, s G, exp(b_C - b), 64 each, G_C (16 times),
// then b as two floats (b = bh + bl from a sum in 64 bits: differences of b keep
// their relative accuracy however far the sum has gone).
constexpr int kGateFloats = 6 * kDC + 16;
enum { kGEta = 0, kGEtaG = kDC, kGsG = 2 * kDC, kGEnd = 3 * kDC, kGC = 4 * kDC,
       kGBh = 4 * kDC + 16, kGBl = 5 * kDC + 16 };
constexpr int kGateChain = 4 * kDC + 16;   // the part that the chains read

// A token tensor [B][H][T][d] by its strides in elements (the last is 1).
struct View {
  const void* p;
  long b, h, t;
};

struct DeltaArgs {
  View q, k, v, eta, gam;     // gam.p nullable: no decay
  View out;
  View d_out, dq, dkk, dv_, deta, dgam;
  const int* lengths;         // nullable
  const float* w_in;          // nullable: zero
  float* w_out;               // nullable
  const float* d_w_out;       // nullable: zero
  float* d_w_in;              // nullable
  char* frag;                 // [chunk unit] T, then P, in terms
  bool save;                  // a backward follows
  float* gate;                // [chunk unit][kGateFloats]
  float* wst;                 // [chunk unit][dvp x dkp] chunk-start states (saving), in lane order
  float* ust;                 // [chunk unit][dvp x 64] U^T (saving), in lane order
  float* dwst;                // backward: chunk-end adjoint states, as wst
  float* yst;                 // backward: Y^T, as ust
  int B, HK, H, T, dk, dv, dvp;   // dvp: dv padded to a multiple of 32
  int NC;                     // chunks of the whole call
  int r0, r1;                 // chunks of this launch
  // The launch's chunks in nseg segments of seglen (the last may be shorter):
  int nseg, seglen;
  float* segs;                // [unit][nseg] what the segments start (backward: end) from, in lane
                              // order (dvp x dkp)
  float* segb;                // [unit][nseg] what they make of a zero state, in lane order
  float* segf;                // [unit][nseg] their transitions F (W -> W F): rows in lane order
                              // (dkp x dkp), then the transpose as row operands (operand_at)
  int nc_buf;                 // chunks per unit that the buffers hold (index r - r_base)
  int r_base;
  float scale;
};

// The wave's number in its workgroup, in a scalar register.
__device__ __forceinline__ int wave_id() {
  return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
}

__device__ __forceinline__ int lab(int m, int r) {
  return 32 * (m >> 1) + 8 * (r >> 2) + 4 * (m & 1) + (r & 3);
}
// exp(x) of a finite x: the hardware's power of two at x log2 e rounded, times
// 1 + ln 2 times what the rounding left (2^-23 relative).
__device__ __forceinline__ float exp_finite(float x) {
  const float h = x * 1.44269504f;
  const float l = fmaf(x, 1.44269504f, -h) + x * 1.92596299e-8f;
  const float p = __builtin_amdgcn_exp2f(h);
  return fmaf(p, l * 0.693147181f, p);
}
// Fragment (row tile m, 32-column block a <= m / 2) of a lower triangular matrix.
__host__ __device__ constexpr int fidx(int m, int a) { return m < 2 ? m : 2 * (m - 1) + a; }

// Operands.  X: a value of the io type, exact.  S: an fp32 value; with bf16 io
// the sum of NT = 3 bf16 terms, each the rounding of what the ones before leave: 8
// bits each, 24 in all, so that nothing is lost (of values whose rounding is finite,
// to 3.39e38).  A product with an X operand is then exact up to its fp32 sums.  One of
// two S operands takes the six pairs of terms of combined order 0 to 2; with a term at
// most 2^-8 of the one before, what the other three leave out is at most 2 (2^-8
// 2^-16) = 2^-23 of the product, of either sign.  (Terms cut off instead of rounded
// save up to 2 % of the time, and lose up to 2^-21, always towards zero.)  f32 io: fp32
// MFMA.
template <bool BF> struct DOp;

template <> struct DOp<true> {
  using E = __bf16;
  static constexpr int NT = 3;
  struct X { bf16x8 v; };
  struct S { bf16x8 t[NT]; };
  static __device__ __forceinline__ f32x4 m1(f32x4 acc, const bf16x8& a, const bf16x8& b) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 xx(f32x4 acc, const X& a, const X& b) {
    return m1(acc, a.v, b.v);
  }
  static __device__ __forceinline__ f32x4 xs(f32x4 acc, const X& a, const S& b) {
#pragma unroll
    for (int i = NT - 1; i >= 0; --i) acc = m1(acc, a.v, b.t[i]);
    return acc;
  }
  static __device__ __forceinline__ f32x4 sx(f32x4 acc, const S& a, const X& b) {
#pragma unroll
    for (int i = NT - 1; i >= 0; --i) acc = m1(acc, a.t[i], b.v);
    return acc;
  }
  static __device__ __forceinline__ f32x4 ss(f32x4 acc, const S& a, const S& b) {
#pragma unroll
    for (int n = NT - 1; n >= 0; --n)
#pragma unroll
      for (int i = 0; i <= n; ++i) acc = m1(acc, a.t[i], b.t[n - i]);
    return acc;
  }
  // Two products at once, issued in turn: an MFMA waits for the one before it
  // on the same accumulator twice as long as for the matrix unit.
  static __device__ __forceinline__ void xs2(f32x4& c0, const X& a0, const S& b0, f32x4& c1,
                                             const X& a1, const S& b1) {
#pragma unroll
    for (int i = NT - 1; i >= 0; --i) {
      c0 = m1(c0, a0.v, b0.t[i]);
      c1 = m1(c1, a1.v, b1.t[i]);
    }
  }
  static __device__ __forceinline__ void sx2(f32x4& c0, const S& a0, const X& b0, f32x4& c1,
                                             const S& a1, const X& b1) {
#pragma unroll
    for (int i = NT - 1; i >= 0; --i) {
      c0 = m1(c0, a0.t[i], b0.v);
      c1 = m1(c1, a1.t[i], b1.v);
    }
  }
  static __device__ __forceinline__ void ss2(f32x4& c0, const S& a0, const S& b0, f32x4& c1,
                                             const S& a1, const S& b1) {
#pragma unroll
    for (int n = NT - 1; n >= 0; --n)
#pragma unroll
      for (int i = 0; i <= n; ++i) {
        c0 = m1(c0, a0.t[i], b0.t[n - i]);
        c1 = m1(c1, a1.t[i], b1.t[n - i]);
      }
  }
  static __device__ __forceinline__ S split(f32x4 x, f32x4 y) {
    typedef __attribute__((ext_vector_type(8))) float f8;
    typedef __attribute__((ext_vector_type(4))) unsigned u4;
    S s;
    f8 v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      s.t[i] = __builtin_convertvector(v, bf16x8);
      if (i + 1 < NT) {
        const u4 p = __builtin_bit_cast(u4, s.t[i]);   // (pairs: a term is the upper half of its float)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[2 * e] -= __uint_as_float(p[e] << 16);
          v[2 * e + 1] -= __uint_as_float(p[e] & 0xffff0000u);
        }
      }
    }
    return s;
  }
  static __device__ __forceinline__ void sum(const S& s, f32x4& x, f32x4& y) {   // of all terms
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = ((float)s.t[2][e] + (float)s.t[1][e]) + (float)s.t[0][e];
      y[e] = ((float)s.t[2][4 + e] + (float)s.t[1][4 + e]) + (float)s.t[0][4 + e];
    }
  }
  static __device__ __forceinline__ void values(const X& p, f32x4& x, f32x4& y) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = (float)p.v[e];
      y[e] = (float)p.v[4 + e];
    }
  }
};

template <> struct DOp<false> {
  using E = float;
  static constexpr int NT = 1;
  struct X { f32x4 a, b; };
  using S = X;
  static __device__ __forceinline__ void sum(const S& p, f32x4& x, f32x4& y) {
    x = p.a;
    y = p.b;
  }
  static __device__ __forceinline__ f32x4 xx(f32x4 acc, const X& p, const X& q) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(p.a[e], q.a[e], acc, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(p.b[e], q.b[e], acc, 0, 0, 0);
    return acc;
  }
  static __device__ __forceinline__ f32x4 xs(f32x4 acc, const X& p, const X& q) { return xx(acc, p, q); }
  static __device__ __forceinline__ f32x4 sx(f32x4 acc, const X& p, const X& q) { return xx(acc, p, q); }
  static __device__ __forceinline__ f32x4 ss(f32x4 acc, const X& p, const X& q) { return xx(acc, p, q); }
  static __device__ __forceinline__ void ss2(f32x4& c0, const X& a0, const X& b0, f32x4& c1,
                                             const X& a1, const X& b1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c0 = __builtin_amdgcn_mfma_f32_16x16x4f32(a0.a[e], b0.a[e], c0, 0, 0, 0);
      c1 = __builtin_amdgcn_mfma_f32_16x16x4f32(a1.a[e], b1.a[e], c1, 0, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c0 = __builtin_amdgcn_mfma_f32_16x16x4f32(a0.b[e], b0.b[e], c0, 0, 0, 0);
      c1 = __builtin_amdgcn_mfma_f32_16x16x4f32(a1.b[e], b1.b[e], c1, 0, 0, 0);
    }
  }
  static __device__ __forceinline__ void xs2(f32x4& c0, const X& a0, const X& b0, f32x4& c1,
                                             const X& a1, const X& b1) {
    ss2(c0, a0, b0, c1, a1, b1);
  }
  static __device__ __forceinline__ void sx2(f32x4& c0, const X& a0, const X& b0, f32x4& c1,
                                             const X& a1, const X& b1) {
    ss2(c0, a0, b0, c1, a1, b1);
  }
  static __device__ __forceinline__ S split(f32x4 x, f32x4 y) { return S{x, y}; }
  static __device__ __forceinline__ void values(const X& p, f32x4& x, f32x4& y) {
    x = p.a;
    y = p.b;
  }
};

// A lower triangular 64x64 matrix as the fragments of its terms, in global
// memory and in LDS: 16 bytes a lane and fragment (in the order of frag_slot), the
// fragments of a term together (f32 io: the two halves of a fragment's fp32
// values at lane * 16 and 1024 + lane * 16).
__host__ __device__ constexpr int tri_bytes(bool bf) {
  return bf ? DOp<true>::NT * kDeltaFrags * 1024 : kDeltaFrags * 2048;
}
// Lane l's 16 bytes of a term lie at slot l XOR 4 x, x = 0, 3, 1, 2 for lane
// groups 0 .. 3: the sixteen lanes of a transposing read (four rows of four lane
// groups) and those that a 16-byte read serves together (LTile) meet all banks.
__device__ __forceinline__ int frag_slot(int lane) {
  return lane ^ ((lane >> 3) & 4) ^ ((lane & 16) ? 12 : 0);
}
// One lane's part of fragment f.
template <bool BF>
__device__ __forceinline__ void put_frag(char* p, int f, int lane, f32x4 x, f32x4 y) {
  if constexpr (BF) {
    const auto s = DOp<true>::split(x, y);
#pragma unroll
    for (int i = 0; i < DOp<BF>::NT; ++i)
      *reinterpret_cast<bf16x8*>(p + ((i * kDeltaFrags + f) * 64 + frag_slot(lane)) * 16) = s.t[i];
  } else {
    *reinterpret_cast<f32x4*>(p + f * 2048 + lane * 16) = x;
    *reinterpret_cast<f32x4*>(p + f * 2048 + 1024 + lane * 16) = y;
  }
}
template <bool BF>
__device__ __forceinline__ typename DOp<BF>::S ld_frag(const char* lds, int f, int lane) {
  typename DOp<BF>::S s;
  if constexpr (BF) {
#pragma unroll
    for (int i = 0; i < DOp<BF>::NT; ++i)
      s.t[i] = *reinterpret_cast<const bf16x8*>(lds + ((i * kDeltaFrags + f) * 64 + frag_slot(lane)) * 16);
  } else {
    s.a = *reinterpret_cast<const f32x4*>(lds + f * 2048 + lane * 16);
    s.b = *reinterpret_cast<const f32x4*>(lds + f * 2048 + 1024 + lane * 16);
  }
  return s;
}

// What a chain leaves for the gradients, in the order of its lanes: per 16
// columns and 32 rows, the lanes' first four values, then their second (row
// 16 tile + c, columns 32 blk + 8 g ..; a wave writes whole lines).
__device__ __forceinline__ long lane_at(int tile, int blk, int nblk, int lane) {
  return ((long)(tile * nblk + blk) * 2 * 64 + lane) * 4;
}
// Element (row, column) of a matrix kept as the row operands of a product, rows
// labelled by lab(): per row tile and 32 columns as lane_at.
__device__ __forceinline__ int operand_at(int row, int col, int nblk) {
  const int m = 2 * (row >> 5) + ((row >> 2) & 1), c = 4 * ((row >> 3) & 3) + (row & 3);
  return (((m * nblk + (col >> 5)) * 2 + ((col >> 2) & 1)) * 64 + 16 * ((col >> 3) & 3) + c) * 4 +
         (col & 3);
}
__device__ __forceinline__ void st_lane(float* p, f32x4 x, f32x4 y) {
  *reinterpret_cast<f32x4*>(p) = x;
  *reinterpret_cast<f32x4*>(p + 256) = y;
}

// One transposing LDS read: within each group of 16 lanes, lane c receives
// element c mod 4 of the quads addressed by lanes 4 r + c / 4, r = 0..3.
__device__ __forceinline__ bf16x4 lds_tr4(const __bf16* p) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s4* lds_s4;
  return __builtin_bit_cast(
      bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4) const_cast<__bf16*>(p)));
}
__device__ __forceinline__ bf16x8 cat8(const bf16x4& a, const bf16x4& b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Fragment of the transpose of a lower triangular matrix in LDS: rows j =
// lab(m, c), contraction over i = 32 a + 8 g .. + 7, a >= m / 2.  Element
// (i, j) sits in fragment (2 a + (i / 4) mod 2, m / 2), lane group
// (j mod 32) / 8, lane 4 g + i mod 4, slot j mod 8.
template <bool BF>
__device__ __forceinline__ typename DOp<BF>::S ld_frag_t(const char* lds, int m, int a, int g,
                                                          int c) {
  typename DOp<BF>::S s;
  if constexpr (BF) {
    const int r = c >> 2, cq = c & 3;
#pragma unroll
    for (int i = 0; i < DOp<BF>::NT; ++i) {
      bf16x4 h[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
        h[x] = lds_tr4(reinterpret_cast<const __bf16*>(lds) +
                       ((i * kDeltaFrags + fidx(2 * a + x, m >> 1)) * 64 + frag_slot(16 * cq + 4 * g + r)) * 8 +
                       4 * (m & 1));
      s.t[i] = cat8(h[0], h[1]);
    }
  } else {
    const int gj = c >> 2, sj = 4 * (m & 1) + (c & 3);   // lane group and slot of column j
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = (16 * gj + 4 * g + e) * 16 + (sj >> 2) * 1024 + (sj & 3) * 4;
      s.a[e] = *reinterpret_cast<const float*>(lds + fidx(2 * a, m >> 1) * 2048 + at);
      s.b[e] = *reinterpret_cast<const float*>(lds + fidx(2 * a + 1, m >> 1) * 2048 + at);
    }
  }
  return s;
}

// A tile of rows of D elements of the io type in LDS, in 16-byte pieces; piece
// p of a row lies at p XOR a function of the row's low bits b0 .. b4.  A 16-byte
// read serves lanes 0-3, 12-15, 20-27 together, then 4-11, 16-19, 28-31, and so
// on; an 8-byte transposing read a group of 16.  With bf16 the function spreads
// over the 256 bytes of the banks the rows of a fragment read (b0, b1, b3, b4
// differ; the lane groups 0 and 1, 2 and 3 ask for neighbouring pieces), the four
// rows (b0, b1) of a transposing read.  (b2 stays out: the rows 4 on that such a
// read goes on to are then a constant away; with COLS it is in, for tiles that
// are written by columns, sixteen rows of a piece at a time.)  fp32 fragments are
// two pieces, which takes another one.
template <bool BF, int D, bool COLS = false>
struct LTile {
  using E = typename DOp<BF>::E;
  static constexpr int PE = 16 / (int)sizeof(E);     // elements of a piece
  static constexpr int NP = D / PE;                  // pieces of a row
  static __device__ __forceinline__ int at(int row, int p) {   // element index of a piece
    if constexpr (!BF) return (row * NP + (p ^ (((row & 3) | ((row >> 1) & 12)) & (NP - 1)))) * PE;
    // (rows of 64 and 128 bytes: b0 and b1, b0 move the bank by themselves)
    const int up = NP >= 16 ? (row & 3) << 2 : NP == 8 ? (row & 2) << 1 : 0;
    const int b4 = (row >> 4) & 1, f = up | (((row >> 2) & 2) ^ (3 * b4));
    return (row * NP + (p ^ f ^ (COLS ? (row >> 2) & 1 : 0))) * PE;
  }
  // row `row`, columns 32 kt + 8 g .. + 7
  static __device__ __forceinline__ typename DOp<BF>::X frag(const E* t, int row, int kt, int g) {
    typename DOp<BF>::X x;
    if constexpr (BF) {
      x.v = *reinterpret_cast<const bf16x8*>(t + at(row, 4 * kt + g));
    } else {
      x.a = *reinterpret_cast<const f32x4*>(t + at(row, 8 * kt + 2 * g));
      x.b = *reinterpret_cast<const f32x4*>(t + at(row, 8 * kt + 2 * g + 1));
    }
    return x;
  }
  // Rows 32 a + 8 g .. + 7 of one column: lab(m, c) or, natural, 16 m + c.
  template <bool NAT = false>
  static __device__ __forceinline__ typename DOp<BF>::X frag_t(const E* t, int m, int a, int g,
                                                               int c) {
    typename DOp<BF>::X x;
    if constexpr (BF) {
      const int row = 32 * a + 8 * g + (c >> 2);
      const int p = NAT ? 2 * m + ((c & 3) >> 1) : 4 * (m >> 1) + (c & 3);
      const int e = NAT ? 4 * (c & 1) : 4 * (m & 1);
      x.v = cat8(lds_tr4(t + at(row, p) + e), lds_tr4(t + at(row + 4, p) + e));
    } else {
      const int col = NAT ? 16 * m + c : lab(m, c), p = col >> 2, e4 = col & 3;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x.a[e] = t[at(32 * a + 8 * g + e, p) + e4];
        x.b[e] = t[at(32 * a + 8 * g + 4 + e, p) + e4];
      }
    }
    return x;
  }
};

// The same from the terms of an S operand, each a tile `plane` elements on.
template <bool BF, int D, bool NAT>
__device__ __forceinline__ typename DOp<BF>::S terms_t(const typename DOp<BF>::E* t, int plane,
                                                        int m, int g, int c) {
  if constexpr (BF) {
    typename DOp<BF>::S s;
#pragma unroll
    for (int i = 0; i < DOp<BF>::NT; ++i)
      s.t[i] = LTile<BF, D, true>::template frag_t<NAT>(t + plane * i, m, 0, g, c).v;
    return s;
  } else {
    return LTile<BF, D, true>::template frag_t<NAT>(t, m, 0, g, c);
  }
}
// Eight fp32 values of such a tile's row (columns 8 p8 ..) into LDS as terms.
template <bool BF, int D>
__device__ __forceinline__ void put_terms(typename DOp<BF>::E* t, int plane, int row, int p8,
                                          f32x4 x, f32x4 y) {
  using L = LTile<BF, D, true>;
  if constexpr (BF) {
    const auto s = DOp<true>::split(x, y);
#pragma unroll
    for (int i = 0; i < DOp<true>::NT; ++i)
      *reinterpret_cast<bf16x8*>(t + plane * i + L::at(row, p8)) = s.t[i];
  } else {
    *reinterpret_cast<f32x4*>(t + L::at(row, 2 * p8)) = x;
    *reinterpret_cast<f32x4*>(t + L::at(row, 2 * p8 + 1)) = y;
  }
}

template <class E>
__device__ __forceinline__ const E* row_of(const View& v, int b, int h, int t) {
  return static_cast<const E*>(v.p) + (b * v.b + h * v.h + t * v.t);
}
template <class E>
__device__ __forceinline__ E* row_of_w(const View& v, int b, int h, int t) {
  return static_cast<E*>(const_cast<void*>(v.p)) + (b * v.b + h * v.h + t * v.t);
}
// Tokens of sequence b that the call takes.
__device__ __forceinline__ int live_tokens(const DeltaArgs& a, int b) {
  return a.lengths ? max(0, min(a.T, a.lengths[b])) : a.T;
}

// Memory from a uniform address on, addressed by byte offsets of 31 bits; an
// access at kNowhere or behind it is dropped (reads zero).  A masked lane then
// needs no branch, and without branches between them the compiler knows how many
// stores are younger than a load: waiting for it does not wait for them.
typedef __amdgpu_buffer_rsrc_t Buf;
constexpr unsigned kNowhere = 0x80000000u;
__device__ __forceinline__ Buf buf_of(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00020000);
}
__device__ __forceinline__ u32x4 buf_ld(Buf b, unsigned at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, 0, 0));
}
__device__ __forceinline__ void buf_st(Buf b, unsigned at, f32x4 x) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), b, (int)at, 0, 0);
}
// Four neighbouring values of the io type, streaming.
template <bool BF>
__device__ __forceinline__ void buf_st_io(Buf b, unsigned at, f32x4 x) {
  typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
  if constexpr (BF)
    __builtin_amdgcn_raw_buffer_store_b64(
        __builtin_bit_cast(u32x2, bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]}), b,
        (int)at, 0, 2);
  else
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), b, (int)at, 0, 2);
}

struct DeltaStepArgs {
  View q, k, v, eta, gam, out;
  float* w;
  const int* slots;      // nullable: sequence b at state b
  int nslots;
  int B, HK, H, T, dk, dv;
  float scale;
};

// -------------------------------------------------------------- launchers
hipError_t launch_delta_step(const DeltaStepArgs& a, bool bf, hipStream_t stream);
hipError_t launch_delta_prep(const DeltaArgs& a, bool bf, hipStream_t stream);
// The chain over every segment from its start (end) state: `state`, only what
// the segments make of a zero state and their transitions.
hipError_t launch_delta_chain(const DeltaArgs& a, bool bf, bool save, bool state, hipStream_t stream);
hipError_t launch_delta_chain_bwd(const DeltaArgs& a, bool bf, bool state, hipStream_t stream);
// bf16, dk in 33..64, no segments: the chain over r0 .. r1 - 1 beside the preparation
// of the np chunks from p0 on, or the gradients of the ng from g0 on.
hipError_t launch_delta_chain_prep(const DeltaArgs& a, bool save, int p0, int np, hipStream_t stream);
hipError_t launch_delta_chain_bwd_grads(const DeltaArgs& a, int g0, int ng, hipStream_t stream);
// The segments' start states from their parts, one after the other.
hipError_t launch_delta_join(const DeltaArgs& a, bool bf, bool bwd, hipStream_t stream);
hipError_t launch_delta_grads(const DeltaArgs& a, bool bf, hipStream_t stream);
// padded key dimension (32, 64 or 128) and value dimension (a multiple of 32)
inline int delta_dkp(int dk) { return dk <= 32 ? 32 : dk <= 64 ? 64 : 128; }
inline int delta_dvp(int dv) { return (dv + 31) & ~31; }

}  // namespace e2ttt
