// Shared pieces of the attention kernels (attn_*.hip).
//
// Per sequence, query head and query t at position p = t + S - T, over the keys
// j that it sees (p - left <= j <= p + right, j before the sequence's end):
//   s_j = scale q . k_j,  lse = log sum_j e^s_j,  P_j = e^(s_j - lse),  o = sum_j P_j v_j
// and, with D = sum_c do_c o_c - d_lse,
//   dv_j += P_j do,  dS_j = P_j (do . v_j - D),  dq = scale sum_j dS_j k_j,
//   dk_j += scale dS_j q.
//
// Layouts.  Products are MFMA tiles of 32 x 32; the accumulator of a tile holds, in
// lane (h, c) = (lane / 32, lane mod 32), rows 8 a + 4 h + i (register 4 a + i, a, i =
// 0..3) of column c.  A step of a product contracts 16 indices, eight from each
// half of the wave.  The scores are formed so that what is contracted next runs
// over their rows: registers 8 s .. 8 s + 7 are then, after rounding, an operand of
// step s as they stand, over the indices 16 s + 8 (j / 4) + 4 h + j mod 4.  The other
// operand takes the same indices from LDS (rows_t).  Scores never leave the lane.
#pragma once

#include <algorithm>

#include "delta_common.h"
#include "div.h"

namespace e2ttt {

typedef __attribute__((ext_vector_type(16))) float f32x16;

// What a workgroup works on.  Workgroups are dealt to the 8 XCDs in turn: those of a key
// head, which share its keys and values, go to one of them and its L2, the key heads in
// turn (12 sequences of 250 to 3000 tokens, 8 query and 2 key heads of 128: 180 us, backward
// 600; with an eighth of the workgroups in a row to each XCD 235 and 1017).  What 8 does not
// divide stays as it is dealt.
//   Where rows are of unequal length (causal, say) a head deals its long ones first, and the
// next head's long ones would begin late: heads that fill an XCD's places together are
// dealt in turn, row by row (dk and dv, 2 x 16 x 2048 x 128: 162 us one head after the
// other, 121 by two, 142 by four; of 64: 59, 57 and 52; 8 x 16 x 2048 x 64: 193 and 179 by
// four; forward and dq, 32 heads of 4096 x 128: 175 + 254 and 154 + 216 by two).  Where two
// workgroups share a CU (position y with y + 32) long and short ones meet by `fold` (forward
// 2 x 8 x 4096 x 128 111 us without and 89 with it, 16 x 8192 x 64 202 and 177; dq 216 and
// 222; where they do not, float32 4 x 8 x 2048 x 64: 157 + 233 and 197 + 294).
struct Work {
  Div row, tiles, heads, HK;     // workgroups of a head; tiles of them; heads of a key head
  Div bunch, block, rest;        // heads that are dealt in turn; their workgroups; the last heads
  unsigned bunches;              // whole ones of an XCD
  unsigned full;                 // workgroups of the key heads that 8 divides
  bool fold;                     // every second 32 of an XCD's workgroups in reverse
};
// uneven: the places of an XCD that are filled at once where rows are of unequal length, else 0
inline Work work_of(int B, int HK, int heads, int tiles, int splits, unsigned uneven, bool fold) {
  const unsigned row = (unsigned)tiles * splits, each = (unsigned)((long)B * HK / 8 * heads);
  const unsigned n = std::max(1u, std::min(each, (uneven + row - 1) / row));
  return Work{div_by(row), div_by((unsigned)tiles), div_by((unsigned)heads), div_by((unsigned)HK),
              div_by(n), div_by(n * row), div_by(std::max(1u, each % n)), each / n, each * 8 * row, fold};
}
struct Place {
  int b, hk, head, split, tile;  // head: of the query heads of a key head
};
__device__ __forceinline__ Place place_of(const Work& w, unsigned id) {
  const bool dealt = id < w.full;
  unsigned y = dealt ? id >> 3 : id, hh, r;
  if (dealt) {
    if (w.fold && (y & 32) && (y | 31) < w.full / 8) y ^= 31;
    const unsigned i = w.block.of(y), j = y - i * w.block.d;
    const Div& n = i < w.bunches ? w.bunch : w.rest;
    r = n.of(j);
    hh = i * w.bunch.d + j - r * n.d;
  } else {
    hh = w.row.of(y);
    r = y - hh * w.row.d;
  }
  const unsigned q = w.heads.of(hh), u = dealt ? (id & 7) + 8 * q : q, b = w.HK.of(u);
  const unsigned split = w.tiles.of(r);
  return Place{(int)b, (int)(u - b * w.HK.d), (int)(hh - q * w.heads.d), (int)split,
               (int)(r - split * w.tiles.d)};
}

struct AttnArgs {
  View q, k, v, out;          // [B][H or HK][T or S][d]
  View d_out, dq, dk, dv;
  float* lse;                 // [B][H][T], nullable in the forward
  const float* d_lse;         // nullable
  float* ex;                  // backward, [B][H][T]: -lse log2 e (-inf for queries that see nothing)
  float* delta;               // backward, [B][H][T]: -D
  const int* lengths;         // nullable
  int B, HK, H, rep, T, S, d;   // rep: query heads of a key head
  int left, right;            // at most 2^30 - 1; negative: no bound
  float scale;
  // A tile of queries (keys) as several workgroups, each over a stretch of the keys
  // (queries): their sums [stretch][row][d] and, in the forward, [stretch][row] {reference,
  // sum} are joined by another kernel.
  int nsplit, nsplit_kv;
  Work work;                  // of a launch
  float* part;
  float2* part_ml;
};

constexpr float kLog2e = 1.44269504088896f;
constexpr float kNegInf = -INFINITY;

// Products on 32 x 32 tiles.  X: eight contraction indices of a row.
template <bool BF> struct MOp;
template <> struct MOp<true> {
  using E = __bf16;
  struct X { bf16x8 v; };
  static __device__ __forceinline__ f32x16 mm(const f32x16& c, const X& a, const X& b) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
  }
  static __device__ __forceinline__ X of(const f32x16& p, int s) {   // registers 8 s .. 8 s + 7
    X x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] = (__bf16)p[8 * s + j];
    return x;
  }
};
template <> struct MOp<false> {
  using E = float;
  struct X { f32x4 a, b; };
  static __device__ __forceinline__ f32x16 mm(f32x16 c, const X& a, const X& b) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.a[j], b.a[j], c, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.b[j], b.b[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ X of(const f32x16& p, int s) {
    X x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x.a[j] = p[8 * s + j];
      x.b[j] = p[8 * s + 4 + j];
    }
    return x;
  }
};

__device__ __forceinline__ f32x16 zero16() {
  f32x16 x;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.0f;
  return x;
}
// Scores of rows before `from` and from `to` on (counted from the first accumulator's) do
// not count.
template <int NT>
__device__ __forceinline__ void cut_rows(f32x16 (&s)[NT], int from, int to, int h) {
  from -= 4 * h;                   // (row 8 (i / 4) + 4 h + i mod 4 of register i)
  to -= 4 * h;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 32 * n + 8 * (i >> 2) + (i & 3);
      s[n][i] = r >= from && r < to ? s[n][i] : kNegInf;
    }
}

// Across the two halves of a wave.
__device__ __forceinline__ void halves(float x, float& lo, float& hi) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  lo = __uint_as_float(r[0]);
  hi = __uint_as_float(r[1]);
}
__device__ __forceinline__ float both_max(float x) {
  float a, b;
  halves(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float both_sum(float x) {
  float a, b;
  halves(x, a, b);
  return a + b;
}

// A tile of rows of D elements in LDS (pieces of 16 bytes placed by LTile, whose
// order keeps both of the reads below off each other's banks: a row read serves
// sixteen rows at a time that differ in bits 0, 1, 3, 4).
template <bool BF, int D>
struct ATile {
  using L = LTile<BF, D>;
  using E = typename L::E;
  using X = typename MOp<BF>::X;
  static constexpr int PE = L::PE, NP = L::NP;
  // Row `row`, columns 16 ks + 8 h .. + 7.
  static __device__ __forceinline__ X rows(const E* t, int row, int ks, int h) {
    X x;
    if constexpr (BF) {
      x.v = *reinterpret_cast<const bf16x8*>(t + L::at(row, 2 * ks + h));
    } else {
      x.a = *reinterpret_cast<const f32x4*>(t + L::at(row, 4 * ks + 2 * h));
      x.b = *reinterpret_cast<const f32x4*>(t + L::at(row, 4 * ks + 2 * h + 1));
    }
    return x;
  }
  // Column 32 m + c, rows r0 + 8 (j / 4) + 4 h + j mod 4.
  static __device__ __forceinline__ X rows_t(const E* t, int r0, int m, int h, int c) {
    X x;
    if constexpr (BF) {
      // (a transposing read: sixteen lanes name four rows of four quads)
      const int row = r0 + 4 * h + ((c & 15) >> 2), col = 32 * m + (c & 16) + 4 * (c & 3);
      x.v = cat8(lds_tr4(t + L::at(row, col >> 3) + (col & 7)),
                 lds_tr4(t + L::at(row + 8, col >> 3) + (col & 7)));
    } else {
      const int p = 8 * m + (c >> 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x.a[j] = t[L::at(r0 + 4 * h + j, p) + (c & 3)];
        x.b[j] = t[L::at(r0 + 8 + 4 * h + j, p) + (c & 3)];
      }
    }
    return x;
  }
};

// Rows from `base` on into a tile, without passing through registers: each of NW
// waves takes its part, a lane one piece per load.  Rows from `n` on and columns
// from `d` on become zeros.  (Rows are at most 2^23 elements apart, so that 64 of
// them lie within a buffer's 31 bits.)
template <bool BF, int D, int ROWS, int NW>
struct Stage {
  using L = LTile<BF, D>;
  using E = typename L::E;
  static constexpr int N = ROWS * L::NP / (64 * NW);
  static_assert(N * 64 * NW == ROWS * L::NP, "whole loads");
  unsigned at[N];             // bytes from base (kNowhere: behind d)
  int row[N];
  __device__ __forceinline__ void init(long stride, int d, int w, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = (w * N + i) * 64 + lane, r = s / L::NP;
      const int p = (s % L::NP) ^ (L::at(r, 0) / L::PE - r * L::NP);
      row[i] = r;
      at[i] = p * L::PE < d ? (unsigned)(r * stride * (long)sizeof(E)) + p * 16u : kNowhere;
    }
  }
  __device__ __forceinline__ void load(E* tile, const E* base, int n, int w) const {
    const Buf b = buf_of(base);
#pragma unroll
    for (int i = 0; i < N; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          b, (__attribute__((address_space(3))) void*)(tile + (w * N + i) * 64 * L::PE), 16,
          (int)(row[i] < n ? at[i] : kNowhere), 0, 0, 0);
  }
};
// 64 floats of a row from base on (zeros from `n` on), by one wave.
__device__ __forceinline__ void stage64(float* to, const float* base, int n, int lane) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(buf_of(base), (__attribute__((address_space(3))) void*)to, 4,
                                           (int)(lane < n ? 4u * lane : kNowhere), 0, 0, 0);
}
__device__ __forceinline__ void staged() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Eight elements of a row as an operand (row null or columns behind d: zeros).
template <bool BF>
__device__ __forceinline__ typename MOp<BF>::X row_frag(const typename MOp<BF>::E* row, int col, int d) {
  typename MOp<BF>::X x{};
  if (row && col < d) {
    if constexpr (BF) {
      x.v = *reinterpret_cast<const bf16x8*>(row + col);
    } else {
      x.a = *reinterpret_cast<const f32x4*>(row + col);
      x.b = *reinterpret_cast<const f32x4*>(row + col + 4);
    }
  }
  return x;
}

// A tile [channels][rows of the lanes] written to the lanes' rows: channels 32 m + ..,
// of the columns before d.
template <bool BF>
__device__ __forceinline__ void st_tile(typename MOp<BF>::E* row, const f32x16& o, float f, int m,
                                        int h, int d) {
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int ch = 32 * m + 8 * a + 4 * h;
    if (ch < d) {
      const f32x4 x{o[4 * a] * f, o[4 * a + 1] * f, o[4 * a + 2] * f, o[4 * a + 3] * f};
      IoT<BF>::st4(row + ch, x);
    }
  }
}

// Queries of sequence b that the call takes.
__device__ __forceinline__ int live_of(const AttnArgs& a, int b) {
  return a.lengths ? max(0, min(a.T, a.lengths[b])) : a.T;
}

// Whether a live query at position p sees a key of a sequence that ends at `end`.
__device__ __forceinline__ bool sees_some(const AttnArgs& a, int p, int end) {
  return (a.left < 0 ? 0 : max(0, p - a.left)) < (a.right < 0 ? end : min(end, p + a.right + 1));
}
// The sum of a query that sees keys: it is positive and finite (the largest of its terms
// is at least one) unless a score has left the range of fp32, which is no sum of zero.
__device__ __forceinline__ float sum_of(float x) { return x > 0.0f && x < INFINITY ? x : NAN; }

// The sums of a lane's row, before they are joined.
__device__ __forceinline__ void st_part(float* row, const f32x16& o, int m, int h, int d) {
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int ch = 32 * m + 8 * a + 4 * h;
    if (ch < d)
      *reinterpret_cast<f32x4*>(row + ch) = f32x4{o[4 * a], o[4 * a + 1], o[4 * a + 2], o[4 * a + 3]};
  }
}
// Stretch `split` of `n` of the range lo .. hi - 1, in whole tiles of `tile`.
__device__ __forceinline__ void stretch_of(int& lo, int& hi, int tile, int split, int n) {
  const int nt = hi > lo ? (hi - lo + tile - 1) / tile : 0;
  const int l = lo;
  lo = l + (int)((long)nt * split / n) * tile;
  hi = min(hi, l + (int)((long)nt * (split + 1) / n) * tile);
}

// Rows of a tile of the inner loops: of keys in the forward and for dq, of queries for dk
// and dv.  (Head dim 128, 2 x 16 x 2048 tokens, causal: backward 221 us with 32 rows for dk
// and dv, 257 with 64; 4 x 32 x 4096, window 1024: 1135 us with 32 for dq, 1170 with 64;
// the forward 361 with 32, 343 with 64.)
constexpr int attn_tile(bool bf, int d) { return !bf && d > 64 ? 32 : 64; }
constexpr int attn_tile_bwd(int d) { return d > 64 ? 32 : 64; }
// Stretches that `groups` workgroups of `tiles` tiles each are split into, for at most
// `places` workgroups (halve: in two where a few more leave CUs to the longest rows).
int attn_splits(long groups, long tiles, long places, bool halve);

hipError_t launch_attn_forward(const AttnArgs& a, bool bf, hipStream_t stream);
hipError_t launch_attn_backward(const AttnArgs& a, bool bf, hipStream_t stream);

}  // namespace e2ttt
