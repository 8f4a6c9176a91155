// Shared pieces of the 4-bit cache kernels (cache_*.hip).
//
// A row of d elements is held as codes of 4 bits (sign, two exponent bits, one of
// mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) times a power of two for each block of 32:
// the least one that leaves the block's elements at most 7, so that nothing is off
// by more than half a step of its neighbours, the top's included (7 goes to 6).  The
// hardware converts between such codes and bf16 or fp32, rounding to nearest, ties
// to even; every value is exact in bf16.
//
// A page holds 64 tokens of one key head, NB = d / 32, in the order in which the
// attention's lanes take it (16 x 16 x 32 products, lane (g, r) = (lane / 16, lane
// mod 16)), each part in whole loads of a lane:
//   K codes   [64 tokens][4 g][NB][4]     channels 32 blk + 8 g + 2 byte, + 1 (high half)
//   K scales  [NB][16 r][4 a]             token 16 a + r: the four row tiles of a lane
//   V codes   [NB][16 r][4 g][4 a][4 i]   token 16 a + 4 g + i, channels 32 blk + 2 r, + 1
//   V scales  [NB][4 g][4 a][4 i]
// V's bytes pair two channels of one token, so that no byte has two writers and two
// tokens' pairs become two channels' pairs by one permutation.  The scores' accumulator
// holds tokens 16 a + 4 g + i in lane group g, which is how V lies.
#pragma once

#include "delta_common.h"
#include "div.h"

namespace e2ttt {

constexpr int kPage = 64;            // tokens of a page
constexpr int kMinExp = 2;           // least scale byte: every value but zero is a normal number
constexpr int kNanExp = 255;         // of a block with a non-finite element: reads as NaN

struct CacheArgs {
  View x, y;                // k, v; q, out for attention: [B][HK or H][T][d]
  float* lse;               // [B][H][T], nullable
  const int* starts;        // [B]: position of a sequence's first token of this call
  const int* lengths;       // nullable
  const int* table;         // [B][P]
  unsigned char* cache;     // [n_pages][HK][68 d]
  float* part;              // attention: partial results
  long n_pages;
  int B, HK, H, T, d, P;
  int left;                 // negative: no bound
  int nsplit;
  Div by_split, by_tile, by_HK, by_rep, by_P;   // attention: of the workgroup's number, of columns, pages
  float scale;
};

// What a sequence holds once the call's tokens are in: positions first .. end - 1.
struct Held {
  long start, end, first;
};
__device__ __forceinline__ Held held_of(const CacheArgs& a, int b) {
  Held x;
  const int live = a.lengths ? max(0, min(a.T, a.lengths[b])) : a.T;
  x.start = a.starts ? a.starts[b] : 0;
  x.end = x.start + live;
  x.first = x.end <= 0 ? 0 : max(0L, ((x.end - 1) / kPage - a.P + 1) * kPage);
  return x;
}
// The page that entry e of a sequence's row of the table names (null: none).
__device__ __forceinline__ unsigned char* page_at(const CacheArgs& a, int b, int hk, int e) {
  const int id = a.table[(long)b * a.P + e];
  if (id < 0 || id >= a.n_pages) return nullptr;
  return a.cache + ((long)id * a.HK + hk) * (68L * a.d);
}

// Byte i of a word of scales, as the factor of the hardware's conversions: of that
// float they take the exponent's bits alone (255: NaN).
template <int I>
__device__ __forceinline__ float scale_of(unsigned w) {
  return __uint_as_float(I == 3 ? w >> 1 : w << (23 - 8 * I));
}

hipError_t launch_cache_write(const CacheArgs& a, bool bf, hipStream_t stream);
hipError_t launch_cache_read(const CacheArgs& a, bool bf, hipStream_t stream);
hipError_t launch_cache_attend(const CacheArgs& a, bool bf, hipStream_t stream);
// Stretches that the keys of a key head are split into, and floats of the partial results.
int cache_splits(const CacheArgs& a);
size_t cache_part_floats(const CacheArgs& a);

}  // namespace e2ttt
