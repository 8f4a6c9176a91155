// C entry points of the 4-bit cache: argument checks and the launches.
#include <math.h>

#include <algorithm>

#include "cache_common.h"
#include "e2ttt.h"
#include "strided.h"

namespace e2ttt {
namespace {

// A launch numbers its threads in 32 bits: 256 to a workgroup that writes or reads, 512 to
// one that attends.
constexpr double kMostRowGroups = 0xffffff, kMostGroups = 0x7fffff;

CacheArgs args_of(const e2ttt_cache_desc* d) {
  CacheArgs a{};
  a.B = d->B; a.HK = d->HK; a.H = d->H; a.T = d->T; a.d = d->d; a.P = d->pages;
  a.left = d->left;
  a.scale = d->scale;
  return a;
}

e2ttt_status check_desc(const e2ttt_cache_desc* d, bool attend) {
  if (!d) return E2TTT_ERR_NULL_ARG;
  if (d->B <= 0 || d->HK <= 0 || d->T <= 0 || d->d <= 0 || d->pages <= 0) return E2TTT_ERR_BAD_SHAPE;
  if (attend && (d->H <= 0 || d->H % d->HK != 0 || !(d->scale >= 1.17549435e-38f) ||
                 !isfinite(d->scale * 1.44269504f)))
    return E2TTT_ERR_BAD_SHAPE;
  if ((d->io != E2TTT_DT_F32 && d->io != E2TTT_DT_BF16) || d->d % 32 || d->d > 128 ||
      d->T > (1 << 29) || d->pages > (1 << 25))
    return E2TTT_ERR_UNSUPPORTED;
  const double rows = (double)d->B * d->HK;
  if (rows * ((d->T + 2) / 4 + 1) * (d->d / 8) > 256 * kMostRowGroups) return E2TTT_ERR_UNSUPPORTED;
  if (attend) {
    const double tiles = ((double)(d->H / d->HK) * d->T + 15) / 16;
    if (rows * tiles > kMostGroups || tiles * 16 > (1 << 30) ||
        rows * (int)tiles * cache_splits(args_of(d)) > kMostGroups)
      return E2TTT_ERR_UNSUPPORTED;
  }
  return E2TTT_OK;
}

// What every call has: pages and where the sequences stand.
e2ttt_status common(const int32_t* starts, const int32_t* lengths, const int32_t* table,
                    const void* cache, int32_t n_pages, CacheArgs* a) {
  if (!table || !cache) return E2TTT_ERR_NULL_ARG;
  if (n_pages <= 0 || misaligned(cache)) return E2TTT_ERR_BAD_SHAPE;
  a->starts = starts;
  a->lengths = lengths;
  a->table = table;
  a->cache = static_cast<unsigned char*>(const_cast<void*>(cache));
  a->n_pages = n_pages;
  return E2TTT_OK;
}

size_t part_bytes(const CacheArgs& a) { return cache_part_floats(a) * sizeof(float); }

}  // namespace
}  // namespace e2ttt

using namespace e2ttt;

extern "C" size_t e2ttt_cache_page_bytes(int32_t HK, int32_t d) {
  return HK <= 0 || d <= 0 || d % 32 || d > 128 ? 0 : (size_t)HK * 68 * d;
}

extern "C" size_t e2ttt_cache_workspace_bytes(const e2ttt_cache_desc* desc) {
  return check_desc(desc, true) == E2TTT_OK ? std::max<size_t>(part_bytes(args_of(desc)), 256) : 0;
}

extern "C" e2ttt_status e2ttt_cache_write(const e2ttt_cache_desc* desc,
                                          const e2ttt_cache_strides* strides, const void* k,
                                          const void* v, const int32_t* starts,
                                          const int32_t* lengths, const int32_t* table, void* cache,
                                          int32_t n_pages, void* stream) {
  e2ttt_status st = check_desc(desc, false);
  if (st != E2TTT_OK) return st;
  CacheArgs a = args_of(desc);
  if (!k || !v) return E2TTT_ERR_NULL_ARG;
  if ((st = common(starts, lengths, table, cache, n_pages, &a)) != E2TTT_OK) return st;
  const RowSpec rows{desc->B, desc->T, desc->d, desc->io};
  if (!rows.read(strides ? &strides->k : nullptr, k, desc->HK, &a.x) ||
      !rows.read(strides ? &strides->v : nullptr, v, desc->HK, &a.y))
    return E2TTT_ERR_BAD_SHAPE;
  return launch_cache_write(a, desc->io == E2TTT_DT_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? E2TTT_OK : E2TTT_ERR_HIP;
}

extern "C" e2ttt_status e2ttt_cache_read(const e2ttt_cache_desc* desc,
                                         const e2ttt_cache_strides* strides, const int32_t* starts,
                                         const int32_t* lengths, const int32_t* table,
                                         const void* cache, int32_t n_pages, void* k, void* v,
                                         void* stream) {
  e2ttt_status st = check_desc(desc, false);
  if (st != E2TTT_OK) return st;
  CacheArgs a = args_of(desc);
  if (!k || !v) return E2TTT_ERR_NULL_ARG;
  if ((st = common(starts, lengths, table, cache, n_pages, &a)) != E2TTT_OK) return st;
  const RowSpec rows{desc->B, desc->T, desc->d, desc->io};
  if (!rows.write(strides ? &strides->k : nullptr, k, desc->HK, &a.x) ||
      !rows.write(strides ? &strides->v : nullptr, v, desc->HK, &a.y))
    return E2TTT_ERR_BAD_SHAPE;
  return launch_cache_read(a, desc->io == E2TTT_DT_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? E2TTT_OK : E2TTT_ERR_HIP;
}

extern "C" e2ttt_status e2ttt_cache_attend(const e2ttt_cache_desc* desc,
                                           const e2ttt_cache_strides* strides, const void* q,
                                           const int32_t* starts, const int32_t* lengths,
                                           const int32_t* table, const void* cache, int32_t n_pages,
                                           void* out, float* lse, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  e2ttt_status st = check_desc(desc, true);
  if (st != E2TTT_OK) return st;
  CacheArgs a = args_of(desc);
  if (!q || !out || !workspace) return E2TTT_ERR_NULL_ARG;
  if ((st = common(starts, lengths, table, cache, n_pages, &a)) != E2TTT_OK) return st;
  const RowSpec rows{desc->B, desc->T, desc->d, desc->io};
  if (!rows.read(strides ? &strides->q : nullptr, q, desc->H, &a.x) ||
      !rows.write(strides ? &strides->out : nullptr, out, desc->H, &a.y) || misaligned(workspace))
    return E2TTT_ERR_BAD_SHAPE;
  if (workspace_bytes < std::max<size_t>(part_bytes(a), 256)) return E2TTT_ERR_WORKSPACE_TOO_SMALL;
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  a.nsplit = cache_splits(a);
  return launch_cache_attend(a, desc->io == E2TTT_DT_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? E2TTT_OK : E2TTT_ERR_HIP;
}
