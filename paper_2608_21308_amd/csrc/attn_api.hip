// C entry points of attention: argument checks and the launches.
#include <math.h>

#include <algorithm>

#include "attn_common.h"
#include "e2ttt.h"
#include "strided.h"

namespace e2ttt {
namespace {

// (a launch numbers its threads in 32 bits: 256 to a tile of 128 queries or keys)
constexpr long kMostTiles = 0xffffff;

e2ttt_status check_desc(const e2ttt_attn_desc* d) {
  if (!d) return E2TTT_ERR_NULL_ARG;
  if (d->B <= 0 || d->HK <= 0 || d->H <= 0 || d->T <= 0 || d->S <= 0 || d->d <= 0 ||
      d->H % d->HK != 0 || !(d->scale > 0.0f) || !isfinite(d->scale * kLog2e))
    return E2TTT_ERR_BAD_SHAPE;
  if ((d->io != E2TTT_DT_F32 && d->io != E2TTT_DT_BF16) || d->d % 8 || d->d > 128 ||
      d->T > (1 << 29) || d->S > (1 << 29))
    return E2TTT_ERR_UNSUPPORTED;
  const double units = (double)d->B * d->H;
  if (units * (((long)d->T + 127) / 128) > kMostTiles ||
      (double)d->B * d->HK * (((long)d->S + 127) / 128) > kMostTiles)
    return E2TTT_ERR_UNSUPPORTED;
  return E2TTT_OK;
}

size_t rows_bytes(const e2ttt_attn_desc* d) {
  return ((size_t)d->B * d->H * d->T * 4 + 255) & ~(size_t)255;
}

AttnArgs args_of(const e2ttt_attn_desc* d, const int32_t* lengths) {
  AttnArgs a{};
  a.B = d->B; a.HK = d->HK; a.H = d->H; a.T = d->T; a.S = d->S; a.d = d->d;
  a.left = std::min(d->left, (1 << 30) - 1);
  a.right = std::min(d->right, (1 << 30) - 1);
  a.scale = d->scale;
  a.lengths = lengths;
  return a;
}

}  // namespace
}  // namespace e2ttt

using namespace e2ttt;

extern "C" size_t e2ttt_attn_scratch_bytes(const e2ttt_attn_desc* desc) {
  return check_desc(desc) == E2TTT_OK ? 2 * rows_bytes(desc) : 0;
}

extern "C" e2ttt_status e2ttt_attn_forward(const e2ttt_attn_desc* desc,
                                           const e2ttt_attn_strides* strides, const void* q,
                                           const void* k, const void* v, const int32_t* lengths,
                                           void* out, float* lse, void* stream) {
  e2ttt_status st = check_desc(desc);
  if (st != E2TTT_OK) return st;
  if (!q || !k || !v || !out) return E2TTT_ERR_NULL_ARG;
  AttnArgs a = args_of(desc, lengths);
  const RowSpec qs{desc->B, desc->T, desc->d, desc->io}, ks{desc->B, desc->S, desc->d, desc->io};
  const e2ttt_attn_strides* s = strides;
  if (!qs.read(s ? &s->q : nullptr, q, desc->H, &a.q) ||
      !ks.read(s ? &s->k : nullptr, k, desc->HK, &a.k) ||
      !ks.read(s ? &s->v : nullptr, v, desc->HK, &a.v) ||
      !qs.write(s ? &s->out : nullptr, out, desc->H, &a.out))
    return E2TTT_ERR_BAD_SHAPE;
  a.lse = lse;
  return launch_attn_forward(a, desc->io == E2TTT_DT_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? E2TTT_OK : E2TTT_ERR_HIP;
}

extern "C" e2ttt_status e2ttt_attn_backward(const e2ttt_attn_desc* desc,
                                            const e2ttt_attn_strides* strides, const void* q,
                                            const void* k, const void* v, const int32_t* lengths,
                                            const void* out, const float* lse, const void* d_out,
                                            const float* d_lse, void* dq, void* dk, void* dv,
                                            void* scratch, size_t scratch_bytes, void* stream) {
  e2ttt_status st = check_desc(desc);
  if (st != E2TTT_OK) return st;
  if (!q || !k || !v || !out || !lse || !d_out || !dq || !dk || !dv || !scratch)
    return E2TTT_ERR_NULL_ARG;
  AttnArgs a = args_of(desc, lengths);
  const RowSpec qs{desc->B, desc->T, desc->d, desc->io}, ks{desc->B, desc->S, desc->d, desc->io};
  const e2ttt_attn_strides* s = strides;
  if (!qs.read(s ? &s->q : nullptr, q, desc->H, &a.q) ||
      !ks.read(s ? &s->k : nullptr, k, desc->HK, &a.k) ||
      !ks.read(s ? &s->v : nullptr, v, desc->HK, &a.v) ||
      !qs.read(s ? &s->out : nullptr, out, desc->H, &a.out) ||
      !qs.read(s ? &s->d_out : nullptr, d_out, desc->H, &a.d_out) ||
      !qs.write(s ? &s->dq : nullptr, dq, desc->H, &a.dq) ||
      !ks.write(s ? &s->dk : nullptr, dk, desc->HK, &a.dk) ||
      !ks.write(s ? &s->dv : nullptr, dv, desc->HK, &a.dv) || misaligned(scratch))
    return E2TTT_ERR_BAD_SHAPE;
  if (scratch_bytes < 2 * rows_bytes(desc)) return E2TTT_ERR_WORKSPACE_TOO_SMALL;
  a.lse = const_cast<float*>(lse);
  a.d_lse = d_lse;
  a.ex = static_cast<float*>(scratch);
  a.delta = reinterpret_cast<float*>(static_cast<char*>(scratch) + rows_bytes(desc));
  return launch_attn_backward(a, desc->io == E2TTT_DT_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? E2TTT_OK : E2TTT_ERR_HIP;
}
