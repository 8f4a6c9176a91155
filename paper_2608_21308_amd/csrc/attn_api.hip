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
      d->H % d->HK != 0 || !(d->scale >= 1.17549435e-38f) || !isfinite(d->scale * kLog2e))
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

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }
size_t rows_bytes(const e2ttt_attn_desc* d) { return up((size_t)d->B * d->H * d->T * 4); }

// How the workgroups of both directions are split, and the bytes that this takes.
struct Plan {
  int nsplit, nsplit_kv;
  size_t ml, forward, backward;
};
// Of n, those within reach of 128 neighbouring tokens.
long within(const e2ttt_attn_desc* d, long n) {
  return d->left < 0 || d->right < 0 ? n : std::min(n, (long)d->left + d->right + 128);
}
Plan plan(const e2ttt_attn_desc* d) {
  Plan p{};
  const long B = d->B, H = d->H, HK = d->HK, T = d->T, S = d->S;
  const bool bf = d->io == E2TTT_DT_BF16, small = bf && d->d <= 64;
  const long tile = attn_tile(bf, d->d), tile_kv = attn_tile_bwd(d->d);
  const long g = B * H * ((T + 127) / 128);
  const bool uneven = (d->left < 0) != (d->right < 0) && 2 * T > S;
  const auto halve = [&](long rows) { return uneven && rows * (bf ? 1 : 4) >= 2560; };
  p.nsplit = attn_splits(g, within(d, S) / tile, small || (bf && 256 / g * g < 208) ? 512 : 256, halve(S));
  p.nsplit_kv = attn_splits(B * HK * ((S + 127) / 128), H / HK * ((within(d, T) + tile_kv - 1) / tile_kv),
                            small ? 512 : 256, halve(H / HK * T));
  const size_t q = p.nsplit > 1 ? up((size_t)p.nsplit * B * H * T * d->d * 4) : 0;
  const size_t kv = p.nsplit_kv > 1 ? up((size_t)p.nsplit_kv * B * HK * S * d->d * 8) : 0;
  p.ml = q;
  p.forward = q ? q + up((size_t)p.nsplit * B * H * T * 8) : 0;
  p.backward = 2 * rows_bytes(d) + std::max(q, kv);
  return p;
}

AttnArgs args_of(const e2ttt_attn_desc* d, const int32_t* lengths) {
  AttnArgs a{};
  a.B = d->B; a.HK = d->HK; a.H = d->H; a.rep = d->H / d->HK; a.T = d->T; a.S = d->S; a.d = d->d;
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
  return check_desc(desc) == E2TTT_OK ? plan(desc).backward : 0;
}

extern "C" size_t e2ttt_attn_workspace_bytes(const e2ttt_attn_desc* desc) {
  return check_desc(desc) == E2TTT_OK ? plan(desc).forward : 0;
}

extern "C" e2ttt_status e2ttt_attn_forward(const e2ttt_attn_desc* desc,
                                           const e2ttt_attn_strides* strides, const void* q,
                                           const void* k, const void* v, const int32_t* lengths,
                                           void* out, float* lse, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  e2ttt_status st = check_desc(desc);
  if (st != E2TTT_OK) return st;
  const Plan p = plan(desc);
  if (!q || !k || !v || !out || (p.forward && !workspace)) return E2TTT_ERR_NULL_ARG;
  AttnArgs a = args_of(desc, lengths);
  const RowSpec qs{desc->B, desc->T, desc->d, desc->io}, ks{desc->B, desc->S, desc->d, desc->io};
  const e2ttt_attn_strides* s = strides;
  if (!qs.read(s ? &s->q : nullptr, q, desc->H, &a.q) ||
      !ks.read(s ? &s->k : nullptr, k, desc->HK, &a.k) ||
      !ks.read(s ? &s->v : nullptr, v, desc->HK, &a.v) ||
      !qs.write(s ? &s->out : nullptr, out, desc->H, &a.out) || misaligned(workspace))
    return E2TTT_ERR_BAD_SHAPE;
  if (workspace_bytes < p.forward) return E2TTT_ERR_WORKSPACE_TOO_SMALL;
  a.lse = lse;
  a.nsplit = p.nsplit;
  a.part = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + p.ml);
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
  const Plan p = plan(desc);
  if (scratch_bytes < p.backward) return E2TTT_ERR_WORKSPACE_TOO_SMALL;
  a.lse = const_cast<float*>(lse);
  a.d_lse = d_lse;
  a.ex = static_cast<float*>(scratch);
  a.delta = reinterpret_cast<float*>(static_cast<char*>(scratch) + rows_bytes(desc));
  a.nsplit = p.nsplit;
  a.nsplit_kv = p.nsplit_kv;
  a.part = reinterpret_cast<float*>(static_cast<char*>(scratch) + 2 * rows_bytes(desc));
  return launch_attn_backward(a, desc->io == E2TTT_DT_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? E2TTT_OK : E2TTT_ERR_HIP;
}
