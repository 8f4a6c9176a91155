// C entry points of the gated delta rule: argument checks, the layout of
// workspace and scratch, and the launches.
#include <math.h>

#include <algorithm>

#include "delta_common.h"
#include "e2ttt.h"
#include "strided.h"

namespace e2ttt {
namespace {

e2ttt_status check_desc(const e2ttt_delta_desc* d, bool save) {
  if (!d) return E2TTT_ERR_NULL_ARG;
  if (d->B <= 0 || d->HK <= 0 || d->H <= 0 || d->T <= 0 || d->dk <= 0 || d->dv <= 0 ||
      d->H % d->HK != 0 || !isfinite(d->scale))
    return E2TTT_ERR_BAD_SHAPE;
  if ((d->io != E2TTT_DT_F32 && d->io != E2TTT_DT_BF16) || d->dk % 8 || d->dv % 8 ||
      d->dk > 128 || d->dv > 256 || d->T > (1 << 30))
    return E2TTT_ERR_UNSUPPORTED;
  // a launch numbers its threads in 32 bits: at most 8 dvp (512) to a unit, and
  // where it takes every chunk at once 512 to a chunk
  const double units = (double)d->B * d->H, nc = ((double)d->T + kDC - 1) / kDC;
  if (units * std::max(512, 8 * delta_dvp(d->dv)) > 4e9 || units * nc > 1e9 ||
      (save && units * nc * 512 > 4e9))
    return E2TTT_ERR_UNSUPPORTED;
  return E2TTT_OK;
}

struct Plan {
  bool bf;
  long U, NC;
  long stretch;                   // chunks of a launch
  long nc_buf;                    // chunks whose gates and fragments are held (all, saving)
  long nseg, seglen;              // segments of a stretch
  long part;                      // chunks of a chain launch beside the next ones' preparation
  size_t o_gate, o_frag, o_state, o_segs, o_segb, o_segf, o_w, o_u, bytes;   // workspace
  size_t s_w, s_u, s_segs, s_segb, s_state, scratch;     // backward scratch
  long w_bytes, u_bytes;
};

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

// Gates and fragments of this many bytes are formed and used at a time.  What
// one launch writes the next reads from the 256 MB last-level cache while it
// is well below that (512 units of 64, 16 chunks: 267 us with 160 MB, 281 with 128,
// 299 at once); segments want long stretches instead, which they divide (16 units
// of 128, 512 chunks: 812 us at once, 902 in three).
constexpr size_t kCacheBytes = (size_t)160 << 20, kStretchBytes = (size_t)512 << 20;

// Segments that `nch` chunks of U units run as (1: none).  A wave holds 16 value
// channels of a unit, and the card takes 2048 such waves at once (`room`: how
// many times the units fit).  n segments take (nch / n) (t_state + t_chain) + n
// t_join, about 5 us and 1 us: least at n = sqrt(5 nch).
//
// They cost a pass over dv + dk channels ahead of the one over dv, so they pay
// where the units' own workgroups leave more than two thirds of the 256 CUs idle,
// three quarters with heads of 128, whose pass takes them twice over (a training
// step, with segments and without: 64 units of 64 x 64, 32 chunks, 275 us and 315; of
// 128 x 128 620 and 625, 128 chunks 2.25 ms and 2.42; 80 of 128, 32 chunks, 746 us and
// 687; 128 units of 64, 64 chunks, forward 407 and 352), and with bf16 where the
// chain is long beside what the pass adds to each of its workgroups (48 units of 128:
// 17 chunks 330 us and 300, 32 chunks 502 and 534; 80 of 64: 8 chunks 134 and 109, 17
// 206 and 197, 32 331 and 348; 64 of 64, 17 chunks, 181 and 185; 80 of 32: 8 chunks 92
// and 88, 17 135 and 153).  fp32 products are slower: four waves a workgroup at 128 too
// (32 units, 17 chunks: 467 us and 508; 48: 650 and 575), and short chains pay (48 units
// of 64, 8 chunks: 139 and 160; 80: 219 and 183).  Chains begin at 8 chunks with bf16 (32
// units of 64: 39 us and 41, 6 chunks 35 and 34), at 6 with fp32 (8 units of 64: 41 and 51).
long room(const e2ttt_delta_desc* d, long U) { return 2048 / (U * (delta_dvp(d->dv) / 16)); }
long segments(const e2ttt_delta_desc* d, long U, long nch) {
  const bool bf = d->io == E2TTT_DT_BF16;
  const int dkp = delta_dkp(d->dk), nw = bf && dkp > 64 ? 8 : 4;
  const long groups = U * ((delta_dvp(d->dv) / 16 + nw - 1) / nw);
  const long n = std::min(std::min(room(d, U), nch / 2), (long)sqrt(5.0 * nch));
  if (groups > (dkp > 64 ? 64 : 80) || groups > nch * (bf ? 256 / dkp : 8)) return 1;
  return n < 3 || nch < (bf ? 8 : 6) ? 1 : n;
}

// Chunks of a part (bf16, dk in 33..64): where the chain's workgroups leave CUs
// idle but are too many for segments, a launch takes a part of the chain beside
// the preparation of the next part, in the backward beside the gradients of the
// part before.  128 units of 64, 64 chunks: 329 us against 358, a training step
// 823 against 852 (96 units: 681 against 744, of 256 chunks 2.43 ms against 2.96;
// 192: 1169 us against 1161).  Launches cost some 10 us, so a part has 16 chunks at
// least (160 units, 64 chunks: 338 us, with parts of 8 399) and there are at most
// eight.
long part_of(const e2ttt_delta_desc* d, long U, long nch, long nseg) {
  const long groups = U * ((delta_dvp(d->dv) + 63) / 64);
  if (d->io != E2TTT_DT_BF16 || delta_dkp(d->dk) != 64 || nseg > 1 || nch < 32 || groups > 160)
    return nch;
  return std::max(16L, (nch + 7) / 8);
}

Plan plan(const e2ttt_delta_desc* d, bool save) {
  Plan p{};
  p.bf = d->io == E2TTT_DT_BF16;
  p.U = (long)d->B * d->H;
  p.NC = ((long)d->T + kDC - 1) / kDC;
  const int dkp = delta_dkp(d->dk), dvp = delta_dvp(d->dv);
  const size_t gate = kGateFloats * sizeof(float);
  const size_t frag = 2 * tri_bytes(p.bf);
  p.w_bytes = 4L * dkp * dvp;
  p.u_bytes = 4L * kDC * dvp;
  const size_t each = (gate + frag) * (size_t)p.U;
  p.nseg = segments(d, p.U, p.NC);
  const long fit = (long)((room(d, p.U) < 2 ? kCacheBytes : kStretchBytes) / each);
  const long n = fit < 1 ? p.NC : (p.NC + fit - 1) / fit;       // stretches of equal length
  p.stretch = (p.NC + n - 1) / n;
  if (save && room(d, p.U) >= 2) p.stretch = p.NC;
  p.nc_buf = save ? p.NC : p.stretch;
  if (p.nseg > 1) p.nseg = std::min(p.nseg, segments(d, p.U, p.stretch));
  p.seglen = (p.stretch + p.nseg - 1) / p.nseg;
  p.nseg = (p.stretch + p.seglen - 1) / p.seglen;
  p.part = part_of(d, p.U, p.stretch, p.nseg);
  const size_t carry = p.part < p.NC ? (size_t)p.U * d->dk * d->dv * 4 : 0;
  const size_t cus = (size_t)p.U * p.nc_buf;
  p.o_gate = 0;
  p.o_frag = up(p.o_gate + cus * gate);
  const size_t segs = p.nseg > 1 ? (size_t)p.U * p.nseg : 0;
  p.o_state = up(p.o_frag + cus * frag);
  p.o_segs = up(p.o_state + carry);
  p.o_segb = up(p.o_segs + segs * p.w_bytes);
  p.o_segf = up(p.o_segb + segs * p.w_bytes);
  p.o_w = up(p.o_segf + segs * 2 * dkp * dkp * 4);
  p.o_u = up(p.o_w + (save ? cus * p.w_bytes : 0));
  p.bytes = up(p.o_u + (save ? cus * p.u_bytes : 0));
  p.s_w = 0;
  p.s_u = up((size_t)p.U * p.NC * p.w_bytes);
  p.s_segs = up(p.s_u + (size_t)p.U * p.NC * p.u_bytes);
  p.s_segb = up(p.s_segs + segs * p.w_bytes);
  p.s_state = up(p.s_segb + segs * p.w_bytes);
  p.scratch = up(p.s_state + carry);
  return p;
}

struct Views {
  e2ttt_strides q, k, v, out, eta, gam, d_out, dq, dk, dv, deta, dgam;
};
e2ttt_status check_views(const e2ttt_delta_desc* d, const e2ttt_delta_strides* s, bool bwd,
                         bool gam, Views* o) {
  const long elt = d->io == E2TTT_DT_BF16 ? 2 : 4;
  const long B = d->B, HK = d->HK, H = d->H, T = d->T;
  o->q = strides_of(s ? &s->q : nullptr, HK, T, d->dk);
  o->k = strides_of(s ? &s->k : nullptr, HK, T, d->dk);
  o->v = strides_of(s ? &s->v : nullptr, H, T, d->dv);
  o->out = strides_of(s ? &s->out : nullptr, H, T, d->dv);
  o->eta = strides_of(s ? &s->eta : nullptr, H, T, 1);
  o->gam = strides_of(s ? &s->log_gamma : nullptr, H, T, 1);
  o->d_out = strides_of(s ? &s->d_out : nullptr, H, T, d->dv);
  o->dq = strides_of(s ? &s->dq : nullptr, HK, T, d->dk);
  o->dk = strides_of(s ? &s->dk : nullptr, HK, T, d->dk);
  o->dv = strides_of(s ? &s->dv : nullptr, H, T, d->dv);
  o->deta = strides_of(s ? &s->d_eta : nullptr, H, T, 1);
  o->dgam = strides_of(s ? &s->d_log_gamma : nullptr, H, T, 1);
  bool ok = rows_ok(o->q, elt, true) && rows_ok(o->k, elt, true) && rows_ok(o->v, elt, true) &&
            rows_ok(o->eta, 4, false) && (!gam || rows_ok(o->gam, 4, false));
  if (!bwd)
    ok = ok && rows_ok(o->out, elt, true) && disjoint(o->out, B, H, T, d->dv);
  else
    ok = ok && rows_ok(o->d_out, elt, true) && rows_ok(o->dq, elt, true) &&
         rows_ok(o->dk, elt, true) && rows_ok(o->dv, elt, true) && rows_ok(o->deta, 4, false) &&
         disjoint(o->dq, B, HK, T, d->dk) && disjoint(o->dk, B, HK, T, d->dk) &&
         disjoint(o->dv, B, H, T, d->dv) && disjoint(o->deta, B, H, T, 1) &&
         (!gam || (rows_ok(o->dgam, 4, false) && disjoint(o->dgam, B, H, T, 1)));
  return ok ? E2TTT_OK : E2TTT_ERR_BAD_SHAPE;
}

void fill(DeltaArgs& a, const e2ttt_delta_desc* d, const Plan& p, char* ws) {
  a.B = d->B; a.HK = d->HK; a.H = d->H; a.T = d->T;
  a.dk = d->dk; a.dv = d->dv; a.dvp = delta_dvp(d->dv);
  a.NC = (int)p.NC;
  a.nc_buf = (int)p.nc_buf;
  a.scale = d->scale;
  a.gate = reinterpret_cast<float*>(ws + p.o_gate);
  a.frag = ws + p.o_frag;
  a.segs = reinterpret_cast<float*>(ws + p.o_segs);
  a.segb = reinterpret_cast<float*>(ws + p.o_segb);
  a.segf = reinterpret_cast<float*>(ws + p.o_segf);
  a.seglen = (int)p.seglen;
  a.wst = reinterpret_cast<float*>(ws + p.o_w);
  a.ust = reinterpret_cast<float*>(ws + p.o_u);
}

}  // namespace
}  // namespace e2ttt

using namespace e2ttt;

extern "C" size_t e2ttt_delta_workspace_bytes(const e2ttt_delta_desc* desc, int save_for_backward) {
  const bool save = save_for_backward != 0;
  return check_desc(desc, save) == E2TTT_OK ? plan(desc, save).bytes : 0;
}

extern "C" size_t e2ttt_delta_scratch_bytes(const e2ttt_delta_desc* desc) {
  return check_desc(desc, true) == E2TTT_OK ? plan(desc, true).scratch : 0;
}

extern "C" e2ttt_status e2ttt_delta_forward(const e2ttt_delta_desc* desc,
                                            const e2ttt_delta_strides* strides, const void* q,
                                            const void* k, const void* v, const float* eta,
                                            const float* log_gamma, const int32_t* lengths,
                                            const float* w_in, void* out, float* w_out,
                                            void* workspace, size_t workspace_bytes,
                                            int save_for_backward, void* stream) {
  e2ttt_status st = check_desc(desc, save_for_backward != 0);
  if (st != E2TTT_OK) return st;
  if (!q || !k || !v || !eta || !out || !workspace) return E2TTT_ERR_NULL_ARG;
  Views vw;
  if ((st = check_views(desc, strides, false, log_gamma != nullptr, &vw)) != E2TTT_OK) return st;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(w_in) ||
      misaligned(w_out) || misaligned(workspace))
    return E2TTT_ERR_BAD_SHAPE;
  const bool save = save_for_backward != 0;
  const Plan p = plan(desc, save);
  if (workspace_bytes < p.bytes) return E2TTT_ERR_WORKSPACE_TOO_SMALL;
  char* ws = static_cast<char*>(workspace);
  DeltaArgs a{};
  fill(a, desc, p, ws);
  a.save = save;
  a.q = view(q, vw.q); a.k = view(k, vw.k); a.v = view(v, vw.v); a.out = view(out, vw.out);
  a.eta = view(eta, vw.eta); a.gam = view(log_gamma, vw.gam);
  a.lengths = lengths;
  float* carry = reinterpret_cast<float*>(ws + p.o_state);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  for (long r0 = 0; r0 < p.NC; r0 += p.stretch) {
    const long r1 = std::min(r0 + p.stretch, p.NC);
    a.r_base = save ? 0 : (int)r0;
    a.r0 = (int)r0;
    a.r1 = (int)std::min(r0 + p.part, r1);
    if (launch_delta_prep(a, p.bf, s) != hipSuccess) return E2TTT_ERR_HIP;
    for (; a.r0 < r1; a.r0 = a.r1) {
      a.r1 = (int)std::min(a.r0 + p.part, r1);
      a.w_in = a.r0 == 0 ? w_in : carry;
      a.w_out = a.r1 == p.NC ? w_out : carry;
      a.nseg = (a.r1 - a.r0 + a.seglen - 1) / a.seglen;  // (the last stretch may be shorter)
      if (a.nseg > 1 && (launch_delta_chain(a, p.bf, false, true, s) != hipSuccess ||
                         launch_delta_join(a, p.bf, false, s) != hipSuccess))
        return E2TTT_ERR_HIP;
      const int next = (int)std::min(p.part, r1 - a.r1);
      if ((next ? launch_delta_chain_prep(a, save, a.r1, next, s)
                : launch_delta_chain(a, p.bf, save, false, s)) != hipSuccess)
        return E2TTT_ERR_HIP;
    }
  }
  return E2TTT_OK;
}

extern "C" e2ttt_status e2ttt_delta_backward(
    const e2ttt_delta_desc* desc, const e2ttt_delta_strides* strides, const void* q, const void* k,
    const void* v, const float* eta, const float* log_gamma, const int32_t* lengths,
    const void* workspace, size_t workspace_bytes, const void* d_out, const float* d_w_out,
    void* dq, void* dk, void* dv, float* d_eta, float* d_log_gamma, float* d_w_in, void* scratch,
    size_t scratch_bytes, void* stream) {
  e2ttt_status st = check_desc(desc, true);
  if (st != E2TTT_OK) return st;
  if (!q || !k || !v || !eta || !workspace || !d_out || !dq || !dk || !dv || !d_eta || !scratch)
    return E2TTT_ERR_NULL_ARG;
  if ((log_gamma == nullptr) != (d_log_gamma == nullptr)) return E2TTT_ERR_NULL_ARG;
  Views vw;
  if ((st = check_views(desc, strides, true, log_gamma != nullptr, &vw)) != E2TTT_OK) return st;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(d_out) || misaligned(dq) ||
      misaligned(dk) || misaligned(dv) || misaligned(d_w_out) || misaligned(d_w_in) ||
      misaligned(workspace) || misaligned(scratch))
    return E2TTT_ERR_BAD_SHAPE;
  const Plan p = plan(desc, true);
  if (workspace_bytes < p.bytes || scratch_bytes < p.scratch) return E2TTT_ERR_WORKSPACE_TOO_SMALL;
  DeltaArgs a{};
  fill(a, desc, p, static_cast<char*>(const_cast<void*>(workspace)));
  a.q = view(q, vw.q); a.k = view(k, vw.k); a.v = view(v, vw.v);
  a.eta = view(eta, vw.eta); a.gam = view(log_gamma, vw.gam);
  a.d_out = view(d_out, vw.d_out);
  a.dq = view(dq, vw.dq); a.dkk = view(dk, vw.dk); a.dv_ = view(dv, vw.dv);
  a.deta = view(d_eta, vw.deta); a.dgam = view(d_log_gamma, vw.dgam);
  a.lengths = lengths;
  a.dwst = reinterpret_cast<float*>(static_cast<char*>(scratch) + p.s_w);
  a.yst = reinterpret_cast<float*>(static_cast<char*>(scratch) + p.s_u);
  a.segs = reinterpret_cast<float*>(static_cast<char*>(scratch) + p.s_segs);
  a.segb = reinterpret_cast<float*>(static_cast<char*>(scratch) + p.s_segb);
  a.r_base = 0;
  if (p.stretch < p.NC) a.seglen = (int)p.NC;   // (no segments)
  float* carry = reinterpret_cast<float*>(static_cast<char*>(scratch) + p.s_state);
  const long part = p.part < p.stretch ? p.part : p.NC;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  for (a.r1 = (int)p.NC; a.r1 > 0; a.r1 = a.r0) {
    a.r0 = (int)std::max(a.r1 - part, 0L);
    a.d_w_out = a.r1 == p.NC ? d_w_out : carry;
    a.d_w_in = a.r0 == 0 ? d_w_in : carry;
    a.nseg = (a.r1 - a.r0 + a.seglen - 1) / a.seglen;
    if (a.nseg > 1 && (launch_delta_chain_bwd(a, p.bf, true, s) != hipSuccess ||
                       launch_delta_join(a, p.bf, true, s) != hipSuccess))
      return E2TTT_ERR_HIP;
    const int done = (int)std::min(part, p.NC - a.r1);
    if ((done ? launch_delta_chain_bwd_grads(a, a.r1, done, s)
              : launch_delta_chain_bwd(a, p.bf, false, s)) != hipSuccess)
      return E2TTT_ERR_HIP;
  }
  a.r1 = (int)((p.NC - 1) % part) + 1;          // the gradients of the last launch's chunks
  if (launch_delta_grads(a, p.bf, s) != hipSuccess) return E2TTT_ERR_HIP;
  return E2TTT_OK;
}

extern "C" e2ttt_status e2ttt_delta_step(const e2ttt_delta_desc* desc,
                                         const e2ttt_delta_strides* strides, const void* q,
                                         const void* k, const void* v, const float* eta,
                                         const float* log_gamma, float* w, const int32_t* slots,
                                         int32_t n_slots, void* out, void* stream) {
  e2ttt_status st = check_desc(desc, false);
  if (st != E2TTT_OK) return st;
  if (!q || !k || !v || !eta || !w || !out) return E2TTT_ERR_NULL_ARG;
  if (n_slots <= 0 || (!slots && n_slots < desc->B)) return E2TTT_ERR_BAD_SHAPE;
  Views vw;
  if ((st = check_views(desc, strides, false, log_gamma != nullptr, &vw)) != E2TTT_OK) return st;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(w))
    return E2TTT_ERR_BAD_SHAPE;
  DeltaStepArgs a{};
  a.q = view(q, vw.q); a.k = view(k, vw.k); a.v = view(v, vw.v); a.out = view(out, vw.out);
  a.eta = view(eta, vw.eta); a.gam = view(log_gamma, vw.gam);
  a.w = w; a.slots = slots; a.nslots = n_slots;
  a.B = desc->B; a.HK = desc->HK; a.H = desc->H; a.T = desc->T;
  a.dk = desc->dk; a.dv = desc->dv; a.scale = desc->scale;
  return launch_delta_step(a, desc->io == E2TTT_DT_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? E2TTT_OK : E2TTT_ERR_HIP;
}
