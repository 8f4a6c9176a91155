// Gated delta rule, recurrent form: a few arriving tokens of every sequence
// update its state and are answered from it, in fp32 on the fp32 state:
//   Wd = exp(g) W,  e = v - Wd k,  W = Wd + eta e k^T,  o = s W q.
// Bound by HBM: a state of 4 dk dv bytes is read once and written once,
// whatever the number of tokens.  Rows of W (value channels) do not meet, so
// the state is dealt out by rows: LPR lanes hold a row as float4 pieces (a wave
// reads whole rows of 64 / LPR channels per load) and sum their partial dots
// by DPP.  A wave takes RS row sets, all loaded before the first is used.
// 128 sequences of 32 heads of 128 x 128: 540 MB in 90 us, 6 TB/s (a part still
// lies in the last-level cache; a large copy reaches 5.2); 8 sequences of 16
// heads of 64 x 64: 4.8 us, which is the launch.
#include "delta_common.h"

namespace e2ttt {

namespace {

template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp_f<0xB1>(v);
  v += dpp_f<0x4E>(v);
  if constexpr (L >= 8) v += dpp_f<0x141>(v);
  return v;
}

template <bool BF, int DK, int RS>
__global__ void __launch_bounds__(256) delta_step_kernel(DeltaStepArgs a, int nblk) {
  using E = typename DOp<BF>::E;
  constexpr int LPR = DK >= 64 ? 8 : 4;     // lanes of a row
  constexpr int NQ = DK / (4 * LPR);        // float4 pieces of a row in a lane
  constexpr int RW = 64 / LPR;              // rows of a set in a wave
  typedef __attribute__((ext_vector_type(4))) E Q;
  const int lane = threadIdx.x & 63, w = wave_id();
  const long bh = blockIdx.x / nblk;
  const int b = (int)(bh / a.H), h = (int)(bh % a.H), hk = h / (a.H / a.HK);
  const int row0 = ((int)(blockIdx.x % nblk) * 4 + w) * RW * RS + lane / LPR;
  const int l = lane % LPR;

  // a token's operands, on their way one token ahead
  Q rk[NQ], rq[NQ];
  E rv[RS];
  float re, rg;
  auto load = [&](int bb, int t) {
    const E* kp = row_of<E>(a.k, bb, hk, t);
    const E* qp = row_of<E>(a.q, bb, hk, t);
    const E* vp = row_of<E>(a.v, bb, h, t);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int col = 4 * (j * LPR + l);
      rk[j] = rq[j] = Q{};
      if (col < a.dk) {
        rk[j] = *reinterpret_cast<const Q*>(kp + col);
        rq[j] = *reinterpret_cast<const Q*>(qp + col);
      }
    }
#pragma unroll
    for (int x = 0; x < RS; ++x) rv[x] = row0 + x * RW < a.dv ? vp[row0 + x * RW] : (E)0.0f;
    re = *row_of<float>(a.eta, bb, h, t);
    rg = a.gam.p ? *row_of<float>(a.gam, bb, h, t) : 0.0f;
  };
  load(b, 0);

  long slot = b;
  bool more = false;
  if (a.slots) {
    // requests that share a slot are taken in the order of their rows by the
    // workgroups of the first of them
    const int s = a.slots[b];
    slot = s;
    if (s < 0 || s >= a.nslots) {           // no state: zero outputs
      for (int t = 0; t < a.T; ++t)
#pragma unroll
        for (int x = 0; x < RS; ++x)
          if (l == 0 && row0 + x * RW < a.dv)
            row_of_w<E>(a.out, b, h, t)[row0 + x * RW] = (E)0.0f;
      return;
    }
    unsigned long before = 0, after = 0;
    for (int x = 0; x < a.B; x += 64) {
      const int y = x + lane;
      const bool eq = y < a.B && a.slots[y] == s;
      before |= __ballot(eq && y < b);
      after |= __ballot(eq && y > b);
    }
    if (before) return;
    more = after != 0;
  }

  float* wp = a.w + (slot * a.H + h) * (long)a.dv * a.dk;
  f32x4 st[RS][NQ];
#pragma unroll
  for (int x = 0; x < RS; ++x)
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int row = row0 + x * RW, col = 4 * (j * LPR + l);
      st[x][j] = zero4();
      if (row < a.dv && col < a.dk)
        st[x][j] = *reinterpret_cast<const f32x4*>(wp + (long)row * a.dk + col);
    }

  for (int bb = b;;) {
    int nb = a.B;                           // the next row of the batch at this slot
    if (more)
      for (nb = bb + 1; nb < a.B && a.slots[nb] != (int)slot;) ++nb;
    for (int t = 0; t < a.T; ++t) {
      f32x4 kv[NQ], qv[NQ];
      float vv[RS];
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          kv[j][e] = (float)rk[j][e];
          qv[j][e] = (float)rq[j][e];
        }
#pragma unroll
      for (int x = 0; x < RS; ++x) vv[x] = (float)rv[x];
      const float eta = re, gm = a.gam.p ? expf(rg) : 1.0f;
      if (t + 1 < a.T)
        load(bb, t + 1);
      else if (nb < a.B)
        load(nb, 0);
#pragma unroll
      for (int x = 0; x < RS; ++x) {
        float d = 0.0f;
#pragma unroll
        for (int j = 0; j < NQ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            st[x][j][e] *= gm;
            d = fmaf(st[x][j][e], kv[j][e], d);
          }
        const float u = eta * (vv[x] - lanes_sum<LPR>(d));
        float o = 0.0f;
#pragma unroll
        for (int j = 0; j < NQ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            st[x][j][e] = fmaf(u, kv[j][e], st[x][j][e]);
            o = fmaf(st[x][j][e], qv[j][e], o);
          }
        o = lanes_sum<LPR>(o);
        const int row = row0 + x * RW;
        if (l == 0 && row < a.dv) row_of_w<E>(a.out, bb, h, t)[row] = (E)(a.scale * o);
      }
    }
    if (nb >= a.B) break;
    bb = nb;
  }
#pragma unroll
  for (int x = 0; x < RS; ++x)
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int row = row0 + x * RW, col = 4 * (j * LPR + l);
      if (row < a.dv && col < a.dk)
        st_stream(reinterpret_cast<f32x4*>(wp + (long)row * a.dk + col), st[x][j]);
    }
}

template <bool BF, int DK, int RS>
hipError_t go(const DeltaStepArgs& a, hipStream_t s) {
  const int per = 4 * (DK >= 64 ? 8 : 16) * RS;     // rows of a workgroup
  const int nblk = (a.dv + per - 1) / per;
  hipLaunchKernelGGL((delta_step_kernel<BF, DK, RS>), dim3((unsigned)((long)a.B * a.H * nblk)),
                     dim3(256), 0, s, a, nblk);
  return hipGetLastError();
}

template <bool BF>
hipError_t pick(const DeltaStepArgs& a, hipStream_t s) {
  if (a.dk <= 16) return go<BF, 16, 1>(a, s);
  if (a.dk <= 32) return go<BF, 32, 1>(a, s);
  if (a.dk <= 64) return go<BF, 64, 2>(a, s);   // (two rows of 256 bytes a lane, one of 512)
  return go<BF, 128, 1>(a, s);
}

}  // namespace

hipError_t launch_delta_step(const DeltaStepArgs& a, bool bf, hipStream_t s) {
  return bf ? pick<true>(a, s) : pick<false>(a, s);
}

}  // namespace e2ttt
