// Channel attention over parts of a long context: a window of the cache with a few first slots
// (wm_channel_attend_window), a prefix that the batch shares next to each sequence's own
// cache (wm_channel_attend_shared), and attention that adds up the weight each slot receives
// (wm_channel_attend_weigh).
//
// Row (l, b, h, i) sits at position t = ctx_len[b] + gq + gs i; with lim = t (paper mask) or
// t + 1 (inclusive) it reads every prefix slot, and the cache slots s < lim with s >= lim -
// window or s < sinks. First form: one wave per row, the head dimension across its lanes.
#include <algorithm>

#include "wm_device.hpp"
#include "wm_internal.hpp"

namespace wm {

template <typename T> struct ReachArgs {
  const T *Q, *Kc, *Vc, *Kd, *Vd;
  const T *Kp, *Vp;  // [k][Hkv][P_cap][d], the shared prefix (P slots)
  const int32_t* ctx_len;
  T* O;
  float* lse;  // [L][B][Hq][T_new], log2 units, or null
  int B, T_new, L, Hq, Hkv, S_cap, P, P_cap, window, sinks, mask_paper;
  int gs, gq, ctx_hi;
  float scale_log2;
  LayerTable chan;
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void reach_rows_kernel(ReachArgs<T> a) {
  constexpr int E = (DH + 63) / 64;
  const long rows = (long)a.L * a.B * a.Hq * a.T_new;
  const long rid = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (rid >= rows) return;
  const int i = (int)(rid % a.T_new), hq = (int)(rid / a.T_new % a.Hq);
  const int b = (int)(rid / a.T_new / a.Hq % a.B), l = (int)(rid / a.T_new / a.Hq / a.B);
  const int c = a.chan.v[l], kvh = hq / (a.Hq / a.Hkv);
  const int lim = min(ctx_at(a.ctx_len, b, a.ctx_hi) + a.gq + a.gs * i + (a.mask_paper ? 0 : 1),
                      a.S_cap);
  const int lo = max(lim - a.window, 0), na = min(a.sinks, lo);
  float q[E], o[E], m = kNegBig, sum = 0.f;
  for (int e = 0; e < E; ++e) {
    q[e] = 64 * e + lane < DH ? to_f32(a.Q[rid * DH + 64 * e + lane]) * a.scale_log2 : 0.f;
    o[e] = 0.f;
  }
  auto slot = [&](const T* kr, const T* vr) {
    float part = 0.f;
    for (int e = 0; e < E; ++e)
      if (64 * e + lane < DH) part += q[e] * to_f32(kr[64 * e + lane]);
    const float sc = wave_sum(part), mn = fmaxf(m, sc);
    const float f = fast_exp2(m - mn), p = fast_exp2(sc - mn);
    sum = sum * f + p;
    for (int e = 0; e < E; ++e)
      o[e] = o[e] * f + (64 * e + lane < DH ? p * to_f32(vr[64 * e + lane]) : 0.f);
    m = mn;
  };
  if (a.mask_paper)
    slot(a.Kd + ((long)c * a.Hkv + kvh) * DH, a.Vd + ((long)c * a.Hkv + kvh) * DH);
  const long pb = ((long)c * a.Hkv + kvh) * a.P_cap * DH;
  for (int s = 0; s < a.P; ++s) slot(a.Kp + pb + (long)s * DH, a.Vp + pb + (long)s * DH);
  const long cb = (((long)c * a.B + b) * a.Hkv + kvh) * a.S_cap * DH;
  for (int s = 0; s < na; ++s) slot(a.Kc + cb + (long)s * DH, a.Vc + cb + (long)s * DH);
  for (int s = lo; s < lim; ++s) slot(a.Kc + cb + (long)s * DH, a.Vc + cb + (long)s * DH);
  T* dst = a.O + ((((long)l * a.B + b) * a.T_new + i) * a.Hq + hq) * DH;
  for (int e = 0; e < E; ++e)
    if (64 * e + lane < DH) dst[64 * e + lane] = from_f32<T>(o[e] / sum);
  if (a.lse && lane == 0) a.lse[rid] = m + __log2f(sum);
}

// weight[c][b][kvh][s] += sum of exp2(score - lse) over the rows that read the slot: a wave per
// slot, its lanes over the rows.
template <typename T, int DH>
__global__ __launch_bounds__(256) void reach_weigh_kernel(ReachArgs<T> a, ChannelGroups cg,
                                                          float* weight) {
  const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int kvh = blockIdx.y % a.Hkv, b = blockIdx.y / a.Hkv % a.B, c = blockIdx.y / a.Hkv / a.B;
  const int p0 = ctx_at(a.ctx_len, b, a.ctx_hi) + a.gq + (a.mask_paper ? 0 : 1);
  if (s >= min(p0 + a.gs * (a.T_new - 1), a.S_cap)) return;
  const int G = a.Hq / a.Hkv, n = (cg.offsets[c + 1] - cg.offsets[c]) * G * a.T_new;
  const T* kr = a.Kc + ((((long)c * a.B + b) * a.Hkv + kvh) * a.S_cap + s) * DH;
  float w = 0.f;
  for (int x = lane; x < n; x += 64) {
    const int i = x % a.T_new, hq = kvh * G + x / a.T_new % G;
    const int l = cg.members[cg.offsets[c] + x / a.T_new / G];
    if (s >= p0 + a.gs * i) continue;
    const long rid = (((long)l * a.B + b) * a.Hq + hq) * a.T_new + i;
    float sc = 0.f;
    for (int e = 0; e < DH; ++e) sc += to_f32(a.Q[rid * DH + e]) * a.scale_log2 * to_f32(kr[e]);
    w += fast_exp2(sc - a.lse[rid]);
  }
  w = wave_sum(w);
  if (lane == 0 && n > 0) weight[(((long)c * a.B + b) * a.Hkv + kvh) * a.S_cap + s] += w;
}

template <typename T>
static ReachArgs<T> reach_args(const Shape& sh, const Reach& r, const LayerTable& chan, const T* Q,
                               const T* Kc, const T* Vc, const T* Kd, const T* Vd,
                               const int32_t* ctx_len, T* O, float* lse) {
  return ReachArgs<T>{Q, Kc, Vc, Kd, Vd, (const T*)r.Kp, (const T*)r.Vp, ctx_len, O, lse, sh.B,
                      sh.T_new, sh.L, sh.Hq, sh.Hkv, sh.S_cap, r.P, r.P_cap, r.window, r.sinks,
                      sh.mask_paper, sh.gs, sh.gq, sh.ctx_hi, kLog2e / sqrtf((float)sh.d), chan};
}

template <typename T>
void launch_reach(const Shape& sh, const Reach& r, const LayerTable& chan, const T* Q, const T* Kc,
                  const T* Vc, const T* Kd, const T* Vd, const int32_t* ctx_len, T* O, float* lse,
                  hipStream_t s) {
  const ReachArgs<T> a = reach_args<T>(sh, r, chan, Q, Kc, Vc, Kd, Vd, ctx_len, O, lse);
  const long rows = (long)sh.L * sh.N() * sh.Hq;
  const dim3 grid((unsigned)((rows + 3) / 4));
  if (sh.d == 32) hipLaunchKernelGGL((reach_rows_kernel<T, 32>), grid, dim3(256), 0, s, a);
  else if (sh.d == 64) hipLaunchKernelGGL((reach_rows_kernel<T, 64>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((reach_rows_kernel<T, 96>), grid, dim3(256), 0, s, a);
}

template <typename T>
void launch_weigh(const Shape& sh, const LayerTable& chan, const ChannelGroups& cg, const T* Q,
                  const T* Kc, const int32_t* ctx_len, const float* lse, float* weight,
                  hipStream_t s) {
  const Reach r{};
  const ReachArgs<T> a = reach_args<T>(sh, r, chan, Q, Kc, nullptr, nullptr, nullptr, ctx_len,
                                       nullptr, const_cast<float*>(lse));
  const long most = (long)sh.ctx_max + sh.span();
  const dim3 grid((unsigned)((most + 3) / 4), (unsigned)(sh.k * sh.B * sh.Hkv));
  if (sh.d == 32) hipLaunchKernelGGL((reach_weigh_kernel<T, 32>), grid, dim3(256), 0, s, a, cg, weight);
  else if (sh.d == 64) hipLaunchKernelGGL((reach_weigh_kernel<T, 64>), grid, dim3(256), 0, s, a, cg, weight);
  else hipLaunchKernelGGL((reach_weigh_kernel<T, 96>), grid, dim3(256), 0, s, a, cg, weight);
}

// ------------------------------------------------------------------ gradients
// With P = exp2(s - lse), D = dO.O, dS = P (dO.v - D): a wave per row sums dq, a wave per slot
// its dk and dv over the rows that read it.
struct ReachBwdArgs {
  ReachArgs<bf16> f;
  const bf16 *Of, *dO;
  float *dQ, *dKc, *dVc, *dKd, *dVd;
  float *dlt, *pd, *dsd;  // per row: D, the dummy's P and dS
  float scale;
};

template <int DH>
__global__ __launch_bounds__(256) void reach_bwd_dq_kernel(ReachBwdArgs g) {
  constexpr int E = (DH + 63) / 64;
  const ReachArgs<bf16>& a = g.f;
  const long rows = (long)a.L * a.B * a.Hq * a.T_new;
  const long rid = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (rid >= rows) return;
  const int i = (int)(rid % a.T_new), hq = (int)(rid / a.T_new % a.Hq);
  const int b = (int)(rid / a.T_new / a.Hq % a.B), l = (int)(rid / a.T_new / a.Hq / a.B);
  const int c = a.chan.v[l], kvh = hq / (a.Hq / a.Hkv);
  const int lim = min(ctx_at(a.ctx_len, b, a.ctx_hi) + a.gq + a.gs * i + (a.mask_paper ? 0 : 1),
                      a.S_cap);
  const int lo = max(lim - a.window, 0), na = min(a.sinks, lo);
  const long tok = ((((long)l * a.B + b) * a.T_new + i) * a.Hq + hq) * DH;
  float q[E], d[E], A[E], Bk[E], m = kNegBig, sum = 0.f, dl = 0.f;
  for (int e = 0; e < E; ++e) {
    const bool ok = 64 * e + lane < DH;
    q[e] = ok ? to_f32(a.Q[rid * DH + 64 * e + lane]) * a.scale_log2 : 0.f;
    d[e] = ok ? to_f32(g.dO[tok + 64 * e + lane]) : 0.f;
    dl += ok ? d[e] * to_f32(g.Of[tok + 64 * e + lane]) : 0.f;
    A[e] = Bk[e] = 0.f;
  }
  const float delta = wave_sum(dl);
  float sd = 0.f, dpd = 0.f;
  auto slot = [&](const bf16* kr, const bf16* vr, bool dummy) {
    float ps = 0.f, pd = 0.f;
    for (int e = 0; e < E; ++e)
      if (64 * e + lane < DH) {
        ps += q[e] * to_f32(kr[64 * e + lane]);
        pd += d[e] * to_f32(vr[64 * e + lane]);
      }
    const float sc = wave_sum(ps), dp = wave_sum(pd), mn = fmaxf(m, sc);
    const float f = fast_exp2(m - mn), p = fast_exp2(sc - mn);
    sum = sum * f + p;
    for (int e = 0; e < E; ++e)
      A[e] = A[e] * f + (64 * e + lane < DH ? p * (dp - delta) * to_f32(kr[64 * e + lane]) : 0.f);
    m = mn;
    if (dummy) sd = sc, dpd = dp;
  };
  if (a.mask_paper)
    slot(a.Kd + ((long)c * a.Hkv + kvh) * DH, a.Vd + ((long)c * a.Hkv + kvh) * DH, true);
  const long cb = (((long)c * a.B + b) * a.Hkv + kvh) * a.S_cap * DH;
  for (int s = 0; s < na; ++s) slot(a.Kc + cb + (long)s * DH, a.Vc + cb + (long)s * DH, false);
  for (int s = lo; s < lim; ++s) slot(a.Kc + cb + (long)s * DH, a.Vc + cb + (long)s * DH, false);
  for (int e = 0; e < E; ++e)
    if (64 * e + lane < DH) g.dQ[rid * DH + 64 * e + lane] = A[e] / sum * g.scale;
  if (lane == 0) {
    const float lse = m + __log2f(sum), p = a.mask_paper ? fast_exp2(sd - lse) : 0.f;
    a.lse[rid] = lse;
    g.dlt[rid] = delta;
    g.pd[rid] = p;
    g.dsd[rid] = p * (dpd - delta);
  }
}

template <int DH>
__global__ __launch_bounds__(256) void reach_bwd_dkv_kernel(ReachBwdArgs g, ChannelGroups cg) {
  constexpr int E = (DH + 63) / 64;
  const ReachArgs<bf16>& a = g.f;
  const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int kvh = blockIdx.y % a.Hkv, b = blockIdx.y / a.Hkv % a.B, c = blockIdx.y / a.Hkv / a.B;
  const int pos0 = ctx_at(a.ctx_len, b, a.ctx_hi) + a.gq, incl = a.mask_paper ? 0 : 1;
  if (s >= pos0 + a.gs * (a.T_new - 1) + 1) return;
  const int G = a.Hq / a.Hkv, nm = cg.offsets[c + 1] - cg.offsets[c];
  const long at = ((((long)c * a.B + b) * a.Hkv + kvh) * a.S_cap + s) * DH;
  float kr[E], vr[E], dk[E], dv[E];
  for (int e = 0; e < E; ++e) {
    const bool ok = 64 * e + lane < DH;
    kr[e] = ok ? to_f32(a.Kc[at + 64 * e + lane]) * a.scale_log2 : 0.f;
    vr[e] = ok ? to_f32(a.Vc[at + 64 * e + lane]) : 0.f;
    dk[e] = dv[e] = 0.f;
  }
  for (int x = 0; x < nm * G; ++x) {
    const int l = cg.members[cg.offsets[c] + x / G], hq = kvh * G + x % G;
    for (int i = 0; i < a.T_new; ++i) {
      const int lim = pos0 + incl + a.gs * i;
      if (s >= lim || (s < lim - a.window && s >= a.sinks)) continue;
      const long rid = (((long)l * a.B + b) * a.Hq + hq) * a.T_new + i;
      const long tok = ((((long)l * a.B + b) * a.T_new + i) * a.Hq + hq) * DH;
      float q[E], d[E], ps = 0.f, pd = 0.f;
      for (int e = 0; e < E; ++e) {
        const bool ok = 64 * e + lane < DH;
        q[e] = ok ? to_f32(a.Q[rid * DH + 64 * e + lane]) : 0.f;
        d[e] = ok ? to_f32(g.dO[tok + 64 * e + lane]) : 0.f;
        ps += q[e] * kr[e];
        pd += d[e] * vr[e];
      }
      const float p = fast_exp2(wave_sum(ps) - a.lse[rid]), ds = p * (wave_sum(pd) - g.dlt[rid]);
      for (int e = 0; e < E; ++e) {
        dk[e] += ds * q[e];
        dv[e] += p * d[e];
      }
    }
  }
  for (int e = 0; e < E; ++e)
    if (64 * e + lane < DH) {
      g.dKc[at + 64 * e + lane] = dk[e] * g.scale;
      g.dVc[at + 64 * e + lane] = dv[e];
    }
}

// The dummy of (channel, KV head): one workgroup, a thread per element.
template <int DH>
__global__ __launch_bounds__(DH) void reach_bwd_dummy_kernel(ReachBwdArgs g, ChannelGroups cg) {
  const ReachArgs<bf16>& a = g.f;
  const int kvh = blockIdx.x % a.Hkv, c = blockIdx.x / a.Hkv, e = threadIdx.x, G = a.Hq / a.Hkv;
  float dk = 0.f, dv = 0.f;
  if (a.mask_paper)
    for (int x = cg.offsets[c]; x < cg.offsets[c + 1]; ++x)
      for (int b = 0; b < a.B; ++b)
        for (int h = kvh * G; h < (kvh + 1) * G; ++h)
          for (int i = 0; i < a.T_new; ++i) {
            const int l = cg.members[x];
            const long rid = (((long)l * a.B + b) * a.Hq + h) * a.T_new + i;
            dk += g.dsd[rid] * to_f32(a.Q[rid * DH + e]);
            dv += g.pd[rid] *
                  to_f32(g.dO[((((long)l * a.B + b) * a.T_new + i) * a.Hq + h) * DH + e]);
          }
  g.dKd[(long)blockIdx.x * DH + e] = dk * g.scale;
  g.dVd[(long)blockIdx.x * DH + e] = dv;
}

size_t reach_backward_rows_bytes(const Shape& sh) {
  return 4ul * sh.L * sh.N() * sh.Hq * sizeof(float);
}

void launch_reach_backward(const Shape& sh, const Reach& r, const LayerTable& chan,
                           const ChannelGroups& cg, const bf16* Q, const bf16* Kc, const bf16* Vc,
                           const bf16* Kd, const bf16* Vd, const bf16* O, const bf16* dO,
                           const int32_t* ctx_len, float* dQ, float* dKc, float* dVc, float* dKd,
                           float* dVd, float* rows, hipStream_t s) {
  const long nr = (long)sh.L * sh.N() * sh.Hq;
  const ReachBwdArgs g{reach_args<bf16>(sh, r, chan, Q, Kc, Vc, Kd, Vd, ctx_len, nullptr, rows),
                       O, dO, dQ, dKc, dVc, dKd, dVd, rows + nr, rows + 2 * nr, rows + 3 * nr,
                       1.0f / sqrtf((float)sh.d)};
  const long most = (long)sh.ctx_max + sh.span();
  const dim3 gr((unsigned)((nr + 3) / 4)),
      gk((unsigned)((most + 3) / 4), (unsigned)(sh.k * sh.B * sh.Hkv)), gd(sh.k * sh.Hkv);
  if (sh.d == 64) {
    hipLaunchKernelGGL(reach_bwd_dq_kernel<64>, gr, dim3(256), 0, s, g);
    hipLaunchKernelGGL(reach_bwd_dkv_kernel<64>, gk, dim3(256), 0, s, g, cg);
    hipLaunchKernelGGL(reach_bwd_dummy_kernel<64>, gd, dim3(64), 0, s, g, cg);
  } else {
    hipLaunchKernelGGL(reach_bwd_dq_kernel<96>, gr, dim3(256), 0, s, g);
    hipLaunchKernelGGL(reach_bwd_dkv_kernel<96>, gk, dim3(256), 0, s, g, cg);
    hipLaunchKernelGGL(reach_bwd_dummy_kernel<96>, gd, dim3(96), 0, s, g, cg);
  }
}

#define WM_INST(T)                                                                                \
  template void launch_reach<T>(const Shape&, const Reach&, const LayerTable&, const T*,          \
                                const T*, const T*, const T*, const T*, const int32_t*, T*,       \
                                float*, hipStream_t);                                             \
  template void launch_weigh<T>(const Shape&, const LayerTable&, const ChannelGroups&, const T*,  \
                                const T*, const int32_t*, const float*, float*, hipStream_t);
WM_INST(float)
WM_INST(bf16)
#undef WM_INST

}  // namespace wm
