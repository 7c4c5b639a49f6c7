// Gradients of the window attention (wm_channel_attend_window_backward; bf16 tensors, head dims 64
// and 96). For a row with scores s_j = q.k_j / sqrt(d) over the slots it reads and the dummy,
// P_j = exp(s_j - LSE), D = dO.O:
//   dS_j = P_j (dO.v_j - D),  dq = sum_j dS_j k_j / sqrt(d),  dk_j += dS_j q / sqrt(d),
//   dv_j += P_j dO.
// Four steps:
//   reach_bwd_dq_kernel    query-major: LSE, D and dq in one walk over the slots that the tile's
//                          rows read, with an online maximum
//   reach_bwd_dkv_kernel   slot-major: 64 slots of one (channel, sequence, KV head) against the
//                          rows whose windows hold them
//   reach_bwd_sink_*       the first slots against the rows whose windows lie past them: all later
//                          rows, which one slot tile would walk alone, cut over waves and
//                          workgroups
//   the dummy              as in wm_backward.hip
// P and dS enter the products as three bf16 parts of 8 bits (cut24), so that fp32 gradients keep
// fp32's digits: with one rounded part they are off by 2e-3 of themselves. That makes 13 products
// of the formula's 5 (S and dP twice, dv, dk and dq three parts each) and as many vector
// instructions for the parts as for the weights, which bounds the kernels.
#include <algorithm>

#include "wm_device.hpp"
#include "wm_frag.hpp"
#include "wm_internal.hpp"
#include "wm_prefill.hpp"

namespace wm {

struct ReachBwdArgs {
  const bf16 *Q, *Kc, *Vc, *Kd, *Vd, *O, *dO;
  const int32_t* ctx_len;
  float *dQ, *dKc, *dVc;
  float *lse, *dlt, *pd, *dsd;  // per row: LSE (log2 units), D, the dummy's P and dS
  float* part;                  // first slots' partial sums [chunks][slices][n32][32][2][d]
  int B, T, L, Hq, Hkv, S_cap, window, sinks, mask_paper, ctx_hi, n_qtiles, n_stiles;
  int gs, gq, n32, chunks;
  float scale_log2, scale;  // log2(e) / sqrt(d), 1 / sqrt(d)
  LayerTable chan;
  ChannelGroups grp;
};

constexpr int kReachBwdWaves = 4;  // waves per workgroup
constexpr float kHiddenScore = -__builtin_inff();

// A thread's share of copying ROWS rows (row_bytes apart in memory) into an LDS block in the
// fragment readers' chunk order: byte offsets of its 16-byte chunks within the block of rows, and
// their rows. Views end at the last row, so rows past it arrive as zeros.
template <int DH, int ROWS, int NW> struct ReachCopy {
  static constexpr int CPR = DH * 2 / 16, TOT = ROWS * CPR, NI = TOT / (64 * NW);
  static_assert(NI * 64 * NW == TOT, "whole instructions per wave");
  uint32_t off[NI];
  int row[NI];
  __device__ __forceinline__ ReachCopy(uint32_t row_bytes, int w, int lane) {
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int pos = (NI * w + n) * 64 + lane, cc = pos % CPR;
      row[n] = pos / CPR;
      off[n] = (uint32_t)row[n] * row_bytes + 16u * (uint32_t)(cc ^ pf_swz<DH>(row[n]));
    }
  }
  // Rows from byte `base` of the view on into LDS at lds_base (this wave's chunks follow its w);
  // rows at or past `na` of the block lie `skip` bytes further on.
  __device__ __forceinline__ void go(uint32_t lds_base, __amdgpu_buffer_rsrc_t view, uint32_t base,
                                     int w, int na = ROWS, uint32_t skip = 0) const {
#pragma unroll
    for (int n = 0; n < NI; ++n)
      lds_dma16(__builtin_amdgcn_readfirstlane(lds_base + (NI * w + n) * 1024),
                base + off[n] + (row[n] >= na ? skip : 0u), view);
  }
};

// --------------------------------------------------------------- dq, LSE, D
// Tile: 128 rows of one (consumer, sequence, query head), 32 per wave; S^T = K q^T and
// dP^T = V dO^T put one row in a lane, and dq^T += K^T dS^T takes dS^T from those registers
// through the transposing read of the K block. Compact slots as in wm_reach.hip.
template <int DH>
__global__ __launch_bounds__(64 * kReachBwdWaves) void reach_bwd_dq_kernel(ReachBwdArgs a) {
  constexpr int NW = kReachBwdWaves, NKS = DH / 16, NDT = DH / 32, ROW = 2 * DH, BLK = 64;
  __shared__ __align__(16) char smem[4 * BLK * ROW];  // two buffers of a K and a V block
  const uint32_t lbase = (uint32_t)(uintptr_t)smem;
  const int tile = xcd_tile(blockIdx.x, (int)gridDim.x);
  const int qtile = a.n_qtiles - 1 - tile % a.n_qtiles;
  int y = tile / a.n_qtiles;
  const int hq = y % a.Hq;
  y /= a.Hq;
  const int b = y % a.B, l = y / a.B;
  const int c = a.chan.v[l], kvh = hq / (a.Hq / a.Hkv);
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pq = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq +
                 (a.mask_paper ? 0 : 1);  // row i reads slots below pq + gs i
  const int q0 = qtile * 32 * NW, qw0 = q0 + 32 * w, qi = qw0 + r;
  const bool valid = qi < a.T;
  const float cl2 = a.scale_log2;

  bf16x8 qf[NKS], df[NKS];
  float dl = 0.f, sdp = 0.f, dpd = 0.f;
  const long dofs = ((long)c * a.Hkv + kvh) * DH;
  const uint32_t dbytes = a.mask_paper ? DH * 2u : 0u;
  const auto kdv = make_view(a.mask_paper ? a.Kd + dofs : nullptr, dbytes);
  const auto vdv = make_view(a.mask_paper ? a.Vd + dofs : nullptr, dbytes);
  {
    const long rowl = ((long)l * a.B + b) * a.T;
    const uint32_t ostride = (uint32_t)a.Hq * DH * 2u;
    const auto qv = make_view(a.Q + (((long)l * a.B + b) * a.Hq + hq) * (long)a.T * DH,
                              (uint32_t)a.T * DH * 2u);
    const auto dv = make_view(a.dO + rowl * a.Hq * DH + (long)hq * DH, (uint32_t)a.T * ostride);
    const auto ov = make_view(a.O + rowl * a.Hq * DH + (long)hq * DH, (uint32_t)a.T * ostride);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const uint32_t col = (uint32_t)(16 * ks + 8 * h) * 2u;
      qf[ks] = buf_frag<bf16>(qv, valid ? (uint32_t)qi * DH * 2u + col : kOffOob);
      df[ks] = buf_frag<bf16>(dv, valid ? (uint32_t)qi * ostride + col : kOffOob);
      const bf16x8 of = buf_frag<bf16>(ov, valid ? (uint32_t)qi * ostride + col : kOffOob);
      const bf16x8 kd = buf_frag<bf16>(kdv, col), vd = buf_frag<bf16>(vdv, col);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dl += (float)df[ks][e] * (float)of[e];
        sdp += (float)qf[ks][e] * (float)kd[e];
        dpd += (float)df[ks][e] * (float)vd[e];
      }
    }
  }
  const float delta = halves_sum(dl);
  const float sd = halves_sum(sdp) * cl2;  // the dummy's score, log2 units
  dpd = halves_sum(dpd);

  const int kend = min(pq + a.gs * (min(q0 + 32 * NW, a.T) - 1), a.S_cap);
  const int lo0 = max(pq + a.gs * q0 - a.window, 0);
  const int na = min(a.sinks, lo0), skip = lo0 - na, n = kend - skip;  // compact slots
  const int lim = pq - skip + a.gs * qi, rlo = lim - a.window;
  const int wlim0 = pq - skip + a.gs * qw0, wlast = min(qw0 + 31, a.T - 1);
  const int wlim1 = wlast >= qw0 ? pq - skip + a.gs * wlast : 0;
  const int nblk = (n + BLK - 1) / BLK;
  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  const auto kv = make_view(a.Kc + cbase, (uint32_t)max(kend, 0) * ROW);
  const auto vv = make_view(a.Vc + cbase, (uint32_t)max(kend, 0) * ROW);
  const PfLane<DH> lo = pf_lane<DH>(lane);

  // running maximum m (log2 units, shared by the two lanes of the row), sum = sum 2^(s - m) and
  // dq~ = sum 2^(s - m) (dP - D) k, rescaled when m grows; lse = m + log2 sum, dq = dq~ / sum
  float m = a.mask_paper ? sd : kNegBig;
  float sum = a.mask_paper && h == 0 ? 1.f : 0.f;
  f32x16 dq[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) dq[dt] = zero16();
  const ReachCopy<DH, BLK, NW> cp(ROW, w, lane);
  auto fetch = [&](int j, uint32_t at) {
    const int left = na - j * BLK;  // first slots from the block's start on
    cp.go(at, kv, (uint32_t)j * BLK * ROW, w, left, (uint32_t)skip * ROW);
    cp.go(at + BLK * ROW, vv, (uint32_t)j * BLK * ROW, w, left, (uint32_t)skip * ROW);
  };
  if (nblk > 0) fetch(0, lbase);
  for (int j = 0; j < nblk; ++j) {
    const uint32_t kb = (uint32_t)(j & 1) * 2 * BLK * ROW;
    wait_vmcnt<0>();
    __syncthreads();  // block j is in LDS; every wave is done with block j - 1
    if (j + 1 < nblk) fetch(j + 1, lbase + (kb ^ (2 * BLK * ROW)));
#pragma unroll
    for (int hg = 0; hg < 2; ++hg) {
      const int sb = j * BLK + 32 * hg;
      // some row of the wave reads some of the 32 slots
      if (sb < wlim1 && (sb + 32 > wlim0 - a.window || sb < a.sinks)) {
        f32x16 sc = zero16(), dp = zero16();
        const uint32_t ho = kb + hg * 32 * ROW;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
          sc = mma32(sc, pf_ldk<DH>(smem, lo, ho, ks), qf[ks]);
          dp = mma32(dp, pf_ldk<DH>(smem, lo, ho + BLK * ROW, ks), df[ks]);
        }
        if (sb + 32 > wlim0 || (sb < wlim1 - a.window && sb + 32 > a.sinks)) {
          const int at = sb + 4 * h;
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const int x = at + 8 * (q >> 2) + (q & 3);
            sc[q] = x >= lim || (x < rlo && x >= a.sinks) ? kHiddenScore : sc[q];
          }
        }
        float mx = sc[0];
#pragma unroll
        for (int q = 1; q < 16; ++q) mx = fmaxf(mx, sc[q]);
        const float mn = fmaxf(m, halves_max(mx) * cl2);
        if (__builtin_expect(__any(mn > m), 0)) {
          const float f = fast_exp2(m - mn);
          sum *= f;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) dq[dt] *= f;
          m = mn;
        }
        f32x16 ds;
        float ps[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const float p = fast_exp2(fmaf(sc[q], cl2, -m));  // 0 when hidden
          ps[q & 1] += p;
          ds[q] = p * (dp[q] - delta);
        }
        sum += ps[0] + ps[1];
        bf16x8 dw[3][2];
        cut24(ds, dw);
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const bf16x8 kf = pf_ldv<DH>(smem, lo, ho, kh, dt);
#pragma unroll
            for (int u = 0; u < 3; ++u) dq[dt] = mma32(dq[dt], kf, dw[u][kh]);
          }
      }
    }
  }
  const float ltot = halves_sum(sum);
  const float lse = m + __log2f(ltot), inv = 1.0f / ltot;
  const float p_d = a.mask_paper ? fast_exp2(sd - lse) : 0.f;
  const float ds_d = p_d * (dpd - delta);
  if (valid) {
    const long idx = (((long)l * a.B + b) * a.Hq + hq) * a.T + qi;
    float* dst = a.dQ + idx * DH;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const bf16x4 kd = __builtin_bit_cast(
            bf16x4, __builtin_amdgcn_raw_buffer_load_b64(kdv, (32 * dt + 8 * g + 4 * h) * 2u, 0, 0));
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = (dq[dt][4 * g + i] * inv + ds_d * (float)kd[i]) * a.scale;
        *(f32x4*)(dst + 32 * dt + 8 * g + 4 * h) = v;
      }
    if (h == 0) {
      a.lse[idx] = lse;
      a.dlt[idx] = delta;
      a.pd[idx] = p_d;
      a.dsd[idx] = ds_d;
    }
  }
}

// The products of 32 rows (block at kb: queries, then dO at kb + dofs) with the 32 slots whose K and
// V rows are kf, vf: P and dS of the rows that `sees` says read the slot (lane (h, r): slot r, rows
// 8 (i / 4) + 4 h + i % 4), then dv^T += dO^T P, dk^T += Q^T dS. lz, nz: the rows' LSE and -D.
template <int DH, class F>
__device__ __forceinline__ void reach_bwd_rows(const char* sm, const PfLane<DH>& lo, uint32_t kb,
                                               uint32_t dofs, const bf16x8 (&kf)[DH / 16],
                                               const bf16x8 (&vf)[DH / 16], const float* lz,
                                               const float* nz, float cl2, int h, bool masked,
                                               F sees, f32x16 (&dk)[DH / 32],
                                               f32x16 (&dv)[DH / 32]) {
  constexpr int NKS = DH / 16, NDT = DH / 32;
  f32x16 sc = zero16(), dp;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4 d4 = *(const f32x4*)(nz + 8 * g + 4 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) dp[4 * g + e] = d4[e];
  }
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) {
    sc = mma32(sc, pf_ldk<DH>(sm, lo, kb, ks), kf[ks]);
    dp = mma32(dp, pf_ldk<DH>(sm, lo, kb + dofs, ks), vf[ks]);
  }
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4 l4 = *(const f32x4*)(lz + 8 * g + 4 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) sc[4 * g + e] = fast_exp2(fmaf(sc[4 * g + e], cl2, -l4[e]));
  }
  if (masked) {  // (dP too: a slot that no row reads may hold anything)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool s = sees(8 * (i >> 2) + 4 * h + (i & 3));
      sc[i] = s ? sc[i] : 0.f;
      dp[i] = s ? dp[i] : 0.f;
    }
  }
  bf16x8 pw[3][2];
  cut24(sc, pw);
#pragma unroll
  for (int kh = 0; kh < 2; ++kh)
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
      const bf16x8 f = pf_ldv<DH>(sm, lo, kb + dofs, kh, dt);
#pragma unroll
      for (int u = 0; u < 3; ++u) dv[dt] = mma32(dv[dt], f, pw[u][kh]);
    }
  dp *= sc;
  cut24(dp, pw);
#pragma unroll
  for (int kh = 0; kh < 2; ++kh)
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
      const bf16x8 f = pf_ldv<DH>(sm, lo, kb, kh, dt);
#pragma unroll
      for (int u = 0; u < 3; ++u) dk[dt] = mma32(dk[dt], f, pw[u][kh]);
    }
}

// ------------------------------------------------------------------- dk, dv
// Tile: 64 slots of one (channel, sequence, KV head), 32 per pair of waves, whose K and V rows stay
// in registers as the column operand. It walks every block of 64 rows whose windows hold some of its
// slots, for every consumer of the channel and every query head of the KV head, the next block
// copied into LDS while the current one is multiplied; a pair's waves take a half of each block, and
// their sums meet in LDS at the end. (One wave per 32 slots, 128 per tile, walks window + 128 rows for
// the window + 32 that each wave needs, and leaves the last of two rounds of workgroups half
// empty: 2 x 2048 tokens, 16 layers of 6/3 heads of 96, window 512 414 us, this way 322.)
template <int DH>
__global__ __launch_bounds__(64 * kReachBwdWaves) __attribute__((amdgpu_waves_per_eu(2)))
void reach_bwd_dkv_kernel(ReachBwdArgs a) {
  constexpr int NW = kReachBwdWaves, NKS = DH / 16, NDT = DH / 32, ROW = 2 * DH, QB = 64;
  constexpr uint32_t BUF = 2 * QB * ROW;  // one buffer: a Q block, then a dO block
  __shared__ __align__(16) char smem[2 * BUF];
  __shared__ __align__(16) float s_lse[2][QB], s_dlt[2][QB];
  const uint32_t lbase = (uint32_t)(uintptr_t)smem;
  const int tile = xcd_tile(blockIdx.x, (int)gridDim.x);
  const int stile = tile % a.n_stiles;
  int y = tile / a.n_stiles;
  const int kvh = y % a.Hkv;
  y /= a.Hkv;
  const int b = y % a.B, c = y / a.B;
  const int G = a.Hq / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pos0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq;
  const int pq = pos0 + (a.mask_paper ? 0 : 1);  // row i reads slots below pq + gs i
  const int send = pos0 + a.gs * (a.T - 1) + 1;  // slots written: [0, send)
  constexpr int SLOTS = 32 * NW / 2;
  const int sbase = stile * SLOTS;
  if (sbase >= send) return;
  const int pair = w & 1, half = w >> 1;  // this wave's slots, its half of every block
  const int ws0 = sbase + 32 * pair, slot = ws0 + r;
  const bool slot_ok = slot < send;

  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  bf16x8 kf[NKS], vf[NKS];
  {
    const auto kv = make_view(a.Kc + cbase, (uint32_t)send * ROW);
    const auto vv = make_view(a.Vc + cbase, (uint32_t)send * ROW);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const uint32_t off = slot_ok ? (uint32_t)slot * ROW + (16 * ks + 8 * h) * 2u : kOffOob;
      kf[ks] = buf_frag<bf16>(kv, off);
      vf[ks] = buf_frag<bf16>(vv, off);
    }
  }
  f32x16 dk[NDT], dv[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) dk[dt] = dv[dt] = zero16();
  const PfLane<DH> lo = pf_lane<DH>(lane);
  // rows i with sbase < pq + gs i (the first) and pq + gs i - window <= sbase + SLOTS - 1
  const int i_num = sbase - pq, l_num = sbase + SLOTS - 1 + a.window - pq;
  const int i_first = i_num < 0 ? 0 : i_num / a.gs + 1;
  const int i_last = l_num < 0 ? -1 : min(l_num / a.gs, a.T - 1);
  const int qb0 = i_first / QB, nqb = i_last >= i_first ? i_last / QB - qb0 + 1 : 0;
  const int nit = (a.grp.offsets[c + 1] - a.grp.offsets[c]) * G * nqb;
  const uint32_t ostride = (uint32_t)a.Hq * DH * 2u;
  const ReachCopy<DH, QB, NW> cq(ROW, w, lane), cd(ostride, w, lane);
  float lse_n = 0.f, dlt_n = 0.f;  // the next block's LSE and -D of row tid (threads < QB)
  auto fetch = [&](int it, uint32_t buf) {
    const int qb = qb0 + it % nqb, x = it / nqb, hq = kvh * G + x % G;
    const int l = a.grp.members[a.grp.offsets[c] + x / G];
    const long rows0 = (((long)l * a.B + b) * a.Hq + hq) * a.T;
    const long rowl = ((long)l * a.B + b) * a.T;
    const auto qv = make_view(a.Q + rows0 * DH, (uint32_t)a.T * DH * 2u);
    const auto dov = make_view(a.dO + rowl * a.Hq * DH + (long)hq * DH, (uint32_t)a.T * ostride);
    cq.go(buf, qv, (uint32_t)(qb * QB) * ROW, w);
    cd.go(buf + QB * ROW, dov, (uint32_t)(qb * QB) * ostride, w);
    if (tid < QB) {
      const int qr = qb * QB + tid;
      lse_n = qr < a.T ? a.lse[rows0 + qr] : 1.0e30f;  // a row past T weighs 0
      dlt_n = qr < a.T ? -a.dlt[rows0 + qr] : 0.f;
    }
  };
  if (nit > 0) fetch(0, lbase);
  for (int it = 0; it < nit; ++it) {
    const int u = it & 1;
    const uint32_t kb = (uint32_t)u * BUF;
    if (tid < QB) {
      s_lse[u][tid] = lse_n;
      s_dlt[u][tid] = dlt_n;
    }
    wait_vmcnt<0>();
    __syncthreads();  // block it is in LDS; every wave is done with block it - 1
    const int qb = qb0 + it % nqb;
    if (it + 1 < nit) fetch(it + 1, lbase + (kb ^ BUF));
    const int qg = qb * QB + 32 * half, qe = min(qg + 31, a.T - 1);  // this wave's rows
    const int lim0 = pq + a.gs * qg, lim1 = pq + a.gs * qe;
    if (qg < a.T && lim1 > ws0 && lim0 - a.window <= ws0 + 31) {
      const bool masked = lim0 <= ws0 + 31 || lim1 - a.window > ws0;
      reach_bwd_rows<DH>(smem, lo, kb + half * 32 * ROW, QB * ROW, kf, vf, &s_lse[u][32 * half],
                         &s_dlt[u][32 * half], a.scale_log2, h, masked,
                         [&](int x) {
                           const int lim = lim0 + a.gs * x;
                           return slot < lim && slot >= lim - a.window;
                         },
                         dk, dv);
    }
  }
  // the second halves' sums through LDS: dk^T and dv^T of 32 slots per pair, as the registers lie
  __syncthreads();
  static_assert(2 * 2 * 64 * 16 * NDT * 4 <= 2 * BUF, "both pairs' sums fit the blocks");
  f32x4* so = (f32x4*)smem + pair * 2 * NDT * 4 * 64 + lane;
  if (half == 1) {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 kq, vq;
#pragma unroll
        for (int i = 0; i < 4; ++i) kq[i] = dk[dt][4 * g + i], vq[i] = dv[dt][4 * g + i];
        so[(2 * (4 * dt + g)) * 64] = kq;
        so[(2 * (4 * dt + g) + 1) * 64] = vq;
      }
  }
  __syncthreads();
  if (half == 1) return;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 kq = so[(2 * (4 * dt + g)) * 64], vq = so[(2 * (4 * dt + g) + 1) * 64];
#pragma unroll
      for (int i = 0; i < 4; ++i) dk[dt][4 * g + i] += kq[i], dv[dt][4 * g + i] += vq[i];
    }
  if (slot_ok) {
    float* dkd = a.dKc + cbase + (long)slot * DH;
    float* dvd = a.dVc + cbase + (long)slot * DH;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 kq, vq;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          kq[i] = dk[dt][4 * g + i] * a.scale;
          vq[i] = dv[dt][4 * g + i];
        }
        *(f32x4*)(dkd + 32 * dt + 8 * g + 4 * h) = kq;
        *(f32x4*)(dvd + 32 * dt + 8 * g + 4 * h) = vq;
      }
  }
}

// ------------------------------------------------------- the first slots' later readers
// 32 first slots of one (channel, sequence, KV head) against the rows whose windows start past them
// (row i reads slot s < sinks with s < lim - window besides its window). The rows are all later
// ones, so they are cut: steps of 32 rows go round the waves of `chunks` workgroups, each wave
// with a ring of two in LDS of its own; the waves' sums meet in LDS, the workgroups' in part,
// added in order by reach_bwd_sink_sum_kernel.
template <int DH>
__global__ __launch_bounds__(64 * kReachBwdWaves) __attribute__((amdgpu_waves_per_eu(2)))
void reach_bwd_sink_kernel(ReachBwdArgs a) {
  constexpr int NW = kReachBwdWaves, NKS = DH / 16, NDT = DH / 32, ROW = 2 * DH, CPR = ROW / 16;
  constexpr int BLK = 32 * ROW, NI = BLK / 1024, STAGE = 2 * BLK, RING = 2 * STAGE;
  constexpr int OLD = DH;  // row stride of the merge staging (floats)
  static_assert(2 * 32 * OLD * 4 <= RING, "the merge staging fits a wave's ring");
  __shared__ __align__(16) char smem[NW * RING];
  __shared__ __align__(16) float s_row[NW][2][2][32];  // a step's LSE and D
  const int chunk = blockIdx.x % a.chunks;
  int y = blockIdx.x / a.chunks;
  const int t32 = y % a.n32, slice = y / a.n32;
  const int kvh = slice % a.Hkv, b = slice / a.Hkv % a.B, c = slice / a.Hkv / a.B;
  const int G = a.Hq / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pos0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq;
  const int pq = pos0 + (a.mask_paper ? 0 : 1);
  const int send = min(pos0 + a.gs * (a.T - 1) + 1, a.sinks);  // slots of this kernel: [0, send)
  const int ws0 = 32 * t32, slot = ws0 + r;
  const bool slot_ok = slot < send;
  // the first row with pq + gs i - window > ws0
  const int i_num = ws0 + a.window - pq;
  const int i_first = i_num < 0 ? 0 : i_num / a.gs + 1;
  const int qb0 = i_first / 32, nqb = (a.T + 31) / 32 - qb0;
  const int nst = nqb > 0 && ws0 < send ? (a.grp.offsets[c + 1] - a.grp.offsets[c]) * G * nqb : 0;
  const int gw = chunk * NW + w, stride = a.chunks * NW;
  const int mine = nst > gw ? (nst - gw + stride - 1) / stride : 0;

  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  bf16x8 kf[NKS], vf[NKS];
  {
    const auto kv = make_view(a.Kc + cbase, (uint32_t)max(send, 0) * ROW);
    const auto vv = make_view(a.Vc + cbase, (uint32_t)max(send, 0) * ROW);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const uint32_t off = slot_ok ? (uint32_t)slot * ROW + (16 * ks + 8 * h) * 2u : kOffOob;
      kf[ks] = buf_frag<bf16>(kv, off);
      vf[ks] = buf_frag<bf16>(vv, off);
    }
  }
  f32x16 dk[NDT], dv[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) dk[dt] = dv[dt] = zero16();
  const PfLane<DH> lo = pf_lane<DH>(lane);
  const uint32_t ostride = (uint32_t)a.Hq * DH * 2u;
  char* ring = smem + w * RING;
  const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
  float lse_n = 0.f, dlt_n = 0.f;  // LSE and -D of the next step's row r
  auto fetch = [&](int j, int st) {  // step j of this wave into ring stage st
    const int it = gw + stride * j, qb = qb0 + it % nqb, x = it / nqb, hq = kvh * G + x % G;
    const int l = a.grp.members[a.grp.offsets[c] + x / G];
    const long rows0 = (((long)l * a.B + b) * a.Hq + hq) * a.T;
    const long rowl = ((long)l * a.B + b) * a.T;
    const auto qv = make_view(a.Q + rows0 * DH, (uint32_t)a.T * DH * 2u);
    const auto dov = make_view(a.dO + rowl * a.Hq * DH + (long)hq * DH, (uint32_t)a.T * ostride);
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int pos = 64 * n + lane, row = pos / CPR, gr = qb * 32 + row;
      const uint32_t cc = 16u * (uint32_t)((pos - row * CPR) ^ pf_swz<DH>(row));
      const uint32_t at = ring_at + st * STAGE + 1024 * n;
      lds_dma16(__builtin_amdgcn_readfirstlane(at), gr < a.T ? (uint32_t)gr * ROW + cc : kOffOob, qv);
      lds_dma16(__builtin_amdgcn_readfirstlane(at + BLK),
                gr < a.T ? (uint32_t)gr * ostride + cc : kOffOob, dov);
    }
    const int qr = qb * 32 + r;
    lse_n = qr < a.T ? a.lse[rows0 + qr] : 1.0e30f;  // a row past T weighs 0
    dlt_n = qr < a.T ? -a.dlt[rows0 + qr] : 0.f;
  };
  if (mine > 0) fetch(0, 0);
  for (int j = 0; j < mine; ++j) {
    const int st = j & 1;
    wait_copies<0>();  // step j has landed
    s_row[w][st][0][r] = lse_n;
    s_row[w][st][1][r] = dlt_n;
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // reads of the stage refilled next
    if (j + 1 < mine) fetch(j + 1, st ^ 1);
    const int qg = (qb0 + (gw + stride * j) % nqb) * 32;
    const int lim0 = pq + a.gs * qg;
    const bool masked = lim0 - a.window <= ws0 + 31 || ws0 + 32 > a.sinks;
    reach_bwd_rows<DH>(ring, lo, st * STAGE, BLK, kf, vf, s_row[w][st][0], s_row[w][st][1],
                       a.scale_log2, h, masked,
                       [&](int x) { return slot_ok && slot < lim0 + a.gs * x - a.window; }, dk, dv);
  }
  // the waves' sums, in order: dk's rows [r][DH], then dv's, in each wave's ring
  float* so = (float*)ring;
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 kq, vq;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        kq[i] = dk[dt][4 * g + i] * a.scale;
        vq[i] = dv[dt][4 * g + i];
      }
      *(f32x4*)(so + r * OLD + 32 * dt + 8 * g + 4 * h) = kq;
      *(f32x4*)(so + (32 + r) * OLD + 32 * dt + 8 * g + 4 * h) = vq;
    }
  __syncthreads();
  float* part = a.part + ((long)chunk * (gridDim.x / a.chunks) + y) * (2 * 32 * DH);
  for (int e = tid; e < 2 * 32 * DH; e += 64 * NW) {
    const int row = e / DH, dd = e - row * DH;
    float v = 0.f;
#pragma unroll
    for (int ww = 0; ww < NW; ++ww) v += ((const float*)(smem + ww * RING))[row * OLD + dd];
    if (a.part) part[e] = v;
    else if (ws0 + (row & 31) < send) {  // one workgroup has the whole sum
      float* dst = (row < 32 ? a.dKc : a.dVc) + cbase + (long)(ws0 + (row & 31)) * DH + dd;
      *dst += v;
    }
  }
}

// dKc and dVc of the first slots += the workgroups' sums, in order.
__global__ __launch_bounds__(256) void reach_bwd_sink_sum_kernel(ReachBwdArgs a, int d, int slices) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x, per = 2l * 32 * d;
  if (i >= (long)slices * a.n32 * per) return;
  const long y = i / per;
  const int e = (int)(i - y * per), row = e / d, slice = (int)(y / a.n32);
  const int b = slice / a.Hkv % a.B, slot = 32 * (int)(y % a.n32) + (row & 31);
  const int send = ctx_at(a.ctx_len, b, a.ctx_hi) + a.gq + a.gs * (a.T - 1) + 1;
  if (slot >= min(send, a.sinks)) return;
  float v = 0.f;
  for (int ch = 0; ch < a.chunks; ++ch) v += a.part[((long)ch * slices * a.n32 + y) * per + e];
  float* dst = (row < 32 ? a.dKc : a.dVc) + ((long)slice * a.S_cap + slot) * d + e % d;
  *dst += v;
}

// First slots in groups of 32: up to this many (chunk, group) pairs of partial sums per slice.
constexpr int kSinkParts = 16;

static size_t reach_rows(const Shape& sh) { return (size_t)sh.L * sh.N() * sh.Hq; }
static size_t sink_part_floats(const Shape& sh) {
  return (size_t)kSinkParts * sh.k * sh.B * sh.Hkv * 2 * 32 * sh.d;
}
size_t reach_backward_bytes(const Shape& sh) {
  return (4 * reach_rows(sh) + sink_part_floats(sh)) * sizeof(float) + dummy_backward_bytes(sh);
}

template <int DH>
static void reach_backward(ReachBwdArgs a, const Shape& sh, hipStream_t s) {
  const int rows = 32 * kReachBwdWaves, slots = rows / 2, slices = sh.k * sh.B * sh.Hkv;
  a.n_qtiles = (sh.T_new + rows - 1) / rows;
  a.n_stiles = (int)(((long)sh.ctx_max + sh.span() + slots - 1) / slots);
  const dim3 blk(64 * kReachBwdWaves);
  hipLaunchKernelGGL(reach_bwd_dq_kernel<DH>,
                     dim3((unsigned)(a.n_qtiles * sh.Hq * sh.B * sh.L)), blk, 0, s, a);
  hipLaunchKernelGGL(reach_bwd_dkv_kernel<DH>, dim3((unsigned)(a.n_stiles * slices)), blk, 0, s, a);
  // the last row's limit less its window: first slots below it have readers past their windows
  const long past = (long)sh.ctx_max + sh.span() - (sh.mask_paper ? 1 : 0) - a.window;
  const long first = std::min<long>(a.sinks, past);
  if (first <= 0) return;
  a.n32 = (int)((first + 31) / 32);
  // chunks of rows while the workgroups fit the CUs at once (LDS: two of them at head dim 64, one at
  // 96), as far as the partial sums' room goes
  const long per = (long)slices * a.n32, want = (DH == 64 ? 2L : 1L) * device_cus() / per;
  const long steps = ((long)sh.L / sh.k + 1) * (sh.Hq / sh.Hkv) * ((sh.T_new + 31) / 32);
  a.chunks = (int)std::max(1L, std::min({want, (long)(kSinkParts / a.n32), steps / 4}));
  if (a.chunks == 1) a.part = nullptr;
  hipLaunchKernelGGL(reach_bwd_sink_kernel<DH>, dim3((unsigned)(per * a.chunks)), blk, 0, s, a);
  if (a.chunks > 1) {
    const long n = per * 2 * 32 * DH;
    hipLaunchKernelGGL(reach_bwd_sink_sum_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s,
                       a, DH, slices);
  }
}

void launch_reach_backward(const Shape& sh, const Reach& r, const LayerTable& chan,
                           const ChannelGroups& cg, const bf16* Q, const bf16* Kc, const bf16* Vc,
                           const bf16* Kd, const bf16* Vd, const bf16* O, const bf16* dO,
                           const int32_t* ctx_len, float* dQ, float* dKc, float* dVc, float* dKd,
                           float* dVd, float* ws, hipStream_t s) {
  const long nr = (long)reach_rows(sh);
  float* part = ws + 4 * nr;
  const ReachBwdArgs a{Q, Kc, Vc, Kd, Vd, O, dO, ctx_len, dQ, dKc, dVc, ws, ws + nr, ws + 2 * nr,
                       ws + 3 * nr, part, sh.B, sh.T_new, sh.L, sh.Hq, sh.Hkv, sh.S_cap, r.window,
                       r.sinks, sh.mask_paper, sh.ctx_hi, 0, 0, sh.gs, sh.gq, 0, 1,
                       kLog2e / sqrtf((float)sh.d), 1.0f / sqrtf((float)sh.d), chan, cg};
  if (sh.d == 64) reach_backward<64>(a, sh, s);
  else reach_backward<96>(a, sh, s);
  launch_dummy_backward(sh, cg, Q, dO, a.pd, a.dsd, part + sink_part_floats(sh), dKd, dVd, s);
}

}  // namespace wm
