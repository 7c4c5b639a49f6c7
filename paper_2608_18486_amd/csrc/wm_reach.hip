// Channel attention over parts of a long context: a window of the cache with a few first slots
// (wm_channel_attend_window), a prefix that the batch shares next to each sequence's own
// cache (wm_channel_attend_shared), and attention that adds up the weight each slot receives
// (wm_channel_attend_weigh).
//
// Row (l, b, h, i) sits at position t = ctx_len[b] + gq + gs i; with lim = t (paper mask) or
// t + 1 (inclusive) it reads every prefix slot, and the cache slots s < lim with s >= lim -
// window or s < sinks. A tile of rows walks the slots that any of its rows reads as one compact
// range x = 0 .. n - 1:
//   window  its na = min(sinks, lo) first slots, then from its first row's window, lo, on:
//           slot x < na ? x : x + skip, skip = lo - na. Where skip > 0 every first slot lies
//           before every row's window, so in compact indexes a row reads x < lim - skip with
//           x >= lim - window - skip or x < sinks in either case.
//   prefix  the prefix padded to whole blocks (the pad hidden), then the cache's slots; in the
//           same terms sinks = P, and lim - window - skip = the padded length for every row.
// Both are a limit, a lowest slot and a bound of first slots per row (ReachRow).
//
// Full-sequence bf16 form at head dims 64 and 96: the pipeline of the prefill attention (128
// rows per workgroup, K and V blocks of 64 slots through LDS rings of three, S(i + 1) and PV(i -
// 1) on the matrix cores while the weights of step i are taken). It differs in what it keeps
// exact: queries enter unscaled, and a weight is exp2(s log2(e) / sqrt(d) - m) from one fma in
// fp32, where the prefill kernel rounds the scaled queries to bf16 (an error of the weights as
// large as their own rounding, for one fma per weight less).
#include <algorithm>

#include "wm_prefill.hpp"

namespace wm {

template <typename T> struct ReachArgs {
  const T *Q, *Kc, *Vc, *Kd, *Vd;
  const T *Kp, *Vp;  // [k][Hkv][P_cap][d], the shared prefix (P slots)
  const int32_t* ctx_len;
  T* O;
  float* lse;  // [L][B][Hq][T_new], log2 units (kernels with LSE)
  int B, T_new, L, Hq, Hkv, S_cap, P, P_cap, window, sinks, mask_paper, n_qtiles;
  int gs, gq, ctx_hi;
  float scale_log2;
  LayerTable chan, lord;  // lord: the consumers in channel order
  // partial states of the batch's rows over the prefix (FLAT): the channels with a reader and
  // their consumers, row tiles per slice, states per row, slots per split
  LayerTable live;
  ChannelGroups cg;
  float* part;
  int z, np, nsplit, split_len;
};

// The compact range of a tile whose rows' limits run from lim0 to kend (inclusive of both rows).
struct ReachSpan {
  int na, skip, n;   // WIN: first slots, slots left out after them, compact slots
  int low;           // a row reads x >= its limit - low (WIN) or x >= low (prefix)
  int first;         // ... or x < first
  int own;           // compact index of cache slot `skip` (prefix: the padded length)
};
constexpr int kReachBlk = 64;
template <typename T, bool PRE>
__device__ __forceinline__ ReachSpan reach_span(const ReachArgs<T>& a, int lim0, int kend) {
  ReachSpan r;
  if constexpr (PRE) {
    r.own = (a.P + kReachBlk - 1) / kReachBlk * kReachBlk;
    r.na = r.skip = 0;
    r.n = r.own + kend;
    r.low = r.own;
    r.first = a.P;
  } else {
    const int lo = max(lim0 - a.window, 0);
    r.na = min(a.sinks, lo);
    r.skip = lo - r.na;
    r.n = kend - r.skip;
    r.low = a.window;
    r.first = a.sinks;
    r.own = 0;
  }
  return r;
}

constexpr float kHidden = -__builtin_inff();  // a hidden slot's score: weight 0 at any reference

// Hides the slots of step i (32 from 32 i on) that this lane's row does not read: those at or
// past lim, and those below lo that are not below first.
__device__ __forceinline__ void reach_mask(f32x16& v, int i, int lim, int lo, int first, int lane) {
  const int base = 32 * i + 4 * (lane >> 5);
  lim -= base, lo -= base, first -= base;
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const int x = 8 * (q >> 2) + (q & 3);
    v[q] = x >= lim || (x < lo && x >= first) ? kHidden : v[q];
  }
}

template <int DH> struct ReachState {  // one wave's running softmax state (2 lanes per row)
  f32x16 o[DH / 32];  // O^T per 32-column tile of the values
  bf16x8 pf[2];       // P(i-1)^T fragments
  float m, lsum;      // reference (log2 units), sum of the weights
};

// One step of 32 slots: PV(i-1), S(i+1) and the weights of S(i) as independent work of one basic
// block, in DH / 16 groups whose LDS reads run one group ahead. sc: the raw scores of step i,
// sn: leaves holding those of step i + 1. LSE: the normaliser adds the weights before their
// rounding to bf16 (the row statistics are then exact to fp32); else the rounded ones, as the
// values are weighted.
template <int DH, bool LSE>
__device__ __forceinline__ void reach_step(const char* sm, const PfLane<DH>& lo, uint32_t kh_cur,
                                           uint32_t kh_nxt, uint32_t vh_prv, int i,
                                           const bf16x8 (&qf)[DH / 16], ReachState<DH>& st,
                                           f32x16& sc, f32x16& sn, float cl2, int lane, int lim,
                                           int rlo, int first, bool masked) {
  if (__builtin_expect(masked, 0)) reach_mask(sc, i, lim, rlo, first, lane);
  constexpr int NG = DH / 16, NDT = DH / 32;
  bf16x8 vf[2], kf[2];
  vf[0] = pf_ldv<DH>(sm, lo, vh_prv, 0, 0);
  kf[0] = pf_ldk<DH>(sm, lo, kh_nxt, 0);
  const float mm = -st.m;
  auto group = [&](auto gc) {
    constexpr int g = decltype(gc)::value;
    constexpr int q0 = (16 * g + NG - 1) / NG, q1 = (16 * (g + 1) + NG - 1) / NG;
    if constexpr (g + 1 < NG) {
      vf[(g + 1) & 1] = pf_ldv<DH>(sm, lo, vh_prv, (g + 1) / NDT, (g + 1) % NDT);
      kf[(g + 1) & 1] = pf_ldk<DH>(sm, lo, kh_nxt, g + 1);
    }
    st.o[g % NDT] = mma32(st.o[g % NDT], vf[g & 1], st.pf[g / NDT]);
    sn = mma32(g == 0 ? zero16() : sn, kf[g & 1], qf[g]);
#pragma unroll
    for (int q = q0; q < q1; ++q) sc[q] = fast_exp2(fmaf(sc[q], cl2, mm));
    __builtin_amdgcn_sched_barrier(0);
  };
  static_for<0, NG>(group);
#pragma unroll
  for (int q = 0; q < 16; ++q) st.pf[q >> 3][q & 7] = (bf16)sc[q];
  float ps = LSE ? tree_sum<0, 16>(sc) : pf_wsum(st.pf[0], st.pf[1]);
  if (__builtin_expect(__any(!(ps <= kGrowSum) || st.m == kNoRef), 0)) {
    // rare: the reference moves to the exact row maximum (never down, but from kNoRef to it)
    f32x16 sr = pf_scores<DH>(sm, lo, kh_cur, qf, zero16());
    if (masked) reach_mask(sr, i, lim, rlo, first, lane);
    float mx = sr[0];
#pragma unroll
    for (int q = 1; q < 16; ++q) mx = fmaxf(mx, sr[q]);
    const float grow = ref_growth(fmaf(halves_max(mx), cl2, -st.m), st.m);
    const float alpha = ref_rescale(grow, st.m);
    st.m += grow;
    st.lsum *= alpha;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) st.o[dt] *= alpha;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      sr[q] = fast_exp2(fmaf(sr[q], cl2, -st.m));
      st.pf[q >> 3][q & 7] = (bf16)sr[q];
    }
    ps = LSE ? tree_sum<0, 16>(sr) : pf_wsum(st.pf[0], st.pf[1]);
  }
  st.lsum += ps;
}

// One tile: 32 rows per wave of one (consumer, sequence, query head). On entry every wave is past
// the previous tile.
template <int DH, bool PRE, bool LSE>
__device__ __forceinline__ void reach_tile(const ReachArgs<bf16>& a, const int tile, char* smem) {
  using P = PfDma<1, DH>;
  constexpr int NKS = P::NKS, NDT = P::NDT;
  // tile order: sequence, KV head, consumer (in channel order), grouped head, query tile (last
  // first): consecutive tiles read neighbouring slots of one K/V slice
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.Hq / a.Hkv;
  const int qtile = a.n_qtiles - 1 - tile % a.n_qtiles;
  int y = tile / a.n_qtiles;
  const int hg = y % G;
  y /= G;
  const int li = y % a.L;
  y /= a.L;
  const int kvh = y % a.Hkv, b = y / a.Hkv;
  const int hq = kvh * G + hg, l = a.lord.v[li], c = a.chan.v[l];
  const int pos0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq;
  const int incl = a.mask_paper ? 0 : 1, gs = a.gs;
  const int q0 = qtile * P::BQ, qw0 = q0 + 32 * w, qi = qw0 + r;
  const float cl2 = a.scale_log2;

  bf16x8 qf[NKS];
  {
    const auto qview = make_view(a.Q + (((long)l * a.B + b) * a.Hq + hq) * (long)a.T_new * DH,
                                 (uint32_t)a.T_new * DH * 2u);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
      qf[ks] = buf_frag<bf16>(qview, qi < a.T_new ? (uint32_t)(qi * DH + 16 * ks + 8 * h) * 2u
                                                  : kOffOob);
  }
  bf16x8 kdv[NKS];
  bf16x4 vdv[NDT][4];
  {
    const long dof = ((long)c * a.Hkv + kvh) * DH;
    const uint32_t dbytes = a.mask_paper ? DH * 2u : 0u;
    const auto kdview = make_view(a.mask_paper ? a.Kd + dof : nullptr, dbytes);
    const auto vdview = make_view(a.mask_paper ? a.Vd + dof : nullptr, dbytes);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) kdv[ks] = buf_frag<bf16>(kdview, (16 * ks + 8 * h) * 2u);
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        vdv[dt][g4] = buf_ld8(vdview, (32 * dt + 8 * g4 + 4 * h) * 2u);
  }

  const int qlast = min(q0 + P::BQ, a.T_new) - 1;
  const int kend = min(pos0 + gs * qlast + incl, a.S_cap);  // cache slots the tile may see
  const ReachSpan sp = reach_span<bf16, PRE>(a, pos0 + gs * q0 + incl, kend);
  const int nblk = (sp.n + P::BKV - 1) / P::BKV;
  // compact limits: this lane's row, the wave's first and last row
  const int off = pos0 + incl + sp.own - sp.skip;
  const int lim = off + gs * qi, wlim0 = off + gs * qw0;
  const int wlast = min(qw0 + 31, a.T_new - 1), wlim1 = off + gs * wlast;
  const int rlo = PRE ? sp.low : lim - sp.low;
  const int wlo0 = PRE ? sp.low : wlim0 - sp.low, wlo1 = PRE ? sp.low : wlim1 - sp.low;
  // a step is unmasked where every row of the wave reads all of it
  auto masked = [&](int i) {
    return 32 * i + 32 > wlim0 || (32 * i < wlo1 && 32 * i + 32 > sp.first);
  };
  const int ilast = wlast >= qw0 ? (wlim1 + 31) / 32 - 1 : -2;  // the wave's last step
  // Steps that no row of the wave reads, between the first slots and its lowest window, are
  // skipped: it runs steps 0 .. a2 (the last one only to add the PV of the step before) and
  // starts again at step r0, with the scores of r0 taken anew.
  const int a2 = sp.first > 0 ? 2 * ((min(sp.first, sp.n) + 63) / 64) : 0;
  int r0 = PRE ? 0 : max(wlo0, 0) / 64 * 2;
  if (r0 <= a2 && a2 > 0) r0 = 0;
  const bool gap = r0 > 0;

  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  const auto kview = make_view(a.Kc + cbase, (uint32_t)max(kend, 0) * P::ROW_BYTES);
  const auto vview = make_view(a.Vc + cbase, (uint32_t)max(kend, 0) * P::ROW_BYTES);
  const long pbase = PRE ? ((long)c * a.Hkv + kvh) * (long)a.P_cap * DH : 0;
  const uint32_t pbytes = PRE ? (uint32_t)a.P * P::ROW_BYTES : 0u;
  const auto kpview = make_view(PRE ? a.Kp + pbase : nullptr, pbytes);
  const auto vpview = make_view(PRE ? a.Vp + pbase : nullptr, pbytes);
  const int pblk = sp.own / P::BKV;
  uint32_t coff[P::NI];  // byte offset of the lane's chunk within block 0
  int crow0[P::NI];
#pragma unroll
  for (int n = 0; n < P::NI; ++n) {
    const int ch = 64 * n + lane, crow = P::RPW * w + ch / P::CPR;
    crow0[n] = crow;
    coff[n] = (uint32_t)crow * P::ROW_BYTES + 16u * (uint32_t)((ch % P::CPR) ^ pf_swz<DH>(crow));
  }
  const uint32_t smem_base = (uint32_t)(uintptr_t)smem;
  // blocks past the range are copied as zeros, so that every wave issues the same sequence (K0
  // K1 V0 | K2 V1 | K3 V2 | ...) and one vmcnt fits every block
  auto issue = [&](int blk, bool v) {
    const bool pre = PRE && blk < pblk;
#pragma unroll
    for (int n = 0; n < P::NI; ++n) {
      uint32_t o = coff[n] + (uint32_t)(pre || !PRE ? blk : blk - pblk) * P::BLK_BYTES;
      if constexpr (!PRE)
        o += blk * P::BKV + crow0[n] >= sp.na ? (uint32_t)sp.skip * P::ROW_BYTES : 0u;
      const uint32_t lds = __builtin_amdgcn_readfirstlane(
          smem_base + (v ? P::V_BASE : 0) + (blk % P::NS) * P::BLK_BYTES +
          P::RPW * w * P::ROW_BYTES + 1024 * n);
      if constexpr (PRE) lds_dma16(lds, o, pre ? (v ? vpview : kpview) : (v ? vview : kview));
      else lds_dma16(lds, o, v ? vview : kview);
    }
  };
  static_assert(P::NS == 3, "the counts of copies in flight below");
  // the first step's PV has no block before it: its (weightless) values are zeros, not what an
  // earlier tile of another sequence left there
  for (int x = 16 * tid; x < 32 * P::ROW_BYTES; x += 16 * P::NT)
    *(i32x4*)(smem + pf_vh<DH>(2, 1) + x) = i32x4{0, 0, 0, 0};
  issue(0, false);
  issue(1, false);
  issue(0, true);

  ReachState<DH> st;
  f32x16 sa, sb;  // scores of even and odd steps
  st.pf[0] = st.pf[1] = zero_frag<bf16>();
  if (a.mask_paper) {
    float part = 0.f;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
      for (int i = 0; i < 8; ++i) part += (float)qf[ks][i] * (float)kdv[ks][i];
    st.m = halves_sum(part) * cl2;
    st.lsum = h == 0 ? 1.f : 0.f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int q = 0; q < 16; ++q) st.o[dt][q] = (float)vdv[dt][q >> 2][q & 3];
  } else {
    st.m = kNoRef;
    st.lsum = 0.f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) st.o[dt] = zero16();
  }
  sa = sb = zero16();
  wait_vmcnt<P::NI * 2>();
  __syncthreads();
  PfLane<DH> lo = pf_lane<DH>(lane);
  auto runs = [&](int i) { return i <= ilast + 1 && (!gap || i < a2 + (a2 > 0) || i >= r0); };
  auto block = [&](const int j, auto uc) {
    constexpr int u = decltype(uc)::value;
    // keep the lane offsets as they are (not one precomputed address per use)
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) asm volatile("" : "+v"(lo.k[ks]));
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) asm volatile("" : "+v"(lo.v[dt][0]), "+v"(lo.v[dt][1]));
    // every wave is past block j-1: the stages of K(j-1) and V(j-2) are free
    __syncthreads();
    issue(j + P::NS - 1, false);
    issue(j + P::NS - 2, true);
    const int i = 2 * j;
    if ((j == 0 || (gap && i == r0)) && i <= ilast)
      sa = pf_scores<DH>(smem, lo, pf_kh<DH>(u, 0), qf, zero16());
    // steps up to ilast + 1: the last one only adds PV(ilast)
    if (runs(i))
      reach_step<DH, LSE>(smem, lo, pf_kh<DH>(u, 0), pf_kh<DH>(u, 1),
                          pf_vh<DH>((u + P::NS - 1) % P::NS, 1), i, qf, st, sa, sb, cl2, lane, lim,
                          rlo, sp.first, masked(i));
    wait_vmcnt<2 * P::NI>();  // K(j+1) and V(j) have landed
    __syncthreads();
    if (runs(i + 1))
      reach_step<DH, LSE>(smem, lo, pf_kh<DH>(u, 1), pf_kh<DH>((u + 1) % P::NS, 0), pf_vh<DH>(u, 0),
                          i + 1, qf, st, sb, sa, cl2, lane, lim, rlo, sp.first, masked(i + 1));
  };
  for (int j = 0; j < nblk; j += P::NS) {
    block(j, std::integral_constant<int, 0>());
    if (j + 1 < nblk) block(j + 1, std::integral_constant<int, 1>());
    if (j + 2 < nblk) block(j + 2, std::integral_constant<int, 2>());
  }
  if (ilast + 1 == 2 * nblk && runs(2 * nblk)) {
    const int u = nblk % P::NS;
    reach_step<DH, LSE>(smem, lo, pf_kh<DH>(u, 0), pf_kh<DH>(u, 1),
                        pf_vh<DH>((u + P::NS - 1) % P::NS, 1), 2 * nblk, qf, st, sa, sb, cl2, lane,
                        lim, rlo, sp.first, true);
  }
  wait_vmcnt<0>();  // no copy may land after the workgroup ends

  const float lt = halves_sum(st.lsum);
  if (qi < a.T_new) {
    const float inv = 1.0f / lt;
    bf16* dst = a.O + ((((long)l * a.B + b) * a.T_new + qi) * a.Hq + hq) * DH;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = st.o[dt][4 * g + i] * inv;
        store4(dst + 32 * dt + 8 * g + 4 * h, v);
      }
    if (LSE && h == 0)
      a.lse[(((long)l * a.B + b) * a.Hq + hq) * a.T_new + qi] = st.m + __log2f(lt);
  }
}

// The place of the t-th tile taken of a share of `count`, which lie head by head (or slice by slice)
// with n tiles each, longest first: in that order, but the last heads that hold `last` tiles
// give all their longest ones first, then the next ones, so that no long tile starts when the
// others end. (All heads this way would read the K and V of all at once: 2 x 2048 tokens, 24 layers
// of 16 heads of 64, no window, 530 us in order, 550 so. Four tiles per workgroup in the
// last heads, in order / so: 2 x 1023 tokens of weighed attention 137 / 133, 4001 tokens of
// 12 layers of 12 heads 379 / 366, under a window of 1024 215 / 211.)
__device__ __forceinline__ int long_first(int t, int count, int n, int last) {
  const int nb = min(count / n, (last + n - 1) / n), v = t - (count - nb * n);
  return v < 0 ? t : t - v + v % nb * n + v / nb;
}

// Grid and work queue as the prefill kernel's (attend_prefill_dma_kernel): one workgroup per tile
// where the CUs hold them all at once, else as many as they hold, each XCD's taking tiles of its
// contiguous share from a counter (queue, reset on the stream before).
template <int DH, bool PRE, bool LSE>
__global__ __launch_bounds__(64 * kPfWaves) __attribute__((amdgpu_waves_per_eu(DH == 64 ? 3 : 2)))
void reach_dma_kernel(ReachArgs<bf16> a, uint32_t* queue) {
  using P = PfDma<1, DH>;
  __shared__ __align__(16) char smem[P::SMEM_BYTES];
  __shared__ int s_tile;
  const int tid = threadIdx.x;
  const int total = a.n_qtiles * a.Hq * a.B * a.L;
  if (!queue) {
    reach_tile<DH, PRE, LSE>(a, xcd_tile(blockIdx.x, total), smem);
    return;
  }
  const int nq = min((int)gridDim.x, kNumXcd), x = blockIdx.x % nq;
  const int per = total / nq, rem = total % nq;
  const int first = x * per + min(x, rem), count = per + (x < rem ? 1 : 0);
  uint32_t* ctr = queue + kQueueStride * x;
  if (tid == 0) s_tile = (int)atomicAdd(ctr, 1u);
  __syncthreads();
  int t = __builtin_amdgcn_readfirstlane(s_tile);
  while (t < count) {
    // (a prefix's tiles are alike but for their own slots: no use in turning their order)
    reach_tile<DH, PRE, LSE>(
        a, first + (PRE ? t : long_first(t, count, a.n_qtiles, 4 * (int)(gridDim.x / nq))), smem);
    if (tid == 0) s_tile = (int)atomicAdd(ctr, 1u);
    __syncthreads();
    t = __builtin_amdgcn_readfirstlane(s_tile);
  }
}

__global__ void reach_queue_kernel(uint32_t* queue) { queue[threadIdx.x] = 0u; }

// ------------------------------------------------ bf16, head dims 64 and 96, few rows per head
// A workgroup takes 32 rows of one head and its four waves cut the compact slots between them, as
// attend_tile_kernel does (wm_tile.hip): blocks of 32 slots go round the waves, each with a ring
// of two in LDS of its own, and the waves' states meet in LDS once. A 128-row tile would leave
// three or two of its four waves without rows, and walk its range as one chain. Slot x of a block
// is found per row of the block, so first slots and window need not start at a block's edge. Times
// beside the rule that chooses it.
template <int DH, bool PRE, bool LSE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void reach_few_kernel(ReachArgs<bf16> a) {
  constexpr int NW = 4, NKS = DH / 16, NDT = DH / 32, ROW = 2 * DH, CPR = ROW / 16, BKV = 32;
  constexpr int BLK = BKV * ROW, NI = BLK / 1024, STAGE = 2 * BLK, RING = 2 * STAGE;
  constexpr int OLD = DH + 4;  // row stride of the merge staging (floats)
  static_assert(32 * OLD * 4 + 256 <= RING, "the merge staging fits a wave's ring");
  __shared__ __align__(16) char smem[NW * RING];
  const int tile = xcd_tile(blockIdx.x, (int)gridDim.x);
  const int qtile = a.n_qtiles - 1 - tile % a.n_qtiles;
  const int G = a.Hq / a.Hkv;
  int y = tile / a.n_qtiles;
  const int hg = y % G;
  y /= G;
  const int li = y % a.L;
  y /= a.L;
  const int kvh = y % a.Hkv, b = y / a.Hkv;
  const int hq = kvh * G + hg, l = a.lord.v[li], c = a.chan.v[l];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pos0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq;
  const int incl = a.mask_paper ? 0 : 1, gs = a.gs;
  const float cl2 = a.scale_log2;
  const int q0 = qtile * 32, qi = q0 + r, qlast = min(q0 + 32, a.T_new) - 1;
  const int kend = min(pos0 + gs * qlast + incl, a.S_cap);
  const ReachSpan sp = reach_span<bf16, PRE>(a, pos0 + gs * q0 + incl, kend);
  const int off = pos0 + incl + sp.own - sp.skip;
  const int lim = off + gs * min(qi, a.T_new - 1), wlim0 = off + gs * q0, wlim1 = off + gs * qlast;
  const int rlo = PRE ? sp.low : lim - sp.low, wlo1 = PRE ? sp.low : wlim1 - sp.low;
  const int nblk = (sp.n + BKV - 1) / BKV, nw = (nblk - w + NW - 1) / NW;

  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  const auto kview = make_view(a.Kc + cbase, (uint32_t)max(kend, 0) * ROW);
  const auto vview = make_view(a.Vc + cbase, (uint32_t)max(kend, 0) * ROW);
  const long pbase = PRE ? ((long)c * a.Hkv + kvh) * (long)a.P_cap * DH : 0;
  const uint32_t pbytes = PRE ? (uint32_t)a.P * ROW : 0u;
  const auto kpview = make_view(PRE ? a.Kp + pbase : nullptr, pbytes);
  const auto vpview = make_view(PRE ? a.Vp + pbase : nullptr, pbytes);
  uint32_t coff[NI];
#pragma unroll
  for (int n = 0; n < NI; ++n) {
    const int ch = 64 * n + lane, row = ch / CPR;
    coff[n] = (uint32_t)row * ROW + 16u * (uint32_t)((ch % CPR) ^ pf_swz<DH>(row));
  }
  char* ring = smem + w * RING;
  const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
  // block j of this wave into stage st (past the wave's last: zeros, so that the copies in flight
  // are the same number at every wait)
  auto issue = [&](int j, int st) {
    const int at = BKV * (w + NW * j);
    const bool pre = PRE && at < sp.own;
    const uint32_t base = j < nw ? (uint32_t)(PRE && !pre ? at - sp.own : at) * ROW : kOffOob;
#pragma unroll
    for (int n = 0; n < 2 * NI; ++n) {
      uint32_t o = base + coff[n % NI];
      if constexpr (!PRE)
        o += j < nw && at + (64 * (n % NI) + lane) / CPR >= sp.na ? (uint32_t)sp.skip * ROW : 0u;
      const uint32_t to = __builtin_amdgcn_readfirstlane(ring_at + st * STAGE + 1024 * n);
      if constexpr (PRE) lds_dma16(to, o, pre ? (n < NI ? kpview : vpview) : (n < NI ? kview : vview));
      else lds_dma16(to, o, n < NI ? kview : vview);
    }
  };

  bf16x8 qf[NKS];
  const auto qv = make_view(a.Q + (((long)l * a.B + b) * a.Hq + hq) * (long)a.T_new * DH,
                            (uint32_t)a.T_new * ROW);
  const bool dummy = a.mask_paper && w == 0;
  const long dof = ((long)c * a.Hkv + kvh) * DH;
  const auto kdv = make_view(dummy ? a.Kd + dof : nullptr, dummy ? ROW : 0u);
  const auto vdv = make_view(dummy ? a.Vd + dof : nullptr, dummy ? ROW : 0u);
  float part = 0.f;
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) {
    const uint32_t col = (uint32_t)(16 * ks + 8 * h) * 2u;
    qf[ks] = buf_frag<bf16>(qv, qi < a.T_new ? (uint32_t)qi * ROW + col : kOffOob);
    const bf16x8 kd = buf_frag<bf16>(kdv, col);
#pragma unroll
    for (int i = 0; i < 8; ++i) part += (float)qf[ks][i] * (float)kd[i];
  }
  f32x16 o[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const bf16x4 vd = buf_ld8(vdv, (32 * dt + 8 * g + 4 * h) * 2u);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[dt][4 * g + i] = (float)vd[i];
    }
  float m = dummy ? halves_sum(part) * cl2 : kNoRef, lsum = dummy && h == 0 ? 1.f : 0.f;

  const PfLane<DH> lo = pf_lane<DH>(lane);
  issue(0, 0);
  int j = 0;
  do {  // (a wave without a block walks one of zeros, every slot of it hidden)
    const int st = j & 1;
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the stage refilled next is read
    issue(j + 1, st ^ 1);
    wait_copies<2 * NI>();
    const uint32_t kh = st * STAGE, vh = kh + BLK;
    const int at = BKV * (w + NW * j);
    const bool masked = at + BKV > wlim0 || (at < wlo1 && at + BKV > sp.first);
    auto scores = [&]() {
      f32x16 s = zero16();
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) s = mma32(s, pf_ldk<DH>(ring, lo, kh, ks), qf[ks]);
      if (masked) reach_mask(s, at / 32, j < nw ? lim : 0, rlo, j < nw ? sp.first : 0, lane);
      return s;
    };
    f32x16 p = scores();
#pragma unroll
    for (int q = 0; q < 16; ++q) p[q] = fast_exp2(fmaf(p[q], cl2, -m));
    bf16x8 pf[2];
#pragma unroll
    for (int q = 0; q < 16; ++q) pf[q >> 3][q & 7] = (bf16)p[q];
    float ps = LSE ? tree_sum<0, 16>(p) : pf_wsum(pf[0], pf[1]);
    if (__builtin_expect(__any(!(ps <= kGrowSum) || m == kNoRef), 0)) {
      p = scores();
      float mx = p[0];
#pragma unroll
      for (int q = 1; q < 16; ++q) mx = fmaxf(mx, p[q]);
      const float grow = ref_growth(fmaf(halves_max(mx), cl2, -m), m), alpha = ref_rescale(grow, m);
      m += grow;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        p[q] = fast_exp2(fmaf(p[q], cl2, -m));
        pf[q >> 3][q & 7] = (bf16)p[q];
      }
      ps = LSE ? tree_sum<0, 16>(p) : pf_wsum(pf[0], pf[1]);
    }
    lsum += ps;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) o[dt] = mma32(o[dt], pf_ldv<DH>(ring, lo, vh, hf, dt), pf[hf]);
  } while (++j < nw);
  wait_copies<0>();  // no copy may land in the staging below, or after the block ends

  // merge the waves' states: each writes its rows [r][DH] and (m, l) to its own ring
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
  float* so = (float*)ring;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = o[dt][4 * g + i];
      *(f32x4*)(so + r * OLD + 32 * dt + 8 * g + 4 * h) = v;
    }
  const float lt = halves_sum(lsum);
  if (h == 0) {
    so[32 * OLD + 2 * r] = m;
    so[32 * OLD + 2 * r + 1] = lt;
  }
  __syncthreads();
  constexpr int C4 = DH / 4;
  for (int e = tid; e < 32 * C4; e += 64 * NW) {
    const int row = e / C4, d4 = 4 * (e - row * C4);
    if (q0 + row >= a.T_new) break;  // rows only grow
    float M = kNegBig;  // of the waves that saw a slot
#pragma unroll
    for (int ww = 0; ww < NW; ++ww) {
      const float* ml = (const float*)(smem + ww * RING) + 32 * OLD + 2 * row;
      M = ml[1] > 0.f ? fmaxf(M, ml[0]) : M;
    }
    float lw = 0.f, ow[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ww = 0; ww < NW; ++ww) {
      const float* sw = (const float*)(smem + ww * RING);
      const float lx = sw[32 * OLD + 2 * row + 1];
      const float al = lx > 0.f ? fast_exp2(sw[32 * OLD + 2 * row] - M) : 0.f;
      lw += lx * al;
      const f32x4 ov = *(const f32x4*)(sw + row * OLD + d4);
#pragma unroll
      for (int i = 0; i < 4; ++i) ow[i] += ov[i] * al;
    }
    const float inv = 1.0f / lw;
#pragma unroll
    for (int i = 0; i < 4; ++i) ow[i] *= inv;
    store4(a.O + ((((long)l * a.B + b) * a.T_new + q0 + row) * a.Hq + hq) * DH + d4, ow);
    if (LSE && d4 == 0)
      a.lse[(((long)l * a.B + b) * a.Hq + hq) * a.T_new + q0 + row] = M + __log2f(lw);
  }
}

// ------------------------------------------- fp32, and bf16 at head dim 32
// The same tiles without the pipeline: 256 rows per workgroup (8 waves of 32), K and V blocks of
// 64 slots double-buffered in LDS through registers, V transposed for fp32 (whose matrix
// instructions have no transposing read). fp32 products run on the fp32 matrix cores, a sixteenth of
// the bf16 rate, which bounds this form. Calls of at most 64 rows per head take 4 waves, two for the
// rows, each pair cutting a block's slots (SW = 2; their states meet in LDS): 5 sequences x 37
// tokens over 777 + 50 slots, 12 layers of 12 heads of 64, 197 us with 8 waves of which two had
// rows, 122 so. FLAT: the rows are the batch's rows of one (channel, KV
// head) side by side, the slots a split of the prefix, the result a partial state per row.
template <typename T, int DH, int SW_> struct ReachCfg {
  static constexpr int SW = SW_, NW = SW == 2 ? 4 : 8, NT = 64 * NW, RW = NW / SW;
  static constexpr int BQ = 32 * RW, BKV = 64;
  typedef PrefillCfg<T, DH> P;
  static constexpr int LDK = P::LDK, LDV = P::LDV, VS = P::VS, NKS = P::NKS, NDT = P::NDT;
  static constexpr bool VTR = P::VTR;
  static constexpr int KIT = P::KIT, VIT = P::VIT;  // fragments (V: or key pairs) of a block
  static constexpr int KFR = (KIT + NT - 1) / NT, VPT = (VIT + NT - 1) / NT;  // ... per thread
  static_assert(SW == 1 || RW * 32 * (DH + 2) * 4 <= 2 * BKV * LDK * (int)sizeof(T),
                "the merge staging fits the K blocks");
};
template <typename T, int DH, bool PRE, bool LSE, bool FLAT = false, int SW = 1>
__global__ __launch_bounds__(SW == 2 ? 256 : 512) void reach_prefill_kernel(ReachArgs<T> a) {
  using C = ReachCfg<T, DH, SW>;
  __shared__ __align__(16) T Ks[2][C::BKV * C::LDK];
  __shared__ __align__(16) T Vt[2][C::VS];
  const int tile = xcd_tile(blockIdx.x, (int)gridDim.x);
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  // this wave's rows, and (SW = 2) its half of every block
  const int w = (tid >> 6) % C::RW, phase = (tid >> 6) / C::RW;
  const float cl2 = a.scale_log2;
  int l = 0, b = 0, hq = 0, kvh, c, q0, kend = 0, split = 0, rows = a.T_new;
  int off = 0, lim, wlim0, wlim1, rlo, wlo0, wlo1;
  ReachSpan sp{};
  long qrow = 0;  // this lane's row of Q
  if constexpr (FLAT) {
    int y = tile / a.z;
    q0 = tile % a.z * C::BQ;
    split = y % a.np;
    y /= a.np;
    kvh = y % a.Hkv;
    const int ci = y / a.Hkv, grp = a.Hq / a.Hkv;
    c = a.live.v[ci];
    const int per_b = (a.cg.offsets[ci + 1] - a.cg.offsets[ci]) * grp * a.T_new;
    rows = per_b * a.B;
    if (q0 >= rows) return;
    const int g = min(q0 + 32 * w + r, rows - 1), x = g % per_b, gl = x / a.T_new;
    const int ml = a.cg.members[a.cg.offsets[ci] + gl / grp];
    qrow = (((long)ml * a.B + g / per_b) * a.Hq + kvh * grp + gl % grp) * a.T_new + x % a.T_new;
    sp.own = (a.P + kReachBlk - 1) / kReachBlk * kReachBlk;  // every slot walked is the prefix's
    sp.n = lim = wlim0 = wlim1 = min((split + 1) * a.split_len, a.P);
    rlo = wlo0 = wlo1 = 0;
  } else {
    const int qtile = a.n_qtiles - 1 - tile % a.n_qtiles;
    int y = tile / a.n_qtiles;
    hq = y % a.Hq;
    y /= a.Hq;
    b = y % a.B, l = y / a.B;
    c = a.chan.v[l], kvh = hq / (a.Hq / a.Hkv);
    q0 = qtile * C::BQ;
    qrow = (((long)l * a.B + b) * a.Hq + hq) * a.T_new + min(q0 + 32 * w + r, a.T_new - 1);
    const int pos0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq;
    const int incl = a.mask_paper ? 0 : 1, gs = a.gs;
    const int qlast = min(q0 + C::BQ, a.T_new) - 1;
    kend = min(pos0 + gs * qlast + incl, a.S_cap);
    sp = reach_span<T, PRE>(a, pos0 + gs * q0 + incl, kend);
    off = pos0 + incl + sp.own - sp.skip;
    const int wl = q0 + 32 * w;
    lim = off + gs * (wl + r), wlim0 = off + gs * wl;
    wlim1 = off + gs * min(wl + 31, a.T_new - 1);
    rlo = PRE ? sp.low : lim - sp.low;
    wlo0 = PRE ? sp.low : wlim0 - sp.low, wlo1 = PRE ? sp.low : wlim1 - sp.low;
  }
  const int qw0 = q0 + 32 * w, qi = qw0 + r;
  const int j0 = FLAT ? split * a.split_len / C::BKV : 0, nblk = (sp.n + C::BKV - 1) / C::BKV;
  const bool live = qw0 < rows;

  frag_t<T> qf[C::NKS];
#pragma unroll
  for (int ks = 0; ks < C::NKS; ++ks)
    qf[ks] = qi < rows ? ld_frag<T>(a.Q + qrow * DH + 16 * ks + 8 * h) : zero_frag<T>();
  float m = kNoRef, lsum = 0.f;
  f32x16 o[C::NDT];
#pragma unroll
  for (int dt = 0; dt < C::NDT; ++dt) o[dt] = zero16();
  if (!FLAT && a.mask_paper && phase == 0) {
    const T* kd = a.Kd + ((long)c * a.Hkv + kvh) * DH;
    const T* vd = a.Vd + ((long)c * a.Hkv + kvh) * DH;
    float part = 0.f;
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks)
#pragma unroll
      for (int i = 0; i < 8; ++i) part += to_f32(qf[ks][i]) * to_f32(kd[16 * ks + 8 * h + i]);
    m = halves_sum(part) * cl2;
    lsum = h == 0 ? 1.f : 0.f;
#pragma unroll
    for (int dt = 0; dt < C::NDT; ++dt)
#pragma unroll
      for (int q = 0; q < 16; ++q) o[dt][q] = to_f32(vd[32 * dt + 8 * (q >> 2) + 4 * h + (q & 3)]);
  }

  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  const auto kview = make_view(FLAT ? nullptr : a.Kc + cbase,
                               FLAT ? 0u : (uint32_t)a.S_cap * DH * sizeof(T));
  const auto vview = make_view(FLAT ? nullptr : a.Vc + cbase,
                               FLAT ? 0u : (uint32_t)a.S_cap * DH * sizeof(T));
  const long pbase = PRE ? ((long)c * a.Hkv + kvh) * (long)a.P_cap * DH : 0;
  const uint32_t pbytes = PRE ? (uint32_t)a.P * DH * sizeof(T) : 0u;
  const auto kpview = make_view(PRE ? a.Kp + pbase : nullptr, pbytes);
  const auto vpview = make_view(PRE ? a.Vp + pbase : nullptr, pbytes);
  frag_t<T> kreg[C::KFR], vreg[C::VPT][C::VTR ? 1 : 2];
  // compact slot x of a block that lies in the prefix (pre) or in the cache
  auto slot_off = [&](int x, int col, bool pre) {
    const int s = PRE ? (pre ? x : x - sp.own) : x < sp.na ? x : x + sp.skip;
    const bool ok = PRE && pre ? s < a.P : s < kend;
    return ok ? (uint32_t)(s * DH + col) * (uint32_t)sizeof(T) : kOffOob;
  };
  auto fetch = [&](int k0) {
    const bool pre = PRE && k0 < sp.own;
    const auto kv = PRE && pre ? kpview : kview, vv = PRE && pre ? vpview : vview;
#pragma unroll
    for (int i = 0; i < C::KFR; ++i) {
      const int f = tid + C::NT * i, key = f / (DH / 8), dc = (f % (DH / 8)) * 8;
      kreg[i] = buf_frag<T>(kv, f < C::KIT ? slot_off(k0 + key, dc, pre) : kOffOob);
    }
#pragma unroll
    for (int i = 0; i < C::VPT; ++i) {
      const int it = tid + C::NT * i;
      const bool ok = it < C::VIT;
      if constexpr (C::VTR) {
        const int key = it / (DH / 8), dc = (it % (DH / 8)) * 8;
        vreg[i][0] = buf_frag<T>(vv, ok ? slot_off(k0 + key, dc, pre) : kOffOob);
      } else {
        const int kp = it % (C::BKV / 2), dg = it / (C::BKV / 2), x = k0 + 2 * kp;
        vreg[i][0] = buf_frag<T>(vv, ok ? slot_off(x, 8 * dg, pre) : kOffOob);
        vreg[i][1] = buf_frag<T>(vv, ok ? slot_off(x + 1, 8 * dg, pre) : kOffOob);
      }
    }
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int i = 0; i < C::KFR; ++i) {
      const int f = tid + C::NT * i, key = f / (DH / 8), dc = (f % (DH / 8)) * 8;
      if (f < C::KIT) st_frag<T>(&Ks[buf][key * C::LDK + dc], kreg[i]);
    }
#pragma unroll
    for (int i = 0; i < C::VPT; ++i) {
      const int it = tid + C::NT * i;
      if (it < C::VIT) {
        if constexpr (C::VTR) {
          const int key = it / (DH / 8), dc = (it % (DH / 8)) * 8;
          st_frag<T>(&Vt[buf][key * C::LDV + dc], vreg[i][0]);
        } else {
          const int kp = it % (C::BKV / 2), dg = it / (C::BKV / 2);
          st_pair_t(&Vt[buf][(8 * dg) * C::LDV + 2 * kp], C::LDV, vreg[i][0], vreg[i][1]);
        }
      }
    }
  };
  // half a block (32 slots from x0 on) against the wave's rows
  auto half = [&](int x0, int kt, const T* ks_, const T* vt_) {
    f32x16 sc = zero16();
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks)
      sc = mma32(sc, ld_frag<T>(ks_ + (32 * kt + r) * C::LDK + 16 * ks + 8 * h), qf[ks]);
    if (x0 + 32 > wlim0 || (x0 < wlo1 && x0 + 32 > sp.first))
      reach_mask(sc, x0 / 32, lim, rlo, sp.first, lane);
    f32x16 pv;
#pragma unroll
    for (int q = 0; q < 16; ++q) pv[q] = fast_exp2(fmaf(sc[q], cl2, -m));
    float ps = tree_sum<0, 16>(pv);
    if (__any(!(ps <= kGrowSum) || m == kNoRef)) {  // rare, as in the pipelined form
      float mx = sc[0];
#pragma unroll
      for (int q = 1; q < 16; ++q) mx = fmaxf(mx, sc[q]);
      const float grow = ref_growth(fmaf(halves_max(mx), cl2, -m), m);
      const float alpha = ref_rescale(grow, m);
      m += grow;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < C::NDT; ++dt) o[dt] *= alpha;
#pragma unroll
      for (int q = 0; q < 16; ++q) pv[q] = fast_exp2(fmaf(sc[q], cl2, -m));
      ps = tree_sum<0, 16>(pv);
    }
    lsum += ps;
    // bf16: the few tokens of FLAT calls keep the weights' 24 bits, as their other slots do
    constexpr int NP = FLAT && sizeof(T) == 2 ? 3 : 1;
    frag_t<T> pf[NP][2];
    if constexpr (NP == 3) {
      cut24(pv, pf);
    } else {
#pragma unroll
      for (int q = 0; q < 16; ++q) pf[0][q >> 3][q & 7] = from_f32<T>(pv[q]);
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int kc = 32 * kt + 16 * hf + 4 * h;
#pragma unroll
      for (int dt = 0; dt < C::NDT; ++dt) {
        frag_t<T> vf;
        if constexpr (C::VTR) {
          vf = ld_vt_tr(vt_, C::LDV, 32 * kt + 16 * hf, dt, 32 * h + r);
        } else {
          const T* vrow = vt_ + (32 * dt + r) * C::LDV;
          vf = ld_frag_4_4<T>(vrow + kc, vrow + kc + 8);
        }
#pragma unroll
        for (int u = 0; u < NP; ++u) o[dt] = mma32(o[dt], vf, pf[u][hf]);
      }
    }
  };
  fetch(j0 * C::BKV);
  stage(j0 & 1);
  __syncthreads();
  for (int j = j0; j < nblk; ++j) {
    const int k0 = j * C::BKV, buf = j & 1;
    fetch(k0 + C::BKV);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int x0 = k0 + 32 * kt;
      // wave-uniform: some row may read some of the 32 slots
      if (live && (SW == 1 || kt == phase) && x0 < wlim1 && (x0 + 32 > wlo0 || x0 < sp.first)) half(x0, kt, Ks[buf], Vt[buf]);
    }
    stage(buf ^ 1);
    __syncthreads();
  }
  float lt = halves_sum(lsum);
  if constexpr (SW == 2) {  // the second half's state joins the first's (every wave is past the loop)
    float* so = (float*)&Ks[0][0] + w * 32 * (DH + 2) + r * (DH + 2);
    if (phase == 1) {
#pragma unroll
      for (int dt = 0; dt < C::NDT; ++dt)
#pragma unroll
        for (int q = 0; q < 16; ++q) so[32 * dt + 8 * (q >> 2) + 4 * h + (q & 3)] = o[dt][q];
      if (h == 0) so[DH] = m, so[DH + 1] = lt;
    }
    __syncthreads();
    if (phase == 1) return;
    const float m2 = so[DH], l2 = so[DH + 1];
    const float M = l2 > 0.f && (m2 > m || !(lt > 0.f)) ? m2 : m;
    const float f1 = lt > 0.f ? fast_exp2(m - M) : 0.f, f2 = l2 > 0.f ? fast_exp2(m2 - M) : 0.f;
    lt = lt * f1 + l2 * f2;
    m = M;
#pragma unroll
    for (int dt = 0; dt < C::NDT; ++dt)
#pragma unroll
      for (int q = 0; q < 16; ++q)
        o[dt][q] = o[dt][q] * f1 + so[32 * dt + 8 * (q >> 2) + 4 * h + (q & 3)] * f2;
  }
  if (qi >= rows) return;
  if constexpr (FLAT) {  // the decode kernels' partial state: o unnormalised, m in score units, l
    float* dst = a.part + (qrow * a.nsplit + split) * (DH + 2);
#pragma unroll
    for (int dt = 0; dt < C::NDT; ++dt)
#pragma unroll
      for (int q = 0; q < 16; ++q) dst[32 * dt + 8 * (q >> 2) + 4 * h + (q & 3)] = o[dt][q];
    if (h == 0) {
      dst[DH] = m / cl2;
      dst[DH + 1] = lt;
    }
    return;
  }
  const float inv = 1.0f / lt;
  T* dst = a.O + ((((long)l * a.B + b) * a.T_new + qi) * a.Hq + hq) * DH;
#pragma unroll
  for (int dt = 0; dt < C::NDT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = o[dt][4 * g + i] * inv;
      store4(dst + 32 * dt + 8 * g + 4 * h, v);
    }
  if (LSE && h == 0) a.lse[(((long)l * a.B + b) * a.Hq + hq) * a.T_new + qi] = m + __log2f(lt);
}

// ---------------------------------------------------------------- weights of longer calls
// weight[c][b][kvh][s] += the sum over the rows that read the slot of exp2(score - lse). A workgroup
// takes 32 CT slots of one slice, whose K rows stay in registers, and its four waves cut the rows
// (32 at a time: a consumer's head's query block): S^T = K Q^T puts one row and 16 slots in a lane,
// so a step adds 16 exponentials per slot tile to the lane's sums, and the rows meet across lanes
// and waves once, at the end, in a fixed order. Query fragments come straight from memory: the
// waves of a CU read the same few blocks (L1 and L2), each for CT slot tiles.
template <typename T, int DH>
__global__ __launch_bounds__(256) void reach_weigh_kernel(ReachArgs<T> a, ChannelGroups cg,
                                                          float* weight) {
  constexpr int NKS = DH / 16, CT = 2;
  __shared__ float s_w[4][32 * CT];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the slot tiles of a slice, which read the same queries, on one XCD
  const int tile = xcd_tile(blockIdx.x, (int)gridDim.x), slice = tile / a.n_qtiles;
  const int kvh = slice % a.Hkv, b = slice / a.Hkv % a.B, c = slice / a.Hkv / a.B;
  const int p0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq +
                 (a.mask_paper ? 0 : 1);  // row i reads slots below p0 + gs i
  const int kend = min(p0 + a.gs * (a.T_new - 1), a.S_cap);
  const int sb = 32 * CT * (tile % a.n_qtiles), G = a.Hq / a.Hkv;
  const int nh = (cg.offsets[c + 1] - cg.offsets[c]) * G;
  if (sb >= kend || nh == 0) return;
  const float cl2 = a.scale_log2;
  const long cbase = ((long)slice * a.S_cap) * DH;
  const auto kview = make_view(a.Kc + cbase, (uint32_t)kend * DH * sizeof(T));
  frag_t<T> kf[CT][NKS];
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
      kf[t][ks] = buf_frag<T>(kview, (uint32_t)((sb + 32 * t + r) * DH + 16 * ks + 8 * h) *
                                         (uint32_t)sizeof(T));
  f32x16 acc[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) acc[t] = zero16();
  // the first row that reads slot sb, rounded down to a block; steps go head by head
  const int i_num = sb - p0, qb0 = (i_num < 0 ? 0 : i_num / a.gs + 1) / 32;
  const int nqb = (a.T_new + 31) / 32 - qb0, nst = nh * nqb;
  frag_t<T> qn[NKS];
  float lse_n = 0.f;
  int qi_n = 0;
  auto fetch = [&](int st) {
    const int x = st / nqb, l = cg.members[cg.offsets[c] + x / G];
    const long row0 = (((long)l * a.B + b) * a.Hq + kvh * G + x % G) * a.T_new;
    qi_n = 32 * (qb0 + st % nqb) + r;
    const auto qview = make_view(a.Q + row0 * DH, (uint32_t)a.T_new * DH * (uint32_t)sizeof(T));
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
      qn[ks] = buf_frag<T>(qview, (uint32_t)(qi_n * DH + 16 * ks + 8 * h) * (uint32_t)sizeof(T));
    lse_n = qi_n < a.T_new ? a.lse[row0 + qi_n] : 0.f;
  };
  if (w < nst) fetch(w);
  for (int st = w; st < nst; st += 4) {
    frag_t<T> qf[NKS];
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = qn[ks];
    const float nl = -lse_n;
    const int qi = qi_n;
    if (st + 4 < nst) fetch(st + 4);
    const int lim = qi < a.T_new ? p0 + a.gs * qi : 0;  // (rows past the last read nothing)
    const int q0 = 32 * (qb0 + st % nqb);
    const bool all = q0 + 32 <= a.T_new && p0 + a.gs * q0 >= sb + 32 * CT;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      f32x16 sc = zero16();
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) sc = mma32(sc, kf[t][ks], qf[ks]);
      if (!all) {
        const int at = sb + 32 * t + 4 * h;
#pragma unroll
        for (int q = 0; q < 16; ++q) sc[q] = at + 8 * (q >> 2) + (q & 3) < lim ? sc[q] : kHidden;
      }
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[t][q] += fast_exp2(fmaf(sc[q], cl2, nl));
    }
  }
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      float v = acc[t][q];
#pragma unroll
      for (int x = 1; x < 32; x <<= 1) v += __shfl_xor(v, x, 64);
      if (r == 0) s_w[w][32 * t + 8 * (q >> 2) + 4 * h + (q & 3)] = v;
    }
  __syncthreads();
  if (tid < 32 * CT && sb + tid < kend) {
    float* dst = weight + (long)slice * a.S_cap + sb + tid;
    *dst += (s_w[0][tid] + s_w[1][tid]) + (s_w[2][tid] + s_w[3][tid]);
  }
}

// bf16 at head dims 64 and 96: the same with the query blocks copied into a ring of three in LDS per
// wave (fragments loaded from memory touch 32 lines an instruction, which the CU's L1 looks up one
// by one), two score sets in turn, and the slot tiles of a slice on one XCD, whose L2 then serves
// its queries to all of them, the longest ones of the last slices first. 2 x 1023 tokens, 16 layers
// of 6/3 heads of 96: 53 us; slice by slice 62, with the tiles over the XCDs 81, from memory 77.
template <int DH>
__global__ __launch_bounds__(256) void reach_weigh_dma_kernel(ReachArgs<bf16> a, ChannelGroups cg,
                                                              float* weight) {
  constexpr int NKS = DH / 16, CT = 2, NS = 3, ROW = 2 * DH, CPR = ROW / 16;
  constexpr int BLK = 32 * ROW, NI = BLK / 1024, STAGE = BLK + 256, RING = NS * STAGE;
  __shared__ __align__(16) char smem[4 * RING];
  __shared__ float s_w[4][32 * CT];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the slot tiles of a slice, which read the same queries, on one XCD
  const int nq = min((int)gridDim.x, kNumXcd), share = (int)gridDim.x / nq;
  int tile = xcd_tile(blockIdx.x, (int)gridDim.x);
  if ((int)gridDim.x % nq == 0)
    tile = tile / share * share + long_first(tile % share, share, a.n_qtiles, a.z);
  const int slice = tile / a.n_qtiles;
  const int kvh = slice % a.Hkv, b = slice / a.Hkv % a.B, c = slice / a.Hkv / a.B;
  const int p0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq +
                 (a.mask_paper ? 0 : 1);
  const int kend = min(p0 + a.gs * (a.T_new - 1), a.S_cap);
  const int sb = 32 * CT * (tile % a.n_qtiles), G = a.Hq / a.Hkv;
  const int nh = (cg.offsets[c + 1] - cg.offsets[c]) * G;
  if (sb >= kend || nh == 0) return;
  const float cl2 = a.scale_log2;
  const auto kview = make_view(a.Kc + (long)slice * a.S_cap * DH, (uint32_t)kend * ROW);
  bf16x8 kf[CT][NKS];
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
      kf[t][ks] = buf_frag<bf16>(kview, (uint32_t)(sb + 32 * t + r) * ROW + (16 * ks + 8 * h) * 2u);
  f32x16 acc[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) acc[t] = zero16();
  const int i_num = sb - p0, qb0 = (i_num < 0 ? 0 : i_num / a.gs + 1) / 32;
  const int nqb = (a.T_new + 31) / 32 - qb0, nst = nh * nqb;
  const int mine = nst > w ? (nst - w + 3) / 4 : 0;  // steps w, w + 4, ... are this wave's
  char* ring = smem + w * RING;
  const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
  uint32_t coff[NI];
#pragma unroll
  for (int n = 0; n < NI; ++n) {
    const int ch = 64 * n + lane, row = ch / CPR;
    coff[n] = (uint32_t)row * ROW + 16u * (uint32_t)((ch % CPR) ^ pf_swz<DH>(row));
  }
  // the next step to copy: head x (of the slice's consumers' heads), query block qb
  int x = 0, qb = w;
  auto issue = [&](int st) {  // its rows and their LSE; past the last step zeros
    if (qb >= nqb) x += qb / nqb, qb %= nqb;
    const bool ok = x < nh;
    const int hx = ok ? x : 0, l = cg.members[cg.offsets[c] + hx / G];
    const long row0 = (((long)l * a.B + b) * a.Hq + kvh * G + hx % G) * a.T_new;
    const auto qview = make_view(a.Q + row0 * DH, (uint32_t)a.T_new * ROW);
    const auto lview = make_view(a.lse + row0, (uint32_t)a.T_new * 4u);
    const uint32_t base = ok ? (uint32_t)(qb0 + qb) * BLK : kOffOob, to = ring_at + st * STAGE;
#pragma unroll
    for (int n = 0; n < NI; ++n)
      lds_dma16(__builtin_amdgcn_readfirstlane(to + 1024 * n), base + coff[n], qview);
    lds_dma4(__builtin_amdgcn_readfirstlane(to + BLK),
             ok ? (uint32_t)(32 * (qb0 + qb) + r) * 4u : kOffOob, lview);
    qb += 4;
  };
  const PfLane<DH> lo = pf_lane<DH>(lane);
  // The scores of step j + 1 are multiplied while the exponentials of step j are taken; two score
  // sets take turns. When step j starts, step j + 1's copies have landed or are waited for, step
  // j + 2's are in flight.
  issue(0);
  issue(1);
  int q_at = w, st = 0;  // the next scored step's query block (of nqb per head), its ring stage
  struct Scored {
    f32x16 sc[CT];
    float nl;
    int q0;
  } sa, sn;
  auto score = [&](Scored& s) {
    if (q_at >= nqb) q_at %= nqb;
    s.q0 = 32 * (qb0 + q_at);
    q_at += 4;
    s.nl = -*(const float*)(ring + st * STAGE + BLK + 4 * r);
#pragma unroll
    for (int t = 0; t < CT; ++t) s.sc[t] = zero16();
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const bf16x8 qf = pf_ldk<DH>(ring, lo, st * STAGE, ks);
#pragma unroll
      for (int t = 0; t < CT; ++t) s.sc[t] = mma32(s.sc[t], kf[t][ks], qf);
    }
    st = st + 1 == NS ? 0 : st + 1;
  };
  auto step = [&](Scored& cur, Scored& nxt) {
    // steps past the last are scored from zeros and not added
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the stage refilled next is read
    issue(st + 1 == NS ? 0 : st + 1);
    wait_copies<NI + 1>();
    if (cur.q0 + 32 > a.T_new || p0 + a.gs * cur.q0 < sb + 32 * CT) {
      const int qi = cur.q0 + r;
      const int lim = qi < a.T_new ? p0 + a.gs * qi : 0;  // (rows past the last read nothing)
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int q = 0; q < 16; ++q)
          cur.sc[t][q] =
              sb + 32 * t + 4 * h + 8 * (q >> 2) + (q & 3) < lim ? cur.sc[t][q] : kHidden;
    }
    score(nxt);
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[t][q] += fast_exp2(fmaf(cur.sc[t][q], cl2, cur.nl));
  };
  if (mine > 0) {
    wait_copies<NI + 1>();
    score(sa);
    for (int j = 0; j < mine; j += 2) {
      step(sa, sn);
      if (j + 1 < mine) step(sn, sa);
    }
  }
  wait_copies<0>();  // no copy may land after the workgroup ends
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      float v = acc[t][q];
#pragma unroll
      for (int y = 1; y < 32; y <<= 1) v += __shfl_xor(v, y, 64);
      if (r == 0) s_w[w][32 * t + 8 * (q >> 2) + 4 * h + (q & 3)] = v;
    }
  __syncthreads();
  if (tid < 32 * CT && sb + tid < kend) {
    float* dst = weight + (long)slice * a.S_cap + sb + tid;
    *dst += (s_w[0][tid] + s_w[1][tid]) + (s_w[2][tid] + s_w[3][tid]);
  }
}

template <typename T>
static ReachArgs<T> reach_args(const Shape& sh, const Reach& r, const LayerTable& chan, const T* Q,
                               const T* Kc, const T* Vc, const T* Kd, const T* Vd,
                               const int32_t* ctx_len, T* O, float* lse) {
  LayerTable lord{};  // consumers sorted by channel, stable
  for (int c = 0, n = 0; c < kMaxLayers && n < sh.L; ++c)
    for (int l = 0; l < sh.L; ++l)
      if (chan.v[l] == c) lord.v[n++] = l;
  return ReachArgs<T>{Q, Kc, Vc, Kd, Vd, (const T*)r.Kp, (const T*)r.Vp, ctx_len, O, lse, sh.B,
                      sh.T_new, sh.L, sh.Hq, sh.Hkv, sh.S_cap, r.P, r.P_cap, r.window, r.sinks,
                      sh.mask_paper, 0, sh.gs, sh.gq, sh.ctx_hi, kLog2e / sqrtf((float)sh.d), chan,
                      lord};
}

template <int DH, bool PRE, bool LSE>
static void reach_dma(ReachArgs<bf16> a, const Shape& sh, uint32_t* queue, hipStream_t s) {
  using P = PfDma<1, DH>;
  // Tiles of 32 rows whose waves cut the slots where a head has no more rows, or up to three of
  // them for two CUs. us a call, 128-row tiles / these: 16 layers of 6/3 heads of 96, window 1024, one
  // sequence of 64 / 128 / 256 tokens (192 / 384 / 768 workgroups) 24 / 27 / 29 and 15 / 24 / 36;
  // 24 layers of 16 heads of 64, window 512, 8 sequences of 16 / 40 tokens 66 / 79 and
  // 63 / 108; over a prefix of 2000, 16 sequences of 16 / 40 257 / 324 and 224 / 389.
  const long few = (long)((sh.T_new + 31) / 32) * sh.Hq * sh.B * sh.L;
  if (sh.T_new <= 32 || 2 * few <= 3l * device_cus()) {
    a.n_qtiles = (sh.T_new + 31) / 32;
    hipLaunchKernelGGL((reach_few_kernel<DH, PRE, LSE>), dim3((unsigned)few), dim3(256), 0, s, a);
    return;
  }
  a.n_qtiles = (sh.T_new + P::BQ - 1) / P::BQ;
  const long tiles = (long)a.n_qtiles * sh.Hq * sh.B * sh.L, resident = (long)device_cus() * P::WPE;
  if (tiles <= resident) {
    hipLaunchKernelGGL((reach_dma_kernel<DH, PRE, LSE>), dim3((unsigned)tiles), dim3(P::NT), 0, s, a,
                       (uint32_t*)nullptr);
    return;
  }
  hipLaunchKernelGGL(reach_queue_kernel, dim3(1), dim3(kQueueWords), 0, s, queue);
  hipLaunchKernelGGL((reach_dma_kernel<DH, PRE, LSE>), dim3((unsigned)resident), dim3(P::NT), 0, s, a,
                     queue);
}

template <typename T, int DH, bool PRE, bool LSE, int SW>
static void reach_plain_go(ReachArgs<T> a, const Shape& sh, hipStream_t s) {
  using C = ReachCfg<T, DH, SW>;
  a.n_qtiles = (sh.T_new + C::BQ - 1) / C::BQ;
  hipLaunchKernelGGL((reach_prefill_kernel<T, DH, PRE, LSE, false, SW>),
                     dim3((unsigned)(a.n_qtiles * sh.Hq * sh.B * sh.L)), dim3(C::NT), 0, s, a);
}
template <typename T, int DH, bool PRE, bool LSE>
static void reach_plain(const ReachArgs<T>& a, const Shape& sh, hipStream_t s) {
  if (sh.T_new <= ReachCfg<T, DH, 2>::BQ) reach_plain_go<T, DH, PRE, LSE, 2>(a, sh, s);
  else reach_plain_go<T, DH, PRE, LSE, 1>(a, sh, s);
}

template <typename T, int DH>
static void prefix_flat(ReachArgs<T> a, int rows, int nlive, hipStream_t s) {
  using C = ReachCfg<T, DH, 1>;
  a.z = (rows + C::BQ - 1) / C::BQ;
  hipLaunchKernelGGL((reach_prefill_kernel<T, DH, true, false, true>),
                     dim3((unsigned)(a.z * a.np * a.Hkv * nlive)), dim3(C::NT), 0, s, a);
}

template <typename T>
void launch_prefix_rows(const Shape& sh, const Reach& r, const LayerTable& live, int nlive,
                        const ChannelGroups& cg, int rows, const T* Q, float* part, int nsplit,
                        int np, int split_len, hipStream_t s) {
  ReachArgs<T> a = reach_args<T>(sh, r, LayerTable{}, Q, nullptr, nullptr, nullptr, nullptr,
                                 nullptr, nullptr, nullptr);
  a.live = live;
  a.cg = cg;
  a.part = part;
  a.np = np;
  a.nsplit = nsplit;
  a.split_len = split_len;
  if constexpr (sizeof(T) == 4) {
    if (sh.d == 64) return prefix_flat<T, 64>(a, rows, nlive, s);
  }
  prefix_flat<T, 32>(a, rows, nlive, s);
}

template <typename T, bool PRE, bool LSE>
static void reach_go(const ReachArgs<T>& a, const Shape& sh, uint32_t* queue, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (sh.d == 64) return reach_dma<64, PRE, LSE>(a, sh, queue, s);
    if (sh.d == 96) return reach_dma<96, PRE, LSE>(a, sh, queue, s);
  } else {
    if (sh.d == 64) return reach_plain<T, 64, PRE, LSE>(a, sh, s);
  }
  reach_plain<T, 32, PRE, LSE>(a, sh, s);
}

template <typename T>
void launch_reach(const Shape& sh, const Reach& r, const LayerTable& chan, const T* Q, const T* Kc,
                  const T* Vc, const T* Kd, const T* Vd, const int32_t* ctx_len, T* O, float* lse,
                  void* queue, hipStream_t s) {
  const ReachArgs<T> a = reach_args<T>(sh, r, chan, Q, Kc, Vc, Kd, Vd, ctx_len, O, lse);
  uint32_t* q = (uint32_t*)queue;
  if (lse) reach_go<T, false, true>(a, sh, q, s);
  else if (r.P > 0) reach_go<T, true, false>(a, sh, q, s);
  else reach_go<T, false, false>(a, sh, q, s);
}

template <typename T>
void launch_weigh(const Shape& sh, const LayerTable& chan, const ChannelGroups& cg, const T* Q,
                  const T* Kc, const int32_t* ctx_len, const float* lse, float* weight,
                  hipStream_t s) {
  const Reach r{};
  ReachArgs<T> a = reach_args<T>(sh, r, chan, Q, Kc, nullptr, nullptr, nullptr, ctx_len, nullptr,
                                 const_cast<float*>(lse));
  const long most = (long)sh.ctx_max + sh.span();
  a.n_qtiles = (int)((most + 63) / 64);  // slot tiles of a slice
  a.z = 4 * device_cus() / kNumXcd;      // tiles whose longest start first: two per place
  const dim3 grid((unsigned)((long)a.n_qtiles * sh.k * sh.B * sh.Hkv));
  if constexpr (sizeof(T) == 2) {
    if (sh.d == 96)
      hipLaunchKernelGGL(reach_weigh_dma_kernel<96>, grid, dim3(256), 0, s, a, cg, weight);
    else if (sh.d == 64)
      hipLaunchKernelGGL(reach_weigh_dma_kernel<64>, grid, dim3(256), 0, s, a, cg, weight);
    if (sh.d != 32) return;
  } else {
    if (sh.d == 64) {
      hipLaunchKernelGGL((reach_weigh_kernel<T, 64>), grid, dim3(256), 0, s, a, cg, weight);
      return;
    }
  }
  hipLaunchKernelGGL((reach_weigh_kernel<T, 32>), grid, dim3(256), 0, s, a, cg, weight);
}

#define WM_INST(T)                                                                                \
  template void launch_reach<T>(const Shape&, const Reach&, const LayerTable&, const T*,          \
                                const T*, const T*, const T*, const T*, const int32_t*, T*,       \
                                float*, void*, hipStream_t);                                      \
  template void launch_prefix_rows<T>(const Shape&, const Reach&, const LayerTable&, int,         \
                                      const ChannelGroups&, int, const T*, float*, int, int, int, \
                                      hipStream_t);                                               \
  template void launch_weigh<T>(const Shape&, const LayerTable&, const ChannelGroups&, const T*,  \
                                const T*, const int32_t*, const float*, float*, hipStream_t);
WM_INST(float)
WM_INST(bf16)
#undef WM_INST

}  // namespace wm
