// Decode form of the channel attention (paper Section 3.1 Step 3, Section 3.2): few new
// tokens per sequence (T_new <= 4) against a long cache.
//
// Split-S over the cache, one workgroup per (split, channel with a reader, sequence, KV head)
// serving every query row that reads that channel and head (all its consumer layers, grouped
// query heads and new tokens), so each channel slice is streamed from HBM once.
#include <algorithm>

#include "wm_device.hpp"
#include "wm_frag.hpp"
#include "wm_prefill.hpp"

namespace wm {

// ------------------------------------------------------------------ decode
// Cache slots per split workgroup: long splits amortise a workgroup's set-up and its
// partial-state write; they are halved (down to 256) while the grid of splits x
// (channel, sequence, KV head) would hold fewer than kDecodeMinBlocks workgroups.
constexpr int kSplitMax = 4096, kSplitMin = 256;
constexpr long kDecodeMinBlocks = 4096;

int decode_split_len(const Shape& sh) {
  const long kend = (long)sh.ctx_max + sh.span();  // upper bound on visible slots
  const long slices = (long)sh.k * sh.B * sh.Hkv;
  int len = kSplitMax;
  while (len > kSplitMin && slices * ((kend + len - 1) / len) < kDecodeMinBlocks) len /= 2;
  return len;
}

int decode_splits(const Shape& sh) {
  const long kend = (long)sh.ctx_max + sh.span();
  const int len = decode_split_len(sh);
  int n = (int)((kend + len - 1) / len);
  return n < 1 ? 1 : n;
}

size_t decode_partials_bytes(const Shape& sh) {
  size_t rows = (size_t)sh.L * sh.B * sh.Hq * sh.T_new;
  return rows * decode_splits(sh) * (sh.d + 2) * sizeof(float);
}

// Slots that a sequence's rows read in all, at most (T_new rows whose windows move on by gs).
long window_slots(const Shape& sh, const Reach& r) {
  return std::min((long)sh.ctx_max + sh.span(),
                  (long)r.sinks + r.window + (long)sh.gs * (sh.T_new - 1));
}

// The partials of a window call of these dims, whatever its window: decode_splits of a walk of
// w slots is ceil(w / 256) until the grid holds kDecodeMinBlocks workgroups, then less than twice
// what that takes, and from there on ceil(w / 4096).
size_t decode_window_bytes(const Shape& sh) {
  const long kend = (long)sh.ctx_max + sh.span(), slices = (long)sh.k * sh.B * sh.Hkv;
  const long some = std::min((kend + kSplitMin - 1) / kSplitMin,
                             std::max(1L, 2 * kDecodeMinBlocks / slices));
  const long n = std::max(std::max(1L, (kend + kSplitMax - 1) / kSplitMax), some);
  return (size_t)sh.L * sh.B * sh.Hq * sh.T_new * n * (sh.d + 2) * sizeof(float);
}

template <typename T> struct DecodeArgs {
  const T *Q, *Kc, *Vc, *Kd, *Vd;
  const int32_t* ctx_len;
  const int32_t* doc;  // [B][T_new] first position of each token's document, or null
  float* part;  // [L][B][Hq][T_new][nsplit][d + 2]: unnormalised o, m, l
  T* O;
  int B, T_new, L, Hq, Hkv, S_cap, mask_paper, nsplit, split_len;
  int gs, gq, ctx_hi;  // query i of sequence b sits at position ctx_len[b] + gq + gs i
  float scale_log2;
  LayerTable chan;
  // the grid's channels, those with a reader: live[i], its consumers offsets[i] .. offsets[i + 1]
  LayerTable live;
  ChannelGroups cg;
  int window, sinks;  // WIN kernels: a row reads its last `window` slots and the first `sinks`
  // weighed attention: raw scores of every row and slot [L][B][Hq][T_new][s_ld] (hidden: -1e30),
  // and the rows' log-sum-exp in log2 units; else null
  float *scores, *lse;
  long s_ld;
};

// The slots that a sequence's rows read in a window, one after the other: `na` first slots, then
// those from lo0 (the first row's window, which starts lowest) on. Compact slot x is slot
// x < na ? x : x + skip of the cache; a row with limit lim reads compact slots below lim - skip
// that are at or past its lo - skip or below `sinks`. (skip > 0 only where every first slot lies
// before every row's window, so that all rows read all of them; else compact = cache slots.)
struct WindowSpan {
  int na, skip, n, lo_last;  // n compact slots; lo_last: the last row's window's first one
};
__device__ __forceinline__ WindowSpan window_span(int lim0, int kend, int window, int sinks) {
  WindowSpan w;
  const int lo0 = max(lim0 - window, 0);
  w.na = min(sinks, lo0);
  w.skip = lo0 - w.na;
  w.n = max(kend - w.skip, 0);
  w.lo_last = max(kend - window, 0) - w.skip;
  return w;
}

// Merge online-softmax state (m2, l2, o2) into (m, l, o).
__device__ __forceinline__ void merge_state(float& m, float& l, float* o, float m2, float l2,
                                            const float* o2, int n, float c) {
  float M = fmaxf(m, m2);
  float a1 = fast_exp2((m - M) * c), a2 = fast_exp2((m2 - M) * c);
  l = l * a1 + l2 * a2;
  for (int i = 0; i < n; ++i) o[i] = o[i] * a1 + o2[i] * a2;
  m = M;
}

// ---------------------------------------------- decode on the matrix cores (bf16)
// bf16, head dims 64 and 96. The rows of one (channel, sequence, KV head) -- consumers x
// grouped heads x new tokens -- are the columns of S^T = K Q^T and O^T = V^T P^T on 32x32x16
// MFMAs, as in the full-sequence kernel, so a slot costs the same for 1 row and for 32.
// (The VALU kernel below spends 16 fused multiply-adds and a butterfly per slot, lane and
// row: at 16 rows, B = 8, ctx 4001, k = 8, 6/3 heads of 96 it ran 383 us on 221 MB of
// cache; this one 47 us. At 2 rows and head dim 64 both run at the rate of the cache
// stream at B = 16, ctx 8191, k = 12; at one consumer over 709 slots this one
// takes 7 us and the VALU kernel 10.6.) What is left is the stream: each of NW waves walks
// every NW-th 32-slot block through a ring of two blocks of its own in LDS (LDS-DMA, no
// barrier: a wave waits only for its own copies). Measured at the two shapes above:
// waves on a CU count for more than copies in flight per wave (three or four blocks per
// ring, with half the waves, 4-30% slower). The weights are the VALU kernel's: scores from the
// unscaled bf16 queries, weights in fp32, cut into three bf16 parts (8 + 8 + 8 bits, exact)
// for three PV products, the normaliser summed from the fp32 ones. (Two rounded parts, 16
// bits, left 2.7e-6 of the terms' sum where two values cancel, three 5e-8; a step at 12 heads
// of 64, k = 12, ctx 8000 99.2 us with two, 100.8 with three; at B = 8, T_new = 4, ctx 4001,
// 6/3 heads of 96 80.7 and 80.8. The parts are truncated: rounding them takes longer, 107.7.)
template <int DH, int NW_> struct DecMfma {
  static constexpr int NW = NW_, NT = 64 * NW, NS = 2, BKV = 32;
  static constexpr int NKS = DH / 16, NDT = DH / 32;
  static constexpr int ROW_BYTES = 2 * DH, CPR = ROW_BYTES / 16;
  static constexpr int BLK = BKV * ROW_BYTES;      // one K (or V) block of 32 slots
  static constexpr int NI = BLK / 1024;            // copy instructions per block
  static constexpr int STAGE = 2 * BLK;            // K then V
  static constexpr int RING = NS * STAGE;          // per wave
  static constexpr int OLD = DH + 4;               // row stride of the merge staging (floats)
  static_assert(32 * OLD * 4 + 256 <= RING, "the merge staging fits a wave's ring");
  static_assert(2 * NI * (NS - 1) <= 63, "the copies in flight behind one vmcnt");
};

// Sum of 16 values as a balanced tree.
__device__ __forceinline__ float sum16(const f32x16& v) {
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = v[i] + v[8 + i];
  return ((t[0] + t[4]) + (t[1] + t[5])) + ((t[2] + t[6]) + (t[3] + t[7]));
}

// lds_dma16 (wm_device.hpp) for bytes that are read once: non-temporal, so the stream does
// not fill L2 and the Infinity Cache with lines nobody reads again (B = 16, ctx 8191, k = 12,
// 16 heads of 64: the step 1004 -> 902 us, its attention 5.6 -> 6.2 TB/s, the rate of a plain
// read of HBM; at B = 8, ctx 4001, whose 221 MB could stay in that cache, 133 -> 124 us).
__device__ __forceinline__ void lds_dma16_stream(uint32_t lds_addr, uint32_t voff,
                                                 __amdgpu_buffer_rsrc_t rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}

// (split, slice y and row tile z of the grid; smem: NW rings)
template <int DH, int NW, bool DOC, bool ONCE, bool WIN, bool SCORES>
__device__ __forceinline__ void decode_block(const DecodeArgs<bf16>& a, const int split, int y,
                                             const int z, char* smem) {
  using C = DecMfma<DH, NW>;
  const int kvh = y % a.Hkv;
  y /= a.Hkv;
  const int b = y % a.B, ci = y / a.B, c = a.live.v[ci];
  const int off = a.cg.offsets[ci], nmem = a.cg.offsets[ci + 1] - off;
  const int grp = a.Hq / a.Hkv;
  const int G = nmem * grp * a.T_new, g0 = 32 * z;
  if (g0 >= G) return;
  const int pos0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq;
  const int gs = a.gs, incl = a.mask_paper ? 0 : 1;
  const int kend = min(pos0 + gs * (a.T_new - 1) + incl, a.S_cap);
  // (WIN: s0, s1 and every slot index below are compact)
  WindowSpan ws{0, 0, 0, 0};
  if constexpr (WIN) ws = window_span(pos0 + incl, kend, a.window, a.sinks);
  const int s0 = split * a.split_len, s1 = min(s0 + a.split_len, WIN ? ws.n : kend);
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float cl2 = a.scale_log2;

  // this lane's row (both halves of the wave share it) and the slots it reads
  auto row_of = [&](int g, int& i) {
    i = g % a.T_new;
    const int gq = (g / a.T_new) % grp, mi = g / (a.T_new * grp);
    const int l = a.cg.members[off + mi], hq = kvh * grp + gq;
    return (((long)l * a.B + b) * a.Hq + hq) * a.T_new + i;
  };
  int vis = 0, lov = 0;
  bf16x8 qf[C::NKS];
  float* srow = nullptr;  // SCORES: where this lane's scores go
  {
    const bool ok = g0 + r < G;
    int i = 0;
    const long rowid = ok ? row_of(g0 + r, i) : 0;
    if (SCORES && ok) srow = a.scores + rowid * a.s_ld + 4 * h;
    if (ok) {
      vis = min(pos0 + gs * i + incl - (WIN ? ws.skip : 0), s1);
      if (DOC) lov = doc_first(a.doc, b, a.T_new, i, pos0 + gs * i);
      if (WIN) lov = max(pos0 + gs * i + incl - a.window, 0) - ws.skip;
    }
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks)
      qf[ks] = ok ? ld_frag<bf16>(a.Q + rowid * DH + 16 * ks + 8 * h) : zero_frag<bf16>();
  }

  const int nblk = s1 > s0 ? (s1 - s0 + C::BKV - 1) / C::BKV : 0;
  const int nw = (nblk - w + C::NW - 1) / C::NW;  // this wave's blocks: w, w + NW, ...
  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  // views end at the last visible slot: rows past it arrive as zeros
  const auto kview = make_view(a.Kc + cbase, (uint32_t)max(kend, 0) * C::ROW_BYTES);
  const auto vview = make_view(a.Vc + cbase, (uint32_t)max(kend, 0) * C::ROW_BYTES);
  uint32_t coff[C::NI];
#pragma unroll
  for (int n = 0; n < C::NI; ++n) {
    const int ch = 64 * n + lane, row = ch / C::CPR;
    coff[n] = (uint32_t)row * C::ROW_BYTES + 16u * (uint32_t)((ch % C::CPR) ^ pf_swz<DH>(row));
  }
  char* ring = smem + w * C::RING;
  const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
  // block j of this wave into ring stage st (blocks past the wave's last are copied as
  // zeros, so the count of copies in flight is the same at every wait)
  auto issue = [&](int j, int st) {
    const uint32_t base =
        j < nw ? (uint32_t)(s0 + C::BKV * (w + C::NW * j)) * C::ROW_BYTES : kOffOob;
#pragma unroll
    for (int n = 0; n < 2 * C::NI; ++n) {
      uint32_t o = base + coff[n % C::NI];
      if constexpr (WIN)
        o += j < nw && s0 + C::BKV * (w + C::NW * j) + (64 * (n % C::NI) + lane) / C::CPR >= ws.na
                 ? (uint32_t)ws.skip * C::ROW_BYTES : 0u;
      const uint32_t lds =
          __builtin_amdgcn_readfirstlane(ring_at + st * C::STAGE + 1024 * n);
      if constexpr (ONCE) lds_dma16_stream(lds, o, n < C::NI ? kview : vview);
      else lds_dma16(lds, o, n < C::NI ? kview : vview);
    }
  };

  // slots below it are visible to every row
  const int all_vis = min(pos0 + incl - (WIN ? ws.skip : 0), s1);
  float m = kNegBig, lsum = 0.f;
  f32x16 o[C::NDT];
#pragma unroll
  for (int dt = 0; dt < C::NDT; ++dt) o[dt] = zero16();
  // (a wave without a block of the split walks one of zeros, every slot of it hidden)
  const PfLane<DH> lo = pf_lane<DH>(lane);
#pragma unroll
  for (int u = 0; u + 1 < C::NS; ++u) issue(u, u);
  int j = 0, st = 0;
  do {
    // the stage block j-1 was read from (its reads have returned) takes block j+NS-1
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    issue(j + C::NS - 1, st == 0 ? C::NS - 1 : st - 1);
    wait_copies<2 * C::NI * (C::NS - 1)>();
    const uint32_t kh = st * C::STAGE, vh = kh + C::BLK;
    f32x16 sc = zero16();
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) sc = mma32(sc, pf_ldk<DH>(ring, lo, kh, ks), qf[ks]);
    const int at = s0 + C::BKV * (w + C::NW * j);  // the block's first slot
    if (DOC || __builtin_expect(at + C::BKV > all_vis ||
                                (WIN && a.T_new > 1 && at < ws.lo_last), 0)) {
      // some row may not read some of the block's slots
      asm volatile("" : "+v"(vis));  // (keeps the comparisons out of the common path)
      const int base = at + 4 * h;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int s = base + 8 * (q >> 2) + (q & 3);
        sc[q] = s >= vis || (DOC && s < lov) || (WIN && s < lov && s >= a.sinks) ? kNegBig : sc[q];
      }
    }
    if constexpr (SCORES) {  // rows of s_ld slots, a multiple of 32: no block ends past one
      if (srow && j < nw) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(f32x4*)(srow + at + 8 * g) = f32x4{sc[4 * g], sc[4 * g + 1], sc[4 * g + 2], sc[4 * g + 3]};
      }
    }
    float mx = sc[0];
#pragma unroll
    for (int q = 1; q < 16; ++q) mx = fmaxf(mx, sc[q]);
    mx = halves_max(mx);
    if (__builtin_expect(__any(mx > m), 0)) {
      const float mn = fmaxf(m, mx), al = fast_exp2((m - mn) * cl2);
      lsum *= al;
#pragma unroll
      for (int dt = 0; dt < C::NDT; ++dt) {
        asm volatile("" : "+v"(o[dt]));  // (keeps the products out of the common path)
        o[dt] *= al;
      }
      m = mn;
    }
    // hidden slots (-1e30) get weight 0, also while the row has seen none (m = -1e30)
    const float mc = m > 0.5f * kNegBig ? m * cl2 : 0.f;
    f32x16 p;
#pragma unroll
    for (int q = 0; q < 16; ++q) p[q] = fast_exp2(fmaf(sc[q], cl2, -mc));
    float ps = sum16(p);
    if (__builtin_expect(__any(!(ps <= 3.0e38f)), 0)) {  // a NaN score weighs nothing
#pragma unroll
      for (int q = 0; q < 16; ++q) p[q] = sc[q] > 0.5f * kNegBig ? p[q] : 0.f;
      ps = sum16(p);
    }
    lsum += ps;
    bf16x8 pw[3][2];
    cut24(p, pw);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      bf16x8 vf[C::NDT];
#pragma unroll
      for (int dt = 0; dt < C::NDT; ++dt) vf[dt] = pf_ldv<DH>(ring, lo, vh, hf, dt);
#pragma unroll
      for (int u = 0; u < 3; ++u)
#pragma unroll
        for (int dt = 0; dt < C::NDT; ++dt) o[dt] = mma32(o[dt], vf[dt], pw[u][hf]);
    }
    st = st + 1 == C::NS ? 0 : st + 1;
  } while (++j < nw);
  wait_copies<0>();  // no copy may land in the staging below, or after the block ends
  // merge the waves' states: each writes its rows [r][DH] and (m, l) to its own ring
  const float lt = halves_sum(lsum);
  float* so = (float*)ring;
#pragma unroll
  for (int dt = 0; dt < C::NDT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = o[dt][4 * g + i];
      *(f32x4*)(so + r * C::OLD + 32 * dt + 8 * g + 4 * h) = v;
    }
  if (h == 0) {
    so[32 * C::OLD + 2 * r] = m;
    so[32 * C::OLD + 2 * r + 1] = lt;
  }
  __syncthreads();
  const int ng = min(32, G - g0);
  for (int e = tid; e < ng * DH; e += C::NT) {
    const int gi = e / DH, dd = e - gi * DH;
    float M = kNegBig;
#pragma unroll
    for (int ww = 0; ww < C::NW; ++ww)
      M = fmaxf(M, ((const float*)(smem + ww * C::RING))[32 * C::OLD + 2 * gi]);
    float lw = 0.f, ow = 0.f;
#pragma unroll
    for (int ww = 0; ww < C::NW; ++ww) {
      const float* sw = (const float*)(smem + ww * C::RING);
      const float al = fast_exp2((sw[32 * C::OLD + 2 * gi] - M) * cl2);
      lw += sw[32 * C::OLD + 2 * gi + 1] * al;
      ow += sw[gi * C::OLD + dd] * al;
    }
    int i;
    float* dst = a.part + (row_of(g0 + gi, i) * a.nsplit + split) * (DH + 2);
    dst[dd] = ow;
    if (dd == 0) {
      dst[DH] = M;
      dst[DH + 1] = lw;
    }
  }
}

template <int DH, int NW, bool DOC, bool ONCE, bool WIN = false, bool SCORES = false>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(3)))
void attend_decode_mfma_kernel(DecodeArgs<bf16> a) {
  __shared__ __align__(16) char smem[NW * DecMfma<DH, NW>::RING];
  decode_block<DH, NW, DOC, ONCE, WIN, SCORES>(a, blockIdx.x, blockIdx.y, blockIdx.z, smem);
}

// ---------------------------------------------- decode on the VALU (fp32, head dim 32)
template <typename T, int DH, int NG, bool WIN = false, bool SCORES = false>
__global__ __launch_bounds__(256) void attend_decode_kernel(DecodeArgs<T> a) {
  // A cache slot is read by LPS lanes of 8 elements each.
  constexpr int LPS = DH / 8;
  static_assert(DH == 32 || DH == 64, "the lanes of a slot sum by butterflies");
  constexpr int SPW = 64 / LPS;  // slots per wave per sweep step
  constexpr int U = NG <= 2 ? 2 : 1;  // sweep steps per batch (U slots per lane)
  constexpr int SPB = 4 * SPW * U;  // slots per batch of the 4 waves
  __shared__ float red[4][NG][DH + 2];

  const int split = blockIdx.x;
  int y = blockIdx.y;
  const int kvh = y % a.Hkv;
  y /= a.Hkv;
  const int b = y % a.B, ci = y / a.B, c = a.live.v[ci];
  const int off = a.cg.offsets[ci], nmem = a.cg.offsets[ci + 1] - off;
  const int grp = a.Hq / a.Hkv;
  const int G = nmem * grp * a.T_new;
  // position of query i: pos0 + gs i (wave-uniform)
  const int pos0 = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_hi)) + a.gq;
  const int gs = a.gs;
  const int incl = a.mask_paper ? 0 : 1;
  const int kend = min(pos0 + gs * (a.T_new - 1) + incl, a.S_cap);
  // (WIN: s0, s1 and every slot index below are compact)
  WindowSpan ws{0, 0, 0, 0};
  if constexpr (WIN) ws = window_span(pos0 + incl, kend, a.window, a.sinks);
  const int s0 = split * a.split_len, s1 = min(s0 + a.split_len, WIN ? ws.n : kend);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int sg = lane / LPS, c8 = lane % LPS;
  const float cl2 = a.scale_log2;
  const float thresh = 8.0f / cl2;  // log2 headroom before a rescale

  const long cbase = (((long)c * a.B + b) * a.Hkv + kvh) * (long)a.S_cap * DH;
  // the slice through buffer views: slots at or past s1 read zeros without a branch
  const __amdgpu_buffer_rsrc_t kview = make_view(a.Kc + cbase, (uint32_t)a.S_cap * DH * sizeof(T));
  const __amdgpu_buffer_rsrc_t vview = make_view(a.Vc + cbase, (uint32_t)a.S_cap * DH * sizeof(T));
  auto slot_off = [&](int s) {
    const int at = WIN && s >= ws.na ? s + ws.skip : s;
    return s < s1 ? (uint32_t)(at * DH + 8 * c8) * (uint32_t)sizeof(T) : kOffOob;
  };

  for (int g0 = 0; g0 < G; g0 += NG) {
    const int ng = min(NG, G - g0);
    float q[NG][8], m[NG], ls[NG], o[NG][8];
    float* srow[NG];       // SCORES: where the row's scores go
    int vis[NG], lov[NG];  // the row reads slots lov <= s < vis
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      m[gi] = kNegBig;
      ls[gi] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[gi][i] = 0.f;
      if (gi < ng) {
        int g = g0 + gi;
        int i = g % a.T_new, gq = (g / a.T_new) % grp, mi = g / (a.T_new * grp);
        int l = a.cg.members[off + mi], hq = kvh * grp + gq;
        long rowid = (((long)l * a.B + b) * a.Hq + hq) * a.T_new + i;
        vis[gi] = pos0 + gs * i + incl - (WIN ? ws.skip : 0);
        lov[gi] = WIN ? max(pos0 + gs * i + incl - a.window, 0) - ws.skip
                      : doc_first(a.doc, b, a.T_new, i, pos0 + gs * i);
        if (SCORES) srow[gi] = a.scores + rowid * a.s_ld;
        load8(a.Q + rowid * DH + 8 * c8, q[gi]);
      } else {
        vis[gi] = 0;
        lov[gi] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) q[gi][i] = 0.f;
      }
    }

    // raw K/V fragments of a batch (U slots per lane), double-buffered across batches
    // (two batches per loop trip keep the buffer indices static)
    frag_t<T> kr0[U], vr0[U], kr1[U], vr1[U];
    auto fetch = [&](int sb, frag_t<T>* kr, frag_t<T>* vr) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t so = slot_off(sb + w * SPW * U + u * SPW + sg);
        kr[u] = buf_frag<T>(kview, so);
        vr[u] = buf_frag<T>(vview, so);
      }
    };
    auto consume = [&](int sb, const frag_t<T>* kr, const frag_t<T>* vr) {
      float p[U][NG];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = sb + w * SPW * U + u * SPW + sg;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
          float d = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) d += q[gi][i] * to_f32(kr[u][i]);
#pragma unroll
          for (int x = 1; x < LPS; x <<= 1) d += __shfl_xor(d, x, 64);
          p[u][gi] = s < s1 && s < vis[gi] && (s >= lov[gi] || (WIN && s < a.sinks)) ? d : kNegBig;
          if constexpr (SCORES) {
            if (c8 == 0 && gi < ng && s < s1) srow[gi][s] = p[u][gi];
          }
        }
      }
#pragma unroll
      for (int gi = 0; gi < NG; ++gi) {
        float mx = p[0][gi];
#pragma unroll
        for (int u = 1; u < U; ++u) mx = fmaxf(mx, p[u][gi]);
        if (mx > m[gi] + thresh) {  // lazy rescale (per lane; merged exactly below)
          const float al = fast_exp2((m[gi] - mx) * cl2);
          ls[gi] *= al;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[gi][i] *= al;
          m[gi] = mx;
        }
        const float mc = m[gi] * cl2;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float pe = p[u][gi] > 0.5f * kNegBig ? fast_exp2(p[u][gi] * cl2 - mc) : 0.f;
          ls[gi] += pe;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[gi][i] += pe * to_f32(vr[u][i]);
        }
      }
    };
    // batches past the split read zeros (and are masked), so the loop runs in pairs
    fetch(s0, kr0, vr0);
    for (int sb = s0; sb < s1; sb += 2 * SPB) {
      fetch(sb + SPB, kr1, vr1);
      consume(sb, kr0, vr0);
      fetch(sb + 2 * SPB, kr0, vr0);
      consume(sb + SPB, kr1, vr1);
    }
    // merge the slot groups of the wave (lanes that share c8)
#pragma unroll
    for (int msk = LPS; msk < 64; msk <<= 1)
#pragma unroll
      for (int gi = 0; gi < NG; ++gi) {
        float m2 = __shfl_xor(m[gi], msk, 64), l2 = __shfl_xor(ls[gi], msk, 64), o2[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o2[i] = __shfl_xor(o[gi][i], msk, 64);
        merge_state(m[gi], ls[gi], o[gi], m2, l2, o2, 8, cl2);
      }
    if (sg == 0) {
#pragma unroll
      for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
        for (int i = 0; i < 8; ++i) red[w][gi][8 * c8 + i] = o[gi][i];
        if (c8 == 0) {
          red[w][gi][DH] = m[gi];
          red[w][gi][DH + 1] = ls[gi];
        }
      }
    }
    __syncthreads();
    for (int e = tid; e < ng * DH; e += 256) {
      int gi = e / DH, dd = e % DH;
      float M = kNegBig;
      for (int ww = 0; ww < 4; ++ww) M = fmaxf(M, red[ww][gi][DH]);
      float Lsum = 0.f, Osum = 0.f;
      for (int ww = 0; ww < 4; ++ww) {
        float sc = fast_exp2((red[ww][gi][DH] - M) * cl2);
        Lsum += red[ww][gi][DH + 1] * sc;
        Osum += red[ww][gi][dd] * sc;
      }
      // recompute the row id for gi (registers are per-lane; rows are uniform)
      int g = g0 + gi;
      int i = g % a.T_new, gq = (g / a.T_new) % grp, mi = g / (a.T_new * grp);
      int l = a.cg.members[off + mi], hq = kvh * grp + gq;
      long rid = (((long)l * a.B + b) * a.Hq + hq) * a.T_new + i;
      float* dst = a.part + (rid * a.nsplit + split) * (DH + 2);
      dst[dd] = Osum;
      if (dd == 0) {
        dst[DH] = M;
        dst[DH + 1] = Lsum;
      }
    }
    __syncthreads();
  }
}

// One wave per query row: fold the dummy slot and all split partials.
template <typename T, int DH, bool LSE = false>
__global__ __launch_bounds__(256) void attend_combine_kernel(DecodeArgs<T> a) {
  constexpr int EPL = (DH + 63) / 64;  // elements per lane: channel 64 e + lane
  const long rows = (long)a.L * a.B * a.Hq * a.T_new;
  const long rid = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (rid >= rows) return;
  long t = rid;
  const int i = (int)(t % a.T_new);
  t /= a.T_new;
  const int hq = (int)(t % a.Hq);
  t /= a.Hq;
  const int b = (int)(t % a.B), l = (int)(t / a.B);
  const int c = a.chan.v[l], kvh = hq / (a.Hq / a.Hkv);
  const float cl2 = a.scale_log2;

  float M, Lsum, o[EPL];
  auto active = [&](int e) { return 64 * e + lane < DH; };
  if (a.mask_paper) {
    const T* q = a.Q + rid * DH;
    const T* kd = a.Kd + ((long)c * a.Hkv + kvh) * DH;
    const T* vd = a.Vd + ((long)c * a.Hkv + kvh) * DH;
    float part = 0.f;
    for (int e = 0; e < EPL; ++e)
      if (active(e)) part += to_f32(q[64 * e + lane]) * to_f32(kd[64 * e + lane]);
    M = wave_sum(part);
    Lsum = 1.f;
    for (int e = 0; e < EPL; ++e) o[e] = active(e) ? to_f32(vd[64 * e + lane]) : 0.f;
  } else {
    M = kNegBig;
    Lsum = 0.f;
    for (int e = 0; e < EPL; ++e) o[e] = 0.f;
  }
  const float* src = a.part + rid * a.nsplit * (DH + 2);
  for (int sidx = 0; sidx < a.nsplit; ++sidx) {
    const float* ps = src + (long)sidx * (DH + 2);
    float o2[EPL];
    for (int e = 0; e < EPL; ++e) o2[e] = active(e) ? ps[64 * e + lane] : 0.f;
    merge_state(M, Lsum, o, ps[DH], ps[DH + 1], o2, EPL, cl2);
  }
  T* dst = a.O + ((((long)l * a.B + b) * a.T_new + i) * a.Hq + hq) * DH;
  for (int e = 0; e < EPL; ++e)
    if (active(e)) dst[64 * e + lane] = from_f32<T>(o[e] / Lsum);
  if (LSE && lane == 0) a.lse[rid] = fmaf(M, cl2, __log2f(Lsum));
}

// weight[c][b][h][s] += the sum over the rows that read (c, b, h) of 2^(score - lse): a thread takes
// four slots, the rows' scores as the decode kernel left them.
template <typename T>
__global__ __launch_bounds__(256) void decode_weigh_kernel(DecodeArgs<T> a, float* weight) {
  int y = blockIdx.y;
  const int kvh = y % a.Hkv;
  y /= a.Hkv;
  const int b = y % a.B, ci = y / a.B, c = a.live.v[ci];
  const int off = a.cg.offsets[ci], nmem = a.cg.offsets[ci + 1] - off, grp = a.Hq / a.Hkv;
  const int pos0 = ctx_at(a.ctx_len, b, a.ctx_hi) + a.gq;
  const int kend = min(pos0 + a.gs * (a.T_new - 1) + (a.mask_paper ? 0 : 1), a.S_cap);
  const int s = 4 * (blockIdx.x * 256 + threadIdx.x);
  if (s >= kend) return;
  f32x4 w = {0.f, 0.f, 0.f, 0.f};
  for (int x = 0; x < nmem * grp; ++x) {
    const int l = a.cg.members[off + x / grp], hq = kvh * grp + x % grp;
    const long row0 = (((long)l * a.B + b) * a.Hq + hq) * a.T_new;
    for (int i = 0; i < a.T_new; ++i) {
      const f32x4 sc = *(const f32x4*)(a.scores + (row0 + i) * a.s_ld + s);
      const float lse = a.lse[row0 + i];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] += sc[e] > 0.5f * kNegBig ? fast_exp2(fmaf(sc[e], a.scale_log2, -lse)) : 0.f;
    }
  }
  float* dst = weight + (((long)c * a.B + b) * a.Hkv + kvh) * a.S_cap + s;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (s + e < kend) dst[e] += w[e];
}

// ------------------------------------------------- the shared prefix, few new tokens
// A prefix slot is read by every sequence, so the rows of one (channel, KV head) are those of the
// whole batch (consumers x grouped heads x new tokens x sequences), each seeing every slot:
// products of up to 128 rows against blocks of 32 slots, where a sequence's own cache meets only
// its own few rows. A workgroup's two waves share the blocks they read: either each has RT tiles of
// 32 rows of its own (RW = 2), wave 0 copying K and wave 1 V into a ring of three blocks, or, where a
// slice has 32 rows at most, both take the same rows and every second block (RW = 1, a ring of two
// pairs). Scores as in decode_block, the weights in 17 bits.
// The workgroups of a prefix's splits and those of the sequences' own caches (decode_block) form
// one grid: the former are bound by their products and exponentials, the latter by the stream of the
// cache, and a CU holds some of each at a time. (64 sequences, 24 layers of 16 heads of 64, 4096 + 300
// slots: 200 us; in two launches, the prefix by waves with rings of their own, 256.)
struct PrefixSpan {
  const bf16 *Kp, *Vp;
  int P, P_cap, nsplit, split_len, z;  // z: workgroups of rows per (slice, split)
  int blocks;                          // workgroups of the prefix, ahead of the caches'
  int own, slices;                     // splits and slices of the sequences' own caches
  float* part;                         // a row's states, the prefix's first
};
template <int DH, int RW, int RT> struct PrefixCfg {
  static constexpr int NW = 2, SW = NW / RW, NS = RW == 2 ? 3 : 2;  // SW: waves that cut the slots
  static constexpr int NKS = DH / 16, NDT = DH / 32, ROW_BYTES = 2 * DH, CPR = ROW_BYTES / 16;
  static constexpr int BLK = 32 * ROW_BYTES, NI = BLK / 1024;
  static constexpr int STAGE = SW * 2 * BLK;     // per block: K then V
  static constexpr int PER = SW * 2 * NI / NW;   // copy instructions of a wave per stage
  static constexpr int ROWS = 32 * RT * RW;      // rows of a workgroup
  static constexpr int OLD = DH + 4, MERGE = 32 * OLD * 4 + 256;  // a tile's state in LDS
  static constexpr int SMEM = NS * STAGE > NW * MERGE ? NS * STAGE : NW * MERGE;
};
template <int DH, int RW, int RT>
__device__ __forceinline__ void prefix_block(const DecodeArgs<bf16>& a, const PrefixSpan& px,
                                             char* smem) {
  using C = PrefixCfg<DH, RW, RT>;
  const int tile = xcd_tile(blockIdx.x, px.blocks);
  const int zt = tile % px.z;
  int y = tile / px.z;
  const int split = y % px.nsplit;
  y /= px.nsplit;
  const int kvh = y % a.Hkv, ci = y / a.Hkv, c = a.live.v[ci];
  const int off = a.cg.offsets[ci], nmem = a.cg.offsets[ci + 1] - off;
  const int grp = a.Hq / a.Hkv, per_b = nmem * grp * a.T_new;
  const int G = per_b * a.B, g0 = C::ROWS * zt;
  if (g0 >= G) return;
  const int s0 = split * px.split_len, s1 = min(s0 + px.split_len, px.P);
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = RW == 2 ? w : 0, sw = RW == 2 ? 0 : w;  // this wave's row tiles, its blocks
  const float cl2 = a.scale_log2;
  int row[RT];  // this lane's rows [l][b][hq][i] (both halves of the wave alike), -1 past the last
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int g = g0 + 32 * (RT * rw + t) + r, b = g / per_b, x = g % per_b, gl = x / a.T_new;
    const int l = a.cg.members[off + gl / grp];
    row[t] = g < G ? ((l * a.B + b) * a.Hq + kvh * grp + gl % grp) * a.T_new + x % a.T_new : -1;
  }
  uint32_t coff[C::NI];
#pragma unroll
  for (int n = 0; n < C::NI; ++n) {
    const int ch = 64 * n + lane, row = ch / C::CPR;
    coff[n] = (uint32_t)row * C::ROW_BYTES + 16u * (uint32_t)((ch % C::CPR) ^ pf_swz<DH>(row));
  }
  const int nblk = (s1 - s0 + 31) / 32, nit = (nblk + C::SW - 1) / C::SW;
  const long cbase = ((long)c * a.Hkv + kvh) * (long)px.P_cap * DH;
  const auto kview = make_view(px.Kp + cbase, (uint32_t)px.P * C::ROW_BYTES);
  const auto vview = make_view(px.Vp + cbase, (uint32_t)px.P * C::ROW_BYTES);
  const uint32_t smem_at = (uint32_t)(uintptr_t)smem;
  // step it into stage st: wave w copies instructions w PER .. of its blocks' K and V (past the
  // last step zeros, so that the copies in flight are the same number at every wait)
  auto issue = [&](int it, int st) {
#pragma unroll
    for (int i = 0; i < C::PER; ++i) {
      const bool v = RW == 2 ? w == 1 : i >= C::NI;
      const int at = s0 + 32 * (it * C::SW + sw);
      const uint32_t base = it < nit ? (uint32_t)at * C::ROW_BYTES : kOffOob;
      lds_dma16(__builtin_amdgcn_readfirstlane(smem_at + st * C::STAGE + 1024 * (w * C::PER + i)),
                base + coff[i % C::NI], v ? vview : kview);
    }
  };
  issue(0, 0);
  if (C::NS == 3) issue(1, 1);
  bf16x8 qf[RT][C::NKS];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks)
      qf[t][ks] = row[t] >= 0 ? ld_frag<bf16>(a.Q + (long)row[t] * DH + 16 * ks + 8 * h)
                           : zero_frag<bf16>();
  }
  float m[RT], lsum[RT];
  f32x16 o[RT][C::NDT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = kNoRef;
    lsum[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < C::NDT; ++dt) o[t][dt] = zero16();
  }
  const PfLane<DH> lo = pf_lane<DH>(lane);
  for (int it = 0, st = 0; it < nit; ++it) {
    wait_copies<(C::NS - 2) * C::PER>();
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    __syncthreads();  // step it has landed, and the stage of step it - 1 is free
    issue(it + C::NS - 1, st == 0 ? C::NS - 1 : st - 1);
    const uint32_t kh = st * C::STAGE + sw * 2 * C::BLK, vh = kh + C::BLK;
    const int at = s0 + 32 * (it * C::SW + sw);
    // scores of both row tiles, then their weights against the rows' references (log2 units),
    // which move only where a weight would pass 2^12 (or at a row's first slots)
    f32x16 p[RT];
    auto scores = [&]() {
#pragma unroll
      for (int t = 0; t < RT; ++t) p[t] = zero16();
#pragma unroll
      for (int ks = 0; ks < C::NKS; ++ks) {
        const bf16x8 kf = pf_ldk<DH>(smem, lo, kh, ks);
#pragma unroll
        for (int t = 0; t < RT; ++t) p[t] = mma32(p[t], kf, qf[t][ks]);
      }
      if (__builtin_expect(at + 32 > s1, 0)) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int q = 0; q < 16; ++q)
            p[t][q] = at + 4 * h + 8 * (q >> 2) + (q & 3) >= s1 ? kNegBig : p[t][q];
      }
    };
    float ps[RT];
    bool far = false;
    scores();
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int q = 0; q < 16; ++q) p[t][q] = fast_exp2(fmaf(p[t][q], cl2, -m[t]));
      ps[t] = sum16(p[t]);
      far |= !(ps[t] <= kGrowSum) || m[t] == kNoRef;
    }
    if (__builtin_expect(__any(far), 0)) {
      scores();
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float mx = p[t][0];
#pragma unroll
        for (int q = 1; q < 16; ++q) mx = fmaxf(mx, p[t][q]);
        mx = halves_max(mx);
        const bool none = !(mx > 0.5f * kNegBig);  // every slot hidden: the reference stays
        const float grow = none ? 0.f : ref_growth(fmaf(mx, cl2, -m[t]), m[t]);
        const float al = ref_rescale(grow, m[t]);
        m[t] += grow;
        lsum[t] *= al;
#pragma unroll
        for (int dt = 0; dt < C::NDT; ++dt) o[t][dt] *= al;
#pragma unroll
        for (int q = 0; q < 16; ++q) p[t][q] = fast_exp2(fmaf(p[t][q], cl2, -m[t]));
        ps[t] = sum16(p[t]);
      }
    }
    // weights in two rounded bf16 parts, 17 bits: off by 2^-18 of each term, where the result is
    // rounded to 2^-9 of itself (with a third part, and the exact maximum at every block, the prefix
    // alone took 87 us instead of 66)
    bf16x8 pw[RT][2][2];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      lsum[t] += ps[t];
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const bf16 hi = (bf16)p[t][q];
        pw[t][0][q >> 3][q & 7] = hi;
        pw[t][1][q >> 3][q & 7] = (bf16)(p[t][q] - (float)hi);
      }
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int dt = 0; dt < C::NDT; ++dt) {
        const bf16x8 vf = pf_ldv<DH>(smem, lo, vh, hf, dt);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u) o[t][dt] = mma32(o[t][dt], vf, pw[t][u][hf]);
      }
    st = st + 1 == C::NS ? 0 : st + 1;
  }
  wait_copies<0>();  // no copy may land in the staging below, or after the block ends
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
  __syncthreads();
  // a tile's states through LDS: a wave's own rows (RW = 2), or the two waves' merged
  float* so = (float*)(smem + w * C::MERGE);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float lt = halves_sum(lsum[t]);
#pragma unroll
    for (int dt = 0; dt < C::NDT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = o[t][dt][4 * g + i];
        *(f32x4*)(so + r * C::OLD + 32 * dt + 8 * g + 4 * h) = v;
      }
    if (h == 0) {
      so[32 * C::OLD + 2 * r] = m[t] / cl2;  // in score units, as decode_block's
      so[32 * C::OLD + 2 * r + 1] = lt;
    }
    __syncthreads();
    for (int e = RW == 2 ? lane : tid; e < 32 * DH; e += RW == 2 ? 64 : 128) {
      const int gi = e / DH, dd = e - gi * DH, to = __shfl(row[t], gi, 64);
      if (to < 0) continue;
      const float* s_a = RW == 2 ? so : (const float*)smem;
      float M = s_a[32 * C::OLD + 2 * gi], lw = s_a[32 * C::OLD + 2 * gi + 1];
      float ow = s_a[gi * C::OLD + dd];
      if constexpr (RW == 1) {
        const float* s_b = (const float*)(smem + C::MERGE);
        merge_state(M, lw, &ow, s_b[32 * C::OLD + 2 * gi], s_b[32 * C::OLD + 2 * gi + 1],
                    s_b + gi * C::OLD + dd, 1, cl2);
      }
      float* dst = px.part + ((long)to * a.nsplit + split) * (DH + 2);
      dst[dd] = ow;
      if (dd == 0) {
        dst[DH] = M;
        dst[DH + 1] = lw;
      }
    }
    __syncthreads();
  }
}

template <int DH, int RW, int RT, bool ONCE>
__global__ __launch_bounds__(128) __attribute__((amdgpu_waves_per_eu(2)))
void attend_shared_mfma_kernel(DecodeArgs<bf16> a, PrefixSpan px) {
  constexpr int kOwn = 2 * DecMfma<DH, 2>::RING, kPre = PrefixCfg<DH, RW, RT>::SMEM;
  __shared__ __align__(16) char smem[kOwn > kPre ? kOwn : kPre];
  if ((int)blockIdx.x < px.blocks) {
    prefix_block<DH, RW, RT>(a, px, smem);
    return;
  }
  const int x = blockIdx.x - px.blocks, y = x / px.own;
  decode_block<DH, 2, false, ONCE, false, false>(a, x % px.own, y % px.slices, y / px.slices, smem);
}

template <typename T, int DH, bool WIN, bool SCORES>
static void decode_rows(const DecodeArgs<T>& a, int G, dim3 grid, hipStream_t s) {
  if (G <= 1)
    hipLaunchKernelGGL((attend_decode_kernel<T, DH, 1, WIN, SCORES>), grid, dim3(256), 0, s, a);
  else if (G <= 2)
    hipLaunchKernelGGL((attend_decode_kernel<T, DH, 2, WIN, SCORES>), grid, dim3(256), 0, s, a);
  else if (G <= 4)
    hipLaunchKernelGGL((attend_decode_kernel<T, DH, 4, WIN, SCORES>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((attend_decode_kernel<T, DH, 8, WIN, SCORES>), grid, dim3(256), 0, s, a);
}

template <typename T, int DH>
static void decode_dispatch(const DecodeArgs<T>& a, int G, dim3 grid, hipStream_t s) {
  if (a.scores) decode_rows<T, DH, false, true>(a, G, grid, s);
  else if (a.window > 0) decode_rows<T, DH, true, false>(a, G, grid, s);
  else decode_rows<T, DH, false, false>(a, G, grid, s);
}

// Splits of the matrix-core kernel: slots per workgroup halved (down to decode_split_len,
// which sizes the partials' workspace) only until the grid holds this many workgroups, 2 per
// CU: a workgroup's set-up and merge cost about as much as 300 slots (B = 8, ctx 4001:
// 512 workgroups or more 132 us a step, 1024 or more 147, 2048 or more 167). Only channels
// with a reader count: layer by layer one of the k has one, and with all of them counted
// (us a layer, query and attention) k = 12, 16 heads of 64, B 2, ctx 8191 took 89 and takes
// 34; k = 12, 12 heads of 64, B 4, ctx 4000 86 and 30; k = 16, 6/3 heads of 96, B 8, ctx 4000
// 54 and 30.
constexpr long kDecodeMfmaBlocks = 512;
// Cache bytes from which a call's slots are taken to be read from HBM. Attention alone, us,
// plain copies / non-temporal ones: 221 MB 133 / 124 a step; at 13 MB that the next call
// reads again (B 1, ctx 709, L 16, layer by layer) 475 / 490 a token, so what the Infinity
// Cache (256 MB) can keep next to the rest of a step stays plain.
constexpr long kDecodeStreamBytes = 128L << 20;

// The matrix-core kernel's grid of the sequences' own slots: splits (a.split_len and a.nsplit are
// set, the latter with `more` states of others), row tiles, and whether the slots are read once.
struct DecodePlan {
  int own, z;
  bool once;
};
template <int DH>
static DecodePlan decode_plan(DecodeArgs<bf16>& a, int G, int nlive, const Shape& sh, int more) {
  const int z = std::max(1, (G + 31) / 32);
  const long slices = (long)nlive * sh.B * sh.Hkv * z, kend = (long)sh.ctx_max + sh.span();
  int len = kSplitMax;
  while (len > a.split_len && slices * ((kend + len - 1) / len) < kDecodeMfmaBlocks) len /= 2;
  a.split_len = len;  // at least decode_split_len, so the partials fit their workspace
  const int own = std::max(1, (int)((kend + len - 1) / len));
  a.nsplit = more + own;
  // a cache read once by one row tile, and larger (all channels: layer by layer, the other
  // layers' calls read theirs in between) than the caches keep from call to call
  const bool once = z == 1 && 4L * sh.k * sh.B * sh.Hkv * kend * DH >= kDecodeStreamBytes;
  return {own, z, once};
}

template <int DH>
static void decode_mfma(DecodeArgs<bf16>& a, int G, int nlive, const Shape& sh, int more,
                        hipStream_t s) {
  const auto [own, z, once] = decode_plan<DH>(a, G, nlive, sh, more);
  const long slices = (long)nlive * sh.B * sh.Hkv * z, kend = (long)sh.ctx_max + sh.span();
  const int len = a.split_len;
  const dim3 grid(own, sh.Hkv * sh.B * nlive, z);
  // Waves per workgroup: 2, which leaves a CU's LDS to five workgroups (three at head dim
  // 96); 1 where a workgroup's walk is at most 128 slots (four blocks); 4 where the workgroups
  // fit the CUs all at once with four (one per CU at head dim 96, two at 64), and at head dim
  // 64 for long walks in several rounds of workgroups. Attention alone with 1 / 2 / 4 waves, us:
  // ctx 100, B 64, L 24, k 12, heads of 64: 77 / 87 / 111; ctx 4000, B 4: 172 / 126 / 133; ctx
  // 1500, B 16, L 12: 144 / 156 / 144; ctx 3000, B 24: 426 / 424 / 400; heads of 96, k = 8: ctx
  // 1000, B 4: 19 / 16.7 / 18.7; ctx 8000, B 1, k = 2: 31 / 26 / 23.6. One layer of 16 heads of
  // 64 with its query, 2 / 4 waves: ctx 700, B 1 19.6 / 19.1; ctx 3000, B 8 38.9 / 33.5; ctx 7948,
  // B 8 62.5 / 57.7; of 12 heads 60.1 / 48.2.
  const long wgs = own * slices, per = std::min<long>(kend, len), cus = device_cus();
  const bool four = DH == 96 ? wgs <= cus : wgs <= 2 * cus || (wgs > 5 * cus && per >= 1024);
  const int waves = per <= 128 ? 1 : four ? 4 : 2;
#define WM_DEC_GO(NW, ...)                                                                    \
  hipLaunchKernelGGL((attend_decode_mfma_kernel<DH, NW, __VA_ARGS__>), grid, dim3(64 * (NW)), \
                     0, s, a)
#define WM_DEC_NW(...)                                                                         \
  do {                                                                                         \
    if (waves == 1) WM_DEC_GO(1, __VA_ARGS__);                                                 \
    else if (waves == 2) WM_DEC_GO(2, __VA_ARGS__);                                            \
    else WM_DEC_GO(4, __VA_ARGS__);                                                            \
  } while (0)
  if (a.doc) {
    if (once) WM_DEC_NW(true, true);
    else WM_DEC_NW(true, false);
  } else if (a.scores) {
    if (once) WM_DEC_NW(false, true, false, true);
    else WM_DEC_NW(false, false, false, true);
  } else if (a.window > 0) {
    if (once) WM_DEC_NW(false, true, true);
    else WM_DEC_NW(false, false, true);
  } else {
    if (once) WM_DEC_NW(false, true);
    else WM_DEC_NW(false, false);
  }
#undef WM_DEC_NW
#undef WM_DEC_GO
}

// Arguments of a call, its channels with a reader in a.live, their number and the most rows of a
// (channel, sequence, KV head) with them.
template <typename T>
static DecodeArgs<T> decode_args(const Shape& sh, const LayerTable& chan_map,
                                 const ChannelGroups& cg, const T* Q, const T* Kc, const T* Vc,
                                 const T* Kd, const T* Vd, const int32_t* ctx_len,
                                 const int32_t* doc, float* partials, T* O, int* nlive, int* G) {
  DecodeArgs<T> a{Q, Kc, Vc, Kd, Vd, ctx_len, doc, partials, O, sh.B, sh.T_new, sh.L, sh.Hq, sh.Hkv,
                  sh.S_cap, sh.mask_paper, decode_splits(sh), decode_split_len(sh), sh.gs, sh.gq,
                  sh.ctx_hi, kLog2e / sqrtf((float)sh.d), chan_map, {}, cg};
  int maxmem = 0, live = 0;
  for (int c = 0; c < sh.k; ++c) {
    int n = cg.offsets[c + 1] - cg.offsets[c];
    if (n == 0) continue;
    a.cg.offsets[live] = cg.offsets[c];
    a.live.v[live++] = c;
    if (n > maxmem) maxmem = n;
  }
  a.cg.offsets[live] = cg.offsets[sh.k];
  *nlive = live;
  *G = maxmem * (sh.Hq / sh.Hkv) * sh.T_new;
  return a;
}

// The splits' partial states from a.part on; a row has a.nsplit in all, `more` of them others'.
template <typename T>
static void decode_states(DecodeArgs<T>& a, const Shape& sh, int G, int nlive, int more,
                          hipStream_t s) {
  if constexpr (sizeof(T) == 2) {  // fp32 at d = 96 is rejected by validation
    if (sh.d == 96) return decode_mfma<96>(a, G, nlive, sh, more, s);
    if (sh.d == 64) return decode_mfma<64>(a, G, nlive, sh, more, s);
  }
  const dim3 grid(a.nsplit, sh.Hkv * sh.B * nlive);
  a.nsplit += more;
  if constexpr (sizeof(T) == 4) {
    if (sh.d == 64) return decode_dispatch<T, 64>(a, G, grid, s);
  }
  decode_dispatch<T, 32>(a, G, grid, s);
}

template <typename T, bool LSE = false>
static void decode_combine(const DecodeArgs<T>& a, int d, hipStream_t s) {
  const long rows = (long)a.L * a.B * a.Hq * a.T_new;
  const dim3 grid((unsigned)((rows + 3) / 4));
  if constexpr (sizeof(T) == 2) {
    if (d == 96) {
      hipLaunchKernelGGL((attend_combine_kernel<bf16, 96, LSE>), grid, dim3(256), 0, s, a);
      return;
    }
  }
  if (d == 64) hipLaunchKernelGGL((attend_combine_kernel<T, 64, LSE>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attend_combine_kernel<T, 32, LSE>), grid, dim3(256), 0, s, a);
}

template <typename T>
void launch_attend_decode(const Shape& shape, const LayerTable& chan_map, const ChannelGroups& cg,
                          const T* Q, const T* Kc, const T* Vc, const T* Kd, const T* Vd,
                          const int32_t* ctx_len, const int32_t* doc, float* partials, T* O,
                          hipStream_t s, const Reach* reach) {
  if (shape.N() <= 0) return;
  Shape sh = shape;
  if (reach) sh.ctx_max = (int)(window_slots(shape, *reach) - shape.span());  // walked slots
  int nlive, G;
  DecodeArgs<T> a = decode_args<T>(sh, chan_map, cg, Q, Kc, Vc, Kd, Vd, ctx_len, doc, partials, O,
                                   &nlive, &G);
  if (reach) a.window = reach->window, a.sinks = reach->sinks;
  decode_states<T>(a, sh, G, nlive, 0, s);
  decode_combine<T>(a, sh.d, s);
}

// -- weighed
static long weigh_ld(const Shape& sh) { return ((long)sh.ctx_max + sh.span() + 31) / 32 * 32; }
size_t decode_scores_bytes(const Shape& sh) {
  return (size_t)sh.L * sh.N() * sh.Hq * weigh_ld(sh) * sizeof(float);
}

template <typename T>
void launch_weigh_decode(const Shape& sh, const LayerTable& chan_map, const ChannelGroups& cg,
                         const T* Q, const T* Kc, const T* Vc, const T* Kd, const T* Vd,
                         const int32_t* ctx_len, float* partials, float* scores, float* lse, T* O,
                         float* weight, hipStream_t s) {
  if (sh.N() <= 0) return;
  int nlive, G;
  DecodeArgs<T> a = decode_args<T>(sh, chan_map, cg, Q, Kc, Vc, Kd, Vd, ctx_len, nullptr, partials,
                                   O, &nlive, &G);
  a.scores = scores;
  a.lse = lse;
  a.s_ld = weigh_ld(sh);
  decode_states<T>(a, sh, G, nlive, 0, s);
  decode_combine<T, true>(a, sh.d, s);
  const dim3 grid((unsigned)((a.s_ld / 4 + 255) / 256), (unsigned)(sh.Hkv * sh.B * nlive));
  hipLaunchKernelGGL(decode_weigh_kernel<T>, grid, dim3(256), 0, s, a, weight);
}

// -- shared prefix
// The prefix's grid by the dims alone (it sizes the workspace): row tiles per workgroup, splits.
struct PrefixPlan {
  int rw, rt, z, nsplit, split_len;
};
static PrefixPlan prefix_plan(const Shape& sh, int P) {
  const long rows = (long)sh.L * sh.B * (sh.Hq / sh.Hkv) * sh.T_new / sh.k;  // of a slice, evenly
  PrefixPlan p{rows > 32 ? 2 : 1, rows > 64 ? 2 : 1, 1, 1, std::max(P, 1)};
  p.z = (int)std::max(1L, (rows + 32 * p.rt * p.rw - 1) / (32 * p.rt * p.rw));
  // Splits until there are three workgroups for two CUs, of 256 slots or more: the sequences' own
  // workgroups take the places left, and every split is a state per row to write and read. (us a
  // call with 2 / 4 / 8 splits: 64 sequences over 4096 + 300 slots, 192 slices of 128 rows 222 /
  // 232 / 248; over 4096 + 100, 24 slices of 256 rows of 96 111 / 72 / 64.)
  const long base = (long)sh.k * sh.Hkv * p.z, cus = device_cus();
  const long most = std::max(1, (P + kSplitMin - 1) / kSplitMin);
  p.nsplit = (int)std::min(most, std::max(1L, (3 * cus / 2 + base - 1) / base));
  p.split_len = ((P + p.nsplit - 1) / p.nsplit + 63) / 64 * 64;
  p.nsplit = std::max(1, (P + p.split_len - 1) / std::max(p.split_len, 1));
  return p;
}
size_t decode_shared_bytes(const Shape& sh, int P) {
  const size_t rows = (size_t)sh.L * sh.B * sh.Hq * sh.T_new;
  return rows * (decode_splits(sh) + (P > 0 ? prefix_plan(sh, P).nsplit : 0)) * (sh.d + 2) *
         sizeof(float);
}

template <int DH>
static void shared_mfma(DecodeArgs<bf16>& a, const Reach& r, const PrefixPlan& p, int G, int nlive,
                        const Shape& sh, hipStream_t s) {
  const DecodePlan d = decode_plan<DH>(a, G, nlive, sh, p.nsplit);
  const int rows = 32 * p.rt * p.rw, z = (G * sh.B + rows - 1) / rows;
  const PrefixSpan px{(const bf16*)r.Kp, (const bf16*)r.Vp, r.P, r.P_cap, p.nsplit, p.split_len, z,
                      z * p.nsplit * sh.Hkv * nlive, d.own, sh.Hkv * sh.B * nlive,
                      a.part};
  a.part += (long)p.nsplit * (DH + 2);
  const dim3 grid((unsigned)(px.blocks + (long)d.own * px.slices * d.z));
#define WM_SHARED_GO(RW, RT)                                                                     \
  do {                                                                                           \
    if (d.once)                                                                                  \
      hipLaunchKernelGGL((attend_shared_mfma_kernel<DH, RW, RT, true>), grid, dim3(128), 0, s, a,  \
                         px);                                                                    \
    else                                                                                         \
      hipLaunchKernelGGL((attend_shared_mfma_kernel<DH, RW, RT, false>), grid, dim3(128), 0, s, a, \
                         px);                                                                    \
  } while (0)
  if (p.rt == 2) WM_SHARED_GO(2, 2);
  else if (p.rw == 2) WM_SHARED_GO(2, 1);
  else WM_SHARED_GO(1, 1);
#undef WM_SHARED_GO
}

template <typename T>
void launch_shared_decode(const Shape& sh, const Reach& r, const LayerTable& chan_map,
                          const ChannelGroups& cg, const T* Q, const T* Kc, const T* Vc,
                          const T* Kd, const T* Vd, const int32_t* ctx_len, float* partials, T* O,
                          hipStream_t s) {
  if (sh.N() <= 0) return;
  int nlive, G;
  DecodeArgs<T> a = decode_args<T>(sh, chan_map, cg, Q, Kc, Vc, Kd, Vd, ctx_len, nullptr, partials,
                                   O, &nlive, &G);
  const PrefixPlan p = prefix_plan(sh, r.P);
  const int more = r.P > 0 ? p.nsplit : 0;
  bool done = false;
  if constexpr (sizeof(T) == 2) {
    done = sh.d != 32 && r.P > 0;
    if (done) sh.d == 96 ? shared_mfma<96>(a, r, p, G, nlive, sh, s)
                         : shared_mfma<64>(a, r, p, G, nlive, sh, s);
  }
  if (!done) {
    a.part = partials + (long)more * (sh.d + 2);
    decode_states<T>(a, sh, G, nlive, more, s);
    if (r.P > 0)
      launch_prefix_rows<T>(sh, r, a.live, nlive, a.cg, G * sh.B, Q, partials, a.nsplit, p.nsplit,
                            p.split_len, s);
  }
  a.part = partials;
  decode_combine<T>(a, sh.d, s);
}

#define WM_INST(T)                                                                              \
  template void launch_attend_decode<T>(const Shape&, const LayerTable&, const ChannelGroups&,  \
                                        const T*, const T*, const T*, const T*, const T*,       \
                                        const int32_t*, const int32_t*, float*, T*, hipStream_t, \
                                        const Reach*);                                          \
  template void launch_weigh_decode<T>(const Shape&, const LayerTable&, const ChannelGroups&,   \
                                       const T*, const T*, const T*, const T*, const T*,        \
                                       const int32_t*, float*, float*, float*, T*, float*,      \
                                       hipStream_t);                                            \
  template void launch_shared_decode<T>(const Shape&, const Reach&, const LayerTable&,          \
                                        const ChannelGroups&, const T*, const T*, const T*,     \
                                        const T*, const T*, const int32_t*, float*, T*,         \
                                        hipStream_t);
WM_INST(float)
WM_INST(bf16)
#undef WM_INST

}  // namespace wm
