// Building blocks of the full-sequence attention kernels (wm_attend.hip, wm_reach.hip): softmax
// references, the tile shapes, and the rings of K/V blocks in LDS.
#pragma once
#include <type_traits>

#include "wm_device.hpp"
#include "wm_frag.hpp"
#include "wm_internal.hpp"

namespace wm {

template <typename T>
__device__ __forceinline__ frag_t<T> ld_frag_4_4(const T* p0, const T* p1);
template <>
__device__ __forceinline__ bf16x8 ld_frag_4_4<bf16>(const bf16* p0, const bf16* p1) {
  bf16x4 a = *(const bf16x4*)p0, b = *(const bf16x4*)p1;
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <>
__device__ __forceinline__ f32x8 ld_frag_4_4<float>(const float* p0, const float* p1) {
  f32x4 a = *(const f32x4*)p0, b = *(const f32x4*)p1;
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A lane's sum of 16 softmax weights above this (some weight above 2^12) triggers the
// rescale of the running state; `!(ps <= kGrowSum)` also catches inf and NaN.
constexpr float kGrowSum = 65536.0f;
// Reference of a row that has seen no slot yet, in log2 units. Finite and small, so
// scores offset by it keep their digits; a row still at kNoRef always takes the
// exact-max rescale, which then sets the reference to the row's exact maximum (up or
// down: its state is still zero). Only a step that hides every slot from the row
// leaves it at kNoRef.
constexpr float kNoRef = -100.0f;

// Growth of a row's reference at a rescale, from the step's row maximum mx (in log2
// units relative to the current reference m): never down once a slot has been read;
// from kNoRef, exactly to the row maximum unless the step hid every slot from the row.
__device__ __forceinline__ float ref_growth(float mx, float m) {
  return m == kNoRef ? (mx > 0.5f * kNegBig ? mx : 0.f) : fmaxf(mx, 0.f);
}
// Factor of the running state at that rescale: a row still at kNoRef has a zero state,
// and exp2(-growth) could overflow when the reference moves down.
__device__ __forceinline__ float ref_rescale(float growth, float m) {
  return m == kNoRef ? 0.f : fast_exp2(-growth);
}

#ifndef WM_PREFILL_WAVES
#define WM_PREFILL_WAVES 8
#endif
constexpr int kPrefillWaves = WM_PREFILL_WAVES;  // waves per prefill workgroup

template <typename T, int DH> struct PrefillCfg {
  static constexpr int NW = kPrefillWaves;
  static constexpr int QT = 256 / (32 * NW);  // 32-query tiles per wave (256 queries per block)
  static constexpr int NT = 64 * NW;    // threads
  static constexpr int BQ = 32 * QT * NW;  // queries per workgroup
  static constexpr int BKV = 64;        // keys per block
  static constexpr int PAD = sizeof(T) == 2 ? 8 : 4;
  static constexpr int LDK = DH + PAD;   // Ks: [BKV][LDK]
  // bf16 V is staged row-major like K ([BKV][LDV], read transposed by ds_read_b64_tr_b16);
  // fp32 V is stored transposed ([DH][LDV])
  static constexpr bool VTR = sizeof(T) == 2;
  static constexpr int LDV = VTR ? DH + 16 : BKV + PAD;
  static constexpr int VS = VTR ? BKV * LDV : DH * LDV;  // V stage (elements)
  static constexpr int NKS = DH / 16;    // k16 steps of Q K^T
  static constexpr int NDT = DH / 32;    // 32-row tiles of O^T
  static constexpr int KIT = BKV * DH / 8;             // K fragments per block
  static constexpr int KFR = (KIT + NT - 1) / NT;      // ... per thread
  static constexpr int VIT = VTR ? KIT : (BKV / 2) * (DH / 8);  // V items per block (16-B
                                                                 // fragments, or key pairs)
  static constexpr int VPT = (VIT + NT - 1) / NT;      // ... per thread
};

// Paired-key transposed store of two V rows' 8 columns: Vt[c][key], Vt[c][key+1].
__device__ __forceinline__ void st_pair_t(bf16* vt, int ld, const bf16x8& a, const bf16x8& b) {
#pragma unroll
  for (int i = 0; i < 8; ++i) *(bf16x2*)(vt + i * ld) = bf16x2{a[i], b[i]};
}
__device__ __forceinline__ void st_pair_t(float* vt, int ld, const f32x8& a, const f32x8& b) {
#pragma unroll
  for (int i = 0; i < 8; ++i) *(f32x2*)(vt + i * ld) = f32x2{a[i], b[i]};
}

// V^T fragment for keys kb + 4h + {0..3, 8..11} and value column 32 dt + r from a
// row-major bf16 V tile, with two transposing LDS reads: within each 16-lane group,
// lane i's element t comes from element i % 4 of the 8-byte chunk addressed by lane
// 4t + i / 4, so lane j addresses key (kb + 4h + 8s + j / 4), columns
// 32 dt + 16 (group & 1) + 4 (j % 4) .. + 3, and receives 4 keys of its own column.
__device__ __forceinline__ bf16x8 ld_vt_tr(const bf16* vs, int ldv, int kb, int dt, int lane) {
  const int j = lane & 15, grp = lane >> 4, h = lane >> 5;
  const bf16* p = vs + (kb + 4 * h + (j >> 2)) * ldv + 32 * dt + 16 * (grp & 1) + 4 * (j & 3);
  typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
  const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 8 * ldv));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// -- bf16, head dims 64 and 96: K/V blocks of 64 slots copied straight into LDS -----------
constexpr int kPfWaves = 4, kPfNs = 3, kPfQt = 1;
// work queue of the persistent kernel: one counter per XCD, 64 bytes apart
constexpr int kQueueStride = 16, kQueueWords = kNumXcd * kQueueStride;
static_assert(kQueueWords * 4 == kPrefillQueueBytes, "queue size");
template <int QT, int DH_> struct PfDma {
  static constexpr int NW = kPfWaves, NT = 64 * NW;
  static constexpr int BQ = 32 * QT * NW;              // queries per workgroup
  static constexpr int BKV = 64, DH = DH_;
  static constexpr int NKS = DH / 16;                  // k16 steps of S (= step groups)
  static constexpr int NDT = DH / 32;                  // 32-column tiles of O^T
  static constexpr int ROW_BYTES = DH * 2;             // one slot row of K or V
  static constexpr int CPR = ROW_BYTES / 16;           // 16-B chunks per row
  static constexpr int BLK_BYTES = BKV * ROW_BYTES;    // one K (or V) block
  static constexpr int RPW = BKV / NW;                 // block rows each wave copies
  static constexpr int NI = RPW * ROW_BYTES / 1024;    // ... in copy instructions of 1 KB
  // Two rings of NS blocks. While block j is processed, K of j and j+1 and V of j-1 and
  // j are read; K of j+2 and V of j+1 (and, with 4 blocks, K of j+3 and V of j+2) are
  // in flight.
  static constexpr int NS = kPfNs;
  static constexpr int V_BASE = NS * BLK_BYTES;        // K ring first, then the V ring
  static constexpr int SMEM_BYTES = 2 * NS * BLK_BYTES;
  static constexpr int WPE = DH == 64 ? 3 : 2;         // waves per SIMD
  static_assert((DH == 64 || DH == 96) && NI * 1024 == RPW * ROW_BYTES && (NS == 3 || NS == 4),
                "tile shapes");
  static_assert(SMEM_BYTES % (16 * NT) == 0, "the rings are zeroed in whole passes");
};

// byte offsets of the K and V ring half blocks: ring stage u, half hf
template <int DH> constexpr uint32_t pf_kh(int u, int hf) {
  return u * 64 * 2 * DH + hf * 32 * 2 * DH;
}
template <int DH> constexpr uint32_t pf_vh(int u, int hf) {
  return kPfNs * 64 * 2 * DH + u * 64 * 2 * DH + hf * 32 * 2 * DH;
}

// S^T fragment rows of one step for one query tile: the 32 K slots of the half block
// at kh against the lane's query column, accumulated on top of acc.
template <int DH>
__device__ __forceinline__ f32x16 pf_scores(const char* sm, const PfLane<DH>& lo, uint32_t kh,
                                            const bf16x8 (&qf)[DH / 16], f32x16 acc) {
  bf16x8 kf[DH / 16];
#pragma unroll
  for (int ks = 0; ks < DH / 16; ++ks) kf[ks] = pf_ldk<DH>(sm, lo, kh, ks);
#pragma unroll
  for (int ks = 0; ks < DH / 16; ++ks) acc = mma32(acc, kf[ks], qf[ks]);
  return acc;
}

// 4 bf16 at byte offset off of a buffer view (zeros out of range)
__device__ __forceinline__ bf16x4 buf_ld8(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
}

// f(integral_constant<int, I>) for I = I0 .. N-1, in order.
template <int I0, int N, class F> __device__ __forceinline__ void static_for(F& f) {
  if constexpr (I0 < N) {
    f(std::integral_constant<int, I0>());
    static_for<I0 + 1, N>(f);
  }
}

// Sum of v[Q0 .. Q1) as a balanced tree.
template <int Q0, int Q1> __device__ __forceinline__ float tree_sum(const f32x16& v) {
  if constexpr (Q1 - Q0 == 1) return v[Q0];
  else {
    constexpr int QM = Q0 + (Q1 - Q0) / 2;
    return tree_sum<Q0, QM>(v) + tree_sum<QM, Q1>(v);
  }
}

}  // namespace wm
