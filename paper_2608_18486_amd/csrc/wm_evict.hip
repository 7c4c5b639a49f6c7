// Moves of cache rows to other positions: the eviction of lightly attended slots
// (wm_cache_evict) and the layout of a shared prefix (wm_prefix_share).
//
// The library keeps slot = position: a key is stored rotated to its slot. A row that moves
// from slot s to slot j therefore has its key turned by (j - s) positions,
//   (x1, x2) -> (x1 cos a - x2 sin a, x2 cos a + x1 sin a),  a = (j - s) theta^(-2m/d),
// rounded to the cache's type once (at most half a step per move); values move as they are.
// Angles: turns = (j - s) theta^(-2m/d) / 2 pi and its fraction in fp64 (a position of 10^5 has
// 10^4 turns, whose fraction fp32 would leave with 3 digits), sine and cosine in fp32.
#include <algorithm>

#include "wm_device.hpp"
#include "wm_internal.hpp"

namespace wm {

// Ascending order of the weights as unsigned integers; NaN below everything, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w == w)) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

struct EvictArgs {
  const int32_t* ctx_len;
  const float* weight;  // [slices][S_cap]
  int32_t* idx;         // [slices][idx_ld] the kept slots, ascending
  int32_t* kept;        // [slices][keep] the same for the caller, -1 past the last; or null
  float* weight_out;    // [slices][S_out]
  int32_t* ctx_out;
  int B, Hkv, S_cap, S_out, ctx_max, keep, first, recent, idx_ld;
};

// One workgroup per (channel, sequence, KV head): the slots it keeps. The M = keep - first -
// recent heaviest of the candidates [first, n - recent) are those with a key above the M-th
// largest, t, and the lowest ones at t: t is found digit by digit (8 bits at a time, from the
// top) with a histogram of the candidates that share the digits found so far; then one pass in
// slot order writes the kept slots by their running count.
constexpr int kSelThreads = 1024;
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_prefix, s_left;
  __shared__ int s_above[kSelThreads / 64], s_tie[kSelThreads / 64];
  const int slice = blockIdx.x, b = slice / a.Hkv % a.B;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = ctx_at(a.ctx_len, b, a.ctx_max);
  const float* wt = a.weight + (long)slice * a.S_cap;
  int32_t* idx = a.idx + (long)slice * a.idx_ld;
  int32_t* kept = a.kept ? a.kept + (long)slice * a.keep : nullptr;
  float* wo = a.weight_out + (long)slice * a.S_out;
  const int nk = min(n, a.keep);
  if (slice / a.Hkv < a.B && slice % a.Hkv == 0 && tid == 0) a.ctx_out[b] = nk;
  for (int j = nk + tid; j < a.S_out; j += kSelThreads) wo[j] = 0.f;
  if (kept)
    for (int j = nk + tid; j < a.keep; j += kSelThreads) kept[j] = -1;
  if (n <= a.keep) {
    for (int j = tid; j < n; j += kSelThreads) {
      idx[j] = j;
      if (kept) kept[j] = j;
      wo[j] = wt[j];
    }
    return;
  }
  const int lo = a.first, hi = n - a.recent;  // candidates
  const int M = a.keep - a.first - a.recent;  // 0 <= M < hi - lo
  uint32_t prefix = 0, left = (uint32_t)M;  // digits found; rank still to find among them
  if (M > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
      for (int s = lo + tid; s < hi; s += kSelThreads) {
        const uint32_t key = weight_key(wt[s]);
        if ((key & mask) == prefix) atomicAdd(&hist[key >> shift & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        uint32_t rank = left;
        int digit = 255;
        while (digit > 0 && hist[digit] < rank) rank -= hist[digit--];
        s_prefix = prefix | (uint32_t)digit << shift;
        s_left = rank;
      }
      __syncthreads();
      prefix = s_prefix;
      left = s_left;
    }
  }
  // prefix: the M-th largest key; `left` of the candidates at it are kept, the lowest ones
  int at = 0, ties = 0;  // kept so far, candidates at the threshold so far
  for (int s0 = 0; s0 < n; s0 += kSelThreads) {
    const int s = s0 + tid;
    bool always = false, above = false, tie = false;
    float wv = 0.f;
    if (s < n) {
      wv = wt[s];
      always = s < lo || s >= hi;
      const uint32_t key = weight_key(wv);
      above = !always && M > 0 && key > prefix;
      tie = !always && M > 0 && key == prefix;
    }
    const uint64_t bt = __ballot(tie);
    if (lane == 0) s_tie[w] = __popcll(bt);
    __syncthreads();
    int tb = ties, tall = 0;
    for (int k = 0; k < kSelThreads / 64; ++k) {
      if (k < w) tb += s_tie[k];
      tall += s_tie[k];
    }
    const int tr = tb + __popcll(bt & ((1ull << lane) - 1));  // this tie's rank
    const bool take = always || above || (tie && tr < (int)left);
    const uint64_t bk = __ballot(take);
    if (lane == 0) s_above[w] = __popcll(bk);
    __syncthreads();
    int kb = at, kall = 0;
    for (int k = 0; k < kSelThreads / 64; ++k) {
      if (k < w) kb += s_above[k];
      kall += s_above[k];
    }
    if (take) {
      const int j = kb + __popcll(bk & ((1ull << lane) - 1));
      idx[j] = s;
      if (kept) kept[j] = s;
      wo[j] = wv;
    }
    at += kall;
    ties += tall;
    __syncthreads();
  }
}

struct MoveArgs {
  const void *Kc, *Vc;
  void *Ko, *Vo;
  const int32_t* idx;  // source slot of each destination slot, or null: the same slot
  const int32_t* ctx_len;
  int B, Hkv, S_cap, S_out, ctx_max, keep, idx_ld;
  int b0, nb;          // sequences b0 .. b0 + nb - 1 of the source
  int shift;           // added to the destination's position (idx null)
  double theta;
};

// Rows [0, n) of every destination slice: a thread moves 8 elements of the key's first half,
// the 8 they rotate with, and the same of the value.
template <typename T, int DH>
__global__ __launch_bounds__(256) void move_rows_kernel(MoveArgs a) {
  constexpr int H = DH / 2, C = H / 8;  // threads per row
  __shared__ double turn[H];            // turns per position
  for (int m = threadIdx.x; m < H; m += 256)
    turn[m] = pow(a.theta, -2.0 * (double)m / (double)DH) * 0.15915494309189533577;
  __syncthreads();
  const int slice = blockIdx.y;  // destination (channel, sequence, KV head)
  const int h = slice % a.Hkv, b = slice / a.Hkv % a.nb, c = slice / (a.Hkv * a.nb);
  const int n = a.idx ? min(ctx_at(a.ctx_len, a.b0 + b, a.ctx_max), a.keep) : a.keep;
  const long src = (((long)c * a.B + a.b0 + b) * a.Hkv + h) * a.S_cap * DH;
  const long dst = (long)slice * a.S_out * DH;
  const T* K = (const T*)a.Kc + src;
  const T* V = (const T*)a.Vc + src;
  T* Ko = (T*)a.Ko + dst;
  T* Vo = (T*)a.Vo + dst;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < (long)n * C; i += 256l * gridDim.x) {
    const int j = (int)(i / C), e = (int)(i % C) * 8;
    const int s = a.idx ? a.idx[(long)slice * a.idx_ld + j] : j;
    float x1[8], x2[8];
    load8(K + (long)s * DH + e, x1);
    load8(K + (long)s * DH + H + e, x2);
    const frag_t<T> v1 = ld_frag<T>(V + (long)s * DH + e);
    const frag_t<T> v2 = ld_frag<T>(V + (long)s * DH + H + e);
    const double by = (double)(j + a.shift - s);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const double t = by * turn[e + u];
      float sn, cs;
      sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
      const float p = x1[u], q = x2[u];
      x1[u] = p * cs - q * sn;
      x2[u] = q * cs + p * sn;
    }
    store8(Ko + (long)j * DH + e, x1);
    store8(Ko + (long)j * DH + H + e, x2);
    st_frag<T>(Vo + (long)j * DH + e, v1);
    st_frag<T>(Vo + (long)j * DH + H + e, v2);
  }
}

template <typename T> static void move_rows(const MoveArgs& a, int k, int d, hipStream_t s) {
  const long per = (long)a.keep * (d / 16);
  const dim3 grid((unsigned)std::min<long>((per + 255) / 256, 64), (unsigned)(k * a.nb * a.Hkv));
  if (d == 32) hipLaunchKernelGGL((move_rows_kernel<T, 32>), grid, dim3(256), 0, s, a);
  else if (d == 64) hipLaunchKernelGGL((move_rows_kernel<T, 64>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((move_rows_kernel<T, 96>), grid, dim3(256), 0, s, a);
}

size_t evict_index_bytes(const Shape& sh) {
  return (size_t)sh.k * sh.B * sh.Hkv * std::max(sh.ctx_max, 1) * sizeof(int32_t);
}

void launch_evict(const Shape& sh, const int32_t* ctx_len, int keep, int first, int recent,
                  const float* weight, const void* Kc, const void* Vc, int S_out,
                  int32_t* ctx_out, float* weight_out, void* Ko, void* Vo, int32_t* kept,
                  int32_t* idx, bool bf, hipStream_t s) {
  const int ld = std::max(sh.ctx_max, 1);
  const EvictArgs e{ctx_len, weight, idx, kept, weight_out, ctx_out, sh.B, sh.Hkv, sh.S_cap,
                    S_out, sh.ctx_max, keep, first, recent, ld};
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)(sh.k * sh.B * sh.Hkv)),
                     dim3(kSelThreads), 0, s, e);
  const int most = std::min(keep, sh.ctx_max);
  if (most == 0) return;
  const MoveArgs m{Kc, Vc, Ko, Vo, idx, ctx_len, sh.B, sh.Hkv, sh.S_cap, S_out, sh.ctx_max, most,
                   ld, 0, sh.B, 0, (double)sh.rope_theta};
  if (bf) move_rows<bf16>(m, sh.k, sh.d, s);
  else move_rows<float>(m, sh.k, sh.d, s);
}

void launch_prefix_share(const Shape& sh, const void* Kc, const void* Vc, int seq, int len,
                         int P_cap, void* Kp, void* Vp, bool bf, hipStream_t s) {
  const MoveArgs m{Kc, Vc, Kp, Vp, nullptr, nullptr, sh.B, sh.Hkv, sh.S_cap, P_cap, 0, len, 0,
                   seq, 1, -len, (double)sh.rope_theta};
  if (bf) move_rows<bf16>(m, sh.k, sh.d, s);
  else move_rows<float>(m, sh.k, sh.d, s);
}

}  // namespace wm
