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
#include <cmath>

#include "wm_device.hpp"
#include "wm_internal.hpp"

namespace wm {

// Ascending order of the weights as unsigned integers in [1, 2^32 - 2]; NaN below everything, -0
// as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  const uint32_t k = u >> 31 ? ~u : u | 0x80000000u;
  return w == w ? k : 1u;
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

// One workgroup per (channel, sequence, KV head): the slots it keeps, the `keep` largest keys and
// of equal ones the lowest slots (the first and the recent slots get the largest key of all). The
// keep-th largest key, t, is found digit by digit (11, 11 and 10 bits from the top): a histogram in
// LDS of the keys that share the digits found so far, whose running sum from the largest bin down
// every thread takes part in. Then one pass in slot order writes the slots above t, and as many at t
// as are missing, by their running count. The weights are read once: the first 1024 R slots' keys
// stay in registers (a wave owns 64 R neighbouring slots, so its running count needs the other
// waves' totals only); slots past them are read again for every digit. What bounds it is the issue
// of instructions: two bits at a time by ballots, 16 rounds of 24 compares a wave, took 114 us at
// 1536 slices of up to 8191 slots and 12 at 36 of 900; this way 51 and 8; histograms of 8 bits
// scanned by one thread 155 and 38.
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
template <int R>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(EvictArgs a) {
  constexpr int kBins = 2 * kSelThreads;
  __shared__ uint32_t s_hist[kBins], s_found[2];
  __shared__ int s_above[kSelWaves], s_tie[kSelWaves];
  const int slice = blockIdx.x, b = slice / a.Hkv % a.B;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = __builtin_amdgcn_readfirstlane(ctx_at(a.ctx_len, b, a.ctx_max));
  const float* wt = a.weight + (long)slice * a.S_cap;
  int32_t* idx = a.idx + (long)slice * a.idx_ld;
  int32_t* kept = a.kept ? a.kept + (long)slice * a.keep : nullptr;
  float* wo = a.weight_out + (long)slice * a.S_out;
  const int nk = min(n, a.keep);
  if (slice < a.B * a.Hkv && slice % a.Hkv == 0 && tid == 0) a.ctx_out[b] = nk;
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
  const int lo = a.first, hi = n - a.recent;  // slots in between are chosen by weight
  constexpr int RD = kSelThreads * R;         // slots per round of the registers
  const bool more = n > RD;
  auto slot = [&](int rd, int j) { return rd + (w * R + j) * 64 + lane; };
  auto load = [&](int s) { return s < n ? wt[s] : 0.f; };
  auto key_of = [&](int s, float x) {  // 0 past the last slot: below every threshold
    const uint32_t k = s >= lo && s < hi ? weight_key(x) : ~0u;
    return s < n ? k : 0u;
  };
  uint32_t key[R];
  float wv[R];
#pragma unroll
  for (int j = 0; j < R; ++j) wv[j] = load(slot(0, j));
#pragma unroll
  for (int j = 0; j < R; ++j) key[j] = key_of(slot(0, j), wv[j]);
  uint32_t t = 0, rank = (uint32_t)a.keep;  // digits found; rank among the keys that share them
  int done = 0;                             // bits found
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass < 2 ? 11 : 10, shift = 32 - done - bits;
    s_hist[2 * tid] = s_hist[2 * tid + 1] = 0;
    __syncthreads();
    auto add = [&](uint32_t k) {
      if (done == 0 || k >> (32 - done) == t >> (32 - done))
        atomicAdd(&s_hist[k >> shift & ((1u << bits) - 1)], 1u);
    };
    if (64 * R * w < n) {  // (a wave past the last slot has nothing to count)
#pragma unroll
      for (int j = 0; j < R; ++j) add(key[j]);
    }
    if (more)
      for (int rd = RD; rd < n; rd += RD)
        for (int j = 0; j < R; ++j) {
          const int s = slot(rd, j);
          add(key_of(s, load(s)));
        }
    __syncthreads();
    // this thread's two bins, the largest ones first: thread 0 holds the last two of 2048
    const int bin = kBins - 2 - 2 * tid;
    const uint32_t h1 = s_hist[bin + 1], h0 = s_hist[bin];
    uint32_t run = h1 + h0;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const uint32_t v = __shfl_up(run, x, 64);
      run += lane >= x ? v : 0;
    }
    if (lane == 63) s_above[w] = (int)run;
    __syncthreads();
    uint32_t before = 0;  // keys in larger bins
    for (int v = 0; v < w; ++v) before += (uint32_t)s_above[v];
    before += run - h1 - h0;
    if (before < rank && before + h1 >= rank) s_found[0] = bin + 1, s_found[1] = rank - before;
    else if (before + h1 < rank && before + h1 + h0 >= rank)
      s_found[0] = bin, s_found[1] = rank - before - h1;
    __syncthreads();
    t |= s_found[0] << shift;
    rank = s_found[1];
    done += bits;
  }
  t = __builtin_amdgcn_readfirstlane(t);
  auto exchange = [&](int na, int nt) {  // this wave's counts, everyone's in s_above, s_tie
    if (lane == 0) s_above[w] = na, s_tie[w] = nt;
    __syncthreads();
  };
  auto tally = [&](uint32_t k, int& na, int& nt) {
    na += __popcll(__builtin_amdgcn_ballot_w64(k > t));
    nt += __popcll(__builtin_amdgcn_ballot_w64(k == t));
  };
  int left = a.keep;  // slots at t to take: what the ones above t leave
  if (more) {
    int na = 0, nt = 0;
    for (int rd = RD; rd < n; rd += RD)
      for (int j = 0; j < R; ++j) {
        const int s = slot(rd, j);
        tally(key_of(s, load(s)), na, nt);
      }
    exchange(na, 0);
    for (int v = 0; v < kSelWaves; ++v) left -= s_above[v];
    __syncthreads();
  }
  int at = 0, ties = 0;  // kept, and slots at t, in the rounds before
  for (int rd = 0; rd < n; rd += RD) {
    if (rd > 0) {
#pragma unroll
      for (int j = 0; j < R; ++j) {
        wv[j] = load(slot(rd, j));
        key[j] = key_of(slot(rd, j), wv[j]);
      }
    }
    int na = 0, nt = 0;
#pragma unroll
    for (int j = 0; j < R; ++j) tally(key[j], na, nt);
    exchange(na, nt);
    // before this wave, and in all (lane v holds wave v's counts)
    int ab = lane < w ? s_above[lane % kSelWaves] : 0, tb = lane < w ? s_tie[lane % kSelWaves] : 0;
    int aall = lane < kSelWaves ? s_above[lane % kSelWaves] : 0;
    int tall = lane < kSelWaves ? s_tie[lane % kSelWaves] : 0;
#pragma unroll
    for (int x = 1; x < kSelWaves; x <<= 1) {
      ab += __shfl_xor(ab, x, 64), tb += __shfl_xor(tb, x, 64);
      aall += __shfl_xor(aall, x, 64), tall += __shfl_xor(tall, x, 64);
    }
    ab = __builtin_amdgcn_readfirstlane(ab);
    tb = ties + __builtin_amdgcn_readfirstlane(tb);
    aall = __builtin_amdgcn_readfirstlane(aall);
    tall = __builtin_amdgcn_readfirstlane(tall);
    if (rd == 0) left -= aall;
    // kept before this wave: the rounds before, the waves' above, and the ties taken of theirs
    int kb = at + ab + min(tb, left) - min(ties, left);
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int s = slot(rd, j);
      const uint64_t bt = __builtin_amdgcn_ballot_w64(key[j] == t);
      const bool take = key[j] > t || (key[j] == t && tb + __popcll(bt & below) < left);
      const uint64_t bk = __builtin_amdgcn_ballot_w64(take);
      if (take) {
        const int o = kb + __popcll(bk & below);
        idx[o] = s;
        if (kept) kept[o] = s;
        wo[o] = wv[j];
      }
      kb += __popcll(bk);
      tb += __popcll(bt);
    }
    at += aall + min(ties + tall, left) - min(ties, left);
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
  double log2_theta;
};

// Two halves of 8 elements of a key, from element e of each half on, turned by `by` positions.
__device__ __forceinline__ void turn8(float (&x1)[8], float (&x2)[8], double by,
                                      const double* turn) {
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const double t = by * turn[u];
    float sn, cs;
    sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
    const float p = x1[u], q = x2[u];
    x1[u] = p * cs - q * sn;
    x2[u] = q * cs + p * sn;
  }
}
// Turns per position of a key's element pairs.
template <int DH> __device__ __forceinline__ void turn_table(double* turn, double log2_theta) {
  for (int m = threadIdx.x; m < DH / 2; m += 256)
    turn[m] = exp2(log2_theta * (-2.0 * (double)m / (double)DH)) * 0.15915494309189533577;
  __syncthreads();
}

// y = the rows x turned by `by` positions.
template <typename T, int DH>
__global__ __launch_bounds__(256) void turn_rows_kernel(const T* x, T* y, long rows, int by,
                                                        double log2_theta) {
  constexpr int H = DH / 2, C = H / 8;
  __shared__ double turn[H];
  turn_table<DH>(turn, log2_theta);
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * C) return;
  const long row = i / C;
  const int e = (int)(i % C) * 8;
  float x1[8], x2[8];
  load8(x + row * DH + e, x1);
  load8(x + row * DH + H + e, x2);
  turn8(x1, x2, (double)by, turn + e);
  store8(y + row * DH + e, x1);
  store8(y + row * DH + H + e, x2);
}

// Rows [0, n) of every destination slice: a thread moves 8 elements of the key's first half,
// the 8 they rotate with, and the same of the value.
template <typename T, int DH>
__global__ __launch_bounds__(256) void move_rows_kernel(MoveArgs a) {
  constexpr int H = DH / 2, C = H / 8;  // threads per row
  __shared__ double turn[H];
  turn_table<DH>(turn, a.log2_theta);
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
    turn8(x1, x2, (double)(j + a.shift - s), turn + e);
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
  // keys in registers: up to 1024 slots in one of them, 8192 in 8, else up to 32768 in 32
  const dim3 slices((unsigned)(sh.k * sh.B * sh.Hkv)), blk(kSelThreads);
  if (sh.ctx_max <= kSelThreads)
    hipLaunchKernelGGL(evict_select_kernel<1>, slices, blk, 0, s, e);
  else if (sh.ctx_max <= 8 * kSelThreads)
    hipLaunchKernelGGL(evict_select_kernel<8>, slices, blk, 0, s, e);
  else
    hipLaunchKernelGGL(evict_select_kernel<32>, slices, blk, 0, s, e);
  const int most = std::min(keep, sh.ctx_max);
  if (most == 0) return;
  const MoveArgs m{Kc, Vc, Ko, Vo, idx, ctx_len, sh.B, sh.Hkv, sh.S_cap, S_out, sh.ctx_max, most,
                   ld, 0, sh.B, 0, log2((double)sh.rope_theta)};
  if (bf) move_rows<bf16>(m, sh.k, sh.d, s);
  else move_rows<float>(m, sh.k, sh.d, s);
}

template <typename T>
static void turn_rows(const Shape& sh, const T* x, T* y, int by, hipStream_t s) {
  const long rows = (long)sh.k * sh.Hkv;
  const double lt = log2((double)sh.rope_theta);
  const dim3 grid((unsigned)((rows * (sh.d / 16) + 255) / 256));
  if (sh.d == 32)
    hipLaunchKernelGGL((turn_rows_kernel<T, 32>), grid, dim3(256), 0, s, x, y, rows, by, lt);
  else if (sh.d == 64)
    hipLaunchKernelGGL((turn_rows_kernel<T, 64>), grid, dim3(256), 0, s, x, y, rows, by, lt);
  else
    hipLaunchKernelGGL((turn_rows_kernel<T, 96>), grid, dim3(256), 0, s, x, y, rows, by, lt);
}

void launch_prefix_share(const Shape& sh, const void* Kc, const void* Vc, int seq, int len,
                         int P_cap, void* Kp, void* Vp, const void* Kd, void* Kd_out, bool bf,
                         hipStream_t s) {
  const MoveArgs m{Kc, Vc, Kp, Vp, nullptr, nullptr, sh.B, sh.Hkv, sh.S_cap, P_cap, 0, len, 0,
                   seq, 1, -len, log2((double)sh.rope_theta)};
  if (bf) move_rows<bf16>(m, sh.k, sh.d, s);
  else move_rows<float>(m, sh.k, sh.d, s);
  if (!Kd_out) return;
  if (bf) turn_rows<bf16>(sh, (const bf16*)Kd, (bf16*)Kd_out, -len, s);
  else turn_rows<float>(sh, (const float*)Kd, (float*)Kd_out, -len, s);
}

}  // namespace wm
