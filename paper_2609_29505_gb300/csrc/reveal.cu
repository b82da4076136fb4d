// Reveal step of a masked-token sampler: of a sample's masked positions (inside a window), the n
// with the best scores get their candidates, the others stay masked.
//
// One CTA per sample.  A position's key orders it: the score's order as an unsigned integer (0: not
// to be chosen).  The n-th largest key is found digit by digit, 8 bits at a time from the top,
// with a histogram in shared memory (a radix select); positions with that very key are taken in
// the order of the position.  16 bytes per position and a handful of barriers: latency alone (GB300: 1 x 192
// positions 3.5 us, 16 x 4096 6.5 us).
#include "common.cuh"
#include "kernels.h"

namespace sgd {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;

struct Shared {
  int hist[256];
  int digit, above, same;
  int masked, chosen;
  int warp_count[kWarps];
};

// larger is better; 0 is no score's key.  -0 and +0 are equal, NaN stands with the worst.
__device__ __forceinline__ uint32_t score_key(float s, int lowest) {
  if (lowest) s = -s;
  if (s != s) s = -__builtin_huge_valf();
  const uint32_t b = __float_as_uint(s + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(kThreads) reveal_kernel(const RevealParams p) {
  extern __shared__ uint32_t keys[];  // [n_tokens]
  __shared__ Shared sh;
  const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = static_cast<int64_t>(b) * p.n_tokens;
  const int32_t* ids = p.ids + row;
  int32_t* out = p.ids_out + row;
  const int want = max(p.n_reveal[b], 0);
  int lo = 0, hi = p.n_tokens;
  if (p.window) {
    lo = max(p.window[2 * b], 0);
    hi = min(p.window[2 * b + 1], p.n_tokens);
  }
  if (threadIdx.x == 0) sh.masked = sh.chosen = 0;
  __syncthreads();
  int masked = 0, may = 0;
  for (int i = threadIdx.x; i < p.n_tokens; i += kThreads) {
    const bool is = ids[i] == p.mask_id, in = is && i >= lo && i < hi;
    masked += is;
    may += in;
    keys[i] = in ? score_key(p.score[(row + i) * p.score_stride], p.lowest) : 0u;
  }
  masked = __reduce_add_sync(0xffffffffu, masked);
  may = __reduce_add_sync(0xffffffffu, may);
  if (lane == 0) {
    atomicAdd(&sh.masked, masked);
    atomicAdd(&sh.chosen, may);
  }
  __syncthreads();
  const int candidates = sh.chosen, take = min(want, candidates);
  if (threadIdx.x == 0 && p.n_left) p.n_left[b] = sh.masked - take;

  // taken: the keys from `from` on, and of those equal to `bar` the first `ties`
  uint32_t from = 1, bar = 0;
  int ties = 0;
  if (take == 0) {
    from = 0xFFFFFFFFu;  // above +inf's
  } else if (take < candidates) {
    int left = take;  // of the positions whose upper digits are those of bar
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < p.n_tokens; i += kThreads) {
        const uint32_t k = keys[i];
        if (k != 0 && (shift == 24 || (k >> (shift + 8)) == (bar >> (shift + 8)))) atomicAdd(&sh.hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (warp == 0) {  // digits 255 - 8 lane .. 248 - 8 lane, from the top
        int n[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += n[j] = sh.hist[255 - 8 * lane - j];
        int before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += up;
        }
        before -= sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (before < left && before + n[j] >= left) {
            sh.digit = 255 - 8 * lane - j;
            sh.above = before;
            sh.same = n[j];
          }
          before += n[j];
        }
      }
      __syncthreads();
      bar |= static_cast<uint32_t>(sh.digit) << shift;
      left -= sh.above;
      from = max(bar, 1u);
      if (sh.same == left) {  // all with these digits: everything from bar on
        left = 0;
        break;
      }
    }
    if (left > 0) {
      ties = left;
      from = bar + 1;
    }
  }
  int seen = 0;
  for (int i0 = 0; i0 < p.n_tokens; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const uint32_t k = i < p.n_tokens ? keys[i] : 0u;
    bool chosen = k >= from;
    if (ties > 0) {
      const bool tie = k == bar;
      const uint32_t ballot = __ballot_sync(0xffffffffu, tie);
      if (lane == 0) sh.warp_count[warp] = __popc(ballot);
      __syncthreads();
      int before = seen + __popc(ballot & ((1u << lane) - 1u)), all = 0;
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += sh.warp_count[w];
        all += sh.warp_count[w];
      }
      chosen |= tie && before < ties;
      seen += all;
      __syncthreads();
    }
    if (i < p.n_tokens) out[i] = chosen ? p.cand[(row + i) * p.cand_stride] : ids[i];
  }
}

}  // namespace

cudaError_t reveal_launch(const RevealParams& p, cudaStream_t s) {
  const size_t smem = sizeof(uint32_t) * p.n_tokens;
  if (smem > 40 * 1024) {
    const cudaError_t e =
        cudaFuncSetAttribute(reveal_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(uint32_t) * kRevealMaxTokens);
    if (e != cudaSuccess) return e;
  }
  reveal_kernel<<<p.batch, kThreads, smem, s>>>(p);
  return cudaGetLastError();
}

}  // namespace sgd
