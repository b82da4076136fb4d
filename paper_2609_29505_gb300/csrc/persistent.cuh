// Kernels over rows of logits whose clusters stay for the whole call: which rows a cluster takes, how many
// clusters there are, waits on what other CTAs send.
#pragma once

#include "vocab_rows.cuh"

namespace sgd {
namespace rows {

// mbar_wait_warp on a barrier that other CTAs of the cluster arrive at.
__device__ __forceinline__ bool wait_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* status, int code) {
  uint64_t t0 = 0;
  for (uint32_t i = 1;; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    if (__all_sync(0xffffffffu, ok)) return true;
    if (i % kPollsPerTimer == 0) {
      int stop = *abort_flag;
      if (!stop && wait_expired(t0)) {
        *abort_flag = stop = 1;
        if (status) atomicCAS(status, 0, code);
      }
      if (__any_sync(0xffffffffu, stop)) return false;
    }
  }
}

// The rows of a cluster, of two kinds: those for which first(r) holds, and the others.  Each kind is dealt
// out to the clusters by itself, one after another, so that every cluster gets as many of it, wherever
// the rows of a kind lie.  The lists are made once, in shared memory, by all threads of the CTA; where a
// cluster would have over kRowList rows (and chance evens them out), rows are dealt out as they come
// and looked at one by one (list() is false).
constexpr int kRowList = 448;

struct RowLists {
  int of_first[kRowList + 1], of_rest[kRowList + 1];
  int n_first, n_rest;
  int warp_count[32];
};

template <int kN, typename F>
__device__ __forceinline__ bool make_row_lists(RowLists& l, int rows, int cluster, int clusters, const F& first) {
  constexpr int kLook = 4, kW = kN / 32;
  static_assert(kN % 32 == 0 && kW <= 32, "whole warps");
  if ((rows + clusters - 1) / clusters > kRowList) return false;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int before = 0;  // rows of the first kind ahead of those looked at
  for (int base = 0; base < rows; base += kLook * kN) {
    bool is[kLook];
#pragma unroll
    for (int u = 0; u < kLook; ++u) {  // thread t: rows base + kLook t + u
      const int r = base + kLook * static_cast<int>(threadIdx.x) + u;
      is[u] = r < rows && first(r);
    }
    int mine = 0;
#pragma unroll
    for (int u = 0; u < kLook; ++u) mine += is[u];
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    if (lane == 31) l.warp_count[warp] = upto;
    __syncthreads();
    int all = lane < kW ? l.warp_count[lane] : 0;
    const int ahead = __reduce_add_sync(0xffffffffu, lane < warp ? all : 0);
    all = __reduce_add_sync(0xffffffffu, all);
    int rank = before + ahead + upto - mine;
#pragma unroll
    for (int u = 0; u < kLook; ++u) {
      const int r = base + kLook * static_cast<int>(threadIdx.x) + u;
      if (r < rows) {
        const int n = is[u] ? rank : r - rank, turn = n / clusters;
        if (n - turn * clusters == cluster) (is[u] ? l.of_first : l.of_rest)[turn] = r;
      }
      rank += is[u];
    }
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    l.n_first = (before - cluster + clusters - 1) / clusters;
    l.n_rest = (rows - before - cluster + clusters - 1) / clusters;
  }
  return true;  // (complete after the CTA's next barrier)
}

struct Clusters {
  int size = 0, count = 0;
};

// Clusters of `c` CTAs that run at once: asked for once per kernel, device and size.  Sets the kernel up
// for the shared memory it takes.
template <auto kKernel>
cudaError_t resident_clusters(int c, int threads, size_t smem, int* n) {
  static std::atomic<int> known[64][5];  // (0: not asked yet; else their number + 1)
  int dev = 0, k = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  while ((1 << k) < c) ++k;
  if (dev < 64 && known[dev][k].load() > 0) {
    *n = known[dev][k].load() - 1;
    return cudaSuccess;
  }
  e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(num_sms() / c * c));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = c;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(n, kKernel, &cfg);
  if (e != cudaSuccess) return e;
  if (dev < 64) known[dev][k].store(*n + 1);
  return cudaSuccess;
}

// The cluster size in [least, most] that leaves the SMs idle least over these rows: rounds, each a share of a
// row long; a larger cluster has to save 5%, as it exchanges more (2048 rows of 32000 bf16 with gradients, 13.5
// rounds of pairs: 60 us, 14 of single CTAs: 47 us).
template <auto kKernel>
cudaError_t choose_clusters(int rows, int least, int most, int threads, size_t smem, Clusters* out) {
  double cost = 0;
  for (int c = least; c <= most; c *= 2) {
    int n = 0;
    const cudaError_t e = resident_clusters<kKernel>(c, threads, smem, &n);
    if (e != cudaSuccess) return e;
    if (n < 1) continue;
    const double t = static_cast<double>((rows + n - 1) / n) / c;
    if (!out->size || t < 0.95 * cost) {
      cost = t;
      *out = Clusters{c, n < rows ? n : rows};
    }
  }
  return out->size ? cudaSuccess : cudaErrorInvalidConfiguration;
}

template <auto kKernel, typename... Args>
cudaError_t launch_clusters(const Clusters& l, int threads, size_t smem, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(l.count) * l.size);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = l.size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kKernel, args...);
}

}  // namespace rows
}  // namespace sgd
