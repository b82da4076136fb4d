// Rows of an embedding table, scaled, and the table's gradient.
//
//   out[r] = scale table[ids[r]];   dtable[t] = scale sum over {r : ids[r] = t} of grad[r], in the order of r.
//
// The gradient goes by the rows sorted by token: every sum has one order, no atomics are added to, and a token with
// half of the rows (the mask of a masked-token model) is split over as many CTAs as the others.
//   sort     (token, row) ascending.  Up to kRankRows rows each row counts the rows before it, N^2 comparisons over the
//            whole GPU in one launch; above, a radix sort (8 bits at a time: histogram, then a stable scatter).
//   sums     CTA (chunk of sorted rows, columns): a run of equal tokens that lies inside the chunk is written
//            to the table; a run that passes a chunk's border leaves a partial sum per chunk in the workspace.  Beside them,
//            unless they are kept, CTAs that clear the rows of the tokens that do not occur: a range of the table each.
//   join     adds the partial sums of such a run in the order of the chunks.
//
// Measured (GB300; a copy moves 6.7 TB/s): 4096 rows, half of them of one token, for a table of 126464 x 4096 bf16: 187 us, 167 of them sums and
// cleared rows (1.07 GB, 6.2 TB/s; a kernel of its own that cleared the table by 16-byte stores took 266 us).  65537 x 1024 for
// 32003 tokens: 83 us, 54 of them the sums (a thread's 16 rows at once; 8: 84 us).  The launches of a call overlap their starts and
// ends (programmatic dependent launch): 88 us without.
#include <atomic>

#include "common.cuh"
#include "kernels.h"

namespace sgd {
namespace {

// ----- elements of the three types -----

template <typename T>
struct Vec {  // 16 bytes
  static constexpr int kN = 16 / static_cast<int>(sizeof(T));
};
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(f16 x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(bf16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ f16 from_f32<f16>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float x) { return __float2bfloat16_rn(x); }

// N values at p, all of them where VEC (then p is aligned to 16 bytes, or to N elements where those are fewer bytes),
// else the first n.
template <bool VEC, int N, typename T>
__device__ __forceinline__ void load(const T* p, int n, float* f) {
  if constexpr (VEC) {
    constexpr int kBytes = N * static_cast<int>(sizeof(T));
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4 u = reinterpret_cast<const uint4*>(p)[i];
        const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
        for (int j = 0; j < Vec<T>::kN; ++j) f[i * Vec<T>::kN + j] = to_f32(e[j]);
      }
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] = to_f32(e[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = j < n ? to_f32(p[j]) : 0.f;
  }
}
template <bool VEC, int N, typename T>
__device__ __forceinline__ void store(T* p, int n, const float* f) {
  if constexpr (VEC) {
    constexpr int kBytes = N * static_cast<int>(sizeof(T));
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        uint4 u;
        T* e = reinterpret_cast<T*>(&u);
#pragma unroll
        for (int j = 0; j < Vec<T>::kN; ++j) e[j] = from_f32<T>(f[i * Vec<T>::kN + j]);
        reinterpret_cast<uint4*>(p)[i] = u;
      }
    } else {
      uint2 u;
      T* e = reinterpret_cast<T*>(&u);
#pragma unroll
      for (int j = 0; j < N; ++j) e[j] = from_f32<T>(f[j]);
      *reinterpret_cast<uint2*>(p) = u;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) p[j] = from_f32<T>(f[j]);
  }
}

template <typename T>
bool vectors(const void* p, int64_t ld, int per, int d) {  // rows of whole vectors, each aligned
  const int64_t bytes = static_cast<int64_t>(sizeof(T)) * per < 16 ? sizeof(T) * per : 16;
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * static_cast<int64_t>(sizeof(T)) % bytes == 0 && d % per == 0;
}

// ----- lookup -----

constexpr int kCols = 8;        // columns of a thread at a time
constexpr int kPiece = 1024;    // columns of a warp's piece of a row
constexpr int kLookWarps = 8;

// Pieces of rows, a warp each, one after another: the next one's values are on their way while a piece is scaled into shared memory, from
// where a bulk copy takes it to `out`.  (Plain stores of 16 bytes a thread wrote 3.9 TB/s: 4096 x 4096 bf16 to fp32 17.2 us.)
template <typename TI, typename TO>
__global__ void __launch_bounds__(32 * kLookWarps, 3) embedding_pieces_kernel(const EmbeddingParams p) {
  constexpr int kPer = kPiece / (32 * kCols), kRaw = kCols * static_cast<int>(sizeof(TI)) / 16;  // runs of 8 columns of a lane, their vectors
  extern __shared__ __align__(128) uint4 pieces[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  TO* buf = reinterpret_cast<TO*>(pieces) + warp * 2 * kPiece;
  const int across = (p.d + kPiece - 1) / kPiece;
  const int64_t all = static_cast<int64_t>(p.rows) * across, step = static_cast<int64_t>(gridDim.x) * kLookWarps;
  const TI* table = static_cast<const TI*>(p.table);
  TO* out = static_cast<TO*>(p.out);
  uint4 next[kPer][kRaw];
  bool next_here = false;
  auto fetch = [&](int64_t q) {
    const int64_t r = q / across;
    const int c0 = static_cast<int>(q - r * across) * kPiece, id = p.ids[r];
    next_here = id >= 0 && id < p.vocab;
    if (!next_here) return;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int c = c0 + (k * 32 + lane) * kCols;
      if (c < p.d)
#pragma unroll
        for (int i = 0; i < kRaw; ++i) next[k][i] = reinterpret_cast<const uint4*>(table + static_cast<int64_t>(id) * p.ld + c)[i];
    }
  };
  int64_t q = static_cast<int64_t>(blockIdx.x) * kLookWarps + warp;
  if (q < all) fetch(q);
  for (int flip = 0; q < all; q += step, flip ^= 1) {
    uint4 now[kPer][kRaw];
    const bool here = next_here;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
#pragma unroll
      for (int i = 0; i < kRaw; ++i) now[k][i] = next[k][i];
    if (q + step < all) fetch(q + step);
    const int64_t r = q / across;
    const int c0 = static_cast<int>(q - r * across) * kPiece, n = min(kPiece, p.d - c0);
    TO* to = buf + flip * kPiece;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");  // the piece before the last has left this place
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int c = (k * 32 + lane) * kCols;
      if (c >= n) continue;
      float f[kCols];
      const TI* e = reinterpret_cast<const TI*>(now[k]);
#pragma unroll
      for (int j = 0; j < kCols; ++j) f[j] = here ? to_f32(e[j]) * p.scale : 0.f;
      store<true, kCols>(to + c, kCols, f);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      bulk_store(out + r * p.ld_out + c0, to, static_cast<uint32_t>(n) * sizeof(TO));
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// Rows of any alignment.
template <typename TI, typename TO>
__global__ void __launch_bounds__(256) embedding_kernel(const EmbeddingParams p) {
  const int64_t all = static_cast<int64_t>(p.rows) * p.d;
  const TI* table = static_cast<const TI*>(p.table);
  TO* out = static_cast<TO*>(p.out);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t r = i / p.d;
    const int c = static_cast<int>(i - r * p.d), id = p.ids[r];
    const float f = id >= 0 && id < p.vocab ? to_f32(table[static_cast<int64_t>(id) * p.ld + c]) * p.scale : 0.f;
    out[r * p.ld_out + c] = from_f32<TO>(f);
  }
}

template <typename TI, typename TO>
cudaError_t lookup(const EmbeddingParams& p, cudaStream_t s) {
  // whole vectors in both, of 8 columns
  if (vectors<TI>(p.table, p.ld, kCols, p.d) && vectors<TO>(p.out, p.ld_out, kCols, p.d)) {
    constexpr int kSmem = kLookWarps * 2 * kPiece * static_cast<int>(sizeof(TO));
    // once per kernel and device
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (kSmem > 48 * 1024 && (dev > 63 || !(ready.load() >> dev & 1))) {
      e = cudaFuncSetAttribute(embedding_pieces_kernel<TI, TO>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
      if (e != cudaSuccess) return e;
      if (dev <= 63) ready.fetch_or(1ull << dev);
    }
    const int64_t ctas = (static_cast<int64_t>(p.rows) * ((p.d + kPiece - 1) / kPiece) + kLookWarps - 1) / kLookWarps, most = 3 * num_sms();
    embedding_pieces_kernel<TI, TO><<<static_cast<unsigned>(ctas < most ? ctas : most), 32 * kLookWarps, kSmem, s>>>(p);
    return cudaGetLastError();
  }
  const int64_t blocks = (static_cast<int64_t>(p.rows) * p.d + 255) / 256, most = 1 << 16;
  embedding_kernel<TI, TO><<<static_cast<unsigned>(blocks < most ? blocks : most), 256, 0, s>>>(p);
  return cudaGetLastError();
}
template <typename TI>
cudaError_t lookup_to(const EmbeddingParams& p, cudaStream_t s) {
  if (p.out_dtype == SGD_F16) return lookup<TI, f16>(p, s);
  if (p.out_dtype == SGD_BF16) return lookup<TI, bf16>(p, s);
  return lookup<TI, float>(p, s);
}

// ----- gradient: the rows sorted by token -----

// Rows that are sorted by counting.  The gradient of rows of 64 columns by counting and by the radix sort, us: 1024 rows 9.8 / 22.5, 4096
// 16.0 / 26.4, 8192 34.8 / 31.7, 12000 52 / 34.
constexpr int kRankRows = 6144;
constexpr int kRankCta = 16;     // of a CTA, 16 threads each
constexpr int kTile = 1024;      // rows of a CTA of the radix sort at a time: 8 warps, 128 each
constexpr int kMaxTiles = 256;   // CTAs: more rows are more at a time
constexpr int kSteps = kTile / 256;
constexpr int kBits = 8, kBins = 1 << kBits;

// A row without a token goes behind all others, as one of the token `vocab`.
__device__ __forceinline__ uint32_t token_of(const int32_t* ids, int r, int vocab) {
  const uint32_t t = static_cast<uint32_t>(ids[r]);
  return min(t, static_cast<uint32_t>(vocab));
}

// rank of row r = number of rows before it in (token, row)
__global__ void __launch_bounds__(256) rank_kernel(const int32_t* ids, int rows, int vocab, uint32_t* tokens, int32_t* order) {
  extern __shared__ uint32_t all[];  // [rows, a multiple of 4], the rest above every token
  pdl_wait_and_trigger();
  const int padded = (rows + 3) & ~3;
  for (int i0 = threadIdx.x; i0 < padded; i0 += 256 * 16) {
    uint32_t t[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) t[u] = i0 + u * 256 < rows ? token_of(ids, i0 + u * 256, vocab) : 0xFFFFFFFFu;
#pragma unroll
    for (int u = 0; u < 16; ++u)
      if (i0 + u * 256 < padded) all[i0 + u * 256] = t[u];
  }
  __syncthreads();
  const int r = blockIdx.x * kRankCta + (threadIdx.x >> 4), part = threadIdx.x & 15;
  int before = 0;
  uint32_t mine = 0;
  if (r < rows) {
    mine = all[r];
    #pragma unroll 4
    for (int i = part * 4; i < padded; i += 64) {
      const uint4 t = *reinterpret_cast<const uint4*>(all + i);
      // an equal token counts where its row is smaller
      before += t.x < mine + (i < r);
      before += t.y < mine + (i + 1 < r);
      before += t.z < mine + (i + 2 < r);
      before += t.w < mine + (i + 3 < r);
    }
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
  if (r < rows && part == 0) {
    tokens[before] = mine;
    order[before] = r;
  }
}

// Radix sort, one digit: counts per (digit, tile), their exclusive scan, and the stable scatter.  FIRST: the keys are
// the rows' tokens, and a row is its own index.
template <bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const int32_t* ids, const uint32_t* keys, int i, int vocab) {
  return FIRST ? token_of(ids, i, vocab) : keys[i];
}
// (A CTA takes `times` tiles, one after another.)
template <bool FIRST>
__global__ void __launch_bounds__(256) radix_count_kernel(const int32_t* ids, const uint32_t* keys, int rows, int times, int vocab, int shift,
                                                          uint32_t* counts) {
  __shared__ uint32_t hist[kBins];
  pdl_wait_and_trigger();
  hist[threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * times * kTile, end = min(first + static_cast<int64_t>(times) * kTile, static_cast<int64_t>(rows));
  for (int64_t i = first + threadIdx.x; i < end; i += 256)
    atomicAdd(&hist[(sort_key<FIRST>(ids, keys, static_cast<int>(i), vocab) >> shift) & (kBins - 1)], 1u);
  __syncthreads();
  counts[blockIdx.x * kBins + threadIdx.x] = hist[threadIdx.x];
}
template <bool FIRST>
__global__ void __launch_bounds__(256) radix_scatter_kernel(const int32_t* ids, const uint32_t* keys, const int32_t* rows_in, int rows, int times,
                                                            int vocab, int shift, const uint32_t* counts, uint32_t* keys_out,
                                                            int32_t* rows_out) {
  __shared__ uint32_t seen[8][kBins];  // of a warp: rows with this digit so far; then where its first one goes
  __shared__ uint32_t warp_sum[8];
  pdl_wait_and_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // where this CTA's rows of digit threadIdx.x go: behind all smaller digits, and the CTAs before it
  uint32_t before = 0, all = 0;
  for (int i0 = 0; i0 < static_cast<int>(gridDim.x); i0 += 32) {
    uint32_t n[32];
#pragma unroll
    for (int u = 0; u < 32; ++u) n[u] = i0 + u < static_cast<int>(gridDim.x) ? counts[(i0 + u) * kBins + threadIdx.x] : 0u;
#pragma unroll
    for (int u = 0; u < 32; ++u) {
      if (i0 + u < static_cast<int>(blockIdx.x)) before += n[u];
      all += n[u];
    }
  }
  uint32_t up = all;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, up, o);
    if (lane >= o) up += x;
  }
  if (lane == 31) warp_sum[warp] = up;
  __syncthreads();
  uint32_t run = up - all + before;
  for (int w = 0; w < warp; ++w) run += warp_sum[w];
  for (int k = 0; k < times; ++k) {
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * times + k) * kTile + warp * (kTile / 8);
    __syncthreads();
    for (int i = threadIdx.x; i < 8 * kBins; i += 256) seen[i / kBins][i % kBins] = 0;
    __syncthreads();
    uint32_t key[kSteps], rank[kSteps];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int64_t i = first + j * 32 + lane;
      key[j] = i < rows ? sort_key<FIRST>(ids, keys, static_cast<int>(i), vocab) : 0u;
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const bool in = first + j * 32 + lane < rows;
      const uint32_t digit = in ? (key[j] >> shift) & (kBins - 1) : kBins;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      const uint32_t below = __popc(same & ((1u << lane) - 1u));
      rank[j] = in ? seen[warp][digit] + below : 0u;
      __syncwarp();
      if (in && below == 0) seen[warp][digit] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const uint32_t n = seen[w][threadIdx.x];
      seen[w][threadIdx.x] = run;
      run += n;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int64_t i = first + j * 32 + lane;
      if (i >= rows) continue;
      const uint32_t at = seen[warp][(key[j] >> shift) & (kBins - 1)] + rank[j];
      keys_out[at] = key[j];
      rows_out[at] = FIRST ? static_cast<int32_t>(i) : rows_in[i];
    }
  }
}

// ----- gradient: sums of runs -----

constexpr int kSumThreads = 128;
constexpr int kMaxChunk = 32;   // rows of a chunk (65537 x 1024: 91 us, 16 rows 103; 4096 x 4096 in chunks of 16 42 us, of 8 30)
constexpr int kJoinCols = 128;  // of a CTA that joins: 32 lanes, 4 columns each

struct Plan {
  int rows, d, chunk, chunks, tiles, times, pd;  // pd: columns of a row of partial sums
  int64_t keys, order, keys2, order2, counts, partial, bytes;  // offsets in the workspace
};
Plan make_plan(int rows, int d) {
  Plan q{};
  q.rows = rows;
  q.d = d;
  // Rows of a chunk: few enough that every SM has some CTAs, and as many as make partial sums a small share of the traffic.
  const int64_t across = (d + 1023) / 1024;
  q.chunk = 8;
  while (q.chunk < kMaxChunk && rows / q.chunk * across > 2048) q.chunk *= 2;
  q.chunks = (rows + q.chunk - 1) / q.chunk;
  q.times = rows / (kTile * kMaxTiles) + 1;
  q.tiles = static_cast<int>((static_cast<int64_t>(rows) + static_cast<int64_t>(kTile) * q.times - 1) / (static_cast<int64_t>(kTile) * q.times));
  q.pd = (d + 7) & ~7;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += (bytes + 255) & ~255ll;
    return here;
  };
  q.keys = take(4ll * rows);
  q.order = take(4ll * rows);
  if (rows > kRankRows) {
    q.keys2 = take(4ll * rows);
    q.order2 = take(4ll * rows);
    q.counts = take(4ll * kBins * q.tiles);
  }
  q.partial = take(8ll * q.chunks * q.pd);
  q.bytes = at;
  return q;
}

struct SumArgs {
  const void* grad;
  int64_t ld_grad;
  const uint32_t* tokens;
  const int32_t* order;
  int rows, vocab, d, chunk, chunks, pd, accumulate;
  float scale;
  int fill, fill_rows;  // CTAs (in x) that clear a range of so many tokens each
  float* partial;  // [chunks, 2, pd]: of the run that came from the chunk before, of the one that goes on to the next
  void* dtable;
  int64_t ld;
};

// scale sum (+ what is there) to the table
template <typename TO, bool VEC, int N>
__device__ __forceinline__ void put(const SumArgs& p, uint32_t token, int c, const float* sum) {
  TO* at = static_cast<TO*>(p.dtable) + static_cast<int64_t>(token) * p.ld + c;
  float f[N];
  if (p.accumulate) {
    if constexpr (VEC) {
      // (ordinary loads: the table is written by this kernel)
      TO v[N];
      constexpr int kBytes = N * static_cast<int>(sizeof(TO));
      if constexpr (kBytes >= 16) {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(v)[i] = reinterpret_cast<const uint4*>(at)[i];
      } else {
        *reinterpret_cast<uint2*>(v) = *reinterpret_cast<const uint2*>(at);
      }
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] = fmaf(p.scale, sum[j], to_f32(v[j]));
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] = c + j < p.d ? fmaf(p.scale, sum[j], to_f32(at[j])) : 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = p.scale * sum[j];
  }
  store<VEC, N>(at, p.d - c, f);
}

constexpr int kZeros = 16384;     // bytes of zeros in shared memory, which copies to the table start from
constexpr int kFillRows = 1024;   // tokens of a range, at most

// The first of the sorted rows [lo, hi) whose token is `token` or more, hi where there is none: a warp, 32 probes at a time.
__device__ __forceinline__ int first_row_of(const uint32_t* tokens, int lo, int hi, uint32_t token) {
  int before = lo - 1;  // lies before it
  const int lane = threadIdx.x & 31;
  while (hi - before > 1) {
    const int step = (hi - before + 31) / 32, at = before + (lane + 1) * step;
    const bool is = at < hi && tokens[at] < token;
    const int more = __popc(__ballot_sync(0xffffffffu, is));
    before += more * step;
    hi = min(hi, before + step);
  }
  return hi;
}

// Clears the rows of the tokens [first, first + n) that do not occur.
template <typename TO, bool VEC>
__device__ __forceinline__ void clear_rows(const SumArgs& p, int first, int n, uint4* zeros, uint32_t* here) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kFillRows / 32; i += kSumThreads) here[i] = 0;
  if (VEC)
    for (int i = threadIdx.x; i < kZeros / 16; i += kSumThreads) zeros[i] = make_uint4(0, 0, 0, 0);
  // the sorted rows of the range, then each token's first one in them
  const uint32_t from = static_cast<uint32_t>(first);
  const int lo = first_row_of(p.tokens, 0, p.rows, from), hi = first_row_of(p.tokens, lo, p.rows, from + n);
  if (VEC) fence_proxy_async_smem();
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kSumThreads) {
    int l = lo, h = hi;
    while (l < h) {
      const int at = l + (h - l) / 2;
      if (p.tokens[at] < from + i) l = at + 1;
      else h = at;
    }
    if (l < hi && p.tokens[l] == from + i) atomicOr(&here[i >> 5], 1u << (i & 31));
  }
  __syncthreads();
  TO* table = static_cast<TO*>(p.dtable);
  for (int i = warp; i < n; i += kSumThreads / 32) {
    if (here[i >> 5] >> (i & 31) & 1) continue;
    TO* at = table + static_cast<int64_t>(first + i) * p.ld;
    if constexpr (VEC) {
      const int64_t bytes = static_cast<int64_t>(p.d) * sizeof(TO);
      for (int64_t o = static_cast<int64_t>(lane) * kZeros; o < bytes; o += 32 * kZeros)
        bulk_store(reinterpret_cast<char*>(at) + o, zeros, static_cast<uint32_t>(min(bytes - o, static_cast<int64_t>(kZeros))));
    } else {
      for (int c = lane; c < p.d; c += 32) at[c] = from_f32<TO>(0.f);
    }
  }
  if (VEC) bulk_store_wait();  // the zeros stay until they are read
}

template <typename TG, typename TO, bool VEC>
__global__ void __launch_bounds__(kSumThreads) embedding_sums_kernel(const SumArgs p) {
  extern __shared__ __align__(16) uint4 zeros[];
  __shared__ uint32_t here[kFillRows / 32];
  pdl_wait_and_trigger();
  if (static_cast<int>(blockIdx.x) < p.fill) {
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * gridDim.y + blockIdx.y) * p.fill_rows;
    if (first < p.vocab)
      clear_rows<TO, VEC>(p, static_cast<int>(first), static_cast<int>(min(static_cast<int64_t>(p.fill_rows), p.vocab - first)), zeros, here);
    return;
  }
  const int chunk = blockIdx.x - p.fill;
  constexpr int N = VEC ? Vec<TG>::kN : 4, kAhead = VEC ? 16 : 8;  // (a row's 16 bytes as they are, or its numbers)
  __shared__ uint32_t tok[kMaxChunk + 2];
  __shared__ int32_t row[kMaxChunk];
  const int first = chunk * p.chunk, n = min(p.chunk, p.rows - first);
  // the tokens of the chunk and of its neighbours (none: one that no row has)
  for (int i = threadIdx.x; i < n + 2; i += kSumThreads) {
    const int at = first + i - 1;
    tok[i] = at >= 0 && at < p.rows ? p.tokens[at] : 0xFFFFFFFFu;
  }
  for (int i = threadIdx.x; i < n; i += kSumThreads) row[i] = p.order[first + i];
  __syncthreads();
  const int c = (blockIdx.y * kSumThreads + threadIdx.x) * N;
  if (c >= p.d) return;
  const TG* grad = static_cast<const TG*>(p.grad) + c;
  float sum[N];
#pragma unroll
  for (int j = 0; j < N; ++j) sum[j] = 0.f;
  bool from_before = tok[1] == tok[0];
  for (int i0 = 0; i0 < n; i0 += kAhead) {
    uint4 raw[VEC ? kAhead : 1];
    float v[VEC ? 1 : kAhead][N];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i0 + u >= n || tok[i0 + u + 1] >= static_cast<uint32_t>(p.vocab)) continue;
      const TG* at = grad + static_cast<int64_t>(row[i0 + u]) * p.ld_grad;
      if constexpr (VEC) raw[u] = *reinterpret_cast<const uint4*>(at);
      else load<false, N>(at, p.d - c, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u;
      if (i >= n) break;
      const uint32_t t = tok[i + 1];
      if (t >= static_cast<uint32_t>(p.vocab)) return;  // the rest has no token
      if constexpr (VEC) {
        const TG* e = reinterpret_cast<const TG*>(&raw[u]);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += to_f32(e[j]);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += v[u][j];
      }
      const bool ends = tok[i + 2] != t, last = i == n - 1;
      if (!ends && !last) continue;
      if (ends && !from_before) {
        put<TO, VEC, N>(p, t, c, sum);
      } else {
        float* at = p.partial + (2 * static_cast<int64_t>(chunk) + (from_before ? 0 : 1)) * p.pd + c;
        if constexpr (VEC) {
#pragma unroll
          for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(at + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j) at[j] = sum[j];  // (a row of partial sums is a multiple of 8 long)
        }
      }
      from_before = false;
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] = 0.f;
    }
  }
}

// Runs that pass a chunk's border: CTA (columns, share of the chunks where such a run begins).
template <typename TO, bool VEC>
__global__ void __launch_bounds__(256) embedding_join_kernel(const SumArgs p) {
  __shared__ int begins[256];
  __shared__ int n_begins;
  __shared__ float4 sums[8][32];
  pdl_wait_and_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c = blockIdx.x * kJoinCols + lane * 4;
  const uint32_t vocab = static_cast<uint32_t>(p.vocab);
  for (int base = blockIdx.y; base < p.chunks; base += 256 * gridDim.y) {
    if (threadIdx.x == 0) n_begins = 0;
    __syncthreads();
    // chunks base, base + gridDim.y, ...: does a run begin here and go on?
    const int64_t mine = base + static_cast<int64_t>(threadIdx.x) * gridDim.y;
    if (mine + 1 < p.chunks) {  // the last chunk's runs end with it
      const int at = static_cast<int>(mine) * p.chunk, end = at + p.chunk;
      const uint32_t t = p.tokens[end - 1], after = p.tokens[end], before = at > 0 ? p.tokens[at - 1] : 0xFFFFFFFFu;
      if (t < vocab && after == t && before != t) begins[atomicAdd(&n_begins, 1)] = static_cast<int>(mine);  // (a run that came from before began there)
    }
    __syncthreads();
    const int n = n_begins;
    for (int k = 0; k < n; ++k) {
      const int c0 = begins[k];
      const uint32_t t = p.tokens[(c0 + 1) * p.chunk - 1];
      // the last chunk of the run: 32 probes at a time between lo (holds the token first) and hi (does not)
      int lo = c0 + 1, hi = p.chunks;
      {  // most runs end in the next few chunks
        const int at = lo + lane + 1;
        const int more = __popc(__ballot_sync(0xffffffffu, at < hi && p.tokens[static_cast<int64_t>(at) * p.chunk] == t));
        lo += more;
        if (more < 32) hi = lo + 1;
      }
      while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int at = lo + (lane + 1) * step;
        const bool in = at < hi && p.tokens[static_cast<int64_t>(at) * p.chunk] == t;
        const int more = __popc(__ballot_sync(0xffffffffu, in));  // (tokens ascend: the first ones)
        const int new_lo = lo + more * step;
        hi = min(hi, new_lo + step);
        lo = new_lo;
      }
      const int parts = lo - c0 + 1;  // tail of c0, heads of c0 + 1 .. lo
      const int per = (parts + 7) / 8, a = warp * per, b = min(a + per, parts);
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c < p.pd) {
#pragma unroll 8
        for (int i = a; i < b; ++i) {
          const int64_t slot = 2 * static_cast<int64_t>(c0 + i) + (i == 0 ? 1 : 0);
          const float4 x = *reinterpret_cast<const float4*>(p.partial + slot * p.pd + c);
          s.x += x.x;
          s.y += x.y;
          s.z += x.z;
          s.w += x.w;
        }
      }
      sums[warp][lane] = s;
      __syncthreads();
      if (warp == 0 && c < p.d) {
#pragma unroll
        for (int w = 1; w < 8; ++w) {
          const float4 x = sums[w][lane];
          s.x += x.x;
          s.y += x.y;
          s.z += x.z;
          s.w += x.w;
        }
        const float f[4] = {s.x, s.y, s.z, s.w};
        put<TO, VEC, 4>(p, t, c, f);
      }
      __syncthreads();
    }
    __syncthreads();
  }
}

template <typename TG, typename TO>
cudaError_t sums(SumArgs a, cudaStream_t s) {
  const bool vec = vectors<TG>(a.grad, a.ld_grad, Vec<TG>::kN, a.d) && vectors<TO>(a.dtable, a.ld, Vec<TG>::kN, a.d) && vectors<TO>(a.dtable, a.ld, Vec<TO>::kN, a.d);
  const int n = vec ? Vec<TG>::kN : 4;
  const int across = (a.d + kSumThreads * n - 1) / (kSumThreads * n);
  a.fill = (a.fill + across - 1) / across;
  const dim3 grid(a.fill + a.chunks, across);
  const size_t smem = vec && a.fill ? kZeros : 0;
  cudaError_t e;
  if (a.rows == 0) {  // (the call's only launch)
    if (vec) embedding_sums_kernel<TG, TO, true><<<grid, kSumThreads, smem, s>>>(a);
    else embedding_sums_kernel<TG, TO, false><<<grid, kSumThreads, smem, s>>>(a);
    e = cudaGetLastError();
  } else {
    e = vec ? launch_behind(embedding_sums_kernel<TG, TO, true>, grid, dim3(kSumThreads), smem, s, a)
            : launch_behind(embedding_sums_kernel<TG, TO, false>, grid, dim3(kSumThreads), smem, s, a);
  }
  if (e != cudaSuccess || a.chunks < 2) return e;
  const int tiles = (a.d + kJoinCols - 1) / kJoinCols, high = (8 * num_sms() + tiles - 1) / tiles;
  const dim3 join(tiles, a.chunks < high ? a.chunks : high);
  return vectors<TO>(a.dtable, a.ld, 4, a.d) ? launch_behind(embedding_join_kernel<TO, true>, join, dim3(256), 0, s, a)
                                             : launch_behind(embedding_join_kernel<TO, false>, join, dim3(256), 0, s, a);
}
template <typename TG>
cudaError_t sums_to(const SumArgs& a, int dtype, cudaStream_t s) {
  if (dtype == SGD_F16) return sums<TG, f16>(a, s);
  if (dtype == SGD_BF16) return sums<TG, bf16>(a, s);
  return sums<TG, float>(a, s);
}

cudaError_t sort_rows(const EmbeddingGradParams& p, const Plan& q, char* ws, const uint32_t** tokens, const int32_t** order,
                      cudaStream_t s) {
  uint32_t* k0 = reinterpret_cast<uint32_t*>(ws + q.keys);
  int32_t* r0 = reinterpret_cast<int32_t*>(ws + q.order);
  if (p.rows <= kRankRows) {
    rank_kernel<<<(p.rows + kRankCta - 1) / kRankCta, 256, 4 * ((p.rows + 3) & ~3), s>>>(p.ids, p.rows, p.vocab, k0, r0);
    *tokens = k0;
    *order = r0;
    return cudaGetLastError();
  }
  uint32_t* k1 = reinterpret_cast<uint32_t*>(ws + q.keys2);
  int32_t* r1 = reinterpret_cast<int32_t*>(ws + q.order2);
  uint32_t* counts = reinterpret_cast<uint32_t*>(ws + q.counts);
  for (int shift = 0; shift < 32 && (shift == 0 || p.vocab >> shift); shift += kBits) {
    const dim3 grid(q.tiles), block(256);
    const uint32_t* from = k0;
    const int32_t* rows_from = r0;
    const uint32_t* counted = counts;
    cudaError_t e;
    if (shift == 0) {
      radix_count_kernel<true><<<grid, block, 0, s>>>(p.ids, from, p.rows, q.times, p.vocab, shift, counts);
      e = cudaGetLastError();
      if (e == cudaSuccess)
        e = launch_behind(radix_scatter_kernel<true>, grid, block, 0, s, p.ids, from, rows_from, p.rows, q.times, p.vocab, shift, counted, k1, r1);
    } else {
      e = launch_behind(radix_count_kernel<false>, grid, block, 0, s, p.ids, from, p.rows, q.times, p.vocab, shift, counts);
      if (e == cudaSuccess)
        e = launch_behind(radix_scatter_kernel<false>, grid, block, 0, s, p.ids, from, rows_from, p.rows, q.times, p.vocab, shift, counted, k1, r1);
    }
    if (e != cudaSuccess) return e;
    uint32_t* k = k0;
    k0 = k1;
    k1 = k;
    int32_t* r = r0;
    r0 = r1;
    r1 = r;
  }
  *tokens = k0;
  *order = r0;
  return cudaSuccess;
}

}  // namespace

int64_t embedding_grad_bytes(int rows, int d) { return make_plan(rows, d).bytes; }

cudaError_t embedding_launch(const EmbeddingParams& p, cudaStream_t s) {
  if (p.dtype == SGD_F16) return lookup_to<f16>(p, s);
  if (p.dtype == SGD_BF16) return lookup_to<bf16>(p, s);
  return lookup_to<float>(p, s);
}

cudaError_t embedding_grad_launch(const EmbeddingGradParams& p, cudaStream_t s) {
  if (p.rows == 0 && p.accumulate) return cudaSuccess;
  const Plan q = make_plan(p.rows, p.d);
  char* ws = static_cast<char*>(p.workspace);
  const uint32_t* tokens = nullptr;
  const int32_t* order = nullptr;
  if (p.rows > 0) {
    const cudaError_t e = sort_rows(p, q, ws, &tokens, &order, s);
    if (e != cudaSuccess) return e;
  }
  // ranges of the table: several per SM
  const int64_t vocab = p.vocab, share = (vocab + 8 * num_sms() - 1) / (8 * num_sms());
  const int fill_rows = share < 4 ? 4 : (share > kFillRows ? kFillRows : static_cast<int>(share));
  const int fill = p.accumulate ? 0 : static_cast<int>((vocab + fill_rows - 1) / fill_rows);
  const SumArgs a{p.grad, p.ld_grad, tokens, order, p.rows, p.vocab, p.d, q.chunk, q.chunks, q.pd, p.accumulate, p.scale,
                  fill, fill_rows, reinterpret_cast<float*>(ws + q.partial), p.dtable, p.ld};
  if (p.grad_dtype == SGD_F16) return sums_to<f16>(a, p.dtable_dtype, s);
  if (p.grad_dtype == SGD_BF16) return sums_to<bf16>(a, p.dtable_dtype, s);
  return sums_to<float>(a, p.dtable_dtype, s);
}

}  // namespace sgd
