// Scoring of many long rows (logprobs.cu has the formulas): the rows stream through the SMs.
//
// One CTA per SM stays for the whole call.  A producer warp keeps a ring of 32 KB tiles filled by bulk
// copies, across the ends of rows; 16 warps take the tiles' statistics and wait for nothing but data; 6
// warps finish the rows, each a row of its own (sums, likeliest tokens, outputs: a chain of latency of
// several us, so that as many of them run at once).  Where there are too few rows for the SMs, the CTAs of
// a cluster share each row and the first of them merges their parts.
//
// The likeliest tokens without a second pass over the row: the k-th largest of the 512 streaming threads'
// maxima is a threshold that k elements or a few more reach; of the threads whose maximum reaches it, the
// maxima of four parts of what they saw tell which part to read again (k / 2048 of the row).  One batch of
// loads does: a load takes some 3 us here, behind the copies that keep the memory busy.  For the single
// likeliest token the tile of each thread's first maximum is enough.
//
// Measured (GB300, replayed from a graph over rotating inputs): 4096 x 126464 fp16, the 32 likeliest: 169 us =
// 6.1 TB/s (a copy moves 6.8), bound by HBM; 2048 of 4096 rows, the likeliest one and the entropy: 92 us = 5.7
// TB/s: a tile's 200 instructions a thread (conversion, fma, exponential, two sums, maximum, minimum) and its
// copy take about as long.  8 streaming warps instead of 16: 127 us; two teams of 4 finishing warps instead of
// single ones: 191 and 98 us (a team's barriers); 6 warps or 4: 174 and 193 us for the lists.
//
// Every wait is bounded.  After one has expired (recorded in the status word) each warp leaves its loop.
#include "logprobs.cuh"
#include "persistent.cuh"

namespace sgd {
namespace rows {
namespace {

constexpr int kStreamWarps = 16, kStreamThreads = 32 * kStreamWarps;
constexpr int kDeep = 4, kTile = kStreamThreads * kDeep;  // vectors of a tile: kDeep per thread
constexpr int kFinishWarps = 6;
constexpr int kAll = kStreamThreads + 32 * (kFinishWarps + 1);
constexpr int kTileBytes = kTile * 16;
constexpr int kStreamCluster = 4;
constexpr int kMaxima = kStreamThreads / 32;  // streaming threads' maxima per lane
constexpr int kParts = 4;       // of what a thread sees of a row: consecutive tiles
constexpr int kMaxGroups = 256;
constexpr int kStaged = 96;
constexpr int slots(int top) { return top == kTopMany ? 4 : 5; }

// A row on its way from the streaming warps to its finishing warp, and across the cluster.
struct Row {
  uint64_t part_full, part_free;  // its statistics in this CTA
  uint64_t row_full, row_free;    // its parts from all CTAs, in the first one
  int row;                        // -1: no more
  float result[2];
  float4 part[kStreamWarps];
  float4 slot[kStreamCluster];
  uint32_t max_key[kStreamThreads];
  uint16_t max_tile[kStreamThreads];  // of the first maximum; the threads that are looked at again
};

// What a finishing warp needs for lists of more than one.
struct Many {
  TopShared top;
  __align__(16) uint4 staged[kStaged];
  int staged_at[kStaged];
  uint16_t groups[kMaxGroups];                        // parts that are read again: thread and part
  uint16_t group_key[kParts * kStreamThreads];  // upper halves of the parts' maxima's keys
};

struct Shared {
  uint64_t full[5], empty[5];
  int slot_row[5];  // row of a tile; -1: no more
  int abort_flag;
  Row row[kFinishWarps];
  RowLists lists;
};

template <typename T>
__device__ __forceinline__ int tiles_of(const Slice<T>& sl) { return max(1, (sl.nv + kTile - 1) / kTile); }

template <int kSlots>
struct Ring {
  int slot = 0;
  uint32_t phase = 0;
  __device__ void next() {
    if (++slot == kSlots) {
      slot = 0;
      phase ^= 1;
    }
  }
};

template <typename T>
struct FromRow {
  Slice<T> sl;
  __device__ uint4 operator()(int i) const { return sl.fetch(i); }
};

// Tiles of a part.
__device__ __forceinline__ int tiles_of_part(int tiles) { return (tiles + kParts - 1) / kParts; }

// The slice's k likeliest elements are among the candidates left in many.top.
template <typename T>
__device__ __forceinline__ void candidates(const WarpTeam& team, const Slice<T>& sl, Row& x, int k, Many& many) {
  const int lane = team.tid;
  TopShared& top = many.top;
  uint32_t keys[kMaxima];
#pragma unroll
  for (int h = 0; h < kMaxima; ++h) keys[h] = x.max_key[lane + 32 * h];
  const Threshold th = threshold(team, keys, k, top);
  const uint32_t lo = th.from();
  int n = 0;
#pragma unroll
  for (int h = 0; h < kMaxima; ++h) {
    const uint32_t hit = __ballot_sync(0xffffffffu, keys[h] >= lo);
    if (keys[h] >= lo) x.max_tile[n + __popc(hit & ((1u << lane) - 1u))] = static_cast<uint16_t>(lane + 32 * h);
    n += __popc(hit);
  }
  __syncwarp();
  int groups = 0;
  // (a slice of few tiles has fewer parts: no one has written the others' maxima)
  const int tiles = tiles_of(sl), per_part = tiles_of_part(tiles), parts = (tiles + per_part - 1) / per_part;
  for (int j0 = 0; j0 < n * kParts; j0 += 32) {
    const int j = j0 + lane;
    const int g = j < n * kParts && j % kParts < parts ? j % kParts * kStreamThreads + x.max_tile[j / kParts] : -1;
    const bool is = g >= 0 && many.group_key[max(g, 0)] >= lo >> 16;
    const uint32_t hit = __ballot_sync(0xffffffffu, is);
    const int at = groups + __popc(hit & ((1u << lane) - 1u));
    if (is && at < kMaxGroups) many.groups[at] = static_cast<uint16_t>(g);
    groups += __popc(hit);
  }
  __syncwarp();
  bool crowded = false;  // more than there is room for: a row of many equal values, say
  if (groups <= kMaxGroups) {
    const float bar = key_value(lo);
    const uint4 none = no_elements<T>();
    // 8 lanes take 8 vectors of a part; 10 such loads of a lane are on their way at once
    constexpr int kAhead = 10;
    const int vectors = per_part * kDeep, per = (vectors + 7) >> 3;
    const float per_inv = 1.f / per;
    auto vector = [&](int c) {  // local vector of chunk c for this lane; -1: none, or not whole
      if (c >= groups * per) return -1;
      const int q = static_cast<int>((c + 0.5f) * per_inv);  // c / per: exact, c is far below 2^22
      const int w = (c - q * per) * 8 + (lane & 7), g = many.groups[q], thread = g % kStreamThreads;
      const int i = (g / kStreamThreads * vectors + w) * kStreamThreads + thread;
      return w < vectors && i < sl.nv && sl.whole(i) ? i : -1;
    };
#pragma unroll 1
    for (int first = 0; first < groups * per; first += 4 * kAhead) {  // (as often in every lane: the warp meets in it)
      const int c0 = first + (lane >> 3);
      uint4 v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = vector(c0 + 4 * u);
        v[u] = none;
        if (i >= 0) v[u] = *reinterpret_cast<const uint4*>(sl.row + sl.first_element(i));
      }
      // the few that hold something are put side by side, so that a lane has one of them to sort out
      int staged = 0;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const bool is = vec_max<1>(&v[u], static_cast<const T*>(nullptr)) >= bar;
        const uint32_t hit = __ballot_sync(0xffffffffu, is);
        if (hit == 0) continue;
        const int at = staged + __popc(hit & ((1u << lane) - 1u));
        const int i = is && at < kStaged ? vector(c0 + 4 * u) : -1;
        if (is && at < kStaged) {
          many.staged[at] = v[u];
          many.staged_at[at] = i >= 0 ? sl.first_element(i) : -Elem<T>::kPer;  // (no vector: the threshold is -inf)
        }
        staged += __popc(hit);
      }
      __syncwarp();
      if (staged > kStaged) {
        crowded = true;
        break;
      }
#pragma unroll 1
      for (int i = lane; i < staged; i += 32) append<T>(many.staged[i], many.staged_at[i], sl.vocab, lo, &top);
      __syncwarp();
    }
    if (lane < 2 && sl.nv > 0) {  // the slice's ragged ends
      const int i = lane ? sl.nv - 1 : 0;
      if (!sl.whole(i) && !(lane && i == 0)) append<T>(sl.gather(i), sl.first_element(i), sl.vocab, lo, &top);
    }
  }
  __syncwarp();
  const int found = top.n;
  __syncwarp();
  if (crowded || groups > kMaxGroups || found > kCap) candidates_of_many(team, sl, FromRow<T>{sl}, th.lo, th.top, k, top);
  else if (th.tied && found < k) collect_ties(team, sl, FromRow<T>{sl}, th.lo, k - found, top);
}

// The rows of one finishing warp, one after another.
template <typename T, int TOP, bool ENT>
__device__ __forceinline__ void finish_rows(const ScoreArgs& p, Row& x, Many& many, uint64_t* lists, volatile int* abort_flag,
                                            const int rank, const int n_ctas) {
  const T* logits = static_cast<const T*>(p.logits);
  const float c = p.scale * kLog2e;
  const int lane = lane_id();
  const WarpTeam team{lane};
  for (uint32_t phase = 0;; phase ^= 1) {
    if (!mbar_wait_warp(smem_u32(&x.part_full), phase, abort_flag, p.status, 66)) break;
    const int r = x.row;
    if (r < 0) break;
    const T* row = logits + r * p.ld;
    const Slice<T> sl(row, p.vocab, rank, n_ctas);
    Given<T> given;
    if (rank == 0) given.fetch_token(p, r, lane);
    float4 v = make_float4(-kInf, 0.f, 0.f, 0.f);
    if (lane < kStreamWarps) v = x.part[lane];
    const float m = key_value(__reduce_max_sync(0xffffffffu, order_key(v.x)));
    int best = 0x7FFFFFFF;
    if (TOP == kTopOne) {
      const uint32_t key = order_key(m);
      int mine[kMaxima], tile = 0x7FFFFFFF;
#pragma unroll
      for (int h = 0; h < kMaxima; ++h) {
        const int i = lane + 32 * h;
        mine[h] = x.max_key[i] == key ? x.max_tile[i] : 0x7FFFFFFF;
        tile = min(tile, mine[h]);
      }
      tile = __reduce_min_sync(0xffffffffu, tile);
      if (m == -kInf) {
        if (sl.nv > 0) best = max(sl.first_element(0), 0);
      } else {
#pragma unroll
        for (int h = 0; h < kMaxima; ++h) {
          if (mine[h] != tile) continue;
          for (int u = 0; u < kDeep; ++u) {
            const int i = tile * kTile + u * kStreamThreads + 32 * h + lane;
            if (i >= sl.nv) continue;
            float f[Elem<T>::kPer];
            unpack(sl.fetch(i), f, static_cast<const T*>(nullptr));
#pragma unroll
            for (int j = 0; j < Elem<T>::kPer; ++j)
              if (f[j] == m) best = min(best, sl.first_element(i) + j);
          }
        }
        best = __reduce_min_sync(0xffffffffu, best);
      }
    }
    if (rank == 0) given.fetch_logit(p, row);
    if (TOP == kTopMany) candidates(team, sl, x, p.top_k, many);
    // to the first CTA, once it is done with this warp's row before
    if (n_ctas > 1 && !wait_cluster(&x.row_free, phase ^ 1u, abort_flag, p.status, 67)) break;
    if (TOP == kTopMany) {
      const uint32_t to = map_to_rank(smem_u32(lists + rank * p.top_k), 0);
      rank_candidates(team, many.top, p.top_k, [&](int place, uint64_t y) { st_cluster(to + 8 * place, y); });
    }
    rebase(v.x, c, m, reference(m, c), v.y, v.z);
    v.y = warp_sum(v.y);
    if (ENT) v.z = warp_sum(v.z);
    if (lane == 0) st_cluster(map_to_rank(smem_u32(&x.slot[rank]), 0), make_float4(m, v.y, v.z, __int_as_float(best)));
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(&x.part_free);
      if (n_ctas > 1) mbar_arrive_cluster(map_to_rank(smem_u32(&x.row_full), 0));
    }
    if (rank == 0) {
      __syncwarp();
      if (n_ctas > 1 && !wait_cluster(&x.row_full, phase, abort_flag, p.status, 68)) break;
      finish<T, TOP, ENT>(team, p, r, row, given, x.slot, lists, n_ctas, x.result);
      __syncwarp();
      if (n_ctas > 1 && lane < n_ctas) mbar_arrive_cluster(map_to_rank(smem_u32(&x.row_free), lane));
    }
    __syncwarp();
  }
}

template <typename T, int TOP, bool ENT>
__global__ void __launch_bounds__(kAll, 1) logprobs_stream_kernel(const ScoreArgs p) {
  constexpr int kSlots = slots(TOP);
  extern __shared__ __align__(128) uint4 buf[];
  __shared__ Shared sh;
  Many* many = reinterpret_cast<Many*>(buf + kSlots * kTile);          // (kTopMany: of each finishing warp)
  uint64_t* lists = reinterpret_cast<uint64_t*>(many + kFinishWarps);  // [kFinishWarps][n_ctas][top_k]
  const int rank = cluster_rank(), n_ctas = cluster_ctas();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &sh.abort_flag;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], kStreamWarps);
    }
    for (int i = 0; i < kFinishWarps; ++i) {
      mbar_init(&sh.row[i].part_full, kStreamWarps);
      mbar_init(&sh.row[i].part_free, 1);
      mbar_init(&sh.row[i].row_full, n_ctas);
      mbar_init(&sh.row[i].row_free, 1);
    }
    sh.abort_flag = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  const int cluster = blockIdx.x / n_ctas, clusters = gridDim.x / n_ctas;
  const bool listed = p.row_ids && make_row_lists<kAll>(sh.lists, p.rows, cluster, clusters,
                                                        [&](int r) { return p.row_ids[r] == p.row_id; });
  __syncthreads();
  cluster_sync();
  const T* logits = static_cast<const T*>(p.logits);
  const float c = p.scale * kLog2e;
  const float lowest = lowest_value(c);

  if (warp == kStreamWarps + kFinishWarps) {
    // ----- producer
    int at = listed ? 0 : cluster;
    auto next_row = [&]() {
      if (listed) return at < sh.lists.n_first ? sh.lists.of_first[at++] : -1;
      if (p.row_ids) {  // 32 of the cluster's rows at a time
        while (at < p.rows) {
          const int64_t r = at + static_cast<int64_t>(lane) * clusters;
          const uint32_t asked = __ballot_sync(0xffffffffu, r < p.rows && p.row_ids[r] == p.row_id);
          const int64_t to = at + static_cast<int64_t>(asked ? __ffs(asked) - 1 : 32) * clusters;
          at = static_cast<int>(to < p.rows ? to : p.rows);
          if (asked) break;
        }
      }
      const int r = at < p.rows ? at : -1;
      if (r >= 0) at = clusters < p.rows - at ? at + clusters : p.rows;
      return r;
    };
    Ring<kSlots> ring;
    bool ok = true;
    int issued = 0;
    while (ok) {
      const int r = next_row();
      const Slice<T> sl(logits + (r < 0 ? 0 : r) * p.ld, p.vocab, rank, n_ctas);
      const char* src = reinterpret_cast<const char*>(sl.row + sl.first_element(0));
      const int lo = sl.nv > 0 && !sl.whole(0) ? 1 : 0;
      const int hi = sl.nv > 0 && !sl.whole(sl.nv - 1) ? sl.nv - 1 : sl.nv;
      const int tiles = r < 0 ? 1 : tiles_of(sl);
      for (int t = 0; t < tiles && ok; ++t, ring.next()) {
        if (lane == 0) {
          ok = mbar_wait(&sh.empty[ring.slot], ring.phase ^ 1u, abort_flag, p.status, 63);
          if (ok) {
            sh.slot_row[ring.slot] = r;
            const int a = max(t * kTile, lo), b = min((t + 1) * kTile, hi);
            if (r >= 0 && b > a) {
              mbar_arrive_expect_tx(&sh.full[ring.slot], (b - a) * 16u);
              bulk_load(buf + ring.slot * kTile + (a - t * kTile), src + static_cast<int64_t>(a) * 16, (b - a) * 16u,
                        &sh.full[ring.slot]);
            } else {
              mbar_arrive(&sh.full[ring.slot]);
            }
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        issued += ok;
      }
      if (r < 0) break;
    }
    if (!ok && lane == 0) {  // no copy may land after the CTA has left
      for (int i = 0; i < kSlots && i < issued; ++i) {
        const int n = issued - 1 - i;
        mbar_drain(&sh.full[n % kSlots], (n / kSlots) & 1);
      }
    }
  } else if (warp < kStreamWarps) {
    // ----- statistics
    Ring<kSlots> ring;
    const uint4 none = no_elements<T>();
    int n = 0;  // finishing warp of the row
    uint32_t phase = 0;
    for (bool ok = true;; phase ^= ++n == kFinishWarps, n = n == kFinishWarps ? 0 : n) {
      if (!mbar_wait_warp(smem_u32(&sh.full[ring.slot]), ring.phase, abort_flag, p.status, 64)) break;
      const int r = sh.slot_row[ring.slot];
      if (r < 0) {  // every finishing warp has to know
        for (int i = 0; i < kFinishWarps; ++i) {
          Row& x = sh.row[n];
          if (!mbar_wait_warp(smem_u32(&x.part_free), phase ^ 1u, abort_flag, p.status, 65)) break;
          if (threadIdx.x == 0) x.row = -1;
          __syncwarp();
          if (lane == 0) mbar_arrive(&x.part_full);
          phase ^= ++n == kFinishWarps;
          if (n == kFinishWarps) n = 0;
        }
        break;
      }
      Row& x = sh.row[n];
      if (!mbar_wait_warp(smem_u32(&x.part_free), phase ^ 1u, abort_flag, p.status, 65)) break;
      const Slice<T> sl(logits + r * p.ld, p.vocab, rank, n_ctas);
      const int tiles = tiles_of(sl), per_part = tiles_of_part(tiles);
      const int lo = sl.nv > 0 && !sl.whole(0) ? 1 : 0, hi = sl.nv > 0 && !sl.whole(sl.nv - 1) ? sl.nv - 1 : sl.nv;
      Stat st;
      int at = 0, in_part = 0;
      float part = -kInf;
      uint16_t* part_key = many[n].group_key + threadIdx.x;
      for (int t = 0; t < tiles; ++t) {
        if (t > 0 && !(ok = mbar_wait_warp(smem_u32(&sh.full[ring.slot]), ring.phase, abort_flag, p.status, 64))) break;
        uint4 v[kDeep];
        const uint4* tile = buf + ring.slot * kTile + threadIdx.x;
        const int k0 = t * kTile + threadIdx.x;
        if (t * kTile >= lo && (t + 1) * kTile <= hi) {
#pragma unroll
          for (int u = 0; u < kDeep; ++u) v[u] = tile[u * kStreamThreads];
        } else {  // the slice's ends: copies bring whole vectors alone
#pragma unroll
          for (int u = 0; u < kDeep; ++u) {
            const int k = k0 + u * kStreamThreads;
            v[u] = k >= lo && k < hi ? tile[u * kStreamThreads] : none;
            if (k < sl.nv && (k < lo || k >= hi)) v[u] = sl.gather(k);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.empty[ring.slot]);
        ring.next();
        const float before = st.m, m = stat_add<T, kDeep, ENT>(st, v, c, lowest);
        if (TOP == kTopOne && m > before) at = t;
        if (TOP == kTopMany) {
          part = fmaxf(part, m);
          if (++in_part == per_part || t == tiles - 1) {
            *part_key = static_cast<uint16_t>(order_key(part) >> 16);
            part_key += kStreamThreads;
            in_part = 0;
            part = -kInf;
          }
        }
      }
      if (!ok) break;
      if (TOP != kTopNone) x.max_key[threadIdx.x] = order_key(st.m);
      if (TOP == kTopOne) x.max_tile[threadIdx.x] = static_cast<uint16_t>(at);
      const float3 w_stat = warp_stat<T, ENT>(st, c, threadIdx.x, kStreamThreads, sl.nv, FromRow<T>{sl});
      if (lane == 0) x.part[warp] = make_float4(w_stat.x, w_stat.y, w_stat.z, 0.f);
      if (threadIdx.x == 0) x.row = r;
      __syncwarp();
      if (lane == 0) mbar_arrive(&x.part_full);
    }
  } else {
    // ----- the rest of a row
    const int i = warp - kStreamWarps;
    finish_rows<T, TOP, ENT>(p, sh.row[i], many[i], lists + i * n_ctas * p.top_k, abort_flag, rank, n_ctas);
  }
  __syncwarp();
  cluster_sync();  // no CTA leaves while another may still write to it
}

size_t smem_bytes(int top_k, int cluster) {
  if (top_k <= 1) return slots(kTopOne) * kTileBytes;
  return slots(kTopMany) * kTileBytes + kFinishWarps * (sizeof(Many) + sizeof(uint64_t) * cluster * top_k);
}
static_assert(slots(kTopMany) * kTileBytes + kFinishWarps * (sizeof(Many) + sizeof(uint64_t) * kStreamCluster * kMaxTop) +
                      sizeof(Shared) <= 226 * 1024 &&
                  slots(kTopOne) * kTileBytes + sizeof(Shared) <= 226 * 1024,
              "a CTA's shared memory");
static_assert((kMaxRowBytes / 16 + 2) / kTile < 65535, "tiles of a row in 16 bits");

template <auto kKernel>
cudaError_t launch_stream(const ScoreArgs& p, cudaStream_t s) {
  Clusters l;
  const cudaError_t e =
      choose_clusters<kKernel>(p.rows, 1, kStreamCluster, kAll, smem_bytes(p.top_k > 1 ? kMaxTop : 1, kStreamCluster), &l);
  return e != cudaSuccess ? e : launch_clusters<kKernel>(l, kAll, smem_bytes(p.top_k, l.size), s, p);
}

template <typename T, int TOP>
cudaError_t stream_ent(const ScoreArgs& p, cudaStream_t s) {
  return p.entropy ? launch_stream<&logprobs_stream_kernel<T, TOP, true>>(p, s)
                   : launch_stream<&logprobs_stream_kernel<T, TOP, false>>(p, s);
}

}  // namespace

// Streaming against a cluster per row, us, the likeliest token and the entropy / the 8 likeliest tokens, fp16:
// rows of 253 KB: 64 MB 18.8 / 20.3 against 22.5 / 30.6, 32 MB 13.1 / 14.8 against 14.2 / 20.6, 16 MB 11.2 / 13.8
// against 8.7 / 12.1; of 128 KB: 128 MB 30.2 / 34.4 against 38.1 / 51.0, 64 MB 23.2 / 27.6 against 22.3 / 31.2, 32
// MB 18.7 / 24.4 against 14.2 / 20.1; of 64 KB: 512 MB 131 / 176 against 125 / 150.
// Longer rows do not make the stream's start shorter (clusters of at most 4 CTAs, where a row of its own takes up to 16), so
// that it takes as many bytes: 494 KB 64 rows 12.5 / 15.1 against 13.7 / 16.1, 48 rows 11.6 / 14.1 against 9.4 / 10.8, 16
// rows 9.5 / 12.2 against 6.0 / 8.7; 1 MB 32 rows 12.3 / 15.1 against 13.9 / 17.4, 24 rows 11.5 / 14.0 against 12.2 / 15.4, 8 rows
// 10.6 / 12.9 against 6.4 / 8.5; 1.9 MB 16 rows 18.2 / 19.1 against 22.4 / 26.8, 12 rows 18.0 / 18.9 against 15.8 / 19.3,
// 1 row 16.9 / 17.7 against 7.2 / 9.4; 3 MB 12 rows 17.0 / 19.7 against 17.7 / 20.4, 4 rows 16.5 / 19.1 against 9.1 / 11.0.
bool stream_pays(int rows, int64_t row_bytes) {
  const double share = (256 << 10) / static_cast<double>(row_bytes), least = share > 1.08 ? 24 * share * share : 28;  // MB
  return row_bytes >= 96 * 1024 && rows * row_bytes >= least * (1 << 20);
}

template <typename T>
cudaError_t score_stream(const ScoreArgs& p, cudaStream_t s) {
  if (p.top_k == 0) return stream_ent<T, kTopNone>(p, s);
  if (p.top_k == 1) return stream_ent<T, kTopOne>(p, s);
  return stream_ent<T, kTopMany>(p, s);
}
template cudaError_t score_stream<f16>(const ScoreArgs&, cudaStream_t);
template cudaError_t score_stream<bf16>(const ScoreArgs&, cudaStream_t);
template cudaError_t score_stream<float>(const ScoreArgs&, cudaStream_t);

}  // namespace rows
}  // namespace sgd
