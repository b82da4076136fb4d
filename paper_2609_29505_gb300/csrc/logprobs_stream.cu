// Scoring of many long rows (logprobs.cu has the formulas): the rows stream through the SMs.
//
// One CTA per SM stays for the whole call.  A producer warp keeps a ring of 16 KB tiles filled by bulk
// copies, across the ends of rows; 8 warps take the tiles' statistics and never wait for anything but
// data; 4 warps finish a row (sums, likeliest tokens, outputs) while the others are at the next one.
// Where there are too few rows for the SMs, the CTAs of a cluster share each row and the first of
// them merges their parts.
//
// The likeliest tokens without a second pass over the row: the streaming warps leave the maximum of
// each group of vectors (of one thread, in consecutive tiles; at most 4096 groups).  The k-th largest of
// the 256 threads' maxima is a threshold that k elements or a few more reach; only the groups whose
// maximum reaches it are read again (some 64 bytes each, from L2).  For the single likeliest token
// the tile of each thread's first maximum is enough.
//
// Every wait is bounded.  After one has expired (recorded in the status word) each role leaves its loop;
// the teams that share a hardware barrier leave together.
#include "logprobs.cuh"
#include "persistent.cuh"

namespace sgd {
namespace rows {
namespace {

constexpr int kStreamWarps = 16, kStreamThreads = 32 * kStreamWarps;
constexpr int kDeep = 4, kTile = kStreamThreads * kDeep;  // vectors of a tile: kDeep per thread
constexpr int kFinishWarps = 4, kFinishThreads = 32 * kFinishWarps;  // of each of two teams, which take turns
constexpr int kAll = kStreamThreads + 2 * kFinishThreads + 32;
constexpr int kSlots = 5;
constexpr int kTileBytes = kTile * 16;
constexpr int kGroupTiles = 8;   // groups of one thread
constexpr int kMaxGroups = 256;  // groups read again
constexpr int kStreamCluster = 8;
constexpr int kMaxima = kStreamThreads / kFinishThreads;  // streaming threads' maxima per finishing thread

struct Shared {
  uint64_t full[kSlots], empty[kSlots];
  uint64_t part_full[2], part_free[2];    // a row's statistics in this CTA
  uint64_t row_full[2], row_free[2];      // its parts from all CTAs, in the first one
  int abort_flag;
  int slot_row[kSlots];                   // row of a tile; -1: no more
  int part_row[2];
  float4 part[2][kStreamWarps];
  uint32_t max_key[2][kStreamThreads];
  int max_tile[2][kStreamThreads];
  float4 slot[2][kStreamCluster];
  float result[2][2];
  int first_tile[2], best[2];
  int n_groups[2];
  RowLists rows;
};
struct Many {
  TopShared top[2];
  int groups[2][kMaxGroups];
  uint32_t group_key[2][kGroupTiles * kStreamThreads];
};

template <typename T>
__device__ __forceinline__ int tiles_of(const Slice<T>& sl) { return max(1, (sl.nv + kTile - 1) / kTile); }

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

// The rows whose statistics are left in buffer b, one after another: their likeliest tokens in this CTA, and in
// the cluster's first CTA their outputs.
template <typename T, int TOP, bool ENT, typename Tm>
__device__ __forceinline__ void finish_rows(const Tm team, const int b, const ScoreArgs& p, Shared& sh, Many& many,
                                            uint64_t* lists, const int rank, const int n_ctas) {
  const T* logits = static_cast<const T*>(p.logits);
  const float c = p.scale * kLog2e;
  const int tid = team.tid;
  volatile int* abort_flag = &sh.abort_flag;
  TopShared& top = many.top[b];
  for (uint32_t phase = 0;; phase ^= 1) {
    bool ok = mbar_wait_warp(smem_u32(&sh.part_full[b]), phase, abort_flag, p.status, 66);
    const int r = ok ? sh.part_row[b] : -1;
    if (tid == 0) {
      sh.best[b] = sh.first_tile[b] = 0x7FFFFFFF;
      sh.n_groups[b] = 0;
    }
    if (team.count(!ok) || r < 0) break;
    const T* row = logits + r * p.ld;
    const Slice<T> sl(row, p.vocab, rank, n_ctas);
    Given<T> given;
    if (rank == 0) given.fetch(p, row, r, tid);
    auto fetch = [&](int i) { return sl.fetch(i); };
    float m = -kInf;
#pragma unroll
    for (int w = 0; w < kStreamWarps; ++w) m = fmaxf(m, sh.part[b][w].x);
    if (TOP == kTopOne) {
      const uint32_t key = order_key(m);
      int mine[kMaxima], first = 0x7FFFFFFF;
#pragma unroll
      for (int h = 0; h < kMaxima; ++h) {
        const int i = tid + h * kFinishThreads;
        mine[h] = sh.max_key[b][i] == key ? sh.max_tile[b][i] : 0x7FFFFFFF;
        first = min(first, mine[h]);
      }
      first = __reduce_min_sync(0xffffffffu, first);
      if ((tid & 31) == 0) atomicMin(&sh.first_tile[b], first);
      team.sync();
      const int tile = sh.first_tile[b];
      if (m == -kInf) {
        if (tid == 0 && sl.nv > 0) sh.best[b] = max(sl.first_element(0), 0);
      } else {
        int found = 0x7FFFFFFF;
#pragma unroll
        for (int h = 0; h < kMaxima; ++h) {
          if (mine[h] != tile) continue;
#pragma unroll
          for (int u = 0; u < kDeep; ++u) {
            const int i = tile * kTile + u * kStreamThreads + h * kFinishThreads + tid;
            if (i >= sl.nv) continue;
            float f[Elem<T>::kPer];
            unpack(sl.fetch(i), f, static_cast<const T*>(nullptr));
#pragma unroll
            for (int j = 0; j < Elem<T>::kPer; ++j)
              if (f[j] == m) found = min(found, sl.first_element(i) + j);
          }
        }
        if (found != 0x7FFFFFFF) atomicMin(&sh.best[b], found);
      }
      team.sync();
    }
    if (TOP == kTopMany) {
      const int tiles = tiles_of(sl), per_group = (tiles + kGroupTiles - 1) / kGroupTiles;
      const int n_keys = (tiles + per_group - 1) / per_group * kStreamThreads;
      uint32_t keys[kMaxima];
#pragma unroll
      for (int h = 0; h < kMaxima; ++h) keys[h] = sh.max_key[b][tid + h * kFinishThreads];
      uint32_t above;
      const uint32_t lo = threshold(team, keys, p.top_k, top, above);
      for (int i = 4 * tid; i < n_keys; i += 4 * kFinishThreads) {
        const uint4 k = *reinterpret_cast<const uint4*>(&many.group_key[b][i]);
        const uint32_t q[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (q[j] >= lo) {
            const int n = atomicAdd(&sh.n_groups[b], 1);
            if (n < kMaxGroups) many.groups[b][n] = i + j;
          }
      }
      team.sync();
      const int n = sh.n_groups[b], per = per_group * kDeep;  // vectors of a group
      if (n <= kMaxGroups) {
        const float bar = key_value(lo);
        for (int j = tid; j < n * per; j += kFinishThreads) {
          const int q = j / per, w = j - q * per, grp = many.groups[b][q];
          const int tile = grp / kStreamThreads * per_group + w / kDeep;
          const int i = tile * kTile + (w % kDeep) * kStreamThreads + grp % kStreamThreads;
          if (i >= sl.nv) continue;
          const uint4 v = sl.fetch(i);
          if (lo > kKeyNegInf && !(vec_max<1>(&v, static_cast<const T*>(nullptr)) >= bar)) continue;
          append(sl, v, sl.first_element(i), lo, top);
        }
      }
      team.sync();
      if (n > kMaxGroups || top.n > kCap) candidates_of_many(team, sl, fetch, lo, above, p.top_k, top);
    }
    // to the first CTA, once it is done with the row before the last
    if (n_ctas > 1) {
      ok = wait_cluster(&sh.row_free[b], phase ^ 1u, abort_flag, p.status, 67);
      if (team.count(!ok)) break;
    }
    if (TOP == kTopMany) {
      const uint32_t to = map_to_rank(smem_u32(lists + (b * n_ctas + rank) * p.top_k), 0);
      rank_candidates(team, top, p.top_k, [&](int place, uint64_t x) { st_cluster(to + 8 * place, x); });
    }
    if (tid < 32) {
      float s = 0.f, t = 0.f;
      if (tid < kStreamWarps) {
        s = sh.part[b][tid].y;
        t = sh.part[b][tid].z;
        rebase(sh.part[b][tid].x, c, reference(m, c), s, t);
      }
      s = warp_sum(s);
      if (ENT) t = warp_sum(t);
      if (tid == 0)
        st_cluster(map_to_rank(smem_u32(&sh.slot[b][rank]), 0), make_float4(m, s, t, __int_as_float(TOP == kTopOne ? sh.best[b] : 0)));
    }
    team.sync();
    if (tid == 0) {
      mbar_arrive(&sh.part_free[b]);
      if (n_ctas > 1) mbar_arrive_cluster(map_to_rank(smem_u32(&sh.row_full[b]), 0));
    }
    if (rank == 0) {
      if (n_ctas > 1) {
        ok = wait_cluster(&sh.row_full[b], phase, abort_flag, p.status, 68);
        if (team.count(!ok)) break;
      }
      finish<T, TOP, ENT>(team, p, r, row, given, sh.slot[b], lists + b * n_ctas * p.top_k, n_ctas, sh.result[b]);
      team.sync();
      if (n_ctas > 1 && tid < n_ctas) mbar_arrive_cluster(map_to_rank(smem_u32(&sh.row_free[b]), tid));
    }
  }
}

template <typename T, int TOP, bool ENT>
__global__ void __launch_bounds__(kAll, 1) logprobs_stream_kernel(const ScoreArgs p) {
  extern __shared__ __align__(128) uint4 buf[];
  __shared__ Shared sh;
  Many& many = *reinterpret_cast<Many*>(buf + kSlots * kTile);  // (kTopMany)
  uint64_t* lists = reinterpret_cast<uint64_t*>(buf + kSlots * kTile + sizeof(Many) / 16);  // [2][n_ctas][top_k]
  const int rank = cluster_rank(), n_ctas = cluster_ctas();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &sh.abort_flag;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], kStreamWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.part_full[i], kStreamWarps);
      mbar_init(&sh.part_free[i], 1);
      mbar_init(&sh.row_full[i], n_ctas);
      mbar_init(&sh.row_free[i], 1);
    }
    sh.abort_flag = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  const int cluster = blockIdx.x / n_ctas, clusters = gridDim.x / n_ctas;
  const bool listed = p.row_ids && make_row_lists<kAll>(sh.rows, p.rows, cluster, clusters,
                                                        [&](int r) { return p.row_ids[r] == p.row_id; });
  __syncthreads();
  cluster_sync();
  const T* logits = static_cast<const T*>(p.logits);
  const float c = p.scale * kLog2e;

  if (warp == kStreamWarps + 2 * kFinishWarps) {
    // ----- producer
    int at = listed ? 0 : cluster;
    auto next_row = [&]() {
      if (listed) return at < sh.rows.n_first ? sh.rows.of_first[at++] : -1;
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
    Ring ring;
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
    Ring ring;
    const uint4 none = no_elements<T>();
    for (int it = 0;; ++it) {
      const int b = it & 1;
      if (!mbar_wait_warp(smem_u32(&sh.full[ring.slot]), ring.phase, abort_flag, p.status, 64)) break;
      const int r = sh.slot_row[ring.slot];
      if (!mbar_wait_warp(smem_u32(&sh.part_free[b]), ((it >> 1) & 1) ^ 1u, abort_flag, p.status, 65)) break;
      if (r < 0) {  // both teams have to know
        const int o = b ^ 1;
        if (!mbar_wait_warp(smem_u32(&sh.part_free[o]), (((it + 1) >> 1) & 1) ^ 1u, abort_flag, p.status, 65)) break;
        if (threadIdx.x == 0) sh.part_row[0] = sh.part_row[1] = -1;
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.part_full[b]);
          mbar_arrive(&sh.part_full[o]);
        }
        break;
      }
      const Slice<T> sl(logits + r * p.ld, p.vocab, rank, n_ctas);
      const int tiles = tiles_of(sl), per_group = (tiles + kGroupTiles - 1) / kGroupTiles;
      Stat st;
      int at = 0;
      float group = -kInf;
      int in_group = 0, g = 0;
      bool ok = true;
      for (int t = 0; t < tiles; ++t) {
        if (t > 0 && !(ok = mbar_wait_warp(smem_u32(&sh.full[ring.slot]), ring.phase, abort_flag, p.status, 64))) break;
        uint4 v[kDeep];
        const uint4* tile = buf + ring.slot * kTile + threadIdx.x;
        if (t > 0 && t < tiles - 1) {
#pragma unroll
          for (int u = 0; u < kDeep; ++u) v[u] = tile[u * kStreamThreads];
        } else {  // the slice's ends
#pragma unroll
          for (int u = 0; u < kDeep; ++u) {
            const int k = t * kTile + u * kStreamThreads + threadIdx.x;
            v[u] = k >= sl.nv ? none : (sl.whole(k) ? tile[u * kStreamThreads] : sl.gather(k));
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.empty[ring.slot]);
        ring.next();
        const float before = st.m, m = stat_add<T, kDeep, ENT>(st, v, c);
        if (TOP == kTopOne && m > before) at = t;
        if (TOP == kTopMany) {
          group = fmaxf(group, m);
          if (++in_group == per_group || t == tiles - 1) {
            many.group_key[b][g * kStreamThreads + threadIdx.x] = order_key(group);
            ++g;
            in_group = 0;
            group = -kInf;
          }
        }
      }
      if (!ok) break;
      if (TOP != kTopNone) sh.max_key[b][threadIdx.x] = order_key(st.m);
      if (TOP == kTopOne) sh.max_tile[b][threadIdx.x] = at;
      const float m = key_value(__reduce_max_sync(0xffffffffu, order_key(st.m)));
      float s = st.s, u = st.t;
      rebase(st.m, c, reference(m, c), s, u);
      s = warp_sum(s);
      if (ENT) u = warp_sum(u);
      if (lane == 0) sh.part[b][warp] = make_float4(m, s, u, 0.f);
      if (threadIdx.x == 0) sh.part_row[b] = r;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.part_full[b]);
    }
  } else if (warp < kStreamWarps + kFinishWarps) {
    finish_rows<T, TOP, ENT>(Team<kFinishThreads, 1>{static_cast<int>(threadIdx.x) - kStreamThreads}, 0, p, sh, many, lists, rank, n_ctas);
  } else {
    finish_rows<T, TOP, ENT>(Team<kFinishThreads, 2>{static_cast<int>(threadIdx.x) - kStreamThreads - kFinishThreads}, 1, p, sh, many, lists,
                             rank, n_ctas);
  }
  __syncwarp();
  cluster_sync();  // no CTA leaves while another may still write to it
}

size_t smem_bytes(const ScoreArgs& p, int cluster) {
  return kSlots * kTileBytes + (p.top_k > 1 ? sizeof(Many) + 2 * sizeof(uint64_t) * cluster * p.top_k : 0);
}
static_assert(sizeof(Many) % 16 == 0, "the lists follow it");
constexpr size_t kMaxLists = 2 * sizeof(uint64_t) * kStreamCluster * kMaxTop;
static_assert(kSlots * kTileBytes + sizeof(Many) + kMaxLists + sizeof(Shared) <= 226 * 1024, "a CTA's shared memory");

template <auto kKernel>
cudaError_t launch_stream(const ScoreArgs& p, cudaStream_t s) {
  const size_t most = kSlots * kTileBytes + (p.top_k > 1 ? sizeof(Many) + kMaxLists : 0);
  Clusters l;
  const cudaError_t e = choose_clusters<kKernel>(p.rows, 1, kStreamCluster, kAll, most, &l);
  return e != cudaSuccess ? e : launch_clusters<kKernel>(l, kAll, smem_bytes(p, l.size), s, p);
}

template <typename T, int TOP>
cudaError_t stream_ent(const ScoreArgs& p, cudaStream_t s) {
  return p.entropy ? launch_stream<&logprobs_stream_kernel<T, TOP, true>>(p, s)
                   : launch_stream<&logprobs_stream_kernel<T, TOP, false>>(p, s);
}

}  // namespace

bool stream_pays(int rows, int64_t row_bytes) { return row_bytes >= 32 * 1024 && rows * row_bytes >= (32 << 20); }

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
