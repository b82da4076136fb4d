// Log-probabilities of given tokens, entropy and the likeliest tokens of rows of logits.
//
// With x_j = scale z_j, m = max x and s = sum e^(x_j - m):
//   ln p_t = (x_t - m) - ln s,   H = ln s - sum (x_j - m) e^(x_j - m) / s,
// and the likeliest tokens by (z descending, index ascending).  One pass over the row from HBM
// (vocab_rows.cuh); the likeliest tokens come from a second pass over the slice in shared memory,
// of the threads alone that hold one:
//   - the k-th largest of the 256 threads' maxima (found by bisection, counting with the barrier)
//     is at most the slice's k-th largest value, and few values lie above it: those are collected;
//   - should they be many (rows that are nearly constant, or sorted so that few threads hold the
//     largest values), the threshold is bisected over all values until it is the k-th largest one
//     itself or few lie above it, and what is equal to it is taken in the order of the index;
//   - every candidate's rank among the candidates is counted, and the cluster's leader merges the
//     CTAs' sorted lists.
#include "vocab_rows.cuh"

namespace sgd {
namespace {

using namespace rows;

constexpr int kCap = 512;  // candidates a CTA ranks

// value of a candidate above, (reversed) index below: larger is likelier, ties to the lower index
__device__ __forceinline__ uint64_t candidate(uint32_t key, int index) {
  return static_cast<uint64_t>(key) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(index));
}
__device__ __forceinline__ int candidate_index(uint64_t c) {
  return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(c));
}

struct TopShared {
  uint64_t list[kCap];
  int n;
  uint32_t lo, hi;
  uint32_t warp_lo[kWarps], warp_hi[kWarps];
  int count[3];
  int warp_count[kWarps];
};

// Elements of the slice with a key of at least `bar`, over the CTA (every thread gets the count).
// `turn`: 0, 1, 2, 0, ... over the calls; the slot of the call after the next is cleared in each.
template <typename T>
__device__ int count_from(const Slice<T>& sl, const uint4* buf, uint32_t bar, TopShared& sh, int turn) {
  int n = 0;
  for (int i = threadIdx.x; i < sl.nv; i += kThreads) {
    float f[Elem<T>::kPer];
    unpack(buf[i], f, static_cast<const T*>(nullptr));
    const int e = sl.first_element(i);
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; ++j) n += order_key(f[j]) >= bar && e + j >= 0 && e + j < sl.vocab;
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if ((threadIdx.x & 31) == 0 && n) atomicAdd(&sh.count[turn], n);
  if (threadIdx.x == 0) sh.count[(turn + 1) % 3] = 0;
  __syncthreads();
  return sh.count[turn];
}

// Appends the slice's elements with a key of at least `from` to the list (as many as it holds) and
// adds their number to sh.n; `mine`: whether this thread may hold one.
template <typename T>
__device__ void collect(const Slice<T>& sl, const uint4* buf, uint32_t from, bool mine, TopShared& sh) {
  if (mine) {
    const float bar = key_value(from);
    for (int i = threadIdx.x; i < sl.nv; i += kThreads) {
      const uint4 v = buf[i];
      if (from > kKeyNegInf && !(vec_max<1>(&v, static_cast<const T*>(nullptr)) >= bar)) continue;
      float f[Elem<T>::kPer];
      unpack(v, f, static_cast<const T*>(nullptr));
      const int e = sl.first_element(i);
#pragma unroll
      for (int j = 0; j < Elem<T>::kPer; ++j) {
        const uint32_t key = order_key(f[j]);
        if (key >= from && e + j >= 0 && e + j < sl.vocab) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < kCap) sh.list[at] = candidate(key, e + j);
        }
      }
    }
  }
  __syncthreads();
}

// The first `need` elements of key `key` in the order of the index are put behind the list.
template <typename T>
__device__ void collect_ties(const Slice<T>& sl, const uint4* buf, uint32_t key, int need, TopShared& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int have = 0;
  const int base = sh.n;
  __syncthreads();
  for (int i0 = 0; i0 < sl.nv && have < need; i0 += kThreads) {
    const int i = i0 + threadIdx.x, e = sl.first_element(i);
    uint32_t hit = 0;
    if (i < sl.nv) {
      float f[Elem<T>::kPer];
      unpack(buf[i], f, static_cast<const T*>(nullptr));
#pragma unroll
      for (int j = 0; j < Elem<T>::kPer; ++j)
        hit |= (order_key(f[j]) == key && e + j >= 0 && e + j < sl.vocab ? 1u : 0u) << j;
    }
    int before = __popc(hit);
    const int mine = before;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += up;
    }
    if (lane == 31) sh.warp_count[warp] = before;
    before -= mine;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += sh.warp_count[w];
      all += sh.warp_count[w];
    }
    before += have;
    for (; hit && before < need; hit &= hit - 1, ++before)
      sh.list[base + before] = candidate(key, e + __ffs(hit) - 1);
    have += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) sh.n = base + min(have, need);
  __syncthreads();
}

// The slice's k likeliest elements are among the candidates left in sh.list (sh.n of them, at most
// kCap); thread_max: the largest of this thread's elements.
template <typename T>
__device__ void candidates(const Slice<T>& sl, const uint4* buf, float thread_max, int k, TopShared& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t key = order_key(thread_max);
  const uint32_t wlo = __reduce_min_sync(0xffffffffu, key), whi = __reduce_max_sync(0xffffffffu, key);
  if (lane == 0) {
    sh.warp_lo[warp] = wlo;
    sh.warp_hi[warp] = whi;
  }
  if (threadIdx.x == 0) sh.n = sh.count[0] = sh.count[1] = 0;
  __syncthreads();
  uint32_t lo = sh.warp_lo[0], hi = sh.warp_hi[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) {
    lo = min(lo, sh.warp_lo[w]);
    hi = max(hi, sh.warp_hi[w]);
  }
  const uint32_t top = hi + 1;  // no key is as large (the largest is that of +inf)
  hi = top;
  // count(maxima >= lo) >= k > count(maxima >= hi): 256 threads are more than k
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const int n = __syncthreads_count(key >= mid);
    if (n >= k) lo = mid; else hi = mid;
    if (n >= k && n <= k + k / 4) break;
  }
  collect(sl, buf, lo, key >= lo, sh);
  if (sh.n <= kCap) return;
  __syncthreads();
  // Too many: count(all >= lo) > kCap >= k.  A row of many equal values is over at once (none is
  // larger than the threshold, or too few); the others take up to 32 counts.
  hi = top;
  int turn = 0, n = 0;
  uint32_t mid = lo + 1;
  while (hi - lo > 1) {
    n = count_from(sl, buf, mid, sh, turn);
    turn = (turn + 1) % 3;
    if (n >= k) lo = mid; else hi = mid;
    if (n >= k && n <= kCap) break;
    mid = lo + (hi - lo) / 2;
  }
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  if (n >= k && n <= kCap) {
    collect(sl, buf, lo, true, sh);
    return;
  }
  // fewer than k above lo: those, and the first of those equal to it
  collect(sl, buf, lo + 1, true, sh);
  collect_ties(sl, buf, lo, k - sh.n, sh);
}

struct Params {
  const void* logits;
  int64_t ld;
  int vocab;
  float scale;
  const int32_t* row_ids;
  int row_id;
  const int32_t* tokens;
  int n_tokens;
  float* token_logprobs;
  float* entropy;
  int top_k;
  int32_t* top_ids;
  float* top_logprobs;
  uint32_t top_offset;  // of the leader's lists in dynamic shared memory
  int* status;
};

enum { kTopNone = 0, kTopOne = 1, kTopMany = 2 };

template <typename T, int TOP, bool ENT>
__global__ void __launch_bounds__(kThreads, 3) logprobs_kernel(const Params p) {
  extern __shared__ __align__(128) uint4 buf[];
  __shared__ uint64_t bars[kMaxPieces];
  __shared__ int abort_flag;
  __shared__ float4 warp_stat[kWarps];
  __shared__ float4 slot[kMaxCluster];
  __shared__ float result[2];  // m, ln s
  __shared__ int best;
  __shared__ __align__(16) unsigned char top_raw[TOP == kTopMany ? sizeof(TopShared) : 16];
  const int rank = cluster_rank();
  uint32_t n_ctas;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n_ctas));
  const int64_t r = blockIdx.x / n_ctas;
  if (p.row_ids && p.row_ids[r] != p.row_id) return;  // the whole cluster
  const T* row = static_cast<const T*>(p.logits) + r * p.ld;
  const Slice<T> sl(row, p.vocab, rank, n_ctas);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i * kPiece < sl.nv; ++i) mbar_init(&bars[i], 1);
    fence_mbar_init();
    fence_proxy_async_smem();
    abort_flag = 0;
    best = 0x7FFFFFFF;
    start_copies(sl, buf, bars);
  }
  fill_ends(sl, buf);
  // the leader's given tokens, fetched while the copies run
  float given = 0.f;
  int token = -1;
  if (rank == 0 && threadIdx.x < p.n_tokens) {
    token = p.tokens[r * p.n_tokens + threadIdx.x];
    given = token >= 0 && token < p.vocab ? to_f(row[token]) : kNan;
  }
  __syncthreads();
  cluster_arrive();

  const float c = p.scale * kLog2e;
  Stat st;
  int at = 0;  // piece in which the maximum was met first
  const uint4 none = [] {
    uint4 v;
    T* e = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; ++j) e[j] = neg_inf<T>();
    return v;
  }();
  for (int i = 0; i * kPiece < sl.nv; ++i) {
    wait_piece(bars, i, &abort_flag, p.status, 61);
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = i * kPiece + u * kThreads + threadIdx.x;
      v[u] = k < sl.nv ? buf[k] : none;
    }
    if (stat_add<T, kUnroll, ENT>(st, v, c)) at = i;
  }

  // the CTA's statistics
  float m = key_value(__reduce_max_sync(0xffffffffu, order_key(st.m)));
  {
    float s = st.s, t = st.t;
    rebase(st.m, c, reference(m, c), s, t);
    s = warp_sum(s);
    if (ENT) t = warp_sum(t);
    if (lane == 0) warp_stat[warp] = make_float4(m, s, t, 0.f);
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) m = fmaxf(m, warp_stat[w].x);
  if (TOP == kTopOne) {
    if (m == -kInf) {
      if (threadIdx.x == 0 && sl.nv > 0) best = max(sl.first_element(0), 0);
    } else if (st.m == m) {
      int found = 0x7FFFFFFF;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int k = at * kPiece + u * kThreads + threadIdx.x;
        if (k < sl.nv && found == 0x7FFFFFFF) {
          float f[Elem<T>::kPer];
          unpack(buf[k], f, static_cast<const T*>(nullptr));
#pragma unroll
          for (int j = Elem<T>::kPer - 1; j >= 0; --j)
            if (f[j] == m) found = sl.first_element(k) + j;
        }
      }
      atomicMin(&best, found);
    }
    __syncthreads();
  }
  uint64_t* lists = reinterpret_cast<uint64_t*>(reinterpret_cast<char*>(buf) + p.top_offset);
  TopShared& top = *reinterpret_cast<TopShared*>(top_raw);
  if (TOP == kTopMany) candidates(sl, buf, st.m, p.top_k, top);
  cluster_wait();  // every CTA of the cluster runs: the leader's shared memory may be written
  if (TOP == kTopMany) {
    const uint32_t to = map_to_rank(smem_u32(lists + rank * p.top_k), 0);
    const int n = top.n;
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const uint64_t x = top.list[i];
      int place = 0;
      for (int j = 0; j < n; ++j) place += top.list[j] > x;
      if (place < p.top_k) st_cluster(to + 8 * place, x);
    }
    for (int i = n + threadIdx.x; i < p.top_k; i += kThreads) st_cluster(to + 8 * i, static_cast<uint64_t>(0));
  }
  if (warp == 0) {
    float s = 0.f, t = 0.f;
    if (lane < kWarps) {
      s = warp_stat[lane].y;
      t = warp_stat[lane].z;
      rebase(warp_stat[lane].x, c, reference(m, c), s, t);
    }
    s = warp_sum(s);
    if (ENT) t = warp_sum(t);
    if (lane == 0)
      st_cluster(map_to_rank(smem_u32(&slot[rank]), 0), make_float4(m, s, t, __int_as_float(TOP == kTopOne ? best : 0)));
  }
  __syncwarp();
  cluster_sync();
  if (rank != 0) return;

  // the row's statistics and what follows from them
  if (warp == 0) {
    float4 v = make_float4(-kInf, 0.f, 0.f, 0.f);
    if (lane < n_ctas) v = slot[lane];
    const float all = key_value(__reduce_max_sync(0xffffffffu, order_key(v.x)));
    const float R = reference(all, c);
    float s = v.y, t = v.z;
    rebase(v.x, c, R, s, t);
    s = warp_sum(s);
    if (ENT) t = warp_sum(t);
    // the CTA of the lowest rank that has the maximum has it at the lowest index
    const int index = __reduce_min_sync(0xffffffffu, lane < n_ctas && v.x == all ? __float_as_int(v.w) : 0x7FFFFFFF);
    if (lane == 0) {
      const bool empty = all == -kInf && s == 0.f;  // (NaN: s is NaN)
      const float delta = all == -kInf ? 0.f : fmaf(all, c, -R);
      const float ln_s = empty ? 0.f : logf(s) - delta * kLn2;
      result[0] = empty ? kInf : all;  // an empty row: every difference to it is -inf
      result[1] = ln_s;
      // H / ln 2 = log2 s' - t / s'; the reference's rounding cancels in the difference
      if (ENT) p.entropy[r] = empty ? 0.f : logf(s) - kLn2 * (t / s);
      if (TOP == kTopOne) {
        if (p.top_ids) p.top_ids[r] = index;
        if (p.top_logprobs) p.top_logprobs[r] = empty ? -kInf : (s != s ? kNan : -ln_s);
      }
    }
  }
  __syncthreads();
  const float all = result[0], ln_s = result[1];
  auto logprob = [&](float z) { return (z - all) * p.scale - ln_s; };
  if (threadIdx.x < p.n_tokens) p.token_logprobs[r * p.n_tokens + threadIdx.x] = token < 0 ? 0.f : logprob(given);
  for (int i = threadIdx.x + kThreads; i < p.n_tokens; i += kThreads) {
    token = p.tokens[r * p.n_tokens + i];
    p.token_logprobs[r * p.n_tokens + i] =
        token < 0 ? 0.f : (token < p.vocab ? logprob(to_f(row[token])) : kNan);
  }
  if (TOP == kTopMany) {
    const int k = p.top_k;
    for (int i = threadIdx.x; i < static_cast<int>(n_ctas) * k; i += kThreads) {
      const uint64_t x = lists[i];
      if (x == 0) continue;
      const int own = i / k;
      int place = i - own * k;
      for (int l = 0; l < static_cast<int>(n_ctas) && place < k; ++l) {
        if (l == own) continue;
        int a = 0, b = k;  // first entry of list l that is smaller
        while (a < b) {
          const int mid = (a + b) >> 1;
          if (lists[l * k + mid] > x) a = mid + 1; else b = mid;
        }
        place += a;
      }
      if (place < k) {
        if (p.top_ids) p.top_ids[r * k + place] = candidate_index(x);
        if (p.top_logprobs) p.top_logprobs[r * k + place] = logprob(key_value(static_cast<uint32_t>(x >> 32)));
      }
    }
  }
}

template <typename T, int TOP>
cudaError_t launch_ent(const Params& p, int rows, const Launch& l, size_t smem, cudaStream_t s) {
  return p.entropy ? launch<&logprobs_kernel<T, TOP, true>>(rows, l, smem, s, p)
                   : launch<&logprobs_kernel<T, TOP, false>>(rows, l, smem, s, p);
}
template <typename T>
cudaError_t launch_top(const Params& p, int rows, const Launch& l, size_t smem, cudaStream_t s) {
  if (p.top_k == 0) return launch_ent<T, kTopNone>(p, rows, l, smem, s);
  if (p.top_k == 1) return launch_ent<T, kTopOne>(p, rows, l, smem, s);
  return launch_ent<T, kTopMany>(p, rows, l, smem, s);
}

}  // namespace

cudaError_t logprobs_launch(const LogprobsParams& q, cudaStream_t s) {
  const int elem = q.dtype == SGD_F32 ? 4 : 2;
  const Launch l = plan(q.rows, q.vocab, elem);
  Params p{q.logits, q.ld, q.vocab, q.scale, q.row_ids, q.row_id, q.tokens, q.n_tokens, q.token_logprobs,
           q.entropy, q.top_k, q.top_ids, q.top_logprobs, static_cast<uint32_t>(l.slice_bytes), device_status_ptr()};
  const size_t smem = l.slice_bytes + (q.top_k > 1 ? sizeof(uint64_t) * l.cluster * q.top_k : 0);
  if (q.dtype == SGD_F16) return launch_top<f16>(p, q.rows, l, smem, s);
  if (q.dtype == SGD_BF16) return launch_top<bf16>(p, q.rows, l, smem, s);
  return launch_top<float>(p, q.rows, l, smem, s);
}

}  // namespace sgd
