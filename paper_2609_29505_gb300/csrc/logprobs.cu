// Log-probabilities of given tokens, entropy and the likeliest tokens of rows of logits.
//
// With x_j = scale z_j, m = max x and s = sum e^(x_j - m):
//   ln p_t = (x_t - m) - ln s,   H = ln s - sum (x_j - m) e^(x_j - m) / s,
// and the likeliest tokens by (z descending, index ascending).
//
// The kernel here is for few or short rows: a cluster takes one row, a slice per CTA, and leaves
// (vocab_rows.cuh); many long rows stream through logprobs_stream.cu.
//
// Measured (GB300): 1 x 126464 fp16, the 4 likeliest tokens, entropy and one given token, on a cluster of 16:
// 5.8 us, latency (the copy, four reductions, the cluster's barrier); 1003 x 32003 bf16, the 8 likeliest,
// entropy, 4 given tokens: 30 us = 2.1 TB/s: three CTAs of 64 KB an SM, each without a copy on its way for
// half of its time.
#include "logprobs.cuh"

namespace sgd {
namespace {

using namespace rows;

template <typename T, int TOP, bool ENT, int kThreads>
__global__ void __launch_bounds__(kThreads, 768 / kThreads) logprobs_kernel(const ScoreArgs p, uint32_t list_offset) {
  constexpr int kWarps = kThreads / 32, kStep = kThreads * kUnroll;
  static_assert(kPiece % kStep == 0, "a thread's vectors lie in one piece");
  extern __shared__ __align__(128) uint4 buf[];
  __shared__ uint64_t bars[kMaxPieces];
  __shared__ int abort_flag;
  __shared__ float4 parts[kWarps];
  __shared__ float4 slot[kMaxCluster];
  __shared__ float result[2];
  __shared__ int best;
  __shared__ int n_reaching;
  __shared__ uint16_t reaching[TOP == kTopMany ? kThreads : 1];
  __shared__ __align__(16) unsigned char top_raw[TOP == kTopMany ? sizeof(TopShared) : 16];
  const Team<kThreads, 0> team{static_cast<int>(threadIdx.x)};
  const int rank = cluster_rank(), n_ctas = cluster_ctas();
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
    n_reaching = 0;
    start_copies(sl, buf, bars);
  }
  fill_ends(sl, buf);
  Given<T> given;
  if (rank == 0) given.fetch_token(p, r, threadIdx.x);
  __syncthreads();
  cluster_arrive();

  const float c = p.scale * kLog2e;
  const float lowest = lowest_value(c);
  Stat st;
  int at = 0;  // step in which the maximum was met first
  const uint4 none = no_elements<T>();
  for (int i = 0; i * kStep < sl.nv; ++i) {
    if (i * kStep % kPiece == 0) wait_piece(bars, i * kStep / kPiece, &abort_flag, p.status, 61);
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = i * kStep + u * kThreads + threadIdx.x;
      v[u] = k < sl.nv ? buf[k] : none;
    }
    const float before = st.m;
    if (stat_add<T, kUnroll, ENT>(st, v, c, lowest) > before) at = i;
  }

  if (rank == 0) given.fetch_logit(p, row);

  // the CTA's statistics
  const float3 w_stat = warp_stat<T, ENT>(st, c, threadIdx.x, kThreads, sl.nv, InShared{buf});
  if (lane == 0) parts[warp] = make_float4(w_stat.x, w_stat.y, w_stat.z, 0.f);
  __syncthreads();
  float m = w_stat.x;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) m = fmaxf(m, parts[w].x);
  if (TOP == kTopOne) {
    if (m == -kInf) {
      if (threadIdx.x == 0 && sl.nv > 0) best = max(sl.first_element(0), 0);
    } else if (st.m == m) {
      int found = 0x7FFFFFFF;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int k = at * kStep + u * kThreads + threadIdx.x;
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
  uint64_t* lists = reinterpret_cast<uint64_t*>(reinterpret_cast<char*>(buf) + list_offset);
  TopShared& top = *reinterpret_cast<TopShared*>(top_raw);
  if (TOP == kTopMany) {
    const uint32_t keys[1] = {order_key(st.m)};
    const Threshold th = threshold(team, keys, p.top_k, top);
    const uint32_t from = th.from();
    // what the threads hold whose maximum reaches the threshold, looked at by all threads
    if (keys[0] >= from) reaching[atomicAdd(&n_reaching, 1)] = static_cast<uint16_t>(threadIdx.x);
    __syncthreads();
    const float bar = key_value(from);
    const int steps = (sl.nv + kThreads - 1) / kThreads, all = n_reaching * steps;
    const float steps_inv = 1.f / steps;
    for (int j = threadIdx.x; j < all; j += kThreads) {
      const int q = static_cast<int>((j + 0.5f) * steps_inv);  // j / steps: exact, j is far below 2^22
      const int i = (j - q * steps) * kThreads + reaching[q];
      if (i >= sl.nv) continue;
      const uint4 v = buf[i];
      if (from > kKeyNegInf && !(vec_max<1>(&v, static_cast<const T*>(nullptr)) >= bar)) continue;
      append<T>(v, sl.first_element(i), sl.vocab, from, &top);
    }
    __syncthreads();
    const int found = top.n;
    __syncthreads();
    if (found > kCap) candidates_of_many(team, sl, InShared{buf}, th.lo, th.top, p.top_k, top);
    else if (th.tied && found < p.top_k) collect_ties(team, sl, InShared{buf}, th.lo, p.top_k - found, top);
  }
  __syncwarp();
  cluster_wait();  // every CTA of the cluster runs: the leader's shared memory may be written
  if (TOP == kTopMany) {
    const uint32_t to = map_to_rank(smem_u32(lists + rank * p.top_k), 0);
    rank_candidates(team, top, p.top_k, [&](int place, uint64_t x) { st_cluster(to + 8 * place, x); });
  }
  if (warp == 0) {
    float s = 0.f, t = 0.f;
    if (lane < kWarps) {
      s = parts[lane].y;
      t = parts[lane].z;
      rebase(parts[lane].x, c, m, reference(m, c), s, t);
    }
    s = warp_sum(s);
    if (ENT) t = warp_sum(t);
    if (lane == 0)
      st_cluster(map_to_rank(smem_u32(&slot[rank]), 0), make_float4(m, s, t, __int_as_float(TOP == kTopOne ? best : 0)));
  }
  __syncwarp();
  cluster_sync();
  if (rank == 0) finish<T, TOP, ENT>(team, p, r, row, given, slot, lists, n_ctas, result);
}

template <typename T, int TOP>
cudaError_t launch_ent(const ScoreArgs& p, const Launch& l, size_t smem, cudaStream_t s) {
  const uint32_t lists = l.slice_bytes;
  if (l.threads == 64)
    return p.entropy ? launch<&logprobs_kernel<T, TOP, true, 64>>(p.rows, l, smem, s, p, lists)
                     : launch<&logprobs_kernel<T, TOP, false, 64>>(p.rows, l, smem, s, p, lists);
  return p.entropy ? launch<&logprobs_kernel<T, TOP, true, 256>>(p.rows, l, smem, s, p, lists)
                   : launch<&logprobs_kernel<T, TOP, false, 256>>(p.rows, l, smem, s, p, lists);
}
template <typename T>
cudaError_t launch_type(const ScoreArgs& p, cudaStream_t s) {
  if (stream_pays(p.rows, static_cast<int64_t>(p.vocab) * sizeof(T))) return score_stream<T>(p, s);
  const Launch l = plan(p.rows, p.vocab, sizeof(T));
  const size_t smem = l.slice_bytes + (p.top_k > 1 ? sizeof(uint64_t) * l.cluster * p.top_k : 0);
  if (p.top_k == 0) return launch_ent<T, kTopNone>(p, l, smem, s);
  if (p.top_k == 1) return launch_ent<T, kTopOne>(p, l, smem, s);
  return launch_ent<T, kTopMany>(p, l, smem, s);
}

}  // namespace

cudaError_t logprobs_launch(const LogprobsParams& q, cudaStream_t s) {
  const ScoreArgs p{q.logits, q.ld, q.rows, q.vocab, q.scale, q.row_ids, q.row_id, q.tokens, q.n_tokens,
                    q.token_logprobs, q.entropy, q.top_k, q.top_ids, q.top_logprobs, device_status_ptr()};
  if (q.dtype == SGD_F16) return launch_type<f16>(p, s);
  if (q.dtype == SGD_BF16) return launch_type<bf16>(p, s);
  return launch_type<float>(p, s);
}

}  // namespace sgd
