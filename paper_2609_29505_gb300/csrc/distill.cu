// Distillation of rows of logits from another model's likeliest tokens: loss and gradient.
//
// p = softmax(scale z).  A row's list gives q_i = e^(lq_i) for the tokens of a set S, Q = sum q_i:
//   renorm: q^_i = q_i / Q,          L = sum q^_i (ln q^_i - ln p_i),
//           dL/dz_j = scale (p_j - q^_j);
//   bucket: q_T = 1 - Q, p_T = sum_{j not in S} p_j,
//           L = sum q_i (ln q_i - ln p_i) + q_T (ln q_T - ln p_T),
//           dL/dz_j = scale (p_j - q_j) in S,  scale p_j (1 - q_T / p_T) outside;
//           with p_T = 0 the second term of L is left out: scale (Q p_j - q_j) in S.
//           (Q > 1, no distribution: q_T = 0, and the gradient is as for Q = 1.)
// The row is held in shared memory (vocab_rows.cuh), so that it is read once for both the loss and the
// gradient: 2 passes over it on chip, sizeof(logit) + sizeof(gradient) bytes per token in HBM.
//
// S is taken out of the row (its values are replaced by -inf in shared memory) before the sum, so
// that p_T is a sum of its own: 1 - sum_S p would leave nothing of a small tail.  In the gradient's
// pass -inf gives S the gradient 0, and its k entries are written after it.
//
// 1 - Q is taken of the fp64 sum of the rounded q_i (their rounding then cancels from the loss to first
// order); what else is done for a loss that is a difference of larger terms stands at row_loss().
//
// The kernel here is for few or short rows: a cluster takes one row, a slice per CTA, and leaves;
// many long rows stream through distill_stream.cu.
#include "distill.cuh"

namespace sgd {
namespace {

using namespace rows;

template <typename T, typename G, int kThreads>
__global__ void __launch_bounds__(kThreads, 768 / kThreads) distill_kernel(const DistillArgs p) {
  constexpr bool kGrad = !std::is_same<G, NoGrad>::value;
  constexpr int E = Elem<T>::kPer, kWarps = kThreads / 32, kStep = kThreads * kUnroll;
  static_assert(kThreads >= kMaxList, "a thread per entry of the list");
  extern __shared__ __align__(128) uint4 buf[];
  __shared__ uint64_t bars[kMaxPieces];
  __shared__ int abort_flag;
  __shared__ int ids[kMaxList];
  __shared__ double q_sum[2];
  __shared__ float q_max[2];
  __shared__ int q_any[2];
  __shared__ float2 parts[kWarps], slot[kMaxCluster];  // {maximum, sum} of the tail, of warps and CTAs
  __shared__ float list_z[kMaxList];                   // the list's logits, in every CTA
  const int rank = cluster_rank();
  const uint32_t n_ctas = cluster_ctas();
  const int64_t r = blockIdx.x / n_ctas;
  const T* row = static_cast<const T*>(p.logits) + r * p.ld;
  const Slice<T> sl(row, p.vocab, rank, n_ctas);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float w = p.weight ? p.weight[r] : 1.f;

  auto nothing = [&] {  // a row that counts for nothing: loss and gradient 0
    if constexpr (kGrad) {
      write_grad<T, G>(sl, static_cast<G*>(p.grad) + r * p.ld_grad, threadIdx.x, kThreads, [](int, float* f) {
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] = 0.f;
      });
    }
    if (rank == 0 && threadIdx.x == 0) p.loss[r] = 0.f;
  };
  if (w == 0.f) {  // the logits are not read
    nothing();
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i * kPiece < sl.nv; ++i) mbar_init(&bars[i], 1);
    fence_mbar_init();
    fence_proxy_async_smem();
    abort_flag = 0;
    start_copies(sl, buf, bars);
  }
  fill_ends(sl, buf);
  // the list: one thread an entry; a token's first place counts, what is no token is left out
  int id = -1;
  float lq = 0.f, q = 0.f;
  if (threadIdx.x < kMaxList) {
    if (threadIdx.x < p.k) {
      id = p.ids[r * p.k + threadIdx.x];
      lq = p.logq[r * p.k + threadIdx.x];
      if (id < 0 || id >= p.vocab) id = -1;
    }
    ids[threadIdx.x] = id;
  }
  __syncthreads();
  if (threadIdx.x < kMaxList) {
    if (id >= 0)
      for (int j = 0; j < static_cast<int>(threadIdx.x); ++j)
        if (ids[j] == id) {
          id = -1;
          break;
        }
    if (id < 0) list_z[threadIdx.x] = -kInf;  // no entry
    q = id >= 0 ? expf(lq) : 0.f;
    __syncwarp();
    const double sum = warp_sum(static_cast<double>(q));
    const int any = __any_sync(0xffffffffu, id >= 0);
    const float top = key_value(__reduce_max_sync(0xffffffffu, order_key(id >= 0 ? lq : -kInf)));
    if (lane == 0) {
      q_sum[warp] = sum;
      q_max[warp] = top;
      q_any[warp] = any;
    }
  }
  __syncthreads();
  cluster_arrive();
  const float q_top = fmaxf(q_max[0], q_max[1]);
  if (!p.bucket && out_of_scale(q_top)) {  // (in every thread of the cluster)
    if (threadIdx.x < kMaxList) {
      lq -= q_top;
      q = id >= 0 ? expf(lq) : 0.f;
      const double sum = warp_sum(static_cast<double>(q));
      if (lane == 0) q_sum[warp] = sum;
    }
    __syncthreads();
  }
  const double Q = q_sum[0] + q_sum[1];
  const bool pulls = (q_any[0] | q_any[1]) && (p.bucket || Q != 0.0);

  // S out of the row
  for (int i = 0; i * kPiece < sl.nv; ++i) wait_piece(bars, i, &abort_flag, p.status, 62);
  cluster_wait();  // every CTA of the cluster runs: its shared memory may be written
  if (!pulls) {    // no token in the list: the whole cluster leaves
    nothing();
    return;
  }
  float z = -kInf;
  const int vec = id >= 0 ? sl.vector_of(id) : -1;
  if (vec >= 0) {
    T* e = reinterpret_cast<T*>(buf + vec) + sl.place_of(id);
    z = to_f(*e);
    *e = neg_inf<T>();
    for (uint32_t i = 0; i < n_ctas; ++i) st_cluster(map_to_rank(smem_u32(&list_z[threadIdx.x]), i), z);
  }
  __syncthreads();

  const float c = p.scale * kLog2e;
  Stat st;
  const uint4 none = no_elements<T>();
  for (int i = 0; i < sl.nv; i += kStep) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = i + u * kThreads + threadIdx.x;
      v[u] = k < sl.nv ? buf[k] : none;
    }
    stat_add<T, kUnroll, false>(st, v, c, 0.f);
  }
  // the tail's sums, over the CTA and the cluster
  const float3 of_warp = warp_stat<T, false>(st, c, threadIdx.x, kThreads, sl.nv, InShared{buf});
  if (lane == 0) parts[warp] = make_float2(of_warp.x, of_warp.y);
  __syncthreads();
  const float2 none_here = make_float2(-kInf, 0.f);
  float2 v = none_here;
  if (n_ctas > 1) {
    if (warp == 0) {
      v = join_parts(lane < kWarps ? parts[lane] : none_here, c);
      if (lane < n_ctas) st_cluster(map_to_rank(smem_u32(&slot[rank]), lane), v);
    }
    __syncwarp();
    cluster_sync();
    if (lane < n_ctas) v = slot[lane];
    else v = none_here;
  } else if (lane < kWarps) {
    v = parts[lane];
  }
  const RowSums sums = sums_with_list(v, list_z[lane], list_z[lane + 32], c);
  const ListSums ls = list_sums(Q, p.bucket);
  const RowScale o = row_scale(sums, ls, w, p.scale, p.bucket, c);
  if constexpr (kGrad) {
    G* grow = static_cast<G*>(p.grad) + r * p.ld_grad;
    write_tail_grad<T, G>(sl, buf, grow, threadIdx.x, kThreads, outside(o, sums, c), c);
    __syncthreads();
    if (vec >= 0) grow[id] = Out<G>::one(ex2_approx(exponent(z, sums.all, o.R, c)) * o.inv_s * o.f_in - q * o.q_in);
  }
  if (rank != 0) return;

  __shared__ float list_q[kMaxList], list_lq[kMaxList];
  if (threadIdx.x < kMaxList) {
    list_q[threadIdx.x] = q;
    list_lq[threadIdx.x] = lq;
  }
  __syncthreads();
  if (warp == 0) {
    const float qs[2] = {list_q[lane], list_q[lane + 32]}, lqs[2] = {list_lq[lane], list_lq[lane + 32]};
    const float zs[2] = {list_z[lane], list_z[lane + 32]};
    const float loss = row_loss(o, sums, ls, w, p.bucket, p.scale, c, qs, lqs, zs);
    if (lane == 0) p.loss[r] = loss;
  }
}

template <typename T, int kThreads>
cudaError_t launch_threads(const DistillArgs& p, int grad_dtype, const Launch& l, cudaStream_t s) {
  const size_t smem = l.slice_bytes;
  if (!p.grad) return launch<&distill_kernel<T, NoGrad, kThreads>>(p.rows, l, smem, s, p);
  if (grad_dtype == SGD_F16) return launch<&distill_kernel<T, f16, kThreads>>(p.rows, l, smem, s, p);
  if (grad_dtype == SGD_BF16) return launch<&distill_kernel<T, bf16, kThreads>>(p.rows, l, smem, s, p);
  return launch<&distill_kernel<T, float, kThreads>>(p.rows, l, smem, s, p);
}
template <typename T>
cudaError_t launch_type(const DistillArgs& p, int grad_dtype, cudaStream_t s) {
  const int64_t row_bytes = static_cast<int64_t>(p.vocab) * sizeof(T);
  if (distill_stream_pays(p.rows, row_bytes, p.grad)) return distill_stream<T>(p, grad_dtype, s);
  Launch l = plan(p.rows, p.vocab, sizeof(T));
  if (p.grad && row_bytes <= kShortGradRow && p.rows * row_bytes >= kManyBytes) l.threads = 64;
  return l.threads == 64 ? launch_threads<T, 64>(p, grad_dtype, l, s) : launch_threads<T, 256>(p, grad_dtype, l, s);
}

}  // namespace

cudaError_t distill_launch(const DistillParams& q, cudaStream_t s) {
  const DistillArgs p{q.logits, q.ld, q.rows, q.vocab, q.scale, q.ids, q.logq, q.k, q.weight, q.tail == SGD_TAIL_BUCKET,
                      q.loss, q.grad, q.ld_grad, device_status_ptr()};
  if (q.dtype == SGD_F16) return launch_type<f16>(p, q.grad_dtype, s);
  if (q.dtype == SGD_BF16) return launch_type<bf16>(p, q.grad_dtype, s);
  return launch_type<float>(p, q.grad_dtype, s);
}

}  // namespace sgd
