// Distillation of rows of logits from another model's likeliest tokens: loss and gradient.
//
// p = softmax(scale z).  A row's list gives q_i = e^(lq_i) for the tokens of a set S, Q = sum q_i:
//   renorm: q^_i = q_i / Q,          L = sum q^_i (ln q^_i - ln p_i),
//           dL/dz_j = scale (p_j - q^_j);
//   bucket: q_T = 1 - Q, p_T = sum_{j not in S} p_j,
//           L = sum q_i (ln q_i - ln p_i) + q_T (ln q_T - ln p_T),
//           dL/dz_j = scale (p_j - q_j) in S,  scale p_j (1 - q_T / p_T) outside.
// The row is held in shared memory (vocab_rows.cuh), so that it is read once for both the loss and the
// gradient: 2 passes over it on chip, sizeof(logit) + sizeof(gradient) bytes per token in HBM.
//
// S is taken out of the row (its values are replaced by -inf in shared memory) before the sum, so
// that p_T is a sum of its own: 1 - sum_S p would leave nothing of a small tail.  In the gradient's
// pass -inf gives S the gradient 0, and its k entries are written after it.
//
// The loss is a difference of larger terms where the two models agree, so that the scalars of a row
// are kept apart: its terms are summed in fp64, 1 - Q is taken of the fp64 sum of the rounded
// q_i (their rounding then cancels to first order), and ln p_T is ln(1 - P) by log1p.
#include <type_traits>

#include "vocab_rows.cuh"

namespace sgd {
namespace {

using namespace rows;

constexpr int kMaxList = kMaxTop;
static_assert(kMaxList == 64, "two warps hold the list");

struct Params {
  const void* logits;
  int64_t ld;
  int vocab;
  float scale;
  const int32_t* ids;
  const float* logq;
  int k;
  const float* weight;
  int bucket;
  float* loss;
  void* grad;
  int64_t ld_grad;
  int* status;
};

struct NoGrad {};

template <typename G>
struct Out;
template <>
struct Out<float> {
  __device__ static float one(float x) { return x; }
};
template <>
struct Out<f16> {  // rounded as they are: a gradient out of fp16's range is inf, as a loss scaler expects
  __device__ static f16 one(float x) { return __float2half_rn(x); }
};
template <>
struct Out<bf16> {
  __device__ static bf16 one(float x) { return __float2bfloat16_rn(x); }
};

// N values to an address aligned to N sizeof(G) (at most 16) bytes
template <int N>
__device__ __forceinline__ void store_vec(float* to, const float* f) {
#pragma unroll
  for (int i = 0; i < N; i += 4) reinterpret_cast<float4*>(to)[i / 4] = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
}
template <int N>
__device__ __forceinline__ void store_words(void* to, const uint32_t* w) {
  if constexpr (N == 8) *static_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
  else *static_cast<uint2*>(to) = make_uint2(w[0], w[1]);
}
template <int N>
__device__ __forceinline__ void store_vec(bf16* to, const float* f) {
  uint32_t w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  store_words<N>(to, w);
}
template <int N>
__device__ __forceinline__ void store_vec(f16* to, const float* f) {
  uint32_t w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  store_words<N>(to, w);
}

// The slice's part of a gradient row: value(f) of the logits' vector f, stored whole where the
// address allows it.
template <typename T, typename G, typename F>
__device__ __forceinline__ void write_grad(const Slice<T>& sl, const uint4* buf, G* grow, const F& value) {
  constexpr int E = Elem<T>::kPer;
  constexpr uintptr_t kAlign = E * sizeof(G) < 16 ? E * sizeof(G) : 16;
  G* g0 = grow - sl.shift;
  const bool aligned = (reinterpret_cast<uintptr_t>(g0) & (kAlign - 1)) == 0;
  for (int i = threadIdx.x; i < sl.nv; i += kThreads) {
    float f[E];
    value(i, f);
    const int e = sl.first_element(i);
    G* to = grow + e;
    if (aligned && sl.whole(i)) {
      store_vec<E>(to, f);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (e + j >= 0 && e + j < sl.vocab) to[j] = Out<G>::one(f[j]);
    }
  }
}

template <typename T, typename G>
__global__ void __launch_bounds__(kThreads, 3) distill_kernel(const Params p) {
  constexpr bool kGrad = !std::is_same<G, NoGrad>::value;
  constexpr int E = Elem<T>::kPer;
  extern __shared__ __align__(128) uint4 buf[];
  __shared__ uint64_t bars[kMaxPieces];
  __shared__ int abort_flag;
  __shared__ int ids[kMaxList];
  __shared__ double q_sum[2];
  __shared__ int q_any[2];
  __shared__ float4 warp_stat[kWarps];
  __shared__ float4 slot[kMaxCluster];
  __shared__ float list_z[kMaxList];  // leader: the list's logits
  __shared__ double loss_sum[2];
  const int rank = cluster_rank();
  const uint32_t n_ctas = cluster_ctas();
  const int64_t r = blockIdx.x / n_ctas;
  const T* row = static_cast<const T*>(p.logits) + r * p.ld;
  const Slice<T> sl(row, p.vocab, rank, n_ctas);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float w = p.weight ? p.weight[r] : 1.f;

  auto nothing = [&] {  // a row that counts for nothing: loss and gradient 0
    if constexpr (kGrad) {
      write_grad<T, G>(sl, buf, static_cast<G*>(p.grad) + r * p.ld_grad, [](int, float* f) {
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
    q = id >= 0 ? expf(lq) : 0.f;
    __syncwarp();
    const double sum = warp_sum(static_cast<double>(q));
    const int any = __any_sync(0xffffffffu, id >= 0);
    if (lane == 0) {
      q_sum[warp] = sum;
      q_any[warp] = any;
    }
  }
  __syncthreads();
  cluster_arrive();
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
    st_cluster(map_to_rank(smem_u32(&list_z[threadIdx.x]), 0), z);
  }
  __syncthreads();

  const float c = p.scale * kLog2e;
  Stat st;
  const uint4 none = no_elements<T>();
  for (int i = 0; i < sl.nv; i += kPiece) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = i + u * kThreads + threadIdx.x;
      v[u] = k < sl.nv ? buf[k] : none;
    }
    stat_add<T, kUnroll, false>(st, v, c);
  }
  // the CTA's sums, of the tail and of its part of S
  float m = key_value(__reduce_max_sync(0xffffffffu, max(order_key(st.m), order_key(z))));
  {
    const float R = reference(m, c);
    float s = st.s, unused = 0.f;
    rebase(st.m, c, R, s, unused);
    float in = vec >= 0 ? ex2_approx(fmaf(z, c, -R)) : 0.f;
    s = warp_sum(s);
    in = warp_sum(in);
    if (lane == 0) warp_stat[warp] = make_float4(m, s, in, 0.f);
  }
  __syncthreads();
  if (warp == 0) {
    float4 v = lane < kWarps ? warp_stat[lane] : make_float4(-kInf, 0.f, 0.f, 0.f);
    m = key_value(__reduce_max_sync(0xffffffffu, order_key(v.x)));
    const float R = reference(m, c);
    float unused = 0.f;
    rebase(v.x, c, R, v.y, unused);
    rebase(v.x, c, R, v.z, unused);
    v.y = warp_sum(v.y);
    v.z = warp_sum(v.z);
    if (lane < n_ctas) st_cluster(map_to_rank(smem_u32(&slot[rank]), lane), make_float4(m, v.y, v.z, 0.f));
  }
  __syncwarp();
  cluster_sync();

  // the row's sums
  float all = -kInf;
  for (uint32_t i = 0; i < n_ctas; ++i) all = fmaxf(all, slot[i].x);
  const float R = reference(all, c);
  float tail = 0.f, in = 0.f, unused = 0.f;
  for (uint32_t i = 0; i < n_ctas; ++i) {
    float4 v = slot[i];
    rebase(v.x, c, R, v.y, unused);
    rebase(v.x, c, R, v.z, unused);
    tail += v.y;
    in += v.z;
  }
  const float s = tail + in;
  const bool empty = all == -kInf && s == 0.f;  // every logit -inf: p = 0
  const float inv_s = empty ? 0.f : 1.f / s;
  const double q_tail = p.bucket ? fmax(0.0, 1.0 - Q) : 0.0;
  const bool has_tail = p.bucket && tail > 0.f;

  if constexpr (kGrad) {
    const float f_in = w * p.scale, q_in = p.bucket ? f_in : static_cast<float>(f_in / Q);
    // p_j (1 - q_T / p_T) = 2^y (1 / s - q_T / tail); finite apart from f_in: tail >= 2^-126
    const float f_out = inv_s - (has_tail ? static_cast<float>(q_tail) / tail : 0.f);
    G* grow = static_cast<G*>(p.grad) + r * p.ld_grad;
    const uint64_t c2 = pack_f32x2(c, c), r2 = pack_f32x2(-R, -R);
    write_grad<T, G>(sl, buf, grow, [&](int i, float* f) {
      unpack(buf[i], f, static_cast<const T*>(nullptr));
#pragma unroll
      for (int j = 0; j < E; j += 2) {
        const uint64_t y = fma_f32x2(pack_f32x2(f[j], f[j + 1]), c2, r2);
        f[j] = f_in * (f_out * ex2_approx(lo_f32x2(y)));
        f[j + 1] = f_in * (f_out * ex2_approx(hi_f32x2(y)));
      }
    });
    __syncthreads();
    if (vec >= 0) grow[id] = Out<G>::one(ex2_approx(fmaf(z, c, -R)) * inv_s * f_in - q * q_in);
  }
  if (rank != 0) return;

  if (threadIdx.x < kMaxList) {
    double term = 0.0;
    if (q != 0.f) {  // (a NaN too)
      const float delta = all == -kInf ? 0.f : fmaf(all, c, -R);
      int e = 0;
      const float f = frexpf(s, &e);  // ln s without the rounding of a large sum's logarithm
      const double ln_s = static_cast<double>(logf(f)) + (e - static_cast<double>(delta)) * 0.6931471805599453;
      const double ln_p = empty ? -HUGE_VAL : (static_cast<double>(list_z[threadIdx.x]) - all) * p.scale - ln_s;
      term = q * (lq - ln_p);
    }
    term = warp_sum(term);
    if (lane == 0) loss_sum[warp] = term;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double L = loss_sum[0] + loss_sum[1];
    if (!p.bucket) {
      int e = 0;
      const float f = frexpf(static_cast<float>(Q), &e);
      L = L / Q - (static_cast<double>(logf(f)) + e * 0.6931471805599453);
    } else if (has_tail && q_tail > 0.0) {
      const float P = in / s;
      const float ln_pt = P < 0.5f ? log1pf(-P) : logf(tail / s);
      const float ln_qt = Q < 0.5 ? log1pf(-static_cast<float>(Q)) : logf(static_cast<float>(q_tail));
      L += q_tail * (static_cast<double>(ln_qt) - ln_pt);
    }
    p.loss[r] = static_cast<float>(w * L);
  }
}

template <typename T>
cudaError_t launch_grad(const Params& p, const DistillParams& q, const Launch& l, size_t smem, cudaStream_t s) {
  if (!q.grad) return launch<&distill_kernel<T, NoGrad>>(q.rows, l, smem, s, p);
  if (q.grad_dtype == SGD_F16) return launch<&distill_kernel<T, f16>>(q.rows, l, smem, s, p);
  if (q.grad_dtype == SGD_BF16) return launch<&distill_kernel<T, bf16>>(q.rows, l, smem, s, p);
  return launch<&distill_kernel<T, float>>(q.rows, l, smem, s, p);
}

}  // namespace

cudaError_t distill_launch(const DistillParams& q, cudaStream_t s) {
  const Launch l = plan(q.rows, q.vocab, q.dtype == SGD_F32 ? 4 : 2);
  const Params p{q.logits, q.ld, q.vocab, q.scale, q.ids, q.logq, q.k, q.weight, q.tail == SGD_TAIL_BUCKET, q.loss,
                 q.grad, q.ld_grad, device_status_ptr()};
  const size_t smem = l.slice_bytes;
  if (q.dtype == SGD_F16) return launch_grad<f16>(p, q, l, smem, s);
  if (q.dtype == SGD_BF16) return launch_grad<bf16>(p, q, l, smem, s);
  return launch_grad<float>(p, q, l, smem, s);
}

}  // namespace sgd
