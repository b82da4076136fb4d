// Distillation of many long rows (distill.cu has the formulas): the rows stream through clusters that stay
// for the whole call.
//
// A CTA holds slices of several rows in shared memory, a buffer each.  8 warps work on them in turn: the
// sums of one row, then the gradient of an earlier one, whose sums have crossed the cluster meanwhile.
// Each buffer has a warp of its own that sees a row through, one step after another: it starts the bulk
// copies, takes the list's tokens out of the slice (they become -inf), adds up the sums, exchanges them
// with the cluster's other CTAs, gives the gradient its scalars, prepares the next row's list while the
// gradient is written, starts the next copies and writes the list's own gradients.  Once the scalars are there the row
// goes (in the CTA of the cluster whose turn it is) to one of the warps that do the losses.  These steps are chains of latency (a
// few us a row); as many of them as there are buffers run at once, and the 8 warps wait for none of them
// but through the barriers of the buffers.
//
// What a CTA sends to the others alternates between two places per buffer: the second row after a row is
// sent when all CTAs have sent the one between, after they have read the first.
//
// The loss alone keeps a buffer only until the sums are taken: the next row's copies start before they are
// exchanged.  Rows of weight 0 are dealt out to the clusters apart from the others, and a warp of its own
// writes their zeros: in a buffer's turn they would keep it from loading.
//
// Measured (GB300, replayed from a graph over rotating inputs), lists of 32, 126464 fp16 logits a row: 4096 rows
// with a bf16 gradient 341 us = 6.1 TB/s (a copy moves 6.8): the 8 warps are busy for 5.1 of the 5.9 thousand
// clocks of a row (sums 2.6, gradient 2.5), the rest is waiting for copies.  The loss alone, 1024 rows: 63 us
// = 4.1 TB/s: a buffer's chain (copy, list, sums, exchange) over three buffers.  Three slices of 64 KB are what
// an SM holds; clusters of 8 with slices of half the size leave 32 SMs idle (15 of them fit: 495 us).
// Tried at 338 us: 12 working warps 349 us, the next vectors fetched ahead of the sums 356 us, slices copied
// and given free in four pieces 367 us.  The gradient a row later than the next row's sums: no difference.
//
// Every wait is bounded.  After one has expired (recorded in the status word) each warp leaves its loop.
#include "distill.cuh"
#include "persistent.cuh"

namespace sgd {
namespace rows {
namespace {

constexpr int kWorkWarps = 8, kWork = 32 * kWorkWarps;
constexpr int kMinBuffers = 3, kMaxBuffers = 5;
constexpr int kLossWarps = 4;
constexpr int kAllThreads = kWork + 32 * (kMaxBuffers + kLossWarps + 1);  // the last warp: zeros
constexpr int kDeep = 4;
constexpr int kBufferBytes = 200 * 1024;
constexpr int kMaxStreamCluster = 8;
constexpr int kHalves = kMaxList / 32;  // list entries of a lane

struct Buffer {
  uint64_t full;       // the slice has arrived
  uint64_t ready;      // and the list's tokens are out of it
  uint64_t part_full;  // the working warps' sums are there
  uint64_t sums_full[2];  // and those of all CTAs
  uint64_t scaled;     // the gradient's scalars are there
  uint64_t done;       // the gradient is written
  int row;             // -1: no more
  int live;            // 0: loss and gradient are 0
  Outside out;         // of the gradient
  RowSums sums;        // of the row, and its gradient's scalars (as registers they spill: read back behind the copies)
  RowScale scale;
  float2 part[kWorkWarps];
  float4 slot[2][kMaxStreamCluster];
  float list_z[2][kMaxList];  // the list's logits, in the CTA that puts down the loss
  uint64_t loss_full, loss_free;
  __align__(16) int ids[32];
};

// Buffers of `vectors` vectors (a multiple of kWork) each.
struct Shape {
  int vectors, buffers;
};

// A row's list, kHalves entries a lane.
struct List {
  int row;
  bool copied;  // it has a weight
  bool lives;   // and its list a token
  float w;
  int id[kHalves];  // -1: none
  float q[kHalves], lq[kHalves];
  ListSums sums;
};

// What a row's loss is made of, on its way to the warp that does it.
struct LossRow {
  int row;  // -1: no more
  bool lives;
  float w;
  ListSums list;
  RowSums sums;
  float q[kMaxList], lq[kMaxList], z[kMaxList];
};

template <typename T, typename G>
__global__ void __launch_bounds__(kAllThreads, 1) distill_stream_kernel(const DistillArgs p, const Shape shape) {
  constexpr bool kGrad = !std::is_same<G, NoGrad>::value;
  constexpr int E = Elem<T>::kPer;
  extern __shared__ __align__(128) uint4 buf[];
  __shared__ Buffer buffers[kMaxBuffers];
  __shared__ LossRow losses[kMaxBuffers];
  __shared__ int abort_shared;
  __shared__ RowLists rows;
  const int rank = cluster_rank(), n_ctas = cluster_ctas();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &abort_shared;
  if (threadIdx.x < shape.buffers) {
    Buffer& b = buffers[threadIdx.x];
    mbar_init(&b.full, 1);
    mbar_init(&b.ready, 1);
    mbar_init(&b.part_full, kWorkWarps);
    mbar_init(&b.sums_full[0], n_ctas);
    mbar_init(&b.sums_full[1], n_ctas);
    mbar_init(&b.scaled, 1);
    mbar_init(&b.done, kWorkWarps);
    mbar_init(&b.loss_full, 1);
    mbar_init(&b.loss_free, 1);
    fence_mbar_init();
  }
  if (threadIdx.x == 0) abort_shared = 0;
  // behind a slice's vectors its buffer holds -inf: no copy writes there
  const uint4 none = no_elements<T>();
  for (int i = threadIdx.x; i < shape.vectors * shape.buffers; i += kAllThreads) buf[i] = none;
  fence_proxy_async_smem();
  const int cluster = blockIdx.x / n_ctas, clusters = gridDim.x / n_ctas;
  const bool listed = p.weight && make_row_lists<kAllThreads>(rows, p.rows, cluster, clusters, [&](int r) { return p.weight[r] != 0.f; });
  __syncthreads();
  cluster_sync();
  const T* logits = static_cast<const T*>(p.logits);
  const float c = p.scale * kLog2e;
  auto slice_of = [&](int r) { return Slice<T>(logits + r * p.ld, p.vocab, rank, n_ctas); };

  if (warp < kWorkWarps) {
    // ----- sums of a row, gradient of an earlier one
    auto take_sums = [&](int n) {
      Buffer& b = buffers[n];
      if (b.live) {
        const uint4* at = buf + n * shape.vectors + threadIdx.x;
        const int nv = slice_of(b.row).nv;
        int left = (nv + kWork - 1) / kWork;
        Stat st;
        for (; left >= kDeep; left -= kDeep, at += kDeep * kWork) {
          uint4 v[kDeep];
#pragma unroll
          for (int u = 0; u < kDeep; ++u) v[u] = at[u * kWork];
          stat_add<T, kDeep, false>(st, v, c, 0.f);
        }
        for (; left > 0; --left, at += kWork) {
          const uint4 v = *at;
          stat_add<T, 1, false>(st, &v, c, 0.f);
        }
        const float3 w_stat = warp_stat<T, false>(st, c, threadIdx.x, kWork, nv, InShared{buf + n * shape.vectors});
        if (lane == 0) b.part[warp] = make_float2(w_stat.x, w_stat.y);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.part_full);
    };
    auto put_gradient = [&](int n, uint32_t phase) {  // false: a wait has expired
      if constexpr (kGrad) {
        Buffer& b = buffers[n];
        if (!mbar_wait_warp(smem_u32(&b.scaled), phase, abort_flag, p.status, 71)) return false;
        const Slice<T> sl = slice_of(b.row);
        G* grow = static_cast<G*>(p.grad) + b.row * p.ld_grad;
        if (b.live) {
          write_tail_grad<T, G>(sl, buf + n * shape.vectors, grow, threadIdx.x, kWork, b.out, c);
        } else {
          write_grad<T, G>(sl, grow, threadIdx.x, kWork, [](int, float* f) {
#pragma unroll
            for (int j = 0; j < E; ++j) f[j] = 0.f;
          });
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.done);
      }
      return true;
    };
    uint32_t over = 0, phase = 0;      // buffers without further rows
    int n = 0, late = -1;              // the buffer of the row whose gradient is still to be written
    uint32_t late_phase = 0;
    bool ok = true;
    auto catch_up = [&]() {
      if (late >= 0) ok = put_gradient(late, late_phase);
      late = -1;
    };
    while (ok && over != (1u << shape.buffers) - 1u) {
      if (!(over >> n & 1)) {
        // (near the end of the rows the other buffers may have none: this one's next row waits for its gradient)
        if (late == n) catch_up();
        ok = ok && mbar_wait_warp(smem_u32(&buffers[n].ready), phase, abort_flag, p.status, 70);
        if (!ok) break;
        if (buffers[n].row < 0) {
          over |= 1u << n;
        } else {
          take_sums(n);
          if (kGrad) {
            catch_up();
            late = n;
            late_phase = phase;
          }
        }
      }
      if (++n == shape.buffers) {
        n = 0;
        phase ^= 1;
      }
    }
    if (ok) catch_up();
  } else if (warp >= kWorkWarps + kMaxBuffers && warp < kWorkWarps + kMaxBuffers + kLossWarps) {
    // ----- losses: of the buffers first, first + kLossWarps, ... in turn, as the working warps go through them
    const int first = warp - kWorkWarps - kMaxBuffers;
    uint32_t all = 0, over = 0, phases = 0;
    for (int n = first; n < shape.buffers; n += kLossWarps) all |= 1u << n;
    for (int n = first; over != all; n = n + kLossWarps < shape.buffers ? n + kLossWarps : first) {
      if (over >> n & 1) continue;
      Buffer& b = buffers[n];
      if (!mbar_wait_warp(smem_u32(&b.loss_full), phases >> n & 1, abort_flag, p.status, 77)) break;
      phases ^= 1u << n;
      const LossRow& x = losses[n];
      const int row = x.row;
      if (row < 0) {
        over |= 1u << n;
        continue;
      }
      float loss = 0.f;
      if (x.lives) {
        float q[kHalves], lq[kHalves], z[kHalves];
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          q[h] = x.q[lane + 32 * h];
          lq[h] = x.lq[lane + 32 * h];
          z[h] = x.z[lane + 32 * h];
        }
        const RowSums sums = x.sums;
        const ListSums list = x.list;
        loss = row_loss(row_scale(sums, list, x.w, p.scale, p.bucket, c), sums, list, x.w, p.bucket, p.scale, c, q, lq, z);
      }
      if (lane == 0) p.loss[row] = loss;
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.loss_free);
    }
  } else if (warp == kWorkWarps + kMaxBuffers + kLossWarps) {
    // ----- rows of weight 0
    for (int i = 0; listed && i < rows.n_rest; ++i) {
      const int r = rows.of_rest[i];
      if constexpr (kGrad)
        write_grad<T, G>(slice_of(r), static_cast<G*>(p.grad) + r * p.ld_grad, lane, 32, [](int, float* f) {
#pragma unroll
          for (int j = 0; j < E; ++j) f[j] = 0.f;
        });
      if (rank == 0 && lane == 0) p.loss[r] = 0.f;
    }
  } else if (warp - kWorkWarps < shape.buffers) {
    // ----- one buffer's rows
    const int n = warp - kWorkWarps;
    Buffer& b = buffers[n];
    uint4* slice = buf + n * shape.vectors;
    int turn = n;  // of the cluster's rows
    auto next_row = [&]() {
      const int i = turn;
      turn += shape.buffers;
      if (listed) return i < rows.n_first ? rows.of_first[i] : -1;
      const int64_t r = cluster + static_cast<int64_t>(i) * clusters;
      return r < p.rows ? static_cast<int>(r) : -1;
    };
    // the next row's list as it is in memory; used later
    auto fetch_list = [&]() {
      List x;
      x.row = next_row();
      x.w = 1.f;
      if (x.row >= 0 && p.weight) x.w = p.weight[x.row];
      x.copied = x.row >= 0 && x.w != 0.f;
      x.lives = false;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const int i = lane + 32 * h;
        const int64_t at = static_cast<int64_t>(x.row) * p.k + i;
        x.id[h] = x.copied && i < p.k ? p.ids[at] : -1;
        x.lq[h] = x.copied && i < p.k ? p.logq[at] : 0.f;
      }
      return x;
    };
    // an id counts at its first place; what is no token is left out
    auto sort_out = [&](List& x) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        if (x.id[h] < 0 || x.id[h] >= p.vocab) x.id[h] = -1;
        if (lane != __ffs(__match_any_sync(0xffffffffu, x.id[h])) - 1) x.id[h] = -1;
        if (32 * (h + 1) >= p.k) break;  // (the other halves hold no id)
        if (h + 1 < kHalves) b.ids[lane] = x.id[h];
      }
      if (p.k > 32) {
        static_assert(kHalves == 2, "the second half is compared with the first");
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const int4 o = *reinterpret_cast<const int4*>(&b.ids[j]);
          if (x.id[1] == o.x || x.id[1] == o.y || x.id[1] == o.z || x.id[1] == o.w) x.id[1] = -1;
        }
        __syncwarp();
      }
      uint32_t key = kKeyNegInf;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) key = max(key, x.id[h] >= 0 ? order_key(x.lq[h]) : kKeyNegInf);
      const float top = key_value(__reduce_max_sync(0xffffffffu, key));
      if (!p.bucket && out_of_scale(top)) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) x.lq[h] -= top;
      }
      double sum = 0.0;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        x.q[h] = x.id[h] >= 0 ? expf(x.lq[h]) : 0.f;
        sum += x.q[h];
      }
      const double Q = warp_sum(sum);
      bool any = false;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) any |= x.id[h] >= 0;
      x.sums = list_sums(Q, p.bucket);
      x.lives = __any_sync(0xffffffffu, any) && x.copied && (p.bucket || Q != 0.0);
    };

    List x = fetch_list(), old;  // of the row to come, and of the one in the buffer
    old.row = -1;
    float z[kHalves] = {-kInf, -kInf};
    int vec[kHalves] = {-1, -1};
    int place = 0;  // of what the others send
    int owner = 0;  // the CTA that puts down the loss of the buffer's row: each in turn
    uint32_t full_phase = 0, phase = 0, sums_phase = 0;
    // the old row's sums across the cluster, and its scalars; false: a wait has expired
    auto exchange = [&]() {
      const float2 v = lane < kWorkWarps ? b.part[lane] : make_float2(-kInf, 0.f);
      const float m = key_value(__reduce_max_sync(0xffffffffu, order_key(v.x)));
      const float m_list = key_value(__reduce_max_sync(0xffffffffu, max(order_key(z[0]), order_key(z[1]))));
      const float R_list = reference(m_list, c);
      float tail = v.y, unused = 0.f, in = 0.f;
      rebase(v.x, c, m, reference(m, c), tail, unused);
#pragma unroll
      for (int h = 0; h < kHalves; ++h) in += vec[h] >= 0 ? ex2_approx(exponent(z[h], m_list, R_list, c)) : 0.f;
      tail = warp_sum(tail);
      in = warp_sum(in);
      RowSums sums;
      if (n_ctas == 1) {
        sums = join_sums(m, tail, m_list, in, c);
      } else {
        if (lane < n_ctas) st_cluster(map_to_rank(smem_u32(&b.slot[place][rank]), lane), make_float4(m, tail, m_list, in));
        __syncwarp();
        if (lane < n_ctas) mbar_arrive_cluster(map_to_rank(smem_u32(&b.sums_full[place]), lane));
        __syncwarp();
        if (!wait_cluster(&b.sums_full[place], sums_phase, abort_flag, p.status, 74)) return false;
        sums = row_sums(b.slot[place], n_ctas, c);
      }
      if (lane == 0) b.sums = sums;
      if constexpr (kGrad) {
        const RowScale scale = row_scale(sums, old.sums, old.w, p.scale, p.bucket, c);
        if (lane == 0) {
          b.scale = scale;
          b.out = outside(scale, sums, c);
        }
      }
      __syncwarp();
      return true;
    };
    // the old row to the warp that does the losses, once that is done with this buffer's last one
    uint32_t loss_phase = 0;
    auto send_loss = [&](int row) {
      if (!mbar_wait_warp(smem_u32(&b.loss_free), loss_phase ^ 1u, abort_flag, p.status, 76)) return false;
      loss_phase ^= 1;
      LossRow& l = losses[n];
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const int i = lane + 32 * h;
        l.q[i] = old.q[h];
        l.lq[i] = old.lq[h];
        l.z[i] = row >= 0 && old.lives && old.id[h] >= 0 ? b.list_z[place][i] : -kInf;
      }
      if (lane == 0) {
        l.row = row;
        l.lives = old.lives;
        l.w = old.w;
        l.list = old.sums;
        l.sums = b.sums;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.loss_full);
      return true;
    };
    for (;; phase ^= 1) {
      const Slice<T> sl = slice_of(max(x.row, 0));
      if (lane == 0) {
        b.row = x.row;
        if (x.copied) {
          const char* src = reinterpret_cast<const char*>(sl.row + sl.first_element(0));
          const int lo = sl.nv > 0 && !sl.whole(0) ? 1 : 0;
          const int hi = sl.nv > 0 && !sl.whole(sl.nv - 1) ? sl.nv - 1 : sl.nv;
          const uint32_t bytes = hi > lo ? (hi - lo) * 16u : 0u;
          mbar_arrive_expect_tx(&b.full, bytes);
          for (int a = lo; a < hi; a += kPiece)
            bulk_load(slice + a, src + static_cast<int64_t>(a) * 16, min(kPiece, hi - a) * 16u, &b.full);
        }
      }
      __syncwarp();
      bool ok = true;
      if (old.row < 0) {
        sort_out(x);  // (of the first row: its copies are under way; the others' lists are ready before)
      } else {  // what is left of the old row
        if (old.lives) {
          if constexpr (kGrad) {
            const RowScale& scale = b.scale;
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
              if (vec[h] >= 0)
                (static_cast<G*>(p.grad) + old.row * p.ld_grad)[old.id[h]] =
                    Out<G>::one(ex2_approx(exponent(z[h], b.sums.all, scale.R, c)) * scale.inv_s * scale.f_in - old.q[h] * scale.q_in);
          } else {
            ok = exchange();
          }
        }
        if (!kGrad && ok && rank == owner) ok = send_loss(old.row);
        owner = owner + 1 == n_ctas ? 0 : owner + 1;
        if (old.lives) {
          place ^= 1;
          sums_phase ^= place == 0;
        }
      }
      if (ok && x.row < 0) {
        if (lane == 0) mbar_arrive(&b.ready);
        send_loss(-1);
        break;
      }
      old = x;
      x = fetch_list();
      if (old.copied) {
        // the row's ragged ends, and what lies behind the slice (rows that start elsewhere in a vector have a
        // few vectors more or less in it)
        const bool ragged = lane < 2 * E && sl.nv > 0 && !(lane >= E && sl.nv == 1) && !sl.whole(lane < E ? 0 : sl.nv - 1);
        const int e = sl.first_element(lane < E ? 0 : sl.nv - 1) + lane % E;
        T end = neg_inf<T>();
        if (ragged && e >= 0 && e < sl.vocab) end = sl.row[e];
        if (!mbar_wait_warp(smem_u32(&b.full), full_phase, abort_flag, p.status, 72)) {
          mbar_drain(&b.full, full_phase);  // no copy may land after the CTA has left
          break;
        }
        full_phase ^= 1;
        if (ragged) reinterpret_cast<T*>(slice + (lane < E ? 0 : sl.nv - 1))[lane % E] = end;
        if (lane <= kMaxStreamCluster && sl.nv + lane < shape.vectors) slice[sl.nv + lane] = none;
        __syncwarp();
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          z[h] = -kInf;
          // (of a row that lives alone: the others' sums cross the cluster for no other, so that nothing would order
          // a write to list_z for it against the writes for later rows)
          vec[h] = old.lives && old.id[h] >= 0 ? sl.vector_of(old.id[h]) : -1;
          if (vec[h] >= 0) {
            T* at = reinterpret_cast<T*>(slice + vec[h]) + sl.place_of(old.id[h]);
            z[h] = to_f(*at);
            *at = neg_inf<T>();
            st_cluster(map_to_rank(smem_u32(&b.list_z[place][lane + 32 * h]), owner), z[h]);
          }
        }
        fence_proxy_async_smem();
      }
      if (!ok) break;
      if (lane == 0) b.live = old.lives;
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.ready);
      if (!kGrad) sort_out(x);
      if (!mbar_wait_warp(smem_u32(&b.part_full), phase, abort_flag, p.status, 73)) break;
      if constexpr (kGrad) {
        if (old.lives && !exchange()) break;
        if (lane == 0) mbar_arrive(&b.scaled);
        if (rank == owner && !send_loss(old.row)) break;  // (while the gradient is written)
        sort_out(x);
        if (!mbar_wait_warp(smem_u32(&b.done), phase, abort_flag, p.status, 75)) break;
      }
    }
  }
  __syncwarp();
  cluster_sync();  // no CTA leaves while another may still write to it
}

// Vectors of a buffer for rows of these bytes over c CTAs (one more where a row starts inside one).
int buffer_vectors(int64_t row_bytes, int c) {
  const int64_t total = (row_bytes + 15) / 16 + 1, per = (total + c - 1) / c;
  return static_cast<int>((per + kWork - 1) / kWork * kWork);
}

template <typename T, typename G>
cudaError_t launch_stream(const DistillArgs& p, cudaStream_t s) {
  const int64_t bytes = static_cast<int64_t>(p.vocab) * sizeof(T);
  auto buffers = [&](int c) { return kBufferBytes / (16 * buffer_vectors(bytes, c)); };
  int least = 1;
  while (least < kMaxStreamCluster && buffers(least) < kMinBuffers) least *= 2;
  constexpr auto kKernel = &distill_stream_kernel<T, G>;
  Clusters l;
  const cudaError_t e = choose_clusters<kKernel>(p.rows, least, kMaxStreamCluster, kAllThreads, kBufferBytes, &l);
  if (e != cudaSuccess) return e;
  Shape shape;
  shape.vectors = buffer_vectors(bytes, l.size);
  shape.buffers = buffers(l.size) < kMaxBuffers ? buffers(l.size) : kMaxBuffers;
  return launch_clusters<kKernel>(l, kAllThreads, static_cast<size_t>(shape.buffers) * shape.vectors * 16, s, p, shape);
}
static_assert(kBufferBytes + kMaxBuffers * (sizeof(Buffer) + sizeof(LossRow)) + sizeof(RowLists) <= 226 * 1024, "a CTA's shared memory");

}  // namespace

// Streaming against a cluster per row, us, the loss / with a bf16 gradient, fp16 logits:
//   row       32 MB                 64 MB                  128 MB                   512 MB
//   253 KB    17 / 21, 18 / 22      23 / 33, 27 / 39       35 / 54, 46 / 68         107 / 175, 160 / 231
//   64 KB     17 / 26, 18 / 22      21 / 33, 28 / 38       31 / 54, 48 / 67         90 / 172, 168 / 232
//   32 KB     16 / 25, 18 / 21      23 / 45, 32 / 42       36 / 82, 57 / 76         113 / 296, 208 / 284
//   16 KB     18 / 38, 29 / 32      29 / 72, 50 / 60       48 / 138, 100 / 116      166 / 532, 377 / 435
//   8.4 KB    28 / 67, 48 / 54      48 / 130, 90 / 104     89 / 254, 180 / 201      329 / 994, 704 / 783
// with 256 threads a row.  With 64 threads, 64 and 512 MB: 253 KB 30 / 47, 179 / 278; 64 KB 31 / 47, 180 / 275; 32 KB 28 / 41,
// 161 / 231; 16 KB 30 / 41, 198 / 259; 8.4 KB 49 / 60, 351 / 423.  So gradients of rows of up to 32 KB take 64 threads a row
// (of the stream's time there a third is the loss warps' code beside the working warps' in the instruction cache), losses
// alone stream from 8 KB on; below that 64 threads win the gradients and cost the losses little (4 KB, 512 MB: 675 / 765
// against 608 / 1791).
bool distill_stream_pays(int rows, int64_t row_bytes, bool grad) {
  return row_bytes > (grad ? kShortGradRow : 16 * kShortSlice) && rows * row_bytes >= kManyBytes &&
         kBufferBytes / (16 * static_cast<int64_t>(buffer_vectors(row_bytes, kMaxStreamCluster))) >= kMinBuffers;
}

template <typename T>
cudaError_t distill_stream(const DistillArgs& p, int grad_dtype, cudaStream_t s) {
  if (!p.grad) return launch_stream<T, NoGrad>(p, s);
  if (grad_dtype == SGD_F16) return launch_stream<T, f16>(p, s);
  if (grad_dtype == SGD_BF16) return launch_stream<T, bf16>(p, s);
  return launch_stream<T, float>(p, s);
}
template cudaError_t distill_stream<f16>(const DistillArgs&, int, cudaStream_t);
template cudaError_t distill_stream<bf16>(const DistillArgs&, int, cudaStream_t);
template cudaError_t distill_stream<float>(const DistillArgs&, int, cudaStream_t);

}  // namespace rows
}  // namespace sgd
