// A token drawn from each row of logits: temperature, top-k, min-p and top-p, from two given random numbers.
//
// With x = scale z, w_i = e^(x_i - max x), and the tokens in the order (z descending, index ascending):
//   K1 = the first top_k of the order that have w_i >= min_p;  K = the shortest prefix of K1 with a mass (sum of w)
//   of at least top_p times K1's.
// The vocabulary is cut into blocks of 512 tokens.  The first block whose cumulative mass (of K alone) is above
// u0 mass(K) is drawn, then the first token in it whose cumulative mass is above u1 mass(block).
//
// Why two steps: one fp32 number has 24 bits, too few for a tail of 126464 tokens.  And why blocks: a border between tokens
// moves with every rounding of the sum before it, so that a draw among 1e5 tokens by fp32 sums is another token than by exact
// ones once in a hundred rows.  A block's border is met with 500 times less often, so that fp32 sums do unless the number
// falls within their error of a border, which is seen, and the masses are taken anew; inside a block, and where a cut is
// looked for, masses are whole numbers (weight() below): their sums have no error and no order.
//
// A row is read once from HBM: warps take blocks and leave their maxima and, where masses are needed, their sums of
// exponentials against the maximum (kError below).  What comes after looks, from L2, only at blocks whose maximum reaches
// a bound zl that the cut cannot be below:
//   top-k: the k-th largest of the blocks' maxima, for large k a quantile of a sample of the row;  min-p: max + ln(min_p) / scale;
//   top-p alone: the 64th largest of the maxima where the maxima above it already have the mass; else from the sample (one token of 8
//   in a histogram of its weights), which also gives a bound zh that the cut is not above.  What is above zh is summed, what lies
//   between is listed; if the cut is not in between after all (counts and sums tell), the whole row is searched.
// The cut is found in the list, or the row, by histograms of counts and masses over the order's integers, 1024 bins at a time,
// down to 256 tokens, which are ranked by comparing all with all.
//
// Many rows: a CTA each, three per SM, so that one's search hides behind the others' reading.  Few: a cluster reads a row.
#include "sample.cuh"

namespace sgd {
namespace {

using namespace rows;

constexpr int kSampled = 16384;  // rows from this many tokens on are sampled
constexpr int kShort = 4;          // blocks of a row that 64 threads take
constexpr int kQueue = 64;       // tokens of a block that a warp puts side by side

// Adds a mass to one in shared memory that others add to as well (two 32-bit additions: whole numbers have no order).
__device__ __forceinline__ void add_shared(uint32_t* lo, uint32_t* hi, uint64_t w) {
  const uint32_t low = static_cast<uint32_t>(w), was = atomicAdd(lo, low);
  const uint32_t high = static_cast<uint32_t>(w >> 32) + (was + low < was);
  if (high) atomicAdd(hi, high);
}

template <int kThreads>
struct __align__(16) Shared {
  static constexpr int kWarps = kThreads / 32;
  static constexpr int kCap = 16 * kThreads;  // tokens of the list
  static constexpr int kHist = 4 * kThreads;  // bins
  uint64_t list[kCap];
  uint32_t count[kHist], lo[kHist], hi[kHist];
  uint64_t small[kThreads], small_w[kThreads];
  uint64_t queue[kWarps][kQueue];
  uint64_t pow2[32];
  uint64_t wide[2][kWarps];
  float part[kWarps];
  uint32_t part_n[kWarps];
  uint32_t groups[kThreads];
  uint64_t best;
  uint64_t cut, cut_before, cut_upto;
  uint64_t above_w;
  uint32_t above_n, bin_n, bin;
  int n, found, bad;
  int edge[4];
  uint32_t edge_n[2];
};

struct Cut {
  uint64_t place;         // of the last token that is kept
  uint64_t before, upto;  // the kept mass without it and with it
};

template <typename T, bool VEC, int kThreads>
struct Row {
  using Sh = Shared<kThreads>;
  static constexpr int kWarps = kThreads / 32, kSmall = kThreads, kCap = Sh::kCap, kHist = Sh::kHist;
  static constexpr int kBinBits = kThreads == 256 ? 10 : 8;
  static_assert(kHist == 1 << kBinBits, "bins");
  const SampleArgs& a;
  const T* row;
  const float* max_of;  // [n_blocks] maxima
  uint64_t* mass;       // [n_blocks]
  Sh& sh;
  float m;              // the row's maximum
  int warp, lane;

  __device__ __forceinline__ uint64_t w_of(float z) const { return weight(z, m, a, sh.pow2); }

  // f(b, its tokens) for the blocks whose maximum is at least `least`, a warp each, with the next one's tokens on their way
  template <typename F>
  __device__ __forceinline__ void blocks(float least, F f) const {
    auto next = [&](int b) {
      while (b < a.n_blocks && !(max_of[b] >= least)) b += kWarps;
      return b;
    };
    int b = next(warp);
    if (b >= a.n_blocks) return;
    Raw<T> raw = fetch<T, VEC>(row, a.p.vocab, b, lane);
    while (b < a.n_blocks) {
      const int after = next(b + kWarps);
      Raw<T> ahead;
      if (after < a.n_blocks) ahead = fetch<T, VEC>(row, a.p.vocab, after, lane);
      f(b, raw);
      raw = ahead;
      b = after;
    }
  }
  // f(place, value) for the tokens of a block that are marked in `on` (bit j: the lane's token j), side by side in the lanes where they
  // are few, else one of each lane at a time
  template <typename F>
  __device__ __forceinline__ void marked(int b, const float* z, uint32_t on, F f) const {
    const int mine = __popc(on);
    int up = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, up, o);
      if (lane >= o) up += x;
    }
    const int all = __shfl_sync(0xffffffffu, up, 31);
    if (all == 0) return;
    if (all <= kQueue) {
      int at = up - mine;
      if (on) {
#pragma unroll
        for (int j = 0; j < kPerLane; ++j)
          if (on >> j & 1) sh.queue[warp][at++] = place(order_key(z[j]), token_at<T, VEC>(b, lane, j));
      }
      __syncwarp();
      for (int i = lane; i < all; i += 32) f(sh.queue[warp][i], value_of(sh.queue[warp][i]));
      __syncwarp();
      return;
    }
#pragma unroll 1
    while (__any_sync(0xffffffffu, on)) {
      if (on) {
        const int e = token_at<T, VEC>(b, lane, __ffs(on) - 1);
        on &= on - 1;
        if (e < a.p.vocab) {
          const float x = to_f(row[e]);
          f(place(order_key(x), e), x);
        }
      }
      __syncwarp();
    }
  }
  // f(place, value) for the row's tokens at or before `from` in the order
  template <typename F>
  __device__ __forceinline__ void each(uint64_t from, F f) const {
    const float least = value_of(from);
    blocks(least, [&](int b, const Raw<T>& raw) {
      float z[kPerLane];
      numbers(raw, z);
      uint32_t on = 0;
#pragma unroll
      for (int j = 0; j < kPerLane; ++j) on |= (z[j] >= least && token_at<T, VEC>(b, lane, j) < a.p.vocab ? 1u : 0u) << j;
      marked(b, z, on, [&](uint64_t x, float y) {
        if (x >= from) f(x, y);
      });
    });
  }

  // Sums over the CTA; a barrier before and after.
  __device__ ulonglong2 cta_sum(uint64_t v, uint64_t w) const {
    v = warp_sum_u64(v);
    w = warp_sum_u64(w);
    __syncthreads();
    if (lane == 0) {
      sh.wide[0][warp] = v;
      sh.wide[1][warp] = w;
    }
    __syncthreads();
    ulonglong2 s = make_ulonglong2(0, 0);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      s.x += sh.wide[0][i];
      s.y += sh.wide[1][i];
    }
    return s;
  }
  __device__ uint64_t cta_sum(uint64_t v) const { return cta_sum(v, 0).x; }

  // Place in a list of n counted so far (one atomic for the lanes that are here).
  __device__ __forceinline__ int slot(int* n) const {
    const uint32_t here = __activemask();
    const int first = __ffs(here) - 1;
    int at = 0;
    if (lane == first) at = atomicAdd(n, __popc(here));
    return __shfl_sync(here, at, first) + __popc(here & ((1u << lane) - 1u));
  }

  struct Rest {
    uint64_t above, tail, error;
  };
  // Tokens above zh: their masses by blocks, and in rest->above together; those from zl to zh: into the list, as far as it goes; with
  // TAIL those below: their mass from fp32 sums, and how far it may be off (`mass` holds the blocks' masses at the call).
  // Returns how many are from zl to zh.
  template <bool TAIL>
  __device__ int bracket(float zl, float zh, Rest* rest) const {
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    uint64_t above = 0, tail = 0, skipped = 0;
    for (int b = threadIdx.x; b < a.n_blocks; b += kThreads)
      if (!(max_of[b] >= zl)) {
        if (TAIL) skipped += mass[b];
        mass[b] = 0;
      }
    blocks(zl, [&](int b, const Raw<T>& raw) {
      float z[kPerLane];
      numbers(raw, z);
      uint32_t on = 0;
      float low[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kPerLane; ++j) {
        const bool is = z[j] >= zl;
        on |= (is ? 1u : 0u) << j;
        if (TAIL) low[j & 1] += is ? 0.f : ex2_approx(__fmul_rn(z[j] - zl, a.c));
      }
      if (zl == -kInf)  // (what is no token is -inf)
#pragma unroll
        for (int j = 0; j < kPerLane; ++j)
          if (token_at<T, VEC>(b, lane, j) >= a.p.vocab) on &= ~(1u << j);
      uint64_t s = 0;
      marked(b, z, on, [&](uint64_t x, float y) {
        if (y > zh) {
          s += w_of(y);
        } else {
          const int at = slot(&sh.n);
          if (at < kCap) sh.list[at] = x;
        }
      });
      if (__any_sync(0xffffffffu, s != 0)) s = warp_sum_u64(s);
      const float l = TAIL ? warp_sum(low[0] + low[1]) : 0.f;
      if (lane == 0) {
        mass[b] = s;
        above += s;
        if (TAIL) tail += block_mass(zl, l, m, a, sh.pow2);
      }
    });
    const ulonglong2 both = cta_sum(above, tail);
    rest->above = both.x;
    if (TAIL) {
      // of the tail's sums against zl: 18 u, and three roundings of an exponent t whose mean over the mass S (of zl's weight) is at
      // most log2(vocab) - log2(S); and tokens below 2^-43
      skipped = cta_sum(skipped);
      const float s = static_cast<float>(both.y), spread = s > 0.f ? log2f(a.p.vocab * (static_cast<float>(w_of(zl)) + 1.f) / s) : 0.f;
      rest->tail = both.y + skipped;
      rest->error = static_cast<uint64_t>(a.n_blocks) + a.p.vocab +
                    __double2ull_ru(kError * static_cast<double>(skipped) +
                                    (20.0 + 2.1 * fmaxf(spread, 0.f)) * 5.9604645e-8 * static_cast<double>(both.y));
    }
    return sh.n;
  }

  // Masses of the blocks, of the tokens at or before `cut` in the order; returns the whole.
  __device__ uint64_t masses(uint64_t cut) const {
    const float least = value_of(cut);
    uint64_t all = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < a.n_blocks; b += kThreads)
      if (!(max_of[b] >= least)) mass[b] = 0;
    blocks(least, [&](int b, const Raw<T>& raw) {
      const uint64_t s = warp_sum_u64(raw_mass<T, VEC>(raw, b, lane, a.p.vocab, cut, m, a, sh.pow2));
      if (lane == 0) {
        mass[b] = s;
        all += s;
      }
    });
    return cta_sum(all);
  }
  // Adds the list's tokens that are kept to the blocks' masses.
  __device__ void add_list(int n, uint64_t cut) const {
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const uint64_t x = sh.list[i];
      if (x < cut) continue;
      uint32_t* to = reinterpret_cast<uint32_t*>(mass + index_of(x) / kBlock);
      add_shared(to, to + 1, w_of(value_of(x)));
    }
    __syncthreads();
  }

  // Where a cut is looked for: the list, or the row.
  struct List {
    static constexpr bool kRow = false;
    const Row& r;
    int n;
    template <typename F>
    __device__ __forceinline__ void each(uint64_t from, F f) const {
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t x = r.sh.list[i];
        if (x >= from) f(x, value_of(x));
      }
    }
  };
  struct Whole {
    static constexpr bool kRow = true;
    const Row& r;
    template <typename F>
    __device__ __forceinline__ void each(uint64_t from, F f) const {
      r.each(from, f);
    }
  };
  __device__ uint64_t sum_of_list(int n, uint64_t from) const {
    uint64_t s = 0;
    List{*this, n}.each(from, [&](uint64_t, float z) { s += w_of(z); });
    return cta_sum(s);
  }

  // The last token of the shortest prefix of the order, among the tokens of src with places lo .. hi (n at most) and those above them (above_n
  // tokens with the mass above_w), that has `count` tokens or (count 0) a mass of at least `target`.
  template <typename S>
  __device__ Cut find_cut(const S& src, int n, uint64_t lo, uint64_t hi, uint32_t count, uint64_t target, uint32_t above_n,
                          uint64_t above_w) const {
    while (n > kSmall) {
      const int shift = max(0, 64 - __clzll(hi - lo) - kBinBits);
      __syncthreads();
      for (int i = threadIdx.x; i < kHist; i += kThreads) sh.count[i] = sh.lo[i] = sh.hi[i] = 0;
      __syncthreads();
      src.each(lo, [&](uint64_t x, float z) {
        if (x > hi) return;
        const uint32_t bin = static_cast<uint32_t>((hi - x) >> shift);
        atomicAdd(&sh.count[bin], 1u);
        add_shared(&sh.lo[bin], &sh.hi[bin], w_of(z));
      });
      __syncthreads();
      pick_bin(count, target, above_n, above_w);
      above_n = sh.above_n;
      above_w = sh.above_w;
      n = sh.bin_n;
      hi -= static_cast<uint64_t>(sh.bin) << shift;
      const uint64_t width = (1ull << shift) - 1ull;
      if (hi - lo > width) lo = hi - width;
      if constexpr (S::kRow) {
        if (n <= kCap && n > kSmall) {
          gather(src, lo, hi, sh.list, kCap);
          return find_cut(List{*this, n}, n, lo, hi, count, target, above_n, above_w);
        }
      }
    }
    gather(src, lo, hi, sh.small, kSmall);
    n = sh.n;
    const int t = threadIdx.x;
    const uint64_t x = t < n ? sh.small[t] : 0;
    const uint64_t w = t < n ? w_of(value_of(x)) : 0;
    sh.small_w[t] = w;
    if (t == 0) sh.cut = 0;
    __syncthreads();
    uint32_t rank = above_n;
    uint64_t cum = above_w;
    if (t < n)
      for (int i = 0; i < n; ++i)
        if (sh.small[i] >= x) {
          ++rank;
          cum += sh.small_w[i];
        }
    // (where rounding leaves none, the last one)
    const bool it = t < n && (count ? rank == count : cum >= target && cum - w < target);
    auto write = [&] {
      sh.cut = x;
      sh.cut_before = cum - w;
      sh.cut_upto = cum;
    };
    if (it) write();
    __syncthreads();
    const bool none = sh.cut == 0;
    __syncthreads();
    if (none && t < n && rank == above_n + n) write();
    __syncthreads();
    const Cut cut{sh.cut, sh.cut_before, sh.cut_upto};
    __syncthreads();
    return cut;
  }
  template <typename S>
  __device__ void gather(const S& src, uint64_t lo, uint64_t hi, uint64_t* to, int cap) const {
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    src.each(lo, [&](uint64_t x, float) {
      if (x > hi) return;
      const int at = slot(&sh.n);
      if (at < cap) to[at] = x;
    });
    __syncthreads();
  }
  // The histogram's first bin with which the target is reached (where rounding leaves none, the last one that holds anything),
  // and what is above it.
  __device__ void pick_bin(uint32_t count, uint64_t target, uint32_t above_n, uint64_t above_w) const {
    if (warp == 0) {
      constexpr int kPer = kHist / 32;  // neighbouring bins of a lane
      uint32_t n = 0;
      uint64_t w = 0;
      for (int j = 0; j < kPer; ++j) {
        const int i = lane * kPer + j;
        n += sh.count[i];
        w += static_cast<uint64_t>(sh.hi[i]) << 32 | sh.lo[i];
      }
      uint32_t before_n = n;
      uint64_t before_w = above_w + warp_scan_u64(w, lane) - w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, before_n, o);
        if (lane >= o) before_n += x;
      }
      before_n += above_n - n;
      auto reached = [&](uint32_t cn, uint64_t cw) { return count ? cn >= count : cw >= target; };
      const uint32_t lanes = __ballot_sync(0xffffffffu, n > 0 && reached(before_n + n, before_w + w));
      const uint32_t held = __ballot_sync(0xffffffffu, n > 0);
      const int which = lanes ? __ffs(lanes) - 1 : 31 - __clz(held);
      if (lane == which) {
        for (int j = 0; j < kPer; ++j) {
          const int i = lane * kPer + j;
          const uint32_t cn = sh.count[i];
          if (cn == 0) continue;
          sh.bin = i;
          sh.bin_n = cn;
          sh.above_n = before_n;
          sh.above_w = before_w;
          before_n += cn;
          before_w += static_cast<uint64_t>(sh.hi[i]) << 32 | sh.lo[i];
          if (reached(before_n, before_w)) break;
        }
      }
    }
    __syncthreads();
  }

  // Key of the k-th largest of kThreads groups' maxima (k <= kThreads): at least k tokens have it or more.
  __device__ uint32_t bound_of_k(int k) const {
    float g = -kInf;
    for (int b = threadIdx.x; b < a.n_blocks; b += kThreads) g = fmaxf(g, max_of[b]);
    const uint32_t mine = order_key(g);
    sh.groups[threadIdx.x] = mine;
    __syncthreads();
    int more = 0;
#pragma unroll 4
    for (int i = 0; i < kThreads; i += 4) {
      const uint4 x = *reinterpret_cast<const uint4*>(sh.groups + i);
      const int t = threadIdx.x;
      more += (x.x > mine || (x.x == mine && i < t)) + (x.y > mine || (x.y == mine && i + 1 < t)) +
              (x.z > mine || (x.z == mine && i + 2 < t)) + (x.w > mine || (x.w == mine && i + 3 < t));
    }
    if (more == k - 1) sh.above_n = mine;
    __syncthreads();
    const uint32_t key = sh.above_n;
    __syncthreads();
    return key;
  }

  // Weights of a sample of the row, one token of 8 or more, in runs of 8: count[i] of those in the i-th 1/32 of an octave from the
  // maximum down.  Returns how many were looked at.
  __device__ int sampled() const {
    const int vocab = a.p.vocab, runs = max(4, (vocab / 8 + 8 * kThreads - 1) / (8 * kThreads));  // of a thread
    __syncthreads();
    for (int i = threadIdx.x; i < kHist; i += kThreads) sh.count[i] = 0;
    if (threadIdx.x < 2) sh.edge[threadIdx.x] = kHist;
    __syncthreads();
    const int64_t all = static_cast<int64_t>(runs) * kThreads;
    for (int k = 0; k < runs; ++k) {
      int e = static_cast<int>((static_cast<int64_t>(k) * kThreads + threadIdx.x) * (vocab - 8) / all);
      float z[8];
      if (VEC) {
        e &= ~7;
#pragma unroll
        for (int i = 0; i < 8 / Elem<T>::kPer; ++i)
          unpack(reinterpret_cast<const uint4*>(row + e)[i], z + i * Elem<T>::kPer, static_cast<const T*>(nullptr));
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = to_f(row[e + j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) atomicAdd(&sh.count[static_cast<int>(fminf((m - z[j]) * a.c * 32.f, kHist - 1.f))], 1u);
    }
    __syncthreads();
    return static_cast<int>(8 * all);
  }
  // A value that about 1.3 k + 400 tokens reach, from the sample.
  __device__ float sampled_bound_of_k(int k) const {
    constexpr int kPer = kHist / kThreads;
    const int looked = sampled();
    uint32_t n[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) n[j] = sum += sh.count[threadIdx.x * kPer + j];
    uint32_t up = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, up, o);
      if (lane >= o) up += x;
    }
    if (lane == 31) sh.part_n[warp] = up;
    __syncthreads();
    up -= sum;
    for (int i = 0; i < warp; ++i) up += sh.part_n[i];
    const double want = (1.3 * k + 400.0) * looked / a.p.vocab;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (up + n[j] >= want) atomicMin(&sh.edge[0], static_cast<int>(threadIdx.x) * kPer + j + 1);
    __syncthreads();
    const int edge = sh.edge[0];
    return edge >= kHist ? -kInf : m - edge / (32.f * a.c);
  }
  // Bounds {zl, zh} on the cut by mass, from the sample: tokens below the cut have the mass `share` (of the maximum's weight)
  // together.  Nothing is lost where they are wrong but time.
  __device__ float2 sampled_bounds(double share) const {
    constexpr int kPer = kHist / kThreads;  // bins of a thread
    const int looked = sampled();
    // from the low end: tokens in a thread's bins and below, and their mass
    uint32_t n[kPer + 1];
    float f[kPer + 1];
    n[kPer] = 0;
    f[kPer] = 0.f;
#pragma unroll
    for (int j = kPer - 1; j >= 0; --j) {
      const int i = threadIdx.x * kPer + j;
      n[j] = n[j + 1] + sh.count[i];
      f[j] = f[j + 1] + sh.count[i] * ex2_approx(-(i + 0.5f) / 32.f);
    }
    uint32_t up_n = n[0];
    float up_f = f[0];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_down_sync(0xffffffffu, up_n, o);
      const float y = __shfl_down_sync(0xffffffffu, up_f, o);
      if (lane + o < 32) {
        up_n += x;
        up_f += y;
      }
    }
    if (lane == 0) {
      sh.part_n[warp] = up_n;
      sh.part[warp] = up_f;
    }
    __syncthreads();
    up_n -= n[0];
    up_f -= f[0];
    for (int i = warp + 1; i < kWarps; ++i) {
      up_n += sh.part_n[i];
      up_f += sh.part[i];
    }
    const float want = static_cast<float>(share * looked / a.p.vocab);
    // edge 0: the first bin below which (and with it) there is less than 0.95 of the mass; edge 1: 1.05
#pragma unroll
    for (int j = kPer - 1; j >= 0; --j) {
      const float here = f[j] + up_f;
      const int i = threadIdx.x * kPer + j;
      if (here <= 0.95f * want) atomicMin(&sh.edge[0], i);
      if (here <= 1.05f * want) atomicMin(&sh.edge[1], i);
    }
    __syncthreads();
    const int low = sh.edge[0], high = sh.edge[1];
    // 64 sampled tokens more below, 32 above: 800 of the row, which the list has room for
    if (threadIdx.x == 0) {
      sh.edge[2] = kHist;
      sh.edge[3] = 0;
      sh.edge_n[0] = sh.edge_n[1] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      if (i == low) sh.edge_n[0] = n[j] + up_n;
      if (i == high) sh.edge_n[1] = n[j] + up_n;
    }
    __syncthreads();
    const uint32_t n_low = sh.edge_n[0], n_high = sh.edge_n[1];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      if (n_low >= 64 && n[j] + up_n <= n_low - 64) atomicMin(&sh.edge[2], i);
      if (n[j] + up_n >= n_high + 32) atomicMax(&sh.edge[3], i);
    }
    __syncthreads();
    const int zl = sh.edge[2], zh = sh.edge[3];
    __syncthreads();
    return make_float2(zl >= kHist ? -kInf : m - zl / (32.f * a.c), zh <= 0 ? kInf : m - zh / (32.f * a.c));
  }
};

template <typename T, bool VEC, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? 3 : 12) sample_kernel(const SampleArgs a) {
  constexpr int kWarps = kThreads / 32;
  using Sh = Shared<kThreads>;
  extern __shared__ __align__(16) unsigned char dynamic[];  // Shared, then [n_blocks] masses and maxima
  Sh& sh = *reinterpret_cast<Sh*>(dynamic);
  const SampleParams& p = a.p;
  uint64_t* mass = reinterpret_cast<uint64_t*>(dynamic + sizeof(Sh));
  float* max_of = reinterpret_cast<float*>(mass + a.n_blocks);
  const int rank = cluster_rank(), n_ctas = cluster_ctas();
  const int64_t r = blockIdx.x / n_ctas;
  if (p.row_ids && p.row_ids[r] != p.row_id) return;  // the whole cluster
  const T* row = static_cast<const T*>(p.logits) + r * p.ld;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (n_ctas > 1) cluster_arrive();
  const bool by_k = p.top_k > 0 && p.top_k < p.vocab, by_m = a.drop != -HUGE_VAL, by_p = p.top_p < 1.0;
  const bool sums = p.logprobs || !(by_k || by_m);
  const float u0 = p.uniforms[2 * r], u1 = p.uniforms[2 * r + 1];
  {
    // two blocks of 16-bit logits, or one of fp32, in hand and as many on their way
    constexpr int kPair = sizeof(T) == 2 ? 2 : 1;
    const int stride = kWarps * n_ctas;
    int b = warp * n_ctas + rank;
    Raw<T> next[kPair];
#pragma unroll
    for (int u = 0; u < kPair; ++u)
      if (b + u * stride < a.n_blocks) next[u] = fetch<T, VEC>(row, p.vocab, b + u * stride, lane);
    if (threadIdx.x < 32) sh.pow2[threadIdx.x] = kPow2[threadIdx.x];
    if (threadIdx.x == 0) {
      sh.bad = 0;
      sh.best = 0;
    }
    const uint32_t to_max = map_to_rank(smem_u32(max_of), 0), to_mass = map_to_rank(smem_u32(mass), 0);
    if (n_ctas > 1) cluster_wait();  // every CTA of the cluster runs: the leader's shared memory may be written
    for (; b < a.n_blocks; b += kPair * stride) {
      Raw<T> cur[kPair];
#pragma unroll
      for (int u = 0; u < kPair; ++u) {
        cur[u] = next[u];
        if (b + (kPair + u) * stride < a.n_blocks) next[u] = fetch<T, VEC>(row, p.vocab, b + (kPair + u) * stride, lane);
      }
      const float2 st = block_stats<T, kPair>(cur, sums, a.c, lane);
      const int at = kPair == 2 && lane >= 16 ? b + stride : b;
      if ((lane == 0 || (kPair == 2 && lane == 16)) && at < a.n_blocks) {
        if (n_ctas == 1) {
          max_of[at] = st.x;
          mass[at] = __float_as_uint(st.y);
        } else {
          st_cluster(to_max + 4 * at, st.x);
          st_cluster(to_mass + 8 * at, static_cast<uint64_t>(__float_as_uint(st.y)));
        }
      }
    }
  }
  if (n_ctas > 1) {
    __syncwarp();
    cluster_sync();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }

  // the row's maximum
  float m = -kInf;
  bool bad = false;
  for (int b = threadIdx.x; b < a.n_blocks; b += kThreads) {
    const float x = max_of[b];
    bad |= x != x;
    m = fmaxf(m, x);
  }
  m = key_value(__reduce_max_sync(0xffffffffu, order_key(m)));
  if (lane == 0) sh.part[warp] = m;
  if (bad) sh.bad = 1;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWarps; ++i) m = fmaxf(m, sh.part[i]);
  if (sh.bad || m == -kInf) {
    // no distribution: the first token of the order
    const uint64_t first = first_of_order(row, p.vocab, threadIdx.x, kThreads);
    if (lane == 0) atomicMax(reinterpret_cast<unsigned long long*>(&sh.best), static_cast<unsigned long long>(first));
    __syncthreads();
    if (threadIdx.x == 0) {
      p.ids[r] = index_of(sh.best);
      if (p.logprobs) p.logprobs[r] = sh.bad ? kNan : -kInf;
    }
    return;
  }

  using R = Row<T, VEC, kThreads>;
  const R t{a, row, max_of, mass, sh, m, warp, lane};
  // masses of whole blocks from their fp32 sums, and the row's
  uint64_t whole = 0;
  if (sums) {
    for (int b = threadIdx.x; b < a.n_blocks; b += kThreads) {
      const uint64_t x = block_mass(max_of[b], __uint_as_float(static_cast<uint32_t>(mass[b])), m, a, sh.pow2);
      mass[b] = x;
      whole += x;
    }
    whole = t.cta_sum(whole);
  }

  uint64_t cut = kEverything;
  bool exact = false;
  if (by_k || by_m || by_p) {
    const uint64_t top = static_cast<uint64_t>(order_key(m)) << 32 | 0xFFFFFFFFu;
    float zl = -kInf, zh = kInf;
    if (by_m) zl = __double2float_ru(static_cast<double>(m) + a.drop);
    const float floor_m = zl;
    if (by_k) {
      // (as many groups as there are blocks have a maximum)
      if (p.top_k <= min(a.n_blocks, kThreads)) zl = fmaxf(zl, key_value(t.bound_of_k(p.top_k)));
      else if (p.vocab >= kSampled) zl = fmaxf(zl, t.sampled_bound_of_k(p.top_k));
    }
    if (!by_k && !by_m) {
      // the maxima from the 64th largest on, if they have the mass already
      const uint32_t key = t.bound_of_k(min(64, (a.n_blocks + 3) / 4));
      uint64_t s = 0;
      for (int b = threadIdx.x; b < a.n_blocks; b += kThreads)
        if (order_key(max_of[b]) >= key) s += t.w_of(max_of[b]);
      if (static_cast<double>(t.cta_sum(s)) >= p.top_p * static_cast<double>(whole) * (1.0 + kError)) {
        zl = key_value(key);
      } else if (p.vocab >= kSampled) {
        const float2 z = t.sampled_bounds((1.0 - p.top_p) * static_cast<double>(whole) * (1.0 / (1ull << kOne)));
        zl = z.x;
        zh = z.y;
      } else {
        // tokens below (1 - top_p) Z / vocab have less than the share 1 - top_p together (half a percent aside, for the sums' error)
        const float least = static_cast<float>(0.995 * (1.0 - p.top_p) / p.vocab) * (static_cast<float>(whole) * (1.f / (1ull << kOne)));
        zl = m + logf(least) / p.scale - 1e-6f * fabsf(m);
      }
    }
    zl = fminf(zl, m);
    if (!(zh >= zl)) zh = kInf;
    typename R::Rest rest{};
    const bool alone = !by_k && !by_m;
    int n = alone ? t.template bracket<true>(zl, zh, &rest) : t.template bracket<false>(zl, zh, &rest);
    if (by_k && n < p.top_k && zl > floor_m) {  // the sample misled
      zl = floor_m;
      n = t.template bracket<false>(zl, zh, &rest);
    }
    bool listed = n <= R::kCap;
    const typename R::List list{t, n};
    const typename R::Whole whole_row{t};
    uint64_t lo = static_cast<uint64_t>(order_key(zl)) << 32;
    if (!alone) {
      cut = lo;
      uint64_t kept = 0;
      if (by_k && p.top_k < n) {
        const Cut k = listed ? t.find_cut(list, n, lo, top, p.top_k, 0, 0, 0) : t.find_cut(whole_row, n, lo, top, p.top_k, 0, 0, 0);
        lo = cut = k.place;
        kept = k.upto;
      } else if (by_p) {
        kept = listed ? t.sum_of_list(n, lo) : t.masses(lo);
      }
      if (by_p) {
        const uint64_t target = __double2ull_ru(p.top_p * static_cast<double>(kept));
        // (a search of the row leaves what it found last in the list)
        cut = listed ? t.find_cut(list, n, lo, top, 0, target, 0, 0).place : t.find_cut(whole_row, n, lo, top, 0, target, 0, 0).place;
      }
    } else {
      const uint64_t hi = zh < m ? static_cast<uint64_t>(order_key(zh)) << 32 | 0xFFFFFFFFu : top;
      const uint64_t above = rest.above, upto = listed ? above + t.sum_of_list(n, lo) : above;
      // the row's mass is known but for the error of the tail's
      uint64_t total = upto + rest.tail, error = rest.error;
      for (bool sure = false;; sure = true) {
        const uint64_t target = __double2ull_ru(p.top_p * static_cast<double>(total));
        if (listed && above + error < target && target + error <= upto) {
          const Cut k = t.find_cut(list, n, lo, hi, 0, target, 0, above);
          cut = k.place;
          if (sure || (target > k.before + error && k.upto >= target + error)) break;
        } else if (sure) {
          listed = false;
          cut = t.find_cut(whole_row, p.vocab, kEverything, top, 0, target, 0, 0).place;
          break;
        }
        // within the error of another cut, or not between the bounds: the row's mass anew (the blocks' masses above zh have to be kept)
        uint64_t s = 0;
        t.blocks(-kInf, [&](int b, const Raw<T>& raw) { s += raw_mass<T, VEC>(raw, b, lane, p.vocab, kEverything, m, a, sh.pow2); });
        total = t.cta_sum(s);
        error = 0;
      }
    }
    if (listed) t.add_list(n, cut);
    else t.masses(cut);
    exact = true;
  }

  __syncthreads();
  for (;;) {
    if (warp == 0) {
      const int b = pick_block(mass, a.n_blocks, u0, exact, lane);
      if (b >= 0) draw_token<T, VEC>(a, row, r, b, u1, cut, m, whole, sh.pow2, lane);
      if (lane == 0) sh.found = b;
    }
    if (exact) return;
    __syncthreads();
    if (sh.found >= 0) return;
    t.masses(kEverything);
    exact = true;
  }
}

template <typename T, bool VEC, int kThreads>
cudaError_t launch_rows(const SampleArgs& a, cudaStream_t s) {
  // few rows: a cluster reads a row, down to a block or two per warp
  Launch l{1, 0, kThreads};
  while (l.cluster < kMaxCluster && static_cast<int64_t>(a.p.rows) * l.cluster < num_sms() && a.n_blocks / l.cluster > 8) l.cluster *= 2;
  return launch<&sample_kernel<T, VEC, kThreads>>(a.p.rows, l, sizeof(Shared<kThreads>) + 12 * static_cast<size_t>(a.n_blocks), s, a);
}
template <typename T>
cudaError_t launch_type(const SampleArgs& a, cudaStream_t s) {
  const bool vec = reinterpret_cast<uintptr_t>(a.p.logits) % 16 == 0 && (a.p.rows == 1 || a.p.ld * static_cast<int64_t>(sizeof(T)) % 16 == 0);
  if (a.n_blocks <= kShort) return vec ? launch_rows<T, true, 64>(a, s) : launch_rows<T, false, 64>(a, s);
  return vec ? launch_rows<T, true, 256>(a, s) : launch_rows<T, false, 256>(a, s);
}

}  // namespace

cudaError_t sample_launch(const SampleParams& p, cudaStream_t s) {
  const double c = static_cast<double>(p.scale) * 1.4426950408889634073599;
  SampleArgs a{p, static_cast<float>(c), 0.f, p.min_p > 0.0 ? log(p.min_p) / static_cast<double>(p.scale) : -HUGE_VAL,
               (p.vocab + kBlock - 1) / kBlock, device_status_ptr()};
  a.c_lo = static_cast<float>(c - static_cast<double>(a.c));
  if (p.dtype == SGD_F16) return launch_type<f16>(a, s);
  if (p.dtype == SGD_BF16) return launch_type<bf16>(a, s);
  return launch_type<float>(a, s);
}

}  // namespace sgd
