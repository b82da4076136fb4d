// A token drawn from each row of logits: temperature, top-k, min-p and top-p, from two given random numbers a row.
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
// A row is read once from HBM: warps take a block each and leave its maximum and, where masses are needed, its sum of
// exponentials against that maximum.  What comes after looks again only at blocks whose maximum reaches a bound on the cut
// (the k-th largest of maxima for top-k; max + ln(min_p) / scale; (1 - top_p) Z / vocab for top-p, as all tokens below it have
// less than the share 1 - top_p together), from L2.  What reaches the bound is sorted in shared memory, or, where it is more than
// kCap tokens, narrowed first by histograms (counts and masses) of the order's integers.
//
// Many rows: a CTA each, several per SM, so that one's search hides behind the others' reading.  Few: a cluster reads a row.
#include <math.h>

#include "vocab_rows.cuh"

namespace sgd {
namespace {

using namespace rows;

constexpr int kBlock = SGD_SAMPLE_BLOCK;
constexpr int kPerLane = kBlock / 32;
constexpr int kCap = 1024;   // tokens that are sorted
constexpr int kBinBits = 10;
constexpr int kHist = 1 << kBinBits;
constexpr int kOne = 43;     // weight() of the row's maximum is 2^43: 2^20.6 of them (a row of 3 MiB) add up in 64 bits
static_assert(kBlock == 512, "a lane takes 16 tokens");

struct Args {
  SampleParams p;
  float c, c_lo;    // scale log2(e), as the sum of two floats
  double drop;      // ln(min_p) / scale: a token at or above max + drop passes (-inf: every token)
  int n_blocks;
};

struct __align__(16) Shared {
  uint64_t list[kCap];
  union {
    uint64_t cum[kCap];
    struct {
      uint32_t count[kHist], lo[kHist], hi[kHist];
    };
  };
  uint64_t pow2[32];
  uint64_t wide[32];
  float part[32];
  uint64_t total, best;
  double target;
  int n, found, bad;
  uint64_t cut, above_w, mass;
  uint32_t above_n, bin_n, bin;
  uint32_t groups[256];
};

// 2^(j / 32) 2^62, j = 0 .. 31
__constant__ uint64_t kPow2[32] = {
    0x4000000000000000ull, 0x4166C34C5615D0ECull, 0x42D561B3E6243D8Aull, 0x444C0740496D4294ull,
    0x45CAE0F1F545EB73ull, 0x47521CC5A2E6A9E0ull, 0x48E1E9B9D588E19Bull, 0x4A7A77D47F7B84B1ull,
    0x4C1BF828C6DC54B8ull, 0x4DC69CDCEAA72A9Cull, 0x4F7A993048D088D7ull, 0x513821818624B40Cull,
    0x52FF6B54D8A89C75ull, 0x54D0AD5A753E077Cull, 0x56AC1F752150A563ull, 0x5891FAC0E95612C8ull,
    0x5A827999FCEF3242ull, 0x5C7DD7A3B17DCF75ull, 0x5E8451CFAC061B5Full, 0x6096266533384A2Bull,
    0x62B39508AA836D6Full, 0x64DCDEC3371793D1ull, 0x6712460A8FC24072ull, 0x69540EC8F895722Dull,
    0x6BA27E656B4EB57Aull, 0x6DFDDBCBED791BABull, 0x70666F76154A7089ull, 0x72DC8373BE41A454ull,
    0x75606373EE921C97ull, 0x77F25CCDEE6D7AE6ull, 0x7A92BE8A92436616ull, 0x7D41D96DB915019Dull,
};

// Weight 2^((z - m) c) of a logit against the row's maximum m as a whole number, 2^43 for the maximum: exact to about 2^-31
// relative and half a unit.  z - m = d + dl exactly, (d + dl) c = t + tl to 2^-45; t + tl = n + j / 32 + g with |g| <= 1/64;
// 2^g - 1 = g ln2 + ... to the fourth power (the fifth is 1.3e-12).
__device__ __forceinline__ uint64_t weight(float z, float m, const Args& a, const uint64_t* pow2) {
  const float d = z - m;
  const float t = __fmul_rn(d, a.c);
  if (!(t > -48.f)) return 0;
  const float back = d - z;
  const float dl = (z - (d - back)) + (-m - back);
  const float tl = fmaf(d, a.c, -t) + fmaf(d, a.c_lo, dl * a.c);
  constexpr float kMagic = 393216.f;  // 1.5 2^18: its unit is 1/32
  const float y = __fadd_rn(t, kMagic);
  const int k = __float_as_int(y) - __float_as_int(kMagic);
  const float g = (t - (y - kMagic)) + tl;
  const float e = g * fmaf(g, fmaf(g, fmaf(g, 0.009618129f, 0.05550411f), 0.24022651f), 0.6931472f);
  const uint64_t base = pow2[k & 31];
  const int64_t more = static_cast<int64_t>(static_cast<int32_t>(base >> 32)) * __float2int_rn(e * 4294967296.f);
  const uint64_t w = base + static_cast<uint64_t>(more);  // 2^62 .. 2^63
  const int shift = 62 - kOne - (k >> 5);
  return shift > 62 ? 0 : (w + (1ull << (shift - 1))) >> shift;
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
constexpr uint32_t kKeyFinite = 0xFF7FFFFFu;  // of the largest finite value
constexpr uint32_t kKeyNan = 0xFFFFFFFFu;
constexpr uint64_t kEverything = static_cast<uint64_t>(kKeyNegInf) << 32;  // the place that no token is behind

__device__ __forceinline__ uint64_t warp_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ uint64_t warp_scan_u64(uint64_t v, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// A token's place in the order: larger comes first.
__device__ __forceinline__ uint64_t place(uint32_t key, int i) {
  return static_cast<uint64_t>(key) << 32 | static_cast<uint32_t>(0xFFFFFFFFu - static_cast<uint32_t>(i));
}
__device__ __forceinline__ int index_of(uint64_t place) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(place)); }

// Maximum of a block (NaN where it holds one) and its sum of 2^((z - maximum) c).  VEC: rows start at 16-byte boundaries.
template <typename T, bool VEC>
__device__ __forceinline__ void load_block(const T* row, int vocab, int b, int lane, float* f) {
  const int first = b * kBlock;
  constexpr int E = Elem<T>::kPer;
  if (VEC && first + kBlock <= vocab) {
#pragma unroll
    for (int i = 0; i < kPerLane / E; ++i)
      unpack(reinterpret_cast<const uint4*>(row + first)[i * 32 + lane], f + i * E, static_cast<const T*>(nullptr));
  } else {
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
      const int e = first + j * 32 + lane;
      f[j] = e < vocab ? to_f(row[e]) : -kInf;
    }
  }
}
template <bool SUM>
__device__ __forceinline__ float2 block_stat(const float* f, float c) {
  float m = f[0];
#pragma unroll
  for (int j = 1; j < kPerLane; ++j) m = max_nan(m, f[j]);
  const uint32_t key = __reduce_max_sync(0xffffffffu, m != m ? kKeyNan : order_key(m));
  if (key > kKeyFinite) return make_float2(kNan, kNan);  // NaN or +inf
  m = key_value(key);
  if (!SUM || m == -kInf) return make_float2(m, 0.f);
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) s[j & 3] += ex2_approx(__fmul_rn(f[j] - m, c));
  return make_float2(m, warp_sum((s[0] + s[1]) + (s[2] + s[3])));
}

template <typename T, int kThreads>
struct Row {
  static constexpr int kWarps = kThreads / 32;
  const Args& a;
  const T* row;
  const float* max_of;  // [n_blocks] maxima
  uint64_t* mass;       // [n_blocks]
  Shared& sh;
  float m;              // the row's maximum
  int warp, lane;

  __device__ uint64_t w_of(float z) const { return weight(z, m, a, sh.pow2); }

  // f(key, index, value) for the tokens of blocks whose maximum is at least `least`
  template <typename F>
  __device__ void each(float least, F f) const {
    for (int b = warp; b < a.n_blocks; b += kWarps) {
      if (!(max_of[b] >= least)) continue;
      float z[kPerLane];
#pragma unroll
      for (int j = 0; j < kPerLane; ++j) {
        const int e = b * kBlock + j * 32 + lane;
        z[j] = e < a.p.vocab ? to_f(row[e]) : kNan;
      }
#pragma unroll
      for (int j = 0; j < kPerLane; ++j)
        if (z[j] == z[j]) f(order_key(z[j]), b * kBlock + j * 32 + lane, z[j]);
    }
  }

  // Sum over the CTA; a barrier before and after.
  __device__ uint64_t cta_sum(uint64_t v) const {
    v = warp_sum_u64(v);
    __syncthreads();
    if (lane == 0) sh.wide[warp] = v;
    __syncthreads();
    uint64_t s = 0;
    for (int i = 0; i < kWarps; ++i) s += sh.wide[i];
    return s;
  }

  // Masses of the blocks, of the tokens at or before `cut` in the order.
  __device__ void masses(uint64_t cut) const {
    const float least = key_value(static_cast<uint32_t>(cut >> 32));
    for (int b = warp; b < a.n_blocks; b += kWarps) {
      uint64_t s = 0;
      if (max_of[b] >= least) {
        float z[kPerLane];
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
          const int e = b * kBlock + j * 32 + lane;
          z[j] = e < a.p.vocab ? to_f(row[e]) : -kInf;
        }
#pragma unroll
        for (int j = 0; j < kPerLane; ++j)
          if (place(order_key(z[j]), b * kBlock + j * 32 + lane) >= cut) s += w_of(z[j]);
        s = warp_sum_u64(s);
      }
      if (lane == 0) mass[b] = s;
    }
    __syncthreads();
  }

  // Sorts the n tokens of the list (descending) and leaves the cumulative masses in cum.
  __device__ void sort(int n) const {
    if (n <= kThreads) {
      const uint64_t mine = threadIdx.x < n ? sh.list[threadIdx.x] : 0;
      int before = 0;
      if (threadIdx.x < n)
        for (int i = 0; i < n; ++i) before += sh.list[i] > mine;
      __syncthreads();
      if (threadIdx.x < n) sh.list[before] = mine;
      __syncthreads();
    } else {
      int all = kThreads;
      while (all < n) all *= 2;
      for (int i = n + threadIdx.x; i < all; i += kThreads) sh.list[i] = 0;
      __syncthreads();
      for (int size = 2; size <= all; size *= 2) {
        for (int step = size / 2; step > 0; step /= 2) {
          for (int i = threadIdx.x; i < all / 2; i += kThreads) {
            const int x = 2 * i - (i & (step - 1)), y = x + step;
            const uint64_t p = sh.list[x], q = sh.list[y];
            const bool descending = (x & size) == 0;
            if ((p < q) == descending) {
              sh.list[x] = q;
              sh.list[y] = p;
            }
          }
          __syncthreads();
        }
      }
    }
    // inclusive sums, kCap / kThreads neighbours a thread
    constexpr int kPer = kCap / kThreads;
    uint64_t w[kPer], s = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      s += w[j] = i < n ? w_of(key_value(static_cast<uint32_t>(sh.list[i] >> 32))) : 0;
    }
    const uint64_t up = warp_scan_u64(s, lane);
    if (lane == 31) sh.wide[warp] = up;
    __syncthreads();
    uint64_t run = up - s;
    for (int i = 0; i < warp; ++i) run += sh.wide[i];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      run += w[j];
      if (i < n) sh.cum[i] = run;
    }
    __syncthreads();
  }

  // Tokens with keys lo .. hi into the list; returns how many there are (the list holds the first kCap that came).
  __device__ int gather(uint32_t lo, uint32_t hi) const {
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    each(key_value(lo), [&](uint32_t key, int i, float) {
      if (key >= lo && key <= hi) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < kCap) sh.list[at] = place(key, i);
      }
    });
    __syncthreads();
    return sh.n;
  }

  // Number of the first n cumulative masses (plus `above`) that are below `target`.
  __device__ int below(int n, uint64_t above, double target) const {
    __syncthreads();
    if (threadIdx.x == 0) sh.found = 0;
    __syncthreads();
    int k = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) k += static_cast<double>(above + sh.cum[i]) < target;
    k = __reduce_add_sync(0xffffffffu, k);
    if (lane == 0 && k) atomicAdd(&sh.found, k);
    __syncthreads();
    return sh.found;
  }

  // The last token of the shortest prefix of the order, among the tokens with keys lo .. hi, that has `count` tokens or
  // (count 0) a mass of at least `target`.  *mass_of: the prefix's mass.
  __device__ uint64_t find_cut(uint32_t lo, uint32_t hi, uint32_t count, double target, uint64_t* mass_of) const {
    uint32_t above_n = 0;
    uint64_t above_w = 0;
    for (;;) {
      const int shift = max(0, 32 - __clz(hi - lo) - kBinBits);
      __syncthreads();
      for (int i = threadIdx.x; i < kHist; i += kThreads) sh.count[i] = sh.lo[i] = sh.hi[i] = 0;
      __syncthreads();
      each(key_value(lo), [&](uint32_t key, int, float z) {
        if (key < lo || key > hi) return;
        const uint32_t bin = (hi - key) >> shift;
        const uint64_t w = w_of(z);
        atomicAdd(&sh.count[bin], 1u);
        const uint32_t low = static_cast<uint32_t>(w), was = atomicAdd(&sh.lo[bin], low);
        const uint32_t high = static_cast<uint32_t>(w >> 32) + (was + low < was);
        if (high) atomicAdd(&sh.hi[bin], high);
      });
      __syncthreads();
      if (warp == 0) {  // kHist / 32 neighbouring bins a lane
        constexpr int kPer = kHist / 32;
        uint32_t n = 0;
        uint64_t w = 0;
        for (int j = 0; j < kPer; ++j) {
          const int i = lane * kPer + j;
          n += sh.count[i];
          w += static_cast<uint64_t>(sh.hi[i]) << 32 | sh.lo[i];
        }
        uint32_t before_n = n;
        uint64_t before_w = warp_scan_u64(w, lane) - w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t x = __shfl_up_sync(0xffffffffu, before_n, o);
          if (lane >= o) before_n += x;
        }
        before_n -= n;
        before_n += above_n;
        before_w += above_w;
        auto reached = [&](uint32_t cn, uint64_t cw) { return count ? cn >= count : static_cast<double>(cw) >= target; };
        // the lane where the target is reached; where rounding leaves none, the last one that holds anything
        uint32_t lanes = __ballot_sync(0xffffffffu, n > 0 && reached(before_n + n, before_w + w));
        const uint32_t held = __ballot_sync(0xffffffffu, n > 0);
        const int which = lanes ? __ffs(lanes) - 1 : 31 - __clz(held);
        if (lane == which) {
          int last = 0;
          uint32_t last_n = 0;
          uint64_t last_w = 0;
          for (int j = 0; j < kPer; ++j) {
            const int i = lane * kPer + j;
            const uint32_t cn = sh.count[i];
            const uint64_t cw = static_cast<uint64_t>(sh.hi[i]) << 32 | sh.lo[i];
            if (cn == 0) continue;
            last = i;
            last_n = before_n;
            last_w = before_w;
            before_n += cn;
            before_w += cw;
            if (reached(before_n, before_w)) break;
          }
          sh.bin = last;
          sh.bin_n = sh.count[last];
          sh.above_n = last_n;
          sh.above_w = last_w;
        }
      }
      __syncthreads();
      above_n = sh.above_n;
      above_w = sh.above_w;
      const uint32_t inside = sh.bin_n;
      hi -= sh.bin << shift;
      const uint32_t width = (1u << shift) - 1u;
      lo = hi - lo > width ? hi - width : lo;
      if (inside <= kCap) {
        const int n = gather(lo, hi);
        sort(n);
        int k = count ? static_cast<int>(count - above_n) - 1 : below(n, above_w, target);
        k = min(max(k, 0), n - 1);
        const uint64_t cut = sh.list[k];
        *mass_of = above_w + sh.cum[k];
        __syncthreads();
        return cut;
      }
      if (shift == 0) {  // equal logits alone: the first `take` of them
        const uint64_t w = w_of(key_value(hi));
        uint32_t take;
        if (count) take = count - above_n;
        else if (w == 0) take = inside;
        else {
          const double need = ceil((target - static_cast<double>(above_w)) / static_cast<double>(w));
          take = need >= inside ? inside : static_cast<uint32_t>(max(need, 1.0));
        }
        take = min(max(take, 1u), inside);
        *mass_of = above_w + w * take;
        return place(hi, tie(hi, take));
      }
    }
  }

  // Index of the n-th token (n >= 1) whose key is `key`: counts per block, then inside the block.
  __device__ int tie(uint32_t key, uint32_t n) const {
    const float z = key_value(key);
    for (int b = warp; b < a.n_blocks; b += kWarps) {
      uint32_t k = 0;
      if (max_of[b] >= z)
        for (int j = 0; j < kPerLane; ++j) {
          const int e = b * kBlock + j * 32 + lane;
          if (e < a.p.vocab) k += order_key(to_f(row[e])) == key;
        }
      k = __reduce_add_sync(0xffffffffu, k);
      if (lane == 0) mass[b] = k;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t left = n;
      int b = 0;
      while (b < a.n_blocks - 1 && mass[b] < left) left -= static_cast<uint32_t>(mass[b++]);
      int e = b * kBlock;
      for (; e < a.p.vocab; ++e)
        if (order_key(to_f(row[e])) == key && --left == 0) break;
      sh.found = min(e, a.p.vocab - 1);
    }
    __syncthreads();
    const int at = sh.found;
    __syncthreads();
    return at;
  }

  // Lower bound on the key of the top_k-th token: the k-th largest of 256 groups' maxima.
  __device__ uint32_t bound_of_k(int k) const {
    static_assert(kThreads >= 256, "a thread per group");
    if (k > 256) return 0;
    float g = -kInf;
    if (threadIdx.x < 256) {
      for (int b = threadIdx.x; b < a.n_blocks; b += 256) g = fmaxf(g, max_of[b]);
      sh.groups[threadIdx.x] = order_key(g);
    }
    if (threadIdx.x == 0) sh.found = 0;
    __syncthreads();
    if (threadIdx.x < 256) {
      const uint32_t mine = sh.groups[threadIdx.x];
      int more = 0;
      for (int i = 0; i < 256; ++i) {
        const uint32_t x = sh.groups[i];
        more += x > mine || (x == mine && i < threadIdx.x);
      }
      if (more == k - 1) sh.found = static_cast<int>(mine);
    }
    __syncthreads();
    return static_cast<uint32_t>(sh.found);
  }
};

template <typename T, bool VEC, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) sample_kernel(const Args a) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ __align__(16) unsigned char dynamic[];  // Shared, then [n_blocks] masses and maxima
  Shared& sh = *reinterpret_cast<Shared*>(dynamic);
  const SampleParams& p = a.p;
  uint64_t* mass = reinterpret_cast<uint64_t*>(dynamic + sizeof(Shared));
  float* max_of = reinterpret_cast<float*>(mass + a.n_blocks);
  const int rank = cluster_rank(), n_ctas = cluster_ctas();
  const int64_t r = blockIdx.x / n_ctas;
  if (p.row_ids && p.row_ids[r] != p.row_id) return;  // the whole cluster
  const T* row = static_cast<const T*>(p.logits) + r * p.ld;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  cluster_arrive();
  if (threadIdx.x < 32) sh.pow2[threadIdx.x] = kPow2[threadIdx.x];
  if (threadIdx.x == 0) {
    sh.bad = 0;
    sh.best = 0;
  }
  const bool by_k = p.top_k > 0 && p.top_k < p.vocab, by_m = a.drop != -HUGE_VAL, by_p = p.top_p < 1.0;
  const bool sums = p.logprobs || !(by_k || by_m);
  cluster_wait();  // every CTA of the cluster runs: the leader's shared memory may be written
  {
    const uint32_t to_max = map_to_rank(smem_u32(max_of), 0), to_mass = map_to_rank(smem_u32(mass), 0);
    constexpr int kAhead = 2;
    const int stride = kWarps * n_ctas;
    for (int b = warp * n_ctas + rank; b < a.n_blocks; b += kAhead * stride) {
      float f[kAhead][kPerLane];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (b + u * stride < a.n_blocks) load_block<T, VEC>(row, p.vocab, b + u * stride, lane, f[u]);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int at = b + u * stride;
        if (at >= a.n_blocks) break;
        const float2 s = sums ? block_stat<true>(f[u], a.c) : block_stat<false>(f[u], a.c);
        if (lane == 0) {
          st_cluster(to_max + 4 * at, s.x);
          st_cluster(to_mass + 8 * at, static_cast<uint64_t>(__float_as_uint(s.y)));
        }
      }
    }
  }
  __syncwarp();
  cluster_sync();
  if (rank != 0) return;

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
    uint64_t first = 0;
    bool nan = false;
    for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
      const float z = to_f(row[i]);
      nan |= z != z || z == kInf;
      const uint64_t x = place(order_key(z), i);
      first = x > first ? x : first;
    }
    atomicMax(reinterpret_cast<unsigned long long*>(&sh.best), static_cast<unsigned long long>(first));
    __syncthreads();
    if (threadIdx.x == 0) {
      p.ids[r] = index_of(sh.best);
      if (p.logprobs) p.logprobs[r] = sh.bad ? kNan : -kInf;
    }
    return;
  }

  const Row<T, kThreads> t{a, row, max_of, mass, sh, m, warp, lane};
  // masses of whole blocks from their fp32 sums, and the row's
  uint64_t all = 0;
  if (sums) {
    for (int b = threadIdx.x; b < a.n_blocks; b += kThreads) {
      const float s = __uint_as_float(static_cast<uint32_t>(mass[b]));
      const uint64_t x = max_of[b] == -kInf ? 0 : __double2ull_rn(static_cast<double>(s) * static_cast<double>(t.w_of(max_of[b])));
      mass[b] = x;
      all += x;
    }
    all = t.cta_sum(all);
  }
  const double whole = static_cast<double>(all);

  uint64_t cut = kEverything;
  bool exact = false;
  if (by_k || by_m || by_p) {
    uint32_t lo = kKeyNegInf;
    const uint32_t top = order_key(m);
    if (by_m) lo = max(lo, order_key(__double2float_ru(static_cast<double>(m) + a.drop)));
    if (by_k) lo = max(lo, t.bound_of_k(p.top_k));
    if (!by_k && !by_m) {
      // tokens below (1 - top_p) Z / vocab: together below the share 1 - top_p (half a percent aside, for the sums' error)
      const double least = 0.995 * (1.0 - p.top_p) * (whole * (1.0 / (1ull << kOne))) / p.vocab;
      const float z = m + static_cast<float>(log(least)) / p.scale - 1e-6f * fabsf(m);
      lo = max(lo, order_key(z));
    }
    if (lo > top) lo = top;
    int n = t.gather(lo, top);
    if (n <= kCap) {
      t.sort(n);
      int keep = by_k ? min(p.top_k, n) : n;
      if (by_p) {
        double target = p.top_p * (by_k || by_m ? static_cast<double>(sh.cum[keep - 1]) : whole);
        int k = t.below(keep, 0, target);
        if (!by_k && !by_m) {
          // is the cut another one within the error of the sums?
          const int k0 = t.below(keep, 0, target * (1.0 - 4e-6)), k1 = t.below(keep, 0, target * (1.0 + 4e-6));
          if (k0 != k1) {
            uint64_t w = 0;
            t.each(-kInf, [&](uint32_t, int, float z) { w += t.w_of(z); });
            k = t.below(keep, 0, p.top_p * static_cast<double>(t.cta_sum(w)));
          }
        }
        keep = min(k + 1, keep);
      }
      cut = sh.list[keep - 1];
      __syncthreads();
    } else {
      cut = static_cast<uint64_t>(lo) << 32;
      uint64_t kept = 0;
      const bool cut_k = by_k && p.top_k < n;
      if (cut_k) {
        cut = t.find_cut(lo, top, p.top_k, 0.0, &kept);
        lo = static_cast<uint32_t>(cut >> 32);
      }
      if (by_p) {
        if (!cut_k) {
          const float least = by_k || by_m ? key_value(lo) : -kInf;
          t.each(least, [&](uint32_t, int, float z) {
            if (z >= least) kept += t.w_of(z);
          });
          kept = t.cta_sum(kept);
        }
        uint64_t unused;
        cut = t.find_cut(lo, top, 0, p.top_p * static_cast<double>(kept), &unused);
      }
    }
    __syncthreads();
    t.masses(cut);
    exact = true;
  }

  // the block
  const float u0 = p.uniforms[2 * r], u1 = p.uniforms[2 * r + 1];
  for (;;) {
    __syncthreads();
    if (warp == 0) {
      const int per = (a.n_blocks + 31) / 32, from = min(lane * per, a.n_blocks), to = min(from + per, a.n_blocks);
      uint64_t s = 0;
      for (int b = from; b < to; ++b) s += mass[b];
      const uint64_t up = warp_scan_u64(s, lane), total = __shfl_sync(0xffffffffu, up, 31);
      const double target = static_cast<double>(fminf(fmaxf(u0, 0.f), 1.f)) * static_cast<double>(total);
      const uint32_t above = __ballot_sync(0xffffffffu, s > 0 && static_cast<double>(up) > target), held = __ballot_sync(0xffffffffu, s > 0);
      const int which = above ? __ffs(above) - 1 : 31 - __clz(held);
      if (lane == which) {
        uint64_t before = up - s, cum = before;
        int b = from;
        for (int i = from; i < to; ++i) {
          if (mass[i] == 0) continue;
          b = i;
          before = cum;
          cum += mass[i];
          if (static_cast<double>(cum) > target) break;
        }
        // fp32 sums are off by 37 2^-24 = 2.2e-6 relative at most (a term by 2^-22 and three roundings of its exponent, at most 9 in
        // the mean; 8 sums): a border by half of that of the whole
        const double error = exact ? 0.0 : 1.2e-6 * static_cast<double>(total);
        const bool sure = exact || ((before == 0 || target - static_cast<double>(before) > error) &&
                                    (cum == total || static_cast<double>(cum) - target > error));
        sh.found = sure ? b : -1;
      }
    }
    __syncthreads();
    if (sh.found >= 0) break;
    t.masses(kEverything);
    exact = true;
  }
  if (warp != 0) return;
  // the token: 16 neighbours a lane
  const int first = sh.found * kBlock + lane * kPerLane;
  uint64_t s = 0;
#pragma unroll 4
  for (int j = 0; j < kPerLane; ++j) {
    const float z = first + j < p.vocab ? to_f(row[first + j]) : -kInf;
    if (place(order_key(z), first + j) >= cut) s += t.w_of(z);
  }
  const uint64_t up = warp_scan_u64(s, lane), total = __shfl_sync(0xffffffffu, up, 31);
  const double target = static_cast<double>(fminf(fmaxf(u1, 0.f), 1.f)) * static_cast<double>(total);
  const uint32_t above = __ballot_sync(0xffffffffu, s > 0 && static_cast<double>(up) > target), held = __ballot_sync(0xffffffffu, s > 0);
  const int which = above ? __ffs(above) - 1 : (held ? 31 - __clz(held) : 0);
  if (lane != which) return;
  uint64_t cum = up - s;
  int id = first;
  float z_id = -kInf;
  for (int j = 0; j < kPerLane; ++j) {
    const float z = first + j < p.vocab ? to_f(row[first + j]) : -kInf;
    const uint64_t w = place(order_key(z), first + j) >= cut ? t.w_of(z) : 0;
    if (w == 0) continue;
    id = first + j;
    z_id = z;
    cum += w;
    if (static_cast<double>(cum) > target) break;
  }
  p.ids[r] = id;
  if (p.logprobs) p.logprobs[r] = (z_id - m) * p.scale - logf(static_cast<float>(whole * (1.0 / (1ull << kOne))));
}

template <typename T, bool VEC>
cudaError_t launch_rows(const Args& a, cudaStream_t s) {
  // few rows: a cluster reads a row, down to a block or two per warp
  Launch l{1, 0, 256};
  while (l.cluster < kMaxCluster && static_cast<int64_t>(a.p.rows) * l.cluster < num_sms() && a.n_blocks / l.cluster > 8) l.cluster *= 2;
  return launch<&sample_kernel<T, VEC, 256>>(a.p.rows, l, sizeof(Shared) + 12 * static_cast<size_t>(a.n_blocks), s, a);
}
template <typename T>
cudaError_t launch_type(const Args& a, cudaStream_t s) {
  const bool vec = reinterpret_cast<uintptr_t>(a.p.logits) % 16 == 0 && (a.p.rows == 1 || a.p.ld * static_cast<int64_t>(sizeof(T)) % 16 == 0);
  return vec ? launch_rows<T, true>(a, s) : launch_rows<T, false>(a, s);
}

}  // namespace

cudaError_t sample_launch(const SampleParams& p, cudaStream_t s) {
  const double c = static_cast<double>(p.scale) * 1.4426950408889634073599;
  Args a{p, static_cast<float>(c), 0.f, p.min_p > 0.0 ? log(p.min_p) / static_cast<double>(p.scale) : -HUGE_VAL,
         (p.vocab + kBlock - 1) / kBlock};
  a.c_lo = static_cast<float>(c - static_cast<double>(a.c));
  if (p.dtype == SGD_F16) return launch_type<f16>(a, s);
  if (p.dtype == SGD_BF16) return launch_type<bf16>(a, s);
  return launch_type<float>(a, s);
}

}  // namespace sgd
