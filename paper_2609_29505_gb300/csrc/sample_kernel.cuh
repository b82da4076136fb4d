// The kernel that draws tokens (sample.cu has the definition, and what bounds it), compiled for each type of the logits.
#pragma once

#include <math.h>
#include <stddef.h>

#include "sample.cuh"

namespace sgd {
namespace rows {

constexpr int kBlock = SGD_SAMPLE_BLOCK;
constexpr int kPerLane = kBlock / 32;
// Blocks of a row that 64 threads take, and 128 instead of 256: what a row costs beside its tokens is barriers, and more rows are under way.
// 4096 fp16 rows, every token / top-p 0.9, us: 1000 tokens 64 threads 23 / 54, 128 23 / 75, 256 41 / 142; 2000: 23 / 76 and 41 / 145;
// 4000: 22 / 88 and 40 / 159; 8000: 26 / 131 and 39 / 223.
constexpr int kShortest = 2, kShort = 16;
constexpr int kSampled = 16384;  // rows from this many tokens on are sampled
constexpr int kOne = 43;         // weight() of the row's maximum is 2^43: 2^20.6 of them (a row of 3 MiB) add up in 64 bits
static_assert(kBlock == 512, "a lane takes 16 tokens");

// A block's sum in fp32 is off by at most this much of it (u = 2^-24): a term by 4 u (ex2.approx) and three roundings of its exponent,
// ln2 3 |t| u, whose mean over the block's mass is at most ln2 3 log2(512) u = 18.7 u; 10 u from being added up, 2 u as a
// multiple of 2^-22: 35 u.
constexpr double kError = 2.2e-6;


// 2^(j / 32) 2^62, j = 0 .. 31
static __constant__ uint64_t kPow2[32] = {
    0x4000000000000000ull, 0x4166C34C5615D0ECull, 0x42D561B3E6243D8Aull, 0x444C0740496D4294ull,
    0x45CAE0F1F545EB73ull, 0x47521CC5A2E6A9E0ull, 0x48E1E9B9D588E19Bull, 0x4A7A77D47F7B84B1ull,
    0x4C1BF828C6DC54B8ull, 0x4DC69CDCEAA72A9Cull, 0x4F7A993048D088D7ull, 0x513821818624B40Cull,
    0x52FF6B54D8A89C75ull, 0x54D0AD5A753E077Cull, 0x56AC1F752150A563ull, 0x5891FAC0E95612C8ull,
    0x5A827999FCEF3242ull, 0x5C7DD7A3B17DCF75ull, 0x5E8451CFAC061B5Full, 0x6096266533384A2Bull,
    0x62B39508AA836D6Full, 0x64DCDEC3371793D1ull, 0x6712460A8FC24072ull, 0x69540EC8F895722Dull,
    0x6BA27E656B4EB57Aull, 0x6DFDDBCBED791BABull, 0x70666F76154A7089ull, 0x72DC8373BE41A454ull,
    0x75606373EE921C97ull, 0x77F25CCDEE6D7AE6ull, 0x7A92BE8A92436616ull, 0x7D41D96DB915019Dull,
};

// Weight 2^((z - m) c) of a logit against the row's maximum m as a whole number, 2^43 for the maximum: off by 2^-29
// of itself and half a unit at most.  (Roundings of g, of the polynomial's last sum, of its product and of that as a whole number: at most 1.4, 1, 1
// and 0.25 of 2^-31, and 0.1 of the rest; 2^-29.36 is the most that has been seen.)  (z - m) f = d + dl exactly, (d + dl) c = t + tl to 2^-45; t + tl = n + j / 32 + g with |g| <= 1/64;
// 2^g - 1 = g ln2 + ... to the fourth power (the fifth is 1.3e-12).  (With the factor f = 1 an fma is the difference.)
__device__ __forceinline__ uint64_t weight(float z, float m, const SampleArgs& a, const uint64_t* pow2) {
  const float mf = __fmul_rn(m, a.f), d = fmaf(z, a.f, -mf);
  const float t = __fmul_rn(d, a.c);
  if (!(t > -48.f)) return 0;
  const float back = fmaf(-z, a.f, d);
  const float dl = fmaf(z, a.f, back - d) + (-mf - back);
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
  return shift > 63 ? 0 : (w + (1ull << (shift - 1))) >> shift;
}

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
// The whole number that a mass is above where it is above u total (u as a multiple of 2^-63).
__device__ __forceinline__ uint64_t share_of(float u, uint64_t total) {
  u = fmaxf(u, 0.f);
  return u >= 1.f ? total : __umul64hi(total, __float2ull_rd(u * 9223372036854775808.f) << 1);
}
// The mass s 2^-22 w of a block, s its sum in [1, 512] against its maximum, whose weight is w.
__device__ __forceinline__ uint64_t times(float s, uint64_t w) {
  return __umul64hi(w << 10, static_cast<uint64_t>(__float2uint_rn(s * 4194304.f)) << 32);
}
// Adds a mass to one in shared memory that others add to as well (two 32-bit additions: whole numbers have no order).
__device__ __forceinline__ void add_shared(uint32_t* lo, uint32_t* hi, uint64_t w) {
  const uint32_t low = static_cast<uint32_t>(w), was = atomicAdd(lo, low);
  const uint32_t high = static_cast<uint32_t>(w >> 32) + (was + low < was);
  if (high) atomicAdd(hi, high);
}

// Additions to the shared memory of another CTA of the cluster.
__device__ __forceinline__ void add_cluster(uint32_t to, uint64_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u64 [%0], %1;" ::"r"(to), "l"(v) : "memory");
}
__device__ __forceinline__ int add_cluster(uint32_t to, int v) {
  int was;
  asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(was) : "r"(to), "r"(v) : "memory");
  return was;
}

// A barrier of the kThreads threads that take a row.
template <int kThreads>
__device__ __forceinline__ void team_sync() {
  asm volatile("barrier.cta.sync.aligned 1, %0;" ::"n"(kThreads) : "memory");
}

// A token's place in the order: larger comes first.
__device__ __forceinline__ uint64_t place(uint32_t key, int i) {
  return static_cast<uint64_t>(key) << 32 | static_cast<uint32_t>(0xFFFFFFFFu - static_cast<uint32_t>(i));
}
__device__ __forceinline__ int index_of(uint64_t x) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(x)); }
__device__ __forceinline__ float value_of(uint64_t x) { return key_value(static_cast<uint32_t>(x >> 32)); }

// ----- a block in a warp's registers -----

// VEC: rows start at 16-byte boundaries, and a lane's tokens are those of its vectors; else every 32nd token.
template <typename T, bool VEC>
__device__ __forceinline__ int token_at(int b, int lane, int j) {
  constexpr int E = Elem<T>::kPer;
  return b * kBlock + (VEC ? (j / E * 32 + lane) * E + j % E : j * 32 + lane);
}
template <typename T>
struct Raw {
  static constexpr int kN = kPerLane / Elem<T>::kPer;
  uint4 v[kN];
};
// (no token: -inf)
template <typename T, bool VEC>
__device__ __forceinline__ Raw<T> fetch(const T* row, int vocab, int b, int lane) {
  Raw<T> r;
  if (VEC && (b + 1) * kBlock <= vocab) {
#pragma unroll
    for (int i = 0; i < Raw<T>::kN; ++i) r.v[i] = reinterpret_cast<const uint4*>(row + static_cast<int64_t>(b) * kBlock)[i * 32 + lane];
  } else {
    T* e = reinterpret_cast<T*>(r.v);
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
      const int at = token_at<T, VEC>(b, lane, j);
      e[j] = at < vocab ? row[at] : neg_inf<T>();
    }
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void numbers(const Raw<T>& r, float* z) {
#pragma unroll
  for (int i = 0; i < Raw<T>::kN; ++i) unpack(r.v[i], z + i * Elem<T>::kPer, static_cast<const T*>(nullptr));
}

// Largest value of a lane's tokens; NaN where there is one.
__device__ __forceinline__ float raw_max(const Raw<float>& r) {
  float z[kPerLane];
  numbers(r, z);
  float m = z[0];
#pragma unroll
  for (int j = 1; j + 1 < kPerLane; j += 2) asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(z[j]), "f"(z[j + 1]));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(z[kPerLane - 1]));
  return m;
}
template <typename P, typename T>
__device__ __forceinline__ float packed_max(const Raw<T>& r) {
  const P* p = reinterpret_cast<const P*>(r.v);
  P m = p[0];
#pragma unroll
  for (int j = 1; j < kPerLane / 2; ++j) m = __hmax2_nan(m, p[j]);
  const float a = to_f(m.x), b = to_f(m.y);
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float raw_max(const Raw<f16>& r) { return packed_max<__half2>(r); }
__device__ __forceinline__ float raw_max(const Raw<bf16>& r) { return packed_max<__nv_bfloat162>(r); }

__device__ __forceinline__ float warp_max_nan(float m) {
  float d;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(m));
  return d;
}

// Sum over a lane's tokens of 2^((z - m) f c).
template <typename T>
__device__ __forceinline__ float raw_sum(const Raw<T>& r, float m, float f, float c) {
  const float mf = __fmul_rn(m, f);
  const uint64_t m2 = pack_f32x2(-mf, -mf), f2 = pack_f32x2(f, f), c2 = pack_f32x2(c, c), none = pack_f32x2(-0.f, -0.f);
  uint64_t s[2] = {pack_f32x2(0.f, 0.f), pack_f32x2(0.f, 0.f)};
  float z[kPerLane];
  numbers(r, z);
#pragma unroll
  for (int j = 0; j < kPerLane; j += 2) {
    // (one rounding each: a product is not contracted into the difference)
    const uint64_t t = fma_f32x2(fma_f32x2(pack_f32x2(z[j], z[j + 1]), f2, m2), c2, none);
    s[j / 2 & 1] = add_f32x2(s[j / 2 & 1], pack_f32x2(ex2_approx(lo_f32x2(t)), ex2_approx(hi_f32x2(t))));
  }
  return sum_f32x2(add_f32x2(s[0], s[1]));
}

// Maxima and sums of two blocks (or of one), in lanes 0 .. 15 those of the first (or in all): the maximum is NaN where it is not
// below +inf; the sum of 2^((z - maximum) f c) is 0 where there is no token, and where SUMS is not.
template <typename T, int kPair>
__device__ __forceinline__ float2 block_stats(const Raw<T>* r, bool sums, float f, float c, int lane) {
  float m[kPair], s[kPair];
#pragma unroll
  for (int u = 0; u < kPair; ++u) m[u] = warp_max_nan(raw_max(r[u]));
#pragma unroll
  for (int u = 0; u < kPair; ++u) s[u] = sums ? raw_sum(r[u], m[u], f, c) : 0.f;
  float v = s[0], most = m[0];
  if (kPair == 2) {
    const bool second = lane >= 16;
    const float give = second ? s[0] : s[kPair - 1];
    v = (second ? s[kPair - 1] : s[0]) + __shfl_xor_sync(0xffffffffu, give, 16);
    if (second) most = m[kPair - 1];
  } else {
    v += __shfl_xor_sync(0xffffffffu, v, 16);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return make_float2(most < kInf ? most : kNan, most == -kInf ? 0.f : v);
}
// A lane's share of a block's mass, of the tokens at or before `cut` in the order.
template <typename T, bool VEC>
__device__ __forceinline__ uint64_t raw_mass(const Raw<T>& r, int b, int lane, int vocab, uint64_t cut, float m, const SampleArgs& a,
                                             const uint64_t* pow2) {
  float z[kPerLane];
  numbers(r, z);
  uint64_t s = 0;
#pragma unroll
  for (int j = 0; j < kPerLane; ++j)  // (no token: -inf, of weight 0)
    if (place(order_key(z[j]), token_at<T, VEC>(b, lane, j)) >= cut) s += weight(z[j], m, a, pow2);
  return s;
}

// The largest place of what a thread's lanes see of the row.
template <typename T>
__device__ __forceinline__ uint64_t first_of_order(const T* row, int vocab, int threads) {
  uint64_t first = 0;
  for (int i = threadIdx.x; i < vocab; i += threads) {
    const uint64_t x = place(order_key(to_f(row[i])), i);
    first = x > first ? x : first;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const uint64_t x = __shfl_xor_sync(0xffffffffu, first, o);
    first = x > first ? x : first;
  }
  return first;
}

constexpr int kQueue = 96;  // tokens that a warp puts side by side: 32 wait at most, and 64 join them

constexpr int kRing = 3;  // tiles of a row on their way or in hand: two blocks (one of fp32) of each warp

// What the first CTA of a cluster asks the others for.
struct Command {
  float m, zl, zh;
  int mode;  // 0: nothing more, 1: a bracket, 2: with the tail
};

template <int kThreads, bool FILTER>
struct __align__(128) Shared {
  static constexpr int kWarps = kThreads / 32;
  static constexpr int kCap = FILTER ? 16 * kThreads : 2;  // tokens of the list
  static constexpr int kHist = FILTER ? 4 * kThreads : 2;  // bins
  static constexpr int kTeam = FILTER ? kThreads : 4;
  union {
    uint4 ring[kRing][kWarps * 2 * kBlock / 8];  // while the row is read
    struct {
      uint64_t list[kCap];
      uint32_t count[kHist], lo[kHist], hi[kHist];
      uint64_t small[kTeam], small_w[kTeam];
    };
  };
  uint64_t full[kRing], empty[kRing];
  alignas(16) Command command;
  uint64_t inside, tail;  // of a cluster's CTAs
  int abort_flag;
  int queue[kWarps][FILTER ? kQueue : 2];
  alignas(16) uint32_t groups[kTeam];  // (read four at a time)
  uint64_t pow2[32];
  uint64_t wide[2][kWarps];
  float part[kWarps];
  uint32_t part_n[kWarps];
  uint64_t best;
  uint64_t cut, cut_before, cut_upto;
  uint64_t above_w;
  uint32_t above_n, bin_n, bin;
  int n, found, bad, n_live;
  int edge[4];
  uint32_t edge_n[2];
};

struct Cut {
  uint64_t place;         // of the last token that is kept
  uint64_t before, upto;  // the kept mass without it and with it
};

template <typename T, bool VEC, int kThreads, bool FILTER>
struct Row {
  using Sh = Shared<kThreads, FILTER>;
  static constexpr int kWarps = kThreads / 32, kHist = Sh::kHist;
  static constexpr int kBinBits = kThreads == 256 ? 10 : kThreads == 128 ? 9 : 8;
  static_assert(!FILTER || kHist == 1 << kBinBits, "bins");
  const SampleArgs& a;
  const T* row;
  const float* max_of;  // [n_blocks] maxima
  uint64_t* mass;       // [n_blocks]
  uint16_t* live;       // [n_blocks] (FILTER: blocks that are looked at)
  Sh& sh;
  float m;              // the row's maximum
  int warp, lane;

  __device__ __forceinline__ uint64_t w_of(float z) const { return weight(z, m, a, sh.pow2); }

  // Sums over the CTA; a barrier before and after.
  __device__ ulonglong2 cta_sum(uint64_t v, uint64_t w) const {
    v = warp_sum_u64(v);
    w = warp_sum_u64(w);
    team_sync<kThreads>();
    if (lane == 0) {
      sh.wide[0][warp] = v;
      sh.wide[1][warp] = w;
    }
    team_sync<kThreads>();
    ulonglong2 s = make_ulonglong2(0, 0);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      s.x += sh.wide[0][i];
      s.y += sh.wide[1][i];
    }
    return s;
  }
  __device__ uint64_t cta_sum(uint64_t v) const {
    v = warp_sum_u64(v);
    team_sync<kThreads>();
    if (lane == 0) sh.wide[0][warp] = v;
    team_sync<kThreads>();
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) s += sh.wide[0][i];
    return s;
  }
  // Inclusive sum over the CTA's threads in their order, and the whole; a barrier before and after.
  __device__ uint64_t cta_scan(uint64_t v, uint64_t* whole) const {
    v = warp_scan_u64(v, lane);
    team_sync<kThreads>();
    if (lane == 31) sh.wide[0][warp] = v;
    team_sync<kThreads>();
    uint64_t all = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) v += sh.wide[0][i];
      all += sh.wide[0][i];
    }
    *whole = all;
    return v;
  }

  // f(b, its tokens) for the blocks whose maximum is at least `least`, a warp each, with the next one's tokens on their way; g(b)
  // for the others, a thread each.
  template <typename F, typename G>
  __device__ __forceinline__ void blocks(float least, F f, G g) const {
    team_sync<kThreads>();
    if (threadIdx.x == 0) sh.n_live = 0;
    team_sync<kThreads>();
    for (int b0 = 0; b0 < a.n_blocks; b0 += kThreads) {
      const int b = b0 + threadIdx.x;
      const bool is = b < a.n_blocks && max_of[b] >= least;
      const uint32_t hit = __ballot_sync(0xffffffffu, is);
      int at = 0;
      if (lane == 0 && hit) at = atomicAdd(&sh.n_live, __popc(hit));
      at = __shfl_sync(0xffffffffu, at, 0);
      if (is) live[at + __popc(hit & ((1u << lane) - 1u))] = static_cast<uint16_t>(b);
      else if (b < a.n_blocks) g(b);
    }
    team_sync<kThreads>();
    const int n = sh.n_live;
    if (warp >= n) return;
    Raw<T> raw = fetch<T, VEC>(row, a.p.vocab, live[warp], lane);
#pragma unroll 1
    for (int i = warp; i < n; i += kWarps) {
      Raw<T> ahead;
      if (i + kWarps < n) ahead = fetch<T, VEC>(row, a.p.vocab, live[i + kWarps], lane);
      f(live[i], raw);
      raw = ahead;
    }
  }
  // Tokens of block b that are at least `least`, one bit each.
  __device__ __forceinline__ uint32_t marks(int b, const Raw<T>& raw, float least) const {
    float z[kPerLane];
    numbers(raw, z);
    uint32_t on = 0;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) on |= z[j] >= least ? 1u << j : 0u;
    if (least == -kInf && (b + 1) * kBlock > a.p.vocab)  // (what is no token is -inf)
#pragma unroll
      for (int j = 0; j < kPerLane; ++j)
        if (token_at<T, VEC>(b, lane, j) >= a.p.vocab) on &= ~(1u << j);
    return on;
  }
  // f(token, value) for the marked tokens of the blocks that a warp looks at, 32 at a time: they wait in the warp's queue for more.
  struct Queue {
    int* at;
    int n = 0;
  };
  template <typename F>
  __device__ __forceinline__ void drain(Queue& q, int least, F f) const {
    int done = 0;
    __syncwarp();
    for (; q.n - done >= least; done += 32) {
      const int i = done + lane;
      if (i < q.n) {
        const int e = q.at[i];
        f(e, to_f(row[e]));
      }
      __syncwarp();
    }
    if (done >= q.n) {
      q.n = 0;
      return;
    }
    if (done) {  // what is left moves to the front
      const int i = done + lane;
      const int e = i < q.n ? q.at[i] : 0;
      __syncwarp();
      if (i < q.n) q.at[lane] = e;
      q.n -= done;
      __syncwarp();
    }
  }
  template <typename F>
  __device__ __forceinline__ void marked(Queue& q, int b, uint32_t on, F f) const {
#pragma unroll 1
    for (;;) {
      const uint32_t here = __ballot_sync(0xffffffffu, on != 0);
      if (!here) return;
      if (on) {
        q.at[q.n + __popc(here & ((1u << lane) - 1u))] = token_at<T, VEC>(b, lane, __ffs(on) - 1);
        on &= on - 1;
      }
      q.n += __popc(here);
      if (q.n > kQueue - 32) drain(q, 32, f);
    }
  }
  // f(place, value) for the row's tokens at or before `from` in the order
  template <typename F>
  __device__ __forceinline__ void each(uint64_t from, F f) const {
    const float least = value_of(from);
    Queue q{sh.queue[warp]};
    auto g = [&](int e, float z) {
      const uint64_t x = place(order_key(z), e);
      if (x >= from) f(x, z);
    };
    blocks(least, [&](int b, const Raw<T>& raw) { marked(q, b, marks(b, raw, least), g); }, [](int) {});
    drain(q, 1, g);
  }

  // Place in a list of n counted so far (one atomic for the lanes that are here).
  __device__ __forceinline__ int slot(int* n) const {
    const uint32_t here = __activemask();
    const int first = __ffs(here) - 1;
    int at = 0;
    if (lane == first) at = atomicAdd(n, __popc(here));
    return __shfl_sync(here, at, first) + __popc(here & ((1u << lane) - 1u));
  }

  struct Rest {
    uint64_t inside, tail, error;
  };
  // The tail's mass: `low` from sums against zl, `skipped` from blocks' sums; and how far it may be off.
  __device__ void tail_error(float zl, uint64_t low, uint64_t skipped, Rest* rest) const {
    // the sums against zl: 18 u, and three roundings of an exponent t whose mean over the mass S (of zl's weight) is at most log2(vocab) -
    // log2(S); half a unit of 2^-22 of zl's weight a block, and tokens below 2^-43
    const uint64_t w_zl = w_of(zl);
    const float wf = static_cast<float>(w_zl) + 1.f;
    const float spread = low > 0 ? fmaxf(log2f(a.p.vocab * wf / static_cast<float>(low)), 0.f) : 0.f;
    rest->tail = low + skipped;
    rest->error = static_cast<uint64_t>(a.p.vocab) + a.n_blocks * (1 + (w_zl >> 22)) +
                  __double2ull_ru((20.0 + 2.1 * spread) * 5.9604645e-8 * static_cast<double>(low) + kError * static_cast<double>(skipped));
  }
  // Tokens from zl to zh: into the list, as far as it goes, and their mass in rest->inside.  Returns how many these are.
  // With TAIL: the mass of those below, from fp32 sums, and how far it may be off; the blocks' masses, which `mass` holds at the call, lose
  // it.  Else: `mass` is cleared.
  template <bool TAIL>
  __device__ int bracket(float zl, float zh, Rest* rest) const {
    if (threadIdx.x == 0) sh.n = 0;
    uint64_t inside = 0, tail = 0, skipped = 0;
    const uint64_t w_zl = TAIL ? w_of(zl) : 0;
    Queue q{sh.queue[warp]};
    auto f = [&](int e, float z) {
      inside += w_of(z);
      const int at = slot(&sh.n);
      if (at < Sh::kCap) sh.list[at] = place(order_key(z), e);
    };
    blocks(zl,
           [&](int b, const Raw<T>& raw) {
             if constexpr (TAIL) {
               float z[kPerLane], s[2] = {0.f, 0.f};
               const float zf = __fmul_rn(zl, a.f);
               numbers(raw, z);
               uint32_t on = 0;
#pragma unroll
               for (int j = 0; j < kPerLane; ++j) {
                 const bool low = z[j] < zl;
                 s[j & 1] += low ? ex2_approx(__fmul_rn(fmaf(z[j], a.f, -zf), a.c)) : 0.f;
                 on |= !low && z[j] <= zh ? 1u << j : 0u;
               }
               if (zl == -kInf) on = marks(b, raw, zl);
               marked(q, b, on, f);
               const float all = warp_sum(s[0] + s[1]);
               if (lane == 0) {
                 const uint64_t w = times(all, w_zl);
                 tail += w;
                 mass[b] -= w;
               }
             } else {
               marked(q, b, marks(b, raw, zl), f);
               if (lane == 0) mass[b] = 0;
             }
           },
           [&](int b) {
             if (TAIL) skipped += mass[b];
             mass[b] = 0;
           });
    drain(q, 1, f);
    const ulonglong2 sum = cta_sum(inside, tail);
    rest->inside = sum.x;
    if constexpr (TAIL) {
      tail_error(zl, sum.y, cta_sum(skipped), rest);
    }
    return sh.n;
  }

  // A cluster's bracket: each CTA takes the blocks that it has read, and sends what it finds to the first one, whose `mass` keeps the blocks'
  // masses, less the tail's, or is not looked at.
  template <bool TAIL>
  __device__ void bracket_share(float zl, float zh, int rank, int n_ctas, int tile) const {
    const uint32_t to_n = map_to_rank(smem_u32(&sh.n), 0), to_list = map_to_rank(smem_u32(sh.list), 0), to_mass = map_to_rank(smem_u32(mass), 0);
    uint64_t inside = 0, tail = 0;
    const uint64_t w_zl = TAIL ? w_of(zl) : 0;
    Queue q{sh.queue[warp]};
    auto f = [&](int e, float z) {
      if (z > zh) return;
      inside += w_of(z);
      const uint32_t here = __activemask();
      const int first = __ffs(here) - 1;
      int at = 0;
      if (lane == first) at = add_cluster(to_n, __popc(here));
      at = __shfl_sync(here, at, first) + __popc(here & ((1u << lane) - 1u));
      if (at < Sh::kCap) st_cluster(to_list + 8 * at, place(order_key(z), e));
    };
    for (int k = rank; k * tile < a.n_blocks; k += n_ctas) {
      for (int b = k * tile + warp; b < min((k + 1) * tile, a.n_blocks); b += kWarps) {
        if (!(max_of[b] >= zl)) continue;
        const Raw<T> raw = fetch<T, VEC>(row, a.p.vocab, b, lane);
        if (TAIL && zl > -kInf) {
          float z[kPerLane], s[2] = {0.f, 0.f};
          const float zf = __fmul_rn(zl, a.f);
          numbers(raw, z);
#pragma unroll
          for (int j = 0; j < kPerLane; ++j) s[j & 1] += z[j] < zl ? ex2_approx(__fmul_rn(fmaf(z[j], a.f, -zf), a.c)) : 0.f;
          const float all = warp_sum(s[0] + s[1]);
          if (lane == 0) {
            const uint64_t w = times(all, w_zl);
            tail += w;
            add_cluster(to_mass + 8 * b, 0 - w);
          }
        }
        marked(q, b, marks(b, raw, zl), f);
      }
    }
    drain(q, 1, f);
    const ulonglong2 sum = cta_sum(inside, tail);
    if (threadIdx.x == 0) {
      add_cluster(map_to_rank(smem_u32(&sh.inside), 0), static_cast<uint64_t>(sum.x));
      if (TAIL) add_cluster(map_to_rank(smem_u32(&sh.tail), 0), static_cast<uint64_t>(sum.y));
    }
  }
  // ... asked for by the first CTA, which takes its share: as bracket().
  template <bool TAIL>
  __device__ int bracket_cluster(float zl, float zh, int n_ctas, int tile, Rest* rest) const {
    if (threadIdx.x == 0) {
      sh.n = 0;
      sh.inside = sh.tail = 0;
    }
    uint64_t skipped = 0;
    for (int b = threadIdx.x; b < a.n_blocks; b += kThreads)
      if (!TAIL || !(max_of[b] >= zl)) {
        if (TAIL) skipped += mass[b];
        mass[b] = 0;
      }
    if (static_cast<int>(threadIdx.x) < n_ctas)
      st_cluster(map_to_rank(smem_u32(&sh.command), threadIdx.x), make_float4(m, zl, zh, __int_as_float(TAIL ? 2 : 1)));
    __syncwarp();
    cluster_sync();
    bracket_share<TAIL>(zl, zh, 0, n_ctas, tile);
    __syncwarp();
    cluster_sync();
    rest->inside = sh.inside;
    if (TAIL) tail_error(zl, sh.tail, cta_sum(skipped), rest);
    return sh.n;
  }

  // Masses of the blocks, of the tokens at or before `cut` in the order; returns the whole.
  __device__ uint64_t masses(uint64_t cut) const {
    uint64_t all = 0;
    blocks(value_of(cut),
           [&](int b, const Raw<T>& raw) {
             const uint64_t s = warp_sum_u64(raw_mass<T, VEC>(raw, b, lane, a.p.vocab, cut, m, a, sh.pow2));
             if (lane == 0) {
               mass[b] = s;
               all += s;
             }
           },
           [&](int b) { mass[b] = 0; });
    return cta_sum(all);
  }
  // The row's mass, and that of the tokens below zl.
  __device__ ulonglong2 total(float zl) const {
    uint64_t s = 0, low = 0;
    blocks(-kInf,
           [&](int, const Raw<T>& raw) {
             float z[kPerLane];
             numbers(raw, z);
#pragma unroll
             for (int j = 0; j < kPerLane; ++j) {
               const uint64_t w = w_of(z[j]);
               s += w;
               if (z[j] < zl) low += w;
             }
           },
           [](int) {});
    return cta_sum(s, low);
  }
  // Adds the list's tokens that are kept to the blocks' masses, or (OUT) takes the others out of them.
  template <bool OUT>
  __device__ void add_list(int n, uint64_t cut) const {
    team_sync<kThreads>();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const uint64_t x = sh.list[i];
      if (OUT ? x >= cut : x < cut) continue;
      uint32_t* to = reinterpret_cast<uint32_t*>(mass + index_of(x) / kBlock);
      const uint64_t w = w_of(value_of(x));
      add_shared(to, to + 1, OUT ? 0 - w : w);
    }
    team_sync<kThreads>();
  }

  // (a block without a token that is kept may be left with less than nothing by the fp32 sums)
  static __device__ __forceinline__ uint64_t positive(uint64_t w) { return static_cast<int64_t>(w) < 0 ? 0 : w; }

  // The first block whose cumulative mass is above u0 of the whole; -1 where the error of the cumulative masses against their whole's share
  // leaves it open.
  __device__ int pick_block(float u0, uint64_t error) const {
    const int per = (a.n_blocks + kThreads - 1) / kThreads, from = min(static_cast<int>(threadIdx.x) * per, a.n_blocks),
              to = min(from + per, a.n_blocks);
    uint64_t s = 0, total;
    for (int b = from; b < to; ++b) s += positive(mass[b]);
    const uint64_t up = cta_scan(s, &total), target = share_of(u0, total);
    if (s > 0 && (target < total ? up > target && up - s <= target : up == total)) {
      uint64_t before = up - s, cum = before;
      int found = from;
      for (int i = from; i < to; ++i) {
        const uint64_t w = positive(mass[i]);
        if (w == 0) continue;
        found = i;
        before = cum;
        cum += w;
        if (cum > target) break;
      }
      if (error && ((before != 0 && target <= before + error) || (cum != total && cum <= target + error))) found = -1;
      sh.found = found;
    }
    team_sync<kThreads>();
    return sh.found;
  }
  // The first token of block b whose cumulative mass, of the tokens at or before `cut`, is above u1 of the block's.
  __device__ void draw_token(int64_t r, int b, float u1, uint64_t cut, uint64_t whole) const {
    const SampleParams& p = a.p;
    constexpr int kPer = kBlock / kThreads;
    const int first = b * kBlock + threadIdx.x * kPer;
    float z[kPer];
    uint64_t w[kPer], s = 0, total;
#pragma unroll
    for (int j = 0; j < kPer; ++j) z[j] = first + j < p.vocab ? to_f(row[first + j]) : -kInf;
#pragma unroll
    for (int j = 0; j < kPer; ++j) s += w[j] = place(order_key(z[j]), first + j) >= cut ? w_of(z[j]) : 0;
    const uint64_t up = cta_scan(s, &total), target = share_of(u1, total);
    if (s > 0 && (target < total ? up > target && up - s <= target : up == total)) {
      uint64_t cum = up - s;
      int id = first;
      float z_id = z[0];
      bool done = false;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        if (w[j] != 0 && !done) {
          id = first + j;
          z_id = z[j];
          cum += w[j];
          done = cum > target;
        }
      }
      p.ids[r] = id;
      if (p.logprobs) p.logprobs[r] = fmaf(z_id, a.f, -__fmul_rn(m, a.f)) * a.scale - logf(static_cast<float>(whole) * (1.f / (1ull << kOne)));
    }
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

  // The last token of the shortest prefix of the order, among the tokens of src with places lo .. hi (n at most) and those above them (above_n
  // tokens with the mass above_w), that has `count` tokens or (count 0) a mass of at least `target`.
  template <typename S>
  __device__ Cut find_cut(const S& src, int n, uint64_t lo, uint64_t hi, uint32_t count, uint64_t target, uint32_t above_n,
                          uint64_t above_w) const {
    while (n > kThreads) {
      const int shift = max(0, 64 - __clzll(hi - lo) - kBinBits);
      team_sync<kThreads>();
      for (int i = threadIdx.x; i < kHist; i += kThreads) sh.count[i] = sh.lo[i] = sh.hi[i] = 0;
      team_sync<kThreads>();
      src.each(lo, [&](uint64_t x, float z) {
        if (x > hi) return;
        const uint32_t bin = static_cast<uint32_t>((hi - x) >> shift);
        atomicAdd(&sh.count[bin], 1u);
        add_shared(&sh.lo[bin], &sh.hi[bin], w_of(z));
      });
      team_sync<kThreads>();
      pick_bin(count, target, above_n, above_w);
      above_n = sh.above_n;
      above_w = sh.above_w;
      n = sh.bin_n;
      hi -= static_cast<uint64_t>(sh.bin) << shift;
      const uint64_t width = (1ull << shift) - 1ull;
      if (hi - lo > width) lo = hi - width;
      if constexpr (S::kRow) {
        if (n <= Sh::kCap && n > kThreads) {
          gather(src, lo, hi, sh.list, Sh::kCap);
          return find_cut(List{*this, n}, n, lo, hi, count, target, above_n, above_w);
        }
      }
    }
    gather(src, lo, hi, sh.small, kThreads);
    n = sh.n;
    const int t = threadIdx.x;
    const uint64_t x = t < n ? sh.small[t] : 0;
    const uint64_t w = t < n ? w_of(value_of(x)) : 0;
    sh.small_w[t] = w;
    if (t == 0) sh.cut = 0;
    team_sync<kThreads>();
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
    team_sync<kThreads>();
    const bool none = sh.cut == 0;
    team_sync<kThreads>();
    if (none && t < n && rank == above_n + n) write();
    team_sync<kThreads>();
    const Cut cut{sh.cut, sh.cut_before, sh.cut_upto};
    team_sync<kThreads>();
    return cut;
  }
  template <typename S>
  __device__ void gather(const S& src, uint64_t lo, uint64_t hi, uint64_t* to, int cap) const {
    team_sync<kThreads>();
    if (threadIdx.x == 0) sh.n = 0;
    team_sync<kThreads>();
    src.each(lo, [&](uint64_t x, float) {
      if (x > hi) return;
      const int at = slot(&sh.n);
      if (at < cap) to[at] = x;
    });
    team_sync<kThreads>();
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
    team_sync<kThreads>();
  }

  // A key that at least k tokens have or more: the k-th largest of the maxima of kThreads groups (k <= kThreads) of blocks, or of tokens.
  // (Without its last bits, whose place the group's number takes: no two are equal.)
  template <bool TOKENS>
  __device__ uint32_t bound_of_k(int k) const {
    constexpr uint32_t kLow = kThreads - 1;
    float g = -kInf;
    if (TOKENS) {
#pragma unroll 8
      for (int i = threadIdx.x; i < a.p.vocab; i += kThreads) g = fmaxf(g, to_f(row[i]));
    } else {
      for (int b = threadIdx.x; b < a.n_blocks; b += kThreads) g = fmaxf(g, max_of[b]);
    }
    const uint32_t mine = (order_key(g) & ~kLow) | threadIdx.x;
    sh.groups[threadIdx.x] = mine;
    team_sync<kThreads>();
    int more = 0;
#pragma unroll 8
    for (int i = 0; i < kThreads; i += 4) {
      const uint4 x = *reinterpret_cast<const uint4*>(sh.groups + i);
      more += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
    }
    if (more == k - 1) sh.above_n = mine & ~kLow;
    team_sync<kThreads>();
    const uint32_t key = max(sh.above_n, kKeyNegInf);
    team_sync<kThreads>();
    return key;
  }

  // Weights of a sample of the row, one token of 8 or more, in runs of 8: count[i] of those in the i-th 1/32 of an octave from the
  // maximum down.  Returns how many were looked at.
  __device__ int sampled() const {
    const int vocab = a.p.vocab, runs = max(4, (vocab / 8 + 8 * kThreads - 1) / (8 * kThreads));  // of a thread
    team_sync<kThreads>();
    for (int i = threadIdx.x; i < kHist; i += kThreads) sh.count[i] = 0;
    if (threadIdx.x < 2) sh.edge[threadIdx.x] = kHist;
    team_sync<kThreads>();
    const int all = runs * kThreads;
    const float step = static_cast<float>(vocab - 8) / static_cast<float>(all), c32 = a.c * 32.f, mf = __fmul_rn(m, a.f);
    constexpr int kAhead = 4, kV = 8 / Elem<T>::kPer;  // loads on their way
    for (int k0 = 0; k0 < runs; k0 += kAhead) {
      uint4 v[kAhead][kV];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (k0 + u >= runs) break;
        const int e = min(static_cast<int>(((k0 + u) * kThreads + threadIdx.x) * step), vocab - 8);
        if (VEC) {
#pragma unroll
          for (int i = 0; i < kV; ++i) v[u][i] = reinterpret_cast<const uint4*>(row + (e & ~7))[i];
        } else {
          T* t = reinterpret_cast<T*>(v[u]);
#pragma unroll
          for (int j = 0; j < 8; ++j) t[j] = row[e + j];
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (k0 + u >= runs) break;
        float z[8];
#pragma unroll
        for (int i = 0; i < kV; ++i) unpack(v[u][i], z + i * Elem<T>::kPer, static_cast<const T*>(nullptr));
#pragma unroll
        for (int j = 0; j < 8; ++j) atomicAdd(&sh.count[static_cast<int>(fminf(fmaf(-z[j], a.f, mf) * c32, kHist - 1.f))], 1u);
      }
    }
    team_sync<kThreads>();
    return 8 * all;
  }
  // The value that lies bins / 32 of an octave below the maximum (-inf: out of fp32's range).
  __device__ float below_max(int bins) const { return (__fmul_rn(m, a.f) - bins / (32.f * a.c)) / a.f; }
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
    team_sync<kThreads>();
    up -= sum;
    for (int i = 0; i < warp; ++i) up += sh.part_n[i];
    const double want = (1.3 * k + 400.0) * looked / a.p.vocab;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (up + n[j] >= want) atomicMin(&sh.edge[0], static_cast<int>(threadIdx.x) * kPer + j + 1);
    team_sync<kThreads>();
    const int edge = sh.edge[0];
    return edge >= kHist ? -kInf : below_max(edge);
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
    team_sync<kThreads>();
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
    team_sync<kThreads>();
    const int low = sh.edge[0], high = sh.edge[1];
    // 64 sampled tokens more below, 32 above: 800 of the row, which the list has room for
    if (threadIdx.x == 0) {
      sh.edge[2] = kHist;
      sh.edge[3] = 0;
      sh.edge_n[0] = sh.edge_n[1] = 0;
    }
    team_sync<kThreads>();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      if (i == low) sh.edge_n[0] = n[j] + up_n;
      if (i == high) sh.edge_n[1] = n[j] + up_n;
    }
    team_sync<kThreads>();
    const uint32_t n_low = sh.edge_n[0], n_high = sh.edge_n[1];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      if (n_low >= 64 && n[j] + up_n <= n_low - 64) atomicMin(&sh.edge[2], i);
      if (n[j] + up_n >= n_high + 32) atomicMax(&sh.edge[3], i);
    }
    team_sync<kThreads>();
    const int zl = sh.edge[2], zh = sh.edge[3];
    team_sync<kThreads>();
    return make_float2(zl >= kHist ? -kInf : below_max(zl), zh <= 0 ? kInf : below_max(zh));
  }
};

template <typename T, bool VEC, int kThreads, bool FILTER>
__global__ void __launch_bounds__(kThreads, (FILTER ? 768 : 1024) / kThreads) sample_kernel(const SampleArgs a) {
  constexpr int kWarps = kThreads / 32;
  using Sh = Shared<kThreads, FILTER>;
  extern __shared__ __align__(128) unsigned char dynamic[];  // Shared, then [n_blocks] masses, maxima, and numbers
  Sh& sh = *reinterpret_cast<Sh*>(dynamic);
  static_assert(offsetof(Sh, groups) % 16 == 0 && offsetof(Sh, ring) % 16 == 0 && sizeof(Sh) % 16 == 0, "vectors of 16 bytes");
  const SampleParams& p = a.p;
  uint64_t* mass = reinterpret_cast<uint64_t*>(dynamic + sizeof(Sh));
  float* max_of = reinterpret_cast<float*>(mass + a.n_blocks);
  uint16_t* live = reinterpret_cast<uint16_t*>(max_of + a.n_blocks);
  const int rank = cluster_rank(), n_ctas = cluster_ctas();
  const int64_t r = blockIdx.x / n_ctas;
  if (p.row_ids && p.row_ids[r] != p.row_id) return;  // the whole cluster
  const T* row = static_cast<const T*>(p.logits) + r * p.ld;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (n_ctas > 1) cluster_arrive();
  const bool by_k = FILTER && p.top_k > 0 && p.top_k < p.vocab, by_m = FILTER && a.drop != -HUGE_VAL, by_p = FILTER && p.top_p < 1.0;
  const bool sums = !FILTER || p.logprobs || !(by_k || by_m);
  const float u0 = p.uniforms[2 * r], u1 = p.uniforms[2 * r + 1];
  constexpr int kPair = sizeof(T) == 2 ? 2 : 1, kTile = kWarps * kPair;  // blocks of a warp at a time, of the CTA
  if (threadIdx.x < 32) sh.pow2[threadIdx.x] = kPow2[threadIdx.x];
  if (threadIdx.x == 0) {
    sh.bad = 0;
    sh.best = 0;
    sh.abort_flag = 0;
  }
  const uint32_t to_max = map_to_rank(smem_u32(max_of), 0), to_mass = map_to_rank(smem_u32(mass), 0);
  auto put = [&](const Raw<T>* cur, int b) {  // blocks b and b + kWarps
    const float2 st = block_stats<T, kPair>(cur, sums, a.f, a.c, lane);
    const int at = kPair == 2 && lane >= 16 ? b + kWarps : b;
    if ((lane == 0 || (kPair == 2 && lane == 16)) && at < a.n_blocks) {
      if (FILTER && rank != 0) max_of[at] = st.x;  // (for this CTA's share of a bracket)
      if (n_ctas == 1) {
        max_of[at] = st.x;
        mass[at] = __float_as_uint(st.y);
      } else {
        st_cluster(to_max + 4 * at, st.x);
        st_cluster(to_mass + 8 * at, static_cast<uint64_t>(__float_as_uint(st.y)));
      }
    }
  };
  const int tiles = (a.n_blocks + kTile - 1) / kTile;
  if constexpr (VEC) {
    // Tiles of 16 KB (256 threads) by bulk copies: long stretches of a row at a time.  With loads of the warps' own, 1 KB each, some sizes
    // of the whole took half as long again as others.
    constexpr int kTileBytes = kTile * kBlock * static_cast<int>(sizeof(T)), E = Elem<T>::kPer;
    static_assert(kTileBytes == static_cast<int>(sizeof(sh.ring[0])), "the ring's tiles");
    volatile int* abort_flag = &sh.abort_flag;
    const int64_t whole_bytes = static_cast<int64_t>(p.vocab / E) * 16;
    auto issue = [&](int k) {  // one thread
      const int64_t from = (static_cast<int64_t>(k) * n_ctas + rank) * kTileBytes;
      const int64_t left = whole_bytes - from;
      uint64_t* bar = &sh.full[k % kRing];
      if (left > 0) {
        const uint32_t bytes = left < kTileBytes ? static_cast<uint32_t>(left) : kTileBytes;
        mbar_arrive_expect_tx(bar, bytes);
        bulk_load(sh.ring[k % kRing], reinterpret_cast<const char*>(row) + from, bytes, bar);
      } else {
        mbar_arrive(bar);
      }
    };
    const int mine = tiles > rank ? (tiles - rank + n_ctas - 1) / n_ctas : 0;
    if (threadIdx.x == 0) {
      for (int i = 0; i < kRing; ++i) {
        mbar_init(&sh.full[i], 1);
        mbar_init(&sh.empty[i], kWarps);
      }
      fence_mbar_init();
      fence_proxy_async_smem();
      for (int k = 0; k < min(kRing, mine); ++k) issue(k);
    }
    team_sync<kThreads>();
    if (n_ctas > 1) cluster_wait();  // every CTA of the cluster runs: the leader's shared memory may be written
    for (int k = 0; k < mine; ++k) {
      if (threadIdx.x == 0 && k > 0 && k - 1 + kRing < mine) {  // the tile before has been read by all: another into its place
        if (mbar_wait(&sh.empty[(k - 1) % kRing], ((k - 1) / kRing) & 1, abort_flag, a.status, 71)) issue(k - 1 + kRing);
        else mbar_arrive(&sh.full[(k - 1) % kRing]);
      }
      __syncwarp();
      // (after an expired wait, which is recorded, the kernel goes on with what is there; no copy lands after the CTA has left)
      if (!mbar_wait_warp(smem_u32(&sh.full[k % kRing]), (k / kRing) & 1, abort_flag, a.status, 72))
        mbar_drain(&sh.full[k % kRing], (k / kRing) & 1);
      const int b = (k * n_ctas + rank) * kTile + warp;
      Raw<T> cur[kPair];
#pragma unroll
      for (int u = 0; u < kPair; ++u) {
        const uint4* from = sh.ring[k % kRing] + (warp + u * kWarps) * (kBlock / E);
        const int first = (b + u * kWarps) * kBlock;
        if (first + kBlock <= p.vocab) {
#pragma unroll
          for (int i = 0; i < Raw<T>::kN; ++i) cur[u].v[i] = from[i * 32 + lane];
        } else {  // the row's end: copies bring whole vectors alone
#pragma unroll
          for (int i = 0; i < Raw<T>::kN; ++i) {
            const int e = first + (i * 32 + lane) * E;
            if (e + E <= p.vocab) {
              cur[u].v[i] = from[i * 32 + lane];
            } else {
              T* t = reinterpret_cast<T*>(&cur[u].v[i]);
#pragma unroll
              for (int j = 0; j < E; ++j) t[j] = e + j < p.vocab ? row[e + j] : neg_inf<T>();
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.empty[k % kRing]);
      put(cur, b);
    }
  } else {
    if (n_ctas > 1) cluster_wait();
    int b = rank * kTile + warp;
    Raw<T> next[kPair];
#pragma unroll
    for (int u = 0; u < kPair; ++u)
      if (b + u * kWarps < a.n_blocks) next[u] = fetch<T, VEC>(row, p.vocab, b + u * kWarps, lane);
    for (; b < a.n_blocks; b += kTile * n_ctas) {
      Raw<T> cur[kPair];
#pragma unroll
      for (int u = 0; u < kPair; ++u) {
        const int ahead = b + u * kWarps + kTile * n_ctas;
        cur[u] = next[u];
        if (ahead < a.n_blocks) next[u] = fetch<T, VEC>(row, p.vocab, ahead, lane);
      }
      put(cur, b);
    }
  }
  if (n_ctas > 1) {
    __syncwarp();
    cluster_sync();
    if (rank != 0) {
      if constexpr (FILTER) {
        cluster_sync();  // the command has come
        const Command c = sh.command;
        if (c.mode == 0) return;
        const Row<T, VEC, kThreads, FILTER> t{a, row, max_of, mass, live, sh, c.m, warp, lane};
        if (c.mode == 2) t.template bracket_share<true>(c.zl, c.zh, rank, n_ctas, kTile);
        else t.template bracket_share<false>(c.zl, c.zh, rank, n_ctas, kTile);
        __syncwarp();
        cluster_sync();
      }
      return;
    }
  } else {
    team_sync<kThreads>();
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
  team_sync<kThreads>();
#pragma unroll
  for (int i = 0; i < kWarps; ++i) m = fmaxf(m, sh.part[i]);
  if (sh.bad || m == -kInf) {
    if (FILTER && n_ctas > 1) {
      if (static_cast<int>(threadIdx.x) < n_ctas)
        st_cluster(map_to_rank(smem_u32(&sh.command), threadIdx.x), make_float4(0.f, 0.f, 0.f, __int_as_float(0)));
      __syncwarp();
      cluster_sync();
    }
    // no distribution: the first token of the order
    const uint64_t first = first_of_order(row, p.vocab, kThreads);
    if (lane == 0) atomicMax(reinterpret_cast<unsigned long long*>(&sh.best), static_cast<unsigned long long>(first));
    team_sync<kThreads>();
    if (threadIdx.x == 0) {
      p.ids[r] = index_of(sh.best);
      if (p.logprobs) p.logprobs[r] = sh.bad ? kNan : -kInf;
    }
    return;
  }

  using R = Row<T, VEC, kThreads, FILTER>;
  const R t{a, row, max_of, mass, live, sh, m, warp, lane};
  // masses of whole blocks from their fp32 sums, and the row's
  uint64_t whole = 0;
  if (sums) {
    for (int b = threadIdx.x; b < a.n_blocks; b += kThreads) {
      const uint64_t x = times(__uint_as_float(static_cast<uint32_t>(mass[b])), t.w_of(max_of[b]));
      mass[b] = x;
      whole += x;
    }
    whole = t.cta_sum(whole);
  }

  uint64_t cut = kEverything;
  uint64_t pick_error = 0;
  if constexpr (FILTER) {
    const uint64_t top = static_cast<uint64_t>(order_key(m)) << 32 | 0xFFFFFFFFu;
    float zl = -kInf, zh = kInf;
    if (by_m) zl = __double2float_ru(static_cast<double>(m) + a.drop);
    const float floor_m = zl;
    auto bound_by_k = [&] {
      // (as many groups of blocks as there are blocks have a maximum)
      if (p.top_k <= min(a.n_blocks, kThreads)) return fmaxf(zl, key_value(t.template bound_of_k<false>(p.top_k)));
      if (p.vocab >= kSampled) return fmaxf(zl, t.sampled_bound_of_k(p.top_k));
      if (p.top_k <= kThreads) return fmaxf(zl, key_value(t.template bound_of_k<true>(p.top_k)));
      return zl;
    };
    // (half a percent of the maximum's weight leaves few tokens by itself, as a rule)
    const bool by_m_first = by_m && p.min_p >= 0.005;
    if (by_k && !by_m_first) zl = bound_by_k();
    if (!by_k && !by_m) {
      // the maxima from the 64th largest on, if they have the mass already
      uint64_t s = 0;
      uint32_t key = 0;
      if (a.n_blocks >= 16) {
        key = t.template bound_of_k<false>(min(64, a.n_blocks / 4));
        for (int b = threadIdx.x; b < a.n_blocks; b += kThreads)
          if (order_key(max_of[b]) >= key) s += t.w_of(max_of[b]);
        s = t.cta_sum(s);
      }
      if (static_cast<double>(s) >= p.top_p * static_cast<double>(whole) * (1.0 + kError)) {
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
    team_sync<kThreads>();
    int n;
    if (n_ctas > 1) n = alone ? t.template bracket_cluster<true>(zl, zh, n_ctas, kTile, &rest) : t.template bracket_cluster<false>(zl, zh, n_ctas, kTile, &rest);
    else n = alone ? t.template bracket<true>(zl, zh, &rest) : t.template bracket<false>(zl, zh, &rest);
    if (by_k && by_m_first ? n > Sh::kCap : by_k && n < p.top_k && zl > floor_m) {  // it did not; or the sample misled
      zl = by_m_first ? bound_by_k() : floor_m;
      team_sync<kThreads>();
      n = t.template bracket<false>(zl, zh, &rest);
      if (n < p.top_k && zl > floor_m) {
        zl = floor_m;
        team_sync<kThreads>();
        n = t.template bracket<false>(zl, zh, &rest);
      }
    }
    bool listed = n <= Sh::kCap;
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
        kept = rest.inside;
      }
      if (by_p) {
        const uint64_t target = __double2ull_ru(p.top_p * static_cast<double>(kept));
        // (a search of the row leaves what it found last in the list)
        cut = listed ? t.find_cut(list, n, lo, top, 0, target, 0, 0).place : t.find_cut(whole_row, n, lo, top, 0, target, 0, 0).place;
      }
    } else {
      // What is not kept has at most the share 1 - top_p of the row's mass T: the tail, and the list from its end on.  The mass of the list that
      // is kept is then at least tail + list - (1 - top_p) T, which is off by the tail's error and, little, by T's.
      const uint64_t hi = zh < m ? static_cast<uint64_t>(order_key(zh)) << 32 | 0xFFFFFFFFu : top;
      uint64_t total = whole, error = rest.error + __double2ull_ru((1.0 - p.top_p) * kError * static_cast<double>(whole));
      bool sure = false;
      for (;;) {
        const uint64_t out = __double2ull_rd((1.0 - p.top_p) * static_cast<double>(total)), held = rest.tail + rest.inside;
        if (listed && out + error < held && held - out + error <= rest.inside) {
          const uint64_t target = held - out;
          const Cut k = t.find_cut(list, n, lo, hi, 0, target, 0, 0);
          cut = k.place;
          if (sure || (target > k.before + error && k.upto >= target + error)) break;
        }
        if (sure) {
          listed = false;
          cut = t.find_cut(whole_row, p.vocab, kEverything, top, 0, __double2ull_ru(p.top_p * static_cast<double>(total)), 0, 0).place;
          break;
        }
        // within the error of another cut, or not between the bounds: both anew
        const ulonglong2 sums_anew = t.total(zl);
        total = sums_anew.x;
        rest.tail = sums_anew.y;
        error = 0;
        sure = true;
      }
    }
    if (!listed) t.masses(cut);
    else if (alone) t.template add_list<true>(n, cut);
    else t.template add_list<false>(n, cut);
    pick_error = listed && alone ? 2 * (rest.error + static_cast<uint64_t>(kError * static_cast<double>(whole))) : 0;
  } else {
    // (errors e of the masses before a border, kError at most, move it by e u (1 - u) of the whole, and those behind it as much)
    pick_error = 1 + static_cast<uint64_t>(0.5 * kError * static_cast<double>(whole));
  }

  team_sync<kThreads>();
  int b = t.pick_block(u0, pick_error);
  if (b < 0) {
    t.masses(cut);
    b = t.pick_block(u0, 0);
  }
  t.draw_token(r, b, u1, cut, whole);
}

// few rows: a cluster reads a row, down to a block or two per warp
template <typename T, bool VEC, int kThreads, bool FILTER>
cudaError_t launch_rows(const SampleArgs& a, cudaStream_t s) {
  Launch l{1, 0, kThreads};
  while (l.cluster < kMaxCluster && static_cast<int64_t>(a.p.rows) * l.cluster < num_sms() && a.n_blocks / l.cluster > 8) l.cluster *= 2;
  const size_t smem = sizeof(Shared<kThreads, FILTER>) + 14 * static_cast<size_t>(a.n_blocks);
  return launch<&sample_kernel<T, VEC, kThreads, FILTER>>(a.p.rows, l, smem, s, a);
}
template <typename T, bool FILTER>
cudaError_t sample_rows(const SampleArgs& a, cudaStream_t s) {
  const bool vec = reinterpret_cast<uintptr_t>(a.p.logits) % 16 == 0 && (a.p.rows == 1 || a.p.ld * static_cast<int64_t>(sizeof(T)) % 16 == 0);
  if (!vec) return a.n_blocks <= kShort ? launch_rows<T, false, 128, FILTER>(a, s) : launch_rows<T, false, 256, FILTER>(a, s);
  if (a.n_blocks <= kShortest) return launch_rows<T, true, 64, FILTER>(a, s);
  return a.n_blocks <= kShort ? launch_rows<T, true, 128, FILTER>(a, s) : launch_rows<T, true, 256, FILTER>(a, s);
}

}  // namespace rows
}  // namespace sgd
