// What the two kernels that draw tokens share (sample.cu has the definition): exact weights, a block's statistics, the last
// two steps of a row.
#pragma once

#include <math.h>

#include "vocab_rows.cuh"

namespace sgd {
namespace rows {

constexpr int kBlock = SGD_SAMPLE_BLOCK;
constexpr int kPerLane = kBlock / 32;
constexpr int kOne = 43;  // weight() of the row's maximum is 2^43: 2^20.6 of them (a row of 3 MiB) add up in 64 bits
static_assert(kBlock == 512, "a lane takes 16 tokens");

// A block's sum in fp32 is off by at most this much of it (u = 2^-24): a term by 4 u (ex2.approx) and three roundings of its exponent,
// ln2 3 |t| u, whose mean over the block's mass is at most ln2 3 log2(512) u = 18.7 u; 10 u from being added up: 33 u.
constexpr double kError = 2.2e-6;

struct SampleArgs {
  SampleParams p;
  float c, c_lo;    // scale log2(e), as the sum of two floats
  double drop;      // ln(min_p) / scale: a token at or above max + drop passes (-inf: every token)
  int n_blocks;
  int* status;
};

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

// Weight 2^((z - m) c) of a logit against the row's maximum m as a whole number, 2^43 for the maximum: exact to about 2^-31
// relative and half a unit.  z - m = d + dl exactly, (d + dl) c = t + tl to 2^-45; t + tl = n + j / 32 + g with |g| <= 1/64;
// 2^g - 1 = g ln2 + ... to the fourth power (the fifth is 1.3e-12).
__device__ __forceinline__ uint64_t weight(float z, float m, const SampleArgs& a, const uint64_t* pow2) {
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
// The whole number that a mass is above where it is above u total.
__device__ __forceinline__ uint64_t share_of(float u, uint64_t total) {
  return __double2ull_rd(static_cast<double>(fminf(fmaxf(u, 0.f), 1.f)) * static_cast<double>(total));
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

// Sum over a lane's tokens of 2^((z - m) c).
template <typename T>
__device__ __forceinline__ float raw_sum(const Raw<T>& r, float m, float c) {
  const uint64_t m2 = pack_f32x2(-m, -m), c2 = pack_f32x2(c, c), none = pack_f32x2(-0.f, -0.f);
  uint64_t s[2] = {pack_f32x2(0.f, 0.f), pack_f32x2(0.f, 0.f)};
  float z[kPerLane];
  numbers(r, z);
#pragma unroll
  for (int j = 0; j < kPerLane; j += 2) {
    // (one rounding each: a product is not contracted into the difference)
    const uint64_t t = fma_f32x2(add_f32x2(pack_f32x2(z[j], z[j + 1]), m2), c2, none);
    s[j / 2 & 1] = add_f32x2(s[j / 2 & 1], pack_f32x2(ex2_approx(lo_f32x2(t)), ex2_approx(hi_f32x2(t))));
  }
  return sum_f32x2(add_f32x2(s[0], s[1]));
}

// Maxima and sums of two blocks (or of one), in lanes 0 .. 15 those of the first (or in all): the maximum is NaN where it is not
// below +inf; the sum of 2^((z - maximum) c) is 0 where there is no token, and where SUMS is not.
template <typename T, int kPair>
__device__ __forceinline__ float2 block_stats(const Raw<T>* r, bool sums, float c, int lane) {
  float m[kPair], s[kPair];
#pragma unroll
  for (int u = 0; u < kPair; ++u) m[u] = warp_max_nan(raw_max(r[u]));
#pragma unroll
  for (int u = 0; u < kPair; ++u) s[u] = sums ? raw_sum(r[u], m[u], c) : 0.f;
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
// A block's mass from its statistics.
__device__ __forceinline__ uint64_t block_mass(float m_block, float s, float m, const SampleArgs& a, const uint64_t* pow2) {
  return s == 0.f ? 0 : __double2ull_rn(static_cast<double>(s) * static_cast<double>(weight(m_block, m, a, pow2)));
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

// The first block whose cumulative mass is above u0 of the whole (one warp); -1 where the masses' error (`exact`: none) leaves it open.
__device__ __forceinline__ int pick_block(const uint64_t* mass, int n_blocks, float u0, bool exact, int lane) {
  const int per = (n_blocks + 31) / 32, from = min(lane * per, n_blocks), to = min(from + per, n_blocks);
  uint64_t s = 0;
#pragma unroll 4
  for (int b = from; b < to; ++b) s += mass[b];
  const uint64_t up = warp_scan_u64(s, lane), total = __shfl_sync(0xffffffffu, up, 31);
  const uint64_t target = share_of(u0, total);
  const uint32_t above = __ballot_sync(0xffffffffu, s > 0 && up > target), held = __ballot_sync(0xffffffffu, s > 0);
  const int which = above ? __ffs(above) - 1 : 31 - __clz(held);
  int found = 0;
  if (lane == which) {
    uint64_t before = up - s, cum = before;
    found = from;
    for (int i = from; i < to; ++i) {
      const uint64_t w = mass[i];
      if (w == 0) continue;
      found = i;
      before = cum;
      cum += w;
      if (cum > target) break;
    }
    // (errors e of the masses before a border, kError at most, move it by e u (1 - u) of the whole, and those behind it as much)
    const uint64_t error = exact ? 0 : __double2ull_ru(0.5 * kError * static_cast<double>(total));
    if (!exact && ((before != 0 && target <= before + error) || (cum != total && cum <= target + error))) found = -1;
  }
  return __shfl_sync(0xffffffffu, found, which);
}

// The first token of block b whose cumulative mass, of the tokens at or before `cut`, is above u1 of the block's (one warp).
template <typename T, bool VEC>
__device__ __forceinline__ void draw_token(const SampleArgs& a, const T* row, int64_t r, int b, float u1, uint64_t cut, float m, uint64_t whole,
                                           const uint64_t* pow2, int lane) {
  const SampleParams& p = a.p;
  const int first = b * kBlock + lane * kPerLane;  // 16 neighbours a lane
  float z[kPerLane];
  uint64_t w[kPerLane], s = 0;
  if (VEC && first + kPerLane <= p.vocab) {
#pragma unroll
    for (int i = 0; i < Raw<T>::kN; ++i)
      unpack(reinterpret_cast<const uint4*>(row + first)[i], z + i * Elem<T>::kPer, static_cast<const T*>(nullptr));
  } else {
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) z[j] = first + j < p.vocab ? to_f(row[first + j]) : -kInf;
  }
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {
    w[j] = place(order_key(z[j]), first + j) >= cut ? weight(z[j], m, a, pow2) : 0;
    s += w[j];
  }
  const uint64_t up = warp_scan_u64(s, lane), total = __shfl_sync(0xffffffffu, up, 31);
  const uint64_t target = share_of(u1, total);
  const uint32_t above = __ballot_sync(0xffffffffu, s > 0 && up > target), held = __ballot_sync(0xffffffffu, s > 0);
  const int which = above ? __ffs(above) - 1 : (held ? 31 - __clz(held) : 0);
  if (lane != which) return;
  uint64_t cum = up - s;
  int id = first;
  float z_id = -kInf;
  bool done = false;
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {
    if (w[j] != 0 && !done) {
      id = first + j;
      z_id = z[j];
      cum += w[j];
      done = cum > target;
    }
  }
  p.ids[r] = id;
  if (p.logprobs) p.logprobs[r] = (z_id - m) * p.scale - logf(static_cast<float>(whole) * (1.f / (1ull << kOne)));
}

// A row without a distribution takes the first token of the order (lanes of `threads` threads; their best places, 0 at first, in *best).
template <typename T>
__device__ __forceinline__ uint64_t first_of_order(const T* row, int vocab, int tid, int threads) {
  uint64_t first = 0;
  for (int i = tid; i < vocab; i += threads) {
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

// Unfiltered draws of many long rows (sample_stream.cu).
bool sample_stream_pays(const SampleArgs& a, int elem);
template <typename T>
cudaError_t sample_stream(const SampleArgs& a, cudaStream_t s);

}  // namespace rows
}  // namespace sgd
