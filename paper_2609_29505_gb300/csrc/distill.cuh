// What the two distillation kernels share: parameters, the list, a row's scalars and the stores of a gradient.
#pragma once

#include <type_traits>

#include "vocab_rows.cuh"

namespace sgd {
namespace rows {

constexpr int kMaxList = kMaxTop;
static_assert(kMaxList == 64, "two warps hold the list");

struct DistillArgs {
  const void* logits;
  int64_t ld;
  int rows, vocab;
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

// The slice's part of a gradient row: value(i, f) gives vector i of the logits' slice; stored whole where
// the gradient's address allows it.
template <typename T, typename G, typename F>
__device__ __forceinline__ void write_grad(const Slice<T>& sl, G* grow, int tid, int threads, const F& value) {
  constexpr int E = Elem<T>::kPer;
  constexpr uintptr_t kAlign = E * sizeof(G) < 16 ? E * sizeof(G) : 16;
  if (sl.nv == 0) return;
  G* g0 = grow + sl.first_element(0);
  const bool aligned = (reinterpret_cast<uintptr_t>(g0) & (kAlign - 1)) == 0;
  const int lo = aligned && sl.whole(0) ? 0 : 1, hi = aligned && sl.whole(sl.nv - 1) ? sl.nv : sl.nv - 1;
  if (aligned) {
    // (the loop's size counts, as a streaming CTA's roles share the instruction cache: unrolled by 8 2052 x 126464 fp16
    // takes 200 us, by 4 175 to 179 and by 2 175; 300 rows in fp32 74, 67 to 75 and 67)
#pragma unroll 2
    for (int i = lo + tid; i < hi; i += threads) {
      float f[E];
      value(i, f);
      store_vec<E>(g0 + static_cast<int64_t>(i) * E, f);
    }
    if (lo == 0 && hi == sl.nv) return;
  }
  // element by element: the row's ends, or all of it
  for (int i = tid; i < sl.nv; i += threads) {
    if (aligned && i >= lo && i < hi) continue;
    float f[E];
    value(i, f);
    const int e = sl.first_element(i);
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (e + j >= 0 && e + j < sl.vocab) grow[e + j] = Out<G>::one(f[j]);
  }
}

// The gradient outside the list: mul 2^(c x - ref), or mul 2^((x - m) c - ref) where the reference is far.
struct Outside {
  float ref, mul, m;
  bool far;
};

template <typename T, typename G>
__device__ __noinline__ void write_far_grad(const Slice<T> sl, const uint4* slice, G* grow, int tid, int threads, const Outside o, float c) {
  for (int i = tid; i < sl.nv; i += threads) {
    float f[Elem<T>::kPer];
    unpack(slice[i], f, static_cast<const T*>(nullptr));
    const int e = sl.first_element(i);
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; ++j)
      if (e + j >= 0 && e + j < sl.vocab) grow[e + j] = Out<G>::one(o.mul * ex2_approx(fmaf(f[j] - o.m, c, -o.ref)));
  }
}
template <typename T, typename G>
__device__ __forceinline__ void write_tail_grad(const Slice<T>& sl, const uint4* slice, G* grow, int tid, int threads, const Outside o,
                                                float c) {
  if (o.far) {
    write_far_grad<T, G>(sl, slice, grow, tid, threads, o, c);
    return;
  }
  const uint64_t c2 = pack_f32x2(c, c), r2 = pack_f32x2(-o.ref, -o.ref);
  const float mul = o.mul;
  write_grad<T, G>(sl, grow, tid, threads, [&](int i, float* f) {
    unpack(slice[i], f, static_cast<const T*>(nullptr));
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; j += 2) {
      const uint64_t y = fma_f32x2(pack_f32x2(f[j], f[j + 1]), c2, r2);
      f[j] = mul * ex2_approx(lo_f32x2(y));
      f[j + 1] = mul * ex2_approx(hi_f32x2(y));
    }
  });
}

// A row's sums: its maximum, the tail's with the sum of the tail's terms against that (in units of the row's maximum a tail
// that is far below would be 0), and the sum of the list's terms against the row's maximum.
struct __align__(16) RowSums {
  float all, tail_max, tail, in;
};
// `in` against the list's own maximum.
__device__ __forceinline__ RowSums join_sums(float tail_max, float tail, float list_max, float in, float c) {
  const float all = fmaxf(tail_max, list_max);
  float unused = 0.f;
  rebase(list_max, c, all, reference(all, c), in, unused);
  return RowSums{all, tail_max, tail, in};
}

// A warp's {maximum, sum} of the tail as one.
__device__ __forceinline__ float2 join_parts(float2 v, float c) {
  const float m = key_value(__reduce_max_sync(0xffffffffu, order_key(v.x)));
  float unused = 0.f;
  rebase(v.x, c, m, reference(m, c), v.y, unused);
  return make_float2(m, warp_sum(v.y));
}
// From the parts of the tail {maximum, sum} and the list's logits, two a lane (a whole warp; every lane gets them).
__device__ __forceinline__ RowSums sums_with_list(float2 v, float z0, float z1, float c) {
  const float list_max = key_value(__reduce_max_sync(0xffffffffu, max(order_key(z0), order_key(z1))));
  const float2 tail = join_parts(v, c);
  const float all = fmaxf(tail.x, list_max), R = reference(all, c);
  const float in = warp_sum(ex2_approx(exponent(z0, all, R, c)) + ex2_approx(exponent(z1, all, R, c)));
  return RowSums{all, tail.x, tail.y, in};
}

// From the CTAs' parts {the tail's maximum and sum, the list's} (a whole warp; every lane gets them).
__device__ __forceinline__ RowSums row_sums(const float4* slot, int n_ctas, float c) {
  const int lane = lane_id();
  float4 v = make_float4(-kInf, 0.f, -kInf, 0.f);
  if (lane < n_ctas) v = slot[lane];
  const float tail_max = key_value(__reduce_max_sync(0xffffffffu, order_key(v.x)));
  const float list_max = key_value(__reduce_max_sync(0xffffffffu, order_key(v.z)));
  float unused = 0.f;
  rebase(v.x, c, tail_max, reference(tail_max, c), v.y, unused);
  rebase(v.z, c, list_max, reference(list_max, c), v.w, unused);
  return join_sums(tail_max, warp_sum(v.y), list_max, warp_sum(v.w), c);
}

// Sums of two floats, hi + lo, for a row's scalars.  (fp64 instructions take some 15 cycles a warp here: a
// division of them costs more than a row's exponentials do.)
struct Float2 {
  float hi, lo;
};
__device__ __forceinline__ Float2 two_sum(float a, float b) {  // a + b exactly
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  return Float2{s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Float2 operator+(Float2 a, Float2 b) {
  const Float2 s = two_sum(a.hi, b.hi);
  return Float2{s.hi, s.lo + (a.lo + b.lo)};
}
__device__ __forceinline__ Float2 operator-(Float2 a) { return Float2{-a.hi, -a.lo}; }
__device__ __forceinline__ Float2 two_prod(float a, float b) {  // a b exactly
  const float p = __fmul_rn(a, b);
  return Float2{p, fmaf(a, b, -p)};
}
// ln(j / 16), j = 8 .. 16, in two parts (constant memory: a load from global memory takes microseconds here).
__constant__ float kLnHigh[9] = {-0.693147182f, -0.575364172f, -0.470003635f, -0.374693453f, -0.287682086f,
                                     -0.207639366f, -0.133531392f, -0.0645385236f, 0.f};
__constant__ float kLnLow[9] = {1.90465421e-09f, 2.75550871e-08f, 5.44550272e-09f,  3.87050969e-09f, 1.37775436e-08f,
                                    1.61007641e-09f, -1.00388664e-09f, 2.41723086e-09f, 0.f};
// ln x of a normal x > 0, to some 4e-9: the exponent times ln 2 in two parts (the first one short: e times it is
// exact), the logarithm of the nearest j / 16 to the significand, and log1pf of what is left (at most 1 / 16).
__device__ __forceinline__ Float2 ln2parts(float x) {
  int e = 0;
  const float f = 16.f * frexpf(x, &e), j = rintf(f), n = static_cast<float>(e);
  const int i = min(max(static_cast<int>(j) - 8, 0), 8);  // (x may be no number)
  return Float2{n * 0.693145751953125f, n * 1.42860677e-6f} + Float2{kLnHigh[i], kLnLow[i]} + Float2{log1pf((f - j) / j), 0.f};
}

// What a row's list adds up to: Q in two parts, and q_T.
struct ListSums {
  float Q, Q_lo, q_tail;
};
__device__ __forceinline__ ListSums list_sums(double Q, bool bucket) {
  const float hi = static_cast<float>(Q), lo = static_cast<float>(Q - hi);
  return ListSums{hi, lo, bucket ? fmaxf(0.f, (1.f - hi) - lo) : 0.f};
}

// Whether a renormalised list's largest entry ln q is so low or high that exponentials lose bits or are out of range:
// then they are taken against it, as only their ratios count.
__device__ __forceinline__ bool out_of_scale(float top) { return fabsf(top) > 60.f && top > -kInf; }

// The scalars of a row's gradient: p_j = inv_s 2^y, y its exponent against (m, R); inside the list the gradient is
// p_j f_in - q q_in.  (m is the row's maximum.)
struct RowScale {
  float R, inv_s, f_in, q_in;
  float ref, mul;  // of the gradient outside
  float tail, s;   // the tail's sum, and that of all, against the row's maximum
  bool empty;
  bool pulls;      // the list leaves the tail a probability, and there is one
};

__device__ __forceinline__ RowScale row_scale(const RowSums& r, const ListSums& l, float w, float scale, bool bucket, float c) {
  RowScale o;
  o.R = reference(r.all, c);
  const float R_tail = reference(r.tail_max, c);
  const float to_all = r.tail_max == -kInf ? 0.f : ex2_approx(shift(r.tail_max, R_tail, r.all, o.R, c));
  o.tail = r.tail * to_all;
  o.s = o.tail + r.in;
  o.empty = r.all == -kInf && o.s == 0.f;  // every logit -inf: p = 0
  o.inv_s = o.empty ? 0.f : 1.f / o.s;
  o.pulls = bucket && r.tail > 0.f && l.q_tail > 0.f;
  const float ws = w * scale;
  o.q_in = bucket ? ws : ws / l.Q;
  // p's factor is the weight of all terms: 1, or Q where a tail that is masked altogether leaves the second term out
  o.f_in = bucket && l.q_tail > 0.f && r.tail == 0.f ? ws * l.Q : ws;
  // w scale p_j (1 - q_T / p_T) = F 2^y, F = w scale (2^d / s - q_T / tail) with y and tail against the tail's maximum, d from
  // there to the row's.  F's exponent k goes into the reference; what rounding the reference takes goes into the
  // factor.
  const float g = o.pulls ? o.inv_s * to_all - l.q_tail / r.tail : o.inv_s;
  int k = 0, k2 = 0;
  float f = ws * g;
  if (isfinite(ws) && isfinite(g)) f = frexpf(g, &k) * frexpf(ws, &k2);
  const float R = o.pulls ? R_tail : o.R;
  const Float2 ref = two_sum(is_far(R) ? 0.f : R, -static_cast<float>(k + k2));
  o.ref = ref.hi;
  o.mul = f * ex2_approx(-ref.lo);
  return o;
}

__device__ __forceinline__ Outside outside(const RowScale& o, const RowSums& r, float c) {
  const float m = o.pulls ? r.tail_max : r.all;
  return Outside{o.ref, o.mul, m, is_far(reference(m, c))};
}

// The loss (a whole warp; every lane gets it), from entries lane, lane + 32, ... of the list.  Where the two
// models agree it is a difference of terms some ten to a thousand times its size, so that these are kept apart:
//   - the list's sum is taken anew, with expf of exponents that are not rounded, and added up in fp64 (an error of
//     1e-7 in it moved losses by 2e-6; one of the tail's sum cancels);
//   - ln q - ln p is a sum of pairs of floats, and the terms are added up in fp64;
//   - ln q_T - ln p_T is ln(1 + (in - Q s) / tail), unless the tail is far below.
template <int N>
__device__ __forceinline__ float row_loss(const RowScale& o, const RowSums& r, const ListSums& l, float w, bool bucket, float scale,
                                          float c, const float (&q)[N], const float (&lq)[N], const float (&z)[N]) {
  if (o.s != o.s) return kNan;  // (NaN or +inf in the row, wherever it stands, also where the list has no weight)
  // in units of e^(scale m), m the row's maximum: the sums hold 2^delta of it, delta = c m - R
  const float delta = delta_of(r.all, c, o.R);
  Float2 x[N];  // scale (z - m)
  double sum = 0.0;
#pragma unroll
  for (int h = 0; h < N; ++h) {
    const Float2 d = two_sum(z[h], -r.all), p = two_prod(d.hi, scale);
    x[h] = Float2{p.hi, fmaf(d.lo, scale, p.lo)};
    if (!isfinite(p.hi)) x[h] = Float2{-kInf, 0.f};  // (out of fp32's range, or z is -inf)
    if (q[h] == 0.f || z[h] == -kInf) continue;  // no entry, or no weight (left to `in`), or no probability
    const float e = expf(x[h].hi);
    sum += static_cast<double>(fmaf(e, x[h].lo, e));
  }
  sum = warp_sum(sum);
  // what has no weight in the list belongs to its sum too; then the sum is taken as it is
  bool all_weighted = true;
#pragma unroll
  for (int h = 0; h < N; ++h) all_weighted &= !(q[h] == 0.f && z[h] > -kInf);
  const float tail = o.tail * ex2_approx(-delta);
  const float in0 = r.in * ex2_approx(-delta);
  const bool anew = __all_sync(0xffffffffu, all_weighted) && r.all > -kInf;
  const float in = anew ? static_cast<float>(sum) : in0, in_lo = anew ? static_cast<float>(sum - in) : 0.f;
  const Float2 s = Float2{tail, 0.f} + Float2{in, in_lo};
  const Float2 ln_s = ln2parts(s.hi) + Float2{s.lo / s.hi, 0.f};
  double terms = 0.0;
#pragma unroll
  for (int h = 0; h < N; ++h) {
    if (q[h] == 0.f) continue;  // (a NaN is no 0)
    const Float2 diff = Float2{lq[h], 0.f} + -x[h] + ln_s;
    if (x[h].hi > -kInf) terms += q[h] * (diff.hi + diff.lo);
    else terms += o.empty || z[h] == -kInf ? q[h] * kInf : -q[h] * scale * (static_cast<double>(z[h]) - r.all);
  }
  terms = warp_sum(terms);
  const float hi = static_cast<float>(terms);
  if (!isfinite(hi)) return w * hi;
  if (!bucket) {  // terms / Q - ln Q
    const float q1 = hi / l.Q, rest = fmaf(-q1, l.Q, hi) + static_cast<float>(terms - hi) - q1 * l.Q_lo;
    const Float2 L = Float2{q1, rest / l.Q} + -ln2parts(l.Q) + Float2{-l.Q_lo / l.Q, 0.f};
    return w * (L.hi + L.lo);
  }
  double of_tail = 0.0;
  if (o.pulls && tail < 1e-18f * s.hi) {
    const float delta_tail = delta_of(r.tail_max, c, reference(r.tail_max, c));
    const double below = scale * (static_cast<double>(r.tail_max) - r.all);  // (may be out of fp32's range)
    of_tail = l.q_tail * (logf(l.q_tail) - (logf(r.tail) - delta_tail * kLn2) + (ln_s.hi + ln_s.lo) - below);
  } else if (o.pulls) {
    const Float2 qs = two_prod(l.Q, s.hi);
    const float off = (((in - qs.hi) - qs.lo) + in_lo - l.Q_lo * s.hi - l.Q * s.lo) / tail;
    of_tail = l.q_tail * (off > -0.5f ? log1pf(off) : logf(l.q_tail) - logf(tail / s.hi));
  }
  return w * static_cast<float>(terms + of_tail);
}

template <typename T>
cudaError_t distill_stream(const DistillArgs& p, int grad_dtype, cudaStream_t s);  // distill_stream.cu
constexpr int64_t kManyBytes = 48 << 20;     // of all rows
constexpr int64_t kShortGradRow = 32 * 1024;  // bytes of a row, with a gradient
bool distill_stream_pays(int rows, int64_t row_bytes, bool grad);

}  // namespace rows
}  // namespace sgd
