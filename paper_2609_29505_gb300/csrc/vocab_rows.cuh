// Rows of logits held on chip: what the scoring and the distillation kernel share.
//
// A row (126464 fp16 values are 253 KB) is read from HBM once.  The CTAs of a cluster take a slice
// of it each into shared memory by bulk copies, so that passes over the row after the first (the
// likeliest tokens, the gradient) cost no traffic; a few numbers per CTA cross the cluster.
// A slice is cut at 16-byte boundaries of the address, whatever the row's own alignment: vector v
// of a row holds its elements v E - shift .. v E - shift + E - 1, E = 16 / sizeof(T), and what lies
// before the row's first or after its last element is filled with -inf.
#pragma once

#include <atomic>

#include "common.cuh"
#include "kernels.h"

namespace sgd {
namespace rows {

constexpr int kUnroll = 4;      // vectors a thread takes at a time
constexpr int kPiece = 1024;    // vectors of one bulk copy (16 KB), with a barrier of its own
constexpr int kMaxPieces = 13;  // of a slice: 208 KB
constexpr int kMaxCluster = 16;
constexpr float kInf = __builtin_huge_valf(), kNan = __builtin_nanf("");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T>
struct Elem {
  static constexpr int kPer = 16 / static_cast<int>(sizeof(T));
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(f16 x) { return __half2float(x); }
__device__ __forceinline__ float to_f(bf16 x) { return __bfloat162float(x); }

template <typename T>
__device__ __forceinline__ T neg_inf();
template <>
__device__ __forceinline__ float neg_inf<float>() { return -kInf; }
template <>
__device__ __forceinline__ f16 neg_inf<f16>() { return __ushort_as_half(0xFC00u); }
template <>
__device__ __forceinline__ bf16 neg_inf<bf16>() { return __ushort_as_bfloat16(0xFF80u); }

__device__ __forceinline__ void unpack(const uint4& u, float* f, const float*) {
  f[0] = __uint_as_float(u.x);
  f[1] = __uint_as_float(u.y);
  f[2] = __uint_as_float(u.z);
  f[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack(const uint4& u, float* f, const f16*) { unpack_f16x8(u, f); }
__device__ __forceinline__ void unpack(const uint4& u, float* f, const bf16*) { unpack_bf16x8(u, f); }

// Largest value of n vectors; a NaN is passed over (its exponential makes the row's sum NaN).
template <int N>
__device__ __forceinline__ float vec_max(const uint4* v, const float*) {
  float m = __uint_as_float(v[0].x);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    m = max3(m, __uint_as_float(v[i].x), __uint_as_float(v[i].y));
    m = max3(m, __uint_as_float(v[i].z), __uint_as_float(v[i].w));
  }
  return m != m ? -kInf : m;
}
template <int N, typename P>
__device__ __forceinline__ float vec_max_packed(const uint4* v) {
  const P* p = reinterpret_cast<const P*>(v);
  P m = p[0];
#pragma unroll
  for (int i = 1; i < 4 * N; ++i) m = __hmax2(m, p[i]);
  const float r = fmaxf(to_f(m.x), to_f(m.y));
  return r != r ? -kInf : r;
}
template <int N>
__device__ __forceinline__ float vec_max(const uint4* v, const f16*) { return vec_max_packed<N, __half2>(v); }
template <int N>
__device__ __forceinline__ float vec_max(const uint4* v, const bf16*) { return vec_max_packed<N, __nv_bfloat162>(v); }

// Smallest value of n vectors; a NaN is passed over.
template <int N>
__device__ __forceinline__ float vec_min(const uint4* v, const float*) {
  float m = __uint_as_float(v[0].x);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    m = min3(m, __uint_as_float(v[i].x), __uint_as_float(v[i].y));
    m = min3(m, __uint_as_float(v[i].z), __uint_as_float(v[i].w));
  }
  return m;
}
template <int N, typename P>
__device__ __forceinline__ float vec_min_packed(const uint4* v) {
  const P* p = reinterpret_cast<const P*>(v);
  P m = p[0];
#pragma unroll
  for (int i = 1; i < 4 * N; ++i) m = __hmin2(m, p[i]);
  return fminf(to_f(m.x), to_f(m.y));
}
template <int N>
__device__ __forceinline__ float vec_min(const uint4* v, const f16*) { return vec_min_packed<N, __half2>(v); }
template <int N>
__device__ __forceinline__ float vec_min(const uint4* v, const bf16*) { return vec_min_packed<N, __nv_bfloat162>(v); }

// Order of fp32 values as unsigned integers: -0 and +0 are equal, NaN stands with -inf.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  if (x != x) return 0x007FFFFFu;  // -inf's
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
constexpr uint32_t kKeyNegInf = 0x007FFFFFu;
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

// Where a CTA's slice of a row lies.
template <typename T>
struct Slice {
  const T* row;
  int vocab;
  int shift;  // elements between the 16-byte boundary at or before the row and the row
  int total;  // vectors of the whole row
  int v0;     // first vector of this CTA
  int nv;     // its vectors (0: none)

  __device__ Slice(const T* r, int n, int rank, int n_ctas) : row(r), vocab(n) {  // n_ctas: a power of two
    constexpr int E = Elem<T>::kPer;
    shift = static_cast<int>((reinterpret_cast<uintptr_t>(r) & 15u) / sizeof(T));
    total = (shift + vocab + E - 1) / E;
    const int per = (total + n_ctas - 1) >> (31 - __clz(n_ctas));
    v0 = rank * per;
    nv = min(per, total - v0);
    if (nv < 0) nv = 0;
  }
  __device__ int first_element(int i) const { return (v0 + i) * Elem<T>::kPer - shift; }  // of local vector i
  __device__ bool whole(int i) const {
    const int e = first_element(i);
    return e >= 0 && e + Elem<T>::kPer <= vocab;
  }
  // local vector i from global memory
  __device__ uint4 fetch(int i) const {
    const T* at = row + first_element(i);
    if (whole(i)) return *reinterpret_cast<const uint4*>(at);
    return gather(i);
  }
  // one that is not whole: -inf where there is no element
  __device__ uint4 gather(int i) const {
    const int e = first_element(i);
    uint4 v;
    T* f = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; ++j) f[j] = e + j >= 0 && e + j < vocab ? row[e + j] : neg_inf<T>();
    return v;
  }
  // local vector that holds element e, or -1
  __device__ int vector_of(int e) const {
    const int i = (e + shift) / Elem<T>::kPer - v0;
    return i >= 0 && i < nv ? i : -1;
  }
  __device__ int place_of(int e) const { return (e + shift) % Elem<T>::kPer; }
};

// Starts the slice's bulk copies (thread 0; the barriers are initialised) and fills the row's ragged
// ends (their first and last vector) with ordinary loads.  Those need a __syncthreads before use.
template <typename T>
__device__ __forceinline__ void start_copies(const Slice<T>& s, uint4* buf, uint64_t* bars) {
  const char* src = reinterpret_cast<const char*>(s.row) - s.shift * static_cast<int>(sizeof(T)) +
                    static_cast<int64_t>(s.v0) * 16;
  const int lo = s.nv > 0 && !s.whole(0) ? 1 : 0;
  const int hi = s.nv > 0 && !s.whole(s.nv - 1) ? s.nv - 1 : s.nv;  // whole vectors are [lo, hi)
  for (int p = 0; p * kPiece < s.nv; ++p) {
    const int a = max(p * kPiece, lo), b = min((p + 1) * kPiece, hi);
    const uint32_t bytes = b > a ? static_cast<uint32_t>(b - a) * 16u : 0u;
    mbar_arrive_expect_tx(&bars[p], bytes);
    if (bytes) bulk_load(buf + a, src + static_cast<int64_t>(a) * 16, bytes, &bars[p]);
  }
}
template <typename T>
__device__ __forceinline__ void fill_ends(const Slice<T>& s, uint4* buf) {
  constexpr int E = Elem<T>::kPer;
  const int w = threadIdx.x / E, j = threadIdx.x % E;
  if (w > 1 || s.nv == 0) return;
  const int i = w ? s.nv - 1 : 0;
  if (s.whole(i) || (w && i == 0)) return;
  const int e = s.first_element(i) + j;
  reinterpret_cast<T*>(buf + i)[j] = e >= 0 && e < s.vocab ? s.row[e] : neg_inf<T>();
}

// Waits for piece p of the slice.  After an expired wait (recorded in the status word) the kernel
// goes on with what is there, as every barrier of the cluster has to be reached; the copies are
// waited for once more, so that none lands after the CTA has left.
__device__ __forceinline__ void wait_piece(uint64_t* bars, int p, volatile int* abort_flag, int* status, int code) {
  if (!mbar_wait_warp(smem_u32(&bars[p]), 0, abort_flag, status, code)) mbar_drain(&bars[p], 0);
}

// Exponents are taken in base 2 against a reference, with c = scale log2(e) and the largest value m:
//   x c - R, R = fl(m c): one rounding (an fma).  R's own rounding is taken back at the end, through
//   delta = m c - R = fma(m, c, -R), so that ln sum e^(scale (x - m)) = ln s - delta ln 2.
//   (x - m) c where |m c| is above kFar, as R's rounding would then be an exponent of its own (half a unit of R
//   passes 128 at 2^32, and R overflows for a mask of the type's lowest value).  The reference is m c
//   itself, delta = 0.
constexpr float kFar = 1048576.f;  // 2^20: delta is below 2^-4
// Exponents below this are cut: 2^x is 0 there, and a sum's factor stays finite.
constexpr float kCut = -1000.f;

__device__ __forceinline__ float reference(float m, float c) { return m == -kInf ? 0.f : __fmul_rn(m, c); }
__device__ __forceinline__ bool is_far(float R) { return fabsf(R) > kFar; }
__device__ __forceinline__ float delta_of(float m, float c, float R) {
  return m == -kInf || is_far(R) ? 0.f : fmaf(m, c, -R);
}

// Exponent of x against the reference (m, R).
__device__ __forceinline__ float exponent(float x, float m, float R, float c) {
  return is_far(R) ? __fmul_rn(x - m, c) : fmaf(x, c, -R);
}
// From the reference (m1, R1) to that of M >= m1: what is added to exponents.
__device__ __forceinline__ float shift(float m1, float R1, float M, float R, float c) {
  float d = R1 - R;
  if (is_far(R1) || is_far(R)) d = fmaf(m1 - M, c, delta_of(M, c, R) - delta_of(m1, c, R1));
  return fmaxf(d, kCut);  // (a NaN, of infinities, too)
}

// Running softmax statistics of one thread: s = sum 2^y and, where ENT, t = sum y 2^y over y = x c - R.  R is at least
// -kFar here: where the thread's values lie below, their terms are as small as they come out beside what other
// threads of the warp have, or the warp's maximum is far itself.  Then, and where a value is far above, warp_stat()
// takes the sums anew.
struct Stat {
  float m = -kInf, R = 0.f, s = 0.f, t = 0.f;
};

template <typename T, int N, bool ENT, bool CUT>
__device__ __forceinline__ void add_terms(Stat& st, const uint4* v, float c) {
  const uint64_t c2 = pack_f32x2(c, c), r2 = pack_f32x2(-st.R, -st.R);
  uint64_t s2 = pack_f32x2(st.s, 0.f), t2 = pack_f32x2(st.t, 0.f);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float f[Elem<T>::kPer];
    unpack(v[i], f, static_cast<const T*>(nullptr));
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; j += 2) {
      uint64_t y = fma_f32x2(pack_f32x2(f[j], f[j + 1]), c2, r2);
      const uint64_t e = pack_f32x2(ex2_approx(lo_f32x2(y)), ex2_approx(hi_f32x2(y)));
      s2 = add_f32x2(s2, e);
      if (CUT) y = pack_f32x2(fmaxf(lo_f32x2(y), kCut), fmaxf(hi_f32x2(y), kCut));
      if (ENT) t2 = fma_f32x2(y, e, t2);
    }
  }
  st.s = sum_f32x2(s2);
  if (ENT) st.t = sum_f32x2(t2);
}

// Values up to this one have an exponent that may overflow: x c is above -2^127 where x is above it.
__device__ __forceinline__ float lowest_value(float c) { return fmaxf(-1.5e38f / c, -3.4028234e38f); }

// Takes N vectors in, whose largest value is returned.  The maximum moves at most once per call: no
// rescaling per element.
template <typename T, int N, bool ENT>
__device__ __forceinline__ float stat_add(Stat& st, const uint4* v, float c, float lowest) {
  const float m = vec_max<N>(v, static_cast<const T*>(nullptr));
  if (m > st.m) {
    const float R = fmaxf(__fmul_rn(m, c), -kFar);
    if (st.m != -kInf) {
      const float d = st.R - R, f = ex2_approx(d);
      if (ENT) st.t = f * (st.t + d * st.s);
      st.s *= f;
    }
    st.m = m;
    st.R = R;
  }
  // a masked token (-inf, or a value whose exponent overflows) has the term 0 in t, not -inf times 0: its exponent
  // is cut, where there is one
  if (ENT && vec_min<N>(v, static_cast<const T*>(nullptr)) <= lowest) add_terms<T, N, true, true>(st, v, c);
  else add_terms<T, N, ENT, false>(st, v, c);
  return m;
}

// A vector without an element: of a slice's end.
template <typename T>
__device__ __forceinline__ uint4 no_elements() {
  uint4 v;
  T* e = reinterpret_cast<T*>(&v);
#pragma unroll
  for (int j = 0; j < Elem<T>::kPer; ++j) e[j] = neg_inf<T>();
  return v;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// s and t of a part with maximum m at the reference (M, R) of a maximum M >= m.
__device__ __forceinline__ void rebase(float m, float c, float M, float R, float& s, float& t) {
  const float d = shift(m, reference(m, c), M, R, c), f = m == -kInf ? 0.f : ex2_approx(d);
  t = m == -kInf ? 0.f : f * (t + d * s);
  s *= f;
}

// Vector i of a slice in shared memory.
struct InShared {
  const uint4* buf;
  __device__ uint4 operator()(int i) const { return buf[i]; }
};

// A warp's statistics {maximum, s, t} from its threads'.  Where its maximum is far the sums are taken anew over the
// threads' vectors, which fetch(i) gives for i = tid, tid + threads, ... below nv.
template <typename T, bool ENT, typename F>
__device__ __noinline__ float2 far_sums(float m, float c, int tid, int threads, int nv, F fetch) {
  float s = 0.f, t = 0.f;
#pragma unroll 1
  for (int i = tid; i < nv; i += threads) {
    float x[Elem<T>::kPer];
    unpack(fetch(i), x, static_cast<const T*>(nullptr));
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; ++j) {
      const float y = __fmul_rn(x[j] - m, c), e = ex2_approx(y);
      s += e;
      if (ENT) t = fmaf(fmaxf(y, kCut), e, t);
    }
  }
  return make_float2(s, t);
}
template <typename T, bool ENT, typename F>
__device__ __forceinline__ float3 warp_stat(const Stat& st, float c, int tid, int threads, int nv, const F& fetch) {
  const float m = key_value(__reduce_max_sync(0xffffffffu, order_key(st.m)));
  const float R = reference(m, c);
  float s = 0.f, t = 0.f;
  if (!is_far(R)) {
    const float d = st.R - R, f = st.m == -kInf ? 0.f : ex2_approx(d);
    t = st.m == -kInf ? 0.f : f * (st.t + d * st.s);
    s = st.s * f;
  } else {
    const float2 a = far_sums<T, ENT>(m, c, tid, threads, nv, fetch);
    s = a.x;
    t = a.y;
  }
  return make_float3(m, warp_sum(s), ENT ? warp_sum(t) : 0.f);
}

__device__ __forceinline__ void st_cluster(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
               : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ uint32_t cluster_ctas() {
  uint32_t n;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
  return n;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// kN threads of a CTA (whole warps) with a hardware barrier of their own.
template <int kN, int kBar>
struct Team {
  static constexpr int kSize = kN, kWarps = kN / 32;
  int tid;
  __device__ void sync() const { asm volatile("barrier.cta.sync.aligned %0, %1;" ::"n"(kBar), "n"(kN) : "memory"); }
  // number of threads whose predicate holds; a barrier as well
  __device__ int count(bool p) const {
    int n;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %1, 0;\n\t"
        "barrier.cta.red.popc.aligned.u32 %0, %2, %3, p;\n\t}"
        : "=r"(n)
        : "r"(static_cast<int>(p)), "n"(kBar), "n"(kN)
        : "memory");
    return n;
  }
};

// The same for one warp.
struct WarpTeam {
  static constexpr int kSize = 32, kWarps = 1;
  int tid;
  __device__ void sync() const { __syncwarp(); }
  __device__ int count(bool p) const { return __popc(__ballot_sync(0xffffffffu, p)); }
};

// Grid: a cluster per row.  The cluster size is a power of two: slices of at most kSlice bytes, and
// smaller ones where there are too few rows to fill the SMs.  (Slices of 64 KB, 32 KB and 128 KB: 414, 503 and
// 546 us for 4096 x 126464 fp16 with lists of 32, before such rows streamed.)
struct Launch {
  int cluster;
  int slice_bytes;
  int threads;
};
constexpr int kSlice = 64 * 1024;
// Vectors of a slice that 64 threads take instead of 256: what a row costs beside its elements (barriers,
// reductions) is then a quarter.  512 MB of 2000 fp16 logits a row, 64 threads against 256: 440 / 827 us scored, 675 / 1464
// us for a loss, 765 / 1599 us with a gradient; of 4000 to 4200: 250 / 430, 351 / 704, 423 / 783 us.
constexpr int kShortSlice = 512;
constexpr int kMaxDynamic = (227 - 16) * 1024;  // beside at most 16 KB of static shared memory

inline Launch plan(int rows, int64_t vocab, int elem) {
  const int64_t bytes = vocab * elem;
  int c = 1;
  while (c < kMaxCluster && (bytes + c - 1) / c > kSlice) c *= 2;
  while (c < kMaxCluster && static_cast<int64_t>(rows) * c < num_sms() && bytes / c > 8192) c *= 2;
  const int64_t total = (bytes + 15) / 16 + 1;  // (one more vector where the row starts inside one)
  const int vectors = static_cast<int>((total + c - 1) / c);
  return Launch{c, vectors * 16, vectors <= kShortSlice ? 64 : 256};
}

template <auto kKernel, typename... Args>
cudaError_t launch(int rows, const Launch& l, size_t smem, cudaStream_t stream, Args... args) {
  // once per kernel and device: dynamic shared memory up to the SM's, clusters of more than 8
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev > 63 || !(ready.load() >> dev & 1)) {
    e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxDynamic);
    if (e != cudaSuccess) return e;
    e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    if (dev <= 63) ready.fetch_or(1ull << dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows) * l.cluster);
  cfg.blockDim = dim3(l.threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = l.cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kKernel, args...);
}

}  // namespace rows
}  // namespace sgd
