// Backward pass of the norms: with xhat = (h - mean) rstd (mean 0 for an RMS norm), n = xhat g + b and
// out = n (1 + scale) + shift, given dout:
//   dn = dout (1 + scale), dx = dn g,
//   dh = rstd (dx - mean(dx) - xhat mean(dx xhat)) + residual   (without mean(dx) for an RMS norm),
//   dg = sum dn xhat, db = sum dn over all rows;  dshift = sum dout, dscale = sum dout n over a sample's rows.
//
// All four come from two sums over a sample's rows, A = sum dout and B = sum dout xhat, per column: dshift = A, dscale = g B + b A,
// db = sum over samples of (1 + scale) A, dg = the same of B.  A group of threads takes a row at a time, keeps its columns'
// A and B in registers over all of its rows, and leaves them in the workspace; a second kernel adds them up in a fixed
// order.  The statistics are taken anew from h, which has to be read for xhat anyway.
//
// HBM bounds it, and the chain of a row (statistics, two sums, the result) where rows are few: 4096 x 4096 with bf16 dout and a
// residual 44.5 us, 39 of them the rows (6.0 TB/s of 6.7), the rest 304 pairs of sums; 2048 x 1152 modulated, 8 samples: 15 us, 14 for 5
// rows a group one after another.
#include <atomic>

#include "common.cuh"
#include "kernels.h"

namespace sgd {
namespace {

constexpr int kThreads = 256;
constexpr int kSms = 152;        // of a GB300
constexpr int kRowsPerPart = 3;  // of a sample that several groups share, at least
constexpr int kColsPerCta = 16;  // of the second kernel: 4 threads of 4 columns
constexpr int kShares = 64;      // and as many shares of the sums as there are threads

// Threads of a row: vectors of 4 columns each, two at most, and four in rows of more than 2048 (`wide`): 4096 columns with a residual are
// 40 us per 4096 rows with 256 threads a row and two CTAs per SM, 57 with 512 and one, whose barriers nothing hides.
struct Group {
  int threads;
  bool wide;
};
Group group_of(int d) {
  if (d > 2048) return {256, true};
  int g = 32;
  while (g * 8 < d) g *= 2;
  return {g, false};
}
constexpr int vectors_of(bool wide) { return wide ? 4 : 2; }
constexpr int ctas_per_sm(bool wide) { return wide ? 2 : 3; }
// Narrow rows: how many a group has in hand or on their way, and bytes of shared memory: theirs, and two rows of dh.
constexpr int kStages = 2;
constexpr int smem_of(bool wide, int elem) { return wide ? 0 : kThreads * 2 * (kStages * (32 + 4 * elem) + 32); }
static_assert(kColsPerCta == 16 && kShares == 64, "256 threads");
static_assert(3 * (smem_of(false, 4) + 9 * 1024) <= 226 * 1024, "shared memory");

struct Plan {
  int group, groups;  // threads of a row; rows at a time in a CTA
  bool wide;
  int per, samples;   // rows of a sample
  int parts, part;    // shares of a sample, rows of one
  int ctas, units;    // units: sums in the workspace
};
// per 0: no modulation (one sample; a CTA's groups join their sums)
Plan make_plan(int rows, int d, int per) {
  Plan q{};
  const Group g = group_of(d);
  q.group = g.threads;
  q.wide = g.wide;
  q.groups = kThreads / q.group;
  const int most_ctas = ctas_per_sm(q.wide) * kSms;
  if (per <= 0) {
    q.per = rows;
    q.samples = 1;
    q.ctas = (rows + q.groups - 1) / q.groups;
    if (q.ctas > most_ctas) q.ctas = most_ctas;
    q.parts = q.units = q.ctas;
    return q;
  }
  if (per > rows) per = rows;  // one sample (whatever period says so: rows + per stays in 32 bits)
  q.per = per;
  q.samples = (rows + per - 1) / per;
  const int longest = per;
  q.parts = (most_ctas * q.groups + q.samples - 1) / q.samples;
  const int most = (longest + kRowsPerPart - 1) / kRowsPerPart;
  if (q.parts > most) q.parts = most;
  q.part = (longest + q.parts - 1) / q.parts;
  q.parts = (longest + q.part - 1) / q.part;
  const int64_t units = static_cast<int64_t>(q.samples) * q.parts;
  q.units = static_cast<int>(units);
  q.ctas = static_cast<int>((units + q.groups - 1) / q.groups);
  if (q.ctas > most_ctas) q.ctas = most_ctas;
  return q;
}

__device__ __forceinline__ float4 bf16x4(uint2 u) {
  const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
  const float2 c = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  return make_float4(a.x, a.y, c.x, c.y);
}
// Four values of dout, as they lie in memory and as numbers.
template <typename T>
struct Four {
  using Raw = uint2;
};
template <>
struct Four<float> {
  using Raw = float4;
};
__device__ __forceinline__ float4 numbers(float4 v, const float*) { return v; }
__device__ __forceinline__ float4 numbers(uint2 u, const bf16*) { return bf16x4(u); }
__device__ __forceinline__ float4 numbers(uint2 u, const f16*) {
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&u.x));
  const float2 c = __half22float2(*reinterpret_cast<const __half2*>(&u.y));
  return make_float4(a.x, a.y, c.x, c.y);
}

template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(dst)), "l"(__cvta_generic_to_global(src)), "n"(BYTES) : "memory");
}

struct Args {
  NormGradParams p;
  Plan q;
  float* sums;  // [units, 2, d]
};

// Sum of three values over a row's threads: two floats and, behind them, another (all are needed at once).
template <int G>
__device__ __forceinline__ float3 group_sum(float3 v, float (*red)[3], int warp_in_group, int barrier) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    v.z += __shfl_xor_sync(0xffffffffu, v.z, o);
  }
  if constexpr (G > 32) {
    if ((threadIdx.x & 31) == 0) {
      red[warp_in_group][0] = v.x;
      red[warp_in_group][1] = v.y;
      red[warp_in_group][2] = v.z;
    }
    asm volatile("barrier.cta.sync.aligned %0, %1;" ::"r"(barrier), "n"(G) : "memory");
    v = make_float3(0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < G / 32; ++i) {
      v.x += red[i][0];
      v.y += red[i][1];
      v.z += red[i][2];
    }
  }
  return v;
}

template <typename T, int G, bool WIDE, bool MOD, bool PARAMS>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(WIDE)) norm_grad_kernel(const Args a) {
  constexpr int NV = vectors_of(WIDE), kGroups = kThreads / G, kGroupWarps = G / 32;
  pdl_wait_and_trigger();
  using Raw = typename Four<T>::Raw;
  __shared__ float red[2][kThreads / 32][3];
  const NormGradParams& p = a.p;
  const int tid = threadIdx.x % G, grp = threadIdx.x / G, nv = p.d >> 2;
  const bool centred = p.kind != SGD_NORM_RMS;
  const float inv_d = 1.f / p.d;
  float (*my_red[2])[3] = {red[0] + grp * kGroupWarps, red[1] + grp * kGroupWarps};
  int flip = 0;
  auto total = [&](float3 v) {  // one barrier per sum: the buffers alternate
    v = group_sum<G>(v, my_red[flip], (threadIdx.x >> 5) % kGroupWarps, 1 + grp);
    flip ^= 1;
    return v;
  };
  uint2 g[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = tid + j * G;
    g[j] = make_uint2(0x3F803F80u, 0x3F803F80u);  // 1
    if (p.g && i < nv) g[j] = __ldg(reinterpret_cast<const uint2*>(p.g) + i);
  }
  float4 A[NV], B[NV], sc[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) A[j] = B[j] = sc[j] = make_float4(0.f, 0.f, 0.f, 0.f);

  // Narrow rows: h, dout and residual come by asynchronous copies into places that their thread alone reads; dh leaves from one of two rows in
  // shared memory, by a bulk copy that the group's first thread starts behind the next row's first barrier.
  extern __shared__ __align__(128) float4 dynamic[];
  constexpr int kPlaces = NV * kThreads;
  float4* h_in = dynamic + threadIdx.x;                 // [kStages][NV][kThreads]
  float4* res_in = h_in + kStages * kPlaces;            // the same
  float4* out = dynamic + 2 * kStages * kPlaces + grp * 2 * NV * G;  // [2][NV * G] of the group
  Raw* raw_in = reinterpret_cast<Raw*>(dynamic + 2 * kStages * kPlaces + 2 * kPlaces) + threadIdx.x;
  auto load = [&](int64_t row, int stage) {  // (row -1: none)
    if (row >= 0) {
      const int64_t at = row * p.d;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int i = tid + j * G, to = stage * kPlaces + j * kThreads;
        if (i < nv) {
          copy_async<16>(h_in + to, reinterpret_cast<const float4*>(p.h + at) + i);
          copy_async<sizeof(Raw)>(raw_in + to, reinterpret_cast<const Raw*>(static_cast<const T*>(p.dout) + at) + i);
          if (p.residual) copy_async<16>(res_in + to, reinterpret_cast<const float4*>(p.residual + at) + i);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // what lies behind the row's end, or has no residual, is 0
#pragma unroll
  for (int k = 0; k < (WIDE ? 0 : kStages * NV); ++k) {
    const bool behind = tid + k % NV * G >= nv;
    if (behind) {
      h_in[k * kThreads] = make_float4(0.f, 0.f, 0.f, 0.f);
      raw_in[k * kThreads] = Raw{};
    }
    if (behind || !p.residual) res_in[k * kThreads] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  int64_t stored = -1;  // row of dh that waits to be copied
  int flip_out = 0;
  auto store = [&] {  // behind a barrier of the group
    if (stored >= 0 && tid == 0) {
      bulk_store(p.dh + stored * p.d, out + (flip_out ^ 1) * NV * G, static_cast<uint32_t>(p.d) * 4);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    stored = -1;
  };
  // the first barrier of a row: the dh before the last has been read from shared memory, so that its place is free
  auto first_total = [&](float3 v) {
    if (WIDE) return total(v);
    if (tid == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    v = total(v);
    if (G == 32) __syncwarp();
    store();
    return v;
  };
  auto row_of = [&](int64_t row, int stage) {
    float4 x[NV], dx[NV], res[NV];
    Raw raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (WIDE) {
        const int i = tid + j * G;
        x[j] = res[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        raw[j] = Raw{};
        if (i < nv) {
          x[j] = reinterpret_cast<const float4*>(p.h + row * p.d)[i];
          raw[j] = reinterpret_cast<const Raw*>(static_cast<const T*>(p.dout) + row * p.d)[i];
          if (p.residual) res[j] = reinterpret_cast<const float4*>(p.residual + row * p.d)[i];
        }
      } else {
        const int at = stage * kPlaces + j * kThreads;
        x[j] = h_in[at];
        raw[j] = raw_in[at];
        res[j] = res_in[at];
      }
    }
    float mean = 0.f;
    if (centred) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) s += (x[j].x + x[j].y) + (x[j].z + x[j].w);
      mean = first_total(make_float3(s, 0.f, 0.f)).x * inv_d;
    }
    float3 s = make_float3(0.f, 0.f, 0.f);  // of x^2, dx, dx x
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const float4 dy = numbers(raw[j], static_cast<const T*>(nullptr)), gain = bf16x4(g[j]);
      dx[j] = make_float4(dy.x * gain.x, dy.y * gain.y, dy.z * gain.z, dy.w * gain.w);
      if (MOD) {
        dx[j].x *= 1.f + sc[j].x;
        dx[j].y *= 1.f + sc[j].y;
        dx[j].z *= 1.f + sc[j].z;
        dx[j].w *= 1.f + sc[j].w;
      }
      if (tid + j * G < nv) {
        x[j].x -= mean;
        x[j].y -= mean;
        x[j].z -= mean;
        x[j].w -= mean;
      }
      s.x += (x[j].x * x[j].x + x[j].y * x[j].y) + (x[j].z * x[j].z + x[j].w * x[j].w);
      s.y += (dx[j].x + dx[j].y) + (dx[j].z + dx[j].w);
      s.z += (dx[j].x * x[j].x + dx[j].y * x[j].y) + (dx[j].z * x[j].z + dx[j].w * x[j].w);
    }
    s = centred ? total(s) : first_total(s);
    const float rstd = rsqrtf(s.x * inv_d + p.eps);
    const float m1 = centred ? s.y * inv_d : 0.f, m2 = s.z * inv_d * rstd;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int i = tid + j * G;
      const float4 dy = numbers(raw[j], static_cast<const T*>(nullptr));
      x[j] = make_float4(x[j].x * rstd, x[j].y * rstd, x[j].z * rstd, x[j].w * rstd);
      if (PARAMS) {
        A[j].x += dy.x;
        A[j].y += dy.y;
        A[j].z += dy.z;
        A[j].w += dy.w;
        B[j].x = fmaf(dy.x, x[j].x, B[j].x);
        B[j].y = fmaf(dy.y, x[j].y, B[j].y);
        B[j].z = fmaf(dy.z, x[j].z, B[j].z);
        B[j].w = fmaf(dy.w, x[j].w, B[j].w);
      }
      if (p.dh && i < nv) {
        float4 v;
        v.x = fmaf(rstd, dx[j].x - m1 - x[j].x * m2, res[j].x);
        v.y = fmaf(rstd, dx[j].y - m1 - x[j].y * m2, res[j].y);
        v.z = fmaf(rstd, dx[j].z - m1 - x[j].z * m2, res[j].z);
        v.w = fmaf(rstd, dx[j].w - m1 - x[j].w * m2, res[j].w);
        if (WIDE) reinterpret_cast<float4*>(p.dh + row * p.d)[i] = v;
        else out[flip_out * NV * G + i] = v;
      }
    }
    if (!WIDE && p.dh) {
      fence_proxy_async_smem();
      stored = row;
      flip_out ^= 1;
    }
  };
  // rows from, from + step, ... below to
  auto rows = [&](int64_t from, int64_t to, int64_t step) {
    if constexpr (WIDE) {
      for (int64_t r = from; r < to; r += step) row_of(r, 0);
      return;
    }
#pragma unroll
    for (int k = 0; k < kStages - 1; ++k) load(from + k * step < to ? from + k * step : -1, k);
    int stage = 0;
    for (int64_t r = from; r < to; r += step) {
      const int64_t ahead = r + (kStages - 1) * step;
      load(ahead < to ? ahead : -1, stage == 0 ? kStages - 1 : stage - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      row_of(r, stage);
      if (++stage == kStages) stage = 0;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  };
  auto finish = [&] {  // the last row's dh
    if (WIDE) return;
    if (G == 32) __syncwarp();
    else asm volatile("barrier.cta.sync.aligned %0, %1;" ::"r"(1 + grp), "n"(G) : "memory");
    store();
    if (tid == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  };


  if (MOD) {
    // a group by itself: a share of a sample's rows at a time
    for (int u = blockIdx.x * kGroups + grp; u < a.q.units; u += gridDim.x * kGroups) {
      const int smp = u / a.q.parts, k = u - smp * a.q.parts;
      const int64_t r0 = static_cast<int64_t>(smp) * a.q.per;
      const int64_t end = min(r0 + a.q.per, static_cast<int64_t>(p.rows));
      const int64_t from = r0 + static_cast<int64_t>(k) * a.q.part, to = min(from + a.q.part, end);
      const float* scale = p.scale + static_cast<int64_t>(smp) * p.ld_mod;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int i = (tid + j * G) * 4;
        if (i < p.d) sc[j] = make_float4(scale[i], scale[i + 1], scale[i + 2], scale[i + 3]);
        if (PARAMS) A[j] = B[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      rows(from, to, 1);
      if (PARAMS) {
        float4* sums = reinterpret_cast<float4*>(a.sums + 2 * static_cast<int64_t>(u) * p.d);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int i = tid + j * G;
          if (i < nv) {
            sums[i] = A[j];
            sums[nv + i] = B[j];
          }
        }
      }
    }
    finish();
    return;
  }
  rows(static_cast<int64_t>(blockIdx.x) * kGroups + grp, p.rows, static_cast<int64_t>(gridDim.x) * kGroups);
  finish();
  if (!PARAMS) return;
  // the groups' sums, in their order
  __shared__ float4 joined[kGroups > 1 ? 2 : 1][kGroups > 1 ? NV * G : 1];
  if constexpr (kGroups > 1) {
    for (int k = 0; k < kGroups; ++k) {
      if (grp == k) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int i = tid + j * G;
          if (k > 0) {
            const float4 x = joined[0][i], y = joined[1][i];
            A[j] = make_float4(A[j].x + x.x, A[j].y + x.y, A[j].z + x.z, A[j].w + x.w);
            B[j] = make_float4(B[j].x + y.x, B[j].y + y.y, B[j].z + y.z, B[j].w + y.w);
          }
          joined[0][i] = A[j];
          joined[1][i] = B[j];
        }
      }
      __syncthreads();
    }
  }
  if (kGroups > 1 && grp != kGroups - 1) return;
  float4* sums = reinterpret_cast<float4*>(a.sums + 2 * static_cast<int64_t>(blockIdx.x) * p.d);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = tid + j * G;
    if (i < nv) {
      sums[i] = A[j];
      sums[nv + i] = B[j];
    }
  }
}

// The units' sums added up: CTA (columns, sample) for dshift and dscale, CTA (columns, the last one) for dg and db.
__global__ void __launch_bounds__(256) norm_grad_sums_kernel(const Args a) {
  __shared__ float4 red[2][kShares][kColsPerCta / 4];
  pdl_wait_and_trigger();
  const NormGradParams& p = a.p;
  const int lane = threadIdx.x & 3, share = threadIdx.x >> 2;
  const int i = blockIdx.x * (kColsPerCta / 4) + lane, nv = p.d >> 2;
  const bool modulated = p.scale != nullptr;
  const int samples = modulated && (p.dshift || p.dscale) ? a.q.samples : 0;
  for (int job = blockIdx.y; job < samples + 1; job += gridDim.y) {
    const bool all = job == samples;
    if (all && !p.dg && !p.db) continue;
    const int from = all ? 0 : job * a.q.parts, to = all ? a.q.units : from + a.q.parts;
    float4 A = make_float4(0.f, 0.f, 0.f, 0.f), B = A;
    if (i < nv) {
#pragma unroll 8
      for (int u = from + share; u < to; u += kShares) {
        const float4* at = reinterpret_cast<const float4*>(a.sums + 2 * static_cast<int64_t>(u) * p.d);
        float4 x = at[i], y = at[nv + i];
        if (all && modulated) {
          const float* s = p.scale + static_cast<int64_t>(u / a.q.parts) * p.ld_mod + 4 * i;
          const float4 f = make_float4(1.f + s[0], 1.f + s[1], 1.f + s[2], 1.f + s[3]);
          x = make_float4(x.x * f.x, x.y * f.y, x.z * f.z, x.w * f.w);
          y = make_float4(y.x * f.x, y.y * f.y, y.z * f.z, y.w * f.w);
        }
        A = make_float4(A.x + x.x, A.y + x.y, A.z + x.z, A.w + x.w);
        B = make_float4(B.x + y.x, B.y + y.y, B.z + y.z, B.w + y.w);
      }
    }
    red[0][share][lane] = A;
    red[1][share][lane] = B;
    __syncthreads();
    if (share < 8) {
      for (int k = share + 8; k < kShares; k += 8) {
        const float4 x = red[0][k][lane], y = red[1][k][lane];
        A = make_float4(A.x + x.x, A.y + x.y, A.z + x.z, A.w + x.w);
        B = make_float4(B.x + y.x, B.y + y.y, B.z + y.z, B.w + y.w);
      }
      __syncwarp();
      red[0][share][lane] = A;
      red[1][share][lane] = B;
      __syncwarp();
    }
    if (share == 0 && i < nv) {
      for (int k = 1; k < 8; ++k) {
        const float4 x = red[0][k][lane], y = red[1][k][lane];
        A = make_float4(A.x + x.x, A.y + x.y, A.z + x.z, A.w + x.w);
        B = make_float4(B.x + y.x, B.y + y.y, B.z + y.z, B.w + y.w);
      }
      const float va[4] = {A.x, A.y, A.z, A.w}, vb[4] = {B.x, B.y, B.z, B.w};
      if (all) {
        if (p.db) reinterpret_cast<float4*>(p.db)[i] = A;
        if (p.dg) reinterpret_cast<float4*>(p.dg)[i] = B;
      } else {
        const int64_t at = static_cast<int64_t>(job) * p.ld_dmod + 4 * i;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float gain = p.g ? __bfloat162float(p.g[4 * i + j]) : 1.f, shift = p.b ? __bfloat162float(p.b[4 * i + j]) : 0.f;
          if (p.dshift) p.dshift[at + j] = va[j];
          if (p.dscale) p.dscale[at + j] = fmaf(gain, vb[j], shift * va[j]);
        }
      }
    }
    __syncthreads();
  }
}

template <typename T, int G, bool WIDE, bool MOD, bool PARAMS>
cudaError_t launch_rows(const Args& a, cudaStream_t s) {
  constexpr int kSmem = smem_of(WIDE, sizeof(T));
  // once per kernel and device
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (kSmem > 40 * 1024 && (dev > 63 || !(ready.load() >> dev & 1))) {
    e = cudaFuncSetAttribute(norm_grad_kernel<T, G, WIDE, MOD, PARAMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    if (dev <= 63) ready.fetch_or(1ull << dev);
  }
  norm_grad_kernel<T, G, WIDE, MOD, PARAMS><<<a.q.ctas, kThreads, kSmem, s>>>(a);
  return cudaGetLastError();
}
template <typename T, int G, bool WIDE>
cudaError_t rows_of(const Args& a, bool params, cudaStream_t s) {
  if (a.p.scale) return params ? launch_rows<T, G, WIDE, true, true>(a, s) : launch_rows<T, G, WIDE, true, false>(a, s);
  return params ? launch_rows<T, G, WIDE, false, true>(a, s) : launch_rows<T, G, WIDE, false, false>(a, s);
}
template <typename T>
cudaError_t rows_of_type(const Args& a, bool params, cudaStream_t s) {
  if (a.q.wide) return rows_of<T, 256, true>(a, params, s);
  if (a.q.group == 32) return rows_of<T, 32, false>(a, params, s);
  if (a.q.group == 64) return rows_of<T, 64, false>(a, params, s);
  if (a.q.group == 128) return rows_of<T, 128, false>(a, params, s);
  return rows_of<T, 256, false>(a, params, s);
}

}  // namespace

int64_t norm_grad_bytes(int rows, int d, int rows_per_batch) {
  return rows < 1 ? 0 : 8ll * make_plan(rows, d, rows_per_batch).units * d;
}

cudaError_t norm_grad_launch(const NormGradParams& p, cudaStream_t s) {
  const bool params = p.dg || p.db || p.dshift || p.dscale;
  const Args a{p, make_plan(p.rows, p.d, p.scale ? p.rows_per_batch : 0), static_cast<float*>(p.workspace)};
  const cudaError_t e = p.dtype == SGD_F16 ? rows_of_type<f16>(a, params, s)
                        : p.dtype == SGD_BF16 ? rows_of_type<bf16>(a, params, s) : rows_of_type<float>(a, params, s);
  if (e != cudaSuccess || !params) return e;
  const int jobs = 1 + (p.scale && (p.dshift || p.dscale) ? a.q.samples : 0);
  const dim3 grid((p.d + kColsPerCta - 1) / kColsPerCta, jobs < 1024 ? jobs : 1024);
  return launch_behind(norm_grad_sums_kernel, grid, dim3(256), 0, s, a);
}

}  // namespace sgd
