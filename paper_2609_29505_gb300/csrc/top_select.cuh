// The k likeliest elements of (a slice of) a row of logits, by a team of threads.
//
// Elements are ordered by (value descending, index ascending).  A threshold that at least k elements
// reach, and not many more, is found first; what reaches it is collected and ranked by counting.
#pragma once

#include "vocab_rows.cuh"

namespace sgd {
namespace rows {

constexpr int kCap = 256;  // candidates that are ranked

// value of a candidate above, (reversed) index below: larger is likelier, ties to the lower index
__device__ __forceinline__ uint64_t candidate(uint32_t key, int index) {
  return static_cast<uint64_t>(key) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(index));
}
__device__ __forceinline__ int candidate_index(uint64_t c) {
  return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(c));
}

struct TopShared {
  uint64_t list[kCap];
  int n;
  int count[3];
  uint32_t warp_lo[8], warp_hi[8];
  int warp_count[8];
};

// Appends the elements of vector `v` (its first element: e) with a key of at least `from` to the list, as
// many as it holds, and adds their number to sh->n.  (Not inlined: it is rare, and the loops around it
// should stay in the instruction cache.)
template <typename T>
__device__ __noinline__ void append(uint4 v, int e, int vocab, uint32_t from, TopShared* sh) {
  float f[Elem<T>::kPer];
  unpack(v, f, static_cast<const T*>(nullptr));
#pragma unroll
  for (int j = 0; j < Elem<T>::kPer; ++j) {
    const uint32_t key = order_key(f[j]);
    if (key >= from && e + j >= 0 && e + j < vocab) {
      const int at = atomicAdd(&sh->n, 1);
      if (at < kCap) sh->list[at] = candidate(key, e + j);
    }
  }
}

// All elements of the slice; fetch(i) gives its vector i.
template <typename T, typename Tm, typename F>
__device__ __forceinline__ void collect(const Tm& team, const Slice<T>& sl, const F& fetch, uint32_t from, TopShared& sh) {
  const float bar = key_value(from);
  for (int i = team.tid; i < sl.nv; i += Tm::kSize) {
    const uint4 v = fetch(i);
    if (from > kKeyNegInf && !(vec_max<1>(&v, static_cast<const T*>(nullptr)) >= bar)) continue;
    append<T>(v, sl.first_element(i), sl.vocab, from, &sh);
  }
  team.sync();
}

// Elements of the slice with a key of at least `bar` (every thread gets the count).  `turn`: 0, 1, 2,
// 0, ... over the calls, each of which clears the next one's counter.
template <typename T, typename Tm, typename F>
__device__ int count_from(const Tm& team, const Slice<T>& sl, const F& fetch, uint32_t bar, TopShared& sh, int turn) {
  int n = 0;
  for (int i = team.tid; i < sl.nv; i += Tm::kSize) {
    float f[Elem<T>::kPer];
    unpack(fetch(i), f, static_cast<const T*>(nullptr));
    const int e = sl.first_element(i);
#pragma unroll
    for (int j = 0; j < Elem<T>::kPer; ++j) n += order_key(f[j]) >= bar && e + j >= 0 && e + j < sl.vocab;
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if ((team.tid & 31) == 0 && n) atomicAdd(&sh.count[turn], n);
  if (team.tid == 0) sh.count[(turn + 1) % 3] = 0;
  team.sync();
  return sh.count[turn];
}

// The first `need` elements of key `key`, in the order of the index, behind the list.
template <typename T, typename Tm, typename F>
__device__ void collect_ties(const Tm& team, const Slice<T>& sl, const F& fetch, uint32_t key, int need, TopShared& sh) {
  const int warp = team.tid >> 5, lane = team.tid & 31;
  int have = 0;
  const int base = sh.n;
  team.sync();
  for (int i0 = 0; i0 < sl.nv && have < need; i0 += Tm::kSize) {
    const int i = i0 + team.tid, e = sl.first_element(i);
    uint32_t hit = 0;
    if (i < sl.nv) {
      float f[Elem<T>::kPer];
      unpack(fetch(i), f, static_cast<const T*>(nullptr));
#pragma unroll
      for (int j = 0; j < Elem<T>::kPer; ++j)
        hit |= (order_key(f[j]) == key && e + j >= 0 && e + j < sl.vocab ? 1u : 0u) << j;
    }
    int before = __popc(hit);
    const int mine = before;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += up;
    }
    if (lane == 31) sh.warp_count[warp] = before;
    before -= mine;
    team.sync();
    int all = 0;
    for (int w = 0; w < Tm::kWarps; ++w) {
      if (w < warp) before += sh.warp_count[w];
      all += sh.warp_count[w];
    }
    before += have;
    for (; hit && before < need; hit &= hit - 1, ++before)
      sh.list[base + before] = candidate(key, e + __ffs(hit) - 1);
    have += all;
    team.sync();
  }
  if (team.tid == 0) sh.n = base + min(have, need);
  team.sync();
}

// A threshold on the maxima: count(maxima >= lo) >= k, and near k unless many are equal to lo (`tied`); then
// fewer than k are above it.  `top`: a key above all.
struct Threshold {
  uint32_t lo, top;
  bool tied;
  // what is looked for among all elements: those above lo alone where it is tied, as the equal ones are many
  __device__ uint32_t from() const { return tied ? lo + 1 : lo; }
};

// By bisection over the keys, counting over the team.  N keys per thread, at least k in all.
template <int N, typename Tm>
__device__ Threshold threshold(const Tm& team, const uint32_t (&key)[N], int k, TopShared& sh) {
  const int warp = team.tid >> 5, lane = team.tid & 31;
  uint32_t lo = key[0], hi = key[0];
#pragma unroll
  for (int i = 1; i < N; ++i) {
    lo = min(lo, key[i]);
    hi = max(hi, key[i]);
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) {
    sh.warp_lo[warp] = lo;
    sh.warp_hi[warp] = hi;
  }
  if (team.tid == 0) sh.n = sh.count[0] = sh.count[1] = 0;
  team.sync();
#pragma unroll
  for (int w = 0; w < Tm::kWarps; ++w) {
    lo = min(lo, sh.warp_lo[w]);
    hi = max(hi, sh.warp_hi[w]);
  }
  const uint32_t top = hi = hi + 1;  // the largest key is that of +inf
  bool tied = true;
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    int n = 0;
    if constexpr (Tm::kWarps == 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) n += key[i] >= mid;
      n = __reduce_add_sync(0xffffffffu, n);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) n += team.count(key[i] >= mid);
    }
    if (n >= k) lo = mid; else hi = mid;
    if (n >= k && n <= k + k / 4) {
      tied = false;
      break;
    }
  }
  return Threshold{lo, top, tied};
}

// Where the elements that were looked for do not fit into the list (rows sorted so that few threads hold the
// largest values, say): the threshold is bisected over all elements until few reach it, or it is the
// k-th largest value itself; then what is above it is taken, and the first of those equal to it.
// Up to 32 counts.
template <typename T, typename Tm, typename F>
__device__ __noinline__ void candidates_of_many(const Tm team, const Slice<T> sl, const F fetch, uint32_t lo, uint32_t top, int k,
                                                TopShared& sh) {
  team.sync();
  uint32_t hi = top, mid = lo + 1;
  int turn = 0, n = 0;
  while (hi - lo > 1) {
    n = count_from(team, sl, fetch, mid, sh, turn);
    turn = (turn + 1) % 3;
    if (n >= k) lo = mid; else hi = mid;
    if (n >= k && n <= kCap) break;
    mid = lo + (hi - lo) / 2;
  }
  if (team.tid == 0) sh.n = 0;
  team.sync();
  if (n >= k && n <= kCap) {
    collect(team, sl, fetch, lo, sh);
    return;
  }
  collect(team, sl, fetch, lo + 1, sh);  // fewer than k
  collect_ties(team, sl, fetch, lo, k - sh.n, sh);
}

// The k largest of the sh.n candidates in order at put(place, candidate); places without one get 0.
template <typename Tm, typename P>
__device__ __forceinline__ void rank_candidates(const Tm& team, const TopShared& sh, int k, const P& put) {
  const int n = sh.n;
  for (int i = team.tid; i < n; i += Tm::kSize) {
    const uint64_t x = sh.list[i];
    int place = 0;
    for (int j = 0; j < n; ++j) place += sh.list[j] > x;
    if (place < k) put(place, x);
  }
  for (int i = n + team.tid; i < k; i += Tm::kSize) put(i, static_cast<uint64_t>(0));
}

// The k largest of n_lists sorted lists of k (0: no entry).
template <typename Tm, typename P>
__device__ __forceinline__ void merge_lists(const Tm& team, const uint64_t* lists, int n_lists, int k, const P& put) {
  const int all = n_lists * k;
  if (all <= 256) {  // counted: loads that do not wait for one another
    for (int i = team.tid; i < all; i += Tm::kSize) {
      const uint64_t x = lists[i];
      int place = 0;
#pragma unroll 8
      for (int j = 0; j < all; ++j) place += lists[j] > x;
      if (x != 0 && place < k) put(place, x);
    }
    return;
  }
  for (int i = team.tid; i < n_lists * k; i += Tm::kSize) {
    const uint64_t x = lists[i];
    if (x == 0) continue;
    const int own = i / k;
    int place = i - own * k;
    for (int l = 0; l < n_lists && place < k; ++l) {
      if (l == own) continue;
      int a = 0, b = k;  // first entry of list l that is smaller
      while (a < b) {
        const int mid = (a + b) >> 1;
        if (lists[l * k + mid] > x) a = mid + 1; else b = mid;
      }
      place += a;
    }
    if (place < k) put(place, x);
  }
}

}  // namespace rows
}  // namespace sgd
