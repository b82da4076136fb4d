// What the two scoring kernels share: parameters, and the last step of a row.
#pragma once

#include "top_select.cuh"

namespace sgd {
namespace rows {

struct ScoreArgs {
  const void* logits;
  int64_t ld;
  int rows, vocab;
  float scale;
  const int32_t* row_ids;
  int row_id;
  const int32_t* tokens;
  int n_tokens;
  float* token_logprobs;
  float* entropy;
  int top_k;
  int32_t* top_ids;
  float* top_logprobs;
  int* status;
};

enum { kTopNone = 0, kTopOne = 1, kTopMany = 2 };

// A row's given tokens, one per thread of the team (more in finish()): the token is fetched ahead of the row, its
// logit while the row's statistics are reduced (a thread waits at the first use of what it loads).
template <typename T>
struct Given {
  int token = -1;
  float z = 0.f;
  __device__ __forceinline__ void fetch_token(const ScoreArgs& p, int64_t r, int tid) {
    if (tid < p.n_tokens) token = p.tokens[r * p.n_tokens + tid];
  }
  __device__ __forceinline__ void fetch_logit(const ScoreArgs& p, const T* row) {
    if (token >= 0) z = token < p.vocab ? to_f(row[token]) : kNan;
  }
};

// The row's outputs from its parts: slot[i] = {maximum, s, t, index of the first maximum} of CTA i, and
// their sorted lists of the likeliest elements.  `result`: two floats shared by the team.
template <typename T, int TOP, bool ENT, typename Tm>
__device__ __forceinline__ void finish(const Tm& team, const ScoreArgs& p, int64_t r, const T* row, Given<T> given,
                                       const float4* slot, const uint64_t* lists, int n_ctas, float* result) {
  const float c = p.scale * kLog2e;
  if (team.tid < 32) {
    float4 v = make_float4(-kInf, 0.f, 0.f, 0.f);
    if (team.tid < n_ctas) v = slot[team.tid];
    const float all = key_value(__reduce_max_sync(0xffffffffu, order_key(v.x)));
    const float R = reference(all, c);
    float s = v.y, t = v.z;
    rebase(v.x, c, all, R, s, t);
    s = warp_sum(s);
    if (ENT) t = warp_sum(t);
    // of the CTAs that have the maximum the first has it at the lowest index
    const int index = __reduce_min_sync(0xffffffffu, team.tid < n_ctas && v.x == all ? __float_as_int(v.w) : 0x7FFFFFFF);
    if (team.tid == 0) {
      const bool empty = all == -kInf && s == 0.f;  // (NaN: s is NaN)
      const float delta = delta_of(all, c, R);
      const float ln_s = empty ? 0.f : logf(s) - delta * kLn2;
      result[0] = empty ? kInf : all;  // an empty row: every difference to it is -inf
      result[1] = ln_s;
      // H / ln 2 = log2 s - t / s; the reference's rounding cancels in the difference
      if (ENT) p.entropy[r] = empty ? 0.f : logf(s) - kLn2 * (t / s);
      if (TOP == kTopOne) {
        if (p.top_ids) p.top_ids[r] = index;
        if (p.top_logprobs) p.top_logprobs[r] = empty ? -kInf : -ln_s;
      }
    }
  }
  if (TOP != kTopMany && p.n_tokens == 0) return;
  team.sync();
  const float all = result[0], ln_s = result[1];
  auto logprob = [&](float z) {
    const float d = z - all;  // (where it is out of range it may not be so scaled)
    return (d == -kInf && z > -kInf ? z * p.scale - all * p.scale : d * p.scale) - ln_s;
  };
  if (team.tid < p.n_tokens)
    p.token_logprobs[r * p.n_tokens + team.tid] = given.token < 0 ? 0.f : logprob(given.z);
  for (int i = team.tid + Tm::kSize; i < p.n_tokens; i += Tm::kSize) {
    const int t = p.tokens[r * p.n_tokens + i];
    p.token_logprobs[r * p.n_tokens + i] = t < 0 ? 0.f : (t < p.vocab ? logprob(to_f(row[t])) : kNan);
  }
  if (TOP == kTopMany)
    merge_lists(team, lists, n_ctas, p.top_k, [&](int place, uint64_t x) {
      const int64_t at = r * p.top_k + place;
      if (p.top_ids) p.top_ids[at] = candidate_index(x);
      if (p.top_logprobs) p.top_logprobs[at] = logprob(key_value(static_cast<uint32_t>(x >> 32)));
    });
}

template <typename T>
cudaError_t score_stream(const ScoreArgs& p, cudaStream_t s);  // logprobs_stream.cu
bool stream_pays(int rows, int64_t row_bytes);

}  // namespace rows
}  // namespace sgd
