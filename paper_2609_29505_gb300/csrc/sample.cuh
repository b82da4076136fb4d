// Draws of tokens: what the host hands to the kernels.
#pragma once

#include "vocab_rows.cuh"

namespace sgd {
namespace rows {

struct SampleArgs {
  SampleParams p;
  // Exponents are (z - m) f c in base 2.  f is 1, or 2^-64 for scales below: there logits may lie as far apart as their type has them, farther
  // than an fp32 difference holds, and still both have a share; and the product scale log2(e) may have few bits.
  float f;
  float c, c_lo;    // scale log2(e) / f, as the sum of two floats
  float scale;      // scale / f
  double drop;      // ln(min_p) / scale: a token at or above max + drop passes (-inf: every token)
  int n_blocks;
  int* status;
};

// FILTER: top-k, min-p or top-p.
template <typename T, bool FILTER>
cudaError_t sample_rows(const SampleArgs& a, cudaStream_t s);

}  // namespace rows
}  // namespace sgd
