// Draws of tokens: what the host hands to the kernels.
#pragma once

#include "vocab_rows.cuh"

namespace sgd {
namespace rows {

struct SampleArgs {
  SampleParams p;
  float c, c_lo;    // scale log2(e), as the sum of two floats
  double drop;      // ln(min_p) / scale: a token at or above max + drop passes (-inf: every token)
  int n_blocks;
  int* status;
};

// FILTER: top-k, min-p or top-p.
template <typename T, bool FILTER>
cudaError_t sample_rows(const SampleArgs& a, cudaStream_t s);

}  // namespace rows
}  // namespace sgd
