// Filtered draws of f16 logits (sample.cu).
#include "sample_kernel.cuh"

namespace sgd {
namespace rows {
template cudaError_t sample_rows<f16, true>(const SampleArgs&, cudaStream_t);
}  // namespace rows
}  // namespace sgd
