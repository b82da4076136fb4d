// Filtered draws of f32 logits (sample.cu).
#include "sample_kernel.cuh"

namespace sgd {
namespace rows {
template cudaError_t sample_rows<float, true>(const SampleArgs&, cudaStream_t);
}  // namespace rows
}  // namespace sgd
