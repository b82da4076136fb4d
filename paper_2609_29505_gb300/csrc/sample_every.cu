// Draws of every token, of all types of logits (sample.cu).
#include "sample_kernel.cuh"

namespace sgd {
namespace rows {
template cudaError_t sample_rows<f16, false>(const SampleArgs&, cudaStream_t);
template cudaError_t sample_rows<bf16, false>(const SampleArgs&, cudaStream_t);
template cudaError_t sample_rows<float, false>(const SampleArgs&, cudaStream_t);
}  // namespace rows
}  // namespace sgd
