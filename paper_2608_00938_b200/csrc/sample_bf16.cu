// The kernels of grace_sample for bf16 logits.
#include "sample.cuh"

namespace grace {
grace_status_t run_sample_bf16(const SampleParams& p, cudaStream_t s) { return run_sample<true>(p, s); }
}  // namespace grace
