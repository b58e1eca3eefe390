// grace_sample: arguments, and the kernels for fp32 logits (those for bf16 ones: sample_bf16.cu, a file of their own because
// the compiler takes a minute for each).
#include "sample.cuh"

namespace grace {
grace_status_t run_sample_bf16(const SampleParams& p, cudaStream_t s);
}  // namespace grace

extern "C" grace_status_t grace_sample(const float* logits_f32, const uint16_t* logits_bf16, int64_t ld, const uint64_t* allow_bits,
                                       const float* row_score, const float* row_lse, const float* temperature,
                                       const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                                       int B, int M, int V, int draws, float* out_score, float* out_logq,
                                       int32_t* out_parent, int32_t* out_token, int32_t* d_status, void* stream) {
  using namespace grace;
  if ((logits_f32 == nullptr) == (logits_bf16 == nullptr) || !u || !out_score || !out_token) return GRACE_INVALID_ARG;
  if (B <= 0 || M <= 0 || V <= 0 || draws <= 0 || ld < V) return GRACE_INVALID_ARG;
  const uintptr_t words = reinterpret_cast<uintptr_t>(logits_f32) | reinterpret_cast<uintptr_t>(row_score) | reinterpret_cast<uintptr_t>(row_lse) |
                          reinterpret_cast<uintptr_t>(temperature) | reinterpret_cast<uintptr_t>(top_k) | reinterpret_cast<uintptr_t>(top_p) |
                          reinterpret_cast<uintptr_t>(min_p) | reinterpret_cast<uintptr_t>(u) | reinterpret_cast<uintptr_t>(out_score) |
                          reinterpret_cast<uintptr_t>(out_logq) | reinterpret_cast<uintptr_t>(out_parent) | reinterpret_cast<uintptr_t>(out_token) |
                          reinterpret_cast<uintptr_t>(d_status);
  if ((words & 3) || (reinterpret_cast<uintptr_t>(logits_bf16) & 1) || (reinterpret_cast<uintptr_t>(allow_bits) & 7)) return GRACE_INVALID_ARG;
  if (V > kSampleMostV || draws > kSampleMostDraws || (int64_t)B * M > 0x7fffffffll) return GRACE_UNSUPPORTED_SHAPE;
  SampleParams p = {};
  const bool bf16 = logits_bf16 != nullptr;
  p.logits = bf16 ? (const void*)logits_bf16 : (const void*)logits_f32;
  p.allow = allow_bits; p.row_score = row_score; p.row_lse = row_lse; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
  p.u = u; p.out_score = out_score; p.out_logq = out_logq; p.out_parent = out_parent; p.out_token = out_token; p.d_status = d_status;
  p.ld = ld; p.R = (int64_t)B * M; p.M = M; p.V = V; p.draws = draws;
  p.vec = ((reinterpret_cast<uintptr_t>(p.logits) | (uintptr_t)(ld * (bf16 ? 2 : 4))) & (bf16 ? 7 : 15)) == 0;
  cudaStream_t s = (cudaStream_t)stream;
  return bf16 ? run_sample_bf16(p, s) : run_sample<false>(p, s);
}
