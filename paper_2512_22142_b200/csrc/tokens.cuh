// The operators at the two ends of a step on tokens, and layer norm: launchers and shared pieces (internal).
#pragma once

#include "ops.cuh"

namespace cleave {

inline uint32_t id_bytes(uint32_t t) { return t == CLEAVE_T_I64 ? 8u : (t == CLEAVE_T_I32 ? 4u : 0u); }

// token `i`, or -1 for padding
__device__ __forceinline__ int32_t load_token(const void* ids, uint32_t type, uint64_t i, uint32_t vocab) {
    const int64_t t = type == CLEAVE_T_I64 ? static_cast<const int64_t*>(ids)[i] : (int64_t) static_cast<const int32_t*>(ids)[i];
    return (uint64_t)t < vocab ? (int32_t)t : -1;
}

cudaError_t launch_embedding(const cleave_embedding_t& d, cudaStream_t st);
uint64_t embedding_backward_workspace(uint64_t n, uint32_t vocab, uint32_t cols);
cudaError_t launch_embedding_backward(const cleave_embedding_backward_t& d, void* ws, cudaStream_t st);

cudaError_t launch_layernorm(const cleave_layernorm_t& d, int sms, cudaStream_t st);
uint32_t layernorm_backward_parts(uint64_t rows, uint32_t cols);
cudaError_t launch_layernorm_backward(const cleave_layernorm_backward_t& d, float* ws, cudaStream_t st);

cudaError_t launch_logprobs(const cleave_logprobs_t& d, int sms, cudaStream_t st);
cudaError_t launch_logprobs_backward(const cleave_logprobs_backward_t& d, int sms, cudaStream_t st);
cudaError_t launch_distill(const cleave_distill_t& d, int sms, cudaStream_t st);
cudaError_t launch_distill_backward(const cleave_distill_backward_t& d, int sms, cudaStream_t st);

}  // namespace cleave
