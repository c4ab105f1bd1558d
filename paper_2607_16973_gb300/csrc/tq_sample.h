// Internal declarations of sampling (tq_sample in tq.h).
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace tq {

size_t sample_workspace(int64_t n, int64_t vocab);
cudaError_t launch_sample(const void* logits, int type, int64_t logits_stride, const float* noise, int64_t noise_stride,
                          int64_t n, int vocab, const float* temperature, const int32_t* top_k, const float* top_p,
                          const float* min_p, int32_t* tokens, float* logprobs, void* workspace, cudaStream_t s);

}  // namespace tq
