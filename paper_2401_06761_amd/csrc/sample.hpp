// Sampling: what the host hands to the kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apar.h"

namespace apar {

constexpr int kSampleMaxVocab = 1 << 20;
constexpr int kSampleMaxRows = (1 << 22) - 1;  // (a workgroup of 1024 threads each, and a launch has fewer than 2^32)

struct SampleCall {
    const void* logits;
    int64_t row_stride;               // elements
    const apar_sample_row* rows;      // null: temperature 1, nothing cut
    const float* uniforms;
    int32_t* tokens;
    float* logprobs;                  // may be null
    int32_t n, vocab;
    apar_token_ids ids;
    int32_t weight_bits;              // at most 51: a weight of 1 is 2^weight_bits, and the weights of a row add up to less than 2^63
};

hipError_t launch_sample_tokens(const SampleCall& call, bool f32, hipStream_t st);

}  // namespace apar
