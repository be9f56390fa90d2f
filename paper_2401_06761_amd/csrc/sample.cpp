// Sampling: the entry point's checks.
#include "sample.hpp"

#include "hip_status.hpp"

using namespace apar;

extern "C" {

int apar_sample_workspace_bytes(int n, int vocab, size_t* bytes_out) {
    if (!bytes_out || n < 0 || vocab < 1) return APAR_ERR_INVALID_ARG;
    if (vocab > kSampleMaxVocab || n > kSampleMaxRows) return APAR_ERR_UNSUPPORTED;
    *bytes_out = 0;
    return APAR_OK;
}

int apar_sample_tokens(const void* logits_dev, int dtype, int n, int vocab, int64_t row_stride, const apar_sample_row* rows_dev,
                       const float* uniforms_dev, const apar_token_ids* ids, int32_t* tokens_dev, float* logprobs_dev,
                       void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (n < 0 || vocab < 1 || (dtype != APAR_F32 && dtype != APAR_BF16)) return APAR_ERR_INVALID_ARG;
    if (vocab > kSampleMaxVocab || n > kSampleMaxRows) return APAR_ERR_UNSUPPORTED;
    if (n == 0) return APAR_OK;
    if (!logits_dev || !uniforms_dev || !tokens_dev || row_stride < vocab) return APAR_ERR_INVALID_ARG;
    size_t need = 0;
    const int rc = apar_sample_workspace_bytes(n, vocab, &need);
    if (rc != APAR_OK) return rc;
    if (workspace_bytes < need || (need > 0 && !workspace_dev)) return APAR_ERR_WORKSPACE_LIMIT;
    if (((uintptr_t)logits_dev & (dtype == APAR_F32 ? 3 : 1)) || ((uintptr_t)rows_dev & 3) || ((uintptr_t)uniforms_dev & 3) ||
        ((uintptr_t)tokens_dev & 3) || ((uintptr_t)logprobs_dev & 3) || ((uintptr_t)workspace_dev & 15))
        return APAR_ERR_INVALID_ARG;
    SampleCall call{};
    call.logits = logits_dev;
    call.row_stride = row_stride;
    call.rows = rows_dev;
    call.uniforms = uniforms_dev;
    call.tokens = tokens_dev;
    call.logprobs = logprobs_dev;
    call.n = n;
    call.vocab = vocab;
    call.ids = ids ? *ids : apar_token_ids{-1, -1, -1};
    call.weight_bits = 62;
    while (((int64_t)1 << (62 - call.weight_bits)) < vocab) call.weight_bits -= 1;
    if (call.weight_bits > 51) call.weight_bits = 51;  // (whole_units)
    DeviceOf guard(logits_dev);
    HIP_TRY(launch_sample_tokens(call, dtype == APAR_F32, (hipStream_t)hip_stream));
    return APAR_OK;
}

}  // extern "C"
