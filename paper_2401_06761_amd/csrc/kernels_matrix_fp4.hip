// Prefill attention over 4-bit pools on the 32x32 matrix instructions: the walk of matrix_walk.hpp over tiles of 2176 bytes, widened to bf16
// when they are staged.  A tile is widened once per workgroup of 128 query rows, some fifty vector instructions of one of its wavefronts; the
// row-tile kernel (kernels_attn_fp4.hip) leaves K as it is, but widens V for every 16 or 32 rows.  What bounds it: the matrix pipe and the walk's
// barriers, as on bf16 pools (five prompts of 1 k to 4.5 k tokens, 32/8 heads, 0.565 TFLOP in 570 us, 0.99 PFLOP/s; on row tiles 903).
#include <hip/hip_runtime.h>

#include "matrix_walk.hpp"

namespace apar {

namespace {

__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prefill_fp4(
    const char* __restrict__ pool, const uint16_t* __restrict__ q, const PrefillWg* __restrict__ wgs,
    const int32_t* __restrict__ tables, int n_q, int n_kv, int group, float scale_log2e, uint16_t* __restrict__ out) {
    __shared__ __attribute__((aligned(16))) char lds[2 * kBufBytes];
    prefill_rows<kTilesFp4>(lds, pool, q, wgs, tables, n_q, n_kv, group, scale_log2e, out);
}

}  // namespace

hipError_t launch_prefill_fp4(const Shape& s, const void* pool, const void* q, const PrefillWg* wgs, const int32_t* tables, int n_wg,
                              void* out, hipStream_t st) {
    if (n_wg <= 0) return hipSuccess;
    const int64_t grid = (int64_t)n_wg * s.n_kv;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL(prefill_fp4, dim3((unsigned)grid), dim3(256), 0, st, (const char*)pool, (const uint16_t*)q, wgs, tables, s.n_q, s.n_kv,
                       s.group, s.scale_log2e, (uint16_t*)out);
    return hipGetLastError();
}

}  // namespace apar
