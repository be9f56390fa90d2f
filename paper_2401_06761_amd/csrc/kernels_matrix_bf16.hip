// Attention shaped for the matrix cores (16-bit pools): 32x32 products, 128 query rows per workgroup.
//
// Two kernels share one walk:
//   * prefill_bf16: a workgroup takes up to 128 query rows of ONE thread - consecutive query tokens x the
//     q heads of one kv group - and walks that thread's root path under the causal paragraph-tree mask;
//   * attention_units_bf16: a workgroup takes up to 128 query rows of threads that all hold one shared
//     segment (a decode step's stand-alone unit with many rows) and walks a chunk of that segment's
//     blocks; every row sees every filled slot, and the rows' softmax states go out as partial results.
//
// The walk goes in super-blocks of 32 token slots (two KV blocks).  Every wavefront owns 32 rows as the
// N side of 32x32 products:
//
//   S^T[token][row] = K[token][:] . Q[row][:]            8 x mfma_f32_32x32x16_bf16 per super-block
//   O^T[dim][row]  += V^T[dim][token] . P^T[token][row]   8 x mfma_f32_32x32x16_bf16 per super-block
//
// so a lane holds 16 logits per super-block and the per-tile bookkeeping of the online softmax (row
// maximum, the branch that moves the reference, sums) is spread over four times as many elements as in
// the row-tile kernel, and both products run at the full matrix rate.  The accumulator layout of S^T
// (lane = 32 h + n holds tokens 8 j + 4 h + i of row n) is the B-operand layout of P^T once the token
// index of the second product is permuted the same way, so probabilities never move between lanes.
//
// The four wavefronts share the path through LDS in groups of two super-blocks (four KV blocks, double
// buffered, one barrier per group): each wavefront has one block of the next group on its way to LDS, without
// registers in between, while a group is consumed.  Blocks lie in LDS in operand order, as sealed blocks do in
// HBM; a still open one (only the last block of a walk can be) is put into that order once it has landed, and the
// codes of a full fp8 block are widened on their way.
//
// What bounds it: a super-block is 512 cycles of products and some 450 of vector instructions (16 exp2 are 256 of
// them) on the same SIMD, and with one phase after the other a wavefront pair needs 1250 cycles per super-block.  So a
// wavefront's own vector work is issued between its products: the probabilities of one super-block between the K.Q^T
// products of the next one, the maximum over those between the V^T.P^T products, and LDS operands are read beside
// either, into registers that have just become free (218 registers, two wavefronts per SIMD).  Six prompts of 1 k to 8 k
// tokens, 8 kv heads of 4 (1.75 TFLOP): 1.90 -> 1.64 ms, matrix pipe busy 57 % of the time instead of 41 % at a clock that
// falls from 1.94 to 1.79 GHz; own segments of 982 threads, 32 heads, walks of 529: 1.80 -> 1.65 ms.  The direct loads alone,
// phases one after the other as before, take half of that.
// Masks only matter at the end of a row's range: a super-block wholly below a wavefront's first limit is applied
// without masks, one wholly above its last limit is skipped.
#include <hip/hip_runtime.h>

#include "matrix_walk.hpp"

namespace apar {

namespace {

template <bool F8>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prefill_bf16(
    const char* __restrict__ pool, const uint16_t* __restrict__ q, const PrefillWg* __restrict__ wgs,
    const int32_t* __restrict__ tables, int n_q, int n_kv, int group, float scale_log2e, uint16_t* __restrict__ out) {
    __shared__ __attribute__((aligned(16))) char lds[2 * kBufBytes];
    prefill_rows<F8 ? kTilesFp8 : kTilesBf16>(lds, pool, q, wgs, tables, n_q, n_kv, group, scale_log2e, out);
}

// Stand-alone units of a decode plan with many rows.  The workgroup descriptor's shared tile list is the
// chunk of the segment (full blocks first, the open one last); its first wavefront entry names the
// threads: depth-first ranks grp_lo / n_slices .. + n_grp / n_slices, rows_per_thread rows each, laid
// flat over the 128 rows; part_base is the first thread's partial-result row for this chunk.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void attention_units_bf16(
    const char* __restrict__ pool, const uint16_t* __restrict__ q, PlanDev plan, int wg_first, int n_cand, int n_q,
    int n_kv, int group, float scale_log2e, PartialBuf part) {
    __shared__ __attribute__((aligned(16))) char lds[2 * kBufBytes];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n = lane & 31, h = lane >> 5;
    const int kvh = blockIdx.x % n_kv;
    const WgDesc* wg = plan.wgs + wg_first + blockIdx.x / n_kv;
    const TileRef* tiles = plan.tiles + wg->coop_ofs;
    const int n_blk = wg->n_coop;
    const int rpt = plan.rows_per_thread;
    const int rank0 = wg->w[0].grp_lo / plan.n_slices, n_thr = wg->w[0].n_grp / plan.n_slices;
    const int last_fill = (tiles[n_blk - 1].meta >> 20) & 31;

    const int row = wave * 32 + n;
    const int tr = row / rpt, within = row - tr * rpt;
    Walk wk;
    wk.head_base = pool + (int64_t)kvh * kTileBytes;
    wk.block_stride = (int64_t)n_kv * kTileBytes;
    wk.table = unwritten(&tiles[0].blk);
    wk.table_stride = sizeof(TileRef) / sizeof(int32_t);
    wk.n_blk = n_blk;
    wk.len = (n_blk - 1) * 16 + last_fill;
    wk.row_ok = tr < n_thr;
    wk.pos = wk.len - 1;  // every row sees every filled slot
    wk.wave_ok = wave * 32 < n_thr * rpt;
    wk.w_first = wk.w_last = wk.len - 1;
    const int tr_ok = wk.row_ok ? tr : 0, within_ok = wk.row_ok ? within : 0;
    const int listed = plan.dfs_threads ? plan.dfs_threads[rank0 + tr_ok] : rank0 + tr_ok;
    const int cc = within_ok / group, hq = kvh * group + (within_ok - cc * group);
    wk.q_row = q + (((int64_t)listed * n_cand + cc) * n_q + hq) * 128;
    wk.scale_log2e = scale_log2e;
    f32x16 o[4];
    float m, l;
    walk_blocks<kTilesBf16>(wk, lds, o, m, l);

    // the row's state goes out as a partial result
    const float lt = l + other_half(l);
    if (!wk.row_ok) return;
    const int64_t slot = ((int64_t)(wg->w[0].part_base + tr) * n_cand + cc) * n_q + hq;
    float* dst = part.o + slot * 128 + 4 * h;
    auto write = [&](auto stream) {
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 v = {o[jj][4 * j + 0], o[jj][4 * j + 1], o[jj][4 * j + 2], o[jj][4 * j + 3]};
                f32x4* to = reinterpret_cast<f32x4*>(dst + 32 * jj + 16 * (j & 1) + 8 * (j >> 1));
                if constexpr (decltype(stream)::value) __builtin_nontemporal_store(v, to);
                else *to = v;
            }
    };
    if (part.stream) {
        asm volatile("" ::: "memory");  // (before and after: else the two branches' stores become one, without the hint)
        write(std::true_type{});
        asm volatile("" ::: "memory");
    } else {
        write(std::false_type{});
    }
    if (h == 0) {
        part.ml[slot * 2] = m;
        part.ml[slot * 2 + 1] = lt;
    }
}

}  // namespace

hipError_t launch_prefill_bf16(const Shape& s, const void* pool, const void* q, const PrefillWg* wgs,
                               const int32_t* tables, int n_wg, void* out, hipStream_t st) {
    if (n_wg <= 0) return hipSuccess;
    const int64_t grid = (int64_t)n_wg * s.n_kv;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    if (s.fp4) return launch_prefill_fp4(s, pool, q, wgs, tables, n_wg, out, st);
    if (s.fp8_sealed)
        hipLaunchKernelGGL(prefill_bf16<true>, dim3((unsigned)grid), dim3(256), 0, st, (const char*)pool, (const uint16_t*)q, wgs,
                           tables, s.n_q, s.n_kv, s.group, s.scale_log2e, (uint16_t*)out);
    else
        hipLaunchKernelGGL(prefill_bf16<false>, dim3((unsigned)grid), dim3(256), 0, st, (const char*)pool, (const uint16_t*)q, wgs,
                           tables, s.n_q, s.n_kv, s.group, s.scale_log2e, (uint16_t*)out);
    return hipGetLastError();
}

hipError_t launch_attention_units_bf16(const Shape& s, const void* pool, const void* q, const PlanDev& plan,
                                       int wg_first, int n_wg, int n_cand, PartialBuf part, hipStream_t st) {
    if (n_wg <= 0) return hipSuccess;
    const int64_t grid = (int64_t)n_wg * s.n_kv;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL(attention_units_bf16, dim3((unsigned)grid), dim3(256), 0, st, (const char*)pool,
                       (const uint16_t*)q, plan, wg_first, n_cand, s.n_q, s.n_kv, s.group, s.scale_log2e, part);
    return hipGetLastError();
}

}  // namespace apar
