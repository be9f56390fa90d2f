// Rows into and out of 4-bit pools (APAR_BF16_FP4KV; layout in apar_internal.hpp).
//
// A group of 32 values x of a row becomes e2m1 codes under the scale 2^e, the smallest with max|x| / 2^e <= 6.  With the
// largest magnitude as bf16, (1 + m / 128) 2^(E - 127): 6 = 1.5 * 4, so e + 127 = E - 2 where m <= 64 and E - 1 elsewhere.
// Codes are rounded to nearest even by the hardware conversion that divides by the scale.  Eight dims are a lane's: a
// group is four neighbouring lanes'.  Blocks that a call writes whole have lanes of their own for K and V, and stores of 16 bytes.
// What bounds them: the chain load, largest magnitude of four lanes, conversion, store, once (a prompt of 4 k rows, 8 kv heads,
// 17 MB in and 4.5 out: 14 us, read back in 7.5); short calls their launch.
#include <hip/hip_runtime.h>

#include <cstring>

#include "apar_internal.hpp"

namespace apar {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
constexpr uint32_t kMost = 0x7f407f40u;  // 6 * 2^125 = 1.5 * 2^127, the largest magnitude the format holds, as bf16, twice

// Eight values as the format holds them - magnitudes beyond 6 * 2^125, infinities included, as that; NaN as 0 -, and the largest magnitude.
// Two values at a time; NaN have a branch.
__device__ __forceinline__ uint32_t held_run(u32x4& x) {
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, (uint32_t)(x[i] & 0x7fff7fffu)));
    if (__builtin_amdgcn_ballot_w64(max(top.x, top.y) > 0x7f80) != 0) {
        top = u16x2{0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((x[i] & 0x7fffu) > 0x7f80u) x[i] &= 0xffff0000u;
            if ((x[i] & 0x7fff0000u) > 0x7f800000u) x[i] &= 0xffffu;
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, (uint32_t)(x[i] & 0x7fff7fffu)));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u16x2 mag = __builtin_elementwise_min(__builtin_bit_cast(u16x2, (uint32_t)(x[i] & 0x7fff7fffu)), __builtin_bit_cast(u16x2, kMost));
        x[i] = (x[i] & 0x80008000u) | __builtin_bit_cast(uint32_t, mag);
    }
    return min((uint32_t)max(top.x, top.y), kMost & 0xffffu);
}
// The scale's byte for a group whose largest magnitude is `top`.
__device__ __forceinline__ uint32_t scale_for(uint32_t top) {
    const int b = (int)(top >> 7) - 2 + ((top & 127u) > 64u ? 1 : 0);
    return top == 0u ? 127u : (uint32_t)max(b, 7);
}
__device__ __forceinline__ uint32_t codes_of(const u32x4& x, uint32_t scale) {
    const float s = __uint_as_float(scale << 23);
    // (words of their own: a bit_cast of a vector's element takes the first one, whichever it names)
    const uint32_t w[4] = {x[0], x[1], x[2], x[3]};
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), s, 3);
}

// Eight dims of a row, 16 bytes -> their codes; scale: the byte of the lane's group.  All lanes of a group call together.
__device__ __forceinline__ uint32_t quantise(u32x4 x, uint32_t& scale) {
    uint32_t top = held_run(x);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    scale = scale_for(top);
    return codes_of(x, scale);
}

// Byte offsets in a tile of a token's word c (dims 8 c .. + 7) and of the scale of group g.
__device__ __forceinline__ int k_word(int t, int c) { return 64 * t + 4 * c; }
__device__ __forceinline__ int v_word(int t, int c) { return kFp4V + ((t >> 2) * 16 + c) * 16 + (t & 3) * 4; }
__device__ __forceinline__ int k_scale(int t, int g) { return kFp4KScale + 4 * t + g; }
__device__ __forceinline__ int v_scale(int t, int g) { return kFp4VScale + (t >> 2) * 16 + 4 * g + (t & 3); }

// FROM: where the descriptors and the source rows are (in the kernel's arguments: its first one).  The first workgroups take the
// blocks that are written whole, a wavefront per (block, kv head): V with dims 8 c .. + 7 of tokens 4 g .. + 3 in lane 16 g + c, K with
// group g of token t in lane 4 t + g, so that the codes of either leave as one contiguous KiB and K's groups need no other lane.  The others take the blocks that get a few rows, sixteen lanes per (block, kv head): the rows
// before the new ones where the block is the copy of a shared one, then the new ones.  Scales of V slots that are not written yet are
// set to 0 when a block is begun, so that a reader may widen them.
template <int FROM>
__global__ __launch_bounds__(256) void append_fp4(AppendTables<FROM> tables, char* __restrict__ pool, const char* __restrict__ k,
                                                  const char* __restrict__ v, int n_blocks, int n_open, int n_src, int n_kv) {
    auto block_at = [&](int at) -> AppendBlock {
        if constexpr (FROM == kAppendRun) {
            typedef const int32_t __attribute__((address_space(4))) * Words;
            const auto w = (Words)__builtin_amdgcn_kernarg_segment_ptr();
            const int before = w[0];
            if (at < before) return AppendBlock{w[4 + 4 * at], w[5 + 4 * at], w[6 + 4 * at], w[7 + 4 * at]};
            return AppendBlock{w[4 + 3 * before + at], -1, w[1] + 16 * (at - before), 16 << 8};
        } else if constexpr (FROM == kAppendArguments) {
            typedef const AppendBlock __attribute__((address_space(4))) * Blocks;
            const auto* p = (Blocks)__builtin_amdgcn_kernarg_segment_ptr() + at;
            return AppendBlock{p->dst, p->copy_of, p->first, p->slots};
        } else {
            return reinterpret_cast<const AppendBlock*>(tables.words)[at];
        }
    };
    auto src_of = [&](int i) -> int {
        if constexpr (FROM == kAppendRun) {
            return i;  // (a run has no list of source rows)
        } else if constexpr (FROM == kAppendArguments) {
            typedef const int32_t __attribute__((address_space(4))) * Words;
            return ((Words)__builtin_amdgcn_kernarg_segment_ptr())[4 * n_blocks + i];
        } else {
            return tables.words[4 * n_blocks + i];
        }
    };
    auto row_of = [&](const AppendBlock& b, int slot) -> int64_t {
        const int row = b.first + slot - (b.slots & 255);
        return n_src ? src_of(row) : row;
    };
    const int c = threadIdx.x & 15;
    const int whole_wgs = (int)(((int64_t)(n_blocks - n_open) * n_kv + 3) / 4);
    if ((int)blockIdx.x < whole_wgs) {
        const int g4 = (threadIdx.x & 63) >> 4;
        const int item = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));  // heads fastest
        const int at = item / n_kv, h = item - at * n_kv;
        if (at >= n_blocks - n_open) return;
        const AppendBlock b = block_at(n_open + at);
        char* tile = pool + ((int64_t)b.dst * n_kv + h) * kFp4TileBytes;
        const int lane = threadIdx.x & 63;
        u32x4 kx[4], vx[4];
        const char* k_row = k + (row_of(b, lane >> 2) * n_kv + h) * 256 + (lane & 3) * 64;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kx[i] = *reinterpret_cast<const u32x4*>(k_row + i * 16);
            vx[i] = *reinterpret_cast<const u32x4*>(v + (row_of(b, 4 * g4 + i) * n_kv + h) * 256 + c * 16);
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, held_run(kx[i]));
        const uint32_t ks = scale_for(top);
        *reinterpret_cast<u32x4*>(tile + lane * 16) = u32x4{codes_of(kx[0], ks), codes_of(kx[1], ks), codes_of(kx[2], ks), codes_of(kx[3], ks)};
        *reinterpret_cast<uint8_t*>(tile + kFp4KScale + lane) = (uint8_t)ks;
        u32x4 vc;
        uint32_t vs = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t s;
            vc[i] = quantise(vx[i], s);
            vs |= s << (8 * i);
        }
        *reinterpret_cast<u32x4*>(tile + v_word(4 * g4, c)) = vc;
        if ((c & 3) == 0) *reinterpret_cast<uint32_t*>(tile + v_scale(4 * g4, c >> 2)) = vs;
        return;
    }
    const int pair = ((int)blockIdx.x - whole_wgs) * 16 + (int)(threadIdx.x >> 4);  // (block, kv head), heads fastest
    const int at = pair / n_kv, h = pair - at * n_kv;
    if (at >= n_open) return;
    const AppendBlock b = block_at(at);
    char* tile = pool + ((int64_t)b.dst * n_kv + h) * kFp4TileBytes;
    const int s0 = b.slots & 255, s1 = b.slots >> 8;
    if (b.copy_of >= 0) {
        const char* old = pool + ((int64_t)b.copy_of * n_kv + h) * kFp4TileBytes;
        for (int t = 0; t < s0; ++t) {
            *reinterpret_cast<uint32_t*>(tile + k_word(t, c)) = *reinterpret_cast<const uint32_t*>(old + k_word(t, c));
            *reinterpret_cast<uint32_t*>(tile + v_word(t, c)) = *reinterpret_cast<const uint32_t*>(old + v_word(t, c));
            if ((c & 3) == 0) {
                *reinterpret_cast<uint8_t*>(tile + k_scale(t, c >> 2)) = *reinterpret_cast<const uint8_t*>(old + k_scale(t, c >> 2));
                *reinterpret_cast<uint8_t*>(tile + v_scale(t, c >> 2)) = *reinterpret_cast<const uint8_t*>(old + v_scale(t, c >> 2));
            }
        }
    }
    for (int t = s0; t < s1; ++t) {
        const int64_t from = (row_of(b, t) * n_kv + h) * 256 + c * 16;
        const u32x4 kx = *reinterpret_cast<const u32x4*>(k + from), vx = *reinterpret_cast<const u32x4*>(v + from);
        uint32_t ks, vs;
        const uint32_t kc = quantise(kx, ks), vc = quantise(vx, vs);
        *reinterpret_cast<uint32_t*>(tile + k_word(t, c)) = kc;
        *reinterpret_cast<uint32_t*>(tile + v_word(t, c)) = vc;
        if ((c & 3) == 0) {
            *reinterpret_cast<uint8_t*>(tile + k_scale(t, c >> 2)) = (uint8_t)ks;
            *reinterpret_cast<uint8_t*>(tile + v_scale(t, c >> 2)) = (uint8_t)vs;
        }
    }
    if ((s0 == 0 || b.copy_of >= 0) && (c & 3) == 0)  // the block is begun here
        for (int t = s1; t < 16; ++t) *reinterpret_cast<uint8_t*>(tile + v_scale(t, c >> 2)) = 0;
}

// The first row's slot, then the blocks that the rows lie in: on the device, or (read where they are) the first argument itself.
struct ReadHere {
    int32_t words[kFp4ReadWords];
};
struct ReadThere {
    const int32_t* words;
};
template <class TABLE>
__global__ __launch_bounds__(256) void read_rows_fp4(TABLE table, const char* __restrict__ pool, uint16_t* __restrict__ k,
                                                     uint16_t* __restrict__ v, int n_rows, int n_kv) {
    typedef const int32_t __attribute__((address_space(4))) * Words;
    Words words;
    if constexpr (sizeof(TABLE) == sizeof(ReadThere)) words = (Words)table.words;
    else words = (Words)__builtin_amdgcn_kernarg_segment_ptr();
    const int64_t item = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);  // (row, kv head), heads fastest; sixteen lanes each
    const int64_t row = item / n_kv;
    if (row >= n_rows) return;
    const int h = (int)(item - row * n_kv), c = threadIdx.x & 15;
    const int at = words[0] + (int)row, t = at & 15;
    const char* tile = pool + ((int64_t)words[1 + (at >> 4)] * n_kv + h) * kFp4TileBytes;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(tile + (half ? v_word(t, c) : k_word(t, c)));
        const uint32_t b = *reinterpret_cast<const uint8_t*>(tile + (half ? v_scale(t, c >> 2) : k_scale(t, c >> 2)));
        const float s = __uint_as_float(b << 23);
        u32x4 x;
        x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
        x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
        x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
        x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
        *reinterpret_cast<u32x4*>((half ? v : k) + (row * n_kv + h) * 128 + c * 8) = x;
    }
}

}  // namespace

hipError_t launch_append_fp4(const Shape& s, void* pool, const void* k, const void* v, const int32_t* words, bool on_host,
                             int n_blocks, int n_open, int n_src, hipStream_t st) {
    if (n_blocks <= 0) return hipSuccess;
    const int64_t grid = ((int64_t)n_open * s.n_kv + 15) / 16 + ((int64_t)(n_blocks - n_open) * s.n_kv + 3) / 4;
    if (grid > 0x7fffffff || (int64_t)n_blocks * s.n_kv > 0x7fffffff) return hipErrorInvalidValue;
#define APAR_APPEND(FROMV, TABLES)                                                                                                 \
    hipLaunchKernelGGL((append_fp4<FROMV>), dim3((unsigned)grid), dim3(256), 0, st, TABLES, (char*)pool, (const char*)k, (const char*)v, \
                       n_blocks, n_open, n_src, s.n_kv)
    if (!on_host) {
        APAR_APPEND(kAppendDevice, AppendTables<kAppendDevice>{words});
    } else if ((size_t)4 * n_blocks + n_src > sizeof(AppendTables<kAppendArguments>) / sizeof(int32_t)) {
        const AppendBlock* b = (const AppendBlock*)words;
        const int before = n_src == 0 ? append_run(b, n_blocks) : -1;
        if (before < 0) return hipErrorInvalidValue;
        AppendTables<kAppendRun> run;
        run.words[0] = before;
        run.words[1] = b[before].first;
        run.words[2] = run.words[3] = 0;
        memcpy(run.words + 4, b, before * sizeof(AppendBlock));
        for (int i = before; i < n_blocks; ++i) run.words[4 + 3 * before + i] = b[i].dst;
        APAR_APPEND(kAppendRun, run);
    } else {
        AppendTables<kAppendArguments> args;
        memcpy(args.words, words, ((size_t)4 * n_blocks + n_src) * sizeof(int32_t));
        APAR_APPEND(kAppendArguments, args);
    }
#undef APAR_APPEND
    return hipGetLastError();
}

hipError_t launch_read_rows_fp4(const Shape& s, const void* pool, const int32_t* words, int n_rows, void* k_out, void* v_out, hipStream_t st) {
    const int64_t grid = ((int64_t)n_rows * s.n_kv + 15) / 16;
    if (grid > 0x7fffffff || n_rows > 0x7fffffff - 16) return hipErrorInvalidValue;
#define APAR_READ(TABLE, ARG) \
    hipLaunchKernelGGL(read_rows_fp4<TABLE>, dim3((unsigned)grid), dim3(256), 0, st, ARG, (const char*)pool, (uint16_t*)k_out, (uint16_t*)v_out, n_rows, s.n_kv)
    if (n_rows <= kFp4ReadHereRows) {
        ReadHere here;
        memcpy(here.words, words, (1 + (words[0] + (size_t)n_rows + kBlockTokens - 1) / kBlockTokens) * sizeof(int32_t));
        APAR_READ(ReadHere, here);
    } else {
        APAR_READ(ReadThere, ReadThere{words});
    }
#undef APAR_READ
    return hipGetLastError();
}

}  // namespace apar
