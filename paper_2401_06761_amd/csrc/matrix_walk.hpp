// The walk of the kernels shaped for the 32x32 matrix instructions (kernels_matrix_bf16.hip says what it is), and the prefill kernels'
// body around it.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "apar_internal.hpp"

namespace apar {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

union Op {  // 16 bytes: a load, or an 8-wide bf16 operand
    u32x4 u;
    bf16x8 b8;
};

constexpr float kSlack = 8.0f;      // a probability may exceed 1 by at most 2^kSlack before the reference moves
constexpr int kTileBytes = 8192;    // one (block, kv head) in operand order: 4 KiB of K, 4 KiB of V
constexpr int kHalf = 4096;
constexpr int kBufBytes = 4 * kTileBytes;  // one staged group: four blocks, each K half then V half

__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {  // round to nearest even
    const f32x2 x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

__device__ __forceinline__ float other_half(float x) {  // the value of lane ^ 32
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r.x : r.y);
}

// fp8 codes in x[0], x[1] times the half's power-of-two scale -> the half's four bf16 pieces x[0..3].
__device__ __forceinline__ void widen(u32x4 (&x)[4], float scale) {
    const u32x4 raw[2] = {x[0], x[1]};
#pragma unroll
    for (int rp = 0; rp < 2; ++rp)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            x[2 * rp + (w >> 1)][2 * (w & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[rp][w], scale, false));
            x[2 * rp + (w >> 1)][2 * (w & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[rp][w], scale, true));
        }
}

// Eight 4-bit codes times a power of two -> eight bf16 values (exact).
__device__ __forceinline__ u32x4 widen_fp4_word(uint32_t w, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
__device__ __forceinline__ void widen_fp4(const u32x4& codes, float scale, u32x4 (&x)[4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = widen_fp4_word(codes[r], scale);
}

// What a wavefront brings to the walk.  `len` token slots are filled along the walk's block list
// (entry i of the list is table[i * table_stride]); the lane's row sees slots 0 .. pos.
struct Walk {
    const char* head_base;   // the pool at this kv head
    int64_t block_stride;
    const int32_t* table;
    int table_stride;
    int n_blk;               // blocks that hold a slot some row of the workgroup sees
    int len;
    bool wave_ok;            // the wavefront has rows at all
    int w_first, w_last;     // smallest and largest pos over the wavefront's rows (wavefront-uniform)
    bool row_ok;
    int pos;
    const uint16_t* q_row;   // the lane's query row (any valid row if !row_ok)
    float scale_log2e;
};

// Memory to LDS without a register in between: the lane's 16 bytes at from + ofs go to LDS address lds + 16 lane; dma_half
// brings the three KiB after that too.  Statements of their own rather than the builtin: the compiler takes that one for an
// access that either counter may count, and then has every operand read from LDS wait for all others.  Whoever requests
// waits for vmcnt(0) before anybody reads.  (The wait states cover a scalar register that a vector instruction has just
// written.)
__device__ __forceinline__ void dma_piece(const char* from, uint32_t ofs, uint32_t lds) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 4\n\t"
        "global_load_lds_dwordx4 %1, %2"
        :
        : "s"(lds), "v"(ofs), "s"(from)
        : "memory", "m0");
}
__device__ __forceinline__ void dma_half(const char* from, uint32_t ofs, uint32_t lds) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 4\n\t"
        "global_load_lds_dwordx4 %1, %2\n\t"
        "global_load_lds_dwordx4 %1, %2 offset:1024\n\t"
        "global_load_lds_dwordx4 %1, %2 offset:2048\n\t"
        "global_load_lds_dwordx4 %1, %2 offset:3072"
        :
        : "s"(lds), "v"(ofs), "s"(from)
        : "memory", "m0");
}

// What the pool holds: bf16 rows; full blocks in fp8 codes with two scales; 4-bit codes with a scale per 32 values.  Codes are widened when
// they are staged, so that LDS holds a bf16 tile.
enum { kTilesBf16, kTilesFp8, kTilesFp4 };
constexpr int tile_bytes_of(int tiles) { return tiles == kTilesFp4 ? kFp4TileBytes : kTileBytes; }

// The dim of O^T that a lane holds of its row in o[jj][4 j + i].  (A lane that stages a 4-bit V tile has eight consecutive dims of four
// slots; put where sealed bf16 blocks have them, they would leave it in eight stores that meet in a sixteenth of the banks.  They
// leave in four of 16 bytes, and the matrix rows stand for other dims.)
__device__ __forceinline__ constexpr int dim_of(int tiles, int jj, int j, int h, int i) {
    return tiles == kTilesFp4 ? 8 * (4 * h + i + 8 * (j >> 1)) + 2 * jj + (j & 1) : 32 * jj + 16 * (j & 1) + 8 * (j >> 1) + 4 * h + i;
}

// Runs the walk; leaves the lane's share of O^T (dim_of), the row's reference m and this lane's half of the row's sum l.
template <int TILES>
__device__ __forceinline__ void walk_blocks(const Walk& wk, char* lds, f32x16 (&o)[4], float& m, float& l) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n = lane & 31, h = lane >> 5;   // column (query row) and half of the 32x32 products
    // For the paths that only open blocks take: what is derived from it is not kept in registers over the walk.
    auto recomputed_lane = [&]() {
        int x = lane;
        asm volatile("" : "+v"(x));
        return x;
    };
    const char* head_base = wk.head_base;
    const int64_t block_stride = wk.block_stride;
    const int w_first = wk.w_first, pos = wk.pos;
    const float scale_log2e = wk.scale_log2e;

    // Q as the B operand: lane (n, h) holds dims 8 (2 s + h) .. + 8 of its row for product step s
    Op qv[8];
    {
        const u32x4* qp = reinterpret_cast<const u32x4*>(wk.q_row);
#pragma unroll
        for (int s = 0; s < 8; ++s) qv[s].u = wk.row_ok ? qp[2 * s + h] : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int jj = 0; jj < 4; ++jj)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[jj][i] = 0.0f;
    m = -INFINITY, l = 0.0f;
    float bias = -INFINITY;  // -m, or -inf as long as the row has seen nothing

    // groups of four blocks (64 token slots)
    const int n_blk = wk.n_blk;
    const int n_grp = (n_blk + 3) / 4;
    const int n_sb = wk.wave_ok ? (wk.w_last >> 5) + 1 : 0;  // super-blocks that some row of the wavefront sees
    // This wavefront stages block `wave` of every group (a group's last blocks may lie past the walk's last block: they
    // are masked, re-read the last one): request() when the group before is about to be consumed, land() when it has been.
    // Sealed blocks lie in LDS as they lie in HBM, and so do open ones once they have landed.
    const uint32_t lds_addr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    constexpr bool F8 = TILES == kTilesFp8, F4 = TILES == kTilesFp4;
    u32x4 sk[2], sv[2];        // the codes of a block in flight (fp8: of a full one; 4 bits: one piece of either half),
    f32x2 ssc = {1.0f, 1.0f};  // and its scales,
    uint32_t sk4 = 0, sv4 = 0; // or the bytes of this lane's
    auto request = [&](int g) {
        const int blk = min(4 * g + wave, n_blk - 1);
        const int fill = min(16, wk.len - blk * 16);
        const char* tile = head_base + __builtin_amdgcn_readfirstlane(wk.table[blk * wk.table_stride]) * block_stride;
        const uint32_t to = lds_addr + (g & 1) * kBufBytes + wave * kTileBytes;
        if constexpr (F4) {  // (a block that is still filling looks like a full one)
            sk[0] = *reinterpret_cast<const u32x4*>(tile + (lane & 15) * 64 + (lane >> 4) * 16);
            sv[0] = *reinterpret_cast<const u32x4*>(tile + kFp4V + lane * 16);
            sk4 = *reinterpret_cast<const uint8_t*>(tile + kFp4KScale + (lane & 15) * 4 + (lane >> 4));
            sv4 = *reinterpret_cast<const uint32_t*>(tile + kFp4VScale + (lane >> 4) * 16 + (lane & 12));
        } else if (F8 && fill == 16) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                sk[r] = *reinterpret_cast<const u32x4*>(tile + r * 1024 + lane * 16);
                sv[r] = *reinterpret_cast<const u32x4*>(tile + kFp8HalfBytes + r * 1024 + lane * 16);
            }
            ssc = *reinterpret_cast<const f32x2*>(tile + kFp8ScaleOfs);
        } else if (fill == 16) {
            dma_half(tile, lane * 16, to);
            dma_half(tile + kHalf, lane * 16, to + kHalf);
        } else {
            // the walk's last block is still open: row-major.  Piece r of this lane belongs to token row
            // 4r + g4; rows past the fill count re-read row 0 (finite values under probability 0)
            const int ln = recomputed_lane();
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int trow = 4 * r + (ln >> 4) < fill ? 4 * r + (ln >> 4) : 0;
                dma_piece(tile, trow * 256 + (ln & 15) * 16, to + r * 1024);
                dma_piece(tile + kHalf, trow * 256 + (ln & 15) * 16, to + kHalf + r * 1024);
            }
        }
    };
    // (the caller has waited for this wavefront's requests)
    auto land = [&](int g) {
        const int blk = min(4 * g + wave, n_blk - 1);
        const bool sealed = wk.len - blk * 16 >= 16;
        char* dst = lds + (g & 1) * kBufBytes + wave * kTileBytes;
        if constexpr (F4) {
            // K: dims 32 g .. + 31 of token c, as they lie in a sealed block
            u32x4 x[4];
            widen_fp4(sk[0], __uint_as_float(sk4 << 23), x);
#pragma unroll
            for (int r = 0; r < 4; ++r) *reinterpret_cast<u32x4*>(dst + r * 1024 + lane * 16) = x[r];
            // V: dims 8 c .. + 7 of slots 4 g + i; piece jj: dims 8 c + 2 jj, + 1 of the four slots
            u32x4 y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = widen_fp4_word(sv[0][i], __uint_as_float(((sv4 >> (8 * i)) & 0xffu) << 23));
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
                *reinterpret_cast<u32x4*>(dst + kHalf + jj * 1024 + lane * 16) =
                    u32x4{__builtin_amdgcn_perm(y[1][jj], y[0][jj], 0x05040100u), __builtin_amdgcn_perm(y[3][jj], y[2][jj], 0x05040100u),
                          __builtin_amdgcn_perm(y[1][jj], y[0][jj], 0x07060302u), __builtin_amdgcn_perm(y[3][jj], y[2][jj], 0x07060302u)};
        } else if (F8 && sealed) {
            // two 16-byte loads hold a half's four pieces at one byte per element (a code times a power of two: exact)
            u32x4 x[4] = {sk[0], sk[1], sk[0], sk[1]};
            widen(x, ssc[0]);
#pragma unroll
            for (int r = 0; r < 4; ++r) *reinterpret_cast<u32x4*>(dst + r * 1024 + lane * 16) = x[r];
            x[0] = sv[0], x[1] = sv[1];
            widen(x, ssc[1]);
#pragma unroll
            for (int r = 0; r < 4; ++r) *reinterpret_cast<u32x4*>(dst + kHalf + r * 1024 + lane * 16) = x[r];
        } else if (!sealed) {
            // piece r of this lane = slot 4r + g4, dims 8c .. 8c + 7 of the open block: put where a sealed one has them
            const int ln = recomputed_lane();
            u32x4 x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = *reinterpret_cast<const u32x4*>(dst + r * 1024 + ln * 16);
            asm volatile("" ::: "memory");  // (lanes read and write each other's pieces)
#pragma unroll
            for (int r = 0; r < 4; ++r) *reinterpret_cast<u32x4*>(dst + bf16_k_offset(4 * r + (ln >> 4), 8 * (ln & 15))) = x[r];
            dst += kHalf;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = *reinterpret_cast<const u32x4*>(dst + r * 1024 + ln * 16);
            asm volatile("" ::: "memory");  // (lanes read and write each other's pieces)
            // V: lanes c, 16 + c, 32 + c, 48 + c hold four slots of the same eight dims and swap words until each has all four
            // slots of two dims (thirty-two 2-byte stores per lane otherwise, eight lanes of each into the same bank)
            const int g4 = ln >> 4, c = ln & 15;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const u32x2 a = __builtin_amdgcn_permlane32_swap(x[r][0], x[r][2], false, false);
                const u32x2 b = __builtin_amdgcn_permlane32_swap(x[r][1], x[r][3], false, false);
                const u32x2 t01 = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false);  // word g4 of slots 4r, 4r + 1
                const u32x2 t23 = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);  // ... 4r + 2, 4r + 3
                const u32x2 even = {(t01.x & 0xffffu) | (t01.y << 16), (t23.x & 0xffffu) | (t23.y << 16)};
                const u32x2 odd = {(t01.x >> 16) | (t01.y & 0xffff0000u), (t23.x >> 16) | (t23.y & 0xffff0000u)};
                *reinterpret_cast<u32x2*>(dst + bf16_v_offset(4 * r, 8 * c + 2 * g4)) = even;
                *reinterpret_cast<u32x2*>(dst + bf16_v_offset(4 * r, 8 * c + 2 * g4 + 1)) = odd;
            }
        }
    };
    // every wavefront's requests have landed, and everyone has read what it needs of the group before
    auto hand_over = [&](int g) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
        land(g);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // Operands of the super-block whose two blocks lie at `at`.  K: lane (n as token slot, h) reads dims 8 (2 s + h) .. + 8 of
    // slot n % 16 of block n / 16.  V: lane (n as matrix row, h) reads slots 4h .. 4h + 3, then 8 + 4h .. 8 + 4h + 3, of one
    // dim; which of the 32 dims a matrix row stands for is chosen so that eight chunks of 16 bytes - two dims each -
    // serve sixteen lanes (the sixteen lanes of dims c = 0..15 instead would meet in half the banks, twice).
    const int k_lane = (n >> 4) * kTileBytes + (n & 15) * 16 + h * 1024;
    const int v_lane = kHalf + (h * 16 + (n & 7) + 8 * (n >> 4)) * 16 + 8 * ((n >> 3) & 1);
    Op ka[8], va[8];
    float top = -INFINITY;  // the largest of the lane's logits of the super-block to come, unscaled
    auto load_k = [&](const char* at, int k) {
        ka[k].u = *reinterpret_cast<const u32x4*>(at + k_lane + (k & 1) * 2048 + (k >> 1) * 256);
    };
    auto load_v = [&](const char* at, int k) {  // k = 4 block + jj
        const char* p = at + v_lane + (k >> 2) * kTileBytes + (k & 3) * 1024;
        const u32x2 lo = *reinterpret_cast<const u32x2*>(p), hi = *reinterpret_cast<const u32x2*>(p + 512);
        va[k].u = u32x4{lo.x, lo.y, hi.x, hi.y};
    };
    // slot t0 + 8 (i / 4) + 4 h + i % 4 is visible up to the row's pos; only super-blocks near the rows' limits need it
    auto mask = [&](f32x16& s, int t0) {
        if (t0 + 31 > w_first) {
            const int room = pos - t0 - 4 * h;  // visible iff 8 (i / 4) + i % 4 <= room
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = (8 * (i >> 2) + (i & 3) <= room) ? s[i] : -INFINITY;
        }
    };
    // If some row ran away from its reference (always so on a row's first super-block): move every row's reference to its
    // running maximum (the two lanes of a row agree on it) and rescale.
    auto settle = [&]() {
        const float t = top * scale_log2e;
        if (__builtin_amdgcn_ballot_w64(t > m + kSlack) != 0) {
            const float mx = fmaxf(t, other_half(t));
            const float m_new = fmaxf(m, mx);
            const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
            l *= alpha;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[jj][i] *= alpha;
            m = m_new;
            bias = m != -INFINITY ? -m : -INFINITY;
        }
    };
    // Probabilities of the super-block whose logits are s, among the K.Q^T products of the one after it (logits sn, first
    // slot t0n), then the V^T.P^T products among the maximum over sn.  The order is fixed: a wavefront's vector instructions
    // run beside its own products only if they are issued between them.  (After a wavefront's last super-block sn comes from
    // whatever is staged and nobody looks at it: eight products too many per walk, between vector instructions.)
    auto weigh = [&](const f32x16& s, f32x16& sn, int t0n, auto beside_k, auto beside_v) {
        Op pb[2];
        float x0 = __builtin_fmaf(s[0], scale_log2e, bias), x1 = __builtin_fmaf(s[1], scale_log2e, bias);
        float sum0 = 0.0f, sum1 = 0.0f, p0 = 0.0f, p1 = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sn[i] = 0.0f;
#pragma unroll
        for (int step = 0; step < 8; ++step) {
            sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[step].b8, qv[step].b8, sn, 0, 0, 0);
            beside_k(step);
            const float e0 = __builtin_amdgcn_exp2f(x0), e1 = __builtin_amdgcn_exp2f(x1);
            if (step < 7) {
                x0 = __builtin_fmaf(s[2 * step + 2], scale_log2e, bias);
                x1 = __builtin_fmaf(s[2 * step + 3], scale_log2e, bias);
            }
            if (step > 0) {
                sum0 += p0;
                sum1 += p1;
                uint32_t w = pack_pair(p0, p1);
                asm volatile("" : "+v"(w), "+v"(sum0), "+v"(sum1));  // (else they sink below the branch that masks sn)
                pb[(step - 1) >> 2].u[(step - 1) & 3] = w;
            }
            p0 = e0, p1 = e1;
            asm volatile("" : "+v"(p0), "+v"(p1));
            __builtin_amdgcn_sched_barrier(0);
        }
        l += (sum0 + p0) + (sum1 + p1);
        pb[1].u[3] = pack_pair(p0, p1);
        mask(sn, t0n);
        top = fmaxf(sn[0], sn[1]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            o[k & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[k].b8, pb[k >> 2].b8, o[k & 3], 0, 0, 0);
            beside_v(k);
            if (k > 0) top = fmaxf(fmaxf(top, sn[2 * k]), sn[2 * k + 1]);
            asm volatile("" : "+v"(top));
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    request(0);
    hand_over(0);
    if (n_grp > 1) request(1);
    f32x16 s0, s1;
    int g = 0;
    if (n_sb > 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) load_k(lds, k);
#pragma unroll
        for (int i = 0; i < 16; ++i) s0[i] = 0.0f;
#pragma unroll
        for (int s = 0; s < 8; ++s) s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[s].b8, qv[s].b8, s0, 0, 0, 0);
        mask(s0, 0);
        top = s0[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s0[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) load_k(lds + 2 * kTileBytes, k);
        // Group by group; at the top of the loop s0 holds the logits of the group's first super-block and ka the K operands
        // of its second one.  Operands are read from LDS beside products, into registers that have just become free.
        for (; 2 * g < n_sb; ++g) {
            const char* buf = lds + (g & 1) * kBufBytes;
            const char* other = lds + ((g + 1) & 1) * kBufBytes;
            settle();
            weigh(s0, s1, 64 * g + 32, [&](int k) { load_v(buf, k); }, [&](int k) { load_v(buf + 2 * kTileBytes, k); });
            if (2 * g + 1 >= n_sb) break;
            if (g + 1 < n_grp) {
                hand_over(g + 1);
                if (g + 2 < n_grp) request(g + 2);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) load_k(other, k);
            settle();
            weigh(s1, s0, 64 * g + 64, [](int) {}, [&](int k) { load_k(other + 2 * kTileBytes, k); });
        }
    }
    for (; g + 1 < n_grp; ++g) {  // a wavefront without rows, or whose rows end before the walk does, goes on staging
        hand_over(g + 1);
        if (g + 2 < n_grp) request(g + 2);
    }
    __syncthreads();
}

// A workgroup of a prefill kernel: up to 128 query rows of one thread.  lds: 2 * kBufBytes.
template <int TILES>
__device__ __forceinline__ void prefill_rows(char* lds, const char* __restrict__ pool, const uint16_t* __restrict__ q, const PrefillWg* __restrict__ wgs,
                                             const int32_t* __restrict__ tables, int n_q, int n_kv, int group, float scale_log2e,
                                             uint16_t* __restrict__ out) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n = lane & 31, h = lane >> 5;
    const int kvh = blockIdx.x % n_kv;
    const PrefillWg wg = wgs[blockIdx.x / n_kv];

    // this lane's query row: token tq of the workgroup's chunk, q head hg of the kv group
    const int row = wave * 32 + n;
    const int tq = row / group, hg = row - tq * group;
    const int w_tok0 = (wave * 32) / group;
    Walk wk;
    wk.head_base = pool + (int64_t)kvh * tile_bytes_of(TILES);
    wk.block_stride = (int64_t)n_kv * tile_bytes_of(TILES);
    wk.table = tables + wg.table_ofs;
    wk.table_stride = 1;
    wk.n_blk = (wg.p0 + wg.n_tok - 1) / 16 + 1;  // blocks that hold an attended token
    wk.len = wg.len;
    wk.row_ok = tq < wg.n_tok;
    wk.pos = wg.p0 + (wk.row_ok ? tq : 0);  // position of the row's token in the thread
    // first and last query position of the wavefront
    wk.wave_ok = w_tok0 < wg.n_tok;
    wk.w_first = wg.p0 + w_tok0;
    wk.w_last = wg.p0 + min(wg.n_tok - 1, (wave * 32 + 31) / group);
    const int64_t qrow = ((int64_t)(wg.q_row0 + (wk.row_ok ? tq : 0)) * n_q) + kvh * group + hg;
    wk.q_row = q + qrow * 128;
    wk.scale_log2e = scale_log2e;
    f32x16 o[4];
    float m, l;
    walk_blocks<TILES>(wk, lds, o, m, l);

    // Normalise and write.  The rows go through LDS (the walk ended with a barrier) so that a store instruction writes
    // four whole rows of 256 bytes: a lane holds its row in runs of four dims, and stores of 8 bytes per lane, 16 per
    // row, leave the L2 as partial lines (80 requests, 480 segments of 107 tokens, walks of 300, 32 heads, 0.85 GB of
    // queries and outputs: 1580 us with non-temporal stores of 8 bytes, 678 with plain ones, 650 this way).
    const float lt = l + other_half(l);
    const float inv = 1.0f / lt;
    constexpr int kStride = 256 + 16;  // padded: the rows of a column of lanes start in different banks
    char* rows = lds + wave * 32 * kStride;
    if constexpr (TILES == kTilesFp4) {
#pragma unroll
        for (int jh = 0; jh < 2; ++jh)
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // eight consecutive dims
                u32x4 pk;
#pragma unroll
                for (int jj = 0; jj < 4; ++jj) pk[jj] = pack_pair(o[jj][8 * jh + i] * inv, o[jj][8 * jh + 4 + i] * inv);
                *reinterpret_cast<u32x4*>(rows + n * kStride + dim_of(TILES, 0, 2 * jh, h, i) * 2) = pk;
            }
    } else {
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x2 pk;
                pk.x = pack_pair(o[jj][4 * j + 0] * inv, o[jj][4 * j + 1] * inv);
                pk.y = pack_pair(o[jj][4 * j + 2] * inv, o[jj][4 * j + 3] * inv);
                *reinterpret_cast<u32x2*>(rows + n * kStride + dim_of(TILES, jj, j, h, 0) * 2) = pk;
            }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int it = 0; it < 8; ++it) {
        const int r = 4 * it + (lane >> 4);
        const u32x4 x = *reinterpret_cast<const u32x4*>(rows + r * kStride + (lane & 15) * 16);
        const int t2 = (wave * 32 + r) / group, h2 = wave * 32 + r - t2 * group;
        if (t2 >= wg.n_tok) continue;
        uint16_t* dst = out + (((int64_t)(wg.q_row0 + t2) * n_q) + kvh * group + h2) * 128;
        __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(dst) + (lane & 15));
    }
}

}  // namespace

}  // namespace apar
