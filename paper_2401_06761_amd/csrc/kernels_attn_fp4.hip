// Attention over tiles that hold K and V in 4 bits (APAR_BF16_FP4KV pools; layout in apar_internal.hpp) on the gfx950 matrix cores.
//
// The same plan as the other row-tile kernels: query rows on the N side of 16x16 products, token slots on the M side,
// two tiles (32 token slots) at a time:
//
//   S^T[token][row] = K[token][:] . Q[row][:]       2 x mfma_scale_f32_16x16x128_f8f6f4 per tile
//   O^T[dim][row]  += V^T[dim][token] . P^T[token][row]   8 x mfma_f32_16x16x32_bf16 per pair of tiles
//
// K is never widened: a lane's 16 bytes are the 32 dims of one group of its token, e2m1 codes as the instruction takes them, and
// the group's power-of-two scale is its scale operand.  The other operand has at least 8 bits per value where either is
// more than 4, so Q goes in as the sum of two e4m3 values under power-of-two scales per 32 dims: the nearest one, and what it
// leaves (at most half a step of it, 2^-4 of it), under 1/16 of the scale.  A bf16 value has 8 significant bits and each term 4, so
// that sum is exact down to 2^-10 of the group's largest value, and off by no more than 2^-22 of that below.
// (The instruction's own sums: off by 4.6e-5 in the mean square for products that reach 45, 4.1e-4 for 720, i.e. some 6e-7
// of the largest.)
// With lane = 16 g + c:
//   K:  dims 32 g .. + 31 of token c        Q: dims 16 g .. + 15 and 64 + 16 g .. + 15 of row c
//   V:  dims 8 c .. 8 c + 7 of tokens 4 g .. 4 g + 3, widened by the conversion that multiplies by the scale (exact in bf16); product
//       jj contracts the tokens 4 g + i of both tiles into dims 8 m + jj
//   S:  logits of tokens 4 g + i of row c, which is the operand layout of P (no lane exchange)
//   O:  dims 8 (4 g + i) + jj of row c: 32 consecutive ones
// so every load is as wide as a lane's share of the tile, no value moves between lanes and nothing is staged: a tile goes from memory
// to operand registers, for the tiles of the shared list as for a wavefront's own (the four wavefronts of a workgroup meet in
// the caches).  A block that is still filling looks like a full one.
//
// A row that does not see a slot meets it with probability 0, and 0 times an infinity is a NaN: what is stored is always
// finite (infinities and NaN have no code), unwritten slots have finite scales (written when the block is begun), logits are
// replaced, not biased, where a row does not see the token.  Candidates' rows are the caller's: where one is not finite, its
// thread's are taken one by one.
//
// What bounds it: HBM where a tile serves few rows (256 requests of four threads, 2 k to 4 k tokens, 32/8 heads: 1.16 GB in 210 us, 5.5 TB/s, where a bare
// read of 2176-byte tiles reaches 6.1), vector instructions behind that (181 for a pair of tiles and 16 rows, 12 matrix ones), and
// those alone where it serves many (60 requests of five threads of 48 rows: 0.36 PFLOP/s); a short call its launch.
#include <hip/hip_runtime.h>

#include <cstring>
#include <type_traits>

#include "apar_internal.hpp"
#include "attn_split.hpp"

namespace apar {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kSlack = 8.0f;  // a probability may exceed 1 by at most 2^kSlack before the reference moves

__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {  // round to nearest even
    const f32x2 x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

struct Row {  // the 16 rows of one tile: query operands (nearest e4m3 values, what they leave, their scales) and softmax state
    i32x8 hi, lo;
    int32_t hi_scale, lo_scale;  // of dims 32 g .. + 31
    f32x4 o[8];
    float m, l;
};

struct Tile {  // as this lane has it: codes, the byte of its K group's scale, the bytes of its four tokens' V scales
    u32x4 k, v;
    uint32_t ks, vs;
};

// The query operands of this lane's row; `src`: the row (any one where there is none: no branch around a load).
__device__ __forceinline__ void load_query(Row& st, const uint16_t* src, bool ok, int g4, int c) {
    const u32x4* p = reinterpret_cast<const u32x4*>(src + 16 * g4);
    const u32x4 u[2][2] = {{p[0], p[1]}, {p[8], p[9]}};
    float x[2][16];
    float top[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        top[h] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = ok ? u[h][i >> 2][i & 3] : 0u;
            x[h][2 * i] = __uint_as_float(w << 16);
            x[h][2 * i + 1] = __uint_as_float(w & 0xffff0000u);
            top[h] = fmaxf(top[h], fmaxf(fabsf(x[h][2 * i]), fabsf(x[h][2 * i + 1])));
        }
        top[h] = fmaxf(top[h], __shfl_xor(top[h], 16, 64));  // (dims 64 h + 32 (g / 2) .. + 31 are two lanes')
    }
    int e[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const bool fine = top[h] < INFINITY;
        int k = 0;
        const float f = frexpf(fine ? top[h] : 0.0f, &k);  // top = f * 2^k, f in [0.5, 1); 448 = 0.875 * 2^9
        e[h] = top[h] > 0.0f && fine ? max(f <= 0.875f ? k - 9 : k - 8, -120) : 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            float y[4], r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fine ? ldexpf(x[h][4 * w + i], -e[h]) : __builtin_nanf("");
            uint32_t n = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            n = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], n, true);
            r[0] = (y[0] - __builtin_amdgcn_cvt_f32_fp8(n, 0)) * 16.0f;
            r[1] = (y[1] - __builtin_amdgcn_cvt_f32_fp8(n, 1)) * 16.0f;
            r[2] = (y[2] - __builtin_amdgcn_cvt_f32_fp8(n, 2)) * 16.0f;
            r[3] = (y[3] - __builtin_amdgcn_cvt_f32_fp8(n, 3)) * 16.0f;
            uint32_t d = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false);
            d = __builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], d, true);
            st.hi[4 * h + w] = (int32_t)n;
            st.lo[4 * h + w] = (int32_t)d;
        }
    }
    // group g of 32 dims lies with lanes 2 (g % 2) and 2 (g % 2) + 1 of the row, in half g / 2
    const int from = (2 * (g4 & 1)) * 16 + c;
    const int a = __shfl(e[0], from, 64), b = __shfl(e[1], from, 64);
    st.hi_scale = (g4 < 2 ? a : b) + 127;
    st.lo_scale = st.hi_scale - 4;
}

__device__ __forceinline__ f32x4 products(const Tile& t, const Row& st) {
    const i32x8 k = {(int32_t)t.k[0], (int32_t)t.k[1], (int32_t)t.k[2], (int32_t)t.k[3], 0, 0, 0, 0};
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, st.lo, s, 4, 0, 0, (int32_t)t.ks, 0, st.lo_scale);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, st.hi, s, 4, 0, 0, (int32_t)t.ks, 0, st.hi_scale);
}

// Moves every row's reference to its running maximum where some row's logits ran away from it (its four lanes agree on it).
__device__ __forceinline__ void move_reference(Row& st, float top) {
    if (__builtin_amdgcn_ballot_w64(top > st.m + kSlack) == 0) return;
    float mx = fmaxf(top, __shfl_xor(top, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(st.m, mx);
    const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(st.m - m_new);
    st.l *= alpha;
#pragma unroll
    for (int jj = 0; jj < 8; ++jj) st.o[jj] *= alpha;
    st.m = m_new;
}

// Two tiles' logits (-inf where this lane's row does not see the token) -> the operand of their probabilities, added to the row's sum.
__device__ __forceinline__ bf16x8 probabilities(Row& st, const f32x4& a, const f32x4& b, float scale_log2e) {
    const float top = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3]))) * scale_log2e;
    move_reference(st, top);
    const float bias = st.m != -INFINITY ? -st.m : -INFINITY;  // (a row that has seen nothing yet)
    float p[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(a[i], scale_log2e, bias));
        p[4 + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(b[i], scale_log2e, bias));
    }
    st.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    const u32x4 pw = {pack_pair(p[0], p[1]), pack_pair(p[2], p[3]), pack_pair(p[4], p[5]), pack_pair(p[6], p[7])};
    return __builtin_bit_cast(bf16x8, pw);
}

// This lane's V values of a tile: w[j] = tokens 4 g, + 1 and 4 g + 2, + 3 of dim 8 c + 2 j, then of the next dim.
__device__ __forceinline__ void widen(const Tile& t, uint32_t (&w)[4][4]) {
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = __uint_as_float(((t.vs >> (8 * i)) & 0xffu) << 23);
    auto two_dims = [&](auto J) {
        constexpr int j = decltype(J)::value;
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[i], s[i], j));
        w[j][0] = low_halves(x[0], x[1]);
        w[j][1] = low_halves(x[2], x[3]);
        w[j][2] = high_halves(x[0], x[1]);
        w[j][3] = high_halves(x[2], x[3]);
    };
    two_dims(std::integral_constant<int, 0>{});
    two_dims(std::integral_constant<int, 1>{});
    two_dims(std::integral_constant<int, 2>{});
    two_dims(std::integral_constant<int, 3>{});
}

// O^T += V^T.P^T for a pair of tiles.
__device__ __forceinline__ void add_values(Row& st, const bf16x8& p, const uint32_t (&wa)[4][4], const uint32_t (&wb)[4][4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const u32x4 even = {wa[j][0], wa[j][1], wb[j][0], wb[j][1]}, odd = {wa[j][2], wa[j][3], wb[j][2], wb[j][3]};
        st.o[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), p, st.o[2 * j], 0, 0, 0);
        st.o[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), p, st.o[2 * j + 1], 0, 0, 0);
    }
}

constexpr int kFoldFloats = 8 * 256 + 128;  // one wavefront's state: eight accumulator quads, reference and share of the sum per lane

template <bool SPLIT, bool INLINE>
__device__ __forceinline__ Slice unit_of_block(PlanDev& plan, int n_kv) {
    if constexpr (INLINE) plan_from_arguments(plan);
    Slice slice;
    if constexpr (SPLIT) {
        slice = slice_of_block(plan.split, 0, n_kv);
    } else {
        slice.wg = blockIdx.x / n_kv;
    }
    return slice;
}

// NT = 16-row tiles per wavefront; SPLIT: several workgroups per unit, each with a slice of its lists (attn_split.hpp).
// lds: the wavefronts' row states when a unit is divided among them
template <int NT, bool SPLIT>
__device__ __forceinline__ void attend_unit(float (&lds)[4][kFoldFloats], const Slice& slice, const char* __restrict__ pool,
                                            const uint16_t* __restrict__ q, const PlanDev& plan, int n_cand, int n_q, int n_kv, int group,
                                            float scale_log2e, const PartialBuf& part, const uint16_t* __restrict__ cand_k,
                                            const uint16_t* __restrict__ cand_v, const uint8_t* __restrict__ cand_mask,
                                            uint16_t* __restrict__ out) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int g4 = lane >> 4, c = lane & 15;
    const int kvh = blockIdx.x % n_kv;
    const WgDesc* wg = plan.wgs + slice.wg;
    WaveItem wi = wg->w[wave];
    if (wi.n_grp == 0) return;  // (a wave-split unit's wavefronts all have rows; nobody waits for this one)
    int coop_ofs = wg->coop_ofs, n_coop = wg->n_coop, n_full = 0;
    if constexpr (SPLIT) {
        cut_list(slice, coop_ofs, n_coop, n_full);
        cut_list(slice, wi.tile_ofs, wi.n_tiles, n_full);
    }
    const char* head_base = pool + (int64_t)kvh * kFp4TileBytes;
    const int64_t block_stride = (int64_t)n_kv * kFp4TileBytes;

    // Row geometry: column c of row tile nt is row `within` of the wavefront's row group nt * cap + c / rps.
    const int rps = plan.rows_per_slice, n_sl = plan.n_slices, rpt = plan.rows_per_thread;
    const int cap = 16 / rps;
    auto row_of = [&](int nt, int col, int& j, int& listed, int& cc, int64_t& qrow, int64_t& slot) -> bool {
        const int jc = col / rps, within = col - jc * rps;
        j = nt * cap + jc;
        const int grp = wi.grp_lo + j;
        const int rank = grp / n_sl, rr = (grp - rank * n_sl) * rps + within;
        if (jc >= cap || j >= wi.n_grp || rr >= rpt) return false;
        listed = plan.dfs_threads ? plan.dfs_threads[rank] : rank;
        cc = rr / group;
        const int hq = kvh * group + (rr - cc * group);
        qrow = ((int64_t)listed * n_cand + cc) * n_q + hq;
        slot = ((int64_t)(wi.part_base + rank - wi.grp_lo / n_sl) * n_cand + cc) * n_q + hq;
        return true;
    };
    Row st[NT];
    int my_j[NT];  // row group of this lane's row, relative to the wavefront's first; -1: no row
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        int j, listed, cc;
        int64_t qrow, slot;
        const bool ok = row_of(nt, c, j, listed, cc, qrow, slot);
        my_j[nt] = ok ? j : -1;
        st[nt].m = -INFINITY;
        st[nt].l = 0.0f;
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) st[nt].o[jj] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        load_query(st[nt], q + (ok ? qrow * 128 : 0), ok, g4, c);
    }
    // how many of a tile's tokens the row `ahead` row groups past its first one sees (causal tiles: one more per group)
    auto seen = [](int meta, int ahead) -> int {
        const int fill = (meta >> 20) & 31;
        return (meta >> 30) ? min(fill, max(0, ((meta >> 25) & 31) + ahead)) : fill;
    };
    const uint32_t k_ofs = c * 64 + g4 * 16, v_ofs = kFp4V + lane * 16;
    const uint32_t ks_ofs = kFp4KScale + c * 4 + g4, vs_ofs = kFp4VScale + g4 * 16 + (c & 12);
    auto fetch = [&](const TileRef& r) -> Tile {
        const char* tile = head_base + r.blk * block_stride;
        return Tile{*reinterpret_cast<const u32x4*>(tile + k_ofs), *reinterpret_cast<const u32x4*>(tile + v_ofs),
                    *reinterpret_cast<const uint8_t*>(tile + ks_ofs), *reinterpret_cast<const uint32_t*>(tile + vs_ofs)};
    };
    // Both lists, one after the other; `shift`: the shared list's ranges count row groups from the workgroup's first.
    for (int list = 0; list < 2; ++list) {
        const TileRef* tiles = plan.tiles + (list == 0 ? coop_ofs : wi.tile_ofs);
        const int n = list == 0 ? n_coop : wi.n_tiles;
        const int shift = list == 0 ? wi.grp_lo - wg->grp_base : 0;
        if (n == 0) continue;
        // Tiles of the shared list that no row of this wavefront sees are passed over; its own list has none.
        auto next = [&](int t) {
            for (; list == 0 && t < n; ++t) {
                const int meta = tiles[t].meta;
                if ((meta & 1023) - shift < wi.n_grp && ((meta >> 10) & 1023) - shift > 0) break;
            }
            return t;
        };
        struct Pair {
            TileRef a, b;
            bool any;
        };
        int t = 0;
        // the pair from t on; without a second tile the first one again, seen by nobody; past the end the last tile, not used
        auto next_pair = [&]() -> Pair {
            Pair p;
            t = next(t);
            p.any = t < n;
            p.a = tiles[min(t, n - 1)];
            t = next(t + 1);
            p.b = tiles[min(t, n - 1)];
            if (t >= n) p.b = TileRef{p.a.blk, 0};
            ++t;
            return p;
        };
        // does every row group of the wavefront see all of the tile?
        auto whole = [&](int meta) {
            return (meta & 1023) - shift <= 0 && ((meta >> 10) & 1023) - shift >= wi.n_grp && meta >> 20 == 16;
        };
        // The next pair is fetched as soon as V is widened; the words of the pair after that are on their way too.  (With two to four pairs
        // on their way, at two wavefronts per SIMD instead of three, calls were slower: 64 requests of group 8 38 -> 45 us, 16 long ones
        // 30 -> 33; with V widened between the products and four wavefronts per SIMD 38 -> 40, 30 -> 34.)
        Pair now = next_pair();
        if (!now.any) continue;
        Tile ta = fetch(now.a), tb = fetch(now.b);
        Pair coming = next_pair();
        while (true) {
            f32x4 sa[NT], sb[NT];
            uint32_t wa[4][4], wb[4][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sa[nt] = products(ta, st[nt]), sb[nt] = products(tb, st[nt]);
            widen(ta, wa);
            widen(tb, wb);
            ta = fetch(coming.a), tb = fetch(coming.b);
            const Pair after = next_pair();
            if (!(whole(now.a.meta) && whole(now.b.meta))) {  // (rows that are none take part in whole tiles: nobody writes them)
                const int alo = (now.a.meta & 1023) - shift, ahi = ((now.a.meta >> 10) & 1023) - shift;
                const int blo = (now.b.meta & 1023) - shift, bhi = ((now.b.meta >> 10) & 1023) - shift;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int mine_a = (my_j[nt] >= max(alo, 0) && my_j[nt] < ahi ? seen(now.a.meta, my_j[nt] - alo) : 0) - 4 * g4;
                    const int mine_b = (my_j[nt] >= max(blo, 0) && my_j[nt] < bhi ? seen(now.b.meta, my_j[nt] - blo) : 0) - 4 * g4;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sa[nt][i] = i < mine_a ? sa[nt][i] : -INFINITY;
                        sb[nt][i] = i < mine_b ? sb[nt][i] : -INFINITY;
                    }
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) add_values(st[nt], probabilities(st[nt], sa[nt], sb[nt], scale_log2e), wa, wb);
            if (!coming.any) break;
            now = coming;
            coming = after;
        }
    }

    // A multi-candidate call's candidates (bf16, a row every n_kv * 128 elements): tiles of as many threads' as fit sixteen slots, each
    // visible to the rows whose mask names it; the unit that writes the rows directly adds them.  (Thread by thread, their loads wait
    // for each other: 192 threads of one candidate 26 -> 22 us.)
    if ((wi.flags & kWaveDirect) && cand_mask != nullptr && (wave == 0 || !(wi.flags & kWaveSplit)) && slice.s == 0) {
        const int64_t tok_stride = (int64_t)n_kv * 128;
        const int rank_hi = (wi.grp_lo + wi.n_grp - 1) / n_sl, threads = 16 / n_cand;
        for (int ru = wi.grp_lo / n_sl; ru <= rank_hi; ru += threads) {
            // where slot x's row starts (past the last candidate: the first one's, seen by nobody)
            auto row_at = [&](int x) -> int64_t {
                const int u = x / n_cand, rank = ru + u;
                const bool real = u < threads && rank <= rank_hi;
                const int from = real ? rank : ru;
                const int listed_u = plan.dfs_threads ? plan.dfs_threads[from] : from;
                return ((int64_t)listed_u * n_cand + (real ? x - u * n_cand : 0)) * tok_stride + kvh * 128;
            };
            // K: dims 32 g .. + 31 of slot c; V: dims 8 c .. + 7 of slots 4 g + i
            u32x4 ck[4], cv[4];
            const uint16_t* k_row = cand_k + row_at(c) + 32 * g4;
            bool fine = true;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                ck[r] = *reinterpret_cast<const u32x4*>(k_row + 8 * r);
                cv[r] = *reinterpret_cast<const u32x4*>(cand_v + row_at(4 * g4 + r) + 8 * c);
            }
            uint32_t sees[NT];
            u32x4 x[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                int j, listed, cc;
                int64_t qrow, slot;
                const bool ok = row_of(nt, c, j, listed, cc, qrow, slot);
                const int u = ok ? (wi.grp_lo + j) / n_sl - ru : -1;
                const bool here = u >= 0 && u < threads;
                // (a row that is none: any one's mask and query; nobody looks at its products)
                const uint32_t tm = cand_mask[here ? (int64_t)listed * n_cand + cc : 0] & ((1u << n_cand) - 1u);
                sees[nt] = here ? tm << (u * n_cand) : 0u;
#pragma unroll
                for (int r = 0; r < 4; ++r) x[nt][r] = *reinterpret_cast<const u32x4*>(q + (here ? qrow * 128 : 0) + 32 * g4 + 8 * r);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) fine = fine && (cv[r][i] & 0x7f80u) != 0x7f80u && (cv[r][i] & 0x7f800000u) != 0x7f800000u;
            const bool all_fine = __builtin_amdgcn_ballot_w64(!fine) == 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (__builtin_amdgcn_ballot_w64(sees[nt] != 0) == 0) continue;
                f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ck[r]), __builtin_bit_cast(bf16x8, x[nt][r]), s, 0, 0, 0);
                const uint32_t mine = sees[nt] >> (4 * g4);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = ((mine >> i) & 1u) ? s[i] : -INFINITY;
                if (all_fine) {
                    const f32x4 none = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    const bf16x8 pb = probabilities(st[nt], s, none, scale_log2e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const u32x4 even = {low_halves(cv[0][j], cv[1][j]), low_halves(cv[2][j], cv[3][j]), 0u, 0u};
                        const u32x4 odd = {high_halves(cv[0][j], cv[1][j]), high_halves(cv[2][j], cv[3][j]), 0u, 0u};
                        st[nt].o[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pb, st[nt].o[2 * j], 0, 0, 0);
                        st[nt].o[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pb, st[nt].o[2 * j + 1], 0, 0, 0);
                    }
                    continue;
                }
                // one by one, each only into the rows that see it
                move_reference(st[nt], fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) * scale_log2e);
                for (int cp = 0; cp < 16; ++cp) {
                    const float logit = __shfl(cp & 2 ? (cp & 1 ? s[3] : s[2]) : (cp & 1 ? s[1] : s[0]), (cp >> 2) * 16 + c, 64);
                    if ((sees[nt] >> cp) & 1u) {  // (the four lanes of a row agree)
                        const float pr = logit == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(__builtin_fmaf(logit, scale_log2e, -st[nt].m));
                        if (g4 == 0) st[nt].l += pr;
                        const uint16_t* vr = cand_v + row_at(cp) + 32 * g4;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int jj = 0; jj < 8; ++jj) st[nt].o[jj][i] += pr * __uint_as_float((uint32_t)vr[8 * i + jj] << 16);
                    }
                }
            }
        }
    }

    // ---- results --------------------------------------------------------------------------------
    // Accumulators j0 .. j0 + J - 1 of the lane's row of row tile nt: the dims 8 (4 g + i) + jj.
    auto write = [&](auto count, int j0, int nt) {
        constexpr int J = decltype(count)::value;
        float lt = st[nt].l;
        lt += __shfl_xor(lt, 16, 64);
        lt += __shfl_xor(lt, 32, 64);
        int j, listed, cc;
        int64_t qrow, slot;
        if (!row_of(nt, c, j, listed, cc, qrow, slot)) return;
        if (wi.flags & kWaveDirect) {
            const float inv = 1.0f / lt;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t x[J / 2];
#pragma unroll
                for (int h = 0; h < J / 2; ++h) x[h] = pack_pair(st[nt].o[2 * h][i] * inv, st[nt].o[2 * h + 1][i] * inv);
                uint16_t* to = out + qrow * 128 + 32 * g4 + 8 * i + j0;
                if constexpr (J == 8) *reinterpret_cast<u32x4*>(to) = u32x4{x[0], x[1], x[2], x[3]};
                else *reinterpret_cast<uint32_t*>(to) = x[0];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float* to = part.o + slot * 128 + 32 * g4 + 8 * i + j0;
                if constexpr (J == 8) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        *reinterpret_cast<f32x4*>(to + 4 * h) =
                            f32x4{st[nt].o[4 * h][i], st[nt].o[4 * h + 1][i], st[nt].o[4 * h + 2][i], st[nt].o[4 * h + 3][i]};
                } else {
                    *reinterpret_cast<f32x2*>(to) = f32x2{st[nt].o[0][i], st[nt].o[1][i]};
                }
            }
            if (g4 == 0 && j0 == 0) {
                part.ml[slot * 2] = st[nt].m;
                part.ml[slot * 2 + 1] = lt;
            }
        }
    };
    if (NT == 1 && (wi.flags & kWaveSplit)) {
        // the four wavefronts hold the same rows over different tiles: every one folds two of the eight accumulators, of its
        // workgroup's wavefronts through LDS and then of the unit's slices.  (One wavefront folding all of the slices: one thread family of 32 k
        // tokens, 8 kv heads, 32 slices 27.6 us a call, this way 24.6.)
        float* to = lds[wave];
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) *reinterpret_cast<f32x4*>(to + (jj * 64 + lane) * 4) = st[0].o[jj];
        *reinterpret_cast<f32x2*>(to + 2048 + lane * 2) = f32x2{st[0].m, st[0].l};
        __syncthreads();
        const int j0 = 2 * wave;
        f32x2 ml[4];
        f32x4 o[4][2];
#pragma unroll
        for (int w2 = 0; w2 < 4; ++w2) {
            ml[w2] = *reinterpret_cast<const f32x2*>(&lds[w2][2048 + lane * 2]);
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) o[w2][jj] = *reinterpret_cast<const f32x4*>(&lds[w2][((j0 + jj) * 64 + lane) * 4]);
        }
        const float mx = fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0]));
        st[0].m = mx;
        st[0].l = 0.0f;
        st[0].o[0] = st[0].o[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w2 = 0; w2 < 4; ++w2) {
            // a wavefront that saw no tile of a row left m = -inf and sums of zero for it
            const float a = ml[w2][0] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml[w2][0] - mx);
            st[0].l += a * ml[w2][1];
            st[0].o[0] += a * o[w2][0];
            st[0].o[1] += a * o[w2][1];
        }
        if constexpr (SPLIT)
            if (!fold_slices<1, 2, 8>(plan.split, slice, n_kv, kvh, wave, 1, lane, reinterpret_cast<Row(&)[1]>(st), j0)) return;
        write(std::integral_constant<int, 2>{}, j0, 0);
        return;
    }
    if constexpr (SPLIT)
        if (!fold_slices<NT, 8>(plan.split, slice, n_kv, kvh, wave, 4, lane, st)) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) write(std::integral_constant<int, 8>{}, 0, nt);
}

// Units of one row tile per wavefront.
template <bool SPLIT, bool INLINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void attention_fp4_one(
    PlanWords<INLINE>, const char* __restrict__ pool, const uint16_t* __restrict__ q, PlanDev plan, int n_cand, int n_q, int n_kv, int group,
    float scale_log2e, PartialBuf part, const uint16_t* __restrict__ cand_k, const uint16_t* __restrict__ cand_v,
    const uint8_t* __restrict__ cand_mask, uint16_t* __restrict__ out) {
    __shared__ __attribute__((aligned(16))) float lds[4][kFoldFloats];
    const Slice slice = unit_of_block<SPLIT, INLINE>(plan, n_kv);
    tables_unwritten(plan);
    attend_unit<1, SPLIT>(lds, slice, pool, q, plan, n_cand, n_q, n_kv, group, scale_log2e, part, cand_k, cand_v, cand_mask, out);
}

// Units of either row-tile class, in one launch.  INLINE (with SPLIT): the plan's tables come with the kernel's arguments.
template <bool SPLIT, bool INLINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void attention_fp4(
    PlanWords<INLINE>, const char* __restrict__ pool, const uint16_t* __restrict__ q, PlanDev plan, int n_cand, int n_q, int n_kv, int group,
    float scale_log2e, PartialBuf part, const uint16_t* __restrict__ cand_k, const uint16_t* __restrict__ cand_v,
    const uint8_t* __restrict__ cand_mask, uint16_t* __restrict__ out) {
    __shared__ __attribute__((aligned(16))) float lds[4][kFoldFloats];
    const Slice slice = unit_of_block<SPLIT, INLINE>(plan, n_kv);
    tables_unwritten(plan);
    if ((plan.wgs[slice.wg].row_tiles & 255) == 2)
        attend_unit<2, SPLIT>(lds, slice, pool, q, plan, n_cand, n_q, n_kv, group, scale_log2e, part, cand_k, cand_v, cand_mask, out);
    else
        attend_unit<1, SPLIT>(lds, slice, pool, q, plan, n_cand, n_q, n_kv, group, scale_log2e, part, cand_k, cand_v, cand_mask, out);
}

}  // namespace

hipError_t launch_attention_fp4(const Shape& s, const void* pool, const void* q, const PlanDev& plan, int n_cand, PartialBuf part,
                                const void* cand_k, const void* cand_v, const uint8_t* mask, void* out, hipStream_t st) {
    if (plan.n_inline_words > kPlanInlineWords) return hipErrorInvalidValue;
    const bool split = plan.split.blocks != nullptr || plan.inline_words;
    const int32_t* n_class = split ? plan.split.n_blocks_class : plan.n_wg_class;
    const int64_t n = ((int64_t)n_class[1] + n_class[2]) * s.n_kv;
    if (n > 0x7fffffff || n_class[0] > 0) return hipErrorInvalidValue;  // (4-bit pools have no matrix units)
    if (n == 0) return hipSuccess;
#define APAR_LAUNCH_KERNEL(KERNEL, WORDS)                                                                               \
    hipLaunchKernelGGL(KERNEL, dim3((unsigned)n), dim3(256), 0, st, WORDS,                                              \
                       (const char*)pool, (const uint16_t*)q, plan, n_cand, s.n_q, s.n_kv, s.group, s.scale_log2e,      \
                       part, (const uint16_t*)cand_k, (const uint16_t*)cand_v, mask, (uint16_t*)out)
#define APAR_LAUNCH(SPLITV, INLINEV, WORDS)                                                            \
    do {                                                                                               \
        if (n_class[1] == 0) APAR_LAUNCH_KERNEL((attention_fp4_one<SPLITV, INLINEV>), WORDS);          \
        else APAR_LAUNCH_KERNEL((attention_fp4<SPLITV, INLINEV>), WORDS);                              \
    } while (0)
    if (plan.inline_words) {
        PlanWords<true> words;
        memcpy(words.words, plan.inline_words, (size_t)plan.n_inline_words * sizeof(int32_t));
        APAR_LAUNCH(true, true, words);
    } else if (split) {
        APAR_LAUNCH(true, false, PlanWords<false>{});
    } else {
        APAR_LAUNCH(false, false, PlanWords<false>{});
    }
#undef APAR_LAUNCH
#undef APAR_LAUNCH_KERNEL
    return hipGetLastError();
}

}  // namespace apar
