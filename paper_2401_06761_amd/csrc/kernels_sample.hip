// Sampling of tokens (gfx950): one workgroup per row of logits.
//
// A row's tokens stand in one order, value descending, index ascending.  With w = exp((x - max) / T) every cut is a prefix of it:
//   top-k: the first k;  top-p: the shortest prefix with mass >= p * (mass of the first k);  min-p: w >= min_p;
// and the token is the first one whose cumulated mass exceeds u * (mass of what is kept).  So a row never has to be sorted: each of these
// is the place where a cumulated count or mass reaches a target, found by digits of the values' ordered bit patterns (keys), 12, 12 and
// 8 bits: a histogram of counts and masses over the first digit, then over the next one of the values that share the first, and so
// on; among equal values the place follows from their weight, and the index from counting them.
// Masses are sums of whole numbers, w 2^weight_bits rounded (42 to 51 bits by the size of the vocabulary, w computed in 64): they
// do not depend on the order of the additions, and all prefixes agree with each other.
//
// bf16 rows (sample_rows_bf16): there are 65536 values, and a workgroup has room to count each of them (128 KiB of LDS, a word for the
// two values of a magnitude).  A weight is then worked out once per value and not once per token (tens of vector instructions in 64 bits): per run
// of 64 values that occur at all, by a wavefront each, to a count and a mass; and every target is reached by one wavefront, first among those
// runs, then among the 64 values of one.  The row stays in registers for the pass that looks for the token's index.  A value
// that occurs more than 65535 times shows in the counters' sum; such a row goes through the digits.  Both ways give the same token.
// What bounds it: memory, behind that the passes over the counters, which nothing fills where a compute unit has one row.
// (256 rows of 128000 in 23 to 25 us, 65 MB; one row of 32000 in 12 us, with all cuts 15, the largest token alone 8; of these 5 are a launch.)  Rows of more than 131072 tokens
// are read twice, with nothing on its way (64 rows of 200000 in 33 us).  Tokens of one value meet in one counter, 64 updates of a wavefront
// one after the other, the masked ones of a row among them: 256 rows of 128000, half of each -inf, 71 us; nine tenths, which go through the
// digits, 244, of the type's lowest value 382.
//
// fp32 rows (sample_rows_f32): every token has a weight of its own.  Its mass goes into one of 8192 bins of equal width between the largest value
// and the lightest that counts, a few tokens each where the row is dense; the tokens of the bin a target falls into become a list, and a
// token's place in it comes from comparing all with all.  That is a pass for the range, one for the masses and one per list, where digits
// take up to three per target and one for the index.  What bounds it: those passes' reads.  256 rows of 128000 with nothing cut are three passes,
// 393 MB, in 81 us, 4.6 TB/s (173 through the digits), with top-k, top-p and min-p in every row 427 MB in 110; the weights, some fifteen 64-bit
// instructions per token, keep the vector units busy for half of that time.  A row by itself is one compute unit's: 32000 in 23 to 30 us (52),
// 128000 in 57 to 73.
#include <hip/hip_runtime.h>

#include "apar_internal.hpp"
#include "sample.hpp"

namespace apar {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 4096;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

__device__ __forceinline__ uint32_t key_of(float x) {  // (-0 counts as 0)
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key ^ 0x80000000u : ~key); }

struct Found {
    uint32_t key;      // the value the target is reached on,
    uint32_t rank;     // and on which of the tokens that have it (by index, from 0)
    uint32_t above;    // tokens with larger values
    u64 mass_above;
};

struct Shared {
    u64 mass0[kBins], mass1[kBins];    // first digit's, and a later one's
    uint32_t count0[kBins], count1[kBins];
    u64 wave_mass[kWaves];
    uint32_t wave_count[kWaves];
    uint32_t hit_bin, hit_count;
    u64 hit_mass;
    u64 total_mass, minp_mass;
    uint32_t total_count, minp_count;
    uint32_t top;
    uint32_t chunk_count[kSampleMaxVocab / (4 * kThreads) + 2];
};

// Goes through a row, 16 bytes a lane; take(index, value) for every element of it, in no order.
template <class T, class Take>
__device__ __forceinline__ void each(const T* row, int vocab, Take take) {
    constexpr int W = 16 / sizeof(T);
    const int head = min(vocab, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));
    const int n = (vocab - head) / W;
    auto value = [](T x) -> float {
        if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)x << 16);
        else return x;
    };
    for (int i = threadIdx.x; i < n; i += kThreads) {
        union {
            u32x4 u;
            T x[W];
        } v;
        v.u = *reinterpret_cast<const u32x4*>(row + head + i * W);
#pragma unroll
        for (int j = 0; j < W; ++j) take(head + i * W + j, value(v.x[j]));
    }
    if ((int)threadIdx.x < head) take((int)threadIdx.x, value(row[threadIdx.x]));
    const int tail = head + n * W + (int)threadIdx.x;
    if (tail < vocab) take(tail, value(row[tail]));
}

// Inclusive sum over the wavefront's lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 from_lane(u64 x) {
    return (u64)from_lane<CTRL, ROWS>((uint32_t)x) | (u64)from_lane<CTRL, ROWS>((uint32_t)(x >> 32)) << 32;
}
template <class N>
__device__ __forceinline__ N prefix_sum(N x) {
    x += from_lane<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8: within sixteen lanes
    x += from_lane<0x112, 0xf>(x);
    x += from_lane<0x114, 0xf>(x);
    x += from_lane<0x118, 0xf>(x);
    x += from_lane<0x142, 0xa>(x);  // lane 15 of a row to the next one, lane 31 to the upper half
    x += from_lane<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ uint32_t at_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ u64 at_lane(u64 x, int lane) {
    return (u64)at_lane((uint32_t)x, lane) | (u64)at_lane((uint32_t)(x >> 32), lane) << 32;
}

// Inclusive sums over the threads of the workgroup, in their order.
template <class S>
__device__ __forceinline__ void scan(S& s, uint32_t& count, u64& mass) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    count = prefix_sum(count);
    mass = prefix_sum(mass);
    if (lane == 63) s.wave_count[wave] = count, s.wave_mass[wave] = mass;
    __syncthreads();
    for (int w = 0; w < wave; ++w) count += s.wave_count[w], mass += s.wave_mass[w];
    __syncthreads();
}

// The bin, from the largest down, in which the cumulated count or mass (of what lies above the bins, `above`, and the bins) reaches
// the target; what lies above that bin.
template <class S>
__device__ __forceinline__ int reach(S& s, const uint32_t* counts, const u64* masses, int bins, bool by_mass, u64 target,
                                     uint32_t& above, u64& mass_above) {
    const int per = (bins + kThreads - 1) / kThreads;
    uint32_t c = 0;
    u64 m = 0;
    const int first = bins - 1 - (int)threadIdx.x * per;  // this thread's bins: first, first - 1, ...
    for (int j = 0; j < per; ++j)
        if (first - j >= 0) c += counts[first - j], m += masses[first - j];
    uint32_t ci = c;
    u64 mi = m;
    scan(s, ci, mi);
    uint32_t cb = above + ci - c;
    u64 mb = mass_above + mi - m;
    const u64 before = by_mass ? mb : cb, behind = by_mass ? mb + m : cb + c;
    if (before < target && target <= behind) {
        for (int j = 0; j < per && first - j >= 0; ++j) {
            const uint32_t cj = counts[first - j];
            const u64 mj = masses[first - j];
            if ((by_mass ? mb + mj : (u64)(cb + cj)) >= target) {
                s.hit_bin = first - j, s.hit_count = cb, s.hit_mass = mb;
                break;
            }
            cb += cj, mb += mj;
        }
    }
    __syncthreads();
    above = s.hit_count;
    mass_above = s.hit_mass;
    const int bin = s.hit_bin;
    __syncthreads();
    return bin;
}

// A token's number as the caller wants it.
__device__ __forceinline__ void write_token(const SampleCall& call, int r, int index) {
    call.tokens[r] = index == call.ids.fork ? APAR_TOKEN_FORK : index == call.ids.child ? APAR_TOKEN_CHILD
                     : index == call.ids.eos ? APAR_TOKEN_EOS : index;
}
__device__ __forceinline__ void write_none(const SampleCall& call, int r) {
    call.tokens[r] = APAR_TOKEN_NONE;
    if (call.logprobs) call.logprobs[r] = -INFINITY;
}

// 2^t for t <= 0 in 64 bits: the series of exp(y) up to y^12 for the fraction, |y| <= ln 2 / 2, where y^13 / 13! is 1.7e-16.  (Half the
// instructions of the library's exp, whose range and special values nobody needs here.)
__device__ __forceinline__ double exp2_below_one(double t) {
    if (!(t > -1000.0)) return 0.0;
    const double n = __builtin_rint(t), y = (t - n) * 0.69314718055994530942;
    double p = 1.0 / 479001600.0;
    p = __builtin_fma(p, y, 1.0 / 39916800.0);
    p = __builtin_fma(p, y, 1.0 / 3628800.0);
    p = __builtin_fma(p, y, 1.0 / 362880.0);
    p = __builtin_fma(p, y, 1.0 / 40320.0);
    p = __builtin_fma(p, y, 1.0 / 5040.0);
    p = __builtin_fma(p, y, 1.0 / 720.0);
    p = __builtin_fma(p, y, 1.0 / 120.0);
    p = __builtin_fma(p, y, 1.0 / 24.0);
    p = __builtin_fma(p, y, 1.0 / 6.0);
    p = __builtin_fma(p, y, 0.5);
    p = __builtin_fma(p, y, 1.0);
    p = __builtin_fma(p, y, 1.0);
    return __builtin_ldexp(p, (int)n);
}

// w in whole units, to nearest even: a unit is at least 2^-51, and a sum with 2^52 has the number in its last 52 bits.
__device__ __forceinline__ u64 whole_units(double w, double one) {
    return (u64)__double_as_longlong(__builtin_fma(w, one, 4503599627370496.0)) & 0xfffffffffffffull;
}

// A row's weights: w = exp((x - max) / T), and in whole units.  `scale`: log2(e) / T.
struct Weights {
    double top, scale, one;
    __device__ __forceinline__ Weights(float t, float temperature, double unit)
        : top(t), scale(1.4426950408889634074 / (double)temperature), one(unit) {}
    __device__ __forceinline__ double of(float x) const { return (double)x == top ? 1.0 : exp2_below_one(((double)x - top) * scale); }
    __device__ __forceinline__ u64 whole(double w) const { return whole_units(w, one); }
    __device__ __forceinline__ u64 units(float x) const { return whole(of(x)); }
    __device__ __forceinline__ float logprob(float x, u64 mass) const {
        const double z = (double)x == top ? 0.0 : ((double)x - top) * scale * 0.69314718055994530942;
        return (float)(z - log((double)mass / one));
    }
};
__device__ __forceinline__ double unit_of(const SampleCall& call) { return (double)(1ull << call.weight_bits); }

// Targets that the cuts and the draw set.
__device__ __forceinline__ u64 top_p_target(float top_p, u64 mass) {
    return max((u64)1, min((u64)ceil((double)fmaxf(top_p, 0.0f) * (double)mass), mass));
}
__device__ __forceinline__ u64 draw_target(float u, u64 mass) {  // the first prefix of more than u times the mass
    return min((u64)((double)fminf(fmaxf(u, 0.0f), 1.0f) * (double)mass) + 1, mass);
}

// By digits, any type and size.
template <class T>
__device__ void sample_by_digits(Shared& s, const SampleCall& call, int r) {
    const int vocab = call.vocab;
    const T* row = (const T*)call.logits + (int64_t)r * call.row_stride;
    const apar_sample_row p = call.rows ? call.rows[r] : apar_sample_row{1.0f, 0, 1.0f, 0.0f};
    const bool greedy = !(p.temperature > 0.0f);

    for (int i = threadIdx.x; i < kBins; i += kThreads) s.count0[i] = 0, s.mass0[i] = 0;
    if (threadIdx.x == 0) s.top = 0, s.total_count = s.minp_count = 0, s.total_mass = s.minp_mass = 0;
    __syncthreads();
    uint32_t top = 0;  // (no value's key)
    each<T>(row, vocab, [&](int, float x) {
        if (x > -INFINITY) top = max(top, key_of(x));
    });
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if ((threadIdx.x & 63) == 0) atomicMax(&s.top, top);
    __syncthreads();
    top = s.top;
    if (top == 0) {  // nothing but -inf and NaN
        if (threadIdx.x == 0) write_none(call, r);
        return;
    }
    const Weights weights(value_of(top), p.temperature, unit_of(call));

    Found token{top, 0, 0, 0};
    u64 kept_mass = 0;
    if (!greedy) {
        const double least = p.min_p > 0.0f ? fmin((double)p.min_p, 1.0) : 0.0;
        uint32_t n = 0, n_min = 0;
        u64 m = 0, m_min = 0;
        each<T>(row, vocab, [&](int, float x) {
            if (!(x > -INFINITY)) return;
            const uint32_t key = key_of(x);
            const double wd = weights.of(x);
            const u64 w = weights.whole(wd);
            atomicAdd(&s.count0[key >> 20], 1u);
            atomicAdd(&s.mass0[key >> 20], w);
            n += 1, m += w;
            if (!(wd < least)) n_min += 1, m_min += w;
        });
        atomicAdd(&s.total_count, n);
        atomicAdd(&s.total_mass, m);
        atomicAdd(&s.minp_count, n_min);
        atomicAdd(&s.minp_mass, m_min);
        __syncthreads();

        auto find = [&](bool by_mass, u64 target) -> Found {
            Found f{0, 0, 0, 0};
            const uint32_t d0 = reach(s, s.count0, s.mass0, kBins, by_mass, target, f.above, f.mass_above);
            f.key = d0 << 20;
            // bf16 values: the digits below the sixteenth bit say nothing
            for (int digit = 1; digit < (sizeof(T) == 2 ? 2 : 3); ++digit) {
                const int shift = digit == 1 ? 8 : 0, bins = digit == 1 ? kBins : 256;
                const uint32_t prefix = f.key >> (shift + (digit == 1 ? 12 : 8));
                for (int i = threadIdx.x; i < bins; i += kThreads) s.count1[i] = 0, s.mass1[i] = 0;
                __syncthreads();
                each<T>(row, vocab, [&](int, float x) {
                    const uint32_t key = key_of(x);
                    if (!(x > -INFINITY) || key >> (shift + (digit == 1 ? 12 : 8)) != prefix) return;
                    atomicAdd(&s.count1[(key >> shift) & (bins - 1)], 1u);
                    atomicAdd(&s.mass1[(key >> shift) & (bins - 1)], weights.units(x));
                });
                __syncthreads();
                f.key |= (uint32_t)reach(s, s.count1, s.mass1, bins, by_mass, target, f.above, f.mass_above) << shift;
            }
            if (sizeof(T) == 2) f.key = f.key >> 31 ? f.key & 0xffff0000u : f.key | 0xffffu;
            const u64 left = target - (by_mass ? f.mass_above : f.above);  // of the tokens with this value, from 1
            const u64 w = weights.units(value_of(f.key));
            f.rank = (uint32_t)(by_mass ? (left + w - 1) / w - 1 : left - 1);
            return f;
        };
        auto mass_to = [&](const Found& f) -> u64 { return f.mass_above + (f.rank + 1) * weights.units(value_of(f.key)); };

        uint32_t kept = s.total_count;
        kept_mass = s.total_mass;
        const uint32_t min_count = s.minp_count;
        const u64 min_mass = s.minp_mass;
        if (p.top_k > 0 && (uint32_t)p.top_k < kept) {
            const Found f = find(false, (u64)p.top_k);
            kept = (uint32_t)p.top_k;
            kept_mass = mass_to(f);
        }
        if (p.top_p < 1.0f) {
            const Found f = find(true, top_p_target(p.top_p, kept_mass));
            kept = min(kept, f.above + f.rank + 1);
            kept_mass = mass_to(f);
        }
        if (min_count < kept) kept_mass = min_mass;
        token = find(true, draw_target(call.uniforms[r], kept_mass));
    }

    // Which of the tokens with that value: the rank-th by index.  Counted by chunks of the row, then inside the one it lies in.
    constexpr int W = 16 / sizeof(T), kChunk = kThreads * W;
    const int chunks = (vocab + kChunk - 1) / kChunk;
    for (int i = threadIdx.x; i < chunks; i += kThreads) s.chunk_count[i] = 0;
    __syncthreads();
    each<T>(row, vocab, [&](int i, float x) {
        if (x > -INFINITY && key_of(x) == token.key) atomicAdd(&s.chunk_count[i / kChunk], 1u);
    });
    __syncthreads();
    uint32_t rank = token.rank;
    int chunk = 0;
    while (chunk + 1 < chunks && s.chunk_count[chunk] <= rank) rank -= s.chunk_count[chunk++];
    uint32_t mine = 0, bits = 0;
    const int first = chunk * kChunk + (int)threadIdx.x * W;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        if (first + j >= vocab) continue;
        float x;
        if constexpr (sizeof(T) == 2) x = __uint_as_float((uint32_t)row[first + j] << 16);
        else x = row[first + j];
        if (x > -INFINITY && key_of(x) == token.key) bits |= 1u << j, mine += 1;
    }
    uint32_t upto = mine;
    u64 none = 0;
    scan(s, upto, none);
    if (upto - mine <= rank && rank < upto) {
        uint32_t skip = rank - (upto - mine);
        while (skip-- > 0) bits &= bits - 1;
        write_token(call, r, first + __builtin_ctz(bits));
        if (call.logprobs) call.logprobs[r] = greedy ? 0.0f : weights.logprob(value_of(token.key), kept_mass);
    }
}

// ---- f32 rows: bins of equal width, and a list ------------------------------------------------------
constexpr int kFine = 8192, kList = 1024;

// The weights of a row whose values are all finite, w = 2^n 2^(k/64) 2^y with |y| <= 1/128: the middle factor from a table, the last one from the
// series of exp(y ln 2) up to y^5 (the next term is 4e-17).  A third of the 64-bit instructions of a weight without a table, and a row has one per token.
struct TableWeights {
    double top, scale, one;
    const double* table;  // 2^(k/64)
    __device__ __forceinline__ TableWeights(float t, float temperature, double unit, const double* powers)
        : top(t), scale(fmin(1.4426950408889634074 / (double)temperature, 1e300)), one(unit), table(powers) {}
    __device__ __forceinline__ double of(float x) const {
        constexpr double kRound = 105553116266496.0;  // 1.5 2^46: a sum with it is a multiple of 1/64
        const double t = fmax(((double)x - top) * scale, -1000.0);
        const double q = t + kRound, y = t - (q - kRound);
        const int k = (int)(uint32_t)__double_as_longlong(q);  // t in sixty-fourths
        double p = 1.3333558146428443423e-3;  // ln(2)^5 / 5!, ...
        p = __builtin_fma(p, y, 9.6181291076284771619e-3);
        p = __builtin_fma(p, y, 5.5504108664821579953e-2);
        p = __builtin_fma(p, y, 2.4022650695910071233e-1);
        p = __builtin_fma(p, y, 6.9314718055994530942e-1);
        p = __builtin_fma(p, y, 1.0);
        p *= table[k & 63];
        return __longlong_as_double(__double_as_longlong(p) + ((long long)(k >> 6) << 52));
    }
    __device__ __forceinline__ u64 whole(double w) const { return whole_units(w, one); }
    __device__ __forceinline__ u64 units(float x) const { return whole(of(x)); }
    __device__ __forceinline__ float logprob(float x, u64 mass) const {
        return (float)(((double)x - top) * scale * 0.69314718055994530942 - log((double)mass / one));
    }
};

struct Item {
    u64 order;  // key and, the other way round, index: one token's is larger than another's that stands behind it
    u64 units;
};
struct Binned {
    u64 mass[kFine];
    uint32_t count[kFine];       // (with top-k)
    Item list[kList];
    u64 list_mass[kList];        // up to and with an item
    uint32_t list_count[kList];
    double powers[64];
    u64 wave_mass[kWaves], wave_all[kWaves], wave_least[kWaves];
    float wave_top[kWaves], wave_low[kWaves];
    uint32_t wave_count[kWaves], wave_tokens[kWaves];
    uint32_t hit_bin, hit_count;
    u64 hit_mass, hit_order;
    uint32_t listed;
};
union RoomsF32 {
    Shared digits;
    Binned binned;
};
static_assert(sizeof(RoomsF32) <= 160 * 1024, "LDS of a compute unit");

__global__ __launch_bounds__(kThreads) void sample_rows_f32(SampleCall call) {
    __shared__ RoomsF32 rooms;
    Binned& s = rooms.binned;
    const int r = blockIdx.x, vocab = call.vocab;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const float* row = (const float*)call.logits + (int64_t)r * call.row_stride;
    const int head = min(vocab, (int)((16 - ((uintptr_t)row & 15)) & 15) / 4);
    const int n_body = (vocab - head) / 4, tail = head + n_body * 4;
    const u32x4* body = reinterpret_cast<const u32x4*>(row + head);
    const int edge = (int)threadIdx.x < head ? (int)threadIdx.x : tail + (int)threadIdx.x - 512;  // a head or (threads from 512 on) a tail element
    const bool has_edge = (int)threadIdx.x < head || ((int)threadIdx.x >= 512 && edge < vocab);
    const float edge_value = has_edge ? row[edge] : -INFINITY;
    const apar_sample_row p = call.rows ? call.rows[r] : apar_sample_row{1.0f, 0, 1.0f, 0.0f};
    const float u = call.uniforms[r];
    // take(index, value) for every element of the row, in no order.  Two pieces of 16 bytes a thread are looked at while the next two are on their
    // way (past the row's end the last one again, not looked at).  With four a call takes 1 to 3 % longer, with six 10 to 30 %.
    constexpr int kPieces = 2;
    auto elements = [&](auto take) __attribute__((always_inline)) {
        u32x4 x[kPieces];
        auto fetch = [&](int at0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) x[i] = body[min(at0 + i * kThreads, n_body - 1)];
        };
        if ((int)threadIdx.x < n_body) fetch(threadIdx.x);
        for (int at0 = threadIdx.x; at0 < n_body; at0 += kPieces * kThreads) {
            u32x4 now[kPieces];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) now[i] = x[i];
            fetch(at0 + kPieces * kThreads);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int at = at0 + i * kThreads;
                if (at >= n_body) break;
                const uint32_t word[4] = {now[i][0], now[i][1], now[i][2], now[i][3]};
#pragma unroll
                for (int j = 0; j < 4; ++j) take(head + at * 4 + j, __uint_as_float(word[j]));
            }
        }
        if (has_edge) take(edge, edge_value);
    };
    auto order_of = [](int i, float x) -> u64 { return (u64)key_of(x) << 32 | (uint32_t)~i; };

    if (!(p.temperature > 0.0f)) {  // the first token
        u64 best = 0;  // (no token's)
        elements([&](int i, float x) __attribute__((always_inline)) {
            if (x > -INFINITY) best = max(best, order_of(i, x));
        });
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) best = max(best, (u64)__shfl_xor((long long)best, o, 64));
        if (lane == 0) s.wave_all[wave] = best;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) best = max(best, s.wave_all[w]);
        if (threadIdx.x != 0) return;
        if (best == 0) return write_none(call, r);
        write_token(call, r, (int)~(uint32_t)best);
        if (call.logprobs) call.logprobs[r] = 0.0f;
        return;
    }

    // ---- the largest and the smallest value
#pragma unroll
    for (int i = 0; i < kFine / kThreads; ++i) s.mass[i * kThreads + threadIdx.x] = 0, s.count[i * kThreads + threadIdx.x] = 0;
    if (threadIdx.x < 64) s.powers[threadIdx.x] = 2.0 * exp2_below_one((double)threadIdx.x / 64.0 - 1.0);
    float top = -INFINITY, low = INFINITY;
    elements([&](int, float x) __attribute__((always_inline)) { top = fmaxf(top, x), low = fminf(low, x); });  // (of a number and a NaN: the number)
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64)), low = fminf(low, __shfl_xor(low, o, 64));
    if (lane == 0) s.wave_top[wave] = top, s.wave_low[wave] = low;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s.wave_top[w]), low = fminf(low, s.wave_low[w]);
    if (top == -INFINITY) {  // nothing but -inf and NaN
        if (threadIdx.x == 0) write_none(call, r);
        return;
    }
    const TableWeights weights(top, p.temperature, unit_of(call), s.powers);
    // A bin is a width of values below the largest one, places from 0 on; the subtraction, the product and their roundings keep the order.  What is
    // lighter than half a unit weighs nothing, and the places need not reach that far: it stands in the last one.  (kFine - 1 - place: the largest
    // values in the last bin.)
    const double span = fmin((double)top - (double)low, (double)(call.weight_bits + 2) * 0.69314718055994530942 * (double)p.temperature);
    const float per = span > 0.0 ? fminf((float)((kFine - 1) / span), 3.4028234e38f) : 0.0f;
    auto place_of = [&](float x) -> float { return fminf((top - x) * per, (float)(kFine - 1)); };
    const bool counted = p.top_k > 0, cut_by_weight = p.min_p > 0.0f;

    bool crowded = top == INFINITY;  // or more tokens in a bin than the list holds: such a row goes through the digits
    if (!crowded) {
        // ---- every bin's mass
        const double least = fmin((double)p.min_p, 1.0);
        u64 mass = 0, mass_least = 0;
        uint32_t n = 0;
        elements([&](int, float x) __attribute__((always_inline)) {
            if (!(x > -INFINITY)) return;
            const double wd = weights.of(x);
            const u64 w = weights.whole(wd);
            const int b = kFine - 1 - (int)place_of(x);
            if (w) atomicAdd(&s.mass[b], w);
            if (counted) atomicAdd(&s.count[b], 1u), n += 1;
            mass += w;
            if (cut_by_weight) mass_least += wd < least ? 0 : w;
        });
        mass = prefix_sum(mass);
        mass_least = prefix_sum(mass_least);
        n = prefix_sum(n);
        if (lane == 63) s.wave_all[wave] = mass, s.wave_least[wave] = mass_least, s.wave_tokens[wave] = n;
        __syncthreads();
        u64 kept_mass = 0, min_mass = 0;
        uint32_t kept = 0;
        for (int w = 0; w < kWaves; ++w) kept_mass += s.wave_all[w], min_mass += s.wave_least[w], kept += s.wave_tokens[w];

        // The token on which the cumulated count or mass reaches a target: its bin; the bin's tokens as a list, with what lies above each of them
        // (all against all); and the one of them.  With a small top-k the list begins at the first token: the cuts behind that one and the
        // draw find their tokens in it.  (Lists of up to 1024 tokens from the first
        // one: top-k of up to 1000 in 16 rows of 128000 takes 11 us longer.)
        int listed_from = kFine, listed_to = -1;
        struct Hit {
            u64 order, mass;  // the token, the mass up to and with it
        };
        auto find = [&](bool by_mass, u64 target) __attribute__((always_inline)) -> Hit {
            uint32_t above = 0;
            u64 mass_above = 0;
            const int b = reach(s, s.count, s.mass, kFine, by_mass, target, above, mass_above);
            if (!by_mass && s.mass[b] == 0) return Hit{0, mass_above};
            if (b < listed_from || b > listed_to) {
                const bool from_first = counted && above + s.count[b] <= kList / 4;
                listed_from = b;
                listed_to = from_first ? kFine - 1 : b;
                if (from_first) above = 0, mass_above = 0;
                if (threadIdx.x == 0) s.listed = 0;
                s.list_mass[threadIdx.x] = mass_above;
                s.list_count[threadIdx.x] = above;
                __syncthreads();
                const float first = (float)(kFine - 1 - listed_to), end = (float)(kFine - listed_from);
                elements([&](int i, float x) __attribute__((always_inline)) {
                    const float at = place_of(x);
                    if (!(at >= first && at < end)) return;
                    if (!(x > -INFINITY)) return;
                    const uint32_t slot = atomicAdd(&s.listed, 1u);
                    if (slot < kList) s.list[slot].order = order_of(i, x);
                });
                __syncthreads();
                const int m = (int)s.listed;
                if (m > kList) {
                    crowded = true;
                    return Hit{0, 0};
                }
                if ((int)threadIdx.x < m) s.list[threadIdx.x].units = weights.units(value_of((uint32_t)(s.list[threadIdx.x].order >> 32)));
                __syncthreads();
                const int parts = kThreads / m, i = (int)threadIdx.x % m, part = (int)threadIdx.x / m;  // (a token's others in parts)
                if (part < parts) {
                    const int per_part = (m + parts - 1) / parts, stop = min((part + 1) * per_part, m);
                    const u64 order = s.list[i].order;
                    u64 sum = 0;
                    uint32_t tokens = 0;
#pragma unroll 4
                    for (int j = part * per_part; j < stop; ++j) {
                        const Item other = s.list[j];
                        if (other.order >= order) sum += other.units, tokens += 1;
                    }
                    atomicAdd(&s.list_mass[i], sum);
                    atomicAdd(&s.list_count[i], tokens);
                }
                __syncthreads();
            }
            const int t = (int)threadIdx.x;
            if (t < (int)s.listed) {
                const u64 units = s.list[t].units, to = by_mass ? s.list_mass[t] : s.list_count[t], before = to - (by_mass ? units : 1);
                if (before < target && target <= to) s.hit_order = s.list[t].order, s.hit_mass = s.list_mass[t];
            }
            __syncthreads();
            return Hit{s.hit_order, s.hit_mass};
        };
        if (counted && (uint32_t)p.top_k < kept) kept_mass = find(false, (u64)p.top_k).mass;
        if (!crowded && p.top_p < 1.0f) kept_mass = find(true, top_p_target(p.top_p, kept_mass)).mass;
        if (!crowded) {
            if (cut_by_weight) kept_mass = min(kept_mass, min_mass);  // (of two prefixes the shorter one)
            const Hit token = find(true, draw_target(u, kept_mass));
            if (!crowded && threadIdx.x == 0) {
                write_token(call, r, (int)~(uint32_t)token.order);
                if (call.logprobs) call.logprobs[r] = weights.logprob(value_of((uint32_t)(token.order >> 32)), kept_mass);
            }
        }
    }
    if (crowded) {
        __syncthreads();
        sample_by_digits<float>(rooms.digits, call, r);
    }
}

// ---- bf16 rows: a counter per value ---------------------------------------------------------------
constexpr int kRuns = 1024;  // runs of 64 bit patterns: 0 .. 510 positive values, 512 .. 1021 negative ones, the others no numbers

struct Counted {
    uint32_t counts[32768];        // per magnitude (bit pattern without the sign): positive values in the low half, negative ones in the high
    u64 present[128];              // bytes; byte 64 w + 16 k + j, bit i: sixteenth j of run 32 w + 4 i + k has a counter that is not 0 ...
    u64 present_below[128];        // ... and of the same run of negative values
    uint16_t run[kRuns];           // the runs that occur, in order of value
    uint32_t run_count[kRuns];     // their tokens, then the tokens up to and with them,
    u64 run_mass[kRuns];           // and masses
    uint32_t wave_sum[kWaves];
    uint32_t chunk_count[kSampleMaxVocab / (8 * kThreads) + 3];
    uint32_t n_runs, tokens;
    uint32_t pattern, rank;        // the token's value, and which of those with it
    u64 kept_mass;
};
union Rooms {
    Shared digits;
    Counted counted;
};
static_assert(sizeof(Rooms) <= 160 * 1024, "LDS of a compute unit");

__device__ __forceinline__ float bf16_value(uint32_t pattern) { return __uint_as_float(pattern << 16); }
// The bit pattern of place l in a run: values fall from the largest on.
__device__ __forceinline__ uint32_t pattern_of(int run, int l) { return (uint32_t)(run * 64 + (run < 512 ? 63 - l : l)); }

// NV: 16-byte pieces of a row per thread, kept in registers (0: rows of any size, read again).
template <int NV>
__global__ __launch_bounds__(kThreads) void sample_rows_bf16(SampleCall call) {
    __shared__ Rooms rooms;
    Counted& s = rooms.counted;
    const int r = blockIdx.x, vocab = call.vocab;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint16_t* row = (const uint16_t*)call.logits + (int64_t)r * call.row_stride;
    const int head = min(vocab, (int)((16 - ((uintptr_t)row & 15)) & 15) / 2);
    const int n_body = (vocab - head) / 8, tail = head + n_body * 8;
    const u32x4* body = reinterpret_cast<const u32x4*>(row + head);
    // Pieces on their way: a few at a time, others behind those that are counted (all at once, the wavefronts stand at their own loads
    // for as long as the row takes, and nobody counts).
    constexpr int kAhead = NV < 4 ? NV : 4;
    u32x4 v[NV > 0 ? NV : 1];
    auto fetch = [&](int i) {  // (past the row's end the last piece again, not looked at: no branch around a load)
        v[i] = __builtin_nontemporal_load(body + min(i * kThreads + (int)threadIdx.x, n_body - 1));
    };
    if (NV > 0 && n_body > 0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(i);
    }
    const int edge = (int)threadIdx.x < head ? (int)threadIdx.x : tail + (int)threadIdx.x - 512;  // a head or (threads from 512 on) a tail element
    const bool has_edge = (int)threadIdx.x < head || ((int)threadIdx.x >= 512 && edge < vocab);
    uint32_t edge_pattern = 0xffffu;
    if (has_edge) edge_pattern = row[edge];
    const apar_sample_row p = call.rows ? call.rows[r] : apar_sample_row{1.0f, 0, 1.0f, 0.0f};
    const float u = call.uniforms[r];
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(&s.counts[(i * kThreads + threadIdx.x) * 4]) = u32x4{0u, 0u, 0u, 0u};
    const int chunks = NV > 0 ? NV : (n_body + kThreads - 1) / kThreads;
    for (int i = threadIdx.x; i < chunks + 2; i += kThreads) s.chunk_count[i] = 0;
    // (a barrier for LDS alone: the row is still on its way, and its first pieces are counted while the others come)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");

    // ---- how often each value occurs
    auto count = [&](uint32_t pattern) { atomicAdd(&s.counts[pattern & 0x7fffu], 1u + (pattern >> 15) * 0xffffu); };
    auto count_piece = [&](const u32x4& x) {
#pragma unroll
        for (int j = 0; j < 4; ++j) count(x[j] & 0xffffu), count(x[j] >> 16);
    };
    if constexpr (NV > 0) {
        if (n_body > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i + kAhead < NV) fetch(i + kAhead);
                asm volatile("" ::: "memory");
                if (i * kThreads + (int)threadIdx.x < n_body) count_piece(v[i]);
                asm volatile("" ::: "memory");
            }
        }
    } else {
        for (int at = threadIdx.x; at < n_body; at += kThreads) count_piece(body[at]);
    }
    if (has_edge) count(edge_pattern);
    __syncthreads();
    // zeros of both signs are one value
    bool crowded = false;  // (a counter too small)
    if (threadIdx.x == 0) {
        const uint32_t z = (s.counts[0] & 0xffffu) + (s.counts[0] >> 16);
        s.tokens = z >> 16;
        s.counts[0] = z & 0xffffu;
    }
    __syncthreads();
    // ---- runs that occur (a wavefront looks at 32 of either sign), their order, and whether any counter overflowed
    uint32_t all = 0, up = 0, down = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // (a run is sixteen lanes' pieces)
        const u32x4 x = *reinterpret_cast<const u32x4*>(&s.counts[((wave * 8 + i) * 64 + lane) * 4]);
        const uint32_t any = x[0] | x[1] | x[2] | x[3];
        up |= (any & 0xffffu) != 0 ? 1u << i : 0u;
        down |= any >> 16 != 0 ? 1u << i : 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) all = __builtin_amdgcn_sad_u16(x[j], 0u, all);  // (both half words)
    }
    reinterpret_cast<uint8_t*>(s.present)[wave * 64 + lane] = (uint8_t)up;
    reinterpret_cast<uint8_t*>(s.present_below)[wave * 64 + lane] = (uint8_t)down;
    if (vocab > 65535) {
        all = prefix_sum(all);
        if (lane == 63) s.wave_sum[wave] = all;
        __syncthreads();
        all = 0;
        for (int w = 0; w < kWaves; ++w) all += s.wave_sum[w];
        crowded = s.tokens != 0 || all != (uint32_t)vocab;
    }
    __syncthreads();
    if (crowded) {  // (every counter's sum is one less, at least, per 65536 tokens that a half word lost)
        sample_by_digits<uint16_t>(rooms.digits, call, r);
        return;
    }
    {
        const int t = threadIdx.x;
        const int run = t <= 510 ? 510 - t : t + 1;  // 510 .. 0, then 512 .. 1021
        const u64* flags = run < 512 ? s.present : s.present_below;
        const int at = ((run & 511) >> 5) * 8 + (run & 3) * 2;
        bool here = t < 1021 && (((flags[at] | flags[at + 1]) >> ((run >> 2) & 7)) & 0x0101010101010101ull) != 0;
        if (run == 510) here = here && (s.counts[0x7f80] & 0xffffu) != 0;  // +inf; the rest of that run are NaN
        const u64 which = __builtin_amdgcn_ballot_w64(here);
        if (lane == 0) s.wave_sum[wave] = __builtin_popcountll(which);
        __syncthreads();
        uint32_t before = 0, total = 0;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += s.wave_sum[w];
            total += s.wave_sum[w];
        }
        if (here) s.run[before + __builtin_popcountll(which & ((1ull << lane) - 1))] = (uint16_t)run;
        if (t == 0) s.n_runs = total;
    }
    __syncthreads();
    const int n_runs = s.n_runs;
    if (n_runs == 0) {  // nothing but -inf and NaN
        if (threadIdx.x == 0) write_none(call, r);
        return;
    }
    auto counter = [&](int run, int l) -> uint32_t {
        const uint32_t x = pattern_of(run, l), c = s.counts[x & 0x7fffu];
        return run == 510 && l < 63 ? 0u : run < 512 ? c & 0xffffu : c >> 16;
    };
    const int top_run = __builtin_amdgcn_readfirstlane((int)s.run[0]);
    const int top_place = __builtin_ctzll(__builtin_amdgcn_ballot_w64(counter(top_run, lane) != 0));
    const uint32_t top_pattern = pattern_of(top_run, top_place);
    const bool greedy = !(p.temperature > 0.0f);
    uint32_t pattern = top_pattern, rank = 0;
    if (!greedy) {
        const Weights weights(bf16_value(top_pattern), p.temperature, unit_of(call));
        // ---- tokens and mass of every run
        for (int e = wave; e < n_runs; e += kWaves) {
            const int run = __builtin_amdgcn_readfirstlane((int)s.run[e]);
            const uint32_t c = counter(run, lane);
            u64 m = 0;
            if (c) m = c * weights.units(bf16_value(pattern_of(run, lane)));
            const uint32_t tokens = prefix_sum(c);
            m = prefix_sum(m);
            if (lane == 63) s.run_count[e] = tokens, s.run_mass[e] = m;
        }
        __syncthreads();
        if (wave == 0) {
            uint32_t tokens = 0;
            u64 mass = 0;
            for (int e0 = 0; e0 < n_runs; e0 += 64) {
                const int e = e0 + lane;
                uint32_t c = e < n_runs ? s.run_count[e] : 0;
                u64 m = e < n_runs ? s.run_mass[e] : 0;
                c = prefix_sum(c) + tokens;
                m = prefix_sum(m) + mass;
                if (e < n_runs) s.run_count[e] = c, s.run_mass[e] = m;
                tokens = at_lane(c, 63);
                mass = at_lane(m, 63);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            struct Place {
                uint32_t pattern, above;  // the value a target is reached on, and what lies above it
                u64 mass_above, unit;     // its weight
            };
            // the first run for which `reached(e)` holds (none: the last one), and the place in it for which `reached_place(tokens, mass, weight)` holds
            auto find = [&](auto reached, auto reached_place) -> Place {
                int at = n_runs - 1;
                for (int e0 = 0; e0 < n_runs; e0 += 64) {
                    const u64 hit = __builtin_amdgcn_ballot_w64(e0 + lane < n_runs && reached(e0 + lane));
                    if (hit) {
                        at = e0 + __builtin_ctzll(hit);
                        break;
                    }
                }
                const int run = __builtin_amdgcn_readfirstlane((int)s.run[at]);
                const uint32_t c = counter(run, lane);
                const uint32_t x = pattern_of(run, lane);
                const double w = c ? weights.of(bf16_value(x)) : 0.0;
                const u64 unit = c ? weights.whole(w) : 0;
                const u64 m = c * unit;
                const uint32_t before = at ? s.run_count[at - 1] : 0;
                const u64 mass_before = at ? s.run_mass[at - 1] : 0;
                const uint32_t ci = prefix_sum(c) + before;
                const u64 mi = prefix_sum(m) + mass_before;
                const u64 hit = __builtin_amdgcn_ballot_w64(c != 0 && reached_place(ci, mi, w));
                if (hit == 0) return Place{0, at_lane(ci, 63), at_lane(mi, 63), 0};  // (only min_p asks for what may be in the next run)
                const int l = __builtin_ctzll(hit);
                return Place{at_lane(x, l), at_lane(ci - c, l), at_lane(mi - m, l), at_lane(unit, l)};
            };
            auto by_count = [&](uint32_t target) {
                return find([&](int e) { return s.run_count[e] >= target; }, [&](uint32_t c, u64, double) { return c >= target; });
            };
            auto by_mass = [&](u64 target) {
                return find([&](int e) { return s.run_mass[e] >= target; }, [&](uint32_t, u64 m, double) { return m >= target; });
            };
            // of the tokens with the value, the one (from 0) on which the mass is reached
            auto rank_of = [](const Place& f, u64 target) -> uint32_t { return (uint32_t)((target - f.mass_above + f.unit - 1) / f.unit - 1); };
            uint32_t kept = tokens;
            u64 kept_mass = mass;
            if (p.top_k > 0 && (uint32_t)p.top_k < kept) {
                const Place f = by_count((uint32_t)p.top_k);
                kept = (uint32_t)p.top_k;
                kept_mass = f.mass_above + (kept - f.above) * f.unit;
            }
            if (p.top_p < 1.0f) {
                const u64 target = top_p_target(p.top_p, kept_mass);
                const Place f = by_mass(target);
                const uint32_t k = rank_of(f, target);
                kept = min(kept, f.above + k + 1);
                kept_mass = f.mass_above + (k + 1) * f.unit;
            }
            if (p.min_p > 0.0f) {
                // what lies above the first value that is too light (the last value of a run stands for the run: it need not occur)
                const double least = fmin((double)p.min_p, 1.0);
                const Place f = find([&](int e) { return weights.of(bf16_value(pattern_of(s.run[e], 63))) < least; },
                                     [&](uint32_t, u64, double w) { return w < least; });
                if (f.above < kept) kept_mass = f.mass_above;
            }
            const u64 target = draw_target(u, kept_mass);
            const Place f = by_mass(target);
            if (lane == 0) s.pattern = f.pattern, s.rank = rank_of(f, target), s.kept_mass = kept_mass;
        }
        __syncthreads();
        pattern = s.pattern;
        rank = s.rank;
        if (call.logprobs && threadIdx.x == kThreads - 1) call.logprobs[r] = weights.logprob(bf16_value(pattern), s.kept_mass);
    } else if (call.logprobs && threadIdx.x == 0) {
        call.logprobs[r] = 0.0f;
    }

    // ---- which of the tokens with that value: the rank-th by index, by chunks of the row (head, pieces, tail), then in one
    const uint32_t both = pattern * 0x10001u, ignored = pattern == 0 ? 0x7fff7fffu : 0xffffffffu;  // (zeros: of either sign)
    auto matches = [&](const u32x4& x) -> uint32_t {  // bit j: element j
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t y = (x[j] ^ both) & ignored;
            bits |= ((y & 0xffffu) == 0 ? 1u : 0u) << (2 * j) | (y >> 16 == 0 ? 2u : 0u) << (2 * j);
        }
        return bits;
    };
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    auto any = [&](const u32x4& x) -> bool {  // (for zeros: perhaps)
        u16x2 least = {0xffff, 0xffff};
#pragma unroll
        for (int j = 0; j < 4; ++j) least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, x[j] ^ both));
        const uint32_t l = __builtin_bit_cast(uint32_t, least);
        return (l & 0xffffu) == 0 || l >> 16 == 0 || pattern == 0;
    };
    const bool edge_matches = has_edge && (edge_pattern ^ (pattern & 0xffffu)) == 0 || (has_edge && pattern == 0 && edge_pattern == 0x8000u);
    if (edge_matches) atomicAdd(&s.chunk_count[edge < head ? 0 : chunks + 1], 1u);
    auto count_matches = [&](int i, const u32x4& x) {
        if (any(x)) atomicAdd(&s.chunk_count[i + 1], (uint32_t)__builtin_popcount(matches(x)));
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * kThreads + (int)threadIdx.x < n_body) count_matches(i, v[i]);
    } else {
        for (int i = 0; i < chunks; ++i)
            if (i * kThreads + (int)threadIdx.x < n_body) count_matches(i, body[i * kThreads + threadIdx.x]);
    }
    __syncthreads();
    int chunk = 0;
    while (chunk < chunks + 1 && s.chunk_count[chunk] <= rank) rank -= s.chunk_count[chunk++];
    chunk = __builtin_amdgcn_readfirstlane(chunk);
    uint32_t bits = 0;
    int first = edge;
    if (chunk == 0 || chunk == chunks + 1) {
        bits = edge_matches && (edge < head) == (chunk == 0) ? 1u : 0u;
    } else {
        const int at = (chunk - 1) * kThreads + (int)threadIdx.x;
        first = head + at * 8;
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i == chunk - 1 && at < n_body) bits = matches(v[i]);
        } else {
            if (at < n_body) bits = matches(body[at]);
        }
    }
    const uint32_t mine = __builtin_popcount(bits);
    uint32_t upto = prefix_sum(mine);
    if (lane == 63) s.wave_sum[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += s.wave_sum[w];
    if (upto - mine <= rank && rank < upto) {
        uint32_t skip = rank - (upto - mine);
        while (skip-- > 0) bits &= bits - 1;
        write_token(call, r, first + __builtin_ctz(bits));
    }
}

}  // namespace

hipError_t launch_sample_tokens(const SampleCall& call, bool f32, hipStream_t st) {
    if (call.n <= 0) return hipSuccess;
#define APAR_SAMPLE(KERNEL) hipLaunchKernelGGL((KERNEL), dim3((unsigned)call.n), dim3(kThreads), 0, st, call)
    const int pieces = (call.vocab / 8 + kThreads - 1) / kThreads;  // of a bf16 row, per thread
    if (f32) APAR_SAMPLE(sample_rows_f32);
    else if (pieces <= 4) APAR_SAMPLE(sample_rows_bf16<4>);
    else if (pieces <= 8) APAR_SAMPLE(sample_rows_bf16<8>);
    else if (pieces <= 16) APAR_SAMPLE(sample_rows_bf16<16>);
    else APAR_SAMPLE(sample_rows_bf16<0>);
#undef APAR_SAMPLE
    return hipGetLastError();
}

}  // namespace apar
