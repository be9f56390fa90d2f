// Sampling of tokens (gfx950): one workgroup per row of logits.
//
// A row's tokens stand in one order, value descending, index ascending.  With w = exp((x - max) / T) every cut is a prefix of it:
//   top-k: the first k;  top-p: the shortest prefix with mass >= p * (mass of the first k);  min-p: w >= min_p;
// and the token is the first one whose cumulated mass exceeds u * (mass of what is kept).  So a row never has to be sorted: each of these
// is the place where a cumulated count or mass reaches a target, found by digits of the values' ordered bit patterns (keys), 12, 12 and
// 8 bits: a histogram of counts and masses over the first digit, then over the next one of the values that share the first, and so
// on; among equal values the place follows from their weight, and the index from counting them.
// Masses are sums of whole numbers, w 2^weight_bits rounded (42 to 61 bits by the size of the vocabulary, w computed in 64): they
// do not depend on the order of the additions, and all prefixes agree with each other.
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

// Inclusive sums over the threads of the workgroup, in their order.
__device__ __forceinline__ void scan(Shared& s, uint32_t& count, u64& mass) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t c = __shfl_up(count, o, 64);
        const u64 m = __shfl_up(mass, o, 64);
        if (lane >= o) count += c, mass += m;
    }
    if (lane == 63) s.wave_count[wave] = count, s.wave_mass[wave] = mass;
    __syncthreads();
    for (int w = 0; w < wave; ++w) count += s.wave_count[w], mass += s.wave_mass[w];
    __syncthreads();
}

// The bin, from the largest down, in which the cumulated count or mass (of what lies above the bins, `above`, and the bins) reaches
// the target; what lies above that bin.
__device__ __forceinline__ int reach(Shared& s, const uint32_t* counts, const u64* masses, int bins, bool by_mass, u64 target,
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

template <class T>
__global__ __launch_bounds__(kThreads) void sample_rows(SampleCall call) {
    __shared__ Shared s;
    const int r = blockIdx.x, vocab = call.vocab;
    const T* row = (const T*)call.logits + (int64_t)r * call.row_stride;
    const apar_sample_row p = call.rows ? call.rows[r] : apar_sample_row{1.0f, 0, 1.0f, 0.0f};
    const double one = ldexp(1.0, call.weight_bits);
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
        if (threadIdx.x == 0) {
            call.tokens[r] = APAR_TOKEN_NONE;
            if (call.logprobs) call.logprobs[r] = -INFINITY;
        }
        return;
    }
    const double x_top = value_of(top);
    const double temperature = p.temperature;
    auto weight = [&](float x) -> double { return (double)x == x_top ? 1.0 : exp(((double)x - x_top) / temperature); };
    auto whole = [&](double w) -> u64 { return (u64)(w * one + 0.5); };

    Found token{top, 0, 0, 0};
    u64 kept_mass = whole(1.0);
    if (!greedy) {
        uint32_t n = 0, n_min = 0;
        u64 m = 0, m_min = 0;
        each<T>(row, vocab, [&](int, float x) {
            if (!(x > -INFINITY)) return;
            const uint32_t key = key_of(x);
            const double wd = weight(x);
            const u64 w = whole(wd);
            atomicAdd(&s.count0[key >> 20], 1u);
            atomicAdd(&s.mass0[key >> 20], w);
            n += 1, m += w;
            if (!(wd < (double)p.min_p) || key == top) n_min += 1, m_min += w;
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
                    atomicAdd(&s.mass1[(key >> shift) & (bins - 1)], whole(weight(x)));
                });
                __syncthreads();
                f.key |= (uint32_t)reach(s, s.count1, s.mass1, bins, by_mass, target, f.above, f.mass_above) << shift;
            }
            if (sizeof(T) == 2) f.key = f.key >> 31 ? f.key & 0xffff0000u : f.key | 0xffffu;
            const u64 left = target - (by_mass ? f.mass_above : f.above);  // of the tokens with this value, from 1
            const u64 w = whole(weight(value_of(f.key)));
            f.rank = (uint32_t)(by_mass ? (left + w - 1) / w - 1 : left - 1);
            return f;
        };
        auto mass_to = [&](const Found& f) -> u64 { return f.mass_above + (f.rank + 1) * whole(weight(value_of(f.key))); };

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
            const double target = ceil((double)fmaxf(p.top_p, 0.0f) * (double)kept_mass);
            const Found f = find(true, max((u64)1, min((u64)target, kept_mass)));
            kept = min(kept, f.above + f.rank + 1);
            kept_mass = mass_to(f);
        }
        if (min_count < kept) kept_mass = min_mass;
        const double u = fminf(fmaxf(call.uniforms[r], 0.0f), 1.0f);
        token = find(true, min((u64)(u * (double)kept_mass) + 1, kept_mass));
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
        const int index = first + __builtin_ctz(bits);
        call.tokens[r] = index == call.ids.fork ? APAR_TOKEN_FORK : index == call.ids.child ? APAR_TOKEN_CHILD
                         : index == call.ids.eos ? APAR_TOKEN_EOS : index;
        if (call.logprobs) {
            const double z = greedy || token.key == top ? 0.0 : ((double)value_of(token.key) - x_top) / temperature;
            call.logprobs[r] = greedy ? 0.0f : (float)(z - log((double)kept_mass / one));
        }
    }
}

}  // namespace

hipError_t launch_sample_tokens(const SampleCall& call, bool f32, hipStream_t st) {
    if (call.n <= 0) return hipSuccess;
    if (f32) hipLaunchKernelGGL(sample_rows<float>, dim3((unsigned)call.n), dim3(kThreads), 0, st, call);
    else hipLaunchKernelGGL(sample_rows<uint16_t>, dim3((unsigned)call.n), dim3(kThreads), 0, st, call);
    return hipGetLastError();
}

}  // namespace apar
