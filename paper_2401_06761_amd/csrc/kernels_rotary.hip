// Rotary positions (gfx950): q and k rows, head by head, pairs of dims turned by the angle position * theta_i.
//
//   y_a = s (x_a cos - x_b sin),  y_b = s (x_b cos + x_a sin)        transposed: sin -> -sin
//
// Angles are kept in turns and in 64 bits until the fraction of a turn is left: position * theta / 2 pi of a far position loses
// as many bits in 32 as it has whole turns.  The fraction, at most half, is then good to 2^-26 in 32 bits, 9e-8 of angle.
// A workgroup takes a few rows: its threads work out the sines and cosines of the rows' pairs once, in LDS, and then go through
// all heads of those rows, 16 bytes of a's and 16 of b's a lane (the bytes of a pair's partner in another lane would need an
// exchange).  What bounds it: memory, every row read and written once (16 k rows of 40 bf16 heads, 335 MB in 62 us, 5.4 TB/s); calls of few
// rows: the launch (48 rows 4.3 us).
#include <hip/hip_runtime.h>

#include <cstring>

#include "apar_internal.hpp"
#include "rotary.hpp"

namespace apar {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// W consecutive elements (16 bytes, or one) to and from floats; bf16: round to nearest even.
__device__ __forceinline__ void load_run(const float* p, float (&x)[4]) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
}
__device__ __forceinline__ void load_run(const uint16_t* p, float (&x)[8]) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(v[i] << 16), x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
}
__device__ __forceinline__ void load_run(const float* p, float (&x)[1]) { x[0] = *p; }
__device__ __forceinline__ void load_run(const uint16_t* p, float (&x)[1]) { x[0] = __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    const f32x2 p = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
}
__device__ __forceinline__ void store_run(float* p, const float (&x)[4]) { *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]}; }
__device__ __forceinline__ void store_run(uint16_t* p, const float (&x)[8]) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_pair(x[0], x[1]), pack_pair(x[2], x[3]), pack_pair(x[4], x[5]), pack_pair(x[6], x[7])};
}
__device__ __forceinline__ void store_run(float* p, const float (&x)[1]) { *p = x[0]; }
__device__ __forceinline__ void store_run(uint16_t* p, const float (&x)[1]) { *p = (uint16_t)pack_pair(x[0], x[0]); }

template <class T, int W>
struct Piece { typedef u32x4 type; };  // W elements as they are
template <class T>
struct Piece<T, 1> { typedef T type; };

// W pairs a lane: 16 bytes of either half (1: sizes or addresses that do not allow that).  PAIRS: the dims of a pair lie side by side.
template <class T, int W, bool PAIRS>
__global__ __launch_bounds__(256) void rotate_rows(RotaryArgs args, RotaryCall call) {
    extern __shared__ f32x2 turns[];  // [rows of the workgroup][pairs]: cosine, sine
    const int64_t row0 = (int64_t)blockIdx.x * call.rows_per_wg;
    const int n_rows = (int)min((int64_t)call.rows_per_wg, call.n_rows - row0);
    const int pairs = call.rotary_dim / 2;
    // the tables are the first argument, read where they are
    typedef const double __attribute__((address_space(4))) * Doubles;
    typedef const int32_t __attribute__((address_space(4))) * Words;
    const auto theta = (Doubles)__builtin_amdgcn_kernarg_segment_ptr();
    const auto inlined = (Words)(theta + kRotaryMaxPairs);
    auto word = [&](int i) -> int { return call.tables ? call.tables[i] : inlined[i]; };
    for (int at = threadIdx.x; at < n_rows * pairs; at += 256) {
        const int r = at / pairs, i = at - r * pairs;
        const int64_t row = row0 + r;
        int64_t pos;
        if (call.positions) {
            pos = call.positions[row];
        } else if (call.rows_per_entry > 0) {  // as many rows for every listed thread
            const int entry = (int)(row / call.rows_per_entry);
            pos = word(entry);
            const int own = (int)(row - (int64_t)entry * call.rows_per_entry);
            if (call.mask)  // a candidate's ancestors are the others that it sees
                pos += __builtin_popcount(call.mask[row] & ((1u << call.rows_per_entry) - 1u) & ~(1u << own));
            else
                pos += own;
        } else {  // the last listed thread whose first row is not behind this one
            int lo = 0, hi = call.n_entries;
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (word(2 * mid) <= row) lo = mid;
                else hi = mid;
            }
            pos = word(2 * lo + 1) + (row - word(2 * lo));
        }
        const double t = (double)pos * theta[i];
        float s, c;
        sincospif(2.0f * (float)(t - rint(t)), &s, &c);
        turns[at] = f32x2{c * call.magnitude, s * (call.transposed ? -call.magnitude : call.magnitude)};
    }
    __syncthreads();
    const int heads = call.q.n_heads + call.k.n_heads;
    const int pieces = call.head_dim / (2 * W), turned = call.rotary_dim / (2 * W);  // a piece is 2 W dims of a head
    const int total = n_rows * heads * pieces;
    for (int at = threadIdx.x; at < total; at += 256) {
        const int rh = at / pieces, piece = at - rh * pieces;
        const int r = rh / heads, head = rh - r * heads;
        const bool is_q = head < call.q.n_heads;
        const RotaryRows& x = is_q ? call.q : call.k;
        const int h = is_q ? head : head - call.q.n_heads;
        const T* in = (const T*)x.in + (row0 + r) * x.in_stride + (int64_t)h * call.head_dim;
        T* out = (T*)x.out + (row0 + r) * x.out_stride + (int64_t)h * call.head_dim;
        if (piece >= turned) {  // dims behind the turned ones: taken over
            if (in == out) continue;
            typedef typename Piece<T, W>::type Bits;
            const Bits* from = reinterpret_cast<const Bits*>(in + 2 * W * piece);
            Bits* to = reinterpret_cast<Bits*>(out + 2 * W * piece);
            const Bits first = from[0], second = from[1];
            to[0] = first;
            to[1] = second;
            continue;
        }
        float u[W], v[W];
        const int a = PAIRS ? 2 * W * piece : W * piece, b = PAIRS ? a + W : a + pairs;
        load_run(in + a, u);
        load_run(in + b, v);
        const f32x2* cs = turns + r * pairs + W * piece;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            // pair j of the piece: elements j of u and of v, or 2 j and 2 j + 1 of the two together
            float& ea = !PAIRS ? u[j] : 2 * j < W ? u[2 * j % W] : v[2 * j % W];
            float& eb = !PAIRS ? v[j] : 2 * j + 1 < W ? u[(2 * j + 1) % W] : v[(2 * j + 1) % W];
            const float fa = ea, fb = eb;
            ea = fa * cs[j].x - fb * cs[j].y;
            eb = fb * cs[j].x + fa * cs[j].y;
        }
        store_run(out + a, u);
        store_run(out + b, v);
    }
}

}  // namespace

hipError_t launch_rotate_rows(const RotaryArgs& args, RotaryCall call, bool f32, hipStream_t st) {
    if (call.n_rows <= 0) return hipSuccess;
    const int e = f32 ? 4 : 2, w = 16 / e;
    auto wide = [&](const RotaryRows& x) {
        return x.n_heads == 0 || ((((uintptr_t)x.in | (uintptr_t)x.out) & 15) == 0 && x.in_stride % w == 0 && x.out_stride % w == 0);
    };
    const bool vec = call.rotary_dim % (2 * w) == 0 && call.head_dim % (2 * w) == 0 && wide(call.q) && wide(call.k);
    // Rows per workgroup: enough workgroups for the chip first, then rows that keep all threads at sines and cosines.
    call.rows_per_wg = call.n_rows >= 2048 ? kRotaryMostRowsPerWg : call.n_rows >= 1024 ? 2 : 1;
    const int64_t grid = (call.n_rows + call.rows_per_wg - 1) / call.rows_per_wg;
    if (call.n_rows > kRotaryMaxRows) return hipErrorInvalidValue;
    const size_t lds = (size_t)call.rows_per_wg * (call.rotary_dim / 2) * sizeof(f32x2);
#define APAR_ROTATE(TV, WV, PV) hipLaunchKernelGGL((rotate_rows<TV, WV, PV>), dim3((unsigned)grid), dim3(256), lds, st, args, call)
#define APAR_ROTATE_PAIRS(TV, WV)                 \
    do {                                          \
        if (call.pairs) APAR_ROTATE(TV, WV, true); \
        else APAR_ROTATE(TV, WV, false);          \
    } while (0)
    if (f32) {
        if (vec) APAR_ROTATE_PAIRS(float, 4);
        else APAR_ROTATE_PAIRS(float, 1);
    } else {
        if (vec) APAR_ROTATE_PAIRS(uint16_t, 8);
        else APAR_ROTATE_PAIRS(uint16_t, 1);
    }
#undef APAR_ROTATE_PAIRS
#undef APAR_ROTATE
    return hipGetLastError();
}

}  // namespace apar
