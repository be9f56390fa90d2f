// Rotary positions: what the host hands to the kernel.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apar.h"

namespace apar {

constexpr int kRotaryMaxPairs = 128;
constexpr int kRotaryInlineWords = 512;
constexpr int kRotaryMostRowsPerWg = 4;
constexpr int64_t kRotaryMaxRows = (int64_t)kRotaryMostRowsPerWg * ((1 << 24) - 1);  // (a launch has fewer than 2^32 threads)

struct RotaryArgs {                       // the kernel's first argument, read from the head of the argument segment
    double theta[kRotaryMaxPairs];        // turns per position
    int32_t words[kRotaryInlineWords];    // a small call's tables of positions
};

struct RotaryRows {
    const void* in;
    void* out;
    int64_t in_stride, out_stride;        // elements from row to row; heads lie side by side
    int32_t n_heads;
};

struct RotaryCall {
    RotaryRows q, k;
    const int32_t* positions;             // per row, on the device; or null, and ...
    const int32_t* tables;                // ... positions of the listed threads' first rows, on the device (null: RotaryArgs::words):
    int32_t rows_per_entry;               // > 0: one word per thread, this many rows each; 0: first row and its position per thread
    int32_t n_entries;
    const uint8_t* mask;                  // candidates: a row's position is as many places behind its thread's as it sees others
    int64_t n_rows;
    int32_t head_dim, rotary_dim, pairs, transposed, rows_per_wg;
    float magnitude;
};

hipError_t launch_rotate_rows(const RotaryArgs& args, RotaryCall call, bool f32, hipStream_t st);

}  // namespace apar

struct apar_rotary {
    apar_rotary_config cfg;
    apar::RotaryArgs args;
};
