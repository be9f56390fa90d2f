// What operators beside the pool need of it: its shape, and the way small tables go to the device.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

#include "apar_internal.hpp"

namespace apar {

struct PoolFacts {
    const Shape* shape;
    const void* kv;   // null on a dry-run pool
    int device;
    bool dry_run;
};
PoolFacts facts_of(const apar_pool* p);

// Words on their way to the device through one of the pool's staging slots; staged_words_read once the kernels that read them are
// enqueued.  The pool's device is the current one.
struct StagedWords {
    const int32_t* dev;
    void* slot;
};
int stage_words(apar_pool* p, const int32_t* words, size_t n, hipStream_t st, StagedWords* out);
int staged_words_read(const StagedWords& w, hipStream_t st);

}  // namespace apar
