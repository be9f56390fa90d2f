// Rotary positions: frequencies, checks, positions of listed threads' rows.
#include "rotary.hpp"

#include <cmath>
#include <cstring>
#include <new>
#include <unordered_map>
#include <vector>

#include "apar_internal.hpp"
#include "hip_status.hpp"
#include "pool_access.hpp"

using namespace apar;

namespace {

// Checks of the rows a call turns (q or k; null: none of them), and their place in `out`.
int rotary_rows(const apar_rotary& r, const apar_rotary_rows* x, RotaryRows& out) {
    out = RotaryRows{};
    if (!x) return APAR_OK;
    if (x->head_dim != 0 && x->head_dim != r.cfg.head_dim) return APAR_ERR_INVALID_ARG;
    const int64_t row = (int64_t)x->n_heads * r.cfg.head_dim;
    if (!x->in_dev || !x->out_dev || x->n_heads < 1 || x->in_stride < row || x->out_stride < row) return APAR_ERR_INVALID_ARG;
    if (x->in_dev == x->out_dev && x->in_stride != x->out_stride) return APAR_ERR_INVALID_ARG;
    out = RotaryRows{x->in_dev, x->out_dev, x->in_stride, x->out_stride, x->n_heads};
    return APAR_OK;
}

// The last checks of a call, and what it takes from the handle.  Nothing is enqueued before them.
int rotary_ready(const apar_rotary& r, RotaryCall& call, bool f32, int transposed) {
    if (call.n_rows > kRotaryMaxRows) return APAR_ERR_UNSUPPORTED;
    if (((int64_t)call.q.n_heads + call.k.n_heads) * r.cfg.head_dim > INT32_MAX / 4) return APAR_ERR_UNSUPPORTED;
    const uintptr_t odd = (uintptr_t)call.q.in | (uintptr_t)call.q.out | (uintptr_t)call.k.in | (uintptr_t)call.k.out;
    if (odd & (f32 ? 3 : 1)) return APAR_ERR_INVALID_ARG;
    call.head_dim = r.cfg.head_dim;
    call.rotary_dim = r.cfg.rotary_dim;
    call.pairs = r.cfg.layout == APAR_ROTARY_PAIRS;
    call.transposed = transposed != 0;
    call.magnitude = (float)r.cfg.magnitude;
    return APAR_OK;
}

// Launches on the device that `on` lies on.
int rotary_launch(const RotaryArgs& args, const RotaryCall& call, bool f32, const void* on, void* hip_stream) {
    DeviceOf guard(on);
    HIP_TRY(launch_rotate_rows(args, call, f32, (hipStream_t)hip_stream));
    return APAR_OK;
}

// Where the listed threads' rows lie, in the kernel's terms (RotaryCall::rows_per_entry).
int positions_of(apar_pool* p, const apar_thread* threads, const int32_t* m, int n, int where, int n_cand, std::vector<int32_t>& words,
                 RotaryCall& call) {
    bool uniform = true, ascending = true;
    for (int i = 1; i < n; ++i) {
        uniform = uniform && (!m || m[i] == m[0]);
        ascending = ascending && threads[i] > threads[i - 1];  // (no thread twice, then)
    }
    // rows to come follow those that an earlier entry of the same thread has
    std::unordered_map<int32_t, int64_t> ahead;
    const bool follow = where == APAR_ROWS_NEXT && n_cand == 0 && !ascending;
    int64_t row = 0;
    words.reserve(uniform ? (size_t)n : 2 * (size_t)n);
    for (int i = 0; i < n; ++i) {
        int64_t len = 0;
        const int rc = apar_thread_len(p, threads[i], &len);
        if (rc != APAR_OK) return rc;
        const int64_t rows = n_cand > 0 ? n_cand : m ? m[i] : 1;
        if (rows < (where == APAR_ROWS_LAST ? 1 : 0) || (where == APAR_ROWS_LAST && rows > len)) return APAR_ERR_INVALID_ARG;
        int64_t first = where == APAR_ROWS_LAST ? len - rows : len;
        if (follow) {
            int64_t& a = ahead[threads[i]];
            first += a;
            a += rows;
        }
        if (first + rows - 1 > INT32_MAX || row + rows > INT32_MAX) return APAR_ERR_UNSUPPORTED;
        if (uniform) {
            words.push_back((int32_t)first);
        } else if (rows > 0) {
            words.push_back((int32_t)row);
            words.push_back((int32_t)first);
        }
        row += rows;
    }
    call.n_rows = row;
    call.rows_per_entry = uniform ? (int32_t)(row / n) : 0;
    call.n_entries = (int32_t)(uniform ? words.size() : words.size() / 2);
    return APAR_OK;
}

int rotate_threads(apar_pool* p, const apar_rotary* r, int dtype, const apar_thread* threads, const int32_t* m, int n, int where,
                   const uint8_t* mask_dev, int n_cand, const apar_rotary_rows* q, const apar_rotary_rows* k, int transposed,
                   void* hip_stream) {
    if (!p || !r || n < 0 || (where != APAR_ROWS_NEXT && where != APAR_ROWS_LAST)) return APAR_ERR_INVALID_ARG;
    const PoolFacts pool = facts_of(p);
    if (r->cfg.head_dim != pool.shape->d || (!pool.dry_run && dtype != pool.shape->dtype)) return APAR_ERR_INVALID_ARG;
    if (n_cand < 0 || n_cand > 8 || (n_cand > 0 && (m || where != APAR_ROWS_NEXT))) return APAR_ERR_INVALID_ARG;
    if (n == 0) return APAR_OK;
    if (!threads || (n_cand == 0 && mask_dev)) return APAR_ERR_INVALID_ARG;
    if (pool.dry_run ? (q || k || mask_dev) : (!q && !k) || (n_cand > 0 && !mask_dev)) return APAR_ERR_INVALID_ARG;
    if ((q && q->n_heads != pool.shape->n_q) || (k && k->n_heads != pool.shape->n_kv)) return APAR_ERR_INVALID_ARG;
    RotaryCall call{};
    std::vector<int32_t> words;
    int rc;
    if ((rc = rotary_rows(*r, q, call.q)) != APAR_OK || (rc = rotary_rows(*r, k, call.k)) != APAR_OK) return rc;
    if ((rc = positions_of(p, threads, m, n, where, n_cand, words, call)) != APAR_OK) return rc;
    if (pool.dry_run || call.n_rows == 0) return APAR_OK;
    call.mask = mask_dev;
    const bool f32 = dtype == APAR_F32;
    if ((rc = rotary_ready(*r, call, f32, transposed)) != APAR_OK) return rc;
    if (words.size() <= (size_t)kRotaryInlineWords) {
        RotaryArgs args = r->args;
        memcpy(args.words, words.data(), words.size() * sizeof(int32_t));
        return rotary_launch(args, call, f32, pool.kv, hip_stream);
    }
    DeviceGuard guard(pool.device);
    StagedWords staged{};
    if ((rc = stage_words(p, words.data(), words.size(), (hipStream_t)hip_stream, &staged)) != APAR_OK) return rc;
    call.tables = staged.dev;
    rc = rotary_launch(r->args, call, f32, pool.kv, hip_stream);
    const int read = staged_words_read(staged, (hipStream_t)hip_stream);  // (without a kernel too: the upload is under way)
    return rc != APAR_OK ? rc : read;
}

}  // namespace

extern "C" {

int apar_rotary_create(const apar_rotary_config* cfg, apar_rotary** out) {
    if (!cfg || !out) return APAR_ERR_INVALID_ARG;
    *out = nullptr;
    const apar_rotary_config& c = *cfg;
    if (c.head_dim < 2 || c.head_dim % 2 || c.rotary_dim < 2 || c.rotary_dim % 2 || c.rotary_dim > c.head_dim) return APAR_ERR_INVALID_ARG;
    if (c.layout != APAR_ROTARY_HALF && c.layout != APAR_ROTARY_PAIRS) return APAR_ERR_INVALID_ARG;
    if (c.scaling < APAR_ROTARY_SCALE_NONE || c.scaling > APAR_ROTARY_SCALE_RAMP) return APAR_ERR_INVALID_ARG;
    auto positive = [](double x) { return x > 0.0 && std::isfinite(x); };
    if (!positive(c.base) || !positive(c.magnitude) || !std::isfinite((float)c.magnitude)) return APAR_ERR_INVALID_ARG;
    if (c.scaling != APAR_ROTARY_SCALE_NONE && !positive(c.factor)) return APAR_ERR_INVALID_ARG;
    if (c.scaling == APAR_ROTARY_SCALE_BASE && c.rotary_dim == 2) return APAR_ERR_INVALID_ARG;
    if (c.scaling == APAR_ROTARY_SCALE_RAMP &&
        !(positive(c.original_len) && std::isfinite(c.low_turns) && std::isfinite(c.high_turns) && c.low_turns < c.high_turns))
        return APAR_ERR_INVALID_ARG;
    if (c.head_dim > 2 * kRotaryMaxPairs) return APAR_ERR_UNSUPPORTED;
    apar_rotary* r = new (std::nothrow) apar_rotary{};
    if (!r) return APAR_ERR_INVALID_ARG;
    r->cfg = c;
    const double d = c.rotary_dim;
    const double base = c.scaling == APAR_ROTARY_SCALE_BASE ? c.base * std::pow(c.factor, d / (d - 2.0)) : c.base;
    for (int i = 0; i < c.rotary_dim / 2; ++i) {
        double turns = std::pow(base, -2.0 * i / d) / (2.0 * M_PI);
        if (c.scaling == APAR_ROTARY_SCALE_LINEAR) turns /= c.factor;
        if (c.scaling == APAR_ROTARY_SCALE_RAMP) {
            const double keep = std::fmin(std::fmax((c.original_len * turns - c.low_turns) / (c.high_turns - c.low_turns), 0.0), 1.0);
            turns = keep * turns + (1.0 - keep) * turns / c.factor;
        }
        if (!std::isfinite(turns)) {
            delete r;
            return APAR_ERR_INVALID_ARG;
        }
        r->args.theta[i] = turns;
    }
    *out = r;
    return APAR_OK;
}

int apar_rotary_destroy(apar_rotary* r) {
    delete r;
    return APAR_OK;
}

int apar_rotary_frequencies(const apar_rotary* r, double* out, int cap, int* n_out) {
    if (!r || !n_out || cap < 0 || (cap > 0 && !out)) return APAR_ERR_INVALID_ARG;
    *n_out = r->cfg.rotary_dim / 2;
    if (cap < *n_out) return APAR_ERR_INVALID_ARG;
    for (int i = 0; i < *n_out; ++i) out[i] = r->args.theta[i] * (2.0 * M_PI);
    return APAR_OK;
}

int apar_rotate_rows(const apar_rotary* r, int dtype, const int32_t* positions_dev, int64_t n_rows, const apar_rotary_rows* q,
                     const apar_rotary_rows* k, int transposed, void* hip_stream) {
    if (!r || n_rows < 0 || (!q && !k)) return APAR_ERR_INVALID_ARG;
    if (dtype != APAR_F32 && dtype != APAR_BF16) return APAR_ERR_INVALID_ARG;
    if (n_rows == 0) return APAR_OK;
    if (!positions_dev) return APAR_ERR_INVALID_ARG;
    RotaryCall call{};
    int rc;
    if ((rc = rotary_rows(*r, q, call.q)) != APAR_OK || (rc = rotary_rows(*r, k, call.k)) != APAR_OK) return rc;
    call.positions = positions_dev;
    call.n_rows = n_rows;
    if ((rc = rotary_ready(*r, call, dtype == APAR_F32, transposed)) != APAR_OK) return rc;
    return rotary_launch(r->args, call, dtype == APAR_F32, positions_dev, hip_stream);
}

int apar_rotate_threads(apar_pool* p, const apar_rotary* r, int dtype, const apar_thread* threads, const int32_t* m, int n, int where,
                        const uint8_t* mask_dev, int n_cand, const apar_rotary_rows* q, const apar_rotary_rows* k, int transposed,
                        void* hip_stream) {
    try {
        return rotate_threads(p, r, dtype, threads, m, n, where, mask_dev, n_cand, q, k, transposed, hip_stream);
    } catch (...) {  // (no memory for the positions)
        return APAR_ERR_INVALID_ARG;
    }
}

}  // extern "C"
