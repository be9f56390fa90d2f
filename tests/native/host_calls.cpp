// What calls hand on to the kernels, and what a call that fails leaves behind, against the runtime of host_pool.cpp.  Built and run by
// tests/test_host_calls.py, which names the check to run.
#include "apar_internal.hpp"
#include "rotary.hpp"

#define main host_pool_main
#define launch_append_blocks append_nothing
#define launch_read_rows read_nothing
#define hipMemcpyAsync copy_at_once
#define hipEventRecord record_nothing
#define hipEventSynchronize wait_for_nothing
#include "host_pool.cpp"
#undef main
#undef launch_append_blocks
#undef launch_read_rows
#undef hipMemcpyAsync
#undef hipEventRecord
#undef hipEventSynchronize

// Copies to the device that may still be under way: until an event recorded behind one has been waited for, what it reads must not change.
struct Upload {
    const void* from;
    std::vector<char> was;
    long at;
};
static std::vector<Upload> g_uploads;
static std::map<hipEvent_t, long> g_recorded;
static long g_enqueued = 0;
extern "C" {
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) {
    std::memcpy(d, s, n);
    g_uploads.push_back(Upload{s, std::vector<char>((const char*)s, (const char*)s + n), ++g_enqueued});
    return hipSuccess;
}
hipError_t hipEventRecord(hipEvent_t e, hipStream_t) {
    g_recorded[e] = g_enqueued;
    return hipSuccess;
}
hipError_t hipEventSynchronize(hipEvent_t e) {
    const long done = g_recorded[e];
    g_uploads.erase(std::remove_if(g_uploads.begin(), g_uploads.end(), [&](const Upload& u) { return u.at <= done; }), g_uploads.end());
    return hipSuccess;
}
hipError_t hipGetDeviceCount(int* n) {
    *n = 1;
    return hipSuccess;
}
}
static void uploads_unchanged() {
    for (const Upload& u : g_uploads) CHECK(std::memcmp(u.from, u.was.data(), u.was.size()) == 0);
}

static std::vector<const char*> g_k, g_v;  // the rows of every append so far
namespace apar {
hipError_t launch_append_blocks(const Shape&, void*, const void* k, const void* v, const int32_t*, bool, int, int, int, hipStream_t) {
    g_k.push_back((const char*)k);
    g_v.push_back((const char*)v);
    return hipGetLastError();
}
hipError_t launch_read_rows(const Shape&, const void*, const int32_t*, int, void*, void*, hipStream_t) { return hipGetLastError(); }
static hipError_t g_rotation = hipSuccess;  // what the next launches give
static int g_rotations = 0;
hipError_t launch_rotate_rows(const RotaryArgs&, RotaryCall, bool, hipStream_t) {
    g_rotations += g_rotation == hipSuccess;
    return g_rotation;
}
}  // namespace apar

// Requests admitted by one call take their prompts' rows one after the other, and a row is n_kv * 128 elements as the caller has
// them, whatever the pool makes of it.
static void admission() {
    for (int dtype : {APAR_F32, APAR_BF16, APAR_BF16_FP8KV, APAR_BF16_FP4KV})
        for (int n_kv : {1, 2, 8}) {
            apar_pool* p;
            CHECK(create(2 * n_kv, n_kv, dtype, 400, &p) == APAR_OK);
            apar_server_config cfg{};
            cfg.max_running = 8;
            apar_server* s;
            CHECK(apar_server_create(p, &cfg, &s) == APAR_OK);
            const int lens[] = {5, 16, 1, 33, 100};
            std::vector<int32_t> prompt(100, 7);
            for (int n : lens) CHECK(apar_server_submit(s, n, prompt.data(), n) == APAR_OK);
            g_k.clear(), g_v.clear();
            static char rows[2];  // (nothing reads there)
            int32_t admitted = 0;
            int64_t used = 0;
            CHECK(apar_server_admit(s, rows, rows + 1, 1000, nullptr, &admitted, &used) == APAR_OK && admitted == 5 && used == 155);
            CHECK(g_k.size() == 5 && g_v.size() == 5);
            int64_t at = 0;
            for (int i = 0; i < 5; ++i) {
                const int64_t bytes = at * n_kv * 128 * (dtype == APAR_F32 ? 4 : 2);
                CHECK(g_k[i] == rows + bytes && g_v[i] == rows + 1 + bytes);
                at += lens[i];
            }
            CHECK(apar_server_destroy(s) == APAR_OK && apar_pool_destroy(p) == APAR_OK);
        }
}

// Calls whose tables are uploaded and that are refused or cannot launch: nothing that the upload reads is written while it may be under way.
static void failures() {
    apar_pool* p;
    CHECK(create(4, 2, APAR_BF16, 2000, &p) == APAR_OK);
    std::vector<apar_thread> ids;
    for (int i = 0; i < 1500; ++i) ids.push_back(thread_of(p, 1 + i % 16));
    apar_rotary_config cfg{};
    cfg.head_dim = cfg.rotary_dim = 128;
    cfg.base = 10000.0, cfg.magnitude = 1.0;
    apar_rotary* r;
    CHECK(apar_rotary_create(&cfg, &r) == APAR_OK);
    apar_rotary_rows q{}, k{}, odd{}, many{};
    q.in_dev = q.out_dev = kRows, q.in_stride = q.out_stride = 4 * 128, q.n_heads = 4;
    k.in_dev = k.out_dev = kRows, k.in_stride = k.out_stride = 2 * 128, k.n_heads = 2;
    odd = q;
    odd.in_dev = odd.out_dev = g_kv + 1;
    auto rotate = [&](int first, const apar_rotary_rows& x) {
        return apar_rotate_threads(p, r, APAR_BF16, ids.data() + first, nullptr, 1000, APAR_ROWS_NEXT, nullptr, 0, &x, &k, 0, nullptr);
    };
    g_uploads.clear();
    for (int i = 0; i < 3; ++i) {
        const size_t under_way = g_uploads.size();
        CHECK(rotate(i, odd) == APAR_ERR_INVALID_ARG);
        CHECK(g_uploads.size() == under_way);  // (refused before anything is enqueued)
        apar::g_rotation = hipErrorInvalidValue;
        CHECK(rotate(i + 1, q) == APAR_ERR_HIP);
        apar::g_rotation = hipSuccess;
        for (int next = 0; next < 20; ++next) {
            CHECK(rotate(next * 20, q) == APAR_OK);
            uploads_unchanged();
        }
    }
    CHECK(apar::g_rotations == 60);
    CHECK(apar_rotary_destroy(r) == APAR_OK && apar_pool_destroy(p) == APAR_OK);
}

// The same of the pool's own calls, each with tables that are uploaded.
static void failed_launches() {
    for (int dtype : {APAR_F32, APAR_BF16, APAR_BF16_FP4KV})
        for (int kind = 0; kind < 5; ++kind) {
            apar_pool* p;
            CHECK(create(4, 2, dtype, 20000, &p) == APAR_OK);
            std::vector<apar_thread> ids;
            for (int i = 0; i < 700; ++i) ids.push_back(thread_of(p, 100 + i % 16));
            const apar_thread big = thread_of(p, 20000);
            const std::vector<int32_t> ones(700, 1), pieces(700, 90);
            auto call = [&](int n) -> int {
                switch (kind) {
                    case 0: return apar_append_kv_batch(p, ids.data(), n, kRows, kRows, nullptr);
                    case 1: return apar_read_kv_rows(p, big, 0, 17000 + n, kRows, kRows, nullptr);
                    case 2: return apar_decode_attention(p, kRows, ids.data(), n, kRows, nullptr);
                    case 3: return apar_prefill_attention(p, kRows, ids.data(), ones.data(), n, kRows, nullptr);
                    default: return apar_prefill_attention(p, kRows, ids.data(), pieces.data(), n, kRows, nullptr);
                }
            };
            CHECK(apar_set_plan_reuse(p, 0) == APAR_OK);
            g_uploads.clear();
            for (int i = 0; i < 3; ++i) {
                const long before = g_enqueued;
                g_last = hipErrorInvalidValue;
                CHECK(call(690 - i) == APAR_ERR_HIP && g_last == hipSuccess);
                CHECK(g_enqueued > before);  // (the case is one that uploads)
                for (int next = 0; next < 12; ++next) {
                    CHECK(call(500 + next * 10) == APAR_OK);
                    uploads_unchanged();
                }
            }
            CHECK(apar_pool_destroy(p) == APAR_OK);
        }
}

// Reads past a thread's rows are refused, however far past.
static void reads() {
    for (int dtype : {APAR_F32, APAR_BF16, APAR_BF16_FP8KV, APAR_BF16_FP4KV}) {
        apar_pool* p;
        CHECK(create(4, 2, dtype, 2000, &p) == APAR_OK);
        const apar_thread t = thread_of(p, 100);
        struct { int64_t first; int n, status; } const calls[] = {
            {0, 100, APAR_OK}, {99, 1, APAR_OK}, {100, 0, APAR_OK}, {0, 101, APAR_ERR_INVALID_ARG}, {100, 1, APAR_ERR_INVALID_ARG},
            {INT64_MAX, 1, APAR_ERR_INVALID_ARG}, {INT64_MAX - 5, 100, APAR_ERR_INVALID_ARG}, {INT64_MAX, INT32_MAX, APAR_ERR_INVALID_ARG},
            {INT64_MAX, 0, APAR_ERR_INVALID_ARG}, {-1, 1, APAR_ERR_INVALID_ARG}, {0, -1, APAR_ERR_INVALID_ARG}};
        for (const auto& c : calls) CHECK(apar_read_kv_rows(p, t, c.first, c.n, kRows, kRows, nullptr) == c.status);
        CHECK(apar_pool_destroy(p) == APAR_OK);
    }
}

int main(int argc, char** argv) {
    const std::map<std::string, void (*)()> checks = {{"admission", admission}, {"failures", failures}, {"reads", reads}, {"failed_launches", failed_launches}};
    CHECK(argc == 2 && checks.count(argv[1]));
    checks.at(argv[1])();
    std::printf("ok: %s\n", argv[1]);
    return 0;
}
