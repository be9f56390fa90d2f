// What calls hand on to the kernels, against the runtime of host_pool.cpp.  Built and run by tests/test_host_calls.py, which names the
// check to run.
#include "apar_internal.hpp"

#define main host_pool_main
#define launch_append_blocks append_nothing
#include "host_pool.cpp"
#undef main
#undef launch_append_blocks

static std::vector<const char*> g_k, g_v;  // the rows of every append so far
namespace apar {
hipError_t launch_append_blocks(const Shape&, void*, const void* k, const void* v, const int32_t*, bool, int, int, int, hipStream_t) {
    g_k.push_back((const char*)k);
    g_v.push_back((const char*)v);
    return hipGetLastError();
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

int main(int argc, char** argv) {
    const std::map<std::string, void (*)()> checks = {{"admission", admission}};
    CHECK(argc == 2 && checks.count(argv[1]));
    checks.at(argv[1])();
    std::printf("ok: %s\n", argv[1]);
    return 0;
}
