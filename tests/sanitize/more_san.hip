// Host-side self-test of shared prefixes, pages and log-probabilities, built with -fsanitize=address,undefined (tests/test_more_build.py): plans and sizes swept over their
// ranges against what the kernels assume, and refusals with extreme arguments.  No GPU.
#include <climits>
#include <cstdio>
#include <cstring>

#include "../../include/sssd_ops.h"
#include "../../paper_2411_05894_amd/csrc/kv8.h"

static int failures = 0;
#define CHECK(cond)                                                                  \
    do {                                                                             \
        if (!(cond)) {                                                               \
            std::fprintf(stderr, "CHECK failed at line %d: %s\n", __LINE__, #cond);  \
            ++failures;                                                              \
        }                                                                            \
    } while (0)

static void shared_plans()
{
    for (int nkv : {1, 2, 3, 8, 16})
        for (int gq : {1, 3, 4, 8, 64})
            for (int B = 1; B <= 400; B += B < 20 ? 1 : 37)
                for (int n : {1, 2, 5, 9, 17, 32})
                    for (int blocks : {1, 5, 64, 1000, 40000})
                        for (int groups : {0, 1, 2, 3, 17, 400})
                            for (bool f32 : {false, true}) {
                                if (groups > B) continue;
                                const Kv8SharedPlan p = kv8_shared_plan(B, n, gq, nkv, blocks, groups, f32);
                                const Kv8Plan rest = kv8_plan(B, n, gq, nkv, blocks, f32);
                                CHECK(p.rt >= 1 && p.rt <= 2 && (p.wave_rows == 1 || p.wave_rows == 4) && p.share >= 1 && p.share <= 64);
                                CHECK(!(f32 && p.wave_rows == 4 && p.rt == 2));
                                CHECK(p.segments == p.share * 4 / p.wave_rows);
                                // partial results lie within the workspace, whatever the other calls that it serves are
                                const size_t rows = (size_t)B * n * gq * nkv;
                                CHECK((p.segments + rest.share) * rows * (128 * sizeof(float) + 16) <= kv8_shared_ws(B, n, gq, nkv, 128));
                                CHECK((p.segments + rest.share) * rows * (64 * sizeof(float) + 16) <= kv8_shared_ws(B, n, gq, nkv, 64));
                                // there is a workgroup for every tile of rows, however they are grouped: all in one, one large and many small ones
                                const int per = p.wave_rows * p.rt * 16, each = n * gq;
                                auto tiles = [&](int m) { return ((int64_t)m * each + per - 1) / per; };
                                if (groups == 1) CHECK(p.tiles >= tiles(B));
                                if (groups > 1) CHECK(p.tiles >= tiles(B - groups + 1) + (groups - 1) * tiles(1) && p.tiles >= (groups - B % groups) * tiles(B / groups) + B % groups * tiles(B / groups + 1));
                            }
    CHECK(kv8_shared_ws(3, 5, 4, 8, 128) <= kv8_shared_ws(4, 5, 4, 8, 128) && kv8_shared_ws(3, 5, 4, 8, 128) <= kv8_shared_ws(3, 6, 4, 8, 128));
}

static void sizes()
{
    size_t bytes = 0;
    sssd_kv8_config c{SSSD_KV8_E4M3, 80, 64, 8, 128, 64, 131072, 0};
    CHECK(sssd_kv8_pages_sizes(&c, &bytes) == SSSD_OK && bytes > 0);
    c.max_batch = INT_MAX;
    c.max_seq = INT_MAX - 64;
    c.n_pages = 1;
    const int rc = sssd_kv8_pages_sizes(&c, &bytes);
    CHECK(rc == SSSD_OK || rc == SSSD_EINVAL);
    CHECK(sssd_kv8_shared_sizes(&c, INT_MAX, 32, &bytes) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_shared_sizes(&c, INT_MIN, 32, &bytes) == SSSD_EINVAL && sssd_kv8_shared_sizes(&c, 1, INT_MAX, &bytes) == SSSD_ECAPACITY);
    for (int type : {0, 1})
        for (int rows : {1, 9, 1023, 1024, 100000, INT_MAX})
            for (int vocab : {1, 7, 2048, 2049, 128256, INT_MAX})
                for (int top : {0, 1, 64}) {
                    if (top > vocab) continue;
                    const size_t n = sssd_op_logprobs_scratch_bytes(type, rows, vocab, 32, top);
                    CHECK(rows >= 1024 || vocab <= 2048 || vocab > 1 << 30 ? n == 0 : n > 0);
                }
}

static void refusals()
{
    sssd_kv8_config c{SSSD_KV8_INT8, 1, 8, 2, 64, 4, 100, 0};
    size_t cache = 0, ws = 0, pages_ws = 0, shared_ws = 0;
    sssd_kv8_sizes(&c, &cache, &ws, nullptr, nullptr);
    sssd_kv8_pages_sizes(&c, &pages_ws);
    sssd_kv8_shared_sizes(&c, 4, 32, &shared_ws);
    int32_t *fake = (int32_t *)(uintptr_t)(1 << 20);
    sssd_kv8 kv{c, fake, cache, fake, ws, fake, fake, 0};
    sssd_kv8_pages p{fake, fake, fake, pages_ws};
    CHECK(sssd_kv8_reserve(&kv, &p, INT_MAX, INT_MAX, INT_MAX, fake, fake, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_reserve(&kv, &p, INT_MIN, 1, 1, fake, fake, nullptr) == SSSD_EINVAL);
    CHECK(sssd_kv8_fork(&kv, &p, nullptr, fake, nullptr) == SSSD_EINVAL);
    CHECK(sssd_kv8_compact(&kv, &p, &kv, &p, nullptr, nullptr, nullptr) == SSSD_EINVAL);
    p.ws_bytes = 0;
    CHECK(sssd_kv8_compact(&kv, &p, nullptr, nullptr, nullptr, nullptr, nullptr) == SSSD_ECAPACITY);
    sssd_rows r{fake, SSSD_F32, LLONG_MAX, LLONG_MIN, LLONG_MAX};
    CHECK(sssd_kv8_attention_shared(&kv, 0, INT_MAX, 1, &r, &r, fake, nullptr, nullptr, 1, fake, fake, fake, shared_ws, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_attention_shared(&kv, 0, 1, 1, &r, &r, fake, nullptr, nullptr, INT_MAX, fake, fake, fake, shared_ws, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_attention_shared(&kv, 0, 1, 1, &r, &r, fake, nullptr, nullptr, INT_MIN, fake, fake, fake, shared_ws, nullptr) == SSSD_EINVAL);
    CHECK(sssd_op_logprobs(fake, 0, INT_MAX, INT_MAX, LLONG_MAX, 1.f, nullptr, 0, nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, 0, nullptr) == SSSD_ECAPACITY);
}

int main()
{
    shared_plans();
    sizes();
    refusals();
    if (failures) return 1;
    std::printf("host self-test passed\n");
    return 0;
}
