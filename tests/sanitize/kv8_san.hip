// Host-side self-test of the 8-bit cache, built with -fsanitize=address,undefined (tests/test_kv8_build.py): sizes, frequencies, the plans of attention
// and of rotations swept over their ranges against what their kernels assume, and refusals with extreme arguments.  No GPU.
#include <climits>
#include <cstdio>
#include <cstring>
#include <vector>

#include "../../paper_2411_05894_amd/csrc/kv8.h"

static int failures = 0;
#define CHECK(cond)                                                                  \
    do {                                                                             \
        if (!(cond)) {                                                               \
            std::fprintf(stderr, "CHECK failed at line %d: %s\n", __LINE__, #cond);  \
            ++failures;                                                              \
        }                                                                            \
    } while (0)

static void attention_plans()
{
    const size_t ws = kv8_attention_ws(128);
    for (int nkv = 1; nkv <= 16; ++nkv)
        for (int gq : {1, 2, 3, 4, 7, 8, 16, 64})
            for (int B = 1; B <= 300; B += B < 40 ? 1 : 13)
                for (int n = 1; n <= 32; ++n)
                    for (int blocks : {1, 40, 200, 1000, 40000})
                        for (bool f32 : {false, true}) {
                            const Kv8Plan p = kv8_plan(B, n, gq, nkv, blocks, f32);
                            const int tiles = (n * gq + 15) / 16, rt = (tiles + p.passes - 1) / p.passes;
                            CHECK(p.passes >= 1 && rt >= 1 && rt <= KV8_MAX_TILES && p.share >= 1 && p.share <= 64);
                            // partial results lie within the workspace
                            if (p.share > 1) CHECK((size_t)B * nkv * p.share * tiles * 16 * (128 * 4 + 8) + HAND_WORDS <= ws);
                            // groups have a word each, and no workgroup of a group waits for more than what is resident
                            if (p.share > 1 && p.in_die) CHECK(B * nkv * p.passes <= HAND_GROUPS && B * nkv % 8 == 0 && p.share <= 32 && B * nkv * p.passes * p.share <= 512);
                        }
}

static void rotations()
{
    for (int d = 2; d <= 1200; d += d < 140 ? 1 : 97)
        for (int r = 2; r <= d && r <= 1024; r += 2)
            for (int neighbours = 0; neighbours < 2; ++neighbours)
                for (int total : {1, 9, 4095, 100000}) {
                    const int heads = d % 7 * 9 + 1;
                    const RopeWork w = rope_work(1, total, d, heads, r, neighbours, 256, total % 2 ? 1 : 4);
                    CHECK(w.rows >= 1 && w.rows <= (uint32_t)ROPE_ROWS && w.rows * (r / 2) <= (uint32_t)ROPE_TABLE && w.per >= 1 && w.per <= heads);
                    const int turning = neighbours ? r : r / 2;
                    CHECK(turning % w.unit == 0 && (int)w.units == turning / w.unit + (d - r + w.unit - 1) / w.unit);
                    CHECK(w.unit != 1 || !neighbours);
                    CHECK((uint64_t)w.per * w.units * w.units < (uint64_t)1 << 32);      // the quotient by units is exact
                    CHECK(w.unit < 8 || (r % 8 == 0 && (d - r) % 8 == 0));
                }
    const RopeWork w = rope_work(1, 5, 8192, 65535, 2, 0, 256, 1);
    CHECK(w.per >= 1 && (uint64_t)w.per * w.units * w.units < (uint64_t)1 << 32);
}

static void sizes_and_frequencies()
{
    size_t bytes = 0, ws = 0;
    int32_t per = 0, pages = 0;
    for (int heads : {1, 8, 64})
        for (int seq : {1, 31, 32, 33, 1 << 20, INT_MAX - 64, INT_MAX})
            for (int batch : {1, 7, 1 << 12, INT_MAX})
                for (int n_pages : {0, 1, INT_MAX})
                    for (int layers : {1, 80, INT_MAX}) {
                        const sssd_kv8_config c{SSSD_KV8_INT8, layers, heads, heads, 128, batch, seq, n_pages};
                        const int rc = sssd_kv8_sizes(&c, &bytes, &ws, &per, &pages);
                        CHECK(rc == SSSD_OK || rc == SSSD_EINVAL);
                        if (rc == SSSD_OK) CHECK(per == (seq + 31) / 32 && pages > 0 && bytes / layers / pages / heads >= 64 * 128 + 8);
                    }
    std::vector<double> turns(512);
    for (int r = 2; r <= 1024; r += 2)
        for (int scaling = 0; scaling < 3; ++scaling) {
            const sssd_rope_config c{r, 500000.f, scaling, 8.f, 1.f, 4.f, 8192};
            turns.assign(r / 2, 0);
            turns.shrink_to_fit();
            CHECK(sssd_rope_frequencies(&c, turns.data()) == SSSD_OK);
            for (double t : turns) CHECK(t > 0 && t < 0.16);
        }
}

static void refusals()
{
    alignas(256) static char room[1024];
    const sssd_kv8_config c{SSSD_KV8_E4M3, 1, 8, 8, 128, 1 << 20, 1 << 20, 1};
    size_t bytes, ws;
    CHECK(sssd_kv8_sizes(&c, &bytes, &ws, nullptr, nullptr) == SSSD_OK);
    sssd_kv8 kv{c, room, bytes, room, ws, (const int32_t *)room, (int32_t *)room, 0};
    sssd_rows r{room, SSSD_F32, LLONG_MAX, LLONG_MIN, LLONG_MAX};
    const sssd_rope rope{(const double *)room, 128, 0, 1.f};
    const int32_t *ints = (const int32_t *)room;
    CHECK(sssd_kv8_append(&kv, 0, 0, 1 << 20, 1 << 20, &r, &r, ints, nullptr, &rope, nullptr, &r, &r, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_append(&kv, 0, INT_MAX, INT_MAX, INT_MAX, &r, &r, ints, ints, nullptr, nullptr, nullptr, nullptr, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_read(&kv, 0, 0, 1 << 20, INT_MAX, nullptr, ints, &r, &r, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_attention(&kv, 0, 1 << 20, 32, &r, &r, ints, nullptr, nullptr, INT_MAX, INT_MAX, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_kv8_commit_tree(&kv, 1 << 20, 32, (int32_t *)room, ints, ints, nullptr) == SSSD_ECAPACITY);
    CHECK(sssd_op_rope(&r, &r, INT_MAX, INT_MAX, 65535, 8192, ints, &rope, nullptr) == SSSD_ECAPACITY);
    kv.flags = 4;
    CHECK(sssd_kv8_read(&kv, 0, 0, 1, 1, nullptr, nullptr, &r, &r, nullptr) == SSSD_EINVAL);
}

int main()
{
    attention_plans();
    rotations();
    sizes_and_frequencies();
    refusals();
    if (failures) return 1;
    std::puts("host self-test passed");
    return 0;
}
