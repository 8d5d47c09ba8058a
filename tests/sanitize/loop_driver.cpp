// Host side of the serving loop's entries under AddressSanitizer + UndefinedBehaviorSanitizer: validation and the sizes of plans and
// workspaces from the smallest to the largest arguments.  Nothing is launched: every call with device work is one that validation
// turns down, and the descriptors are exactly sized heap blocks.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "mquant.h"

#define CHECK(c) do { if (!(c)) { fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); exit(1); } } while (0)

int main()
{
    void *P = reinterpret_cast<void *>(0x10000), *Q = reinterpret_cast<void *>(0x20000);
    int32_t *I = static_cast<int32_t *>(P);
    float *F = static_cast<float *>(P);
    const int32_t sizes[] = {0, 1, 2, 3, 17, 64, 129, 1000, 4097, 100000, 1 << 20, INT_MAX - 1, INT_MAX};
    for (int32_t T : sizes)
        for (int32_t n_seq : sizes)
            for (int32_t n_groups : sizes)
                for (int32_t max_rows : {0, 1, 2, 100, INT_MAX})
                    for (int32_t prefix : sizes)
                        for (int32_t suffix : {0, 1, 100, 1 << 20, INT_MAX})
                            for (int32_t kv_heads : {1, 8}) {
                                const int64_t n = mquant_paged_attention_shared_workspace_bytes(T, n_seq, n_groups, kv_heads * 7, kv_heads, 128, max_rows,
                                                                                                prefix, suffix);
                                CHECK(n >= 0 || n == MQUANT_ERR_UNSUPPORTED);
                                CHECK(n % 256 == 0 || n < 0);
                            }
    CHECK(mquant_paged_attention_shared_workspace_bytes(INT_MIN, 1, 1, 1, 1, 128, 0, 0, 0) == MQUANT_ERR_BAD_SHAPE);
    for (int32_t rows : sizes)
        for (int32_t V : sizes) {
            const int64_t n = mquant_sample_workspace_bytes(rows, V);
            CHECK(V < 1 ? n == MQUANT_ERR_BAD_SHAPE : V > 1 << 20 ? n == MQUANT_ERR_UNSUPPORTED : n >= 0 && n % 256 == 0);
            const int st = mquant_sample(nullptr, MQUANT_F16, INT64_MAX, F, I, F, F, F, I, F, rows, V, P, INT64_MAX, nullptr);
            CHECK(st == (n < 0 ? n : rows == 0 ? MQUANT_OK : MQUANT_ERR_NULL) || (n >= 0 && st == MQUANT_ERR_UNSUPPORTED));
        }
    for (int32_t page : {0, 1, 8, 16, 24, 64, 4096, 8192, INT_MIN, INT_MAX})
        for (int32_t pages : sizes)
            for (int32_t table : sizes) {
                auto *c = static_cast<mquant_paged_cache_t *>(malloc(sizeof(mquant_paged_cache_t)));
                auto *r = static_cast<mquant_rotary_t *>(malloc(sizeof(mquant_rotary_t)));
                *c = {P, P, I, 3, pages, page, table, 4, 128};
                CHECK(mquant_rotary_init(r, MQUANT_ROTARY_HALVES, 128, 1e4, MQUANT_ROTARY_TURNS, 8.0, 4096.0, 1.0, 32.0) == MQUANT_OK);
                const int st = mquant_paged_attention_shared(nullptr, 3584, c, I, I, I, I, 2, Q, 3584, 9, 28, 0, 0, 0, P, 0, nullptr);
                CHECK(st == MQUANT_ERR_NULL || st == MQUANT_ERR_UNSUPPORTED || st == MQUANT_ERR_BAD_SHAPE);
                CHECK(mquant_rotary_append(P, 3584, Q, 3584, P, 512, nullptr, 512, nullptr, nullptr, 1e-6f, I, I, nullptr, 9, 28, r, c, nullptr) == st);
                const int plan = mquant_step_plan(I, I, I, I, 3, I, table, page, I, pages, I, I, I, I, nullptr, nullptr, 9, nullptr);
                CHECK(plan == MQUANT_ERR_NULL || plan == MQUANT_ERR_UNSUPPORTED || plan == MQUANT_ERR_BAD_SHAPE);
                free(r);
                free(c);
            }
    // sums and products of counts at their ends
    for (int32_t a : {INT_MIN, -1, 0, 1, 64, INT_MAX})
        for (int32_t b : {INT_MIN, -1, 0, 1, 64, INT_MAX})
            for (int32_t axes : {INT_MIN, 0, 1, 2, 3, 4, INT_MAX})
                for (int32_t dim : {INT_MIN, 0, 16, 128, 144, INT_MAX}) {
                    auto *r = static_cast<mquant_rotary_t *>(malloc(sizeof(mquant_rotary_t)));
                    CHECK(mquant_rotary_init(r, MQUANT_ROTARY_INTERLEAVED, 128, 1e4, MQUANT_ROTARY_BASE, 1e3, 0, 0, 0) == MQUANT_OK);
                    r->section[0] = a;
                    r->section[1] = r->section[2] = b;
                    r->n_axes = axes;
                    r->rot_dim = dim;
                    const int st = mquant_rotary_apply(P, 3584, Q, 3584, P, 512, Q, 512, P, P, 1e-6f, nullptr, 4, 28, 4, 128, r, nullptr);
                    CHECK(st == MQUANT_ERR_NULL || st == MQUANT_ERR_UNSUPPORTED || st == MQUANT_ERR_BAD_SHAPE);
                    free(r);
                }
    mquant_rotary_t r;
    for (double base : {0.0, 1.0, 1.0000001, 1e308, static_cast<double>(INFINITY), static_cast<double>(NAN)})
        for (double factor : {0.0, 1.0, 1e308, static_cast<double>(INFINITY), static_cast<double>(NAN)})
            for (double turns : {-1e308, 0.0, 1e-308, 1e308, static_cast<double>(NAN)})
                for (int scaling = -1; scaling < 5; ++scaling) {
                    const int st = mquant_rotary_init(&r, MQUANT_ROTARY_HALVES, 64, base, scaling, factor, 4096.0, 0.0, turns);
                    CHECK(st == MQUANT_OK || st == MQUANT_ERR_BAD_SHAPE);
                    for (int j = 0; st == MQUANT_OK && j < 32; ++j) CHECK(std::isfinite(r.freq[j]));
                }
    const mquant_paged_cache_t c = {P, P, I, 3, 10, 16, 10, 4, 128};
    CHECK(mquant_rotary_init(&r, MQUANT_ROTARY_HALVES, 64, 1e4, MQUANT_ROTARY_NONE, 1.0, 0, 0, 0) == MQUANT_OK);
    CHECK(mquant_paged_attention_shared(P, INT64_MAX, &c, I, I, I, I, INT_MAX, Q, INT64_MAX, INT_MAX, 28, 0, 0, 0, P, 0, nullptr) == MQUANT_ERR_UNSUPPORTED);
    CHECK(mquant_rotary_apply(P, INT64_MAX - 7, Q, INT64_MAX - 7, P, 512, Q, 512, P, P, 1e-6f, I, INT_MAX, INT_MAX, 4, 128, &r, nullptr) ==
          MQUANT_ERR_UNSUPPORTED);
    CHECK(mquant_step_plan(I, I, I, I, INT_MAX, I, INT_MAX, 4096, I, INT_MAX, I, I, I, I, I, nullptr, INT_MAX, nullptr) == MQUANT_ERR_UNSUPPORTED);
    printf("serving loop host sanitizer run ok\n");
    return 0;
}
