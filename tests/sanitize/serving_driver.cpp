// Host side of the serving entries under AddressSanitizer + UndefinedBehaviorSanitizer: validation and the sizes of plans and
// workspaces from the smallest to the largest arguments.  Nothing is launched: every call with device work is one that validation
// turns down, and the cache descriptors are exactly sized heap blocks.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "mquant.h"

#define CHECK(c) do { if (!(c)) { fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); exit(1); } } while (0)

int main()
{
    void *P = reinterpret_cast<void *>(0x10000), *Q = reinterpret_cast<void *>(0x20000);
    const int32_t *I = static_cast<const int32_t *>(P);
    const float *F = static_cast<const float *>(P);
    const int32_t sizes[] = {0, 1, 2, 3, 15, 16, 17, 64, 65, 127, 128, 129, 1000, 4097, 100000, 1 << 20, INT_MAX - 1, INT_MAX};
    for (int32_t T : sizes)
        for (int32_t n_seq : sizes)
            for (int32_t max_rows : sizes)
                for (int32_t max_kv : sizes)
                    for (int32_t kv_heads : {1, 4, 8}) {
                        const int64_t n = mquant_paged_attention_workspace_bytes(T, n_seq, kv_heads * 7, kv_heads, 128, max_rows, max_kv);
                        CHECK(n >= 0 || n == MQUANT_ERR_UNSUPPORTED);
                        CHECK(n % 256 == 0 || n < 0);
                    }
    for (int32_t T : sizes)
        for (int32_t K : {8, 64, 1000, 29568, 1 << 20, INT_MAX - 7})
            for (int32_t rank : {8, 24, 64, 128}) CHECK(mquant_lora_workspace_bytes(T, K, rank) >= (T > 0 ? int64_t{4} * T * rank : 0));
    CHECK(mquant_paged_attention_workspace_bytes(INT_MIN, 1, 1, 1, 128, 0, 0) == MQUANT_ERR_BAD_SHAPE);
    CHECK(mquant_lora_workspace_bytes(INT_MIN, 8, 8) == MQUANT_ERR_BAD_SHAPE && mquant_lora_workspace_bytes(1, INT_MIN, 8) == MQUANT_ERR_BAD_SHAPE);
    for (int32_t page : {0, 1, 8, 16, 24, 64, 4096, 8192, INT_MIN, INT_MAX})
        for (int32_t pages : sizes)
            for (int32_t table : sizes) {
                auto *c = static_cast<mquant_paged_cache_t *>(malloc(sizeof(mquant_paged_cache_t)));
                *c = {P, P, I, 3, pages, page, table, 4, 128};
                const int st = mquant_paged_attention(nullptr, 3584, c, I, I, Q, 3584, 9, 28, 0, 0, P, 0, nullptr);
                CHECK(st == MQUANT_ERR_NULL || st == MQUANT_ERR_UNSUPPORTED || st == MQUANT_ERR_BAD_SHAPE);
                const int ap = mquant_kv_append(P, 3584, Q, 3584, P, 512, nullptr, 512, nullptr, nullptr, 1e-6f, I, I, nullptr, 9, 28, 1e4, c, nullptr);
                CHECK(ap == st);
                free(c);
            }
    mquant_paged_cache_t c = {P, P, I, 3, 10, 16, 10, 4, 128};
    CHECK(mquant_paged_attention(P, INT64_MAX, &c, I, I, Q, INT64_MAX, INT_MAX, 28, 0, 0, P, 0, nullptr) == MQUANT_ERR_UNSUPPORTED);
    CHECK(mquant_paged_attention(P, 3584, &c, I, I, Q, 3584, 3, 28, 1, 160, nullptr, 0, nullptr) == MQUANT_ERR_WORKSPACE);
    CHECK(mquant_qk_norm_rope(P, 3584, Q, 3584, P, 512, Q, 512, P, P, 1e-6f, nullptr, 4, 28, 4, 128, 1e4, nullptr) == MQUANT_ERR_NULL);
    CHECK(mquant_qk_norm_rope(P, INT64_MAX - 7, Q, INT64_MAX - 7, P, 512, Q, 512, P, P, 1e-6f, I, INT_MAX, INT_MAX, 4, 128, 1e4, nullptr) == MQUANT_ERR_UNSUPPORTED);
    CHECK(mquant_kv_append(P, 3584, Q, 3584, P, 512, P, 512, nullptr, nullptr, -1.0f, I, I, nullptr, 9, 28, 1e4, &c, nullptr) == MQUANT_ERR_BAD_SHAPE);
    CHECK(mquant_lora_apply(P, 8, nullptr, I, P, P, F, P, INT_MAX, Q, INT_MAX, INT_MAX, INT_MAX, 8, 8, INT_MAX, P, INT64_MAX, nullptr) ==
          MQUANT_ERR_UNSUPPORTED);
    CHECK(mquant_lora_apply(P, 8, nullptr, I, P, P, F, P, 8, Q, 8, 4, 8, 8, 8, -1, P, 1 << 20, nullptr) == MQUANT_ERR_BAD_SHAPE);
    printf("serving host sanitizer run ok\n");
    return 0;
}
