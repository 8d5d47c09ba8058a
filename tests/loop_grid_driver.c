// Grids and scratch memory of the attention over shared prefixes against stand-ins for HIP (lds_limit_driver.c's): whatever the host
// bounds, every launch has work-groups and fewer than 2^32 threads a dimension, and a bound beyond the table is the table's.
#define main linears_main
#define hipLaunchKernel seen_by_limits
#include "lds_limit_driver.c"
#undef hipLaunchKernel
#undef main

static int calls, bad;
static uint64_t grids;

int hipLaunchKernel(const void *kernel, dim3_t grid, dim3_t block, void **args, size_t lds, void *stream)
{
    const uint64_t x = (uint64_t)grid.x * block.x, y = (uint64_t)grid.y * block.y, z = (uint64_t)grid.z * block.z;
    if (x == 0 || y == 0 || z == 0 || x >> 32 || y >> 32 || z >> 32) ++bad;
    grids = grids * 1000003 + x * 7919 + y * 31 + z;
    return seen_by_limits(kernel, grid, block, args, lds, stream);
}

static int64_t smaller(int64_t a, int64_t b) { return a < b ? a : b; }

int main(int argc, char **argv)
{
    void *lib = argc > 1 ? dlopen(argv[1], RTLD_NOW | RTLD_LOCAL) : NULL;
    if (!lib) { printf("%s\n", dlerror()); return 2; }
    LOAD(mquant_paged_attention_shared); LOAD(mquant_paged_attention_shared_workspace_bytes);
    LOAD(mquant_step_plan); LOAD(mquant_sample); LOAD(mquant_sample_workspace_bytes);
    void *P = (void *)0x10000, *Q = (void *)0x20000;
    const int32_t seqs[] = {1, 2, 31, 200, 2000}, rows[] = {1, 2, 5, 13, 100, 700}, tables[] = {1, 513, 16777216}, groups[] = {0, 1, 3, 200, 3000},
                  bounds[] = {0, 1, 129, 8200, 131072, 0x40000000, 0x7fffff81, 0x7fffffff};
    int failed = 0;
    for (int h = 0; h < 3; ++h)
        for (int s = 0; s < 5; ++s)
            for (int r = 0; r < 6; ++r)
                for (int t = 0; t < 3; ++t)
                    for (int g = 0; g < 5; ++g)
                        for (int b = 0; b < 64; ++b)
                            for (int known = 0; known < 2; ++known) {
                                const int32_t n_kv = h == 0 ? 1 : h == 1 ? 4 : 8, n_q = n_kv * (h == 1 ? 7 : 8), T = seqs[s] * rows[r];
                                const int32_t max_rows = known ? rows[r] : 0, slots = tables[t] * 64, asked[2] = {bounds[b % 8], bounds[b / 8]};
                                const mquant_paged_cache_t c = {P, P, P, seqs[s], 100, 64, tables[t], n_kv, 128};
                                int32_t held[2];
                                int64_t need, wide;
                                for (int i = 0; i < 2; ++i) held[i] = asked[i] > 0 ? (int32_t)smaller(asked[i], slots) : slots;
                                need = mquant_paged_attention_shared_workspace_bytes_(T, seqs[s], groups[g], n_q, n_kv, 128, max_rows, held[0], held[1]);
                                wide = mquant_paged_attention_shared_workspace_bytes_(T, seqs[s], groups[g], n_q, n_kv, 128, max_rows, asked[0] ? asked[0] : slots,
                                                                                      asked[1] ? asked[1] : slots);
                                uint64_t by[2] = {0, 0};
                                for (int own = 0; own < 2; ++own, ++calls) {                 // the caller's bounds, then those that hold
                                    const int32_t *with = own ? held : asked;
                                    grids = 0;
                                    failed += mquant_paged_attention_shared_(P, n_q * 128, &c, P, P, P, P, groups[g], Q, n_q * 128, T, n_q, max_rows, with[0], with[1],
                                                                             P, need, NULL) != MQUANT_OK;
                                    by[own] = grids;
                                }
                                failed += by[0] != by[1];
                                // scratch asked for with the caller's own bounds does, too
                                failed += mquant_paged_attention_shared_(P, n_q * 128, &c, P, P, P, P, groups[g], Q, n_q * 128, T, n_q, max_rows, asked[0], asked[1], P,
                                                                         wide, NULL) != MQUANT_OK;
                            }
    const int32_t counts[] = {0, 1, 255, 256, 4096, 4097, 1 << 20, 0x7fffff00, 0x7fffffff};
    for (int i = 0; i < 9; ++i) {
        failed += mquant_step_plan_(P, P, P, P, 5, P, 9, 64, P, 1000, P, P, P, P, P, P, counts[i], NULL) != MQUANT_OK;
        for (int V = 1; V <= 1 << 20; V = V * 4 + (V == 1)) {
            if (counts[i] == 0 || V > 1 << 20) continue;
            const int64_t need = mquant_sample_workspace_bytes_(counts[i], V);
            const int st = mquant_sample_(P, MQUANT_F32, V, P, P, P, P, P, P, P, counts[i], V, P, need, NULL);
            failed += st != MQUANT_OK && !(st == MQUANT_ERR_UNSUPPORTED && counts[i] >= 1 << 14);
        }
    }
    printf("%d calls, %d launches, %d of them bad, %d failed\n", calls, launches, bad, failed);
    return calls && launches >= calls && !bad && !failed ? 0 : 1;
}
