// Grids and scratch memory of the serving entries against stand-ins for HIP (lds_limit_driver.c's): whatever the host bounds, every launch
// has work-groups and fewer than 2^32 threads a dimension, and a bound beyond the table is the table's.
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
    LOAD(mquant_paged_attention); LOAD(mquant_paged_attention_workspace_bytes);
    void *P = (void *)0x10000, *Q = (void *)0x20000;
    const int32_t seqs[] = {1, 2, 3, 31, 128, 200, 256, 2000}, rows[] = {1, 2, 5, 13, 100, 700}, tables[] = {1, 513, 3000, 33554431},
                  bounds[] = {0, 1, 129, 1281, 8192, 8200, 131072, 0x40000000, 0x7fffff7f, 0x7fffff80, 0x7fffff81, 0x7fffffff};
    int failed = 0;
    for (int h = 0; h < 3; ++h)
        for (int s = 0; s < 8; ++s)
            for (int r = 0; r < 6; ++r)
                for (int t = 0; t < 4; ++t)
                    for (int b = 0; b < 12; ++b)
                        for (int known = 0; known < 2; ++known) {
                            const int32_t n_kv = h == 0 ? 1 : h == 1 ? 4 : 8, n_q = n_kv * (h == 1 ? 7 : 8), T = seqs[s] * rows[r];
                            const int32_t max_rows = known ? rows[r] : 0, slots = tables[t] * 64;
                            const mquant_paged_cache_t c = {P, P, P, seqs[s], 100, 64, tables[t], n_kv, 128};
                            const int32_t bound = bounds[b] > 0 ? (int32_t)smaller(bounds[b], slots) : slots;
                            const int64_t need = mquant_paged_attention_workspace_bytes_(T, seqs[s], n_q, n_kv, 128, max_rows, bound);
                            const int64_t wide = mquant_paged_attention_workspace_bytes_(T, seqs[s], n_q, n_kv, 128, max_rows, bounds[b] > 0 ? bounds[b] : slots);
                            uint64_t by[2] = {0, 0};
                            for (int own = 0; own < 2; ++own, ++calls) {                     // the caller's bound, then the one that holds
                                grids = 0;
                                failed += mquant_paged_attention_(P, n_q * 128, &c, P, P, Q, n_q * 128, T, n_q, max_rows, own ? bound : bounds[b], P, need, NULL) !=
                                          MQUANT_OK;
                                by[own] = grids;
                            }
                            failed += by[0] != by[1];
                            // scratch asked for with the caller's own bound does, too
                            failed += mquant_paged_attention_(P, n_q * 128, &c, P, P, Q, n_q * 128, T, n_q, max_rows, bounds[b], P, wide, NULL) != MQUANT_OK;
                        }
    printf("%d calls, %d launches, %d of them bad, %d failed\n", calls, launches, bad, failed);
    return calls && launches >= calls && !bad && !failed ? 0 : 1;
}
