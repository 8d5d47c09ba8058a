// The dynamic LDS limits of the serving kernels on several devices: the stand-ins for HIP of lds_limit_driver.c and the
// calls that launch every kernel with more than 64 KiB.
#define main linears_main
#include "lds_limit_driver.c"
#undef main

int main(int argc, char **argv)
{
    void *lib = argc > 1 ? dlopen(argv[1], RTLD_NOW | RTLD_LOCAL) : NULL;
    if (!lib) { printf("%s\n", dlerror()); return 2; }
    LOAD(mquant_paged_attention); LOAD(mquant_lora_apply); LOAD(mquant_qk_norm_rope); LOAD(mquant_kv_append);
    void *P = (void *)0x10000, *Q = (void *)0x20000;
    for (dev_now = 0; dev_now < 3; ++dev_now)
        for (int rep = 0; rep < 2; ++rep) {
            const mquant_paged_cache_t c = {P, P, P, 2, 100, 64, 50, 4, 128};
            const int rows[] = {2, 10, 100, 2000};
            for (int i = 0; i < 4; ++i)
                CALL(mquant_paged_attention_(P, 3584, &c, P, P, Q, 3584, rows[i], 28, (rows[i] + 1) / 2, 3000, P, (int64_t)1 << 40, NULL));
            for (int rank = 8; rank <= 128; rank *= 2)
                for (int T = 4; T <= 4000; T *= 10)
                    CALL(mquant_lora_apply_(P, 3584, NULL, P, P, P, P, P, 4608, Q, 4608, T, 4608, 3584, rank, 3, P, (int64_t)1 << 40, NULL));
            CALL(mquant_kv_append_(P, 3584, Q, 3584, P, 512, P, 512, P, P, 1e-6f, P, P, NULL, 100, 28, 1e4, &c, NULL));
            CALL(mquant_qk_norm_rope_(P, 3584, Q, 3584, P, 512, Q, 512, P, P, 1e-6f, P, 100, 28, 4, 128, 1e4, NULL));
        }
    printf("%d launches, %d large, %d without a limit on their device\n", launches, large, missing);
    return launches && large && !missing ? 0 : 1;
}
