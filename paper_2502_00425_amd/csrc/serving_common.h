// What the operators of the serving step share (qk_norm.hip, paged_attention.hip): the paged cache as the
// kernels see it, its checks, and the sequence a row belongs to.
#pragma once

#include <hip/hip_fp16.h>

#include "mquant_internal.h"

namespace mquant {

constexpr int kCacheHeadDim = 128;
constexpr int64_t kMaxThreads = 0xffffffffll;              // of a launch along one dimension

struct PagedCache {
    __half *k, *v;
    const int32_t *table;
    int32_t n_seq, n_pages, page_shift, table_pages, n_kv_heads;
    int64_t page_halves;                   // of one page: n_kv_heads * page_size * 128
};

// Shape and pointers of a cache descriptor.
static inline int check_cache(const mquant_paged_cache_t *c)
{
    if (!c) return MQUANT_ERR_NULL;
    if (c->n_seq < 0 || c->n_kv_heads < 1) return MQUANT_ERR_BAD_SHAPE;
    if (c->head_dim != kCacheHeadDim) return MQUANT_ERR_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0) return MQUANT_ERR_UNSUPPORTED;
    if (c->n_seq == 0) return MQUANT_OK;
    if (c->n_pages < 1 || c->table_pages < 1) return MQUANT_ERR_BAD_SHAPE;
    if (static_cast<int64_t>(c->table_pages) * c->page_size > 0x7fffffc0ll) return MQUANT_ERR_UNSUPPORTED;     // slots in 32 bits
    if (static_cast<int64_t>(c->n_pages) * c->n_kv_heads > 0xffffffffll / (c->page_size / 16)) return MQUANT_ERR_UNSUPPORTED;
    if (!c->k_pages_dev || !c->v_pages_dev || !c->page_table_dev) return MQUANT_ERR_NULL;
    if (!aligned_to(c->k_pages_dev, 16) || !aligned_to(c->v_pages_dev, 16) || !aligned_to(c->page_table_dev, 4))
        return MQUANT_ERR_ALIGNMENT;
    return MQUANT_OK;
}

static inline PagedCache cache_args(const mquant_paged_cache_t *c)
{
    return {static_cast<__half *>(c->k_pages_dev), static_cast<__half *>(c->v_pages_dev), c->page_table_dev, c->n_seq,
            c->n_pages, __builtin_ctz(static_cast<unsigned>(c->page_size)), c->table_pages, c->n_kv_heads,
            static_cast<int64_t>(c->n_kv_heads) * c->page_size * kCacheHeadDim};
}

// Over the 16 lanes of a row, all of which get the result: rotations by 8, 4, 2 and 1 inside the register file (through LDS, as
// general lane exchanges go, each of the four takes the latency of an LDS read).
template <typename F>
__device__ __forceinline__ int row16(int x, F f)
{
    x = f(x, __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(x, x, 0x124, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(x, x, 0x122, 0xf, 0xf, false));
    return f(x, __builtin_amdgcn_update_dpp(x, x, 0x121, 0xf, 0xf, false));
}

__device__ __forceinline__ float row16_sum(float x)
{
    return __int_as_float(row16(__float_as_int(x), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}
__device__ __forceinline__ int32_t row16_max(int32_t x) { return row16(x, [](int a, int b) { return a > b ? a : b; }); }
__device__ __forceinline__ int32_t row16_min(int32_t x) { return row16(x, [](int a, int b) { return a < b ? a : b; }); }

// Sequence of row i: the number of sequences that start at or before it, less one; -1 for a row of none.  A wave looks at
// 64 starts at a time (row_start does not decrease).
__device__ __forceinline__ int32_t sequence_of_row(const int32_t *__restrict__ row_start, int32_t n_seq, int32_t i)
{
    const int lane = threadIdx.x & 63;
    int32_t n = 0;
    for (int32_t at = 0; at <= n_seq; at += 64) {
        const int32_t j = at + lane;
        const int32_t here = __builtin_popcountll(__ballot(j <= n_seq && row_start[j <= n_seq ? j : n_seq] <= i));
        n += here;
        if (here < 64) break;
    }
    return n <= n_seq ? n - 1 : -1;
}

}  // namespace mquant
