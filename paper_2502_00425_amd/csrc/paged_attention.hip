// Attention of a step's rows over a paged cache, for gfx950.
//
// Row i of sequence s sees the slots j <= pos[i]: o = sum_j p_j v_j, p = softmax(q k_j / sqrt(128)), one pass over
// the slots with the running maximum and sum of the softmax.
#include <cmath>

#include "serving_common.h"

using namespace mquant;

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
constexpr int kD = kCacheHeadDim;

// A wave takes one row and query head, 64 slots at a time: a lane's score is that of one slot, its output two channels.
__global__ __launch_bounds__(256) void paged_attention_rows_kernel(const __half *__restrict__ q, int64_t ldq, PagedCache c,
                                                                   const int32_t *__restrict__ row_start,
                                                                   const int32_t *__restrict__ pos, __half *__restrict__ o,
                                                                   int64_t ldo, int32_t T, int32_t n_q, float scale_log2e)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int32_t i = static_cast<int32_t>(item / n_q), h = static_cast<int32_t>(item % n_q);
    if (i >= T) return;
    const int32_t seq = sequence_of_row(row_start, c.n_seq, i);
    if (seq < 0) return;
    const int32_t slots = c.table_pages << c.page_shift, in_page = (1 << c.page_shift) - 1;
    const int32_t p = pos[i], len = p < 0 ? 0 : p < slots ? p + 1 : slots;
    const int64_t head = static_cast<int64_t>(h / (n_q / c.n_kv_heads)) << c.page_shift;
    const __half *qr = q + i * ldq + static_cast<int64_t>(h) * kD;
    const int32_t *table = c.table + static_cast<int64_t>(seq) * c.table_pages;
    float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int32_t j0 = 0; j0 < len; j0 += 64) {
        const int32_t j = j0 + lane < len ? j0 + lane : len - 1;
        int32_t page = table[j >> c.page_shift];
        page = page >= 0 && page < c.n_pages ? page : 0;
        const int64_t row = page * c.page_halves + (head + (j & in_page)) * kD;
        float s = 0.0f;
        for (int d = 0; d < kD; d += 8) {
            const v8h kv = *reinterpret_cast<const v8h *>(c.k + row + d), qv = *reinterpret_cast<const v8h *>(qr + d);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_fmaf(static_cast<float>(kv[e]), static_cast<float>(qv[e]), s);
        }
        s = j0 + lane < len ? s * scale_log2e : -INFINITY;
        float top = s;
        for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
        top = fmaxf(m, top);
        const float alpha = exp2f(m - top), w = exp2f(s - top);
        float sum = w;
        for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
        m = top;
        l = l * alpha + sum;
        o0 *= alpha;
        o1 *= alpha;
        const int n = len - j0 < 64 ? len - j0 : 64;
        for (int t = 0; t < n; ++t) {
            const float wt = __shfl(w, t, 64);
            const int64_t vr = __shfl(row, t, 64);
            const __half2 v2 = *reinterpret_cast<const __half2 *>(c.v + vr + lane * 2);
            o0 = __builtin_fmaf(wt, __low2float(v2), o0);
            o1 = __builtin_fmaf(wt, __high2float(v2), o1);
        }
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    *reinterpret_cast<__half2 *>(o + i * ldo + static_cast<int64_t>(h) * kD + lane * 2) = __floats2half2_rn(o0 * inv, o1 * inv);
}

int check_sizes(int32_t T, int32_t n_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_rows, int32_t max_kv)
{
    if (T < 0 || n_seq < 0 || n_q_heads < 1 || n_kv_heads < 1 || max_rows < 0 || max_kv < 0) return MQUANT_ERR_BAD_SHAPE;
    if (head_dim != kD) return MQUANT_ERR_UNSUPPORTED;
    if (n_q_heads % n_kv_heads != 0) return MQUANT_ERR_BAD_SHAPE;
    return MQUANT_OK;
}

}  // namespace

extern "C" int64_t mquant_paged_attention_workspace_bytes(int32_t T, int32_t n_seq, int32_t n_q_heads, int32_t n_kv_heads,
                                                          int32_t head_dim, int32_t max_rows, int32_t max_kv)
{
    return check_sizes(T, n_seq, n_q_heads, n_kv_heads, head_dim, max_rows, max_kv);
}

extern "C" int mquant_paged_attention(const void *q, int64_t ldq, const mquant_paged_cache_t *cache, const int32_t *row_start,
                                      const int32_t *pos, void *o, int64_t ldo, int32_t T, int32_t n_q_heads, int32_t max_rows,
                                      int32_t max_kv, void *workspace, int64_t workspace_bytes, mquant_stream_t stream)
{
    if (const int st = check_cache(cache); st != MQUANT_OK) return st;
    if (const int st = check_sizes(T, cache->n_seq, n_q_heads, cache->n_kv_heads, cache->head_dim, max_rows, max_kv); st != MQUANT_OK)
        return st;
    if (T == 0 || cache->n_seq == 0) return MQUANT_OK;
    if (!q || !o || !row_start || !pos) return MQUANT_ERR_NULL;
    const int64_t w = static_cast<int64_t>(n_q_heads) * kD;
    if (ldq < w || ldo < w) return MQUANT_ERR_BAD_SHAPE;
    if (ldq % 8 != 0 || ldo % 4 != 0 || !aligned_to(q, 16) || !aligned_to(o, 8) || !aligned_to(pos, 4) || !aligned_to(row_start, 4))
        return MQUANT_ERR_ALIGNMENT;
    const int64_t blocks = ceil_div(static_cast<int64_t>(T) * n_q_heads, 4);
    if (blocks > 0x7fffffff) return MQUANT_ERR_UNSUPPORTED;
    const float scale_log2e = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(kD)));
    MQ_LAUNCH(paged_attention_rows_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, static_cast<hipStream_t>(stream),
              static_cast<const __half *>(q), ldq, cache_args(cache), row_start, pos, static_cast<__half *>(o), ldo, T, n_q_heads,
              scale_log2e);
    return launch_status();
}
