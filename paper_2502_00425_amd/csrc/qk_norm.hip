// Norms of queries and keys per head with the rotary embedding, and with the write of keys and values to
// their pages, in one pass, for gfx950.
//
// For a head x of 128 channels and position p:
//   u = x * w * (sum(x^2) / 128 + eps)^(-1/2)     (no weight: u = x)
//   y[2j] = u[2j] cos a - u[2j+1] sin a,  y[2j+1] = u[2j] sin a + u[2j+1] cos a,  a = p * base^(-2j/128)
// A position of 16384 leaves an fp32 angle accurate to 1e-3 only, so angles are formed in double, in turns (p * base^(-2j/128) / 2 pi):
// whole turns are taken off there, what is left, at most half a turn, is rounded to fp32 (2^-22 of a radian) for its sine and
// cosine.  The squares' sum and the products are fp32, and the result is rounded to fp16 once.
#include <cmath>

#include "serving_common.h"

using namespace mquant;

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
constexpr int kD = kCacheHeadDim;

struct Angles {
    double f[kD / 2];
};

struct Rows {
    const __half *q, *k, *v;
    __half *q_out, *k_out;
    int64_t ldq, ldqo, ldk, ldko, ldv;
    const __half *q_weight, *k_weight;
    const int32_t *pos, *rope_pos, *row_start;
    float eps;
    int32_t T, n_q, n_k;
};

// A wave takes one row and `per` (at most U) groups of four heads (queries first, then keys, then values): 16 lanes a head, 16
// bytes a lane.  Lane l forms the angle of pair l, every lane then takes the four pairs it holds, the same ones in all its
// heads.  `waves` waves share a row and lie next to each other, so that rows are read and written from end to end.  Bound by the bytes: 72
// heads of 16384 rows 104 us, 604 MB, 5.8 TB/s.  Few rows are bound by the launch and two trips to memory: 77 rows of 32 heads 3.2 us.
// Rows that fill the chip go past the caches (72 heads of 16384 rows 121.7 -> 107.5 us, 36 of 4096 with the append 17.8 ->
// 14.9): lines that are written whole need not be looked up there.  Few rows stay, the next kernel reads them.
template <bool PAST>
__device__ __forceinline__ void put(__half *p, v8h v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<v8h *>(p));
    else *reinterpret_cast<v8h *>(p) = v;
}

template <bool APPEND, int U>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(Rows a, PagedCache c, Angles inv, int32_t waves, int32_t per)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t i = static_cast<int32_t>(item / waves);
    if (i >= a.T) return;
    const int32_t part = static_cast<int32_t>(item % waves);
    const int32_t first = part * per * 4 + (lane >> 4), all = a.n_q + a.n_k * (APPEND ? 2 : 1);
    const int32_t heads = all < (part + 1) * per * 4 ? all : (part + 1) * per * 4;         // this wave's end
    const int ch = (lane & 15) * 8;
    const int32_t p = a.pos[i];
    v8h x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t h = first + u * 4;
        const __half *row = h < a.n_q ? a.q + i * a.ldq + static_cast<int64_t>(h) * kD
                            : h < a.n_q + a.n_k ? a.k + i * a.ldk + static_cast<int64_t>(h - a.n_q) * kD
                                                : a.v + i * a.ldv + static_cast<int64_t>(h - a.n_q - a.n_k) * kD;
        x[u] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
        if (h < heads) x[u] = *reinterpret_cast<const v8h *>(row + ch);
    }
    const int32_t seq = APPEND ? sequence_of_row(a.row_start, c.n_seq, i) : 0;
    if (seq < 0) return;
    // the row's slot
    int64_t slot = -1;                                          // halves from a page array's start to head 0's row
    int32_t head_stride = 0;
    if constexpr (APPEND) {
        head_stride = kD << c.page_shift;
        const int32_t page_at = p >> c.page_shift;
        if (p >= 0 && page_at < c.table_pages) {
            const int32_t page = c.table[static_cast<int64_t>(seq) * c.table_pages + page_at];
            if (page >= 0 && page < c.n_pages)
                slot = page * c.page_halves + static_cast<int64_t>(p & ((1 << c.page_shift) - 1)) * kD;
        }
    }
    const double turns = static_cast<double>(APPEND && a.rope_pos ? a.rope_pos[i] : p) * inv.f[lane];
    float sn, cs, co[4], si[4];
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &cs);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        co[e] = __shfl(cs, (lane & 15) * 4 + e, 64);
        si[e] = __shfl(sn, (lane & 15) * 4 + e, 64);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t h = first + u * 4;
        if (U > 1 && u >= per) break;
        const bool is_q = h < a.n_q && h < heads, is_v = APPEND && h >= a.n_q + a.n_k;
        const __half *w = is_q ? a.q_weight : a.k_weight;
        float f[8], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = static_cast<float>(x[u][e]);
            sum = __builtin_fmaf(f[e], f[e], sum);
        }
        sum = row16_sum(sum);
        if (w && h < heads && !is_v) {
            const float r = 1.0f / sqrtf(sum * (1.0f / kD) + a.eps);
            const v8h wt = *reinterpret_cast<const v8h *>(w + ch);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= r * static_cast<float>(wt[e]);
        }
        v8h y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[2 * e] = static_cast<_Float16>(f[2 * e] * co[e] - f[2 * e + 1] * si[e]);
            y[2 * e + 1] = static_cast<_Float16>(f[2 * e] * si[e] + f[2 * e + 1] * co[e]);
        }
        if (is_q) {
            put<(U > 1)>(a.q_out + i * a.ldqo + static_cast<int64_t>(h) * kD + ch, y);
        } else if (!APPEND) {
            if (h < heads) put<(U > 1)>(a.k_out + i * a.ldko + static_cast<int64_t>(h - a.n_q) * kD + ch, y);
        } else if (h < heads && slot >= 0) {
            if (is_v) put<(U > 1)>(c.v + slot + static_cast<int64_t>(h - a.n_q - a.n_k) * head_stride + ch, x[u]);
            else put<(U > 1)>(c.k + slot + static_cast<int64_t>(h - a.n_q) * head_stride + ch, y);
        }
    }
}

int check_side(const void *x, int64_t ldx, const void *out, int64_t ldo, int32_t T, int32_t heads)
{
    if (heads == 0) return MQUANT_OK;
    if (!x || !out) return MQUANT_ERR_NULL;
    const int64_t w = static_cast<int64_t>(heads) * kD;
    if (ldx < w || ldo < w) return MQUANT_ERR_BAD_SHAPE;
    if (x == out && ldx != ldo && T > 1) return MQUANT_ERR_BAD_SHAPE;         // of a single row it says nothing
    if (ldx % 8 != 0 || ldo % 8 != 0 || !aligned_to(x, 16) || !aligned_to(out, 16)) return MQUANT_ERR_ALIGNMENT;
    return MQUANT_OK;
}

int check_norm(const void *q_weight, const void *k_weight, float eps, double base)
{
    if (!(eps >= 0.0f) || !std::isfinite(eps) || !(base > 1.0) || !std::isfinite(base)) return MQUANT_ERR_BAD_SHAPE;
    if (!aligned_to(q_weight, 16) || !aligned_to(k_weight, 16)) return MQUANT_ERR_ALIGNMENT;
    return MQUANT_OK;
}

template <bool APPEND>
int launch(const Rows &a, const PagedCache &c, double base, hipStream_t stream)
{
    const int64_t heads = a.n_q + static_cast<int64_t>(a.n_k) * (APPEND ? 2 : 1);
    Angles inv;
    // base^(-2j/128) / 2 pi, each from the one before in 64-bit fractions (off by 2^-57 at most; 64 calls of pow cost the host 1.3 us)
    const long double ratio = powl(static_cast<long double>(base), -2.0L / kD);
    long double f = 0.159154943091895335768883763372514362L;
    for (int j = 0; j < kD / 2; ++j, f *= ratio) inv.f[j] = static_cast<double>(f);
    // A wave takes four heads where rows are few, since what such a launch waits for is the way of one wave, else up to 16.  Waves of 4 /
    // of up to 16 heads, 32 heads: 512 rows 4.1 / 4.7 us, 700 5.0 / 5.0, 1024 5.8 / 5.3, 4096 15.0 / 11.6; 72 heads: 256 4.4 / 5.0, 512 6.2 / 6.0.
    // (Up to 12 heads at 72 of 16384 rows 102.4 us, 16 101.1: 6.0 TB/s, 20 103.6, 40 107.3; 32 of 4096 12.8, 11.6, 12.3, 12.2.)
    constexpr int U = 4;
    const int64_t groups = ceil_div(heads, 4);
    int64_t waves = ceil_div(groups, U);
    const bool few = a.T * groups < 6000;
    if (few) waves = groups;
    const int64_t blocks = ceil_div(a.T * waves, 4);
    if (blocks > kMaxThreads / 256 || heads > 1 << 20) return MQUANT_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(blocks));
    const int32_t per = static_cast<int32_t>(ceil_div(groups, waves)), n = static_cast<int32_t>(waves);
    if (few) MQ_LAUNCH((qk_norm_rope_kernel<APPEND, 1>), grid, dim3(256), 0, stream, a, c, inv, n, per);
    else MQ_LAUNCH((qk_norm_rope_kernel<APPEND, U>), grid, dim3(256), 0, stream, a, c, inv, n, per);
    return launch_status();
}

}  // namespace

extern "C" int mquant_qk_norm_rope(const void *q, int64_t ldq, void *q_out, int64_t ldqo, const void *k, int64_t ldk, void *k_out,
                                   int64_t ldko, const void *q_weight, const void *k_weight, float eps, const int32_t *pos,
                                   int32_t T, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, double base,
                                   mquant_stream_t stream)
{
    if (T < 0 || n_q_heads < 0 || n_kv_heads < 0 || (n_q_heads == 0 && n_kv_heads == 0)) return MQUANT_ERR_BAD_SHAPE;
    if (head_dim != kD) return MQUANT_ERR_UNSUPPORTED;
    if (const int st = check_norm(q_weight, k_weight, eps, base); st != MQUANT_OK) return st;
    if (T == 0) return MQUANT_OK;
    if (!pos) return MQUANT_ERR_NULL;
    if (!aligned_to(pos, 4)) return MQUANT_ERR_ALIGNMENT;
    if (const int st = check_side(q, ldq, q_out, ldqo, T, n_q_heads); st != MQUANT_OK) return st;
    if (const int st = check_side(k, ldk, k_out, ldko, T, n_kv_heads); st != MQUANT_OK) return st;
    const Rows a = {static_cast<const __half *>(q), static_cast<const __half *>(k), nullptr, static_cast<__half *>(q_out),
                    static_cast<__half *>(k_out), ldq, ldqo, ldk, ldko, 0, static_cast<const __half *>(q_weight),
                    static_cast<const __half *>(k_weight), pos, nullptr, nullptr, eps, T, n_q_heads, n_kv_heads};
    return launch<false>(a, PagedCache{}, base, static_cast<hipStream_t>(stream));
}

extern "C" int mquant_kv_append(const void *q, int64_t ldq, void *q_out, int64_t ldqo, const void *k, int64_t ldk, const void *v,
                                int64_t ldv, const void *q_weight, const void *k_weight, float eps, const int32_t *row_start,
                                const int32_t *pos, const int32_t *rope_pos, int32_t T, int32_t n_q_heads, double base,
                                const mquant_paged_cache_t *cache, mquant_stream_t stream)
{
    if (T < 0 || n_q_heads < 0) return MQUANT_ERR_BAD_SHAPE;
    if (const int st = check_cache(cache); st != MQUANT_OK) return st;
    if (const int st = check_norm(q_weight, k_weight, eps, base); st != MQUANT_OK) return st;
    if (T == 0 || cache->n_seq == 0) return MQUANT_OK;
    if (!row_start || !pos) return MQUANT_ERR_NULL;
    if (!aligned_to(row_start, 4) || !aligned_to(pos, 4) || !aligned_to(rope_pos, 4)) return MQUANT_ERR_ALIGNMENT;
    if (const int st = check_side(q, ldq, q_out, ldqo, T, n_q_heads); st != MQUANT_OK) return st;
    if (const int st = check_side(k, ldk, cache->k_pages_dev, ldk, T, cache->n_kv_heads); st != MQUANT_OK) return st;
    if (const int st = check_side(v, ldv, cache->v_pages_dev, ldv, T, cache->n_kv_heads); st != MQUANT_OK) return st;
    const Rows a = {static_cast<const __half *>(q), static_cast<const __half *>(k), static_cast<const __half *>(v),
                    static_cast<__half *>(q_out), nullptr, ldq, ldqo, ldk, 0, ldv, static_cast<const __half *>(q_weight),
                    static_cast<const __half *>(k_weight), pos, rope_pos, row_start, eps, T, n_q_heads, cache->n_kv_heads};
    return launch<true>(a, cache_args(cache), base, static_cast<hipStream_t>(stream));
}
