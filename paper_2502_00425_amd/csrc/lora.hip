// Low-rank adapters of many requests beside a shared linear, for gfx950:
//   h[i] = x[perm[i]] A_a^T (fp32, in the workspace),  y[i, n] = fp16(base[i, n] + scale[a] * h[i] B_a[n]^T),  a = adapter[i].
#include <hip/hip_fp16.h>

#include "mquant_internal.h"

using namespace mquant;

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

__global__ __launch_bounds__(256) void lora_shrink_kernel(const __half *__restrict__ x, int64_t ldx, const int32_t *__restrict__ perm,
                                                          const int32_t *__restrict__ adapter, const __half *__restrict__ a,
                                                          float *__restrict__ h, int32_t T, int32_t K, int32_t rank, int32_t n_adapters)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t i = blockIdx.x, id = adapter[i];
    if (id < 0 || id >= n_adapters) return;
    int32_t src = perm ? perm[i] : i;
    src = src >= 0 && src < T ? src : 0;
    for (int32_t r = wave; r < rank; r += 4) {
        const __half *ar = a + (static_cast<int64_t>(id) * rank + r) * K;
        float s = 0.0f;
        for (int32_t k = lane * 8; k < K; k += 512) {
            const v8h xv = *reinterpret_cast<const v8h *>(x + src * ldx + k), av = *reinterpret_cast<const v8h *>(ar + k);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_fmaf(static_cast<float>(xv[e]), static_cast<float>(av[e]), s);
        }
        for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m, 64);
        if (lane == 0) h[static_cast<int64_t>(i) * rank + r] = s;
    }
}

__global__ __launch_bounds__(256) void lora_expand_kernel(const float *__restrict__ h, const int32_t *__restrict__ adapter,
                                                          const __half *__restrict__ b, const float *__restrict__ scale,
                                                          const __half *base, int64_t ldb, __half *y, int64_t ldy, int32_t N,
                                                          int32_t rank, int32_t n_adapters)
{
    const int32_t n = blockIdx.x * 256 + threadIdx.x, i = blockIdx.y, id = adapter[i];
    if (n >= N) return;
    float f = __half2float(base[i * ldb + n]);
    if (id >= 0 && id < n_adapters) {
        const __half *br = b + (static_cast<int64_t>(id) * N + n) * rank;
        float s = 0.0f;
        for (int32_t r = 0; r < rank; ++r) s = __builtin_fmaf(h[static_cast<int64_t>(i) * rank + r], __half2float(br[r]), s);
        f = __builtin_fmaf(scale[id], s, f);
    }
    y[i * ldy + n] = __float2half_rn(f);
}

}  // namespace

extern "C" int64_t mquant_lora_workspace_bytes(int32_t T, int32_t K, int32_t rank)
{
    if (T < 0 || K < 0 || rank < 1) return MQUANT_ERR_BAD_SHAPE;
    if (K == 0 || K % 8 != 0 || rank % 8 != 0 || rank > 128) return MQUANT_ERR_UNSUPPORTED;
    return ceil_div(static_cast<int64_t>(T) * rank * 4, 256) * 256;
}

extern "C" int mquant_lora_apply(const void *x, int64_t ldx, const int32_t *perm, const int32_t *adapter, const void *a, const void *b,
                                 const float *scale, const void *base, int64_t ldb, void *y, int64_t ldy, int32_t T, int32_t N,
                                 int32_t K, int32_t rank, int32_t n_adapters, void *workspace, int64_t workspace_bytes,
                                 mquant_stream_t stream_)
{
    if (N < 0 || n_adapters < 0) return MQUANT_ERR_BAD_SHAPE;
    const int64_t need = mquant_lora_workspace_bytes(T, K, rank);
    if (need < 0) return static_cast<int>(need);
    if (T == 0 || N == 0) return MQUANT_OK;
    if (!x || !adapter || !base || !y || (n_adapters > 0 && (!a || !b || !scale))) return MQUANT_ERR_NULL;
    if (ldx < K || ldb < N || ldy < N || (y == base && ldy != ldb)) return MQUANT_ERR_BAD_SHAPE;
    if (ldx % 8 != 0 || !aligned_to(x, 16) || !aligned_to(a, 16) || !aligned_to(b, 16) || !aligned_to(base, 2) || !aligned_to(y, 2) ||
        !aligned_to(adapter, 4) || !aligned_to(perm, 4) || !aligned_to(scale, 4))
        return MQUANT_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < need) return MQUANT_ERR_WORKSPACE;
    if (!aligned_to(workspace, 256)) return MQUANT_ERR_ALIGNMENT;
    if (T > 65535) return MQUANT_ERR_UNSUPPORTED;
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    float *h = static_cast<float *>(workspace);
    MQ_LAUNCH(lora_shrink_kernel, dim3(static_cast<unsigned>(T)), dim3(256), 0, stream, static_cast<const __half *>(x), ldx, perm, adapter,
              static_cast<const __half *>(a), h, T, K, rank, n_adapters);
    if (const int st = launch_status(); st != MQUANT_OK) return st;
    MQ_LAUNCH(lora_expand_kernel, dim3(static_cast<unsigned>(ceil_div(N, 256)), static_cast<unsigned>(T)), dim3(256), 0, stream, h, adapter,
              static_cast<const __half *>(b), scale, static_cast<const __half *>(base), ldb, static_cast<__half *>(y), ldy, N, rank, n_adapters);
    return launch_status();
}
