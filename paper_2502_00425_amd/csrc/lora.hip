// Low-rank adapters of many requests beside a shared linear, for gfx950:
//   h[i] = x[perm[i]] A_a^T,   y[i, n] = fp16(base[i, n] + scale[a] * h[i] B_a[n]^T),   a = adapter[i].
// Two launches: shrink (h, fp32, in slices of K) and expand (adds the slices, multiplies by B, adds to the base).  Both take
// rows 256 at a time and gather the rows of one adapter into a tile, so a tile reads its adapter once, however the
// requests are mixed; rows without an adapter are a tile of their own that copies.  Bound by the bytes of x, base, y and, for few
// rows, of the adapters.
#include <hip/hip_fp16.h>

#include "mquant_internal.h"

using namespace mquant;

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kBlock = 256;                // rows among which a tile is gathered: four a lane
constexpr int kShrinkWaves = 8;
constexpr int kUnit = 64;                  // channels of K that a wave takes at a time: a 128-byte line of every row
constexpr int kExpandWaves = 4;
constexpr int kCols = 64;                  // columns of y that a wave takes at a time
constexpr int kMaxSlices = 16;

struct Lora {
    const __half *x;
    int64_t ldx;
    const int32_t *perm, *adapter;
    const __half *a, *b;
    const float *scale;
    const __half *base;
    int64_t ldb;
    __half *y;
    int64_t ldy;
    float *h;                              // [slices][T][rank]
    int32_t T, N, K, rank, n_adapters, slices, cols;         // cols: columns of a work-group of the expansion
};

__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// Tile number `tile` of the 256 rows from row0 on: the adapters in order of their first row, TR rows of one a tile.  Puts the
// rows into `list` (every wave the same ones) and their number into n; -> adapter, n_adapters for the rows
// without one, -1: no such tile.
template <int TR>
__device__ __forceinline__ int32_t find_tile(const Lora &p, int32_t row0, int32_t tile, int32_t *list, int32_t &n)
{
    const int lane = threadIdx.x & 63;
    int32_t key[4];
    uint64_t left[4], mine[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int32_t i = row0 + q * 64 + lane;
        key[q] = i < p.T ? p.adapter[i] : -1;
        key[q] = key[q] >= 0 && key[q] < p.n_adapters ? key[q] : p.n_adapters;
        left[q] = __ballot(i < p.T);
    }
    int32_t cur = -1, count = 0;
    for (;;) {
        if (left[0] != 0) cur = __builtin_amdgcn_readlane(key[0], __builtin_ctzll(left[0]));
        else if (left[1] != 0) cur = __builtin_amdgcn_readlane(key[1], __builtin_ctzll(left[1]));
        else if (left[2] != 0) cur = __builtin_amdgcn_readlane(key[2], __builtin_ctzll(left[2]));
        else if (left[3] != 0) cur = __builtin_amdgcn_readlane(key[3], __builtin_ctzll(left[3]));
        else return -1;
        count = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            mine[q] = left[q] & __ballot(key[q] == cur);
            left[q] &= ~mine[q];
            count += __builtin_popcountll(mine[q]);
        }
        const int32_t tiles = (count + TR - 1) / TR;
        if (tile < tiles) break;
        tile -= tiles;
    }
    int32_t before = -tile * TR;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int32_t at = before + __builtin_popcountll(mine[q] & ((uint64_t{1} << lane) - 1));
        if (((mine[q] >> lane) & 1) != 0 && at >= 0 && at < TR) list[at] = row0 + q * 64 + lane;
        before += __builtin_popcountll(mine[q]);
    }
    n = count - tile * TR < TR ? count - tile * TR : TR;
    return cur;
}

// h of one tile and slice of K.  The waves take units of 64 channels in turn: x rows are the A operand, rows of A_a the B
// operand of 16x16x32 products, both straight from memory (16 bytes a lane), and their sums meet in LDS by halves.
template <int RT, int RB>
__global__ __launch_bounds__(kShrinkWaves * 64) void lora_shrink_kernel(Lora p)
{
    constexpr int TR = RT * 16;
    __shared__ __attribute__((aligned(16))) v4f sums[kShrinkWaves / 2][RT * RB][64];
    int32_t *list = reinterpret_cast<int32_t *>(sums);         // until the sums meet
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x >> 6);
    int32_t n = 0;
    const int32_t id = find_tile<TR>(p, blockIdx.y * kBlock, blockIdx.x, list, n);
    if (id < 0 || id == p.n_adapters) return;
    __syncthreads();

    int32_t row[RT];                                           // of y, lane l: row l % 16 of each 16
    const __half *xr[RT], *ar[RB];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int j = t * 16 + l16;
        row[t] = list[j < n ? j : n - 1];
        int32_t src = p.perm ? p.perm[row[t]] : row[t];
        src = src >= 0 && src < p.T ? src : 0;
        xr[t] = p.x + src * p.ldx;
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = b * 16 + l16;
        ar[b] = p.a + (static_cast<int64_t>(id) * p.rank + (r < p.rank ? r : p.rank - 1)) * p.K;
    }
    v4f acc[RT][RB];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[t][b] = v4f{0.f, 0.f, 0.f, 0.f};
    const int32_t units = (p.K + kUnit - 1) / kUnit, slice = blockIdx.z;
    const int32_t u0 = static_cast<int32_t>(static_cast<int64_t>(units) * slice / p.slices);
    const int32_t u1 = static_cast<int32_t>(static_cast<int64_t>(units) * (slice + 1) / p.slices);
    v8h xv[RT][2], av[RB][2];
    // K is a multiple of 8; what lies behind it in the last unit is read from the row's last 8 channels and multiplied by zero
    auto load = [&](int32_t u) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int32_t k = u * kUnit + s * 32 + g * 8, at = k < p.K ? k : p.K - 8;
#pragma unroll
            for (int b = 0; b < RB; ++b) av[b][s] = *reinterpret_cast<const v8h *>(ar[b] + at);
#pragma unroll
            for (int t = 0; t < RT; ++t) xv[t][s] = *reinterpret_cast<const v8h *>(xr[t] + at);
        }
    };
    auto multiply = [&](int32_t u) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if ((u + 1) * kUnit > p.K && u * kUnit + s * 32 + g * 8 >= p.K)
#pragma unroll
                for (int b = 0; b < RB; ++b) av[b][s] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int b = 0; b < RB; ++b) acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[t][s], av[b][s], acc[t][b], 0, 0, 0);
        }
    };
    for (int32_t u = u0 + wave; u < u1; u += kShrinkWaves) {
        load(u);
        multiply(u);
    }
    __syncthreads();
#pragma unroll
    for (int half = kShrinkWaves / 2; half >= 1; half >>= 1) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int b = 0; b < RB; ++b) sums[wave - half][t * RB + b][lane] = acc[t][b];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int b = 0; b < RB; ++b) acc[t][b] += sums[wave][t * RB + b][lane];
        __syncthreads();
    }
    if (wave != 0) return;
    float *h = p.h + static_cast<int64_t>(slice) * p.T * p.rank;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t i = __shfl(row[t], g * 4 + r, 64);   // result register r of lane group g is row 4 g + r
            if (t * 16 + g * 4 + r < n)
#pragma unroll
                for (int b = 0; b < RB; ++b)
                    if (b * 16 + l16 < p.rank) h[i * p.rank + b * 16 + l16] = acc[t][b][r];
        }
}

// y of one tile and `cols` columns.  Y^T = B_a h^T: rows of B_a are the A operand, rows of h the B operand, so that a lane is a row
// of y.  A-row rho of product s is column 32 (s / 2) + 8 (rho / 4) + 4 (s % 2) + rho % 4 of the wave's 64: a lane's four products hold two
// times 8 consecutive columns, 16 bytes each.  h goes in as two fp16 parts of h 2^-e, e per row from its largest value: what is lost is
// 2^-22 of that value, and no magnitude of h overflows.
template <int RT, int KS, bool VEC>
__global__ __launch_bounds__(kExpandWaves * 64) void lora_expand_kernel(Lora p)
{
    constexpr int TR = RT * 16;
    __shared__ int32_t list[TR];
    __shared__ float factors[TR];
    __shared__ __attribute__((aligned(16))) v8h parts[RT][KS][2][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x >> 6);
    int32_t n = 0;
    const int32_t id = find_tile<TR>(p, blockIdx.y * kBlock, blockIdx.x, list, n);
    if (id < 0) return;
    const bool none = id == p.n_adapters;
    if (none && p.y == p.base) return;
    __syncthreads();

    int32_t row[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) row[t] = list[t * 16 + l16 < n ? t * 16 + l16 : n - 1];
    v8h bv[4][KS], bs[RT][2];
    // Rows, columns and ranks behind the last repeat it, so that no load is a branch; what they give is multiplied by zero or not stored
    auto load = [&](int32_t c0) {
        if (!none)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int32_t col = c0 + (s >> 1) * 32 + (l16 >> 2) * 8 + (s & 1) * 4 + (l16 & 3);
                const __half *br = p.b + (static_cast<int64_t>(id) * p.N + (col < p.N ? col : p.N - 1)) * p.rank;
#pragma unroll
                for (int k = 0; k < KS; ++k) bv[s][k] = *reinterpret_cast<const v8h *>(br + (k * 32 + g * 8 < p.rank ? k * 32 + g * 8 : p.rank - 8));
            }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int32_t col = c0 + w * 32 + g * 8;
                const __half *base = p.base + row[t] * p.ldb;
                if constexpr (VEC) {
                    bs[t][w] = *reinterpret_cast<const v8h *>(base + (col < p.N ? col : p.N - 8));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) bs[t][w][e] = *reinterpret_cast<const _Float16 *>(base + (col + e < p.N ? col + e : p.N - 1));
                }
            }
    };
    const int32_t first = blockIdx.z * p.cols, end = p.N - first < p.cols ? p.N : first + p.cols;
    load(first + wave * kCols);                                // on its way while the rows' parts are prepared

    // The slices of h are added by all waves: wave w takes 16 rows and every SG-th slice; the groups' sums meet in LDS, and one of
    // them leaves the rows' parts where all waves read them.
    constexpr int SG = kExpandWaves / RT;
    const int nsub = (n + 15) / 16;
    const float scale = none ? 0.0f : p.scale[id];
    const int t_h = wave / SG, part_h = wave % SG;
    float f[KS][8];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) f[s][e] = 0.0f;
    if (!none && t_h < nsub) {
        const int j = t_h * 16 + l16;
        const int64_t slice = static_cast<int64_t>(p.T) * p.rank;
        const float *h = p.h + static_cast<int64_t>(list[j < n ? j : n - 1]) * p.rank;
        constexpr int kAtOnce = KS <= 2 ? 4 : 2;
        for (int32_t c = part_h; c < p.slices; c += kAtOnce * SG) {
            v4f v[kAtOnce][KS][2];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int s = 0; s < KS; ++s) {                 // ranks and slices behind the last repeat it
                    const int r = s * 32 + g * 8;
                    const float *at = h + (c + i * SG < p.slices ? c + i * SG : c) * slice + (r < p.rank ? r : p.rank - 8);
                    v[i][s][0] = reinterpret_cast<const v4f *>(at)[0];
                    v[i][s][1] = reinterpret_cast<const v4f *>(at)[1];
                }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        f[s][e] += c + i * SG < p.slices && s * 32 + g * 8 < p.rank ? v[i][s][e >> 2][e & 3] : 0.0f;
        }
    }
    if constexpr (SG > 1) {
        __shared__ __attribute__((aligned(16))) float meet[RT][SG - 1][KS][64][8];
        if (part_h > 0)
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) meet[t_h][part_h - 1][s][lane][e] = f[s][e];
        __syncthreads();
        if (part_h == 0)
#pragma unroll
            for (int o = 0; o < SG - 1; ++o)
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[s][e] += meet[t_h][o][s][lane][e];
    }
    if (!none && t_h < nsub && part_h == 0) {
        float top = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[s][e]));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        int e2 = static_cast<int>((__float_as_uint(top) >> 23) & 255) - 127 - 14;       // the largest value below 2^15
        e2 = e2 < -100 ? -100 : e2;
        const float down = __uint_as_float(static_cast<uint32_t>(127 - e2) << 23);
        if (g == 0) factors[t_h * 16 + l16] = scale * __uint_as_float(static_cast<uint32_t>(127 + e2) << 23);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            v8h hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = f[s][e] * down;
                hi[e] = static_cast<_Float16>(v);
                lo[e] = static_cast<_Float16>(v - static_cast<float>(hi[e]));
            }
            parts[t_h][s][0][lane] = hi;
            parts[t_h][s][1][lane] = lo;
        }
    }
    __syncthreads();

    float factor[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) factor[t] = factors[t * 16 + l16];
    for (int32_t c0 = first + wave * kCols; c0 < end; c0 += kExpandWaves * kCols) {
        if (c0 != first + wave * kCols) load(c0);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (t >= nsub) break;
            v4f acc[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) acc[s] = v4f{0.f, 0.f, 0.f, 0.f};
            if (!none)
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int part = 1; part >= 0; --part) {
                        const v8h hv = parts[t][k][part][lane];
#pragma unroll
                        for (int s = 0; s < 4; ++s) acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bv[s][k], hv, acc[s], 0, 0, 0);
                    }
            __half *out = p.y + row[t] * p.ldy;
            const bool mine = t * 16 + l16 < n;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int32_t col = c0 + w * 32 + g * 8;
                v8h r = bs[t][w];
                if (!none)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        r[e] = static_cast<_Float16>(__builtin_fmaf(factor[t], acc[w * 2 + (e >> 2)][e & 3], static_cast<float>(r[e])));
                if constexpr (VEC) {
                    if (mine && col < p.N) *reinterpret_cast<v8h *>(out + col) = r;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (mine && col + e < p.N) *reinterpret_cast<_Float16 *>(out + col + e) = r[e];
                }
            }
        }
    }
}

// Rows of a tile and slices of K.  Few rows: tiles of 16, and slices short enough that each wave has about one unit; more: tiles of 64
// (32 at ranks beyond 64: 64 accumulator registers either way), and as many slices as give every compute unit a work-group.
struct Plan {
    int rt, rb;
    int32_t slices, tiles;                 // tiles: at most, per 256 rows, behind the first of every adapter
};

Plan make_plan(int32_t T, int32_t K, int32_t rank)
{
    Plan p;
    p.rb = rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8;
    p.rt = T <= 64 ? 1 : p.rb == 8 ? 2 : 4;
    const int32_t units = static_cast<int32_t>(ceil_div(K, kUnit));
    int64_t s = T <= 64 ? ceil_div(units, kShrinkWaves) : kNumCU / ceil_div(T, p.rt * 16);
    const int64_t most = T <= 64 ? kMaxSlices : ceil_div(units, 2 * kShrinkWaves);
    if (s > most) s = most;
    if (s > kMaxSlices) s = kMaxSlices;
    p.slices = static_cast<int32_t>(s < 1 ? 1 : s);
    p.tiles = static_cast<int32_t>((T < kBlock ? T : kBlock) / (p.rt * 16));
    return p;
}

template <int RT, int RB>
int launch_shrink(const Lora &a, dim3 grid, hipStream_t stream)
{
    MQ_LAUNCH((lora_shrink_kernel<RT, RB>), grid, dim3(kShrinkWaves * 64), 0, stream, a);
    return launch_status();
}

template <int RT, int KS>
int launch_expand(const Lora &a, dim3 grid, bool vec, hipStream_t stream)
{
    if (vec) MQ_LAUNCH((lora_expand_kernel<RT, KS, true>), grid, dim3(kExpandWaves * 64), 0, stream, a);
    else MQ_LAUNCH((lora_expand_kernel<RT, KS, false>), grid, dim3(kExpandWaves * 64), 0, stream, a);
    return launch_status();
}

}  // namespace

extern "C" int64_t mquant_lora_workspace_bytes(int32_t T, int32_t K, int32_t rank)
{
    if (T < 0 || K < 0 || rank < 1) return MQUANT_ERR_BAD_SHAPE;
    if (K == 0 || K % 8 != 0 || rank % 8 != 0 || rank > 128) return MQUANT_ERR_UNSUPPORTED;
    if (T == 0) return 0;
    return ceil_div(static_cast<int64_t>(make_plan(T, K, rank).slices) * T * rank * 4, 256) * 256;
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
    hipStream_t stream = static_cast<hipStream_t>(stream_);

    const Plan p = make_plan(T, K, rank);
    Lora args = {static_cast<const __half *>(x), ldx, perm, adapter, static_cast<const __half *>(a), static_cast<const __half *>(b), scale,
                 static_cast<const __half *>(base), ldb, static_cast<__half *>(y), ldy, static_cast<float *>(workspace), T, N, K, rank,
                 n_adapters, p.slices, T <= 64 ? kExpandWaves * kCols : 2 * kExpandWaves * kCols};
    const int64_t blocks = ceil_div(T, kBlock), chunks = ceil_div(N, args.cols);
    const int32_t in_block = T < kBlock ? T : kBlock;
    // tiles of a block: full ones, and a last one of every adapter (and of the rows without)
    const int32_t tiles = p.tiles + (n_adapters < in_block ? n_adapters + 1 : in_block);
    if (blocks > 65535 || chunks > 65535) return MQUANT_ERR_UNSUPPORTED;
    const bool vec = N % 8 == 0 && ldb % 8 == 0 && ldy % 8 == 0 && aligned_to(base, 16) && aligned_to(y, 16);
    if (n_adapters > 0) {
        const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(blocks), static_cast<unsigned>(p.slices));
        int st;
        if (p.rt == 1) {
            st = p.rb == 1 ? launch_shrink<1, 1>(args, grid, stream) : p.rb == 2 ? launch_shrink<1, 2>(args, grid, stream)
               : p.rb == 4 ? launch_shrink<1, 4>(args, grid, stream) : launch_shrink<1, 8>(args, grid, stream);
        } else {
            st = p.rb == 1 ? launch_shrink<4, 1>(args, grid, stream) : p.rb == 2 ? launch_shrink<4, 2>(args, grid, stream)
               : p.rb == 4 ? launch_shrink<4, 4>(args, grid, stream) : launch_shrink<2, 8>(args, grid, stream);
        }
        if (st != MQUANT_OK) return st;
    }
    const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(blocks), static_cast<unsigned>(chunks));
    if (p.rt == 1)
        return p.rb <= 2 ? launch_expand<1, 1>(args, grid, vec, stream) : p.rb == 4 ? launch_expand<1, 2>(args, grid, vec, stream)
                                                                                    : launch_expand<1, 4>(args, grid, vec, stream);
    return p.rb <= 2 ? launch_expand<4, 1>(args, grid, vec, stream) : p.rb == 4 ? launch_expand<4, 2>(args, grid, vec, stream)
                                                                                : launch_expand<2, 4>(args, grid, vec, stream);
}
