// Low-rank adapters of many requests beside a shared linear, for gfx950:
//   h[i] = x[perm[i]] A_a^T,   y[i, n] = fp16(base[i, n] + scale[a] * h[i] B_a[n]^T),   a = adapter[i].
// Two launches: shrink (h, fp32, in slices of K) and expand (adds the slices, multiplies by B, adds to the base).  Both take
// rows 256 at a time and gather the rows of one adapter into a tile, so a tile reads its adapter once, however the
// requests are mixed; rows without an adapter are a tile of their own that copies.  Bound by the bytes of x, base, y and, for few
// rows, of the adapters.
#include <hip/hip_fp16.h>

#include <cmath>

#include "lds_dma.h"
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
constexpr int kMaxSlices = 16;             // of few rows
constexpr int32_t kMaxSide = 1 << 30;      // of K and N: kernels step past their end in 32 bits

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
    const int quarters = p.T - row0 < kBlock ? (p.T - row0 + 63) / 64 : 4;     // that hold rows
    int32_t key[4] = {0, 0, 0, 0};
    uint64_t left[4] = {0, 0, 0, 0}, mine[4] = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= quarters) break;
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
            if (q >= quarters) break;
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

// h in two fp16 parts of h 2^-e: e from the largest value of a row, so that this lies below 2^15.
__device__ __forceinline__ void scale_of(float &top, float &down, float &up)
{
    top = fmaxf(top, __shfl_xor(top, 16, 64));                 // a row's ranks are spread over the lane groups
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    int e = static_cast<int>((__float_as_uint(top) >> 23) & 255) - 127 - 14;
    e = e < -100 ? -100 : e;
    down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
}

__device__ __forceinline__ void split(const float (&f)[8], float down, v8h &hi, v8h &lo)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = f[e] * down;
        hi[e] = static_cast<_Float16>(v);
        lo[e] = static_cast<_Float16>(v - static_cast<float>(hi[e]));
    }
}

// h of 16 rows and a slice of K.  The waves take units of 64 channels in turn: x rows are the A operand, rows of A_a the B
// operand of 16x16x32 products, both straight from memory (16 bytes a lane), and their sums meet in LDS by halves.  Bound by latency: 4 rows
// of 3584 channels, rank 16, 4.2 us; 48 rows of 12 adapters, 29568 channels, 7.4 (14.2 MB of x and A, 1.9 TB/s: a wave has one to four units).
template <int RB>
__global__ __launch_bounds__(kShrinkWaves * 64) void lora_shrink_kernel(Lora p)
{
    __shared__ int32_t list[16];
    __shared__ __attribute__((aligned(16))) v4f sums[kShrinkWaves / 2][RB][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x >> 6);
    int32_t n = 0;
    const int32_t id = find_tile<16>(p, blockIdx.y * kBlock, blockIdx.z, list, n);
    if (id < 0 || id == p.n_adapters) return;
    __syncthreads();

    const int32_t row = list[l16 < n ? l16 : n - 1];           // of y
    int32_t src = p.perm ? p.perm[row] : row;
    src = src >= 0 && src < p.T ? src : 0;
    const __half *xr = p.x + src * p.ldx, *ar[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = b * 16 + l16;
        ar[b] = p.a + (static_cast<int64_t>(id) * p.rank + (r < p.rank ? r : p.rank - 1)) * p.K;
    }
    v4f acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = v4f{0.f, 0.f, 0.f, 0.f};
    const int32_t units = (p.K + kUnit - 1) / kUnit, slice = blockIdx.x;
    const int32_t u0 = static_cast<int32_t>(static_cast<int64_t>(units) * slice / p.slices);
    const int32_t u1 = static_cast<int32_t>(static_cast<int64_t>(units) * (slice + 1) / p.slices);
    for (int32_t u = u0 + wave; u < u1; u += kShrinkWaves) {
        v8h xv[2], av[RB][2];
        // K is a multiple of 8; what lies behind it in the last unit is read from the row's last 8 channels and multiplied by zero
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int32_t k = u * kUnit + s * 32 + g * 8, at = k < p.K ? k : p.K - 8;
#pragma unroll
            for (int b = 0; b < RB; ++b) av[b][s] = *reinterpret_cast<const v8h *>(ar[b] + at);
            xv[s] = *reinterpret_cast<const v8h *>(xr + at);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if ((u + 1) * kUnit > p.K && u * kUnit + s * 32 + g * 8 >= p.K) xv[s] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < RB; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[s], av[b][s], acc[b], 0, 0, 0);
        }
    }
#pragma unroll
    for (int half = kShrinkWaves / 2; half >= 1; half >>= 1) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int b = 0; b < RB; ++b) sums[wave - half][b][lane] = acc[b];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int b = 0; b < RB; ++b) acc[b] += sums[wave][b][lane];
        __syncthreads();
    }
    if (wave != 0) return;
    float *h = p.h + static_cast<int64_t>(slice) * p.T * p.rank;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int j = g * 4 + r;                               // result register r of lane group g is row 4 g + r
        if (j < n)
#pragma unroll
            for (int b = 0; b < RB; ++b)
                if (b * 16 + l16 < p.rank) h[static_cast<int64_t>(list[j]) * p.rank + b * 16 + l16] = acc[b][r];
    }
}

// y of 16 rows and `cols` columns, 64 a wave.  Y^T = B_a h^T: rows of B_a are the A operand, rows of h the B operand, so that a lane is a row of
// y.  A-row rho of product s is column 32 (s / 2) + 8 (rho / 4) + 4 (s % 2) + rho % 4 of the 64: a lane's four products hold two times 8
// consecutive columns, 16 bytes each.  h goes in as two fp16 parts of h 2^-e, e per row from its largest value: what is lost is 2^-22 of
// that value, and no magnitude of h overflows.  Bound by latency: 4 rows of 4608 columns, rank 16, 5.1 us, 48 rows of 8192 columns 5.9
// (4.7 MB): adapter ids, then slices of h, then the products; base and B_a are on their way meanwhile.
template <int KS, bool VEC>
__global__ __launch_bounds__(kExpandWaves * 64) void lora_expand_kernel(Lora p)
{
    __shared__ int32_t list[16];
    __shared__ float factors[16];
    __shared__ __attribute__((aligned(16))) v8h parts[KS][2][64];
    __shared__ __attribute__((aligned(16))) float meet[kExpandWaves - 1][KS][64][8];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x >> 6);
    int32_t n = 0;
    const int32_t id = find_tile<16>(p, blockIdx.y * kBlock, blockIdx.z, list, n);
    if (id < 0) return;
    const bool none = id == p.n_adapters;
    if (none && p.y == p.base) return;
    __syncthreads();

    const bool mine = l16 < n;
    const int32_t row = list[mine ? l16 : n - 1];
    const __half *base = p.base + row * p.ldb;
    v8h bv[4][KS], bs[2];
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
        for (int w = 0; w < 2; ++w) {
            const int32_t col = c0 + w * 32 + g * 8;
            if constexpr (VEC) {
                bs[w] = *reinterpret_cast<const v8h *>(base + (col < p.N ? col : p.N - 8));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) bs[w][e] = *reinterpret_cast<const _Float16 *>(base + (col + e < p.N ? col + e : p.N - 1));
            }
        }
    };
    const int32_t first = blockIdx.x * p.cols, end = p.N - first < p.cols ? p.N : first + p.cols;
    load(first + wave * kCols);                                // on its way while the rows' parts are prepared

    // The slices of h are added by all waves, every fourth by each; their sums meet in LDS, and the first leaves the rows' parts where all
    // waves read them.
    float f[KS][8];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) f[s][e] = 0.0f;
    if (!none) {
        const int64_t slice = static_cast<int64_t>(p.T) * p.rank;
        const float *h = p.h + static_cast<int64_t>(row) * p.rank;
        constexpr int kAtOnce = KS <= 2 ? 4 : 2;
        for (int32_t c = wave; c < p.slices; c += kAtOnce * kExpandWaves) {
            v4f v[kAtOnce][KS][2];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int s = 0; s < KS; ++s) {                 // ranks and slices behind the last repeat it
                    const int r = s * 32 + g * 8, at_c = c + i * kExpandWaves;
                    const float *at = h + (at_c < p.slices ? at_c : c) * slice + (r < p.rank ? r : p.rank - 8);
                    v[i][s][0] = reinterpret_cast<const v4f *>(at)[0];
                    v[i][s][1] = reinterpret_cast<const v4f *>(at)[1];
                }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        f[s][e] += c + i * kExpandWaves < p.slices && s * 32 + g * 8 < p.rank ? v[i][s][e >> 2][e & 3] : 0.0f;
        }
    }
    if (wave > 0)
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) meet[wave - 1][s][lane][e] = f[s][e];
    __syncthreads();
    if (!none && wave == 0) {
#pragma unroll
        for (int o = 0; o < kExpandWaves - 1; ++o)
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) f[s][e] += meet[o][s][lane][e];
        float top = 0.0f, down, up;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[s][e]));
        scale_of(top, down, up);
        if (g == 0) factors[l16] = p.scale[id] * up;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            v8h hi, lo;
            split(f[s], down, hi, lo);
            parts[s][0][lane] = hi;
            parts[s][1][lane] = lo;
        }
    }
    __syncthreads();

    const float factor = factors[l16];
    __half *out = p.y + row * p.ldy;
    for (int32_t c0 = first + wave * kCols; c0 < end; c0 += kExpandWaves * kCols) {
        if (c0 != first + wave * kCols) load(c0);
        v4f acc[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[s] = v4f{0.f, 0.f, 0.f, 0.f};
        if (!none)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int part = 1; part >= 0; --part) {
                    const v8h hv = parts[k][part][lane];
#pragma unroll
                    for (int s = 0; s < 4; ++s) acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bv[s][k], hv, acc[s], 0, 0, 0);
                }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int32_t col = c0 + w * 32 + g * 8;
            v8h r = bs[w];
            if (!none)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[e] = static_cast<_Float16>(__builtin_fmaf(factor, acc[w * 2 + (e >> 2)][e & 3], static_cast<float>(r[e])));
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

// ------------------------------------------------------------------------------------------------ many rows
//
// Tiles of 64 rows, 16 a wave.  Straight loads of operands take 64 bytes of each of 16 rows an instruction, and the
// path to the registers then moves 15 bytes a clock (37 GB/s a compute unit, measured with 8 waves and 16 KiB in flight
// each); so here all that is read goes 256 bytes of a row at a time, by LDS-DMA or with 16 lanes to a row.
typedef const v8h __attribute__((address_space(3))) *v8h_lds_ptr;
constexpr int kRows = 64;
constexpr int kStage = 128;                // channels of K in LDS at a time, two buffers

template <int N>
__device__ __forceinline__ void wait_copies()
{
    wait_vmcnt<N>();
    asm volatile("" ::: "memory");
}

// h of 64 rows and a slice of K.  Chunk c (16 bytes) of row r lies at chunk c ^ (r & 15): a fragment read takes one chunk of 16 rows.
// 4096 rows of 3584 channels, rank 64: 12 us (29 MB of x, 2.5 TB/s): about one work-group to a compute unit, which waits for a stage of
// 32 KiB at a time (a wave waits 63 % of its life).  Three buffers are no faster where two work-groups still fit a compute unit
// (rank 16 8.1 / 8.6), and cost a second round of work-groups where they do not (rank 64 12.0 / 19.5).  Ranks beyond 64 are a second part, in work-groups of its own: 128 of them
// in one, with stages of 48 KiB and one work-group to a compute unit, took 26.0 us where two parts take 18.4.
template <int RB>
__global__ __launch_bounds__(256) void lora_shrink_rows_kernel(Lora p)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];           // two of: 64 rows of x, RB * 16 rows of A_a, 256 bytes each
    __shared__ int32_t list[kRows];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x >> 6);
    int32_t n = 0;
    const int32_t id = find_tile<kRows>(p, blockIdx.y * kBlock, blockIdx.z, list, n);
    if (id < 0 || id == p.n_adapters) return;
    __syncthreads();

    const int32_t parts = p.rank > RB * 16 ? 2 : 1, r0 = static_cast<int32_t>(blockIdx.x) % parts * RB * 16;    // first rank
    constexpr int kBuffer = (kRows + RB * 16) * 256;
    const uint32_t lds0 = lds_address(smem);
    const __half *xr[4], *ar[RB];                              // where this lane copies from: rows 4 i + g of the wave's 16, of each 16 of A_a
    int32_t xc[4], ac;                                         // and which chunk of them
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = wave * 16 + i * 4 + g;
        const int32_t row = list[j < n ? j : n - 1];
        int32_t src = p.perm ? p.perm[row] : row;
        src = src >= 0 && src < p.T ? src : 0;
        xr[i] = p.x + src * p.ldx;
        xc[i] = (l16 ^ (i * 4 + g)) * 8;
    }
    ac = (l16 ^ (wave * 4 + g)) * 8;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = r0 + b * 16 + wave * 4 + g;
        ar[b] = p.a + (static_cast<int64_t>(id) * p.rank + (r < p.rank ? r : p.rank - 1)) * p.K;
    }
    auto copy = [&](int32_t stage, int buffer) {               // channels behind K repeat its last 8
        const int32_t k = stage * kStage, last = p.K - 8;
        const uint32_t at = lds0 + buffer * kBuffer;
#pragma unroll
        for (int i = 0; i < 4; ++i) lds_dma16_lane_address(xr[i] + (k + xc[i] < p.K ? k + xc[i] : last), at + (wave * 4 + i) * 1024);
#pragma unroll
        for (int b = 0; b < RB; ++b)
            lds_dma16_lane_address(ar[b] + (k + ac < p.K ? k + ac : last), at + kRows * 256 + (b * 4 + wave) * 1024);
    };
    const int32_t stages = (p.K + kStage - 1) / kStage, slice = blockIdx.x / parts;
    const int32_t s0 = static_cast<int32_t>(static_cast<int64_t>(stages) * slice / p.slices);
    const int32_t s1 = static_cast<int32_t>(static_cast<int64_t>(stages) * (slice + 1) / p.slices);
    v4f acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = v4f{0.f, 0.f, 0.f, 0.f};
    if (s0 < s1) copy(s0, 0);
    for (int32_t s = s0; s < s1; ++s) {
        const int buffer = (s - s0) & 1;
        if (s + 1 < s1) {
            copy(s + 1, buffer ^ 1);
            wait_copies<4 + RB>();
        } else {
            wait_copies<0>();
        }
        __syncthreads();
        const uint32_t at = lds0 + buffer * kBuffer + l16 * 256;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const uint32_t chunk = ((ks * 4 + g) ^ l16) << 4;
            v8h xv = *(v8h_lds_ptr)(uintptr_t)(at + wave * 4096 + chunk);
            if (s * kStage + ks * 32 + g * 8 >= p.K) xv = v8h{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < RB; ++b)
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv, *(v8h_lds_ptr)(uintptr_t)(at + kRows * 256 + b * 4096 + chunk), acc[b], 0, 0, 0);
        }
        __syncthreads();
    }
    float *h = p.h + static_cast<int64_t>(slice) * p.T * p.rank;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int j = wave * 16 + g * 4 + r;                   // result register r of lane group g is row 4 g + r
        if (j < n)
#pragma unroll
            for (int b = 0; b < RB; ++b)
                if (r0 + b * 16 + l16 < p.rank) h[static_cast<int64_t>(list[j]) * p.rank + r0 + b * 16 + l16] = acc[b][r];
    }
}

// y of 64 rows and `cols` columns, 128 at a time.  Y = h B_a^T: 16 rows of h are the A operand (a wave prepares its own, in registers), rows of
// B_a the B operand, column 8 c + s of the 128 as column c of product s: a lane then holds 8 consecutive columns of four rows, and 16
// lanes a row, 256 bytes.  The 128 rows of B_a are one run of memory and are copied as such, in two buffers; chunk q (16 bytes) of them lies at q ^ h
// inside its 16, h counting the 8 rows before it, so that a fragment read, one chunk of 16 rows 8 apart, meets no bank twice.
// 4096 rows of 4608 columns, rank 64: 21 us, 75 MB of base and y, 3.6 TB/s; two products for the two parts of h, 512 columns behind one
// preparation of the rows.
template <int KS, bool VEC>
__global__ __launch_bounds__(256) void lora_expand_rows_kernel(Lora p)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];           // two of: 128 rows of B_a
    __shared__ int32_t list[kRows];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x >> 6);
    int32_t n = 0;
    const int32_t id = find_tile<kRows>(p, blockIdx.y * kBlock, blockIdx.z, list, n);
    if (id < 0) return;
    const bool none = id == p.n_adapters;
    if (none && p.y == p.base) return;
    __syncthreads();

    const int32_t chunks = p.rank / 8, pieces = chunks * 2;    // 1 KiB pieces of a block of 128 rows of B_a
    const int shift = 34 - __builtin_clz(chunks);              // h = q >> (3 + log2(chunks)): exact for powers of two, else some banks meet
    const uint32_t lds0 = lds_address(smem), buffer_bytes = pieces * 1024;
    const int32_t first = blockIdx.x * p.cols, end = p.N - first < p.cols ? p.N : first + p.cols, blocks = (end - first + 127) / 128;
    const int sh = shift < 4 ? 4 : shift;
    auto copy_b = [&](int32_t block, int buffer) {
        const uint8_t *from = reinterpret_cast<const uint8_t *>(p.b + (static_cast<int64_t>(id) * p.N + first + block * 128) * p.rank);
        const int32_t rest = p.N - first - block * 128, last = (rest < 128 ? rest : 128) * chunks - 1;     // chunks behind the last row repeat its last one
        for (int i = wave; i < pieces; i += 4) {
            const int32_t at = i * 64 + lane, q = (at & ~15) | ((at & 15) ^ ((at >> sh) & 15));
            lds_dma16_lane_address(from + static_cast<int64_t>(q < last ? q : last) * 16, lds0 + buffer * buffer_bytes + i * 1024);
        }
    };
    const int32_t rows = n - wave * 16 < 16 ? n - wave * 16 : 16;              // of this wave; may be none
    int32_t row[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int j = wave * 16 + g * 4 + r;
        row[r] = list[j < n ? j : n - 1];
    }
    v8h bs[4];
    auto load_base = [&](int32_t block) {                      // columns behind the last repeat it
        const int32_t col = first + block * 128 + l16 * 8;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const __half *base = p.base + row[r] * p.ldb;
            if constexpr (VEC) {
                bs[r] = *reinterpret_cast<const v8h *>(base + (col < p.N ? col : p.N - 8));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) bs[r][e] = *reinterpret_cast<const _Float16 *>(base + (col + e < p.N ? col + e : p.N - 1));
            }
        }
    };
    load_base(0);

    // ---- h of the wave's 16 rows, lane: row l16, ranks 8 g .. of every 32; two parts of h 2^-e
    v8h hi[KS], lo[KS];
    float factor[4] = {0.f, 0.f, 0.f, 0.f};
    if (!none) {
        // The slices are added as they lie in memory, 16 bytes a lane along the rows, and change over to the operand's order in LDS. (Read in
        // that order, 128 bytes of 16 rows a load, a slice took 0.5 us a work-group.)
        const int64_t slice = static_cast<int64_t>(p.T) * p.rank;
        const int32_t per_row = p.rank / 4, pitch = p.rank + 4;                // 16-byte pieces of a row; floats of it in LDS
        constexpr int NI = KS * 2;                             // pieces of a lane, at most
        const float *from[NI];
        v4f sum[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int32_t at = i * 64 + lane, j = wave * 16 + (at / per_row < 16 ? at / per_row : 15);
            from[i] = p.h + static_cast<int64_t>(list[j < n ? j : n - 1]) * p.rank + at % per_row * 4;
            sum[i] = v4f{0.f, 0.f, 0.f, 0.f};
        }
        constexpr int kAtOnce = KS == 1 ? 8 : KS == 2 ? 4 : 2;
        for (int32_t c = 0; c < p.slices; c += kAtOnce) {
            v4f v[kAtOnce][NI];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                for (int i = 0; i < NI; ++i)                   // slices behind the last repeat it
                    v[u][i] = *reinterpret_cast<const v4f *>(from[i] + (c + u < p.slices ? c + u : p.slices - 1) * slice);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
                if (c + u < p.slices)
#pragma unroll
                    for (int i = 0; i < NI; ++i) sum[i] += v[u][i];
        }
        float *mine = reinterpret_cast<float *>(smem) + wave * 16 * pitch;     // of this wave alone
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int32_t at = i * 64 + lane;
            if (at < 16 * per_row) *reinterpret_cast<v4f *>(mine + at / per_row * pitch + at % per_row * 4) = sum[i];
        }
        float f[KS][8], top = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int r = s * 32 + g * 8;
            const float *at = mine + l16 * pitch + (r < p.rank ? r : 0);
            const v4f f0 = reinterpret_cast<const v4f *>(at)[0], f1 = reinterpret_cast<const v4f *>(at)[1];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[s][e] = r < p.rank ? (e < 4 ? f0[e & 3] : f1[e & 3]) : 0.0f;
        }
        const float scale = p.scale[id];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[s][e]));
        float down, up;
        scale_of(top, down, up);
#pragma unroll
        for (int s = 0; s < KS; ++s) split(f[s], down, hi[s], lo[s]);
#pragma unroll
        for (int r = 0; r < 4; ++r) factor[r] = scale * __shfl(up, g * 4 + r, 64);
        wait_copies<0>();                                      // from here on the loop counts what it asks for itself
        __syncthreads();                                       // all waves are done with their sums
        copy_b(0, 0);
    }

    for (int32_t block = 0; block < blocks; ++block) {
        const int buffer = block & 1;
        v4f acc[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) acc[s] = v4f{0.f, 0.f, 0.f, 0.f};
        if (!none) {
            // This block's rows of B_a: behind them at most the base's four loads and the stores of the block before were issued
            if (block == 0) wait_copies<0>();
            else wait_copies<4>();
            __syncthreads();                                   // they are there for all waves, and the other buffer is free
            if (block + 1 < blocks) copy_b(block + 1, buffer ^ 1);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bool in = k * 32 + g * 8 < p.rank;
                const int32_t c = in ? k * 4 + g : chunks - 1;
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const int32_t q = (l16 * 8 + s) * chunks + c, at = (q & ~15) | ((q & 15) ^ ((q >> sh) & 15));
                    const v8h bv = *(v8h_lds_ptr)(uintptr_t)(lds0 + buffer * buffer_bytes + at * 16);
                    acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[k], bv, acc[s], 0, 0, 0);
                    acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[k], bv, acc[s], 0, 0, 0);
                }
            }
        }
        const int32_t col = first + block * 128 + l16 * 8;
        v8h out[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            out[r] = bs[r];
            if (!none)
#pragma unroll
                for (int e = 0; e < 8; ++e) out[r][e] = static_cast<_Float16>(__builtin_fmaf(factor[r], acc[e][r], static_cast<float>(bs[r][e])));
        }
        if (block + 1 < blocks) load_base(block + 1);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            __half *y = p.y + row[r] * p.ldy;
            const bool mine = g * 4 + r < rows;
            if constexpr (VEC) {
                if (mine && col < end) __builtin_nontemporal_store(out[r], reinterpret_cast<v8h *>(y + col));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (mine && col + e < end) *reinterpret_cast<_Float16 *>(y + col + e) = out[r][e];
            }
        }
    }
}

// Few rows: tiles of 16, and slices of K short enough that each wave has about one unit.
int64_t few_slices(int32_t K)
{
    const int64_t s = ceil_div(K, kUnit * kShrinkWaves);
    return s < kMaxSlices ? s : kMaxSlices;
}

// Many: tiles of 64; a slice's stage takes 0.55 us and every slice costs the expansion 0.28, so about sqrt(2 stages) slices (rank 64, K = 3584,
// 28 stages, shrink + expansion in us with 2 / 4 / 8 / 14 slices: 512 rows 25.2 / 20.6 / 19.8 / 21.7, 1024 26.2 / 22.3 / 22.2 / 24.9), but no
// more than give every compute unit a work-group (4096 rows: 4 slices 33.2, 8 41.9).  Two parts of the rank cost twice in the expansion (rank
// 128 with 2 / 3 / 4 slices: 2889 rows 40.0 / 40.2 / 39.3, 4096 48.6 / 48.6 / 54.1, 1000 29.4 / 27.2 / 25.5 and 28.2 with 8).
constexpr int32_t kManyRank = 64;          // ranks of a part
int64_t rank_parts(int32_t rank) { return rank > kManyRank ? 2 : 1; }
int64_t wanted_slices(int32_t K, int64_t parts)
{
    return static_cast<int64_t>(ceil(sqrt(2.0 * static_cast<double>(ceil_div(K, kStage)) / static_cast<double>(parts))));
}
int64_t many_slices(int32_t T, int32_t K, int32_t rank)
{
    int64_t s = wanted_slices(K, rank_parts(rank));
    const int64_t most = kNumCU / (ceil_div(T, kRows) * rank_parts(rank));
    if (s > most) s = most;
    return s < 1 ? 1 : s;
}

// The most that T rows or fewer have of rows times slices: s slices go with up to kNumCU / (s parts) tiles.
int64_t most_row_slices(int32_t T, int32_t K, int64_t parts)
{
    int64_t most = 0, s = wanted_slices(K, parts);
    if (s > kNumCU / parts) s = kNumCU / parts;
    for (; s > 1; --s) {
        const int64_t rows = static_cast<int32_t>(kNumCU) / static_cast<int32_t>(s * parts) * kRows;
        if (T <= rows) break;
        if (s * rows > most) most = s * rows;
    }
    return s * T > most ? s * T : most;
}

// Tiles of 16 rows or of 64: 64 where they are full.  Tiles of 64 / of 16, shrink + expansion in us, K = 3584, N = 4608, rank 16 and 64, 4 adapters:
// 128 rows 10.2 / 9.6 and 14.5 / 13.4, 256 10.6 / 10.9 and 14.9 / 16.5, 512 11.3 / 13.2 and 16.6 / 22.1; 64 adapters, each row another:
// 128 rows 52.4 / 35.8 and 61.0 / 42.7, 512 89 / 61 and 111 / 73, 1024 108 / 107 and 141 / 132.
// The host knows how many adapters there are, not how many the rows use, and takes the one for the other, here and for the tiles of the grids.  Where far
// more are loaded than used that is wrong (K = 3584, N = 4608, rank 64, us): 4096 rows of 5 adapters, 5 / 500 loaded, 34.5 / 104 (26 times the
// work-groups, nearly all of which find no tile), 256 rows of 5 16.3 / 27.8, 1000 rows of one, 1 / 64 loaded, 20.0 / 36.1; up to 48 rows no difference.
constexpr int32_t kFewMax = 1024;
bool few_rows(int32_t T, int32_t n_adapters) { return T <= 128 || (T <= kFewMax && n_adapters >= T / 16); }

// The expansion on its own: with many columns reading B_a for 64 rows at once is worth empty places in a tile from a few tiles of 16 on (N = 37888,
// tiles of 64 / of 16, rank 16 and 64: 100 rows of one adapter 7.6 / 9.3 and 10.1 / 18.6, 156 rows of 15 adapters, each another, 22.5 / 18.9
// and 31.0 / 33.1, 300 of 20 39.7 / 53.7 and 54.3 / 84.5).
bool few_rows_to_expand(int32_t T, int32_t N, int32_t n_adapters) { return T <= 64 || (N < 16384 && few_rows(T, n_adapters)); }

template <int RB>
int launch_shrink(const Lora &a, dim3 grid, hipStream_t stream)
{
    MQ_LAUNCH(lora_shrink_kernel<RB>, grid, dim3(kShrinkWaves * 64), 0, stream, a);
    return launch_status();
}

template <int RB>
int launch_shrink_rows(const Lora &a, dim3 grid, hipStream_t stream)
{
    constexpr int lds = 2 * (kRows + RB * 16) * 256;
    auto kern = lora_shrink_rows_kernel<RB>;
    if constexpr (lds >= 60 * 1024) {                          // next to the list of rows
        static LdsLimit limit;
        if (const int st = limit.raise(reinterpret_cast<const void *>(kern), lds); st != MQUANT_OK) return st;
    }
    MQ_LAUNCH(kern, grid, dim3(256), lds, stream, a);
    return launch_status();
}

template <int KS, bool VEC>
int launch_expand(const Lora &a, bool few, dim3 grid, hipStream_t stream)
{
    if (few) MQ_LAUNCH((lora_expand_kernel<KS, VEC>), grid, dim3(kExpandWaves * 64), 0, stream, a);
    else {
        auto kern = lora_expand_rows_kernel<KS, VEC>;
        if constexpr (KS == 4) {
            static LdsLimit limit;
            if (const int st = limit.raise(reinterpret_cast<const void *>(kern), 2 * 256 * 128); st != MQUANT_OK) return st;
        }
        MQ_LAUNCH(kern, grid, dim3(256), 2 * 256 * a.rank, stream, a);
    }
    return launch_status();
}

}  // namespace

extern "C" int64_t mquant_lora_workspace_bytes(int32_t T, int32_t K, int32_t rank)
{
    if (T < 0 || K < 0 || rank < 1) return MQUANT_ERR_BAD_SHAPE;
    if (K == 0 || K % 8 != 0 || rank % 8 != 0 || rank > 128) return MQUANT_ERR_UNSUPPORTED;
    if (T == 0) return 0;
    // whichever way the number of adapters chooses, and no less than fewer rows or lower ranks take: scratch for the largest step does for all
    const int64_t few = few_slices(K) * (T < kFewMax ? T : kFewMax), many = most_row_slices(T, K, rank_parts(rank));
    int64_t floats = (few > many ? few : many) * rank;
    if (rank > kManyRank) {
        const int64_t lower = most_row_slices(T, K, 1) * kManyRank;
        if (lower > floats) floats = lower;
    }
    return ceil_div(floats * 4, 256) * 256;
}

extern "C" int mquant_lora_apply(const void *x, int64_t ldx, const int32_t *perm, const int32_t *adapter, const void *a, const void *b,
                                 const float *scale, const void *base, int64_t ldb, void *y, int64_t ldy, int32_t T, int32_t N,
                                 int32_t K, int32_t rank, int32_t n_adapters, void *workspace, int64_t workspace_bytes,
                                 mquant_stream_t stream_)
{
    if (N < 0 || n_adapters < 0) return MQUANT_ERR_BAD_SHAPE;
    const int64_t need = mquant_lora_workspace_bytes(T, K, rank);
    if (need < 0) return static_cast<int>(need);
    if (N > kMaxSide || K > kMaxSide) return MQUANT_ERR_UNSUPPORTED;
    if (T == 0 || N == 0) return MQUANT_OK;
    if (!x || !adapter || !base || !y || (n_adapters > 0 && (!a || !b || !scale))) return MQUANT_ERR_NULL;
    if (ldx < K || ldb < N || ldy < N || (y == base && ldy != ldb)) return MQUANT_ERR_BAD_SHAPE;
    if (ldx % 8 != 0 || !aligned_to(x, 16) || !aligned_to(a, 16) || !aligned_to(b, 16) || !aligned_to(base, 2) || !aligned_to(y, 2) ||
        !aligned_to(adapter, 4) || !aligned_to(perm, 4) || !aligned_to(scale, 4))
        return MQUANT_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < need) return MQUANT_ERR_WORKSPACE;
    if (!aligned_to(workspace, 256)) return MQUANT_ERR_ALIGNMENT;
    hipStream_t stream = static_cast<hipStream_t>(stream_);

    const bool few = few_rows(T, n_adapters), few_to_expand = few_rows_to_expand(T, N, n_adapters);
    Lora args = {static_cast<const __half *>(x), ldx, perm, adapter, static_cast<const __half *>(a), static_cast<const __half *>(b), scale,
                 static_cast<const __half *>(base), ldb, static_cast<__half *>(y), ldy, static_cast<float *>(workspace), T, N, K, rank,
                 n_adapters, static_cast<int32_t>(few ? few_slices(K) : many_slices(T, K, rank)),
                 few_to_expand ? kExpandWaves * kCols : rank > 64 ? 1024 : 512};
    // Few rows: a block of columns a wave, two of many columns (34 rows of 12 adapters, rank 32, N = 37888, one / two / four: 11.4 / 8.5 / 9.0 us, 64 of 3,
    // rank 64, 15.7 / 12.4 / 12.7, 4 of 4, rank 16, 4.6 / 4.9 / 5.8; N = 10240, 48 of 12, rank 16, 5.8 / 5.9 / 6.8).
    if (few_to_expand && N >= 16384 && T > 8) args.cols *= 2;
    // Many rows: 512 columns a work-group, which prepares its rows once for all of them, fewer where that leaves compute units idle (K = 3584,
    // N = 4608, rank 64, expansion with 128 / 256 / 512 / 1024 columns: 128 rows 9.1 / 10.4 / 13.4 / 18.9 us, 1024 15.7 / 14.8 / 16.3 / 21.2, 4096
    // 28.2 / 24.4 / 21.7 / 23.1; rank 128, 4096 rows, 512 / 1024: 35.9 / 30.7).
    while (!few_to_expand && args.cols > 128 && ceil_div(T, kRows) * ceil_div(N, args.cols) < kNumCU) args.cols /= 2;
    const int64_t blocks = ceil_div(T, kBlock), chunks = ceil_div(N, args.cols);
    if (blocks > 65535) return MQUANT_ERR_UNSUPPORTED;
    // Tiles of 256 rows: full ones, and a last one of every adapter (and of the rows without), which may not be there: those come last in
    // the grids.
    auto tiles = [&](int32_t rows) {
        const int32_t in_block = T < kBlock ? T : kBlock;
        return static_cast<unsigned>(in_block / rows + (n_adapters < in_block ? n_adapters + 1 : in_block));
    };
    if (n_adapters > 0) {
        const dim3 grid(static_cast<unsigned>(args.slices * (few ? 1 : rank_parts(rank))), static_cast<unsigned>(blocks), tiles(few ? 16 : kRows));
        const int st = few ? (rank <= 16 ? launch_shrink<1>(args, grid, stream) : rank <= 32 ? launch_shrink<2>(args, grid, stream)
                              : rank <= 64 ? launch_shrink<4>(args, grid, stream) : launch_shrink<8>(args, grid, stream))
                     : rank <= 16 ? launch_shrink_rows<1>(args, grid, stream) : rank <= 32 ? launch_shrink_rows<2>(args, grid, stream)
                                  : launch_shrink_rows<kManyRank / 16>(args, grid, stream);
        if (st != MQUANT_OK) return st;
    }
    const dim3 grid(static_cast<unsigned>(chunks), static_cast<unsigned>(blocks), tiles(few_to_expand ? 16 : kRows));
    if (N % 8 == 0 && ldb % 8 == 0 && ldy % 8 == 0 && aligned_to(base, 16) && aligned_to(y, 16))
        return rank <= 32 ? launch_expand<1, true>(args, few_to_expand, grid, stream)
             : rank <= 64 ? launch_expand<2, true>(args, few_to_expand, grid, stream) : launch_expand<4, true>(args, few_to_expand, grid, stream);
    return rank <= 32 ? launch_expand<1, false>(args, few_to_expand, grid, stream)
         : rank <= 64 ? launch_expand<2, false>(args, few_to_expand, grid, stream) : launch_expand<4, false>(args, few_to_expand, grid, stream);
}
