// Attention of a step's rows over a paged cache, for gfx950.
//
// Row i of sequence s sees the slots j <= pos[i] of its sequence: o = sum_j p_j v_j, p = softmax(q k_j / sqrt(128)), in
// one pass over the slots with the running maximum and sum of the softmax (fp32), fp16 matrix operands.  The
// heads that share a key/value head read the same slots, so the queries of a (sequence, key/value head) are the
// pairs (row, head of the group), row-major: query m is row m / G, head m % G.  Two kernels:
//   paged_few_kernel    sequences of at most kFew queries (decode, drafted tokens): a wave walks 32 slots at a time by
//                       itself, bound by the bytes of the cache;
//   paged_chunk_kernel  the others: 128 queries a work-group, 64 slots a tile, bound by the matrix cores.
// Both split the slots of a sequence into pieces where there are too few work-groups otherwise; the pieces' partial
// results (unnormalised sums, maximum, denominator, fp32) meet in paged_combine_kernel.
#include <climits>
#include <cmath>

#include "lds_dma.h"
#include "serving_common.h"

using namespace mquant;

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef __fp16 tr4 __attribute__((vector_size(8)));
typedef tr4 __attribute__((address_space(3))) *tr4_lds_ptr;
typedef const v8h __attribute__((address_space(3))) *v8h_lds_ptr;
typedef v4u __attribute__((address_space(3))) *v4u_lds_ptr;

constexpr int kD = kCacheHeadDim;
constexpr int kFew = 48;                   // queries of a (sequence, key/value head) up to which paged_few_kernel takes it
constexpr int kFewSlots = 32;              // slots a wave takes at a time
constexpr int kFewWaves = 4;
constexpr int kFewStep = kFewSlots * kFewWaves;
constexpr int kFewLds = kFewWaves * 2 * kFewSlots * 256;
constexpr int kFewPitch = kD + 4;          // floats of a query's row where the waves meet
constexpr int kChunkQ = 128;               // queries of a work-group (32 a wave)
constexpr int kChunkK = 64;                // slots of a tile
constexpr int kTileBytes = kChunkK * 256;
constexpr int kChunkLds = 4 * kTileBytes;  // two key and two value tiles
constexpr int kAhead = 4;                  // LDS fragment reads in flight ahead of the MFMA that uses them

// The running maximum that the sums are scaled to follows the true one lazily: only when some query's has grown by more
// than kLazy (a factor 2^8 in the probabilities, harmless in fp16 and fp32) are the sums rescaled.  The exponents see it
// times scale_log2e and rounded, in eighths at a score of 8e6: so sums meet under a factor of the rounded products' difference (exact where the
// factor matters), under one of the maxima's own they would be up to 2^(1/8) apart.  No product is contracted into an addition here (-ffp-contract=off).
constexpr float kLazy = 8.0f;

struct Step {
    const __half *q;
    int64_t ldq, ldo;
    __half *o;
    const int32_t *row_start, *pos;
    int32_t T, n_q, group;                 // group: query heads per key/value head
    float scale_log2e;
    PagedCache c;
    // pieces of slots: how many at most, slots of one, and the partial results of (piece, query): sums [128], then (what they are scaled to, denominator)
    int32_t n_split, piece;
    int32_t few_stride;                    // queries of a (sequence, key/value head) that have room among the partial results
    int32_t all;                           // this kernel takes every sequence, whatever its rows
    float *part;
    float2 *part_ml;
};

__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// Waits for all but N of this wave's copies to LDS; nothing that reads or writes memory moves across.
template <int N>
__device__ __forceinline__ void wait_copies()
{
    wait_vmcnt<N>();
    asm volatile("" ::: "memory");
}

// Rows of a sequence: first and behind the last, inside [0, T).
__device__ __forceinline__ int2 rows_of(const Step &a, int32_t seq)
{
    const int32_t b = a.row_start[seq], e = a.row_start[seq + 1];
    return make_int2(b > 0 ? b : 0, e < a.T ? e : a.T);
}

// Last slot that a row sees, -1: none.
__device__ __forceinline__ int32_t limit_of(const Step &a, int32_t row)
{
    const int32_t p = a.pos[row], last = (a.c.table_pages << a.c.page_shift) - 1;
    return p < 0 ? -1 : p < last ? p : last;
}

// The 16 slots block * 16 .. of a sequence, as the number of 4 KiB blocks before them in a page array.  A block behind the table
// repeats its last one, a page id out of range is page 0: any block is memory of the cache, and what a row does not see
// is not used.
__device__ __forceinline__ uint32_t block_at(const Step &a, int32_t seq, int32_t kvh, int32_t block)
{
    const int32_t shift = a.c.page_shift - 4, last = (a.c.table_pages << shift) - 1, b = block < last ? block : last;
    const int32_t id = a.c.table[static_cast<int64_t>(seq) * a.c.table_pages + (b >> shift)];
    const uint32_t page = static_cast<uint32_t>(id) < static_cast<uint32_t>(a.c.n_pages) ? id : 0;
    return (page * static_cast<uint32_t>(a.c.n_kv_heads) + kvh) * (1u << shift) + (b & ((1 << shift) - 1));
}

__device__ __forceinline__ const uint8_t *block_ptr(const __half *pages, uint32_t block)
{
    return reinterpret_cast<const uint8_t *>(pages) + (static_cast<uint64_t>(block) << 12);
}

__device__ __forceinline__ int32_t pieces_of(const Step &a, int32_t limit)
{
    if (limit < 0) return 0;
    const int32_t n = limit / a.piece + 1;
    return n < a.n_split ? n : a.n_split;
}

// ------------------------------------------------------------------------------------------------ few queries
//
// A work-group: one (sequence, key/value head) and one piece of its slots; wave w takes the 32 slots w, w + 4, ... of it, with
// 16 KiB of LDS of its own for them, so the waves run without barriers:
//   S^T = K Q^T     A = 16 slots from LDS, B = Q^T in registers: a lane is a query, its registers are slots
//   O^T += V^T P^T  B = the same registers as fp16, A = V^T by transposing LDS reads.
// Copies of the next 32 keys start when the fragments of this tile are in registers, those of the values behind the last
// product, so about 14 of the 16 KiB are in flight all the time, for 8 waves a compute unit.
// Key chunk c (16 bytes) of row r lies at chunk c ^ (r & 15): a fragment read takes one chunk of 16 rows.  Value chunk c lies
// at c ^ 2 (r & 7): a transposing read takes 32 bytes of 8 rows.
// Bound by the bytes of the cache where they are many: 32 sequences of 500 to 16384 slots, 64 heads on 8 (633 MB), 126 us with the
// join, 5.0 TB/s (a device copy 4.9).  One row over 1281 slots is five trips to memory, one behind another, and two launches: 8.0 us.
// NQ: 16 queries each, all of them computed, whatever a sequence has: skipping by branches those behind the last query cost the
// others the overlap of their products and exponentials (20.4 against 17.7 us at 8 sequences of 5 rows x 28 heads over 4096 slots), and
// a form for each number beside one another gave nothing (32 sequences of one row among one of 512, 8000 slots each: 194 and 193 us).
template <int NQ>
__global__ __launch_bounds__(kFewWaves * 64, 2) void paged_few_kernel(Step a)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = uniform(tid >> 6);
    const int32_t units = a.c.n_seq * a.c.n_kv_heads;
    const int32_t unit = blockIdx.x % units, piece = blockIdx.x / units;
    const int32_t seq = unit / a.c.n_kv_heads, kvh = unit % a.c.n_kv_heads;
    const int2 rows = rows_of(a, seq);
    if (rows.x >= rows.y) return;
    const int32_t M = (rows.y - rows.x) * a.group;
    if (!a.all && M > kFew) return;

    const uint32_t k_lds = lds_address(smem) + wave * (2 * kFewSlots * 256), v_lds = k_lds + kFewSlots * 256;
    uint32_t k_off[4], v_off[4];                               // where a lane reads in a block of 16 rows
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 4 + g;
        k_off[i] = r * 256 + ((l16 ^ r) << 4);
        v_off[i] = r * 256 + ((l16 ^ ((r & 7) << 1)) << 4);
    }
    for (int32_t m0 = 0; m0 < M; m0 += 16 * NQ) {
        const int nq = M - m0 < 16 * NQ ? (M - m0 + 15) / 16 : NQ;
        const bool split = m0 + 16 * NQ <= a.few_stride;       // the others' slots are all in piece 0
        if (!split && piece > 0) return;
        // page ids, queries and positions are on their way together
        const int32_t begin = split ? piece * a.piece : 0;     // slots, a multiple of kFewStep
        const int32_t first = begin / kFewSlots + wave;
        // lane 2 i + b: block b of this wave's tile i; 32 tiles (4096 slots of the work-group) a time
        auto blocks_from = [&](int32_t tile0) { return block_at(a, seq, kvh, (tile0 + (lane >> 1) * kFewWaves) * 2 + (lane & 1)); };
        uint32_t blocks = blocks_from(first);
        v8h qf[NQ][4];
        int32_t lim[NQ], top = -1, low = INT_MAX;
#pragma unroll
        for (int u = 0; u < NQ; ++u) {
            const int32_t m = m0 + u * 16 + l16, mc = m < M ? m : M - 1;
            const int32_t row = rows.x + mc / a.group;
            const __half *qp = a.q + row * a.ldq + static_cast<int64_t>(kvh * a.group + mc % a.group) * kD + g * 8;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) qf[u][ks] = *reinterpret_cast<const v8h *>(qp + ks * 32);
            lim[u] = limit_of(a, row);
        }
#pragma unroll
        for (int u = 0; u < NQ; ++u) {
            top = lim[u] > top ? lim[u] : top;
            low = lim[u] < low ? lim[u] : low;
        }
        top = uniform(row16_max(top));
        low = uniform(row16_min(low));
        if (begin > top && piece > 0) continue;
        const int32_t end = !split || piece == a.n_split - 1 || top < begin + a.piece ? top + 1 : begin + a.piece;
        const int32_t n_tiles = (end + kFewSlots - 1) / kFewSlots;

        v4f acc[NQ][8];
        float m_ref[NQ], l_run[NQ];
#pragma unroll
        for (int u = 0; u < NQ; ++u) {
            m_ref[u] = -INFINITY;
            l_run[u] = 0.0f;
#pragma unroll
            for (int cb = 0; cb < 8; ++cb) acc[u][cb] = v4f{0.f, 0.f, 0.f, 0.f};
        }
        const float lazy_raw = kLazy / a.scale_log2e;
        for (int32_t tile0 = first; tile0 < n_tiles; tile0 += 32 * kFewWaves) {
            if (tile0 != first) blocks = blocks_from(tile0);
            auto copy = [&](const __half *pages, const uint32_t (&off)[4], uint32_t lds, int it) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint8_t *base = block_ptr(pages, __builtin_amdgcn_readlane(blocks, 2 * it + b));
#pragma unroll
                    for (int i = 0; i < 4; ++i) lds_dma16_uniform_base(base, off[i], lds + b * 4096 + i * 1024);
                }
            };
            wait_copies<0>();                                  // the page ids too: behind this the loop counts copies only
            int n = (n_tiles - tile0 + kFewWaves - 1) / kFewWaves;
            if (n > 32) n = 32;
            copy(a.c.k, k_off, k_lds, 0);
            copy(a.c.v, v_off, v_lds, 0);
            for (int it = 0; it < n; ++it) {
                const int32_t slot0 = (tile0 + it * kFewWaves) * kFewSlots;
                wait_copies<8>();                              // keys are there, values may be on the way
                // For the compiler, other addresses in every tile: the sums of each fragment read, held through the walk, and those of the
                // way out below spilled ten registers at NQ = 3 (11 % of the time of 35 queries over 4096 slots).
                uint32_t k_at = k_lds + l16 * 256, v_at = v_lds;
                asm volatile("" : "+v"(k_at), "+v"(v_at));
                v8h kf[2][4];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        kf[kb][ks] = *(v8h_lds_ptr)(uintptr_t)(k_at + kb * 4096 + (((ks * 4 + g) ^ l16) << 4));
                wait_lgkm0();
                asm volatile("" ::: "memory");
                const bool more = it + 1 < n;
                if (more) copy(a.c.k, k_off, k_lds, it + 1);
                v8h p[NQ];
#pragma unroll
                for (int u = 0; u < NQ; ++u) {
                    v4f s[2] = {v4f{0.f, 0.f, 0.f, 0.f}, v4f{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                        for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[kb][ks], qf[u][ks], s[kb], 0, 0, 0);
                    if (slot0 + kFewSlots - 1 > low) {         // some query does not see some slot
                        const int32_t room = lim[u] - slot0 - 4 * g;
#pragma unroll
                        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (kb * 16 + r > room) s[kb][r] = -INFINITY;
                    }
                    float m = m_ref[u];
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int r = 0; r < 4; ++r) m = fmaxf(m, s[kb][r]);
                    if (__any(m > m_ref[u] + lazy_raw)) {      // also the first visible slot (m_ref = -inf)
                        m = fmaxf(m, __shfl_xor(m, 16, 64));
                        m = fmaxf(m, __shfl_xor(m, 32, 64));
                        const float alpha = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_ref[u] * a.scale_log2e - m * a.scale_log2e);
                        l_run[u] *= alpha;
#pragma unroll
                        for (int cb = 0; cb < 8; ++cb) acc[u][cb] *= alpha;
                        m_ref[u] = m;
                    }
                    const float neg = m_ref[u] == -INFINITY ? 0.0f : -m_ref[u] * a.scale_log2e;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v2h ph;                                // the denominator sums the probabilities as the product sees them
                        ph[0] = static_cast<_Float16>(__builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 1][(e & 1) * 2], a.scale_log2e, neg)));
                        ph[1] = static_cast<_Float16>(__builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 1][(e & 1) * 2 + 1], a.scale_log2e, neg)));
                        l_run[u] = __builtin_amdgcn_fdot2(ph, v2h{1, 1}, l_run[u], false);
                        p[u][e * 2] = ph[0];
                        p[u][e * 2 + 1] = ph[1];
                    }
                }
                if (more) wait_copies<8>();
                else wait_copies<0>();
                if (slot0 + kFewSlots > top + 1) {             // values behind the last slot may be anything: zero times NaN
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (slot0 + b * 16 + i * 4 + g > top)
                                *(v4u_lds_ptr)(uintptr_t)(v_lds + b * 4096 + i * 1024 + lane * 16) = v4u{0, 0, 0, 0};
                    asm volatile("" ::: "memory");
                }
                // Operand slot j of lane group g is the slot that score register j holds there: 4 g + j, 16 + 4 g + j - 4.  A transposing
                // read takes, per 16 lanes, the 32 bytes of four rows that lanes 4 r .. 4 r + 3 point at, and gives lane i channel i.
                const int vr = 4 * g + ((lane >> 2) & 3);
                const uint32_t v_row = v_at + vr * 256 + (lane & 1) * 8;
#pragma unroll
                for (int cb = 0; cb < 8; ++cb) {
                    union {
                        tr4 h[2];
                        v8h f8;
                    } vf;
                    const uint32_t at = v_row + (((cb * 2 + ((lane >> 1) & 1)) ^ ((vr & 7) << 1)) << 4);
                    vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4f16((tr4_lds_ptr)(uintptr_t)at);
                    vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4f16((tr4_lds_ptr)(uintptr_t)(at + 4096));
#pragma unroll
                    for (int u = 0; u < NQ; ++u)
                        acc[u][cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf.f8, p[u], acc[u][cb], 0, 0, 0);
                }
                wait_lgkm0();
                asm volatile("" ::: "memory");
                if (more) copy(a.c.v, v_off, v_lds, it + 1);
            }
        }

        // ---- the four waves meet in LDS, 16 queries at a time: thread t finishes 8 channels of query t / 16
        int t = tid;
        asm volatile("" : "+v"(t));                            // what is worked out from it is not held through the walk
        const int my_q = t & 15, my_ch = (t >> 4 & 3) * 4;
        float *sums = reinterpret_cast<float *>(smem);                          // [4][16][kFewPitch]
        float2 *ml = reinterpret_cast<float2 *>(smem + kFewWaves * 16 * kFewPitch * 4);        // [4][16]
        int32_t *lims = reinterpret_cast<int32_t *>(ml + kFewWaves * 16);       // [16]
        static_assert(kFewWaves * 16 * (kFewPitch * 4 + 8) + 16 * 4 <= kFewLds, "exchange of the waves");
#pragma unroll
        for (int u = 0; u < NQ; ++u) {
            if (u >= nq) break;
            float l = l_run[u];
            l += __shfl_xor(l, 16, 64);
            l += __shfl_xor(l, 32, 64);
            __syncthreads();
#pragma unroll
            for (int cb = 0; cb < 8; ++cb)
                *reinterpret_cast<v4f *>(sums + (wave * 16 + my_q) * kFewPitch + cb * 16 + my_ch) = acc[u][cb];
            if (my_ch == 0) ml[wave * 16 + my_q] = make_float2(m_ref[u] * a.scale_log2e, l);
            if (t < 16) lims[t] = lim[u];
            __syncthreads();
            const int qi = t >> 4, ch = (t & 15) * 8;
            const int32_t m = m0 + u * 16 + qi;
            if (m < M) {
                float top_m = -INFINITY, den = 0.0f, f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) top_m = fmaxf(top_m, ml[w * 16 + qi].x);
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) {
                    const float2 x = ml[w * 16 + qi];
                    const float share = x.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x.x - top_m);
                    den += share * x.y;
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] += share * sums[(w * 16 + qi) * kFewPitch + ch + e];
                }
                const int32_t row = rows.x + m / a.group, limit = lims[qi];
                if (!split || pieces_of(a, limit) <= 1) {
                    if (piece == 0) {
                        const float inv = den > 0.0f ? 1.0f / den : 0.0f;       // a row that sees nothing: zeros
                        __half *out = a.o + row * a.ldo + static_cast<int64_t>(kvh * a.group + m % a.group) * kD + ch;
                        __half h[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) h[e] = __float2half_rn(f[e] * inv);
                        reinterpret_cast<uint2 *>(out)[0] = reinterpret_cast<const uint2 *>(h)[0];
                        reinterpret_cast<uint2 *>(out)[1] = reinterpret_cast<const uint2 *>(h)[1];
                    }
                } else if (limit >= begin) {
                    const int64_t at = (static_cast<int64_t>(piece) * units + unit) * a.few_stride + m;
                    *reinterpret_cast<v4f *>(a.part + at * kD + ch) = v4f{f[0], f[1], f[2], f[3]};
                    *reinterpret_cast<v4f *>(a.part + at * kD + ch + 4) = v4f{f[4], f[5], f[6], f[7]};
                    if (ch == 0) a.part_ml[at] = make_float2(top_m, den);
                }
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ chunks
//
// A work-group: 128 queries of a (sequence, key/value head), four waves of 32, and one piece of the slots; the 64 slots of a tile
// are shared by the waves through LDS.  S^T = K Q^T, softmax, O^T += V^T P^T with 32x32x16 products: a lane is a query, so its
// statistics live in one lane pair and the rescale needs no lane exchange.  While the exponentials of tile j run on the
// vector ALU the matrix core computes the scores of tile j + 1 (written interleaved and pinned).  Tiles come by LDS-DMA, two
// buffers each, keys one step ahead of values, one barrier a tile.
// Consecutive queries are the group's heads of one row, then of the next: a work-group spans 128 / G rows whose limits lie
// close together, so it walks its tiles without skipping any for single waves, and only the last tiles are compared slot by slot.
// Bound by the power of the matrix cores: 4096 rows x 64 heads on 16384 slots 1750 to 1930 us by card, 1.0 to 1.1 PFLOP/s, as a large
// library product; an MFMA is in the matrix pipes 63 % of the cycles, the vector pipes are busy 54 %, the clock is 1.55 GHz.  Few
// work-groups wait for a step's copies instead (KG = 2: two key groups of four waves, which meet in LDS, for those).
__device__ __forceinline__ void halves_of(float x, float &lo, float &hi)
{
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    lo = __int_as_float(sw[0]);
    hi = __int_as_float(sw[1]);
}

// MFMA 32x32 result register r of lane group g holds row (r/4)*8 + g*4 + r%4.
__device__ __forceinline__ int acc_row(int r, int g) { return (r >> 2) * 8 + g * 4 + (r & 3); }

template <int KG>
__global__ __launch_bounds__(KG * 256, 2) void paged_chunk_kernel(Step a, int32_t xcds_per_kv)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];           // KG * kChunkLds
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = uniform((tid >> 6) & 3), kg = KG > 1 ? uniform(tid >> 8) : 0;
    // Work-groups are dealt round-robin to the 8 XCDs, each with its own L2: one key/value head per XCD where they divide
    // evenly, so that an L2 fetches the tiles its work-groups walk together once.
    int32_t kvh, item;
    if (xcds_per_kv > 0) {
        const int32_t xcd = blockIdx.x % 8;
        kvh = xcd / xcds_per_kv;
        item = static_cast<int32_t>(blockIdx.x / 8) * xcds_per_kv + xcd % xcds_per_kv;
    } else {
        kvh = blockIdx.x % a.c.n_kv_heads;
        item = blockIdx.x / a.c.n_kv_heads;
    }
    // Query tiles are dealt from the last of a sequence to the first (the later ones see more slots), up to 64 sequences in order of
    // length, so that long work-groups start first.  Where all work-groups are on the chip at once, two to a compute unit, the second half
    // goes from short to long instead: whoever comes second beside the longest is short (2220 rows of three sequences of 1733 to 5000
    // slots: 122 us in the sequences' order).
    const int32_t piece = item % a.n_split;
    int32_t left = item / a.n_split;
    int32_t seq = -1, tile = 0;
    int2 rows = make_int2(0, 0);
    for (int32_t at = 0; at < a.c.n_seq; at += 64) {
        int32_t s = a.c.n_seq - 1 - at - lane;
        int32_t tiles = 0, length = -1;
        int2 r = make_int2(0, 0);
        if (s >= 0) {
            r = rows_of(a, s);
            const int32_t M = r.y > r.x ? (r.y - r.x) * a.group : 0;
            tiles = a.all || M > kFew ? (M + kChunkQ - 1) / kChunkQ : 0;
        }
        if (a.c.n_seq > 1 && a.c.n_seq <= 64) {
            if (tiles > 0) length = limit_of(a, r.y - 1);
            int32_t rank = 0;
            for (int32_t j = 0; j < a.c.n_seq; ++j) {
                const int32_t other = __builtin_amdgcn_readlane(length, j);
                rank += other > length || (other == length && j < lane) ? 1 : 0;
            }
            if (lane >= a.c.n_seq) rank = lane;                // behind all sequences: where it is
            s = __builtin_amdgcn_ds_permute(rank * 4, s);
            tiles = __builtin_amdgcn_ds_permute(rank * 4, tiles);
        }
        int32_t sum = tiles;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int32_t o = __shfl_up(sum, x, 64);
            if (lane >= x) sum += o;
        }
        const int32_t total = __builtin_amdgcn_readlane(sum, 63);
        if (KG == 1 && a.c.n_seq <= 64 && a.n_split == 1 && total <= 2 * kNumCU / a.c.n_kv_heads) {
            const int32_t half = kNumCU / a.c.n_kv_heads;
            if (left >= half && left < total) left = total - 1 - (left - half);
        }
        const uint64_t behind = __ballot(sum > left);
        if (behind != 0) {
            const int who = __builtin_ctzll(behind);
            seq = __builtin_amdgcn_readlane(s, who);
            tile = __builtin_amdgcn_readlane(sum, who) - 1 - left;
            const int from = a.c.n_seq - 1 - at - seq;         // the lane that looked at it
            rows = make_int2(__builtin_amdgcn_readlane(r.x, from), __builtin_amdgcn_readlane(r.y, from));
            break;
        }
        left -= total;
    }
    if (seq < 0) return;
    const int32_t M = (rows.y - rows.x) * a.group;

    // ---- this lane's query: the slots it sees, Q^T fragments; page ids are on their way with them
    const int32_t m = tile * kChunkQ + wave * 32 + l32, mc = m < M ? m : M - 1;
    const int32_t row = rows.x + mc / a.group, head = kvh * a.group + mc % a.group;
    const int32_t limit = limit_of(a, row);
    v8h qf[kD / 16];
    {
        const __half *qp = a.q + row * a.ldq + static_cast<int64_t>(head) * kD + g * 8;
#pragma unroll
        for (int ks = 0; ks < kD / 16; ++ks) qf[ks] = *reinterpret_cast<const v8h *>(qp + ks * 16);
    }
    // Key group kg takes the tiles t0 + kg, t0 + kg + KG, ...: tile i of its own.  The groups do the same number of steps: the last tile
    // of one may lie behind the piece, and nothing of it is visible then.
    const int32_t piece_tiles = a.piece / kChunkK, t0 = piece * piece_tiles;
    auto tile_of = [&](int32_t i) { return t0 + kg + KG * i; };
    // lane l: block l % 4 of tile 16 j + l / 4, for the keys' tile and for the values', and the next 16 tiles on their way
    auto blocks_from = [&](int32_t i) { return block_at(a, seq, kvh, tile_of(i + (lane >> 2)) * 4 + (lane & 3)); };
    uint32_t k_blocks = blocks_from(0), v_blocks = k_blocks, n_blocks = blocks_from(16);

    int32_t top, low = row16_min(limit);
    {
        __shared__ int32_t tops[4];
        int32_t hi = row16_max(limit);
        low = uniform(min(low, __shfl_xor(low, 16, 64)));      // lanes 32.. hold the same queries
        hi = max(hi, __shfl_xor(hi, 16, 64));
        if (kg == 0 && lane == 0) tops[wave] = hi;
        __syncthreads();
        top = uniform(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
    }
    const int32_t t_all = (top + kChunkK) / kChunkK;           // top = -1: none
    if (t0 >= t_all && piece > 0) return;
    const int32_t t_end = piece == a.n_split - 1 || t_all < t0 + piece_tiles ? t_all : t0 + piece_tiles;
    const int32_t steps = t_end > t0 ? (t_end - t0 + KG - 1) / KG : 0;

    // ---- tile copies: block i of 16 slots is 4 KiB of one page; a wave copies four rows of each block.  Key chunk c of row r lies at
    // chunk c ^ (r & 15) (a fragment read takes one chunk of 16 rows), value chunk c at c ^ 4 (r & 3) (a transposing read: 64 bytes of 4 rows).
    const uint32_t lds0 = lds_address(smem) + kg * kChunkLds;
    const int c_row = wave * 4 + (lane >> 4);
    const uint32_t k_off = c_row * 256 + (((lane & 15) ^ (c_row & 15)) << 4);
    const uint32_t v_off = c_row * 256 + (((lane & 15) ^ ((c_row & 3) << 2)) << 4);
    auto dma_k = [&](int32_t i, int b) {
        const int32_t at = i * 4;
        if ((at & 63) == 0 && at > 0) {
            k_blocks = n_blocks;
            n_blocks = blocks_from(i + 16);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            lds_dma16_uniform_base(block_ptr(a.c.k, __builtin_amdgcn_readlane(k_blocks, (at & 63) + u)), k_off,
                                   lds0 + b * kTileBytes + (u * 4 + wave) * 1024);
    };
    auto dma_v = [&](int32_t i, int b) {                       // one tile behind the keys: their blocks are in k_blocks by then
        const int32_t at = i * 4;
        if ((at & 63) == 0) v_blocks = k_blocks;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            lds_dma16_uniform_base(block_ptr(a.c.v, __builtin_amdgcn_readlane(v_blocks, (at & 63) + u)), v_off,
                                   lds0 + (2 + b) * kTileBytes + (u * 4 + wave) * 1024);
    };
    // Value rows behind the last slot become zeros once they have landed (every lane those it copied): they may hold anything,
    // and a zero probability times NaN is NaN.
    auto zero_tail = [&](int32_t i, int b) {
        const int32_t t = tile_of(i);
        if (t * kChunkK + kChunkK - 1 <= top) return;
        uint32_t at = lds0 + (2 + b) * kTileBytes + wave * 1024 + lane * 16;
        int32_t slot = t * kChunkK + c_row;
        asm volatile("" : "+v"(at), "+v"(slot) : : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (slot + 16 * i > top) *(v4u_lds_ptr)(uintptr_t)(at + i * 4096) = v4u{0, 0, 0, 0};
    };

    v16f acc_o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc_o[dt][r] = 0.0f;
    const v16f zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

    // ---- LDS fragments: MFMA i of the score product is (ks, kb) = (i / 2, i % 2), of the P V product (kk, dt) = (i / 4, i % 4).  Operand
    // slot s of lane group g of the P V product is the slot that score register s holds there: 16 kk + 8 (s / 4) + 4 g + s % 4.
    const int tr_row = (lane >> 2) & 3;
    const uint32_t v_lane = g * 1024 + tr_row * 256 + (tr_row << 6) + (((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) * 16 + (lane & 1) * 8;
    uint32_t k_at[8], v_at[4];
    for (int i = 0; i < 8; ++i) {
        k_at[i] = lds0 + l32 * 256 + (((i * 2 + g) ^ (l32 & 15)) << 4);
        asm volatile("" : "+v"(k_at[i]));
    }
    for (int i = 0; i < 4; ++i) {
        v_at[i] = lds0 + (v_lane ^ (i << 6));
        asm volatile("" : "+v"(v_at[i]));
    }
    auto kfrag = [&](uint32_t kb_lds, int i) { return *(v8h_lds_ptr)(uintptr_t)(k_at[i >> 1] + kb_lds + (i & 1) * 8192); };
    auto vfrag = [&](uint32_t vb_lds, int i) {
        const uint32_t f = v_at[i & 3] + vb_lds + (i >> 2) * 4096;
        union {
            tr4 h[2];
            v8h f8;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4f16((tr4_lds_ptr)(uintptr_t)f);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4f16((tr4_lds_ptr)(uintptr_t)(f + 2048));
        return u.f8;
    };
    auto scores = [&](uint32_t kb_lds, v16f (&s)[2]) {
        v8h fr[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fr[i] = kfrag(kb_lds, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr[i % kAhead], qf[i >> 1], i < 2 ? zero16 : s[i & 1], 0, 0, 0);
            if (i + kAhead < 16) fr[i % kAhead] = kfrag(kb_lds, i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    const float scale_log2e = a.scale_log2e, lazy_raw = kLazy / scale_log2e;
    float m_ref = -INFINITY, l_run = 0.0f;

    // One step: softmax and P V of the group's tile i_cur (scores in s_cur, values in V buffer par) while the scores of its next tile (keys in K
    // buffer par ^ 1) go to s_nxt between the exponentials.  On entry a barrier has published those buffers and freed K
    // buffer par and V buffer par ^ 1.  The last tile computes scores of whatever lies in the other K buffer, which nothing reads: a
    // second form of the step without them cost 69 spilled registers.
    auto step = [&](v16f (&s_cur)[2], v16f (&s_nxt)[2], const int32_t i_cur, const int par) {
        if (i_cur + 2 < steps) dma_k(i_cur + 2, par);
        if (i_cur + 1 < steps) dma_v(i_cur + 1, par ^ 1);
        const int32_t t = t0 + kg + KG * i_cur;
        const uint32_t kb_lds = (par ^ 1) * kTileBytes, vb_lds = (2 + par) * kTileBytes;
        if (t * kChunkK + kChunkK - 1 > low || (KG > 1 && t >= t_end)) {       // some query of the wave does not see some slot
            int32_t room = KG > 1 && t >= t_end ? -1 : limit - t * kChunkK - 4 * g;
            asm volatile("" : "+v"(room));
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (kb * 32 + acc_row(r, 0) > room) s_cur[kb][r] = -INFINITY;
        }
        float m_new = m_ref;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) m_new = fmaxf(m_new, s_cur[kb][r]);
        {
            float lo, hi;
            halves_of(m_new, lo, hi);                          // the query's other 32 slots
            m_new = fmaxf(lo, hi);
        }
        if (__any(m_new > m_ref + lazy_raw)) {                 // also the first visible tile (m_ref = -inf)
            const float m_use = m_new == -INFINITY ? 0.0f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m_ref * scale_log2e - m_use * scale_log2e);
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc_o[dt][r] *= alpha;
            m_ref = m_new;
        }
        const float neg = m_ref == -INFINITY ? 0.0f : -m_ref * scale_log2e;
        v8h p[4], fr[kAhead];
        float l_two[2] = {0.0f, 0.0f}, x[2][2], y[2][2];
        auto arg = [&](int e) {
            x[e & 1][0] = __builtin_fmaf(s_cur[e >> 3][(e & 7) * 2], scale_log2e, neg);
            x[e & 1][1] = __builtin_fmaf(s_cur[e >> 3][(e & 7) * 2 + 1], scale_log2e, neg);
        };
        auto ex = [&](int e) {
            y[e & 1][0] = __builtin_amdgcn_exp2f(x[e & 1][0]);
            y[e & 1][1] = __builtin_amdgcn_exp2f(x[e & 1][1]);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fr[i] = kfrag(kb_lds, i);
        __builtin_amdgcn_sched_barrier(0);
        arg(0);
        ex(0);
        arg(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s_nxt[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr[i % kAhead], qf[i >> 1], i < 2 ? zero16 : s_nxt[i & 1], 0, 0, 0);
            if (i + kAhead < 16) fr[i % kAhead] = kfrag(kb_lds, i + kAhead);
            if (i + 1 < 16) ex(i + 1);
            v2h ph;                                            // the denominator sums the probabilities as the product sees them
            ph[0] = static_cast<_Float16>(y[i & 1][0]);
            ph[1] = static_cast<_Float16>(y[i & 1][1]);
            p[(i >> 3) * 2 + ((i & 7) >> 2)][(i & 3) * 2] = ph[0];
            p[(i >> 3) * 2 + ((i & 7) >> 2)][(i & 3) * 2 + 1] = ph[1];
            if (i + 2 < 16) arg(i + 2);
            l_two[i & 1] = __builtin_amdgcn_fdot2(ph, v2h{1, 1}, l_two[i & 1], false);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fr[i] = vfrag(vb_lds, i);
        __builtin_amdgcn_sched_barrier(0);
        {
            float lo, hi;
            halves_of(l_two[0] + l_two[1], lo, hi);
            l_run += lo + hi;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            acc_o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr[i % kAhead], p[i >> 2], acc_o[i & 3], 0, 0, 0);
            if (i + kAhead < 16) fr[i % kAhead] = vfrag(vb_lds, i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
        wait_copies<0>();
        zero_tail(i_cur + 1, par ^ 1);
        __syncthreads();
    };
    // Two steps a turn of the loop, which has one exit: an odd tile goes ahead of it (a way out between the two steps had the
    // compiler move the 64 sums to other registers every turn).
    if (steps > 0) {
        const int par = steps & 1;
        dma_k(0, par);
        dma_v(0, par);
        if (steps > 1) dma_k(1, par ^ 1);
        wait_copies<0>();
        zero_tail(0, par);
        __syncthreads();
        v16f s_a[2], s_b[2];
        int32_t i = 0;
        if (par != 0) {
            scores(kTileBytes, s_b);
            __syncthreads();                                   // the first tile's K buffer is free
            step(s_b, s_a, i++, 1);
        } else {
            scores(0, s_a);
            __syncthreads();
        }
        for (; i < steps; i += 2) {
            step(s_a, s_b, i, 0);
            step(s_b, s_a, i + 1, 1);
        }
    }

    const float ref = m_ref * scale_log2e;

    // ---- lane = query, registers = head channels (4 consecutive per group)
    const bool partial = a.n_split > 1;
    const bool write = m < M && (!partial || limit >= t0 * kChunkK);
    const int64_t at = (static_cast<int64_t>(piece) * a.T + row) * a.n_q + head;
    __half *out = a.o + row * a.ldo + static_cast<int64_t>(head) * kD;
    auto store4 = [&](int dt, int r4, const v4f &f, float inv_l) {
        if (partial) {
            *reinterpret_cast<v4f *>(a.part + at * kD + dt * 32 + r4 * 8 + g * 4) = f;
            return;
        }
        __half h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = __float2half_rn(f[e] * inv_l);
        *reinterpret_cast<uint2 *>(out + dt * 32 + r4 * 8 + g * 4) = *reinterpret_cast<const uint2 *>(h);
    };
    if constexpr (KG == 1) {
        if (!write) return;
        const float inv_l = l_run > 0.0f ? 1.0f / l_run : 0.0f;                 // a row that sees nothing: zeros
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                store4(dt, r4, v4f{acc_o[dt][r4 * 4], acc_o[dt][r4 * 4 + 1], acc_o[dt][r4 * 4 + 2], acc_o[dt][r4 * 4 + 3]}, inv_l);
        if (partial && g == 0) a.part_ml[at] = make_float2(ref, l_run);
    } else {
        // The two key groups of a query exchange halves of the channels: group kg finishes channels 64 kg .. 64 kg + 63.  The last
        // barrier of the loop has freed the tile buffers.
        float *xch = reinterpret_cast<float *>(smem);          // [8 waves][34][64]
        static_assert(8 * 34 * 64 * 4 <= 2 * kChunkLds, "exchange of the key groups");
        float *mine = xch + (kg * 4 + wave) * (34 * 64) + lane;
        const float *theirs = xch + ((kg ^ 1) * 4 + wave) * (34 * 64) + lane;
        auto give = [&](const v16f &x, const v16f &y) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                mine[r * 64] = x[r];
                mine[(16 + r) * 64] = y[r];
            }
        };
        if (kg == 0) give(acc_o[2], acc_o[3]);
        else give(acc_o[0], acc_o[1]);
        mine[32 * 64] = ref;
        mine[33 * 64] = l_run;
        __syncthreads();
        if (!write) return;
        const float m_o = theirs[32 * 64], l_o = theirs[33 * 64], top_m = fmaxf(ref, m_o);
        const float own = ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref - top_m);
        const float other = m_o == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_o - top_m);
        const float l_all = l_run * own + l_o * other, inv_l = l_all > 0.0f ? 1.0f / l_all : 0.0f;
        auto finish = [&](int dt, const v16f &acc, const float *from) {
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                v4f f;
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = acc[r4 * 4 + e] * own + from[(r4 * 4 + e) * 64] * other;
                store4(dt, r4, f, inv_l);
            }
        };
        if (kg == 0) {
            finish(0, acc_o[0], theirs);
            finish(1, acc_o[1], theirs + 16 * 64);
        } else {
            finish(2, acc_o[2], theirs);
            finish(3, acc_o[3], theirs + 16 * 64);
        }
        if (partial && kg == 0 && g == 0) a.part_ml[at] = make_float2(top_m, l_all);
    }
}

// ------------------------------------------------------------------------------------------------ pieces
//
// A wave joins the pieces of one query: o = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p; 16 lanes hold its channels, the quarters of the wave
// take every fourth piece, and 16 pieces are on their way at once, with the running maximum and sum over the sixteens.  Queries whose slots
// were one piece are finished already, those that the other kernel took are its own.  Bound by latency: 3.5 to 5.5 us, of which a launch
// takes 2 and the way row_start, position and partial results, result the rest.
template <bool CHUNK>
__global__ __launch_bounds__(256) void paged_combine_kernel(Step a)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + uniform(threadIdx.x >> 6);
    int32_t row, head;
    int64_t at, stride;                                        // of the partial results: first piece, between pieces
    if constexpr (CHUNK) {
        row = static_cast<int32_t>(item / a.n_q);
        head = static_cast<int32_t>(item % a.n_q);
        if (row >= a.T) return;
        const int32_t seq = sequence_of_row(a.row_start, a.c.n_seq, row);
        if (seq < 0) return;
        const int2 rows = rows_of(a, seq);
        if (!a.all && (rows.y - rows.x) * a.group <= kFew) return;
        at = item;
        stride = static_cast<int64_t>(a.T) * a.n_q;
    } else {
        const int32_t units = a.c.n_seq * a.c.n_kv_heads;
        const int64_t unit = item / a.few_stride;
        const int32_t m = static_cast<int32_t>(item % a.few_stride);
        if (unit >= units) return;
        const int2 rows = rows_of(a, static_cast<int32_t>(unit / a.c.n_kv_heads));
        if (rows.x >= rows.y) return;
        const int32_t M = (rows.y - rows.x) * a.group;
        if (m >= M || (!a.all && M > kFew)) return;
        row = rows.x + m / a.group;
        head = static_cast<int32_t>(unit % a.c.n_kv_heads) * a.group + m % a.group;
        at = item;
        stride = static_cast<int64_t>(units) * a.few_stride;
    }
    const int32_t limit = limit_of(a, row);
    const int ch = (lane & 15) * 8, quarter = lane >> 4;
    float top = -INFINITY, den = 0.0f, f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    constexpr int kAtOnce = 4;
    int32_t n = a.n_split;
    for (int32_t p0 = 0; p0 < n; p0 += 4 * kAtOnce) {
        v4f v[kAtOnce][2];
        float2 ml[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {                    // asked for before the row's limit is there: what lies in pieces behind it is not used
            const int32_t p = p0 + i * 4 + quarter;
            const int64_t from = at + (p < a.n_split ? p : a.n_split - 1) * stride;
            ml[i] = a.part_ml[from];
            v[i][0] = *reinterpret_cast<const v4f *>(a.part + from * kD + ch);
            v[i][1] = *reinterpret_cast<const v4f *>(a.part + from * kD + ch + 4);
        }
        n = pieces_of(a, limit);
        if (!CHUNK && n <= 1) return;
        float top_p = top;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (p0 + i * 4 + quarter >= n) ml[i].x = -INFINITY;
            top_p = fmaxf(top_p, ml[i].x);
        }
        top_p = fmaxf(top_p, __shfl_xor(top_p, 16, 64));
        top_p = fmaxf(top_p, __shfl_xor(top_p, 32, 64));
        const float keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - top_p);
        top = top_p;
        den *= keep;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= keep;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (ml[i].x == -INFINITY) continue;
            const float share = __builtin_amdgcn_exp2f(ml[i].x - top);
            den = __builtin_fmaf(share, ml[i].y, den);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __builtin_fmaf(share, v[i][e >> 2][e & 3], f[e]);
        }
    }
    den += __shfl_xor(den, 16, 64);
    den += __shfl_xor(den, 32, 64);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] += __shfl_xor(f[e], 16, 64);
        f[e] += __shfl_xor(f[e], 32, 64);
    }
    if (quarter != 0) return;
    const float inv = den > 0.0f ? 1.0f / den : 0.0f;
    __half h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = __float2half_rn(f[e] * inv);
    __half *out = a.o + row * a.ldo + static_cast<int64_t>(head) * kD + ch;
    reinterpret_cast<uint2 *>(out)[0] = reinterpret_cast<const uint2 *>(h)[0];
    reinterpret_cast<uint2 *>(out)[1] = reinterpret_cast<const uint2 *>(h)[1];
}

// ------------------------------------------------------------------------------------------------ dispatch

int check_sizes(int32_t T, int32_t n_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_rows, int32_t max_kv)
{
    if (T < 0 || n_seq < 0 || n_q_heads < 1 || n_kv_heads < 1 || max_rows < 0 || max_kv < 0) return MQUANT_ERR_BAD_SHAPE;
    if (head_dim != kD) return MQUANT_ERR_UNSUPPORTED;
    if (n_q_heads % n_kv_heads != 0) return MQUANT_ERR_BAD_SHAPE;
    // kernels step past the last query in 32 bits (2^30 queries would be 256 GiB)
    if (static_cast<int64_t>(T) * n_q_heads > 1 << 30 || static_cast<int64_t>(n_seq) * n_kv_heads > 0x7fffff) return MQUANT_ERR_UNSUPPORTED;
    return MQUANT_OK;
}

// What a call launches.
struct Plan {
    bool few = false, chunk = false;       // the kernels that may be needed; alone, a kernel takes every sequence
    int32_t few_split = 1, few_piece = 1 << 30, few_stride = 0, few_nq = 1;
    bool chunk_two = false;                // two key groups to a work-group
    int32_t chunk_split = 1, chunk_piece = 1 << 30, chunk_tiles = 0;
    int64_t few_part = 0, chunk_part = 0;  // partial results (queries x pieces)
    int64_t bytes() const
    {
        const int64_t n = few_part + chunk_part;
        return n == 0 ? 0 : ceil_div(n * kD * 4, 256) * 256 + ceil_div(n * 8, 256) * 256;
    }
};

Plan make_plan(int32_t T, int32_t n_seq, int32_t n_q, int32_t n_kv, int32_t max_rows, int32_t max_kv)
{
    Plan p;
    if (T == 0 || n_seq == 0) return p;
    const int32_t G = n_q / n_kv;
    const int64_t most = max_rows > 0 && max_rows < T ? max_rows : T;          // rows of a sequence
    const int64_t least = T - (n_seq - 1) * most;                              // where no row is outside the sequences
    p.chunk = most * G > kFew;
    p.few = !p.chunk || least * G <= kFew;
    const int64_t units = static_cast<int64_t>(n_seq) * n_kv, kv = max_kv > 0 ? max_kv : 1;
    if (p.few) {
        const int64_t m = most * G < kFew ? most * G : kFew;
        p.few_nq = static_cast<int32_t>(ceil_div(m, 16));
        p.few_stride = 16 * p.few_nq;
        // Pieces: each costs a work-group's way in and out and a share of the join, and one work-group to a compute unit is enough to
        // keep the memory busy; but host and device know a longest sequence only, and a long one among short ones must not be what
        // the launch waits for.  us by pieces: 64 heads on 8, 7 sequences of 15000 slots 4 79.4, 9 81.0, 18 84.7; 20 of 6000 1 84.3, 3 91.6, 6 95.2, 20
        // of 600 to 6000 1 44.3, 3 42.9, 6 39.7; 32 of 8192 1 182, 2 189, 4 194, 32 of 500 to 16384 1 177, 2 184, 4 125, 8 131; 28 on 4, 8 of 1000 to
        // 16000 8 24.4, 16 26.7, 32 28.5, 64 of 100 to 8000 1 56.9, 2 58.8, 4 47.5, 16 49.3.
        int64_t split = units < kNumCU / 2 ? kNumCU / units : units < kNumCU ? ceil_div(2 * kNumCU, units) : ceil_div(4 * kNumCU, units);
        if (units < kNumCU / 2 && split < ceil_div(kv, 4096)) split = ceil_div(kv, 4096);
        if (split > ceil_div(kv, kFewStep)) split = ceil_div(kv, kFewStep);
        if (split > kMaxThreads / (kFewWaves * 64) / units) split = kMaxThreads / (kFewWaves * 64) / units;
        if (split > 1) {                                       // one piece has no length: rounded up it would not fit 32 bits
            p.few_piece = static_cast<int32_t>(ceil_div(ceil_div(kv, split), kFewStep) * kFewStep);
            p.few_split = static_cast<int32_t>(ceil_div(kv, p.few_piece));
        }
        if (p.few_split > 1) p.few_part = units * p.few_stride * p.few_split;
    }
    if (p.chunk) {
        const int64_t longer = p.few ? (T / (kFew / G + 1) < n_seq ? T / (kFew / G + 1) : n_seq) : n_seq;    // sequences it may take
        p.chunk_tiles = static_cast<int32_t>(static_cast<int64_t>(T) * G / kChunkQ + longer);
        const int64_t groups = p.chunk_tiles * static_cast<int64_t>(n_kv);
        // Pieces: the fewest estimated us.  A step of the walk, which waits for memory where compute units are idle, takes 1.7 with two key
        // groups, 1.0 where two work-groups share a compute unit; the join is a launch, and partial results are written and read.
        // kv is the longest sequence's: a chunk beside longer sequences of single rows is split by their length (512 rows on 512 slots among 31 rows on
        // 4096: 77.7 us, the chunk alone 15.9, the 31 alone 46.3).
        // us by pieces: 28 heads on 4, 64 rows on 2000 slots 1 35.6, 2 26.3, 4 20.4, 8 18.9, 16 21.4; 256 on 1000 1 22.6, 2 24.8, 6 26.4; 256 on
        // 8000 1 118, 4 49.3, 8 46.6; 512 on 512 1 16.0, 2 27.7; 600 on 2000 1 36.8, 3 41.6; 5 on 1, 300 on 9000 1 131, 8 29.5, 16 26.6.
        const int64_t tiles = ceil_div(kv, kChunkK), queries = static_cast<int64_t>(T) * n_q;
        int64_t best = tiles;                                  // tiles of a piece
        double best_us = INFINITY;
        for (int64_t split = 1; split <= (tiles + 1) / 2 && groups * split <= 2 * kNumCU; ++split) {
            const int64_t piece = ceil_div(tiles, split);
            const double walk = groups * split <= kNumCU ? 1.7 * static_cast<double>((piece + 1) / 2) : static_cast<double>(piece);
            const double us = walk + (split > 1 ? 6.0 + 0.25e-3 * static_cast<double>(queries * split) : 0.0);
            if (us >= best_us) continue;
            best_us = us;
            best = piece;
        }
        if (best < tiles) {
            p.chunk_piece = static_cast<int32_t>(best * kChunkK);
            p.chunk_split = static_cast<int32_t>(ceil_div(tiles, best));
        }
        p.chunk_two = groups * p.chunk_split <= kNumCU;
        if (p.chunk_split > 1) p.chunk_part = static_cast<int64_t>(T) * n_q * p.chunk_split;
    }
    return p;
}

}  // namespace

extern "C" int64_t mquant_paged_attention_workspace_bytes(int32_t T, int32_t n_seq, int32_t n_q_heads, int32_t n_kv_heads,
                                                          int32_t head_dim, int32_t max_rows, int32_t max_kv)
{
    if (const int st = check_sizes(T, n_seq, n_q_heads, n_kv_heads, head_dim, max_rows, max_kv); st != MQUANT_OK) return st;
    return make_plan(T, n_seq, n_q_heads, n_kv_heads, max_rows, max_kv).bytes();
}

extern "C" int mquant_paged_attention(const void *q, int64_t ldq, const mquant_paged_cache_t *cache, const int32_t *row_start,
                                      const int32_t *pos, void *o, int64_t ldo, int32_t T, int32_t n_q_heads, int32_t max_rows,
                                      int32_t max_kv, void *workspace, int64_t workspace_bytes, mquant_stream_t stream_)
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
    const int32_t n_kv = cache->n_kv_heads;
    const int32_t slots = cache->table_pages * cache->page_size;
    Plan p = make_plan(T, cache->n_seq, n_q_heads, n_kv, max_rows, max_kv > 0 && max_kv < slots ? max_kv : slots);
    // scratch that was asked for with a bound beyond the table may be another size: then that bound's pieces are taken
    if (max_kv > slots && workspace_bytes < p.bytes()) p = make_plan(T, cache->n_seq, n_q_heads, n_kv, max_rows, max_kv);
    const int64_t need = p.bytes();
    if (need > 0 && (!workspace || workspace_bytes < need)) return MQUANT_ERR_WORKSPACE;
    if (need > 0 && !aligned_to(workspace, 256)) return MQUANT_ERR_ALIGNMENT;
    hipStream_t stream = static_cast<hipStream_t>(stream_);

    Step a = {static_cast<const __half *>(q), ldq, ldo, static_cast<__half *>(o), row_start, pos, T, n_q_heads, n_q_heads / n_kv,
              static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(kD))), cache_args(cache), 1, 1 << 30, p.few_stride, 0,
              static_cast<float *>(workspace),
              reinterpret_cast<float2 *>(static_cast<uint8_t *>(workspace) + ceil_div((p.few_part + p.chunk_part) * kD * 4, 256) * 256)};
    if (p.chunk) {
        a.n_split = p.chunk_split;
        a.piece = p.chunk_piece;
        a.all = !p.few;
        const int32_t xcds_per_kv = 8 % n_kv == 0 ? 8 / n_kv : 0;
        const int64_t items = static_cast<int64_t>(p.chunk_tiles) * p.chunk_split;
        const int64_t groups = xcds_per_kv > 0 ? 8 * ceil_div(items, xcds_per_kv) : items * n_kv;
        const int key_groups = p.chunk_two ? 2 : 1;
        if (groups * key_groups * 256 > kMaxThreads) return MQUANT_ERR_UNSUPPORTED;
        auto kern = p.chunk_two ? paged_chunk_kernel<2> : paged_chunk_kernel<1>;
        static LdsLimit limits[2];
        if (const int st = limits[p.chunk_two].raise(reinterpret_cast<const void *>(kern), key_groups * kChunkLds); st != MQUANT_OK) return st;
        MQ_LAUNCH(kern, dim3(static_cast<unsigned>(groups)), dim3(key_groups * 256), key_groups * kChunkLds, stream, a, xcds_per_kv);
        if (const int st = launch_status(); st != MQUANT_OK) return st;
        if (p.chunk_split > 1) {
            MQ_LAUNCH(paged_combine_kernel<true>, dim3(static_cast<unsigned>(ceil_div(static_cast<int64_t>(T) * n_q_heads, 4))), dim3(256), 0,
                      stream, a);
            if (const int st = launch_status(); st != MQUANT_OK) return st;
        }
    }
    if (p.few) {
        a.n_split = p.few_split;
        a.piece = p.few_piece;
        a.all = !p.chunk;
        a.part += p.chunk_part * kD;
        a.part_ml += p.chunk_part;
        const int64_t units = static_cast<int64_t>(cache->n_seq) * n_kv, groups = units * p.few_split;
        auto kern = p.few_nq == 1 ? paged_few_kernel<1> : p.few_nq == 2 ? paged_few_kernel<2> : paged_few_kernel<3>;
        static LdsLimit limits[3];
        if (const int st = limits[p.few_nq - 1].raise(reinterpret_cast<const void *>(kern), kFewLds); st != MQUANT_OK) return st;
        MQ_LAUNCH(kern, dim3(static_cast<unsigned>(groups)), dim3(kFewWaves * 64), kFewLds, stream, a);
        if (const int st = launch_status(); st != MQUANT_OK) return st;
        if (p.few_split > 1) {
            MQ_LAUNCH(paged_combine_kernel<false>, dim3(static_cast<unsigned>(ceil_div(units * p.few_stride, 4))), dim3(256), 0, stream, a);
            return launch_status();
        }
    }
    return MQUANT_OK;
}
