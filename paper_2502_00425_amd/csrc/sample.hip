// The next token of every row of logits by temperature, top-k, top-p and min-p from a given random number, for gfx950.
//
// Token i has the weight w = 2^-x, x = (m - l) log2(e) / t >= 0; ranked by logit, the kept tokens are a front of the ranking, and
// which token is drawn is a question of sums of weights.  Weights are formed in double (off by 2^-44 of themselves) and summed as whole
// multiples of 2^-43: such sums do not depend on their order, so that atomics in LDS and any split of the work give the same
// token.  2^20 tokens of weight 1 are 2^63.
//
// Nothing is sorted but a short list.  tile_kernel, a work-group to 16 KiB of a row, takes from every piece of 64 blocks of 16 bytes its
// largest logit and, as the row's settings ask, the weight of every piece or the tokens and weights of the tile by bins of the logit.
// pick_kernel, a work-group to a row, puts them together:
//   rows without filters: the piece in which the sum passes u S, and the token in it;
//   what top-k, top-p and min-p can keep is a short list, by the bins: it is gathered from the pieces whose largest logit can be in it, and
//   everything is decided among its tokens;
//   many tokens are kept: the tokens of the bin in which the ranking is cut are gathered (narrowed by finer bins, then digit by digit of their
//   rank, where they are more than the list holds); with the rank of the last kept token the tiles' bins give the tile in which the
//   sum passes u S, which is looked at token by token;
//   the rest (+inf among the logits, long lists by top-k or min-p alone): bins of the whole row and a walk over it by the one work-group.
#include <cfloat>
#include <cmath>

#include <hip/hip_fp16.h>

#include "mquant_internal.h"

using namespace mquant;

namespace {

typedef unsigned long long u64;
typedef unsigned __int128 u128;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxTokens = 1 << 20;
constexpr int kBins = 1024;                // of walk_row
constexpr int kCoarse = 256;               // bins of a tile: 1/4 of x wide, the last one has all that is left
constexpr int kTileThreads = 256, kTileBlocks = 4, kTilePieces = kTileThreads / 64 * kTileBlocks;
constexpr int kMaxPieces = ((kMaxTokens + 6) / 4 + kTileThreads * kTileBlocks - 1) / (kTileThreads * kTileBlocks) * kTilePieces;    // fp32, tiles filled up
constexpr int kShort = 256;                // tokens of a list up to which each is compared with all others
constexpr int kList = 2048;                // tokens that are sorted at a time, two to a thread
constexpr int kBits = 43;                  // a weight of 1 is 2^43
constexpr u64 kNone = ~0ull;
constexpr int kIndexBits = 24;             // of a rank: logit, then number of the token

struct Args {
    const void *logits;
    int64_t ld;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p, *u;
    int32_t *token;
    float *logprob;
    int32_t V;
    // of every row: pieces and tiles as the workspace has room for (at least as many as the row has)
    int32_t pieces, tiles;
    u64 *piece_sum;                        // [rows, pieces] weight of a piece against its own largest logit
    float *piece_max;                      // [rows, pieces]; NaN where no token can be chosen
    u64 *tile_mass;                        // [rows, tiles, kCoarse] against the tile's largest logit
    uint32_t *tile_count;                  // [rows, tiles, kCoarse]
    float *tile_max;                       // [rows, tiles]; NaN as above
};

// What the tiles of a row are asked for.
enum class Ask { kNothing, kSums, kCount, kMass, kBoth };

struct Settings {
    float t, p, min_p, u;
    int32_t k;
    __device__ Settings(const Args &a, int64_t r)
        : t(a.temperature ? a.temperature[r] : 1.0f), p(a.top_p ? a.top_p[r] : 1.0f), min_p(a.min_p ? a.min_p[r] : 0.0f), u(a.u[r]),
          k(a.top_k ? a.top_k[r] : 0)
    {
        if (k < 0 || k >= a.V) k = 0;
    }
    // Whether the first token of the ranking is all that is kept, which has weight 1.
    __device__ bool first() const { return !(t > 0.0f) || k == 1 || p <= 0.0f || min_p > 1.0f; }
    // Of the first few tokens their number is enough: the weights are worked out in the list.  Min-p alone says itself which tokens are kept.
    __device__ Ask ask() const
    {
        if (first()) return Ask::kNothing;
        if (k > 0) return k <= kList ? Ask::kCount : Ask::kBoth;
        return p < 1.0f ? Ask::kMass : min_p > 0.0f ? Ask::kNothing : Ask::kSums;
    }
};

// 2^(43 - j / 64)
__device__ const double kPower[64] = {
    0x1.0000000000000p+43, 0x1.fa7c1819e90d8p+42, 0x1.f50765b6e4540p+42, 0x1.efa1bee615a27p+42,
    0x1.ea4afa2a490dap+42, 0x1.e502ee78b3ff6p+42, 0x1.dfc97337b9b5fp+42, 0x1.da9e603db3285p+42,
    0x1.d5818dcfba487p+42, 0x1.d072d4a07897cp+42, 0x1.cb720dcef9069p+42, 0x1.c67f12e57d14bp+42,
    0x1.c199bdd85529cp+42, 0x1.bcc1e904bc1d2p+42, 0x1.b7f76f2fb5e47p+42, 0x1.b33a2b84f15fbp+42,
    0x1.ae89f995ad3adp+42, 0x1.a9e6b5579fdbfp+42, 0x1.a5503b23e255dp+42, 0x1.a0c667b5de565p+42,
    0x1.9c49182a3f090p+42, 0x1.97d829fde4e50p+42, 0x1.93737b0cdc5e5p+42, 0x1.8f1ae99157736p+42,
    0x1.8ace5422aa0dbp+42, 0x1.868d99b4492edp+42, 0x1.82589994cce13p+42, 0x1.7e2f336cf4e62p+42,
    0x1.7a11473eb0187p+42, 0x1.75feb564267c9p+42, 0x1.71f75e8ec5f74p+42, 0x1.6dfb23c651a2fp+42,
    0x1.6a09e667f3bcdp+42, 0x1.6623882552225p+42, 0x1.6247eb03a5585p+42, 0x1.5e76f15ad2148p+42,
    0x1.5ab07dd485429p+42, 0x1.56f4736b527dap+42, 0x1.5342b569d4f82p+42, 0x1.4f9b2769d2ca7p+42,
    0x1.4bfdad5362a27p+42, 0x1.486a2b5c13cd0p+42, 0x1.44e086061892dp+42, 0x1.4160a21f72e2ap+42,
    0x1.3dea64c123422p+42, 0x1.3a7db34e59ff7p+42, 0x1.371a7373aa9cbp+42, 0x1.33c08b26416ffp+42,
    0x1.306fe0a31b715p+42, 0x1.2d285a6e4030bp+42, 0x1.29e9df51fdee1p+42, 0x1.26b4565e27cddp+42,
    0x1.2387a6e756238p+42, 0x1.2063b88628cd6p+42, 0x1.1d4873168b9aap+42, 0x1.1a35beb6fcb75p+42,
    0x1.172b83c7d517bp+42, 0x1.1429aaea92de0p+42, 0x1.11301d0125b51p+42, 0x1.0e3ec32d3d1a2p+42,
    0x1.0b5586cf9890fp+42, 0x1.0874518759bc8p+42, 0x1.059b0d3158574p+42, 0x1.02c9a3e778061p+42,
};

// What a row's threads share.
struct Shared {
    u64 mass[kBins];                       // up to and with a bin
    uint32_t count[kBins];
    u64 coarse_mass[kCoarse];
    uint32_t coarse_count[kCoarse];
    union {
        struct {
            u64 rank[kList], sum[kList];
        } list;
        u64 piece[kMaxPieces];             // weight of 64 blocks of 16 bytes
        struct {
            u64 mass[256];
            uint32_t count[256];
        } digit;
    };
    double power[64];                      // kPower
    u64 room[kWaves];
    u64 found[2];
    uint32_t found32[2];
    uint32_t n, n_pieces;
    int32_t todo[kMaxPieces];              // pieces to gather from
};

// ---- a row's logits: the 16-byte blocks that hold it, from the aligned one in which it begins
template <typename E>
struct Row {
    static constexpr int kPer = 16 / sizeof(E);
    const uint4 *block;
    int32_t skip, n_blocks, V;             // elements of the first block ahead of the row
    bool only_inf;                         // where +inf occurs, it counts as 0 and everything else as nothing

    __device__ Row(const Args &a, int64_t row) : V(a.V)
    {
        const uintptr_t p = reinterpret_cast<uintptr_t>(static_cast<const E *>(a.logits) + row * a.ld);
        skip = static_cast<int32_t>((p & 15) / sizeof(E));
        block = reinterpret_cast<const uint4 *>(p & ~static_cast<uintptr_t>(15));
        n_blocks = (skip + V + kPer - 1) / kPer;
        only_inf = false;
    }

    // Token number of element e of block b; outside [0, V): not of the row.
    __device__ int32_t token(int32_t b, int e) const { return b * kPer + e - skip; }

    // The logits of block b, NaN for what is not of the row.
    __device__ void read(const uint4 &raw, int32_t b, float (&l)[kPer]) const
    {
        union {
            uint4 u;
            E e[kPer];
        } x;
        x.u = raw;
#pragma unroll
        for (int e = 0; e < kPer; ++e) l[e] = static_cast<float>(x.e[e]);
        if (b == 0 || b >= n_blocks - 1) {
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (static_cast<uint32_t>(token(b, e)) >= static_cast<uint32_t>(V)) l[e] = NAN;
        }
        if (only_inf) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) l[e] = l[e] == INFINITY ? 0.0f : NAN;
        }
    }
};

// Whether a token with this logit can be chosen: neither -inf nor NaN.
__device__ __forceinline__ bool there(float l) { return l > -INFINITY; }

// ---- sums over the work-group
__device__ __forceinline__ u64 shfl_up64(u64 x, int by)
{
    const uint32_t lo = __shfl_up(static_cast<uint32_t>(x), by, 64), hi = __shfl_up(static_cast<uint32_t>(x >> 32), by, 64);
    return static_cast<u64>(hi) << 32 | lo;
}

__device__ __forceinline__ u64 wave_scan(u64 x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 y = shfl_up64(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// Up to and with this thread; `all`: over all threads.  Ends behind a barrier that frees nothing: a barrier has to come before the next use.
__device__ __forceinline__ u64 scan(u64 x, u64 *room, u64 &all)
{
    const int wave = threadIdx.x >> 6;
    x = wave_scan(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) room[wave] = x;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) x += all;
        all += room[w];
    }
    return x;
}

// ---- ranks: the larger the logit and the lower the token's number, the smaller
__device__ __forceinline__ uint32_t order_of(float l)          // rises with l
{
    const uint32_t b = __float_as_uint(l + 0.0f);              // -0 ranks with 0
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ float float_of(uint32_t order) { return __uint_as_float(order ^ (order >> 31 ? 0x80000000u : 0xffffffffu)); }

__device__ __forceinline__ u64 rank_of(float l, int32_t token)
{
    return static_cast<u64>(~order_of(l)) << kIndexBits | static_cast<uint32_t>(token);
}

__device__ __forceinline__ float logit_of(u64 rank) { return float_of(~static_cast<uint32_t>(rank >> kIndexBits)); }

// ---- weights
struct Scale {
    double x_of;                           // log2(e) / t; not 0, so that x_end is a number
    double x_end;                          // m - l from which weights count as nothing
    float bin_of;                          // 16 x_of, for the bins
    float m;                               // the largest logit

    __device__ Scale(float t, float top) : x_of(fmax(1.4426950408889634074 / static_cast<double>(t), 1e-60)), m(top)
    {
        x_end = (kBits + 1.75) / x_of;
        bin_of = fminf(static_cast<float>(x_of * 16.0), 1e30f);
    }

    // A tile's bins are of the logit itself, 1/4 of x wide, so that those of all tiles fit together.  Falls with l, whatever is rounded.
    __device__ float quarters(float l) const { return l * (-0.25f * bin_of); }
    __device__ int coarse(float l) const { return static_cast<int>(fminf(fmaxf(floorf(quarters(l)), -0x1p29f), 0x1p29f)); }
    // Within such a bin, 1024 of them.
    __device__ int fine(float l, int bin) const
    {
        return static_cast<int>(fminf(fmaxf((quarters(l) - static_cast<float>(bin)) * static_cast<float>(kBins), 0.0f), kBins - 1.0f));
    }

    // The smallest logit in a coarse bin up to `bin`, by bisection of the floats in their order.
    __device__ float least(int bin) const
    {
        uint32_t lo = 0x00800000u, hi = 0xff7fffffu;           // -FLT_MAX and FLT_MAX, of which the largest logit is one at most
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (coarse(float_of(mid)) <= bin) hi = mid;
            else lo = mid + 1;
        }
        return float_of(lo);
    }

    __device__ double x(float l) const { return (static_cast<double>(m) - static_cast<double>(l)) * x_of; }
    // Falls with l, like the rank, whatever is rounded; the last bin has all that is left.
    __device__ int bin(float l) const { return static_cast<int>(fminf((m - l) * bin_of, static_cast<float>(kBins - 1))); }

    // 2^(43 - x), nothing (2^-1.75) for what is no logit: x in steps of 1/64 by the table, the rest by e^-z, |z| <= ln 2 / 128, to z^4
    // (z^5 / 120 is 2^-44.5).  The steps are found by adding 1.5 2^52; their number is in the low bits then.
    __device__ double weight(float l, const double *power) const
    {
        constexpr double kStep = 0.69314718055994530942 / 64.0, kRound = 0x1.8p52;
        const double d = __builtin_fmin(static_cast<double>(m) - static_cast<double>(l), x_end), y_of = x_of * 64.0;
        const double t = __builtin_fma(d, y_of, kRound), n = t - kRound, y = __builtin_fma(d, y_of, -n);
        const int i = static_cast<int>(__double_as_longlong(t));
        double p = __builtin_fma(y, kStep * kStep * kStep * kStep / 24.0, -(kStep * kStep * kStep / 6.0));
        p = __builtin_fma(p, y, kStep * kStep / 2.0);
        p = __builtin_fma(p, y, -kStep);
        p = __builtin_fma(p, y, 1.0);
        return __longlong_as_double(__double_as_longlong(power[i & 63] * p) - (static_cast<long long>(i >> 6) << 52));
    }
    __device__ u64 weigh(float l, const double *power) const;
};

// To the nearest whole number below 2^52.
__device__ __forceinline__ u64 whole(double w) { return static_cast<u64>(__double_as_longlong(w + 0x1p52)) & ((1ull << 52) - 1); }

__device__ __forceinline__ u64 Scale::weigh(float l, const double *power) const { return whole(weight(l, power)); }

// floor(f * n) for f in [0, 1], and its remainder's truth value.
__device__ __forceinline__ u64 share_of(float f, u64 n, bool &rest)
{
    rest = false;
    if (!(f > 0.0f)) return 0;
    if (f >= 1.0f) return n;
    int e;
    const u64 mantissa = static_cast<u64>(ldexpf(frexpf(f, &e), 24));          // f = mantissa 2^(e - 24), e <= 0
    const int down = 24 - e;
    const u128 product = static_cast<u128>(mantissa) * n;                       // below 2^88
    if (down > 120) {
        rest = product != 0;
        return 0;
    }
    rest = (product & ((static_cast<u128>(1) << down) - 1)) != 0;
    return static_cast<u64>(product >> down);
}

// Every block of the row once: f(block number, logits).  Four of a thread's blocks are on their way at a time.
template <typename E, typename F>
__device__ __forceinline__ void walk(const Row<E> &row, F f)
{
    constexpr int kAtOnce = 4;
    for (int32_t b0 = threadIdx.x; b0 < row.n_blocks; b0 += kThreads * kAtOnce) {
        uint4 raw[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int32_t b = b0 + u * kThreads;
            raw[u] = row.block[b < row.n_blocks ? b : row.n_blocks - 1];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int32_t b = b0 + u * kThreads;
            if (b >= row.n_blocks) break;
            float l[Row<E>::kPer];
            row.read(raw[u], b, l);
            f(b, l);
        }
    }
}

// Sorts the n <= kList numbers of v, rising; all threads.
__device__ void sort_list(u64 *v, int n)
{
    int size = 2;
    while (size < n) size <<= 1;
    for (int i = threadIdx.x; i < size; i += kThreads)
        if (i >= n) v[i] = kNone;
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int t = threadIdx.x; t < size >> 1; t += kThreads) {
                const int i = ((t & ~(j - 1)) << 1) | (t & (j - 1));
                const u64 x = v[i], y = v[i + j];
                if ((x > y) == ((i & k) == 0)) {
                    v[i] = y;
                    v[i + j] = x;
                }
            }
        }
    __syncthreads();
}

// Sums of the weights of the list's n tokens, up to and with each; all threads.
__device__ void sum_list(Shared &s, int n, const Scale &sc)
{
    const int i = threadIdx.x * 2;
    const u64 x = i < n ? sc.weigh(logit_of(s.list.rank[i]), s.power) : 0;
    const u64 y = i + 1 < n ? sc.weigh(logit_of(s.list.rank[i + 1]), s.power) : 0;
    u64 all;
    const u64 up = scan(x + y, s.room, all);
    s.list.sum[i] = up - y;
    s.list.sum[i + 1] = up;
    __syncthreads();
}

// The tokens that `take` names are put into the list as far as it has room; returns how many there are.
template <typename E, typename F>
__device__ int gather(Shared &s, const Row<E> &row, F take)
{
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    walk(row, [&](int32_t b, const float (&l)[Row<E>::kPer]) {
#pragma unroll
        for (int e = 0; e < Row<E>::kPer; ++e)
            if (there(l[e]) && take(l[e], row.token(b, e))) {
                const uint32_t at = atomicAdd(&s.n, 1u);
                if (at < kList) s.list.rank[at] = rank_of(l[e], row.token(b, e));
            }
    });
    __syncthreads();
    const int n = s.n;
    __syncthreads();
    return n;
}

// How many of the list's n sorted tokens, with sums of weights up to and with each, come ahead of a cut: the first `count` of them at most,
// and only those with less than `mass` before them.
__device__ int cut_list(Shared &s, int n, u64 count, u64 mass)
{
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    uint32_t mine = 0;
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (static_cast<u64>(i) < count && (i == 0 ? 0 : s.list.sum[i - 1]) < mass) ++mine;
    if (mine > 0) atomicAdd(&s.n, mine);
    __syncthreads();
    const int k = s.n;
    __syncthreads();
    return k;
}

// The rank of the last token that a cut keeps of the n tokens that `of` names, a run of the ranking: by rank the first `count` of them (at
// least 1, at most all), and only those with less than `mass` of their weight before them (the first one has).  kept_mass: the weight of
// those kept.
template <typename E, typename F>
__device__ u64 cut_run(Shared &s, const Row<E> &row, const Scale &sc, F of, u64 n, u64 count, u64 mass, u64 &kept_mass)
{
    u64 prefix = 0, passed = 0;            // digits of the rank that are known, weight of the tokens ahead of them
    int low = 32 + kIndexBits;             // bits that are not
    while (n > kList) {
        low -= 8;
        __syncthreads();
        if (threadIdx.x < 256) {
            s.digit.mass[threadIdx.x] = 0;
            s.digit.count[threadIdx.x] = 0;
        }
        __syncthreads();
        walk(row, [&](int32_t at, const float (&l)[Row<E>::kPer]) {
#pragma unroll
            for (int e = 0; e < Row<E>::kPer; ++e) {
                if (!there(l[e]) || !of(l[e])) continue;
                const u64 r = rank_of(l[e], row.token(at, e));
                if (r >> low >> 8 != prefix) continue;
                atomicAdd(&s.digit.mass[r >> low & 255], sc.weigh(l[e], s.power));
                atomicAdd(&s.digit.count[r >> low & 255], 1u);
            }
        });
        __syncthreads();
        if (threadIdx.x == 0) {            // the digit of the last token that the cut keeps
            u64 c = 0, w = 0;
            int d = -1;
            u64 c_at = 0, w_at = 0;
            for (int i = 0; i < 256; ++i) {
                if (s.digit.count[i] == 0) continue;
                if (d >= 0 && (c >= count || w >= mass)) break;
                d = i;
                c_at = c;
                w_at = w;
                c += s.digit.count[i];
                w += s.digit.mass[i];
            }
            s.found[0] = c_at;
            s.found[1] = w_at;
            s.found32[0] = d;
            s.found32[1] = s.digit.count[d];
        }
        __syncthreads();
        prefix = prefix << 8 | s.found32[0];
        n = s.found32[1];
        count -= s.found[0];
        mass = mass > s.found[1] ? mass - s.found[1] : 0;
        passed += s.found[1];
        __syncthreads();
    }
    const int m = gather(s, row, [&](float l, int32_t token) { return of(l) && rank_of(l, token) >> low == prefix; });
    sort_list(s.list.rank, m);
    sum_list(s, m, sc);
    int k = cut_list(s, m, count, mass);
    if (k < 1) k = 1;
    kept_mass = passed + s.list.sum[k - 1];
    const u64 last = s.list.rank[k - 1];
    __syncthreads();
    return last;
}

// ---- what the tiles of a row find out
__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}

__device__ __forceinline__ u64 wave_sum(u64 x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t lo = __shfl_xor(static_cast<uint32_t>(x), d, 64), hi = __shfl_xor(static_cast<uint32_t>(x >> 32), d, 64);
        x += static_cast<u64>(hi) << 32 | lo;
    }
    return x;
}

__device__ __forceinline__ void set_power(double *power)
{
    if (threadIdx.x < 64) power[threadIdx.x] = kPower[threadIdx.x];
}

template <typename E>
__global__ __launch_bounds__(kTileThreads) void tile_kernel(Args a)
{
    __shared__ u64 mass[kCoarse];
    __shared__ uint32_t count[kCoarse];
    __shared__ double power[64];
    __shared__ float tops[kTileThreads / 64];
    constexpr int kPer = Row<E>::kPer;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r = blockIdx.x / a.tiles;
    const int32_t tile = blockIdx.x % a.tiles;
    const Row<E> row(a, r);
    const int32_t piece0 = tile * kTilePieces + wave * kTileBlocks;
    uint4 raw[kTileBlocks];
#pragma unroll
    for (int j = 0; j < kTileBlocks; ++j) {
        const int32_t b = (piece0 + j) * 64 + lane;
        raw[j] = row.block[b < row.n_blocks ? b : row.n_blocks - 1];
    }
    const Settings set(a, r);
    const Ask ask = set.ask();
    set_power(power);
    mass[tid] = 0;
    count[tid] = 0;
    float l[kTileBlocks][kPer], top[kTileBlocks], wave_top = -INFINITY;
#pragma unroll
    for (int j = 0; j < kTileBlocks; ++j) {
        row.read(raw[j], (piece0 + j) * 64 + lane, l[j]);
        top[j] = -INFINITY;
#pragma unroll
        for (int e = 0; e < kPer; ++e) top[j] = fmaxf(top[j], l[j][e]);
        top[j] = wave_max(top[j]);
        wave_top = fmaxf(wave_top, top[j]);
        if (lane == 0) a.piece_max[r * a.pieces + piece0 + j] = top[j];
    }
    if (ask == Ask::kNothing) return;
    if (ask != Ask::kSums && lane == 0) tops[wave] = wave_top;
    __syncthreads();
    if (ask == Ask::kSums) {
#pragma unroll
        for (int j = 0; j < kTileBlocks; ++j) {
            const Scale sc(set.t, top[j]);
            u64 w = 0;
#pragma unroll
            for (int e = 0; e < kPer; ++e) w += sc.weigh(l[j][e], power);
            w = wave_sum(w);
            if (lane == 0) a.piece_sum[r * a.pieces + piece0 + j] = w;
        }
        return;
    }
    float tile_top = tops[0];
#pragma unroll
    for (int w = 1; w < kTileThreads / 64; ++w) tile_top = fmaxf(tile_top, tops[w]);
    const Scale sc(set.t, tile_top);
    const int base = sc.coarse(tile_top);
#pragma unroll
    for (int j = 0; j < kTileBlocks; ++j)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (!there(l[j][e])) continue;
            const int at = sc.coarse(l[j][e]) - base, bin = at < kCoarse ? at : kCoarse - 1;
            if (ask != Ask::kMass) atomicAdd(&count[bin], 1u);
            if (ask != Ask::kCount) atomicAdd(&mass[bin], sc.weigh(l[j][e], power));
        }
    __syncthreads();
    const int64_t at = (r * a.tiles + tile) * kCoarse + tid;
    if (ask != Ask::kMass) a.tile_count[at] = count[tid];
    if (ask != Ask::kCount) a.tile_mass[at] = mass[tid];
    if (tid == 0) a.tile_max[r * a.tiles + tile] = tile_top;
}

// Weight against the row's largest logit of what weighs `sum` against the logit l.
__device__ __forceinline__ u64 rescaled(u64 sum, float l, const Scale &sc, const double *power)
{
    return static_cast<u64>(rint(static_cast<double>(sum) * (sc.weight(l, power) * 0x1p-43)));
}

// Sum over the 2^log lanes next to each other.
__device__ __forceinline__ u64 lanes_sum(u64 x, int log)
{
    for (int d = 1; d < 1 << log; d <<= 1) {
        const uint32_t lo = __shfl_xor(static_cast<uint32_t>(x), d, 64), hi = __shfl_xor(static_cast<uint32_t>(x >> 32), d, 64);
        x += static_cast<u64>(hi) << 32 | lo;
    }
    return x;
}

// Which of the list's n <= kShort tokens is drawn: each is compared with all, by 4 lanes next to each other, 16 where they are few.
template <typename F>
__device__ void draw_short(Shared &s, int n, int32_t k, float p, double min_w, float u, u64 all_mass, bool all_known, const Scale &sc, F chosen)
{
    static_assert(kShort * 4 == kThreads, "lanes of a token");
    constexpr u64 kTokenMask = (1u << kIndexBits) - 1;
    const int log = n <= kThreads / 16 ? 4 : 2, lanes = 1 << log;
    const int tid = threadIdx.x, me = tid >> log, part = tid & (lanes - 1);
    const bool mine = me < n;
    const u64 rank = mine ? s.list.rank[me] : kNone;
    const double w = mine ? sc.weight(logit_of(rank), s.power) : 0.0;
    const u64 weight = whole(w);
    if (mine && part == 0) s.list.sum[me] = weight;
    if (tid < 2) s.found[tid] = 0;
    __syncthreads();
    u64 before = 0, ahead = 0;             // weight and number of the tokens ahead of mine
    if (mine) {
#pragma unroll 4
        for (int j = part; j < n; j += lanes) {
            const u64 other = s.list.rank[j], sum = s.list.sum[j];
            if (other < rank) {
                ++ahead;
                before += sum;
            }
        }
    }
    ahead = lanes_sum(ahead, log);
    if (p < 1.0f) before = lanes_sum(before, log);
    bool kept = mine && (k <= 0 || ahead < static_cast<u64>(k)), rest;
    if (p < 1.0f) {
        if (!all_known) {
            if (kept && part == 0) atomicAdd(&s.found[0], weight);
            __syncthreads();
            all_mass = s.found[0];
        }
        u64 target = share_of(p, all_mass, rest);
        target += rest ? 1 : 0;
        kept = kept && (before < target || ahead == 0);
    }
    kept = kept && (w >= min_w || ahead == 0);
    __syncthreads();
    if (mine && part == 0) {
        s.list.sum[me] = kept ? weight : 0;
        if (kept) atomicAdd(&s.found[1], weight);
    }
    __syncthreads();
    const u64 sum = s.found[1];
    u64 pass = share_of(u, sum, rest);
    if (pass >= sum) pass = sum - 1;
    u64 at = 0;
    if (kept) {
#pragma unroll 4
        for (int j = part; j < n; j += lanes) {
            const u64 other = s.list.rank[j], w_j = s.list.sum[j];
            if ((other & kTokenMask) < (rank & kTokenMask)) at += w_j;
        }
    }
    at = lanes_sum(at, log);
    if (kept && part == 0 && at <= pass && at + weight > pass) chosen(rank, sum);
}

// The same for more tokens: sorted by rank, then the kept ones by their number.
template <typename F>
__device__ void draw_sorted(Shared &s, int n, int32_t k, float p, double min_w, float u, u64 all_mass, bool all_known, const Scale &sc, F chosen)
{
    const int tid = threadIdx.x;
    constexpr u64 kTokenMask = (1u << kIndexBits) - 1;
    sort_list(s.list.rank, n);
    sum_list(s, n, sc);
    bool rest;
    if (k <= 0 || k > n) k = n;
    u64 target = kNone;
    if (p < 1.0f) {
        target = share_of(p, all_known ? all_mass : s.list.sum[k - 1], rest);
        target += rest ? 1 : 0;
    }
    int kept = cut_list(s, n, k, target);
    if (kept < 1) kept = 1;
    if (min_w > 0.0) {
        if (tid == 0) s.n = 0;
        __syncthreads();
        uint32_t mine = 0;
        for (int i = tid; i < kept; i += kThreads)
            if (sc.weight(logit_of(s.list.rank[i]), s.power) >= min_w) ++mine;
        if (mine > 0) atomicAdd(&s.n, mine);
        __syncthreads();
        kept = s.n > 1 ? s.n : 1;
        __syncthreads();
    }
    const u64 sum = s.list.sum[kept - 1];
    u64 pass = share_of(u, sum, rest);
    if (pass >= sum) pass = sum - 1;
    const int i = tid * 2;
    const u64 r0 = i < kept ? s.list.rank[i] : kNone, r1 = i + 1 < kept ? s.list.rank[i + 1] : kNone;
    __syncthreads();
    // sorted by the token's number, with the place in the ranking behind it
    if (i < kept) s.list.rank[i] = (r0 & kTokenMask) << 12 | static_cast<u64>(i);
    if (i + 1 < kept) s.list.rank[i + 1] = (r1 & kTokenMask) << 12 | static_cast<u64>(i + 1);
    __syncthreads();
    sort_list(s.list.rank, kept);
    auto weight_at = [&](int at) {
        const int place = static_cast<int>(s.list.rank[at] & 0xfff);
        return s.list.sum[place] - (place > 0 ? s.list.sum[place - 1] : 0);
    };
    const u64 x = i < kept ? weight_at(i) : 0, y = i + 1 < kept ? weight_at(i + 1) : 0;
    u64 total;
    const u64 up = scan(x + y, s.room, total);
    if (up - x - y <= pass && up - y > pass) s.found32[0] = static_cast<uint32_t>(s.list.rank[i] & 0xfff);
    if (up - y <= pass && up > pass) s.found32[0] = static_cast<uint32_t>(s.list.rank[i + 1] & 0xfff);
    __syncthreads();
    const int place = s.found32[0];                            // a place has its logit in the thread that held it
    if (place == i) chosen(r0, sum);
    if (place == i + 1) chosen(r1, sum);
}

// The piece in which the sum passes `pass`, of `pieces` sums in s.piece, and the sum ahead of it, for all threads: s.found32[0], s.found[0].
// Returns the whole sum; `pass` is u's share of it.
__device__ u64 find_piece(Shared &s, int32_t pieces, float u, u64 &pass)
{
    // every thread takes the pieces from..to, next to each other
    const int32_t per = (pieces + kThreads - 1) / kThreads, from = threadIdx.x * per, to = from + per < pieces ? from + per : pieces;
    u64 mine = 0, sum;
    for (int32_t i = from; i < to; ++i) mine += s.piece[i];
    const u64 up = scan(mine, s.room, sum);
    bool rest;
    pass = share_of(u, sum, rest);
    if (pass >= sum) pass = sum - 1;
    if (up > pass && up - mine <= pass) {
        u64 at = up - mine;
        int32_t i = from;
        while (at + s.piece[i] <= pass) at += s.piece[i++];
        s.found32[0] = i;
        s.found[0] = at;
    }
    __syncthreads();
    return sum;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void pick_kernel(Args a)
{
    __shared__ Shared s;
    constexpr int kPer = Row<E>::kPer;
    constexpr int32_t kTokenMask = (1 << kIndexBits) - 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r = blockIdx.x;
    Row<E> row(a, r);
    const Settings set(a, r);
    const float *piece_max = a.piece_max + r * a.pieces;
    auto result = [&](int32_t token, double logprob) {
        a.token[r] = token;
        if (a.logprob) a.logprob[r] = static_cast<float>(logprob);
    };

    // ---- the largest logit
    set_power(s.power);
    float top = -INFINITY;
    for (int32_t i = tid; i < a.pieces; i += kThreads) top = fmaxf(top, piece_max[i]);
    top = wave_max(top);
    float *tops = reinterpret_cast<float *>(s.room);
    if (lane == 0) tops[wave] = top;
    if (tid < 2) s.found32[tid] = ~0u;
    if (tid == 0) s.n = s.n_pieces = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w]);
    __syncthreads();
    if (top == -INFINITY) {
        if (tid == 0) result(-1, -INFINITY);
        return;
    }
    auto first_piece = [&] {               // the first one with the largest logit
        for (int32_t i = tid; i < a.pieces; i += kThreads)
            if (piece_max[i] == top) {
                atomicMin(&s.found32[0], static_cast<uint32_t>(i));
                break;
            }
        __syncthreads();
        return static_cast<int32_t>(s.found32[0]);
    };
    if (set.first()) {
        const int32_t b = first_piece() * 64 + lane;
        if (wave != 0) return;
        float l[kPer];
        row.read(row.block[b < row.n_blocks ? b : row.n_blocks - 1], b, l);
        int e = kPer;
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i)
            if (l[i] == top) e = i;
        if (lane == __builtin_ctzll(__ballot(e < kPer))) result(row.token(b, e), 0.0);
        return;
    }
    Scale sc(set.t, top);
    if (top == INFINITY) {
        row.only_inf = true;
        sc = Scale(set.t, 0.0f);
    }
    // log-probability of a token among kept ones of this weight
    auto chosen = [&](u64 rank, u64 all) {
        result(static_cast<int32_t>(rank & kTokenMask),
               -sc.x(logit_of(rank)) * 0.69314718055994530942 - log(static_cast<double>(all) * 0x1p-43));
    };
    const Ask ask = set.ask();
    const float p = set.p, u = set.u;
    int32_t k = set.k;
    const double min_w = set.min_p > 0.0f ? ldexp(static_cast<double>(set.min_p), kBits) : 0.0;

    if (ask == Ask::kSums && top < INFINITY) {
        // ---- the weights of the pieces, then of the piece's tokens, against its own largest logit as the tile summed them
        const u64 *piece_sum = a.piece_sum + r * a.pieces;
        for (int32_t i = tid; i < a.pieces; i += kThreads)
            s.piece[i] = piece_max[i] > -INFINITY ? rescaled(piece_sum[i], piece_max[i], sc, s.power) : 0;
        __syncthreads();
        u64 pass;
        const u64 sum = find_piece(s, a.pieces, u, pass);
        if (wave != 0) return;
        const int32_t piece = s.found32[0], b = piece * 64 + lane;
        const Scale own(set.t, piece_max[piece]);
        float l[kPer];
        row.read(row.block[b < row.n_blocks ? b : row.n_blocks - 1], b, l);
        u64 w[kPer], here = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            w[e] = own.weigh(l[e], s.power);
            here += w[e];
        }
        u64 at = wave_scan(here);
        const u64 all = static_cast<u64>(__shfl(static_cast<uint32_t>(at >> 32), 63, 64)) << 32 | __shfl(static_cast<uint32_t>(at), 63, 64);
        pass = static_cast<u64>(static_cast<double>(pass - s.found[0]) * (static_cast<double>(all) / static_cast<double>(s.piece[piece])));
        if (pass >= all) pass = all - 1;
        at -= here;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (at <= pass && at + w[e] > pass) chosen(rank_of(l[e], row.token(b, e)), sum);
            at += w[e];
        }
        return;
    }

    // rank up to which min-p keeps tokens: all with at least the smallest logit that has the weight
    u64 by_min = kNone;
    auto find_by_min = [&] {
        uint32_t lo = 0x00800000u, hi = order_of(sc.m);        // from -FLT_MAX
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (sc.weight(float_of(mid), s.power) >= min_w) hi = mid;
            else lo = mid + 1;
        }
        by_min = rank_of(float_of(lo), kTokenMask);
    };
    const bool by_weight = min_w > 0.0 && !(p < 1.0f);        // min-p says by itself which tokens can be kept
    if (top < INFINITY && (ask != Ask::kNothing || by_weight)) {
        // ---- tokens and weight by the row's coarse bins, up to and with each; the bin in which the ranking is cut
        const int base = sc.coarse(top);
        int end = kCoarse - 1;
        u64 all_mass = 0, all_count = 0;
        const bool counted = ask == Ask::kCount || ask == Ask::kBoth, weighed = ask == Ask::kMass || ask == Ask::kBoth;
        auto bin_of = [&](u64 up, u64 here, u64 target) {      // of the target's token; all threads
            if (tid < kCoarse && up >= target && up - here < target) s.found32[1] = tid;
            __syncthreads();
            const int bin = s.found32[1];
            __syncthreads();
            return bin;
        };
        u64 target = 0;
        if (counted || weighed) {
            if (tid < kCoarse) {
                s.coarse_mass[tid] = 0;
                s.coarse_count[tid] = 0;
            }
            __syncthreads();
            const int64_t at = r * a.tiles * kCoarse;
            for (int32_t i = tid; i < a.tiles * kCoarse; i += kThreads) {
                const float tile_top = a.tile_max[r * a.tiles + i / kCoarse];
                const uint32_t c = counted ? a.tile_count[at + i] : 0;
                const u64 m = weighed ? a.tile_mass[at + i] : 0;
                if (c == 0 && m == 0) continue;
                const int to = i % kCoarse + sc.coarse(tile_top) - base, bin = to < kCoarse ? to : kCoarse - 1;
                if (c > 0) atomicAdd(&s.coarse_count[bin], c);
                if (m > 0) atomicAdd(&s.coarse_mass[bin], rescaled(m, tile_top, sc, s.power));
            }
            __syncthreads();
            const u64 c = tid < kCoarse && counted ? s.coarse_count[tid] : 0, m = tid < kCoarse && weighed ? s.coarse_mass[tid] : 0;
            const u64 c_up = counted ? scan(c, s.room, all_count) : 0, m_up = weighed ? scan(m, s.room, all_mass) : 0;
            if (tid < kCoarse) {
                s.coarse_count[tid] = static_cast<uint32_t>(c_up);
                s.coarse_mass[tid] = m_up;
            }
            __syncthreads();
            if (counted) {
                if (static_cast<u64>(k) > all_count) k = static_cast<int32_t>(all_count);
                end = bin_of(c_up, c, k);
            } else {
                bool rest;
                target = share_of(p, all_mass, rest);
                target += rest ? 1 : 0;
                if (target == 0) target = 1;                   // the first token
                end = bin_of(m_up, m, target);
            }
        }
        // ---- the tokens up to there, where they are few, from the pieces that can have some
        float lo = end < kCoarse - 1 ? sc.least(base + end) : -FLT_MAX;
        if (by_weight) {                                       // what is rounded here lets a few more in
            const double x = fmax(-log2(static_cast<double>(set.min_p)), 0.0) * (1.0 + 0x1p-20) + 0x1p-20;
            lo = fmaxf(lo, static_cast<float>(static_cast<double>(top) - x / sc.x_of - fabs(static_cast<double>(top)) * 0x1p-22));
        }
        auto gather_from = [&](float from) {
            for (int32_t i = tid; i < a.pieces; i += kThreads)
                if (piece_max[i] >= from) s.todo[atomicAdd(&s.n_pieces, 1u)] = i;
            __syncthreads();
            const int32_t todo = s.n_pieces;
            constexpr int kAtOnce = 4;
            for (int32_t i0 = wave; i0 < todo; i0 += kWaves * kAtOnce) {
                uint4 raw[kAtOnce];
                int32_t b[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    const int32_t at = i0 + i * kWaves;
                    b[i] = s.todo[at < todo ? at : todo - 1] * 64 + lane;
                    raw[i] = row.block[b[i] < row.n_blocks ? b[i] : row.n_blocks - 1];
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    if (i0 + i * kWaves >= todo) break;
                    float l[kPer];
                    row.read(raw[i], b[i], l);
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (l[e] >= from) {
                            const uint32_t to = atomicAdd(&s.n, 1u);
                            if (to < kList) s.list.rank[to] = rank_of(l[e], row.token(b[i], e));
                        }
                }
            }
            __syncthreads();
            const uint32_t n = s.n;
            __syncthreads();
            return n;
        };
        const bool few = !counted || s.coarse_count[end] <= kList || by_weight;
        const uint32_t n = few ? gather_from(lo) : kList + 1;
        if (n <= kShort) {
            draw_short(s, n, k, p, min_w, u, all_mass, ask == Ask::kMass, sc, chosen);
            return;
        }
        if (n <= kList) {
            draw_sorted(s, n, k, p, min_w, u, all_mass, ask == Ask::kMass, sc, chosen);
            return;
        }
        if (weighed) {
            // ---- many tokens are kept: the last one, in the bin of the cut, then the tile in which the sum passes u S
            auto cut = [&](int bin, u64 count, u64 mass, u64 &kept_mass) {
                const float from = bin < kCoarse - 1 ? sc.least(base + bin) : -FLT_MAX, to = bin > 0 ? sc.least(base + bin - 1) : INFINITY;
                const int m = gather(s, row, [&](float l, int32_t) { return l >= from && l < to; });
                if (m <= kList) return cut_run(s, row, sc, [&](float l) { return l >= from && l < to; }, m, count, mass, kept_mass);
                s.mass[tid] = 0;
                s.count[tid] = 0;
                __syncthreads();
                walk(row, [&](int32_t, const float (&l)[kPer]) {
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (l[e] >= from && l[e] < to) {
                            const int at = sc.fine(l[e], base + bin);
                            atomicAdd(&s.count[at], 1u);
                            atomicAdd(&s.mass[at], sc.weigh(l[e], s.power));
                        }
                });
                __syncthreads();
                const u64 c = s.count[tid], w = s.mass[tid];
                u64 all_c, all_w;
                const u64 c_up = scan(c, s.room, all_c), w_up = scan(w, s.room, all_w);
                // the last bin whose first token is kept
                __syncthreads();
                if (tid == 0) s.found32[0] = 0;
                __syncthreads();
                if (c > 0 && c_up - c < count && w_up - w < mass) atomicMax(&s.found32[0], static_cast<uint32_t>(tid));
                __syncthreads();
                const int fine = s.found32[0];
                __syncthreads();
                if (tid == fine) {
                    s.found[0] = c_up - c;
                    s.found[1] = w_up - w;
                    s.found32[1] = static_cast<uint32_t>(c);
                }
                __syncthreads();
                const u64 c0 = s.found[0], w0 = s.found[1], here = s.found32[1];
                __syncthreads();
                const u64 last = cut_run(s, row, sc, [&](float l) { return l >= from && l < to && sc.fine(l, base + bin) == fine; }, here,
                                         count - c0, mass > w0 ? mass - w0 : 0, kept_mass);
                kept_mass += w0;
                return last;
            };
            u64 last = kNone, in_bin;
            int bin = end;
            if (counted) {                                     // top-k, then top-p of the weight of its tokens
                const u64 c0 = bin > 0 ? s.coarse_count[bin - 1] : 0, m0 = bin > 0 ? s.coarse_mass[bin - 1] : 0;
                last = cut(bin, k - c0, kNone, in_bin);
                if (p < 1.0f) {
                    bool rest;
                    target = share_of(p, m0 + in_bin, rest);
                    target += rest ? 1 : 0;
                    if (target == 0) target = 1;
                    const u64 m_up = tid < kCoarse ? s.coarse_mass[tid] : 0, m = m_up - (tid > 0 && tid < kCoarse ? s.coarse_mass[tid - 1] : 0);
                    bin = bin_of(m_up, m, target);
                }
            }
            if (p < 1.0f) {
                const u64 m0 = bin > 0 ? s.coarse_mass[bin - 1] : 0;
                const u64 by_p = cut(bin, kNone, target - m0, in_bin);
                last = by_p < last ? by_p : last;
            }
            if (min_w > 0.0) find_by_min();
            if (by_min < last) last = by_min;
            // ---- kept weight of the tiles: their bins above the one of the last kept token, and of that one token by token
            const float lo_kept = logit_of(last);
            const int cut_at = sc.coarse(lo_kept) - base;
            bin = cut_at < kCoarse - 1 ? cut_at : kCoarse - 1;
            const float above = bin > 0 ? sc.least(base + bin - 1) : INFINITY;
            for (int32_t i = tid; i < a.tiles; i += kThreads) s.piece[i] = 0;
            __syncthreads();
            for (int32_t i = tid; i < a.tiles * kCoarse; i += kThreads) {                  // a wave: 64 bins of a tile
                const float tile_top = a.tile_max[r * a.tiles + i / kCoarse];
                const u64 m = a.tile_mass[r * a.tiles * kCoarse + i];
                const u64 w = wave_sum(m > 0 && i % kCoarse + sc.coarse(tile_top) - base < bin ? rescaled(m, tile_top, sc, s.power) : 0);
                if (lane == 0 && w > 0) atomicAdd(&s.piece[i / kCoarse], w);
            }
            walk(row, [&](int32_t b, const float (&l)[kPer]) {
                u64 w = 0;
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (l[e] >= lo_kept && l[e] < above && rank_of(l[e], row.token(b, e)) <= last) w += sc.weigh(l[e], s.power);
                if (w > 0) atomicAdd(&s.piece[b / (kTileThreads * kTileBlocks)], w);
            });
            __syncthreads();
            u64 pass;
            const u64 sum = find_piece(s, a.tiles, u, pass);
            // ---- the tile's tokens, a block to a thread, against the tile's largest logit, which is kept if any is
            static_assert(kTileThreads * kTileBlocks == kThreads, "blocks of a tile");
            const int32_t tile = s.found32[0], b = tile * kThreads + tid;
            float l[kPer];
            row.read(row.block[b < row.n_blocks ? b : row.n_blocks - 1], b, l);
            const Scale own(set.t, a.tile_max[r * a.tiles + tile]);
            u64 w[kPer], here = 0, all;
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                w[e] = there(l[e]) && rank_of(l[e], row.token(b, e)) <= last ? own.weigh(l[e], s.power) : 0;
                here += w[e];
            }
            const u64 ahead = s.found[0];
            u64 at = scan(here, s.room, all) - here;
            pass = static_cast<u64>(static_cast<double>(pass - ahead) * (static_cast<double>(all) / static_cast<double>(s.piece[tile])));
            if (pass >= all) pass = all - 1;
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (at <= pass && at + w[e] > pass) chosen(rank_of(l[e], row.token(b, e)), sum);
                at += w[e];
            }
            return;
        }
    }

    // ---- the others (+inf, more tokens than a list holds by top-k or min-p alone): tokens and weight by bins of the whole row
    if (min_w > 0.0) find_by_min();
    u64 last = by_min;                     // rank of the last kept token
    if (k > 0 || p < 1.0f) {
        s.mass[tid] = 0;
        s.count[tid] = 0;
        __syncthreads();
        walk(row, [&](int32_t b, const float (&l)[kPer]) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (!there(l[e])) continue;
                const int at = sc.bin(l[e]);
                atomicAdd(&s.count[at], 1u);
                const u64 w = sc.weigh(l[e], s.power);
                if (w > 0) atomicAdd(&s.mass[at], w);
            }
        });
        __syncthreads();
        u64 all_mass, all_count;
        const u64 mass = scan(s.mass[tid], s.room, all_mass);
        const u64 count = scan(s.count[tid], s.room, all_count);
        s.mass[tid] = mass;
        s.count[tid] = static_cast<uint32_t>(count);
        if (k <= 0 || static_cast<u64>(k) > all_count) k = static_cast<int32_t>(all_count);
        if (tid < 2) s.found32[tid] = 0;
        __syncthreads();
        u64 of_k = all_mass;
        auto cut = [&](int bin, u64 count, u64 mass, u64 &kept_mass) {
            const uint32_t n = s.count[bin] - (bin > 0 ? s.count[bin - 1] : 0);
            return cut_run(s, row, sc, [&](float l) { return sc.bin(l) == bin; }, n, count, mass, kept_mass);
        };
        if (static_cast<u64>(k) < all_count) {
            const uint32_t before = tid > 0 ? s.count[tid - 1] : 0;
            if (before < static_cast<uint32_t>(k) && count >= static_cast<uint32_t>(k)) s.found32[0] = tid;
            __syncthreads();
            const int bin = s.found32[0];
            u64 in_bin;
            const u64 by_k = cut(bin, k - (bin > 0 ? s.count[bin - 1] : 0), kNone, in_bin);
            last = by_k < last ? by_k : last;
            of_k = (bin > 0 ? s.mass[bin - 1] : 0) + in_bin;
        }
        if (p < 1.0f) {
            bool rest;
            u64 target = share_of(p, of_k, rest);
            target += rest ? 1 : 0;
            if (target == 0) target = 1;
            if ((tid > 0 ? s.mass[tid - 1] : 0) < target && mass >= target) s.found32[1] = tid;
            __syncthreads();
            const int bin = s.found32[1];
            u64 in_bin;
            const u64 by_p = cut(bin, kNone, target - (bin > 0 ? s.mass[bin - 1] : 0), in_bin);
            last = by_p < last ? by_p : last;
        }
        __syncthreads();
    }

    // ---- the kept weights along the vocabulary, by pieces of 64 blocks
    auto kept = [&](float l, int32_t token) -> u64 { return there(l) && rank_of(l, token) <= last ? sc.weigh(l, s.power) : 0; };
    const int32_t pieces = (row.n_blocks + 63) / 64;
    for (int32_t b0 = tid; b0 < pieces * 64; b0 += kThreads) {
        u64 w = 0;
        if (b0 < row.n_blocks) {
            float l[kPer];
            row.read(row.block[b0], b0, l);
#pragma unroll
            for (int e = 0; e < kPer; ++e) w += kept(l[e], row.token(b0, e));
        }
        w = wave_sum(w);
        if (lane == 0) s.piece[b0 >> 6] = w;
    }
    __syncthreads();
    u64 pass;
    const u64 sum = find_piece(s, pieces, u, pass);
    if (wave != 0) return;
    const int32_t b = s.found32[0] * 64 + lane;
    u64 w[kPer], here = 0;
    float l[kPer];
    row.read(row.block[b < row.n_blocks ? b : row.n_blocks - 1], b, l);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        w[e] = kept(l[e], row.token(b, e));
        here += w[e];
    }
    u64 at = s.found[0] + wave_scan(here) - here;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        if (at <= pass && at + w[e] > pass) chosen(rank_of(l[e], row.token(b, e)), sum);
        at += w[e];
    }
}

// Tiles of a row whose logits take `bytes` each, wherever in a block it begins.
int32_t tiles_of(int32_t V, int32_t bytes)
{
    const int32_t per = 16 / bytes, blocks = (V + 2 * per - 2) / per;
    return static_cast<int32_t>(ceil_div(blocks, kTileThreads * kTileBlocks));
}

// Where the parts of the workspace begin; [5]: its size.
struct Layout {
    int64_t at[6];
    Layout(int32_t rows, int32_t tiles)
    {
        const int64_t n = static_cast<int64_t>(rows) * tiles;
        const int64_t bytes[5] = {n * kTilePieces * 8, n * kCoarse * 8, n * kCoarse * 4, n * kTilePieces * 4, n * 4};
        at[0] = 0;
        for (int i = 0; i < 5; ++i) at[i + 1] = at[i] + ceil_div(bytes[i], 256) * 256;
    }
};

template <typename E>
int launch(Args a, int32_t rows, hipStream_t stream)
{
    MQ_LAUNCH(tile_kernel<E>, dim3(static_cast<unsigned>(rows * a.tiles)), dim3(kTileThreads), 0, stream, a);
    if (const int st = launch_status(); st != MQUANT_OK) return st;
    MQ_LAUNCH(pick_kernel<E>, dim3(static_cast<unsigned>(rows)), dim3(kThreads), 0, stream, a);
    return launch_status();
}

}  // namespace

extern "C" int64_t mquant_sample_workspace_bytes(int32_t rows, int32_t V)
{
    if (rows < 0 || V < 1) return MQUANT_ERR_BAD_SHAPE;
    if (V > kMaxTokens) return MQUANT_ERR_UNSUPPORTED;
    return Layout(rows, tiles_of(V, 4)).at[5];
}

extern "C" int mquant_sample(const void *logits, int32_t type, int64_t ld, const float *temperature, const int32_t *top_k,
                             const float *top_p, const float *min_p, const float *u, int32_t *token, float *logprob, int32_t rows,
                             int32_t V, void *workspace, int64_t workspace_bytes, mquant_stream_t stream)
{
    const int64_t need = mquant_sample_workspace_bytes(rows, V);
    if (need < 0) return static_cast<int>(need);
    if (type != MQUANT_F16 && type != MQUANT_F32) return MQUANT_ERR_BAD_SHAPE;
    if (ld < V) return MQUANT_ERR_BAD_SHAPE;
    if (rows == 0) return MQUANT_OK;
    const int32_t tiles = tiles_of(V, type == MQUANT_F16 ? 2 : 4);
    // 2^32 threads are more than a launch takes
    if (rows >= 1 << 22 || static_cast<int64_t>(rows) * tiles >= 1 << 24) return MQUANT_ERR_UNSUPPORTED;
    if (!logits || !u || !token) return MQUANT_ERR_NULL;
    if (!aligned_to(logits, type == MQUANT_F16 ? 2 : 4) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) ||
        !aligned_to(min_p, 4) || !aligned_to(u, 4) || !aligned_to(token, 4) || !aligned_to(logprob, 4))
        return MQUANT_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < need) return MQUANT_ERR_WORKSPACE;
    if (!aligned_to(workspace, 256)) return MQUANT_ERR_ALIGNMENT;
    const Layout lay(rows, tiles);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    const Args a = {logits, ld, temperature, top_k, top_p, min_p, u, token, logprob, V, tiles * kTilePieces, tiles,
                    reinterpret_cast<u64 *>(ws + lay.at[0]), reinterpret_cast<float *>(ws + lay.at[3]), reinterpret_cast<u64 *>(ws + lay.at[1]),
                    reinterpret_cast<uint32_t *>(ws + lay.at[2]), reinterpret_cast<float *>(ws + lay.at[4])};
    return type == MQUANT_F16 ? launch<_Float16>(a, rows, static_cast<hipStream_t>(stream)) : launch<float>(a, rows, static_cast<hipStream_t>(stream));
}
