// The next token of every row of logits by temperature, top-k, top-p and min-p from a given random number, for gfx950.
//
// Token i has the weight w = 2^-x, x = (m - l) log2(e) / t >= 0; ranked by logit, the kept tokens are a front of the ranking, and
// which token is drawn is a question of sums of weights.  Weights are formed in double (off by 2^-38.7 of themselves) and summed as whole
// multiples of 2^-43: such sums do not depend on their order, so that atomics in LDS give the same token every time.  2^20 tokens of
// weight 1 are 2^63.  Parts of a row are summed against their own largest logit and put together by its weight.
//
// Nothing is sorted but short runs of the ranking.  tile_kernel, a work-group to 16 KiB of a row, takes from every piece of 64 blocks of 16 bytes
// its largest logit and, as the row's settings ask, the weight of four pieces or the tokens or weights of the tile by bins of the logit.
// pick_kernel, a work-group to a row, puts them together:
//   rows without filters: the four pieces in which the sum passes u S, and the token in them;
//   what top-k, top-p and min-p can keep is, by the bins, a list of up to kList tokens: they are gathered from the pieces whose largest logit
//   can be among them, and everything is decided there, by comparing each with all (up to kShort) or by parts of the ranking and the vocabulary;
//   more tokens are kept: those of the bin in which the ranking is cut are gathered (or narrowed in the row itself, by finer bins and then digit by
//   digit of their rank, where LDS does not hold them); with the rank of the last kept token the tiles' bins give the tile in
//   which the sum passes u S, which is looked at token by token;
//   the rest (+inf among the logits, more than kList tokens by top-k or min-p alone): bins of the whole row and a walk over it by the one
//   work-group.
// What bounds them, in us a launch: tile_kernel the weights' arithmetic (256 rows of 128000 fp32 33 drawn from all, 4 TB/s; greedy 20, 6.5 TB/s from the
// last cache; 64 rows of 150001 fp16 10 and 4) or the atomics of the bins (17 by top-p); pick_kernel trips to what other L2s wrote, the gather
// and the code's own way through a cold cache (one row's 50 best of 32000 9, 64 rows' of 150001 11).
#include <cfloat>
#include <cmath>

#include "serving_common.h"

using namespace mquant;

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxTokens = 1 << 20;
constexpr int kBins = 1024;                // parts of a ranking or of the vocabulary, one to a thread
constexpr int kCoarse = 256;               // bins of a tile: 1/4 of x wide, the last one has all that is left
constexpr int kTileThreads = 256, kTileBlocks = 4, kTilePieces = kTileThreads / 64 * kTileBlocks;
constexpr int kMaxPieces = ((kMaxTokens + 6) / 4 + kTileThreads * kTileBlocks - 1) / (kTileThreads * kTileBlocks) * kTilePieces;    // fp32, tiles filled up
constexpr int kShort = 256;                // tokens of a list up to which each is compared with all others
constexpr int kList = 2048;                // tokens that are sorted at a time, two to a thread
constexpr int kHold = 8192;                // tokens that are held in LDS: a list, or those of one bin
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
    float *piece_max;                      // [rows, pieces]; -inf where no token can be chosen
    u64 *four_sum;                         // [rows, pieces / 4] weight of four pieces (of a wave) against their largest logit ..
    float *four_max;                       // .. which is here
    u64 *tile_bins;                        // [rows, tiles, kCoarse] tokens, or weight against the tile's largest logit
    u64 *tile_mass;                        // [rows, tiles, kCoarse] weight, where both are asked for
    float *tile_max;                       // [rows, tiles]; -inf as above
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

// What a row's threads share.
struct Shared {
    u64 mass[kBins];
    uint32_t count[kBins];
    u64 coarse_mass[kCoarse];
    uint32_t coarse_count[kCoarse];
    union {
        struct {
            u64 rank[kList], sum[kList];
        } list;
        u64 piece[kMaxPieces];             // weight of 64 blocks of 16 bytes, or of a tile
        struct {
            u64 mass[256];
            uint32_t count[256];
        } digit;
    };
    u64 held[kHold];                       // tokens by their rank, as they came
    u64 room[kWaves];
    u64 found[2];
    uint32_t found32[2];
    uint32_t n, n_pieces, n_held, at_least;
};

__device__ __forceinline__ Shared &lds()
{
    __shared__ Shared s;
    return s;
}

// ---- a row's logits: the 16-byte blocks that hold it, from the aligned one in which it begins
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

template <typename E>
struct Row {
    static constexpr int kPer = 16 / sizeof(E);
    // in so many words memory: an address that went through a whole number is taken for one that may be in LDS, and a load from it
    // waits for LDS too
    const __attribute__((address_space(1))) v4u *block;
    int32_t skip, n_blocks, V;             // elements of the first block ahead of the row
    bool only_inf;                         // where +inf occurs, it counts as 0 and everything else as nothing

    __device__ __forceinline__ Row(const Args &a, int64_t row) : V(a.V), only_inf(false)
    {
        const uintptr_t p = reinterpret_cast<uintptr_t>(static_cast<const E *>(a.logits) + row * a.ld);
        skip = static_cast<int32_t>((p & 15) / sizeof(E));
        block = (const __attribute__((address_space(1))) v4u *)(p & ~static_cast<uintptr_t>(15));
        n_blocks = (skip + V + kPer - 1) / kPer;
    }

    __device__ __forceinline__ v4u load(int32_t b) const { return block[b < n_blocks ? b : n_blocks - 1]; }

    // Token number of element e of block b; outside [0, V): not of the row.
    __device__ __forceinline__ int32_t token(int32_t b, int e) const { return b * kPer + e - skip; }

    __device__ __forceinline__ float value(float l) const { return !only_inf ? l : l == INFINITY ? 0.0f : NAN; }

    // The logit of a token that is in reach already.
    __device__ __forceinline__ float logit(int32_t token) const { return value(static_cast<float>(((const __attribute__((address_space(1))) E *)block)[token + skip])); }

    // The logits of a block that is all of the row's.
    __device__ __forceinline__ void read(const v4u &raw, float (&l)[kPer]) const
    {
        union {
            v4u u;
            E e[kPer];
        } x;
        x.u = raw;
#pragma unroll
        for (int e = 0; e < kPer; ++e) l[e] = value(static_cast<float>(x.e[e]));
    }

    // Block b with NaN for what is not of the row.
    __device__ __forceinline__ v4u blank(const v4u &raw, int32_t b) const
    {
        union {
            v4u u;
            E e[kPer];
        } x;
        x.u = raw;
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (static_cast<uint32_t>(token(b, e)) >= static_cast<uint32_t>(V)) x.e[e] = static_cast<E>(NAN);
        return x.u;
    }

    // The logits of block b, NaN for what is not of the row.
    __device__ __forceinline__ void read(const v4u &raw, int32_t b, float (&l)[kPer]) const
    {
        read(raw, l);
        if (b == 0 || b >= n_blocks - 1) {
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (static_cast<uint32_t>(token(b, e)) >= static_cast<uint32_t>(V)) l[e] = NAN;
        }
    }
};

// Whether a token with this logit can be chosen: neither -inf nor NaN.
__device__ __forceinline__ bool there(float l) { return l > -INFINITY; }

// ---- over the work-group
__device__ __forceinline__ u64 wave_sum(u64 x) { return from_lane(wave_scan(x), 63); }

// Up to and with this thread; `all`: over all threads.  Ends behind a barrier that frees nothing: a barrier has to come before the next use.
__device__ __forceinline__ u64 scan(u64 x, u64 *room, u64 &all)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    x = wave_scan(x);
    __syncthreads();
    if (lane == 63) room[wave] = x;
    __syncthreads();
    const u64 sums = wave_scan(lane < kWaves ? room[lane] : 0);
    all = from_lane(sums, kWaves - 1);
    return wave > 0 ? x + from_lane(sums, wave - 1) : x;
}

// ---- ranks: the larger the logit and the lower the token's number, the smaller
__device__ __forceinline__ uint32_t order_of(float l)          // rises with l
{
    const uint32_t b = __float_as_uint(l + 0.0f);              // -0 ranks with 0
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ float float_of(uint32_t order) { return __uint_as_float(order ^ (order >> 31 ? 0x80000000u : 0xffffffffu)); }

// The largest of a wave's logits, -inf where there is none (NaN is not one); as whole numbers, since those are moved and compared in one
// instruction.
__device__ __forceinline__ float wave_max(float x)
{
    uint32_t o = order_of(fmaxf(x, -INFINITY));
    auto with = [&](uint32_t y) { o = o > y ? o : y; };
    with(moved<0x111, 0xf>(o, 0u));
    with(moved<0x112, 0xf>(o, 0u));
    with(moved<0x114, 0xf>(o, 0u));
    with(moved<0x118, 0xf>(o, 0u));
    with(moved<0x142, 0xa>(o, 0u));
    with(moved<0x143, 0xc>(o, 0u));
    return float_of(__builtin_amdgcn_readlane(o, 63));
}

// The same of four logits a lane at once: the largest of number i in the lanes 16 i .. 16 i + 15.
__device__ __forceinline__ float four_max(float x0, float x1, float x2, float x3)
{
    auto swapped = [](float a, float b, auto swap) {           // exchanges parts of a wave, then the larger of both
        const auto r = swap(__float_as_uint(a), __float_as_uint(b));
        return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    };
    auto halves = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane32_swap(a, b, false, false); };
    auto rows = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane16_swap(a, b, false, false); };
    uint32_t o = order_of(fmaxf(swapped(swapped(x0, x2, halves), swapped(x1, x3, halves), rows), -INFINITY));
    auto with = [&](uint32_t y) { o = o > y ? o : y; };
    with(moved<0xb1, 0xf>(o, 0u));                             // of a pair, a quad, by mirrored halves and rows
    with(moved<0x4e, 0xf>(o, 0u));
    with(moved<0x141, 0xf>(o, 0u));
    with(moved<0x140, 0xf>(o, 0u));
    return float_of(o);
}

__device__ __forceinline__ u64 rank_of(float l, int32_t token)
{
    return static_cast<u64>(~order_of(l)) << kIndexBits | static_cast<uint32_t>(token);
}

__device__ __forceinline__ float logit_of(u64 rank) { return float_of(~static_cast<uint32_t>(rank >> kIndexBits)); }

// ---- weights
typedef uint32_t words __attribute__((ext_vector_type(2)));    // of a double, the low one first

// As a multiple of 2^-43, to the nearest, below 2^52 of them.
__device__ __forceinline__ u64 whole(double w)
{
    return static_cast<u64>(__double_as_longlong(__builtin_fma(w, 0x1p43, 0x1p52))) & ((1ull << 52) - 1);
}

struct Scale {
    double x_of;                           // log2(e) / t; not 0, so that x_end is a number
    double x_end;                          // m - l at which weights count as nothing
    float bin_of;                          // 16 x_of, for the bins
    float m;                               // the largest logit

    __device__ __forceinline__ Scale(float t, float top) : x_of(fmax(1.4426950408889634074 / static_cast<double>(t), 1e-60)), m(top)
    {
        x_end = fmin(693.14718055994530942 * static_cast<double>(t), 1e63);
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

    // The same by a wave at once, 64 floats around where the bins' border is but for what is rounded.
    __device__ __forceinline__ float least_near(int bin) const
    {
        const float near = static_cast<float>(bin + 1) / (-0.25f * bin_of);
        const float l = float_of(order_of(fminf(fmaxf(near, -1e38f), 1e38f)) + (threadIdx.x & 63) - 32);
        const uint64_t in = __ballot(coarse(l) <= bin);        // of the lanes from some one on
        const int from = in != 0 ? __builtin_ctzll(in) : 0;
        return from > 0 ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l), from)) : least(bin);
    }

    __device__ double x(float l) const { return (static_cast<double>(m) - static_cast<double>(l)) * x_of; }
    // Falls with l, like the rank, whatever is rounded; the last bin has all that is left.
    __device__ int bin(float l) const { return static_cast<int>(fminf((m - l) * bin_of, static_cast<float>(kBins - 1))); }

    // 2^-x, nothing (2^-1000) for what is no logit.  With -n the whole number next to -x, 2^(n - x) is a polynomial of degree 8 in n - x, which is
    // 1 at 0 (interpolated at the zeros of a Chebyshev polynomial, off by 2^-38.7 at most).  -n is found by adding 1.5 2^52 and is in
    // the low bits then.  (A table in LDS for a shorter polynomial is slower: lanes ask for any of its entries.)
    __device__ __forceinline__ double weight(float l) const
    {
        constexpr double kRound = 0x1.8p52;
        const double d = __builtin_fmax(static_cast<double>(l) - static_cast<double>(m), -x_end);
        const double t = __builtin_fma(d, x_of, kRound), n = t - kRound, y = __builtin_fma(d, x_of, -n);
        double p = 0x1.63b2d7971923fp-20;
        p = __builtin_fma(p, y, 0x1.00c0e4e15189cp-16);
        p = __builtin_fma(p, y, 0x1.4308c7183d6a2p-13);
        p = __builtin_fma(p, y, 0x1.5d877598350dep-10);
        p = __builtin_fma(p, y, 0x1.3b2ab70ad2565p-7);
        p = __builtin_fma(p, y, 0x1.c6b08da70cce3p-5);
        p = __builtin_fma(p, y, 0x1.ebfbdff82a734p-3);
        p = __builtin_fma(p, y, 0x1.62e42fef9cc69p-1);
        p = __builtin_fma(p, y, 1.0);
        words w = __builtin_bit_cast(words, p);
        w[1] += __builtin_bit_cast(words, t)[0] << 20;
        return __builtin_bit_cast(double, w);
    }
    __device__ __forceinline__ u64 weigh(float l) const { return whole(weight(l)); }
};

// floor(f * n) for f in [0, 1], and whether there is a remainder: f is a 24-bit number times 2^-down.
__device__ __forceinline__ u64 share_of(float f, u64 n, bool &rest)
{
    rest = false;
    if (!(f > 0.0f)) return 0;
    if (f >= 1.0f) return n;
    const uint32_t bits = __float_as_uint(f), e = bits >> 23;
    const u64 mantissa = e > 0 ? (bits & 0x7fffff) | 0x800000 : bits;
    const int down = e > 0 ? 150 - static_cast<int>(e) : 149;                  // 24 at least
    const u64 lo = (n & 0xffffffff) * mantissa, hi = (n >> 32) * mantissa + (lo >> 32);        // the product is hi 2^32 + lo % 2^32
    const uint32_t low = static_cast<uint32_t>(lo);
    if (down >= 96) {
        rest = n > 0;
        return 0;
    }
    if (down >= 32) {
        rest = low != 0 || (hi & ((1ull << (down - 32)) - 1)) != 0;
        return hi >> (down - 32);
    }
    rest = (low & ((1u << down) - 1)) != 0;
    return hi << (32 - down) | low >> down;
}

// floor(u * sum), below the sum.
__device__ __forceinline__ u64 drawn_at(float u, u64 sum)
{
    bool rest;
    const u64 at = share_of(u, sum, rest);
    return at < sum ? at : sum - 1;
}

// The weight ahead of a token has to be below this to keep it: p * sum, rounded up, 1 at least.
__device__ __forceinline__ u64 target_of(float p, u64 sum)
{
    bool rest;
    const u64 at = share_of(p, sum, rest) + (rest ? 1 : 0);
    return at > 0 ? at : 1;
}

// What to do with the tokens of four blocks that `is` names by their logit: f(logit, token).  Found for all of them first, done one by one, so
// that the code of f is there once.
template <typename E, typename P, typename F>
__device__ __forceinline__ void each_of(const Row<E> &row, const v4u (&raw)[4], const int32_t (&b)[4], P is, F f)
{
    // eight tokens a block: one block at a time, since code that runs once is waited for (four at a time 1 us more, one row of 32000 15.2 us); of
    // four tokens that is no longer so (12.7 us, 13.0 by one)
    constexpr int kPer = Row<E>::kPer, kUnroll = kPer == 8 ? 1 : 4;
    // by name: an array that the program indexes is given 16 KiB of LDS or scratch memory (50 best of 256 rows of 128000: 49 us, 37 by name)
    const int32_t b0 = b[0], b1 = b[1], b2 = b[2], b3 = b[3];
    uint32_t hits = 0;
    v4u r0 = raw[0], r1 = raw[1], r2 = raw[2], r3 = raw[3];
    int32_t c0 = b0, c1 = b1, c2 = b2, c3 = b3;
#pragma unroll kUnroll
    for (int i = 0; i < 4; ++i) {
        float l[kPer];
        row.read(r0, c0, l);
        const bool in = c0 < row.n_blocks;
        hits >>= kPer;
#pragma unroll
        for (int e = 0; e < kPer; ++e) hits |= is(l[e]) && in ? 1u << (3 * kPer + e) : 0u;
        r0 = r1;
        r1 = r2;
        r2 = r3;
        c0 = c1;
        c1 = c2;
        c2 = c3;
    }
#pragma unroll 1
    while (hits != 0) {
        const int h = __builtin_ctz(hits), i = h / kPer;
        hits &= hits - 1;
        int32_t block = b0;
        block = i == 1 ? b1 : block;
        block = i == 2 ? b2 : block;
        block = i == 3 ? b3 : block;
        const int32_t token = row.token(block, h % kPer);
        f(row.logit(token), token);
    }
}

__device__ __forceinline__ void put_held(float l, int32_t token)
{
    const uint32_t at = atomicAdd(&lds().n, 1u);
    if (at < kHold) lds().held[at] = rank_of(l, token);
}

// Takes the tokens of four blocks into the held ones, as far as there is room; n counts them.  A wave asks for its places once.
template <typename E, typename P>
__device__ __forceinline__ void hold_blocks(const Row<E> &row, const v4u (&raw)[4], const int32_t (&b)[4], P is, uint32_t &n)
{
    constexpr int kPer = Row<E>::kPer, kMany = 256;
    uint32_t hits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float l[kPer];
        row.read(raw[i], b[i], l);
#pragma unroll
        for (int e = 0; e < kPer; ++e) hits |= is(l[e]) && b[i] < row.n_blocks ? 1u << (i * kPer + e) : 0u;
    }
    const uint32_t mine = __builtin_popcount(hits), up = wave_scan(mine), total = from_lane(up, 63);
    if (total == 0) return;
    uint32_t at = 0;
    if ((threadIdx.x & 63) == 0) at = atomicAdd(&n, total);
    at = __builtin_amdgcn_readfirstlane(at) + up - mine;
    u64 *to = lds().held;
    if (total > kMany) {                   // one by one, each of a lane's would be waited for
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float l[kPer];
            row.read(raw[i], b[i], l);
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (hits >> (i * kPer + e) & 1) {
                    if (at < kHold) to[at] = rank_of(l[e], row.token(b[i], e));
                    ++at;
                }
        }
        return;
    }
    const int32_t b0 = b[0], b1 = b[1], b2 = b[2], b3 = b[3];
#pragma unroll 1
    for (; hits != 0; hits &= hits - 1, ++at) {
        const int h = __builtin_ctz(hits), i = h / kPer;
        int32_t block = b0;
        block = i == 1 ? b1 : block;
        block = i == 2 ? b2 : block;
        block = i == 3 ? b3 : block;
        const int32_t token = row.token(block, h % kPer);
        if (at < kHold) to[at] = rank_of(row.logit(token), token);
    }
}

// The same for the whole row.
template <typename E>
struct InRow {
    const Row<E> &row;

    template <typename P, typename F>
    __device__ __forceinline__ void each(P is, F f) const
    {
#pragma unroll 1
        for (int32_t b0 = threadIdx.x; b0 < row.n_blocks; b0 += kThreads * 4) {
            v4u raw[4];
            int32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                b[i] = b0 + i * kThreads;
                raw[i] = row.load(b[i]);
            }
            each_of(row, raw, b, is, f);
        }
    }

    template <typename P>
    __device__ __forceinline__ void hold(P is, uint32_t &n) const
    {
#pragma unroll 1
        for (int32_t b0 = threadIdx.x; b0 - static_cast<int32_t>(threadIdx.x & 63) < row.n_blocks; b0 += kThreads * 4) {       // whole waves
            v4u raw[4];
            int32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                b[i] = b0 + i * kThreads;
                raw[i] = row.load(b[i]);
            }
            hold_blocks(row, raw, b, is, n);
        }
    }
};

// And for the n tokens that LDS holds.
struct Held {
    int n;

    template <typename P, typename F>
    __device__ __forceinline__ void each(P is, F f) const
    {
        const u64 *rank = lds().held;
#pragma unroll 1
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float l = logit_of(rank[i]);
            if (is(l)) f(l, static_cast<int32_t>(rank[i] & ((1u << kIndexBits) - 1)));
        }
    }
};

// What a row's work-group knows when its way is one of the functions below.  Those write the row's result themselves and get what they need through
// memory: what is passed or kept around a call would be held in scratch memory by every call, also of rows that go another way.
struct Known {
    Settings set;
    Scale sc;
    float top;
    double min_w;
    int32_t k;
    int base, end;                         // first coarse bin, and the one of the cut
    u64 target;                            // of top-p alone
    u64 all_mass;                          // weight of all tokens that can be chosen, 0: not known
    float least;                           // the smallest logit of a list
};

__device__ __forceinline__ Known &known()
{
    __shared__ u64 room[(sizeof(Known) + 7) / 8];
    return *reinterpret_cast<Known *>(room);
}

// The row's token and its log-probability.
__device__ __forceinline__ void put_result(const Args &a, int64_t r, int32_t token, double logprob)
{
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = static_cast<float>(logprob);
}

// A thread's answer: the token that is drawn, by its rank, among kept ones of this weight; kNone: another thread has it.
struct Drawn {
    u64 rank = kNone, sum = 0;

    __device__ __forceinline__ void write(const Args &a, int64_t r, const Scale &sc) const
    {
        if (rank == kNone) return;
        // the log-probability of a token among kept ones of this weight
        put_result(a, r, static_cast<int32_t>(rank & ((1u << kIndexBits) - 1)),
                -sc.x(logit_of(rank)) * 0.69314718055994530942 - log(static_cast<double>(sum) * 0x1p-43));
    }
};

// ---- lists
__device__ __forceinline__ void put(float l, int32_t token)
{
    const uint32_t at = atomicAdd(&lds().n, 1u);
    if (at < kList) lds().list.rank[at] = rank_of(l, token);
}

// Sorts the n <= kList numbers of the list, rising; all threads.
__device__ __forceinline__ void sort_list(int n)
{
    u64 *v = lds().list.rank;
    int size = 2;
    while (size < n) size <<= 1;
    for (int i = threadIdx.x; i < size; i += kThreads)
        if (i >= n) v[i] = kNone;
#pragma unroll 1
    for (int k = 2; k <= size; k <<= 1)
#pragma unroll 1
        for (int j = k >> 1; j > 0; j >>= 1) {
            // up to a distance of 64 a wave's pairs are its own 128 numbers
            if (j > 64 || (j == 64 && k > 128) || k == 2) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int t = threadIdx.x, i = ((t & ~(j - 1)) << 1) | (t & (j - 1));
            static_assert(kList == 2 * kThreads, "pairs of a thread");
            if (t < size >> 1) {
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
__device__ __forceinline__ void sum_list(int n, const Scale &sc)
{
    Shared &s = lds();
    const int i = threadIdx.x * 2;
    const u64 x = i < n ? sc.weigh(logit_of(s.list.rank[i])) : 0, y = i + 1 < n ? sc.weigh(logit_of(s.list.rank[i + 1])) : 0;
    u64 all;
    const u64 up = scan(x + y, s.room, all);
    s.list.sum[i] = up - y;
    s.list.sum[i + 1] = up;
    __syncthreads();
}

// How many threads' `is` are true, twice a thread.
__device__ __forceinline__ int count_all(bool is, bool is_too)
{
    Shared &s = lds();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    const uint32_t mine = (is ? 1 : 0) + (is_too ? 1 : 0);
    if (mine > 0) atomicAdd(&s.n, mine);
    __syncthreads();
    const int k = s.n;
    __syncthreads();
    return k;
}

// How many of the list's n sorted tokens, with sums of weights up to and with each, a cut keeps: the first `count` of them at most, and only
// those with less than `mass` before them; one at least.
__device__ __forceinline__ int cut_list(int n, u64 count, u64 mass)
{
    const u64 *sum = lds().list.sum;
    const int i = threadIdx.x * 2;
    auto kept = [&](int i) { return i < n && static_cast<u64>(i) < count && (i == 0 ? 0 : sum[i - 1]) < mass; };
    const int k = count_all(kept(i), kept(i + 1));
    return k > 1 ? k : 1;
}

// The first of the kCoarse bins up to which their sum reaches target(whole sum), or the last one, and the sum ahead of it; a wave by
// itself, four bins a lane.
template <typename N, typename F>
__device__ __forceinline__ int bin_in(const N *bins, F target, N &ahead)
{
    static_assert(kCoarse == 4 * 64, "bins of a lane");
    const int lane = threadIdx.x & 63;
    const N b0 = bins[lane * 4], b1 = bins[lane * 4 + 1], b2 = bins[lane * 4 + 2], b3 = bins[lane * 4 + 3];
    const N up = wave_scan<N>(b0 + b1 + b2 + b3);
    const N t = target(from_lane(up, 63));
    const uint64_t reached = __ballot(up >= t);
    const int at = reached != 0 ? __builtin_ctzll(reached) : 63;
    N sum = up - b0 - b1 - b2 - b3;        // of the lane, the bin and the sum ahead of it
    int bin = lane * 4;
    if (sum + b0 < t) sum += b0, ++bin;
    if (bin == lane * 4 + 1 && sum + b1 < t) sum += b1, ++bin;
    if (bin == lane * 4 + 2 && sum + b2 < t) sum += b2, ++bin;
    ahead = from_lane(sum, at);
    return __builtin_amdgcn_readlane(bin, at);
}

// Weight against the row's largest logit of what weighs `sum` against the logit l.
__device__ __forceinline__ u64 rescaled(u64 sum, float l, const Scale &sc)
{
    return static_cast<u64>(rint(static_cast<double>(sum) * sc.weight(l)));
}

// For each of n <= kShort numbers in LDS, how many are less: `ahead`, zeros before (rows of 0 count none).  A lane holds one, and all waves have a share
// of those that it is compared with, which every lane reads at once.
template <typename N>
__device__ __forceinline__ void count_ahead(const N *v, int n, uint32_t *ahead)
{
    static_assert(kShort == 4 * 64 && kWaves == 16, "shares of a wave");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int log2 = n <= 64 ? 0 : n <= 128 ? 1 : 2, group = wave & ((1 << log2) - 1), part = wave >> log2;
    const int t = group * 64 + lane, per = (n + (kWaves >> log2) - 1) >> (4 - log2), from = part * per, to = from + per < n ? from + per : n;
    const N mine = t < n ? v[t] : 0;
    uint32_t count = 0;
#pragma unroll 4
    for (int j = from; j < to; ++j) count += v[j] < mine ? 1 : 0;
    if (count > 0) atomicAdd(&ahead[t], count);
}

// Which of the list's n <= kShort tokens is drawn.  Their places in the ranking and then, of the kept ones, along the vocabulary are counted by all
// waves, not sorted (220 tokens of 64 rows of 150001: 22 us for the kernel, sorted 32).  The rest is the first wave's, four tokens a lane,
// without barriers: an instruction that all 16 waves run takes the work-group 16 cycles, one wave's 4.
__device__ __forceinline__ Drawn draw_short(int n, int32_t k, float p, double min_w, float u, u64 all_mass, bool all_known, const Scale &sc)
{
    Shared &s = lds();
    constexpr uint32_t kTokenMask = (1u << kIndexBits) - 1;
    constexpr int kHeld = kShort / 64;
    uint32_t *place = s.coarse_count, *kept_place = s.count, *kept_token = s.count + kShort;
    static_assert(kBins >= 2 * kShort && kCoarse >= kShort, "room for them");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid < kShort) place[tid] = kept_place[tid] = 0;
    __syncthreads();
    count_ahead(s.held, n, place);
    __syncthreads();
    u64 held[kHeld];
    u64 sum = 0, weight[kHeld];
    uint32_t n_kept = 0;
    if (wave == 0) {
#pragma unroll
        for (int g = 0; g < kHeld; ++g) held[g] = g * 64 + lane < n ? s.held[g * 64 + lane] : kNone;
        // ---- along the ranking: token lane + 64 g goes to its place, then a lane has four places next to each other
        u64 *by_place = s.list.sum;
#pragma unroll
        for (int g = 0; g < kHeld; ++g) {
            weight[g] = 0;
            const int i = g * 64 + lane;
            if (g * 64 < n && i < n) {
                weight[g] = sc.weigh(logit_of(held[g]));
                by_place[place[i]] = weight[g];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        u64 w[kHeld], here = 0;
#pragma unroll
        for (int e = 0; e < kHeld; ++e) here += w[e] = lane * kHeld + e < n ? by_place[lane * kHeld + e] : 0;
        u64 ahead = wave_scan(here) - here;
        if (k <= 0 || k > n) k = n;
        u64 mass = kNone;                                      // a kept token has less ahead of it
        if (p < 1.0f) {
            u64 of_k = 0;
#pragma unroll
            for (int e = 0; e < kHeld; ++e) of_k += lane * kHeld + e < k ? w[e] : 0;
            mass = target_of(p, all_known ? all_mass : wave_sum(of_k));
        }
        u64 at = ahead;
#pragma unroll
        for (int e = 0; e < kHeld; ++e) {
            n_kept += __builtin_popcountll(__ballot(lane * kHeld + e < k && at < mass));
            at += w[e];
        }
        if (min_w > 0.0) {                                     // the kept ones are the ranking's first ones by weight too
            uint32_t heavy = 0;
#pragma unroll
            for (int g = 0; g < kHeld; ++g)
                if (g * 64 < n) heavy += __builtin_popcountll(__ballot(g * 64 + lane < n && sc.weight(logit_of(held[g])) >= min_w));
            n_kept = heavy < n_kept ? heavy : n_kept;
            n_kept = n_kept > 1 ? n_kept : 1;
        }
#pragma unroll
        for (int e = 0; e < kHeld; ++e) sum += lane * kHeld + e < static_cast<int>(n_kept) ? w[e] : 0;
        sum = wave_sum(sum);
#pragma unroll
        for (int g = 0; g < kHeld; ++g) {
            const int i = g * 64 + lane;
            if (g * 64 < n && i < n) {
                const bool kept = place[i] < n_kept;
                kept_token[i] = kept ? static_cast<uint32_t>(held[g]) & kTokenMask : ~0u;
            }
        }
    }
    __syncthreads();
    count_ahead(kept_token, n, kept_place);
    __syncthreads();
    Drawn d;
    if (wave != 0) return d;
    // ---- the kept ones along the vocabulary, as above; the others come last
    u64 *by_place = s.list.sum;
    uint32_t *who = kept_token;
#pragma unroll
    for (int g = 0; g < kHeld; ++g) {
        const int i = g * 64 + lane;
        if (g * 64 < n && i < n && place[i] < n_kept) {        // the others come behind all kept ones
            by_place[kept_place[i]] = weight[g];
            who[kept_place[i]] = i;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    u64 w[kHeld], here = 0;
#pragma unroll
    for (int e = 0; e < kHeld; ++e) here += w[e] = lane * kHeld + e < static_cast<int>(n_kept) ? by_place[lane * kHeld + e] : 0;
    u64 at = wave_scan(here) - here;
    const u64 pass = drawn_at(u, sum);
#pragma unroll
    for (int e = 0; e < kHeld; ++e) {
        if (at <= pass && at + w[e] > pass) d = {s.held[who[lane * kHeld + e]], sum};
        at += w[e];
    }
    return d;
}

// The piece in which the sum passes u's share of it, of `pieces` sums in s.piece, and the sum ahead of it, for all threads: s.found32[0],
// s.found[0].  Returns the whole sum; `pass` is u's share.
__device__ __forceinline__ u64 find_piece(int32_t pieces, float u, u64 &pass)
{
    Shared &s = lds();
    // every thread takes the pieces from..to, next to each other
    const int32_t per = (pieces + kThreads - 1) / kThreads, from = threadIdx.x * per, to = from + per < pieces ? from + per : pieces;
    u64 mine = 0, sum;
#pragma unroll 1
    for (int32_t i = from; i < to; ++i) mine += s.piece[i];
    const u64 up = scan(mine, s.room, sum);
    pass = drawn_at(u, sum);
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

// Of a block's tokens with their weights, the one in which the sum passes `pass`, where `at` is the sum ahead of the block.
template <typename E>
__device__ __forceinline__ u64 pick_token(const Row<E> &row, int32_t b, const float (&l)[Row<E>::kPer], const u64 (&w)[Row<E>::kPer], u64 at, u64 pass)
{
    u64 rank = kNone;
#pragma unroll
    for (int e = 0; e < Row<E>::kPer; ++e) {
        if (at <= pass && at + w[e] > pass) rank = rank_of(l[e], row.token(b, e));
        at += w[e];
    }
    return rank;
}

// ---- long lists
// The rank of the last token that a cut keeps of the n tokens that `of` names by their logit, a run of the ranking: by rank the first `count` of them
// (at least 1, at most all), and only those with less than `mass` of their weight before them (the first one has).  kept_mass: the weight of
// those kept.
template <typename S, typename F>
__device__ __forceinline__ u64 cut_run(const S &tokens, const Scale &sc, F of, u64 n, u64 count, u64 mass, u64 &kept_mass)
{
    Shared &s = lds();
    const int tid = threadIdx.x;
    u64 prefix = 0, passed = 0;            // digits of the rank that are known, weight of the tokens ahead of them
    int low = 32 + kIndexBits;             // bits that are not
#pragma unroll 1
    while (n > kList) {
        low -= 8;
        __syncthreads();
        if (tid < 256) {
            s.digit.mass[tid] = 0;
            s.digit.count[tid] = 0;
        }
        __syncthreads();
        tokens.each(of, [&](float l, int32_t token) {
            const u64 r = rank_of(l, token);
            if (r >> low >> 8 != prefix) return;
            atomicAdd(&s.digit.mass[r >> low & 255], sc.weigh(l));
            atomicAdd(&s.digit.count[r >> low & 255], 1u);
        });
        __syncthreads();
        if (tid == 0) {                    // the digit of the last token that the cut keeps
            u64 c = 0, w = 0, c_at = 0, w_at = 0;
            int d = -1;
#pragma unroll 1
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
    }
    __syncthreads();
    if (tid == 0) s.n = 0;
    __syncthreads();
    tokens.each(of, [&](float l, int32_t token) {
        if (rank_of(l, token) >> low == prefix) put(l, token);
    });
    __syncthreads();
    const int m = s.n;
    __syncthreads();
    if (m <= 64) {                         // by one wave, each compared with all
        if (tid < 64) {
            const u64 mine = tid < m ? s.list.rank[tid] : kNone, weight = tid < m ? sc.weigh(logit_of(mine)) : 0;
            s.list.sum[tid] = weight;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            u64 ahead = 0;
            uint32_t before = 0;
#pragma unroll 2
            for (int j = 0; j < m; ++j) {
                const bool less = s.list.rank[j] < mine;
                before += less ? 1 : 0;
                ahead += less ? s.list.sum[j] : 0;
            }
            const bool kept = tid < m && (before == 0 || (before < count && ahead < mass));
            const u64 sum = wave_sum(kept ? weight : 0);
            if (kept && before + 1 == __builtin_popcountll(__ballot(kept))) {
                s.found[0] = mine;
                s.found[1] = sum;
            }
        }
        __syncthreads();
        const u64 last = s.found[0];
        kept_mass = passed + s.found[1];
        __syncthreads();
        return last;
    }
    sort_list(m);
    sum_list(m, sc);
    const int k = cut_list(m, count, mass);
    kept_mass = passed + s.list.sum[k - 1];
    const u64 last = s.list.rank[k - 1];
    __syncthreads();
    return last;
}

// The same of a run that may be long: counted by kBins parts first, and the part of the cut is then the run.
template <typename S, typename F, typename B>
__device__ __forceinline__ u64 cut_by_parts(const S &tokens, const Scale &sc, F of, B part_of, u64 count, u64 mass, u64 &kept_mass)
{
    Shared &s = lds();
    const int tid = threadIdx.x;
    __syncthreads();
    s.mass[tid] = 0;
    s.count[tid] = 0;
    if (tid == 0) s.found32[0] = 0;
    __syncthreads();
    tokens.each(of, [&](float l, int32_t) {
        const int at = part_of(l);
        atomicAdd(&s.count[at], 1u);
        atomicAdd(&s.mass[at], sc.weigh(l));
    });
    __syncthreads();
    const u64 c = s.count[tid], w = s.mass[tid];
    u64 all;
    const u64 c_up = scan(c, s.room, all), w_up = scan(w, s.room, all);
    if (c > 0 && c_up - c < count && w_up - w < mass) atomicMax(&s.found32[0], static_cast<uint32_t>(tid));    // the last part whose first token is kept
    __syncthreads();
    const int part = s.found32[0];
    __syncthreads();
    if (tid == part) {
        s.found[0] = c_up - c;
        s.found[1] = w_up - w;
        s.found32[1] = static_cast<uint32_t>(c);
    }
    __syncthreads();
    const u64 c0 = s.found[0], w0 = s.found[1], n = s.found32[1];
    __syncthreads();
    const u64 last = cut_run(tokens, sc, [&](float l) { return of(l) && part_of(l) == part; }, n, count - c0, mass > w0 ? mass - w0 : 0, kept_mass);
    kept_mass += w0;
    return last;
}

// Rank up to which min-p keeps tokens: all with at least the smallest logit that has the weight.
__device__ __forceinline__ u64 last_by_weight(const Scale &sc, double min_w)
{
    uint32_t lo = 0x00800000u, hi = order_of(sc.m);            // from -FLT_MAX
#pragma unroll 1
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (sc.weight(float_of(mid)) >= min_w) hi = mid;
        else lo = mid + 1;
    }
    return rank_of(float_of(lo), (1 << kIndexBits) - 1);
}

// Which of the n <= kHold tokens held is drawn: the last kept one by parts of the ranking, then the weights of the kept ones by parts of the
// vocabulary, and of the part in which the sum passes u S a thread has one token.  (Sorted by rank and then by their number, 1900 tokens took
// 45 us.)
__device__ __noinline__ void draw_list(const Args *args, int64_t r, int n)
{
    Shared &s = lds();
    const Known w = known();
    const Scale &sc = w.sc;
    const int tid = threadIdx.x;
    const Held tokens = {n};
    const float p = w.set.p, scale = fmaxf((kBins - 0.5f) / (sc.m - w.least), sc.bin_of);
    auto any = [](float) { return true; };
    auto part_of = [&](float l) { return static_cast<int>(fminf((sc.m - l) * scale, kBins - 1.0f)); };
    u64 last = kNone, of_k = w.all_mass, none;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {                     // top-k (or all tokens, for their weight), then top-p
        if (pass == 0 ? (w.k <= 0 || w.k >= n) && (of_k > 0 || !(p < 1.0f)) : !(p < 1.0f)) continue;
        const u64 by = cut_by_parts(tokens, sc, any, part_of, pass == 0 && w.k > 0 ? w.k : kNone, pass == 0 ? kNone : target_of(p, of_k),
                                    pass == 0 ? of_k : none);
        last = by < last ? by : last;
    }
    auto kept = [&](float l, int32_t token) { return rank_of(l, token) <= last && (!(w.min_w > 0.0) || sc.weight(l) >= w.min_w); };
    int shift = 0;
    while ((args->V - 1) >> shift >= kBins) ++shift;
    static_assert(kMaxTokens <= kBins * kThreads && kThreads <= kList, "tokens of a part");
    __syncthreads();
    s.mass[tid] = 0;
    s.list.sum[tid] = 0;
    __syncthreads();
    tokens.each(any, [&](float l, int32_t token) {
        if (kept(l, token)) atomicAdd(&s.mass[token >> shift], sc.weigh(l));
    });
    __syncthreads();
    const u64 here = s.mass[tid];
    u64 sum;
    const u64 up = scan(here, s.room, sum), pass = drawn_at(w.set.u, sum);
    if (up > pass && up - here <= pass) {
        s.found32[0] = tid;
        s.found[0] = up - here;
    }
    __syncthreads();
    const int part = s.found32[0];
    tokens.each(any, [&](float l, int32_t token) {
        if (token >> shift != part || !kept(l, token)) return;
        s.list.sum[token & ((1 << shift) - 1)] = sc.weigh(l);
        s.list.rank[token & ((1 << shift) - 1)] = rank_of(l, token);
    });
    __syncthreads();
    const u64 mine = s.list.sum[tid];
    u64 all;
    const u64 at = s.found[0] + scan(mine, s.room, all);
    if (at > pass && at - mine <= pass) Drawn{s.list.rank[tid], sum}.write(*args, r, sc);
}

// Many tokens are kept, and the tiles have their weights by coarse bins: the last kept token, in the bin of the cut, then the tile in which the
// sum passes u S, which is looked at token by token.
template <typename E>
__device__ __noinline__ void draw_long(const Args *args, int64_t r)
{
    Shared &s = lds();
    const Args a = *args;
    const Known w = known();
    const Row<E> row(a, r);
    const Scale &sc = w.sc;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float p = w.set.p;
    const u64 *tile_mass = w.k > 0 ? a.tile_mass : a.tile_bins;
    __syncthreads();
    u64 all;
    const u64 m_up = scan(tid < kCoarse ? s.coarse_mass[tid] : 0, s.room, all);
    const u64 c_up = scan(tid < kCoarse ? s.coarse_count[tid] : 0, s.room, all);
    if (tid < kCoarse) {                   // up to and with each
        s.coarse_mass[tid] = m_up;
        s.coarse_count[tid] = static_cast<uint32_t>(c_up);
    }
    __syncthreads();
    u64 last = kNone, in_bin, target = w.target;
    int bin = w.end, held = -1;
    uint32_t n_held = 0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {                     // top-k, then top-p of the weight of its tokens
        if (pass == 0 ? w.k <= 0 : !(p < 1.0f)) continue;
        const u64 c0 = bin > 0 ? s.coarse_count[bin - 1] : 0, m0 = bin > 0 ? s.coarse_mass[bin - 1] : 0;
        const float from = bin < kCoarse - 1 ? sc.least_near(w.base + bin) : -FLT_MAX, to = bin > 0 ? sc.least_near(w.base + bin - 1) : INFINITY;
        auto in = [&](float l) { return l >= from && l < to; };
        if (tid == 0) s.n_held = 0;
        __syncthreads();
        InRow<E>{row}.hold(in, s.n_held);
        __syncthreads();
        held = bin;
        n_held = s.n_held;
        auto part = [&](float l) { return sc.fine(l, w.base + bin); };
        const u64 count = pass == 0 ? w.k - c0 : kNone, mass = pass == 0 ? kNone : target - m0;
        const u64 by = n_held <= kHold ? cut_by_parts(Held{static_cast<int>(n_held)}, sc, in, part, count, mass, in_bin)
                                      : cut_by_parts(InRow<E>{row}, sc, in, part, count, mass, in_bin);
        last = by < last ? by : last;
        if (pass == 0 && p < 1.0f) {
            target = target_of(p, m0 + in_bin);
            if (tid == 0) s.found32[0] = bin;                  // where rounding leaves none
            __syncthreads();
            if (tid < kCoarse && m_up >= target && (tid > 0 ? s.coarse_mass[tid - 1] : 0) < target) s.found32[0] = tid;
            __syncthreads();
            bin = s.found32[0];
            __syncthreads();
        }
    }
    if (w.min_w > 0.0) {
        const u64 by = last_by_weight(sc, w.min_w);
        last = by < last ? by : last;
    }
    // ---- kept weight of the tiles: their bins above the one of the last kept token, and of that one token by token
    const float lo_kept = logit_of(last);
    const int cut_at = sc.coarse(lo_kept) - w.base;
    bin = cut_at < kCoarse - 1 ? cut_at : kCoarse - 1;
    const float above = bin > 0 ? sc.least_near(w.base + bin - 1) : INFINITY;
    static_assert(kCoarse == 4 * 64, "bins of a lane");
#pragma unroll 1
    for (int32_t i = wave; i < a.tiles; i += kWaves) {         // a wave: a tile
        const float tile_top = a.tile_max[r * a.tiles + i];
        const int behind = bin - (sc.coarse(tile_top) - w.base) - lane * 4;
        const u64 *m = tile_mass + (r * a.tiles + i) * kCoarse + lane * 4;
        const u64 m0 = m[0], m1 = m[1], m2 = m[2], m3 = m[3];
        const u64 sum = wave_sum((behind > 0 ? m0 : 0) + (behind > 1 ? m1 : 0) + (behind > 2 ? m2 : 0) + (behind > 3 ? m3 : 0));
        if (lane == 0) s.piece[i] = sum > 0 ? rescaled(sum, tile_top, sc) : 0;
    }
    __syncthreads();
    auto rest = [&](float l) { return l >= lo_kept && l < above; };
    auto add = [&](float l, int32_t token) {
        if (rank_of(l, token) <= last) atomicAdd(&s.piece[(token + row.skip) / (Row<E>::kPer * kTileThreads * kTileBlocks)], sc.weigh(l));
    };
    if (held == bin && n_held <= kHold) Held{static_cast<int>(n_held)}.each(rest, add);
    else InRow<E>{row}.each(rest, add);
    __syncthreads();
    Drawn d;
    u64 pass;
    const u64 sum = find_piece(a.tiles, w.set.u, pass);
    // ---- the tile's tokens, a block to a thread, against the tile's largest logit, which is kept if any is
    static_assert(kTileThreads * kTileBlocks == kThreads, "blocks of a tile");
    const int32_t tile = s.found32[0], b = tile * kThreads + tid;
    float l[Row<E>::kPer];
    row.read(row.load(b), b, l);
    const Scale own(w.set.t, a.tile_max[r * a.tiles + tile]);
    u64 weight[Row<E>::kPer], here = 0;
#pragma unroll
    for (int e = 0; e < Row<E>::kPer; ++e) {
        weight[e] = b < row.n_blocks && there(l[e]) && rank_of(l[e], row.token(b, e)) <= last ? own.weigh(l[e]) : 0;
        here += weight[e];
    }
    const u64 ahead = s.found[0], at = scan(here, s.room, all) - here;
    pass = static_cast<u64>(static_cast<double>(pass - ahead) * (static_cast<double>(all) / static_cast<double>(s.piece[tile])));
    if (pass >= all) pass = all - 1;
    d = {pick_token(row, b, l, weight, at, pass), sum};
    d.write(a, r, sc);
}

// The others (+inf among the logits, more tokens than a list holds by top-k or min-p alone), without the tiles' help: the last kept token
// by parts of the whole row, then the kept weights along the vocabulary.
template <typename E>
__device__ __noinline__ void draw_whole(const Args *args, int64_t r)
{
    Shared &s = lds();
    const Args a = *args;
    const Known w = known();
    Row<E> row(a, r);
    row.only_inf = w.top == INFINITY;
    const Scale &sc = w.sc;
    const int tid = threadIdx.x, lane = tid & 63;
    u64 last = kNone, of_k = 0, none;
    auto all_tokens = [](float l) { return there(l); };
    auto part = [&](float l) { return sc.bin(l); };
    if (w.min_w > 0.0) last = last_by_weight(sc, w.min_w);
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {                     // top-k (or all tokens, for their weight), then top-p
        if (pass == 0 ? w.k <= 0 && !(w.set.p < 1.0f) : !(w.set.p < 1.0f)) continue;
        const u64 by = cut_by_parts(InRow<E>{row}, sc, all_tokens, part, pass == 0 && w.k > 0 ? w.k : kNone, pass == 0 ? kNone : target_of(w.set.p, of_k),
                                    pass == 0 ? of_k : none);
        last = by < last ? by : last;
    }
    auto kept = [&](float l, int32_t token) -> u64 { return there(l) && rank_of(l, token) <= last ? sc.weigh(l) : 0; };
    const int32_t pieces = (row.n_blocks + 63) / 64;
    __syncthreads();
#pragma unroll 1
    for (int32_t b0 = tid; b0 < pieces * 64; b0 += kThreads) {
        float l[Row<E>::kPer];
        row.read(row.load(b0), b0, l);
        u64 weight = 0;
#pragma unroll
        for (int e = 0; e < Row<E>::kPer; ++e) weight += kept(l[e], row.token(b0, e));
        weight = wave_sum(weight);
        if (lane == 0) s.piece[b0 >> 6] = weight;
    }
    __syncthreads();
    Drawn d;
    u64 pass;
    const u64 sum = find_piece(pieces, w.set.u, pass);
    if (tid >= 64) return;
    const int32_t b = s.found32[0] * 64 + lane;
    float l[Row<E>::kPer];
    row.read(row.load(b), b, l);
    u64 weight[Row<E>::kPer], here = 0;
#pragma unroll
    for (int e = 0; e < Row<E>::kPer; ++e) here += weight[e] = kept(l[e], row.token(b, e));
    d = {pick_token(row, b, l, weight, s.found[0] + wave_scan(here) - here, pass), sum};
    d.write(a, r, sc);
}

// ---- what the tiles of a row find out
template <typename E>
__global__ __launch_bounds__(kTileThreads) void tile_kernel(Args a)
{
    __shared__ u64 mass[kCoarse];
    __shared__ uint32_t count[kCoarse];
    __shared__ float tops[kTileThreads / 64];
    constexpr int kPer = Row<E>::kPer;
    static_assert(kTileBlocks == 4, "blocks of a lane, by name");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t r = blockIdx.x / a.tiles;
    const int32_t tile = blockIdx.x % a.tiles;
    const Row<E> row(a, r);
    const int32_t piece0 = tile * kTilePieces + wave * kTileBlocks;
    auto block = [&](int j) {
        const int32_t b = (piece0 + j) * 64 + lane;
        return row.load(b);
    };
    v4u b0 = block(0), b1 = block(1), b2 = block(2), b3 = block(3);
    const Settings set(a, r);
    const Ask ask = set.ask();
    mass[tid] = 0;
    count[tid] = 0;
    if (piece0 == 0 || (piece0 + kTileBlocks) * 64 >= row.n_blocks) {          // the row's first and last blocks
#pragma unroll 1
        for (int j = 0; j < kTileBlocks; ++j) {
            const v4u now = row.blank(b0, (piece0 + j) * 64 + lane);
            b0 = b1;
            b1 = b2;
            b2 = b3;
            b3 = now;
        }
    }
    auto largest = [&](const v4u &raw) {
        float l[kPer], top = -INFINITY;
        row.read(raw, l);
#pragma unroll
        for (int e = 0; e < kPer; ++e) top = fmaxf(top, l[e]);
        return top;
    };
    const float tops4 = four_max(largest(b0), largest(b1), largest(b2), largest(b3));
    if ((lane & 15) == 0) a.piece_max[r * a.pieces + piece0 + (lane >> 4)] = tops4;
    float tile_top = -INFINITY;
#pragma unroll
    for (int j = 0; j < kTileBlocks; ++j) tile_top = fmaxf(tile_top, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(tops4), j * 16)));
    if (ask == Ask::kNothing) return;
    if (ask == Ask::kSums) {               // of the wave's four pieces together
        const Scale sc(set.t, tile_top);
        double w = 0.0;
#pragma unroll 1
        for (int j = 0; j < kTileBlocks; j += 2) {
            float l[kPer], k[kPer];
            row.read(b0, l);
            row.read(b1, k);
#pragma unroll
            for (int e = 0; e < kPer; ++e) w += sc.weight(l[e]) + sc.weight(k[e]);
            b0 = b2;
            b1 = b3;
        }
        const u64 all = wave_sum(whole(w));
        if (lane == 0) {
            a.four_sum[(r * a.pieces + piece0) / kTileBlocks] = all;
            a.four_max[(r * a.pieces + piece0) / kTileBlocks] = tile_top;
        }
        return;
    }
    if (lane == 0) tops[wave] = tile_top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTileThreads / 64; ++w) tile_top = fmaxf(tile_top, tops[w]);
    const Scale sc(set.t, tile_top);
    const int base = sc.coarse(tile_top);
#pragma unroll 1
    for (int j = 0; j < kTileBlocks; ++j) {
        float l[kPer];
        row.read(b0, l);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (!there(l[e])) continue;
            const int at = sc.coarse(l[e]) - base, bin = at < kCoarse ? at : kCoarse - 1;
            if (ask != Ask::kMass) atomicAdd(&count[bin], 1u);
            if (ask != Ask::kCount) atomicAdd(&mass[bin], sc.weigh(l[e]));
        }
        b0 = b1;
        b1 = b2;
        b2 = b3;
    }
    __syncthreads();
    const int64_t at = (r * a.tiles + tile) * kCoarse + tid;
    a.tile_bins[at] = ask == Ask::kMass ? mass[tid] : count[tid];
    if (ask == Ask::kBoth) a.tile_mass[at] = mass[tid];
    if (tid == 0) a.tile_max[r * a.tiles + tile] = tile_top;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void pick_kernel(Args a)
{
    Shared &s = lds();
    constexpr int kPer = Row<E>::kPer;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t r = blockIdx.x;
    const Row<E> row(a, r);
    const float *piece_max = a.piece_max + r * a.pieces;
    // ---- what the tiles found out, on its way at once: to another L2 a trip takes more than a microsecond
    constexpr int kEarly = 4;
    const int32_t n_bins = a.tiles * kCoarse;
    const float *tile_max = a.tile_max + r * a.tiles;
    const u64 *tile_bins = a.tile_bins + r * n_bins;
    u64 bins[kEarly];
    float tile_top[kEarly];
#pragma unroll
    for (int j = 0; j < kEarly; ++j) {
        const int32_t i = tid + j * kThreads < n_bins ? tid + j * kThreads : 0;
        bins[j] = tile_bins[i];
        tile_top[j] = tile_max[i / kCoarse];
    }
    // ---- the largest logit; every wave by itself, without a barrier
    float top = -INFINITY;
#pragma unroll 4
    for (int32_t i = lane; i < a.pieces; i += 64) top = fmaxf(top, piece_max[i]);
    const Settings set(a, r);
    top = wave_max(top);
    if (top == -INFINITY) {
        if (tid == 0) put_result(a, r, -1, -INFINITY);
        return;
    }
    if (set.first()) {
        if (wave != 0) return;
        int32_t i = lane;                  // the first piece with the largest logit, the first token in it
        uint64_t here;
        while ((here = __ballot(i < a.pieces && piece_max[i < a.pieces ? i : 0] == top)) == 0) i += 64;
        const int32_t b = (i - lane + __builtin_ctzll(here)) * 64 + lane;
        float l[kPer];
        row.read(row.load(b), b, l);
        int e = kPer;
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i)
            if (l[i] == top) e = i;
        if (lane == __builtin_ctzll(__ballot(e < kPer))) put_result(a, r, row.token(b, e), 0.0);
        return;
    }
    const Ask ask = set.ask();
    const float p = set.p;
    Known w = {set, Scale(set.t, top == INFINITY ? 0.0f : top), top, set.min_p > 0.0f ? static_cast<double>(set.min_p) : 0.0, set.k, 0,
               kCoarse - 1, 0, 0, 0.0f};
    const Scale &sc = w.sc;
    const bool by_weight = w.min_w > 0.0 && !(p < 1.0f);       // min-p says by itself which tokens can be kept
    const Args *args = reinterpret_cast<const Args *>((const void *)__builtin_amdgcn_kernarg_segment_ptr());   // a, where it is
    if (ask == Ask::kSums && top < INFINITY) {
        // ---- the weights of four pieces each, then of the four pieces' tokens, against their own largest logit as the tile summed them: a
        // wave to a piece
        const int32_t fours = a.pieces / kTileBlocks;
        const float *four_max = a.four_max + r * fours;
        for (int32_t i = tid; i < fours; i += kThreads)
            s.piece[i] = four_max[i] > -INFINITY ? rescaled(a.four_sum[r * fours + i], four_max[i], sc) : 0;
        __syncthreads();
        u64 pass;
        const u64 sum = find_piece(fours, set.u, pass);
        const int32_t four = s.found32[0], b = (four * kTileBlocks + wave) * 64 + lane;
        u64 weight[kPer], here = 0, up = 0;
        float l[kPer];
        if (wave < kTileBlocks) {
            const Scale own(set.t, four_max[four]);
            row.read(row.load(b), b, l);
#pragma unroll
            for (int e = 0; e < kPer; ++e) here += weight[e] = b < row.n_blocks ? own.weigh(l[e]) : 0;
            up = wave_scan(here);
            if (lane == 63) s.room[wave] = up;
        }
        __syncthreads();
        if (wave >= kTileBlocks) return;
        u64 ahead = 0, all = 0;
#pragma unroll
        for (int j = 0; j < kTileBlocks; ++j) {
            if (j == wave) ahead = all;
            all += s.room[j];
        }
        pass = static_cast<u64>(static_cast<double>(pass - s.found[0]) * (static_cast<double>(all) / static_cast<double>(s.piece[four])));
        if (pass >= all) pass = all - 1;
        Drawn{pick_token(row, b, l, weight, ahead + up - here, pass), sum}.write(a, r, sc);
    } else if (top < INFINITY && (ask != Ask::kNothing || by_weight)) {
        // ---- tokens and weight by the row's coarse bins; the bin in which the ranking is cut
        const bool counted = ask == Ask::kCount || ask == Ask::kBoth, weighed = ask == Ask::kMass || ask == Ask::kBoth;
        u64 all_mass = 0;
        uint32_t up_to_end = 0;            // tokens up to that bin
        w.base = sc.coarse(top);
        auto add_bins = [&](int32_t i, float tile_top, u64 n) {
            if (i >= n_bins || n == 0) return;
            const int to = i % kCoarse + sc.coarse(tile_top) - w.base, bin = to < kCoarse ? to : kCoarse - 1;
            if (counted) atomicAdd(&s.coarse_count[bin], static_cast<uint32_t>(n));
            else atomicAdd(&s.coarse_mass[bin], rescaled(n, tile_top, sc));
            if (ask == Ask::kBoth) atomicAdd(&s.coarse_mass[bin], rescaled(a.tile_mass[r * n_bins + i], tile_top, sc));
        };
        if (tid == 0) s.n = s.n_pieces = s.at_least = 0;
        if (tid < kCoarse) {
            s.coarse_mass[tid] = 0;
            s.coarse_count[tid] = 0;
        }
        __syncthreads();
        if (counted || weighed) {
#pragma unroll
            for (int j = 0; j < kEarly; ++j) add_bins(tid + j * kThreads, tile_top[j], bins[j]);
#pragma unroll 1
            for (int32_t i = tid + kEarly * kThreads; i < n_bins; i += kThreads) add_bins(i, tile_max[i / kCoarse], tile_bins[i]);
            __syncthreads();
            // every wave finds the bin by itself, four bins a lane
            if (counted) {
                uint32_t ahead;
                w.end = bin_in(s.coarse_count, [&](uint32_t all) {
                    if (static_cast<uint32_t>(w.k) > all) w.k = static_cast<int32_t>(all);
                    return static_cast<uint32_t>(w.k);
                }, ahead);
                up_to_end = ahead + s.coarse_count[w.end];
            } else {
                u64 ahead;
                w.end = bin_in(s.coarse_mass, [&](u64 all) { return w.target = target_of(p, all_mass = all); }, ahead);
            }
        }
        // ---- the tokens up to there, where they are few: those with at least this logit
        float least = w.end < kCoarse - 1 ? sc.least_near(w.base + w.end) : -FLT_MAX;
        if (by_weight) {                                       // what is rounded here lets a few more in
            const double x = fmax(-log2(static_cast<double>(set.min_p)), 0.0) * (1.0 + 0x1p-20) + 0x1p-20;
            least = fmaxf(least, static_cast<float>(static_cast<double>(top) - x / sc.x_of - fabs(static_cast<double>(top)) * 0x1p-22));
        }
        auto can = [&](float l) { return l >= least; };
        w.all_mass = ask == Ask::kMass ? all_mass : 0;
        w.least = least;
        if (tid == 0) known() = w;                             // for a way that may follow, so that registers need not keep it
        uint32_t n = kList + 1;
        if (!counted || up_to_end <= kList || by_weight) {
            // the pieces that can have such a token, then a wave every 16th of them, four at a time
            uint16_t *todo = reinterpret_cast<uint16_t *>(s.mass);
            static_assert(kMaxPieces <= 0xffff && kMaxPieces * 2 <= sizeof(s.mass) + sizeof(s.count), "pieces by their number");
            // by weight alone: a token of bin b weighs 2^-((b - 1) / 4) at most, so there are at least this many (of the further bins the
            // weights' rounding to 2^-43 would be most)
            if (!counted && weighed && tid <= w.end && tid <= kCoarse / 2) {
                const double n_here = static_cast<double>(s.coarse_mass[tid]) * 0x1p-43 * static_cast<double>(exp2f(0.25f * static_cast<float>(tid - 1)));
                atomicAdd(&s.at_least, static_cast<uint32_t>(n_here < 0x1p21 ? n_here : 0x1p21));
            }
            for (int32_t i = tid; i < a.pieces; i += kThreads)
                if (can(piece_max[i])) todo[atomicAdd(&s.n_pieces, 1u)] = static_cast<uint16_t>(i);
            __syncthreads();
            const int32_t n_todo = s.at_least <= kList + kCoarse ? s.n_pieces : 0;
#pragma unroll 1
            for (int32_t i0 = wave; i0 < n_todo; i0 += kWaves * 4) {
                v4u raw[4];
                int32_t b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int32_t i = i0 + j * kWaves;
                    b[j] = i < n_todo ? todo[i] * 64 + lane : row.n_blocks;
                    raw[j] = row.load(b[j]);
                }
                each_of(row, raw, b, can, put_held);
            }
            __syncthreads();
            n = s.at_least <= kList + kCoarse ? s.n : kList + 1;
            __syncthreads();
        }
        if (n <= kShort) {
            const Known &w = known();
            draw_short(n, w.k, w.set.p, w.min_w, w.set.u, w.all_mass, w.all_mass > 0, w.sc).write(*args, r, w.sc);
            return;
        }
        __syncthreads();
        if (n <= kList) draw_list(args, r, n);
        else if (weighed) draw_long<E>(args, r);
        else draw_whole<E>(args, r);
    } else {
        if (tid == 0) known() = w;
        __syncthreads();
        draw_whole<E>(args, r);
    }
}

// Tiles of a row whose logits take `bytes` each, wherever in a block it begins.
int32_t tiles_of(int32_t V, int32_t bytes)
{
    const int32_t per = 16 / bytes, blocks = (V + 2 * per - 2) / per;
    return static_cast<int32_t>(ceil_div(blocks, kTileThreads * kTileBlocks));
}

// Where the parts of the workspace begin; [6]: its size.
struct Layout {
    int64_t at[7];
    Layout(int32_t rows, int32_t tiles)
    {
        const int64_t n = static_cast<int64_t>(rows) * tiles, waves = kTileThreads / 64;
        const int64_t bytes[6] = {n * kTilePieces * 4, n * waves * 8, n * waves * 4, n * kCoarse * 8, n * kCoarse * 8, n * 4};
        at[0] = 0;
        for (int i = 0; i < 6; ++i) at[i + 1] = at[i] + ceil_div(bytes[i], 256) * 256;
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
    return Layout(rows, tiles_of(V, 4)).at[6];
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
                    reinterpret_cast<float *>(ws + lay.at[0]), reinterpret_cast<u64 *>(ws + lay.at[1]), reinterpret_cast<float *>(ws + lay.at[2]),
                    reinterpret_cast<u64 *>(ws + lay.at[3]), reinterpret_cast<u64 *>(ws + lay.at[4]), reinterpret_cast<float *>(ws + lay.at[5])};
    return type == MQUANT_F16 ? launch<_Float16>(a, rows, static_cast<hipStream_t>(stream)) : launch<float>(a, rows, static_cast<hipStream_t>(stream));
}
