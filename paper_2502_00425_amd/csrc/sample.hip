// The next token of every row of logits by temperature, top-k, top-p and min-p from a given random number, for gfx950.
//
// Token i has the weight w = 2^-x, x = (m - l) log2(e) / t >= 0; ranked by logit, the kept tokens are a front of the ranking, and
// which token is drawn is a question of sums of weights.  Weights are formed in double (off by 2^-44 of themselves) and summed as whole
// multiples of 2^-43: such sums do not depend on their order, so that atomics in LDS and any split of the work give the same
// token.  2^20 tokens of weight 1 are 2^63.
//
// Nothing is sorted but a short list.  A row goes through
//   the maximum;
//   bins of x, 1/16 wide, with the tokens and the weight in each: the bins in which the ranking is cut are found by sums over the bins,
//   and where the tokens up to there are few (kList), they are gathered, sorted and everything is decided among them;
//   otherwise the tokens of the bin in question are gathered and sorted (narrowed digit by digit of their rank where they are more than
//   the list holds), which gives the rank of the last kept token;
//   one walk over the row sums the kept weights by pieces of 64 lanes, and the piece in which the sum passes u S is looked at again.
// Rows without filters need the maximum and that walk only.
#include <cmath>

#include <hip/hip_fp16.h>

#include "mquant_internal.h"

using namespace mquant;

namespace {

typedef unsigned long long u64;
typedef unsigned __int128 u128;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxTokens = 1 << 20;
constexpr int kBins = 1024;
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
};

// What a row's threads share.
struct Shared {
    u64 mass[kBins];                       // up to and with a bin
    uint32_t count[kBins];
    union {
        struct {
            u64 rank[kList], sum[kList];
        } list;
        u64 piece[kMaxTokens / 4 / 64 + 1];        // of a walk: 64 blocks of 16 bytes
        struct {
            u64 mass[256];
            uint32_t count[256];
        } digit;
    };
    double power[64];                      // 2^(43 - j / 64)
    u64 room[kWaves];
    uint32_t room32[kWaves];
    u64 found[2];
    uint32_t found32[2];
    uint32_t n;
};

// ---- a row's logits: the 16-byte blocks that hold it, from the aligned one in which it begins
template <typename E>
struct Row {
    static constexpr int kPer = 16 / sizeof(E);
    const uint4 *block;
    int32_t skip, n_blocks, V;             // elements of the first block ahead of the row
    float inf_as;                          // where +inf occurs, it counts as 0 and everything else as nothing

    __device__ Row(const Args &a, int64_t row) : V(a.V)
    {
        const uintptr_t p = reinterpret_cast<uintptr_t>(static_cast<const E *>(a.logits) + row * a.ld);
        skip = static_cast<int32_t>((p & 15) / sizeof(E));
        block = reinterpret_cast<const uint4 *>(p & ~static_cast<uintptr_t>(15));
        n_blocks = (skip + V + kPer - 1) / kPer;
        inf_as = INFINITY;
    }

    // Token number of element e of block b; outside [0, V): not of the row.
    __device__ int32_t token(int32_t b, int e) const { return b * kPer + e - skip; }

    // The logits of a block, NaN where there is none: not of the row, -inf, NaN.
    __device__ void read(const uint4 &raw, int32_t b, float (&l)[kPer]) const
    {
        union {
            uint4 u;
            E e[kPer];
        } x;
        x.u = raw;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            float f = static_cast<float>(x.e[e]) + 0.0f;       // -0 ranks with 0
            if (inf_as == 0.0f) f = f == INFINITY ? 0.0f : NAN;
            const bool here = static_cast<uint32_t>(token(b, e)) < static_cast<uint32_t>(V) && f > -INFINITY;
            l[e] = here ? f : NAN;
        }
    }
};

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

// ---- weights
struct Scale {
    double x_of;                           // log2(e) / t
    float bin_of;                          // 16 times that, for the bins
    float m;

    __device__ double x(float l) const { return (static_cast<double>(m) - static_cast<double>(l)) * x_of; }
    // Falls with l, like the rank, whatever is rounded; the last bin has all that is left.
    __device__ int bin(float l) const { return static_cast<int>(fminf((m - l) * bin_of, static_cast<float>(kBins - 1))); }
};

// 2^(43 - x): x in steps of 1/64 by the table, the rest by e^-z, |z| <= ln 2 / 128, to z^4 (z^5 / 120 is 2^-44.5).
__device__ __forceinline__ double weight(double x, const double *power)
{
    if (!(x < kBits + 1.5)) return 0.0;
    const double y = x * 64.0, n = rint(y);
    const int i = static_cast<int>(n);
    const double z = (y - n) * (0.69314718055994530942 / 64.0);
    double p = __builtin_fma(z, 1.0 / 24.0, -1.0 / 6.0);
    p = __builtin_fma(p, z, 0.5);
    p = __builtin_fma(p, z, -1.0);
    p = __builtin_fma(p, z, 1.0);
    return ldexp(power[i & 63] * p, -(i >> 6));
}

// To the nearest whole number below 2^52.
__device__ __forceinline__ u64 whole(double w) { return static_cast<u64>(__double_as_longlong(w + 0x1p52)) & ((1ull << 52) - 1); }

__device__ __forceinline__ u64 weight_of(float l, const Scale &sc, const double *power) { return whole(weight(sc.x(l), power)); }

// ---- ranks: the larger the logit and the lower the token's number, the smaller
__device__ __forceinline__ u64 rank_of(float l, int32_t token)
{
    const uint32_t b = __float_as_uint(l);
    const uint32_t rising = b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
    return static_cast<u64>(~rising) << kIndexBits | static_cast<uint32_t>(token);
}

__device__ __forceinline__ float logit_of(u64 rank)
{
    const uint32_t rising = ~static_cast<uint32_t>(rank >> kIndexBits);
    return __uint_as_float(rising ^ (rising >> 31 ? 0x80000000u : 0xffffffffu));
}

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
    const u64 x = i < n ? weight_of(logit_of(s.list.rank[i]), sc, s.power) : 0;
    const u64 y = i + 1 < n ? weight_of(logit_of(s.list.rank[i + 1]), sc, s.power) : 0;
    u64 all;
    const u64 up = scan(x + y, s.room, all);
    s.list.sum[i] = up - y;
    s.list.sum[i + 1] = up;
    __syncthreads();
}

// The tokens that `take` names are put into the list (which has room); returns how many.
template <typename E, typename F>
__device__ int gather(Shared &s, const Row<E> &row, F take)
{
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    walk(row, [&](int32_t b, const float (&l)[Row<E>::kPer]) {
#pragma unroll
        for (int e = 0; e < Row<E>::kPer; ++e)
            if (l[e] == l[e] && take(l[e], row.token(b, e))) {
                const uint32_t at = atomicAdd(&s.n, 1u);
                if (at < kList) s.list.rank[at] = rank_of(l[e], row.token(b, e));
            }
    });
    __syncthreads();
    const int n = s.n < kList ? s.n : kList;
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

// The rank of the last token of bin `b` that a cut keeps: of the bin's tokens by rank the first `count` (at least 1, at most all), and only
// those with less than `mass` of the bin's weight before them (the bin's first one has).  kept_mass: their weight.
template <typename E>
__device__ u64 cut_bin(Shared &s, const Row<E> &row, const Scale &sc, int b, uint32_t in_bin, u64 count, u64 mass, u64 &kept_mass)
{
    u64 prefix = 0, passed = 0;            // digits of the rank that are known, weight of the tokens ahead of them
    int low = 32 + kIndexBits;             // bits that are not
    u64 n = in_bin;
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
                if (!(l[e] == l[e]) || sc.bin(l[e]) != b) continue;
                const u64 r = rank_of(l[e], row.token(at, e));
                if (r >> low >> 8 != prefix) continue;
                atomicAdd(&s.digit.mass[r >> low & 255], weight_of(l[e], sc, s.power));
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
    const int m = gather(s, row, [&](float l, int32_t token) { return sc.bin(l) == b && rank_of(l, token) >> low == prefix; });
    sort_list(s.list.rank, m);
    sum_list(s, m, sc);
    int k = cut_list(s, m, count, mass);
    if (k < 1) k = 1;
    kept_mass = passed + s.list.sum[k - 1];
    const u64 last = s.list.rank[k - 1];
    __syncthreads();
    return last;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void sample_kernel(Args a)
{
    __shared__ Shared s;
    constexpr int kPer = Row<E>::kPer;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r = blockIdx.x;
    Row<E> row(a, r);
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    int32_t k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f, u = a.u[r];
    if (tid < 64) s.power[tid] = exp2(kBits - tid / 64.0);

    // ---- the first token of the ranking
    u64 best = kNone;
    walk(row, [&](int32_t b, const float (&l)[kPer]) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (!(l[e] == l[e])) continue;
            const u64 x = rank_of(l[e], row.token(b, e));
            best = x < best ? x : best;
        }
    });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t lo = __shfl_xor(static_cast<uint32_t>(best), d, 64), hi = __shfl_xor(static_cast<uint32_t>(best >> 32), d, 64);
        const u64 x = static_cast<u64>(hi) << 32 | lo;
        best = x < best ? x : best;
    }
    if (lane == 0) s.room[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = s.room[w] < best ? s.room[w] : best;
    __syncthreads();
    auto result = [&](int32_t token, double logprob) {
        a.token[r] = token;
        if (a.logprob) a.logprob[r] = static_cast<float>(logprob);
    };
    constexpr int32_t kTokenMask = (1 << kIndexBits) - 1;
    if (best == kNone || !(t > 0.0f)) {
        if (tid == 0) result(best == kNone ? -1 : static_cast<int32_t>(best & kTokenMask), best == kNone ? -INFINITY : 0.0);
        return;
    }
    Scale sc;
    sc.m = logit_of(best);
    if (sc.m == INFINITY) {
        row.inf_as = 0.0f;
        sc.m = 0.0f;
        best = rank_of(0.0f, static_cast<int32_t>(best & kTokenMask));
    }
    sc.x_of = 1.4426950408889634074 / static_cast<double>(t);
    sc.bin_of = fminf(static_cast<float>(sc.x_of * 16.0), 1e30f);
    // log-probability of a token among kept ones of this weight
    auto chosen = [&](u64 rank, u64 all) {
        result(static_cast<int32_t>(rank & kTokenMask),
               -sc.x(logit_of(rank)) * 0.69314718055994530942 - log(static_cast<double>(all) * 0x1p-43));
    };
    const double min_w = min_p > 0.0f ? ldexp(static_cast<double>(min_p), kBits) : 0.0;

    u64 last = kNone;                      // rank of the last kept token (min-p aside)
    if (k > 0 || p < 1.0f || min_p > 0.0f) {
        // ---- tokens and weight by bins
        s.mass[tid] = 0;
        s.count[tid] = 0;
        __syncthreads();
        walk(row, [&](int32_t b, const float (&l)[kPer]) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (!(l[e] == l[e])) continue;
                const int at = sc.bin(l[e]);
                atomicAdd(&s.count[at], 1u);
                const u64 w = weight_of(l[e], sc, s.power);
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
        if (tid < 2) s.found32[tid] = kBins - 1;
        __syncthreads();
        // the bin of the k-th token; the one at which top-p ends at the latest; the last one with weights of min-p
        const uint32_t before = tid > 0 ? s.count[tid - 1] : 0;
        if (before < static_cast<uint32_t>(k) && count >= static_cast<uint32_t>(k)) s.found32[0] = tid;
        __syncthreads();
        const int bin_k = s.found32[0];
        bool rest;
        u64 most = share_of(p, s.mass[bin_k], rest);           // of at most the weight up to the k-th token's bin
        most += rest ? 1 : 0;
        if (p < 1.0f && (tid > 0 ? s.mass[tid - 1] : 0) < most && mass >= most) s.found32[1] = tid;
        __syncthreads();
        int end = s.found32[1] < static_cast<uint32_t>(bin_k) ? s.found32[1] : bin_k;
        if (p < 1.0f && most == 0) end = 0;
        if (min_p > 0.0f) {
            const double x = -log2(static_cast<double>(min_p)) * 16.0;
            const int by_min = x < 0.0 ? 1 : x < kBins - 2 ? static_cast<int>(x) + 1 : kBins - 1;          // one more, for what is rounded
            end = by_min < end ? by_min : end;
        }
        const bool all_k = static_cast<u64>(k) == all_count;
        if (p < 1.0f && !all_k) end = bin_k;                   // top-p is of the weight up to the k-th token
        if (s.count[end] <= kList) {
            // ---- everything among few tokens
            const int n = gather(s, row, [&](float l, int32_t) { return sc.bin(l) <= end; });
            sort_list(s.list.rank, n);
            sum_list(s, n, sc);
            u64 target = kNone;
            if (p < 1.0f) {
                target = share_of(p, all_k ? all_mass : s.list.sum[k - 1], rest);
                target += rest ? 1 : 0;
            }
            int kept = cut_list(s, n, k, target);              // fewer than k where the others are cut by top-p or min-p
            if (kept < 1) kept = 1;
            if (min_p > 0.0f) {
                if (tid == 0) s.n = 0;
                __syncthreads();
                uint32_t mine = 0;
                for (int i = tid; i < kept; i += kThreads)
                    if (weight(sc.x(logit_of(s.list.rank[i])), s.power) >= min_w) ++mine;
                if (mine > 0) atomicAdd(&s.n, mine);
                __syncthreads();
                kept = s.n > 1 ? s.n : 1;
                __syncthreads();
            }
            // ---- the kept ones in the order of the vocabulary
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
            // the place in the ranking has to become a logit again: the threads that hold r0 and r1 know it
            if (tid == 0) s.found32[0] = 0;
            __syncthreads();
            if (up - x - y <= pass && up - y > pass) s.found32[0] = static_cast<uint32_t>(s.list.rank[i] & 0xfff);
            if (up - y <= pass && up > pass) s.found32[0] = static_cast<uint32_t>(s.list.rank[i + 1] & 0xfff);
            __syncthreads();
            const int place = s.found32[0];
            if (place == i) chosen(r0, sum);
            if (place == i + 1) chosen(r1, sum);
            return;
        }
        // ---- many tokens are kept: the last one by top-k, then the last one by top-p
        u64 of_k = all_mass;
        if (!all_k) {
            const uint32_t c0 = bin_k > 0 ? s.count[bin_k - 1] : 0;
            const u64 m0 = bin_k > 0 ? s.mass[bin_k - 1] : 0;
            u64 in_bin;
            last = cut_bin(s, row, sc, bin_k, s.count[bin_k] - c0, k - c0, kNone, in_bin);
            of_k = m0 + in_bin;
        }
        if (p < 1.0f) {
            u64 target = share_of(p, of_k, rest);
            target += rest ? 1 : 0;
            if (tid == 0) s.found32[1] = 0;
            __syncthreads();
            if ((tid > 0 ? s.mass[tid - 1] : 0) < target && mass >= target) s.found32[1] = tid;
            __syncthreads();
            const int bin_p = s.found32[1];
            const uint32_t c0 = bin_p > 0 ? s.count[bin_p - 1] : 0;
            const u64 m0 = bin_p > 0 ? s.mass[bin_p - 1] : 0;
            u64 in_bin;
            const u64 by_p = cut_bin(s, row, sc, bin_p, s.count[bin_p] - c0, kNone, target > m0 ? target - m0 : 0, in_bin);
            last = by_p < last ? by_p : last;
        }
        __syncthreads();
    }

    // ---- the kept weights along the vocabulary, by pieces of 64 blocks
    auto kept = [&](float l, int32_t token) -> u64 {
        if (!(l == l)) return 0;
        const double w = weight(sc.x(l), s.power);
        if (w < min_w && rank_of(l, token) != best) return 0;
        return last == kNone || rank_of(l, token) <= last ? whole(w) : 0;
    };
    const int32_t pieces = (row.n_blocks + 63) / 64;
    for (int32_t b0 = tid; b0 < pieces * 64; b0 += kThreads) {
        u64 w = 0;
        if (b0 < row.n_blocks) {
            float l[kPer];
            row.read(row.block[b0], b0, l);
#pragma unroll
            for (int e = 0; e < kPer; ++e) w += kept(l[e], row.token(b0, e));
        }
        w = wave_scan(w);
        if (lane == 63) s.piece[b0 >> 6] = w;
    }
    __syncthreads();
    // every thread takes the pieces from..to, next to each other
    const int32_t per = (pieces + kThreads - 1) / kThreads, from = tid * per, to = from + per < pieces ? from + per : pieces;
    u64 mine = 0, sum;
    for (int32_t i = from; i < to; ++i) mine += s.piece[i];
    const u64 up = scan(mine, s.room, sum);
    bool rest;
    u64 pass = share_of(u, sum, rest);
    if (pass >= sum) pass = sum - 1;
    if (up > pass && up - mine <= pass) {
        u64 at = up - mine;
        int32_t i = from;
        while (at + s.piece[i] <= pass) at += s.piece[i++];
        s.found32[0] = i;
        s.found[0] = at;
    }
    __syncthreads();
    if (wave != 0) return;
    const int32_t b = s.found32[0] * 64 + lane;
    u64 w[kPer], here = 0;
    float l[kPer];
    if (b < row.n_blocks) row.read(row.block[b], b, l);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        w[e] = b < row.n_blocks ? kept(l[e], row.token(b, e)) : 0;
        here += w[e];
    }
    u64 at = s.found[0] + wave_scan(here) - here;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        if (at <= pass && at + w[e] > pass) chosen(rank_of(l[e], row.token(b, e)), sum);
        at += w[e];
    }
}

}  // namespace

extern "C" int64_t mquant_sample_workspace_bytes(int32_t rows, int32_t V)
{
    if (rows < 0 || V < 1) return MQUANT_ERR_BAD_SHAPE;
    if (V > kMaxTokens) return MQUANT_ERR_UNSUPPORTED;
    return 0;
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
    if (rows >= 1 << 22) return MQUANT_ERR_UNSUPPORTED;                          // 2^32 threads are more than a launch takes
    if (!logits || !u || !token) return MQUANT_ERR_NULL;
    if (!aligned_to(logits, type == MQUANT_F16 ? 2 : 4) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) ||
        !aligned_to(min_p, 4) || !aligned_to(u, 4) || !aligned_to(token, 4) || !aligned_to(logprob, 4))
        return MQUANT_ERR_ALIGNMENT;
    if (need > 0 && (!workspace || workspace_bytes < need)) return MQUANT_ERR_WORKSPACE;
    if (need > 0 && !aligned_to(workspace, 256)) return MQUANT_ERR_ALIGNMENT;
    const Args a = {logits, ld, temperature, top_k, top_p, min_p, u, token, logprob, V};
    if (type == MQUANT_F16) MQ_LAUNCH(sample_kernel<_Float16>, dim3(static_cast<unsigned>(rows)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    else MQ_LAUNCH(sample_kernel<float>, dim3(static_cast<unsigned>(rows)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    return launch_status();
}
