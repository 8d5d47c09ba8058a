// The bookkeeping of a serving step for gfx950: pages given back by ended sequences, rows and pages of the others, row_start, positions
// and slots, from the sequences' lengths in device memory.
//
// With r the rows a sequence may get and need its new pages, everything is a sum along the sequences: a sequence is served while both sums
// stay inside T and the free pages, which is a condition that never turns true again, so that sums over all of them place the
// served ones.  plan_kernel, one work-group, walks the sequences 1024 at a time with the sums carried on; pages and rows are dealt to the
// threads by their number and find their sequence by bisection of the sums.  Many rows are written by plan_rows_kernel instead.
#include "serving_common.h"

using namespace mquant;

namespace {

constexpr int kThreads = 1024;
constexpr int kRowsHere = 4096;            // rows up to which the one work-group writes them itself
constexpr int kRowsThread = 4;             // rows of a thread of plan_rows_kernel
constexpr int kStartsLds = 4096;           // starts of sequences that a work-group of plan_rows_kernel holds in LDS

struct Plan {
    const int32_t *length, *rows, *shared, *order;
    int32_t *table, *ring;
    const int32_t *state;
    int32_t *state_out, *length_out, *row_start, *pos;
    int64_t *slot;
    int32_t n_seq, table_pages, page_shift, n_pages, T;
};

__device__ __forceinline__ int64_t shfl_up64(int64_t x, int by)
{
    const int lo = __shfl_up(static_cast<int>(x), by, 64), hi = __shfl_up(static_cast<int>(x >> 32), by, 64);
    return (static_cast<int64_t>(hi) << 32) | static_cast<uint32_t>(lo);
}

// Sum of x over the threads up to this one; `all`: over all threads.  `room` holds a number per wave and may be used again behind the
// next barrier.
__device__ __forceinline__ int64_t scan(int64_t x, int64_t *room, int64_t &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = shfl_up64(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) room[wave] = x;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w == wave) x += all;
        all += room[w];
    }
    return x;
}

// The first of n rising numbers that is above x (n: none).
template <typename N>
__device__ __forceinline__ int32_t above(const N *v, int32_t n, int64_t x)
{
    int32_t lo = 0, hi = n;
    while (lo < hi) {
        const int32_t mid = (lo + hi) >> 1;
        if (static_cast<int64_t>(v[mid]) > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__device__ __forceinline__ int32_t slots_of(const Plan &a) { return a.table_pages << a.page_shift; }

__device__ __forceinline__ int32_t length_of(const Plan &a, int32_t s)
{
    const int32_t n = a.length[s], most = slots_of(a);
    return n < 0 ? 0 : n < most ? n : most;
}

__device__ __forceinline__ int32_t pages_of(const Plan &a, int32_t n) { return static_cast<int32_t>((static_cast<uint32_t>(n) + (1u << a.page_shift) - 1) >> a.page_shift); }

// Position and slot of row i, the (i - start)-th of the n new rows of sequence s (n_seq: of none).
__device__ __forceinline__ void write_row(const Plan &a, int32_t i, int32_t s, int32_t start, int32_t n)
{
    int32_t p = -1;
    int64_t at = -1;
    if (s < a.n_seq) {
        const int32_t o = a.order ? a.order[i] : i - start;
        if (o >= 0 && o < n) {
            p = a.length_out[s] - n + o;
            const int32_t page = a.table[static_cast<int64_t>(s) * a.table_pages + (p >> a.page_shift)];
            if (page >= 0 && page < a.n_pages) at = (static_cast<int64_t>(page) << a.page_shift) + (p & ((1 << a.page_shift) - 1));
        }
    }
    a.pos[i] = p;
    if (a.slot) a.slot[i] = at;
}

__global__ __launch_bounds__(kThreads) void plan_kernel(Plan a, int32_t write_rows)
{
    __shared__ int64_t room[kThreads / 64], sums[kThreads], served[2];
    __shared__ int32_t pages0[kThreads], starts[kThreads];
    const int tid = threadIdx.x;
    int32_t head = a.state[0] % a.n_pages, count = a.state[1];
    if (head < 0) head += a.n_pages;
    count = count < 0 ? 0 : count < a.n_pages ? count : a.n_pages;
    __syncthreads();                                           // state_out may be the same array

    // pages of ended sequences to the ring's end
    int64_t given = 0;
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kThreads) {
        const int32_t s = s0 + tid;
        int32_t n = 0;
        if (s < a.n_seq && a.rows[s] < 0) {
            const int32_t own = a.shared && a.shared[s] > 0 ? a.shared[s] : 0;
            n = pages_of(a, length_of(a, s)) - own;
            n = n > 0 ? n : 0;
        }
        int64_t all;
        sums[tid] = scan(n, room, all);
        if (all > 0) {
            __syncthreads();
            const int32_t tile = a.n_seq - s0 < kThreads ? a.n_seq - s0 : kThreads;
            for (int64_t i = tid; i < all; i += kThreads) {
                const int32_t j = above(sums, tile, i);
                const int64_t first = j > 0 ? sums[j - 1] : 0;
                const int32_t own = a.shared && a.shared[s0 + j] > 0 ? a.shared[s0 + j] : 0;
                const int32_t id = a.table[static_cast<int64_t>(s0 + j) * a.table_pages + own + (i - first)];
                // more pages than the ring holds can only be pages given back twice: they are not written over others
                if (count + given + i < a.n_pages) a.ring[(static_cast<int64_t>(head) + count + given + i) % a.n_pages] = id;
            }
        }
        given += all;
        __syncthreads();
    }
    const int64_t there = count + given < a.n_pages ? count + given : a.n_pages;

    // rows and pages of the others
    if (tid < 2) served[tid] = 0;
    int64_t rows_before = 0, need_before = 0;                  // sums over the sequences behind us, served or not
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kThreads) {
        const int32_t s = s0 + tid;
        int32_t r = 0, before = 0, need = 0;
        bool ended = false;
        if (s < a.n_seq) {
            r = a.rows[s];
            before = length_of(a, s);
            ended = r < 0;
            if (ended || static_cast<int64_t>(before) + r > slots_of(a)) r = 0;
            pages0[tid] = pages_of(a, before);
            need = pages_of(a, before + r) - pages0[tid];
        }
        int64_t all_rows, all_need;
        const int64_t my_rows = rows_before + scan(r, room, all_rows);
        const int64_t my_need = need_before + scan(need, room, all_need);
        const int64_t need_first = served[1];                  // where this tile's pages begin
        const bool ok = s < a.n_seq && my_rows <= a.T && my_need <= there;
        sums[tid] = my_need;
        const int n_ok = __syncthreads_count(ok);              // they are the tile's first ones
        if (tid == n_ok - 1) {
            served[0] = my_rows;
            served[1] = my_need;
        }
        __syncthreads();
        if (s < a.n_seq) {
            const int32_t start = static_cast<int32_t>(ok ? my_rows - r : served[0]);
            a.row_start[s] = start;
            starts[tid] = start;                               // of the last tile, which is the only one where they are used
            a.length_out[s] = ended ? 0 : ok ? before + r : before;
        }
        for (int64_t i = need_first + tid; i < served[1]; i += kThreads) {
            const int32_t j = above(sums, n_ok, i);
            const int64_t first = j > 0 ? sums[j - 1] : need_before;
            a.table[static_cast<int64_t>(s0 + j) * a.table_pages + pages0[j] + (i - first)] = a.ring[(head + i) % a.n_pages];
        }
        rows_before += all_rows;
        need_before += all_need;
        __syncthreads();
    }
    if (a.n_seq == 0) __syncthreads();
    const int32_t rows = static_cast<int32_t>(served[0]);
    if (tid == 0) {
        a.row_start[a.n_seq] = rows;
        a.state_out[0] = static_cast<int32_t>((head + served[1]) % a.n_pages);
        a.state_out[1] = static_cast<int32_t>(there - served[1]);
    }
    if (!write_rows) return;
    for (int32_t i = tid; i < a.T; i += kThreads) {
        int32_t s = a.n_seq, start = 0, end = 0;
        if (i < rows) {
            const int32_t *v = a.n_seq <= kThreads ? starts : a.row_start;
            s = above(v, a.n_seq, i) - 1;
            start = v[s];
            end = s + 1 < a.n_seq ? v[s + 1] : rows;
        }
        write_row(a, i, s, start, end - start);
    }
}

// Rows by the thread, sequences found by bisection of the starts (in LDS, where they fit).
__global__ __launch_bounds__(256) void plan_rows_kernel(Plan a)
{
    __shared__ int32_t lds[kStartsLds];
    const bool here = a.n_seq < kStartsLds;
    if (here)
        for (int32_t s = threadIdx.x; s <= a.n_seq; s += 256) lds[s] = a.row_start[s];
    __syncthreads();
    const int32_t *v = here ? lds : a.row_start;
    const int32_t rows = v[a.n_seq];
#pragma unroll
    for (int u = 0; u < kRowsThread; ++u) {
        const int64_t i = (static_cast<int64_t>(blockIdx.x) * kRowsThread + u) * 256 + threadIdx.x;
        if (i >= a.T) return;
        int32_t s = a.n_seq, start = 0, end = 0;
        if (i < rows) {
            s = above(v, a.n_seq, i) - 1;
            start = v[s];
            end = v[s + 1];
        }
        write_row(a, static_cast<int32_t>(i), s, start, end - start);
    }
}

}  // namespace

extern "C" int mquant_step_plan(const int32_t *length, const int32_t *rows, const int32_t *shared, const int32_t *order, int32_t n_seq,
                                int32_t *page_table, int32_t table_pages, int32_t page_size, int32_t *free_pages, int32_t n_pages,
                                const int32_t *free_state, int32_t *free_state_out, int32_t *length_out, int32_t *row_start,
                                int32_t *pos, int64_t *slot, int32_t T, mquant_stream_t stream_)
{
    if (n_seq < 0 || T < 0 || n_pages < 1) return MQUANT_ERR_BAD_SHAPE;
    if (page_size < 16 || page_size > 4096 || (page_size & (page_size - 1)) != 0 || n_seq > 1 << 20) return MQUANT_ERR_UNSUPPORTED;
    if (!free_pages || !free_state || !free_state_out || !row_start) return MQUANT_ERR_NULL;
    if (n_seq > 0) {
        if (table_pages < 1) return MQUANT_ERR_BAD_SHAPE;
        if (static_cast<int64_t>(table_pages) * page_size > 0x7fffffc0ll) return MQUANT_ERR_UNSUPPORTED;
        if (!length || !rows || !page_table || !length_out) return MQUANT_ERR_NULL;
    }
    if (T > 0 && !pos) return MQUANT_ERR_NULL;
    for (const void *p : {static_cast<const void *>(length), static_cast<const void *>(rows), static_cast<const void *>(shared),
                          static_cast<const void *>(order), static_cast<const void *>(page_table), static_cast<const void *>(free_pages),
                          static_cast<const void *>(free_state), static_cast<const void *>(free_state_out),
                          static_cast<const void *>(length_out), static_cast<const void *>(row_start), static_cast<const void *>(pos)})
        if (!aligned_to(p, 4)) return MQUANT_ERR_ALIGNMENT;
    if (!aligned_to(slot, 8)) return MQUANT_ERR_ALIGNMENT;
    const Plan a = {length, rows, shared, order, page_table, free_pages, free_state, free_state_out, length_out, row_start, pos, slot,
                    n_seq, table_pages, __builtin_ctz(static_cast<unsigned>(page_size)), n_pages, T};
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    const bool here = T <= kRowsHere;
    MQ_LAUNCH(plan_kernel, dim3(1), dim3(kThreads), 0, stream, a, here ? 1 : 0);
    if (const int st = launch_status(); st != MQUANT_OK || here) return st;
    MQ_LAUNCH(plan_rows_kernel, dim3(static_cast<unsigned>(ceil_div(T, 256 * kRowsThread))), dim3(256), 0, stream, a);
    return launch_status();
}
