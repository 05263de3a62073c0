// A step's tables from the sequences' lengths: row starts, pages taken from and given
// back to a ring of free ones, and the slot and place of each new token.
//
// Everything is a sum over the sequences before one: of new tokens, of pages taken, of
// pages given back.  Each workgroup works all three out for itself (seqs pairs of
// numbers, from the caches) and then does its share of the tokens, of the taken pages
// and of the given ones, each found by a search in a chunk's sums in shared memory.  A
// new token's page is read from where the page is taken from, not from the table, so
// that no workgroup waits for another; given pages go behind all free ones, where
// nothing is taken from.  Bound by latency: two dependent rounds of loads and some
// barriers (64 sequences with a token each 3.6 us; 1024 with 1 to 96 tokens, 0.46 MB,
// 8.8 us; with 64-bit sums by shuffles in workgroups of 1024 threads 13.2 and 17.6).
#include <algorithm>

#include "tr_step.h"
#include "tr_wave.h"

namespace tr {
namespace {

constexpr int32_t kImpossible = INT32_MAX;

// Sums that stay at 2^32 - 1 once they are past it: more than any pool or batch of rows.
struct Sums {
    uint32_t fresh, take, give;   // new tokens, pages taken and given back
};

__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y)
{
    return {__builtin_elementwise_add_sat(x.fresh, y.fresh), __builtin_elementwise_add_sat(x.take, y.take),
            __builtin_elementwise_add_sat(x.give, y.give)};
}

// One sequence: its lengths, its pages before and after, and whether they fit.
struct Sequence {
    int32_t length, held, need;
    Sums sums;
    bool fits;
};

__device__ __forceinline__ int32_t pages_for(const PagesArgs& a, int32_t n)
{
    return n ? (int32_t)divide((uint32_t)n - 1, a.by_page) + 1 : 0;
}

__device__ __forceinline__ Sequence sequence_of(const PagesArgs& a, int b)
{
    Sequence s{};
    s.fits = true;
    if (b >= a.seqs) return s;
    const int32_t kv = max(a.kv_len[b], 0), change = a.change[b];
    const int64_t length = max((int64_t)kv + change, (int64_t)0);
    s.length = (int32_t)min(length, (int64_t)INT32_MAX);
    s.held = pages_for(a, kv);
    s.need = pages_for(a, s.length);
    s.sums = {(uint32_t)max(change, 0), (uint32_t)max(s.need - s.held, 0), (uint32_t)max(s.held - s.need, 0)};
    s.fits = length <= INT32_MAX && max(s.held, s.need) <= a.table_width;
    return s;
}

// Inclusive sums over the workgroup's T threads, and the whole sum in `all`.
template <int T>
__device__ __forceinline__ Sums scan(Sums x, Sums& all, uint4 (&shared)[T / 64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto add = [&](int m) { x = x + Sums{dpp_u32(x.fresh, m), dpp_u32(x.take, m), dpp_u32(x.give, m)}; };
    add(1);
    add(2);
    add(4);
    add(8);
    add(15);
    add(31);
    if (lane == 63) shared[wave] = uint4{x.fresh, x.take, x.give, 0};
    __syncthreads();
    Sums before{};
    all = {};
#pragma unroll
    for (int w = 0; w < T / 64; ++w) {
        const uint4 y = shared[w];
        if (w < wave) before = before + Sums{y.x, y.y, y.z};
        all = all + Sums{y.x, y.y, y.z};
    }
    __syncthreads();
    return x + before;
}

// First of a chunk's T ends that is above x, which is below the last one's.
template <int T>
__device__ __forceinline__ int find(const uint32_t* ends, uint32_t x)
{
    int lo = 0;
#pragma unroll
    for (int step = T / 2; step; step >>= 1)
        if (ends[lo + step - 1] <= x) lo += step;
    return lo;
}

// A workgroup's share [first, last) of n < 2^31 things, cut down to [c0, c1).
struct Range {
    uint32_t first, last;
};

__device__ __forceinline__ Range share(uint32_t n, uint32_t c0, uint32_t c1)
{
    const uint32_t each = (n + gridDim.x - 1) / gridDim.x;
    return {max(min(blockIdx.x * each, n), c0), min(min((blockIdx.x + 1) * each, n), c1)};
}

// `tables`: rows, pages, slots and places; `lengths`: kv_out and state_out, by the
// first workgroup (which may be kv_len and state, that other workgroups still read).
template <int T>
__global__ __launch_bounds__(T) void pages_kernel(PagesArgs a, bool tables, bool lengths)
{
    __shared__ uint4 shared[T / 64];
    __shared__ uint32_t fresh_end[T], take_end[T], give_end[T];
    __shared__ int32_t length[T], held[T], need[T];
    const int tid = threadIdx.x;
    const int32_t state0 = a.state[0], state1 = a.state[1];
    const uint32_t pages = (uint32_t)a.pages, first = (uint32_t)min(max(state0, 0), a.pages - 1), free = (uint32_t)min(max(state1, 0), a.pages);
    auto in_ring = [&](uint32_t i) { return i >= pages ? i - pages : i; };       // i < 2 pages

    // ---- the whole step -------------------------------------------------------------
    Sums all{};
    bool fits = true;
    Sequence s{};
    Sums mine{};
    for (int b0 = 0; b0 < a.seqs; b0 += T) {
        s = sequence_of(a, b0 + tid);
        fits = fits && s.fits;
        Sums sum;
        mine = scan<T>(s.sums, sum, shared);
        all = all + sum;
    }
    fits = __syncthreads_and(fits);
    int32_t lacking = 0;
    if (!fits || all.fresh > (uint32_t)a.rows || all.give > pages - free) lacking = kImpossible;
    else if (all.take > free) lacking = (int32_t)min(all.take - free, (uint32_t)kImpossible);
    const bool done = lacking == 0, one = a.seqs <= T;

    // ---- sequences, a chunk at a time -------------------------------------------------
    Sums before{};
    for (int b0 = 0; b0 < a.seqs; b0 += T) {
        const int b = b0 + tid, n = min(T, a.seqs - b0);
        Sums sum = all;
        if (!one) {
            s = sequence_of(a, b);
            mine = scan<T>(s.sums, sum, shared);
        }
        const Sums end = before + mine, past = before + sum;
        if (tid < n) {
            if (lengths && blockIdx.x == 0) a.kv_out[b] = done ? s.length : a.kv_len[b];
            if (tables && blockIdx.x == 0) a.q_start[b + 1] = done ? (int32_t)end.fresh : 0;
        }
        if (!done || !tables) {
            before = past;
            continue;
        }
        fresh_end[tid] = end.fresh;           // threads without a sequence: the last one's
        take_end[tid] = end.take;
        give_end[tid] = end.give;
        length[tid] = s.length;
        held[tid] = s.held;
        need[tid] = s.need;
        __syncthreads();
        const Range takes = share(all.take, before.take, past.take);
        for (uint32_t k = takes.first + tid; k < takes.last; k += T) {
            const int i = find<T>(take_end, k);
            a.table[(b0 + i) * a.table_stride + need[i] - (int32_t)(take_end[i] - k)] = a.ring[in_ring(first + k)];
        }
        const Range gives = share(all.give, before.give, past.give);
        for (uint32_t k = gives.first + tid; k < gives.last; k += T) {
            const int i = find<T>(give_end, k);
            a.ring[in_ring(in_ring(first + free) + k)] = a.table[(b0 + i) * a.table_stride + held[i] - (int32_t)(give_end[i] - k)];
        }
        const Range tokens = share((uint32_t)a.rows, before.fresh, past.fresh);
        for (uint32_t t = tokens.first + tid; t < tokens.last; t += T) {
            const int i = find<T>(fresh_end, t);
            const int32_t p = length[i] - (int32_t)(fresh_end[i] - t), slot = (int32_t)divide((uint32_t)p, a.by_page);
            if (a.pos) a.pos[t] = p;
            if (a.slots) {
                const int32_t taken = slot - held[i];
                const uint32_t from = take_end[i] - (uint32_t)(need[i] - held[i]);
                const int32_t page = taken < 0 ? a.table[(b0 + i) * a.table_stride + slot] : a.ring[in_ring(first + from + (uint32_t)taken)];
                a.slots[t] = (int64_t)page * a.page_size + (p - slot * a.page_size);
            }
        }
        before = past;
        __syncthreads();
    }

    // ---- what belongs to no sequence, and the whole step's numbers ----------------------
    if (tables) {
        const Range rest = share((uint32_t)a.rows, done ? all.fresh : 0, (uint32_t)a.rows);
        for (uint32_t t = rest.first + tid; t < rest.last; t += T) {
            if (a.pos) a.pos[t] = 0;
            if (a.slots) a.slots[t] = -1;
        }
        if (blockIdx.x == 0 && tid == 0) {
            a.q_start[0] = 0;
            *a.short_of = lacking;
        }
    }
    if (lengths && blockIdx.x == 0 && tid == 0) {
        a.state_out[0] = done ? (int32_t)in_ring(first + all.take) : state0;
        a.state_out[1] = done ? (int32_t)(free - all.take + all.give) : state1;
    }
}

}  // namespace

hipError_t launch_pages(const PagesArgs& args, hipStream_t s)
{
    PagesArgs a = args;
    a.by_page = divisor((uint32_t)a.page_size);
    const int64_t groups = std::max((int64_t)1, std::min((int64_t)256, (a.rows + 16 * (int64_t)a.seqs + 4095) / 4096));
    const bool apart = groups > 1 && (a.kv_out == a.kv_len || a.state_out == a.state);
    auto launch = [&](auto kernel, int threads, unsigned n, bool tables, bool lengths) {
        hipLaunchKernelGGL(kernel, dim3(n), dim3(threads), 0, s, a, tables, lengths);
        return hipGetLastError();
    };
    auto step = [&](unsigned n, bool tables, bool lengths) {
        return a.seqs <= 256 ? launch(pages_kernel<256>, 256, n, tables, lengths) : launch(pages_kernel<1024>, 1024, n, tables, lengths);
    };
    const hipError_t e = step((unsigned)groups, true, !apart);
    return e != hipSuccess || !apart ? e : step(1, false, true);
}

}  // namespace tr
