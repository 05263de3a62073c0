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
// barriers.
#include <algorithm>

#include "tr_step.h"

namespace tr {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int32_t kImpossible = INT32_MAX;

struct Sums {
    int64_t fresh, take, give;   // new tokens, pages taken and given back
};

__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) { return {x.fresh + y.fresh, x.take + y.take, x.give + y.give}; }

// One sequence: its lengths, its pages before and after, and whether they fit.
struct Sequence {
    int64_t length;
    int64_t held, need;
    Sums sums;
    bool fits;
};

__device__ __forceinline__ Sequence sequence_of(const PagesArgs& a, int b)
{
    Sequence s{};
    s.fits = true;
    if (b >= a.seqs) return s;
    const int64_t kv = max(a.kv_len[b], 0), change = a.change[b];
    s.length = max(kv + change, (int64_t)0);
    s.held = (kv + a.page_size - 1) / a.page_size;
    s.need = (s.length + a.page_size - 1) / a.page_size;
    s.sums = {max(change, (int64_t)0), max(s.need - s.held, (int64_t)0), max(s.held - s.need, (int64_t)0)};
    s.fits = s.length <= INT32_MAX && max(s.held, s.need) <= a.table_width;
    return s;
}

// Inclusive sums over the workgroup's threads, and the whole sum in `all`.
__device__ __forceinline__ Sums scan(Sums x, Sums& all, Sums (&shared)[kWaves])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const Sums y = {__shfl_up(x.fresh, m), __shfl_up(x.take, m), __shfl_up(x.give, m)};
        if (lane >= m) x = x + y;
    }
    if (lane == 63) shared[wave] = x;
    __syncthreads();
    Sums before{};
    all = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before = before + shared[w];
        all = all + shared[w];
    }
    __syncthreads();
    return x + before;
}

// First of the n ends that is above x.
__device__ __forceinline__ int find(const int32_t* ends, int n, int32_t x)
{
    int lo = 0;
    for (int step = kThreads; step; step >>= 1)
        if (lo + step <= n && ends[lo + step - 1] <= x) lo += step;
    return lo;
}

// A workgroup's share [first, last) of n things, cut down to [c0, c1).
struct Range {
    int32_t first, last;
};

__device__ __forceinline__ Range share(int64_t n, int64_t c0, int64_t c1)
{
    const int64_t each = (n + gridDim.x - 1) / gridDim.x;
    return {(int32_t)max(blockIdx.x * each, c0), (int32_t)min(min((blockIdx.x + 1) * each, n), c1)};
}

// `tables`: rows, pages, slots and places; `lengths`: kv_out and state_out, by the
// first workgroup (which may be kv_len and state, that other workgroups still read).
__global__ __launch_bounds__(kThreads) void pages_kernel(PagesArgs a, bool tables, bool lengths)
{
    __shared__ Sums shared[kWaves];
    __shared__ int32_t fresh_end[kThreads], take_end[kThreads], give_end[kThreads];
    __shared__ int32_t length[kThreads], held[kThreads], need[kThreads];
    const int tid = threadIdx.x;
    const uint32_t pages = (uint32_t)a.pages;
    const int64_t first = min(max(a.state[0], 0), a.pages - 1), free = min(max(a.state[1], 0), a.pages);

    // ---- the whole step -------------------------------------------------------------
    Sums all{};
    bool fits = true;
    Sequence s{};
    Sums mine{};
    for (int b0 = 0; b0 < a.seqs; b0 += kThreads) {
        s = sequence_of(a, b0 + tid);
        fits = fits && s.fits;
        Sums sum;
        mine = scan(s.sums, sum, shared);
        all = all + sum;
    }
    fits = __syncthreads_and(fits);
    int32_t lacking = 0;
    if (!fits || all.fresh > a.rows || free + all.give > a.pages) lacking = kImpossible;
    else if (all.take > free) lacking = (int32_t)(all.take - free);
    const bool done = lacking == 0, one = a.seqs <= kThreads;

    // ---- sequences, a chunk at a time -------------------------------------------------
    Sums before{};
    for (int b0 = 0; b0 < a.seqs; b0 += kThreads) {
        const int b = b0 + tid, n = min(kThreads, a.seqs - b0);
        Sums sum = all;
        if (!one) {
            s = sequence_of(a, b);
            mine = scan(s.sums, sum, shared);
        }
        const Sums end = before + mine;
        if (tid < n) {
            if (lengths && blockIdx.x == 0) a.kv_out[b] = done ? (int32_t)s.length : a.kv_len[b];
            if (tables && blockIdx.x == 0) a.q_start[b + 1] = done ? (int32_t)end.fresh : 0;
        }
        if (!done || !tables) continue;
        fresh_end[tid] = (int32_t)end.fresh;
        take_end[tid] = (int32_t)end.take;
        give_end[tid] = (int32_t)end.give;
        length[tid] = (int32_t)s.length;
        held[tid] = (int32_t)s.held;
        need[tid] = (int32_t)s.need;
        __syncthreads();
        const Sums past = before + sum;
        const Range takes = share(all.take, before.take, past.take);
        for (int32_t k = takes.first + tid; k < takes.last; k += kThreads) {
            const int i = find(take_end, n, k);
            const int32_t slot = need[i] - (take_end[i] - k);
            a.table[(b0 + i) * a.table_stride + slot] = a.ring[(uint32_t)(first + k) % pages];
        }
        const Range gives = share(all.give, before.give, past.give);
        for (int32_t k = gives.first + tid; k < gives.last; k += kThreads) {
            const int i = find(give_end, n, k);
            const int32_t slot = held[i] - (give_end[i] - k);
            a.ring[(uint64_t)(first + free + k) % pages] = a.table[(b0 + i) * a.table_stride + slot];
        }
        const Range tokens = share(a.rows, before.fresh, past.fresh);
        for (int32_t t = tokens.first + tid; t < tokens.last; t += kThreads) {
            const int i = find(fresh_end, n, t);
            const int32_t p = length[i] - (fresh_end[i] - t), slot = p / a.page_size;
            if (a.pos) a.pos[t] = p;
            if (a.slots) {
                const int32_t taken = slot - held[i];
                const int32_t page = taken < 0 ? a.table[(b0 + i) * a.table_stride + slot]
                                               : a.ring[(uint32_t)(first + take_end[i] - (need[i] - held[i]) + taken) % pages];
                a.slots[t] = (int64_t)page * a.page_size + (p - slot * a.page_size);
            }
        }
        before = past;
        __syncthreads();
    }

    // ---- what belongs to no sequence, and the whole step's numbers ----------------------
    if (tables) {
        const Range rest = share(a.rows, done ? all.fresh : 0, a.rows);
        for (int64_t t = (int64_t)rest.first + tid; t < rest.last; t += kThreads) {
            if (a.pos) a.pos[t] = 0;
            if (a.slots) a.slots[t] = -1;
        }
        if (blockIdx.x == 0 && tid == 0) {
            a.q_start[0] = 0;
            *a.short_of = lacking;
        }
    }
    if (lengths && blockIdx.x == 0 && tid == 0) {
        const int32_t f = a.state[0], n = a.state[1];
        a.state_out[0] = done ? (int32_t)((uint32_t)(first + all.take) % pages) : f;
        a.state_out[1] = done ? (int32_t)(free - all.take + all.give) : n;
    }
}

}  // namespace

hipError_t launch_pages(const PagesArgs& a, hipStream_t s)
{
    const int64_t groups = std::max((int64_t)1, std::min((int64_t)256, (a.rows + 16 * (int64_t)a.seqs + 4095) / 4096));
    const bool apart = groups > 1 && (a.kv_out == a.kv_len || a.state_out == a.state);
    hipLaunchKernelGGL(pages_kernel, dim3((unsigned)groups), dim3(kThreads), 0, s, a, true, !apart);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !apart) return e;
    hipLaunchKernelGGL(pages_kernel, dim3(1), dim3(kThreads), 0, s, a, false, true);
    return hipGetLastError();
}

}  // namespace tr
