// What the attention kernels share on the device: their sequences and what a row
// of them sees, the deal of all steps to the workgroups, the parts of items that
// several workgroups work on, and a finished row.
#pragma once

#include "tr_attn.h"
#include "tr_divide.h"
#include "tr_wave.h"

namespace tr {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;

__device__ __forceinline__ float minus_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float from_bf16(uint32_t v) { return __uint_as_float(v << 16); }

// The largest of three, NaN if one is: one instruction, and one that does not
// first quiet a matrix instruction's result in another, as fmaxf does.  Both of
// these stay in the compiler's hands: between a matrix instruction or an
// exponential and a reader of its result there have to be waits, which it counts
// for its own instructions and not for those of inline assembly.
__device__ __forceinline__ float max3(float x, float y, float z)
{
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z);
}

// Two values rounded to bf16, the first one low.
__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}

// Whether a word holds a bf16 that is not finite.
__device__ __forceinline__ bool not_finite(uint32_t w)
{
    return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

// ---- sequences ---------------------------------------------------------------------
// One sequence of the step, its fields clamped to what the tensors hold.
struct Sequence {
    int64_t q0;        // first packed row
    int32_t n;         // new tokens
    int32_t len;       // tokens with the new ones, as given: token i is number len - n + i
    int32_t begin;     // first token that some row sees
    int32_t end;       // past the last one
};

__device__ __forceinline__ Sequence sequence_at(const AttendArgs& a, int b)
{
    Sequence s;
    const int64_t q0 = min(max((int64_t)a.step.q_start[b], (int64_t)0), a.tokens);
    const int64_t q1 = min(max((int64_t)a.step.q_start[b + 1], q0), a.tokens);
    s.q0 = q0;
    s.n = (int32_t)(q1 - q0);
    s.len = a.step.kv_len[b];
    s.end = max(0, min(s.len, a.most));
    s.begin = a.window > 0 ? (int32_t)min((int64_t)s.end, max((int64_t)0, (int64_t)s.len - s.n - a.window + 1)) : 0;
    return s;
}

// The tokens [lo, hi) that new token i sees.
__device__ __forceinline__ void seen_by(const AttendArgs& a, const Sequence& s, int i, int& lo, int& hi)
{
    const int64_t p = (int64_t)s.len - s.n + i;
    hi = a.causal ? (int)max((int64_t)0, min((int64_t)s.end, p + 1)) : s.end;
    lo = a.window > 0 ? (int)max((int64_t)0, p - a.window + 1) : 0;
}

// ---- the deal of the work -------------------------------------------------------------
// The work is the items (sequence, key head, tile of rows), each with its range of
// keys in steps.  All steps of all items in a row are dealt out to the workgroups
// in equal shares, whatever the sequences' lengths: a workgroup's share can end
// inside an item, and then the last of its workgroups to arrive joins the item's
// parts.
constexpr int kFewThreads = 256;
constexpr int kAlign = 32;   // a range of keys begins at a multiple of it

// Where a workgroup is in the row of all steps.  Items of a sequence are its
// tiles of ROWS rows, and of each the key heads one after another.
struct Place {
    int b;             // sequence
    Sequence s;
    int steps;         // of an item of it
    int tiles;         // of rows
    int64_t first;     // its first step in the row
};

// Steps of STEP keys that an item of a sequence takes (STEP 0: an item is one step).
template <int STEP>
__device__ __forceinline__ int steps_of(const Sequence& s)
{
    if constexpr (STEP == 0) return 1;
    else return max(1, (s.end - (s.begin & ~(kAlign - 1)) + STEP - 1) / STEP);
}

template <int ROWS>
__device__ __forceinline__ int tiles_of(const AttendArgs& a, const Sequence& s)
{
    return (int)(((int64_t)s.n * a.group + ROWS - 1) / ROWS);
}

template <int ROWS, int STEP>
__device__ __forceinline__ int64_t cost_of(const AttendArgs& a, int b, int extra)
{
    if (b >= a.step.seqs) return 0;
    const Sequence s = sequence_at(a, b);
    return (int64_t)tiles_of<ROWS>(a, s) * (steps_of<STEP>(s) + extra) * a.kv_heads;
}

// All steps, and a workgroup's share of them: at least 1 / kMostParts of the
// longest item's, so that an item, which may begin inside a share, has at most
// kMostParts + 1 parts, which one workgroup can join.
constexpr int kMostParts = 64;

struct Shares {
    int64_t total, share;
    int extra;         // steps that an item counts for besides its own (first_place)
};

template <int ROWS, int STEP>
__device__ __forceinline__ Shares shares_of(const AttendArgs& a, int lane)
{
    int64_t sum = 0;
    int most = 0;
    for (int b0 = 0; b0 < a.step.seqs; b0 += 64) {
        const int b = b0 + lane;
        if (b < a.step.seqs) {
            const Sequence s = sequence_at(a, b);
            const int steps = steps_of<STEP>(s);
            sum += (int64_t)tiles_of<ROWS>(a, s) * steps * a.kv_heads;
            if (s.n > 0) most = max(most, steps);       // those without new tokens have no items
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        sum += __shfl_xor(sum, m);
        most = max(most, __shfl_xor(most, m));
    }
    Shares r;
    r.total = uniform(sum);
    r.share = max((r.total + gridDim.x - 1) / gridDim.x,
                  (int64_t)((__builtin_amdgcn_readfirstlane(most) + kMostParts - 1) / kMostParts));
    r.extra = 0;
    return r;
}

// Sequences up to which a workgroup may look for an item among all of them, a wavefront
// 64 at a time, instead of walking over those of its share (8 heads of keys of 128,
// a group of 4; 64 sequences of 128 tokens over 512: 135 us by items, 148 by shares;
// 256 of 64: 333 and 321; 1024 of 16: 1027 and 770; 16384 of 16 over 64: 69 and 4.4 ms).
constexpr int kSearched = 128;

// The sequence that step u (< all_steps) lies in, searched from sequence `from`
// on, before which lie `before` (<= u) steps: a workgroup walks the sequences of
// its share once.
template <int ROWS, int STEP>
__device__ __forceinline__ Place place_of(const AttendArgs& a, int64_t u, int lane, int from = 0, int64_t before = 0, int extra = 0)
{
    Place p{};
    for (int b0 = from; b0 < a.step.seqs; b0 += 64) {
        const int64_t c = cost_of<ROWS, STEP>(a, b0 + lane, extra);
        int64_t sum = c;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int64_t o = __shfl_up(sum, m);
            if (lane >= m) sum += o;
        }
        const uint64_t past = __ballot(u < before + sum);
        if (past) {
            const int at = __builtin_ctzll(past);
            p.b = b0 + at;
            p.first = uniform(before + __shfl(sum - c, at));
            break;
        }
        before += uniform(__shfl(sum, 63));
    }
    p.b = __builtin_amdgcn_readfirstlane(p.b);
    p.s = sequence_at(a, p.b);
    p.steps = steps_of<STEP>(p.s) + extra;
    p.tiles = tiles_of<ROWS>(a, p.s);
    return p;
}

// shares_of, and where the workgroup's share begins, with each sequence looked at once
// where a wavefront can (up to 64 of them).  To begin an item and to end it takes a
// workgroup about as long as kItemSteps steps; where shares are long each item counts
// for so many more, at its beginning.  A share has at least LEAST steps.
constexpr int kItemSteps = 3, kLongShare = 8;

template <int ROWS, int STEP, int LEAST>
__device__ __forceinline__ Shares first_place(const AttendArgs& a, int lane, Place& p)
{
    if (a.step.seqs > 64) {
        Shares all = shares_of<ROWS, STEP>(a, lane);
        all.share = max(all.share, (int64_t)LEAST);
        const int64_t u = (int64_t)blockIdx.x * all.share;
        if (u < all.total) p = place_of<ROWS, STEP>(a, u, lane);
        return all;
    }
    Sequence s{};
    int64_t cost = 0, items = 0;
    int steps = 0;
    if (lane < a.step.seqs) {
        s = sequence_at(a, lane);
        steps = steps_of<STEP>(s);
        items = (int64_t)tiles_of<ROWS>(a, s) * a.kv_heads;
        cost = items * steps;
    }
    int64_t sum = cost, all_items = items;
    int most = s.n > 0 ? steps : 0;               // those without new tokens have no items
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int64_t o = __shfl_up(sum, m), i = __shfl_up(all_items, m);
        if (lane >= m) {
            sum += o;
            all_items += i;
        }
        most = max(most, __shfl_xor(most, m));
    }
    Shares r;
    r.total = uniform(__shfl(sum, 63));
    r.extra = r.total >= (int64_t)kLongShare * gridDim.x ? kItemSteps : 0;
    sum += all_items * r.extra;
    cost += items * r.extra;
    r.total = uniform(__shfl(sum, 63));
    r.share = max(max((r.total + gridDim.x - 1) / gridDim.x, (int64_t)LEAST),
                  (int64_t)((__builtin_amdgcn_readfirstlane(most) + r.extra + kMostParts - 1) / kMostParts));
    const uint64_t past = __ballot((int64_t)blockIdx.x * r.share < sum);
    p.b = past ? __builtin_ctzll(past) : 0;
    auto from = [&](int x) { return __builtin_amdgcn_readlane(x, p.b); };
    p.first = uniform(__shfl(sum - cost, p.b));
    p.steps = from(steps) + r.extra;
    p.s.q0 = uniform(__shfl(s.q0, p.b));
    p.s.n = from(s.n);
    p.s.len = from(s.len);
    p.s.begin = from(s.begin);
    p.s.end = from(s.end);
    return r;
}

// N elements from e0 of one finished row: sums over their l, and lse from the
// maximum (of scores in powers of two) and l.
template <int N>
__device__ __forceinline__ void finish_row(const AttendArgs& a, int64_t t, int head, int e0, const float (&acc)[N], float l, float m)
{
    const bool some = l > 0.f || l != l;
    const float f = some ? 1.f / l : 0.f;
    uint16_t* p = static_cast<uint16_t*>(a.out.p) + t * a.out.token + (int64_t)head * a.out.head + e0;
    constexpr int V = N < 8 ? N : 8;
#pragma unroll
    for (int e = 0; e < N; e += V) {
        if (e0 + e >= a.dim) break;
        uint32_t w[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            w[i] = some ? (uint32_t)to_bf16(acc[e + 2 * i] * f) | (uint32_t)to_bf16(acc[e + 2 * i + 1] * f) << 16 : 0u;
        if constexpr (V == 8) *reinterpret_cast<u32x4*>(p + e) = u32x4{w[0], w[1], w[2], w[3]};
        else if constexpr (V == 4) *reinterpret_cast<uint2*>(p + e) = uint2{w[0], w[1]};
        else *reinterpret_cast<uint32_t*>(p + e) = w[0];
    }
    if (a.lse && e0 == 0) a.lse[t * a.heads + head] = some ? fmaf(m, kLn2, __logf(l)) : minus_inf();
}

// ---- parts of items ------------------------------------------------------------------
// A part that another workgroup, on another XCD, is to read is written and read
// past the L2s, by accesses of agent scope.  A workgroup's two parts are the end
// of an item begun before it (0) and the beginning of one that goes on past it (1).
__device__ __forceinline__ void put2(float* p, float x, float y)
{
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ float2 get2(const float* p)
{
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return float2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// Floats of a part: ROWS rows of DH sums, their maxima and l.
template <int DH, int ROWS>
constexpr int kPartFloats = ROWS * DH + 2 * ROWS;

// Floats of a context's parts for each CU, and whether the two parts of each of PER_CU
// workgroups fit: each launch that writes parts asserts that its own do.
template <int DH>
constexpr int kCuFloats = 2 * kPartFloats<DH, DH == 256 ? 128 : 256>;
template <int DH, int ROWS, int PER_CU = 1>
constexpr bool kPartsFit = PER_CU * 2 * kPartFloats<DH, ROWS> <= kCuFloats<DH>;

// One item's parts: `count` of them, this workgroup's is number `mine`, the
// first is workgroup `owner`'s second.
struct Parts {
    int owner, count, mine;
};

__device__ __forceinline__ Parts parts_of(int64_t begin, int64_t end, int64_t share)
{
    Parts p;
    p.owner = (int)(begin / share);
    p.count = (int)((end - 1) / share) - p.owner + 1;
    p.mine = (int)blockIdx.x - p.owner;
    return p;
}

template <int FLOATS>
__device__ __forceinline__ float* part_at(const AttendArgs& a, const Parts& p, int i)
{
    return a.part + ((int64_t)(p.owner + i) * 2 + (i == 0)) * FLOATS;
}

// Whether all other parts are there already; the same in the whole workgroup.
__device__ __forceinline__ bool others_done(const AttendArgs& a, const Parts& p, int* shared)
{
    if (threadIdx.x == 0)
        *shared = __hip_atomic_load(a.arrived + p.owner, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.count - 1;
    __syncthreads();
    return *shared != 0;
}

// After this workgroup's part is written: whether it was the last one.
__device__ __forceinline__ bool last_to_arrive(const AttendArgs& a, const Parts& p, int* shared)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wavefront's stores are done
    __syncthreads();
    if (threadIdx.x == 0)
        *shared = __hip_atomic_fetch_add(a.arrived + p.owner, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.count - 1;
    __syncthreads();
    return *shared != 0;
}

// The count is back at zero for the next call.
__device__ __forceinline__ void joined(const AttendArgs& a, const Parts& p)
{
    if (threadIdx.x == 0) __hip_atomic_store(a.arrived + p.owner, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Address swizzles of a row in shared memory, in pieces of 16 bytes: the 16 rows
// that a read of K's fragments, or a transposing read of V, touches spread over
// all banks.
template <int DH>
__device__ __forceinline__ int k_swizzle(int row)
{
    return DH == 64 ? (row >> 1) & 7 : row & 15;
}

template <int DH>
__device__ __forceinline__ int v_piece(int row, int piece)
{
    return piece ^ ((DH == 64 ? (row >> 1) & 3 : row & 7) << 1);
}

// 16 bytes of keys or values that nothing reads again soon.
__device__ __forceinline__ u32x4 read_once(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x4*>(p)); }

// ---- tiles of many rows ---------------------------------------------------------------
constexpr int kManyTile = 64, kManyRows = 32;

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int DH>
__device__ __forceinline__ int v_swizzle(int row)
{
    return DH == 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2;
}

// Whether the workgroups take whole items in turn instead of equal shares of all
// steps.  Shares count an item's steps as those of all its sequence's rows; where
// tiles see only part of them (a prompt's, half of them on average; those under a
// window, little more than it) the shares of such tiles are done sooner.  Taken
// whole, the steps of the tiles themselves count, and half of the longest tile's
// at the end while other workgroups have none left.  8 heads of keys, a group of 4:
// a prompt of 3800 tokens from an empty cache takes 199 us so and 296 by shares,
// 1500 tokens with a window of 512 over 8000 37 and 65.
template <int ROWS, int STEP>
__device__ __forceinline__ bool items_alone(const AttendArgs& a, const Shares& all, int lane)
{
    if constexpr (STEP == 0) return true;
    else {
        if (!a.causal || a.step.seqs > kSearched) return false;
        float sum = 0.f, most = 0.f;
        const float tile = (float)(ROWS / a.group + 1);             // new tokens of a tile
        for (int b = lane; b < a.step.seqs; b += 64) {
            const Sequence s = sequence_at(a, b);
            if (s.n == 0) continue;
            float mean = max(1.f, ((float)(s.end - s.begin) - 0.5f * max(0.f, (float)s.n - tile)) / STEP), top = (float)steps_of<STEP>(s);
            if (a.window > 0) {
                const float one = ((float)a.window + tile) / STEP + 1.f;
                mean = min(mean, one);
                top = min(top, one);
            }
            sum += mean * (float)tiles_of<ROWS>(a, s) * (float)a.kv_heads;
            most = max(most, top);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            sum += __shfl_xor(sum, m);
            most = max(most, __shfl_xor(most, m));
        }
        const float alone = max(most, sum / (float)gridDim.x + 0.5f * most);
        return __all(alone < (float)all.share) != 0;
    }
}

// 16 bytes a lane from memory into shared memory at lds + 16 lane.  An
// instruction without a register result: the kernel counts and waits itself.
__device__ __forceinline__ void load_lds(uint32_t lds, const void* p)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}

// The same from base + off, the base the wavefront's.
__device__ __forceinline__ void load_lds(uint32_t lds, const void* base, uint32_t off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}

__device__ __forceinline__ void wait_all_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ float max_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

}  // namespace
}  // namespace tr
