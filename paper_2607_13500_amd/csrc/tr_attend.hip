// Attention of packed new tokens over a paged cache:
//   out = sum_j softmax_j(scale q . k_j) v_j  over the tokens j that a row sees,
// in one pass over the keys with a running maximum m and sum l:  a tile's
// weights are exp(s - m'), and what was summed before is scaled by exp(m - m').
// Exponentials are powers of two, scores carry log2(e).
//
// Rows.  The rows of one sequence that share a key head are its new tokens
// times the group of query heads: row r is token r / group, head r % group of
// the group.  Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T:
// a matrix instruction's accumulator then holds a row of queries in a lane's
// registers, so the softmax needs no shared memory, and the weights are already
// where the second product takes them from; only V has to change its order, by
// transposing reads of shared memory.
//
// Weights are rounded to bf16 for the second product (the sum l takes them
// unrounded): its operands have one type, and V is bf16.  A second product with
// what the rounding leaves, for which few rows have the time, would turn infinite
// values into NaN: that rest is 0 or negative as often as not.
#include <algorithm>

#include "tr_attn.h"
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
// j / page_size and r / group for uniform divisors, by multiplication.
__device__ __forceinline__ uint32_t divide(uint32_t x, const Divisor& d) { return (__umulhi(d.mul, x) + x) >> d.shift; }

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

// ---- few rows over many keys -----------------------------------------------------------
// The work is the items (sequence, key head, tile of 16 rows), each with its
// range of keys in steps of kStep.  All steps of all items in a row are dealt
// out to the workgroups in equal shares, whatever the sequences' lengths: a
// workgroup's share can end inside an item, and then the last of its workgroups
// to arrive joins the item's parts.  A workgroup's four wavefronts take tiles of 32 keys in
// turn, each with its own maximum and sums, and join them at the end of an item.
//
// Bound by the bytes of the cache: a wavefront has the next tile's keys and
// values in flight, in registers, while it works on one; 16 rows cost two
// matrix instructions of 16 cycles per 16 x 32 elements of keys.  Rows of a head
// are read whole, a load after another, and past the caches: 5.9-6.2 TB/s (64
// requests over 256 to 16384 tokens 211 us), where 64 bytes of 16 rows at a time
// through the caches reached 5.2.  Three workgroups of a CU instead of two spill
// registers (342 us).
constexpr int kRows = 16, kTile = 32, kStep = 128, kFewThreads = 256;
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
__device__ __forceinline__ int64_t cost_of(const AttendArgs& a, int b)
{
    if (b >= a.step.seqs) return 0;
    const Sequence s = sequence_at(a, b);
    return (int64_t)tiles_of<ROWS>(a, s) * steps_of<STEP>(s) * a.kv_heads;
}

// All steps, and a workgroup's share of them: at least 1 / kMostParts of the
// longest item's, so that an item, which may begin inside a share, has at most
// kMostParts + 1 parts, which one workgroup can join.
constexpr int kMostParts = 64;

struct Shares {
    int64_t total, share;
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
__device__ __forceinline__ Place place_of(const AttendArgs& a, int64_t u, int lane, int from = 0, int64_t before = 0)
{
    Place p{};
    for (int b0 = from; b0 < a.step.seqs; b0 += 64) {
        const int64_t c = cost_of<ROWS, STEP>(a, b0 + lane);
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
    p.steps = steps_of<STEP>(p.s);
    p.tiles = tiles_of<ROWS>(a, p.s);
    return p;
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

// Workgroups of a CU, by their registers.
template <int DH>
constexpr int kFewPerCu = DH == 64 ? 3 : DH == 128 ? 2 : 1;

// PG16: pages of whole halves of a tile (a multiple of 16 tokens, below 2 GB),
// so that a half's page is the wavefront's and a lane's place in it fixed.
// FULL: head_dim is DH.
template <int DH, bool PG16, bool FULL>
__global__ __launch_bounds__(kFewThreads, kFewPerCu<DH>) void attend_few_kernel(AttendArgs a)
{
    constexpr int KF = DH / 32, DT = DH / 16;          // fragments of keys, tiles of elements
    constexpr int PIECES = DH / 8, VR = 64 / PIECES, VN = kTile / VR;   // pieces of a row, rows of a load, loads of a tile
    constexpr int PAD = DH + 4;
    constexpr int BYTES = kTile * DH * 2;
    constexpr int kLds = 4 * (2 * BYTES > kRows * PAD * 4 ? 2 * BYTES : kRows * PAD * 4);
    __shared__ __align__(16) unsigned char smem[kLds];
    __shared__ float ml[4][2][kRows];
    __shared__ int flag;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int vrow = lane / PIECES, piece = lane % PIECES;
    unsigned char* kt = smem + wave * 2 * BYTES;                 // the wavefront's tile
    unsigned char* vt = kt + BYTES;
    const int token_bytes = (int)(a.cache.token * 2);            // PG16
    const int in_lane = vrow * token_bytes + piece * 16;

    const Shares all = shares_of<kRows, kStep>(a, lane);
    int64_t u = (int64_t)blockIdx.x * all.share;
    const int64_t u_end = min(u + all.share, all.total);

    int from = 0;
    int64_t before = 0;
    while (u < u_end) {
        const Place pl = place_of<kRows, kStep>(a, u, lane, from, before);
        from = pl.b;
        before = pl.first;
        const Sequence s = pl.s;
        const int64_t local = u - pl.first;
        const int item = (int)(local / pl.steps), step0 = (int)(local - (int64_t)item * pl.steps);
        const int step1 = (int)min((int64_t)pl.steps, step0 + (u_end - u));
        const int rt = item / a.kv_heads, h = item - rt * a.kv_heads;
        const bool whole = step0 == 0 && step1 == pl.steps;

        // ---- this lane's row ------------------------------------------------------
        const int rows = (int)min((int64_t)kRows, (int64_t)s.n * a.group - (int64_t)rt * kRows);
        const uint32_t r = (uint32_t)(rt * kRows + col);
        const int tok = (int)divide(r, a.by_group), head = h * a.group + (int)(r - (uint32_t)tok * a.group);
        const bool live = col < rows;
        int lo = 0, hi = 0;
        if (live) seen_by(a, s, tok, lo, hi);
        int lo_min, lo_max, hi_min, hi_max;       // over the tile's rows
        {
            const int t0 = (int)divide((uint32_t)rt * kRows, a.by_group), t1 = (int)divide((uint32_t)(rt * kRows + rows - 1), a.by_group);
            seen_by(a, s, t0, lo_min, hi_min);
            seen_by(a, s, t1, lo_max, hi_max);
        }
        bf16x8 qf[KF];
#pragma unroll
        for (int k = 0; k < KF; ++k) {
            u32x4 v{};
            if (live && k * 32 + grp * 8 < a.dim)
                v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q.p) + (s.q0 + tok) * a.q.token + (int64_t)head * a.q.head + k * 32 + grp * 8);
            qf[k] = __builtin_bit_cast(bf16x8, v);
        }
        f32x4 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = minus_inf(), l = 0.f;

        // ---- keys -------------------------------------------------------------------
        const int base = s.begin & ~(kTile - 1);
        const int j_end = min(hi_max, base + step1 * kStep);
        const int first = base + step0 * kStep + wave * kTile;
        // tiles before any row's range are skipped
        int j0 = first;
        if (j0 + kTile <= lo_min) j0 += ((lo_min - j0) / kStep) * kStep;
        if (j0 + kTile <= lo_min) j0 += kStep;
        const int32_t* table = a.step.table + (int64_t)pl.b * a.step.table_stride;
        const uint16_t* kp = static_cast<const uint16_t*>(a.cache.k) + (int64_t)h * a.cache.head;
        const uint16_t* vp = static_cast<const uint16_t*>(a.cache.v) + (int64_t)h * a.cache.head;
        const int last = hi_max - 1;              // tokens past it (and before lo_min) are read as it (as lo_min)

        auto page_at = [&](int slot) { return min(max(table[slot], 0), a.cache.pages - 1); };
        u32x4 kr[VN], vr[VN];
        auto fetch = [&](int j) {
            if constexpr (PG16) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    // rows of a half that no row sees are read all the same (they are in
                    // the page), a half without any in the place of the nearest one
                    const int half = min(max(j + 16 * x, lo_min & ~15), last & ~15);
                    const int slot = (int)divide((uint32_t)half, a.by_page);
                    const int64_t at = (int64_t)page_at(slot) * a.cache.page + (int64_t)(half - slot * a.cache.page_size) * a.cache.token;
                    const int64_t off = uniform(at);
                    const char* kb = reinterpret_cast<const char*>(kp + off) + in_lane;
                    const char* vb = reinterpret_cast<const char*>(vp + off) + in_lane;
#pragma unroll
                    for (int i = 0; i < VN / 2; ++i)
                        if (FULL || piece * 8 < a.dim) {
                            kr[x * (VN / 2) + i] = read_once(kb + i * VR * token_bytes);
                            vr[x * (VN / 2) + i] = read_once(vb + i * VR * token_bytes);
                        }
                }
            } else {
                int64_t koff[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int t = min(max(j + 16 * x + col, lo_min), last);
                    const int slot = (int)divide((uint32_t)t, a.by_page);
                    koff[x] = (int64_t)page_at(slot) * a.cache.page + (int64_t)(t - slot * a.cache.page_size) * a.cache.token;
                }
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    const int64_t off = __shfl(koff[VR * i / 16], (VR * i + vrow) & 15) + piece * 8;
                    if (FULL || piece * 8 < a.dim) {
                        kr[i] = read_once(kp + off);
                        vr[i] = read_once(vp + off);
                    }
                }
            }
        };
        if constexpr (!FULL) {
#pragma unroll
            for (int i = 0; i < VN; ++i) kr[i] = u32x4{};   // pieces past the head stay zero
        }
        if (j0 < j_end) fetch(j0);
        for (; j0 < j_end; j0 += kStep) {
            // rows that see different tokens of this tile: a value that is not
            // finite must not reach the rows that do not see it
            const bool mixed = lo_max > max(j0, lo_min) || hi_min < min(j0 + kTile, hi_max);
            bool bad = false;
            if (mixed) {
#pragma unroll
                for (int i = 0; i < VN; ++i)
                    bad |= not_finite(vr[i].x) || not_finite(vr[i].y) || not_finite(vr[i].z) || not_finite(vr[i].w);
                bad = bad && (FULL || piece * 8 < a.dim);
            }
            // nor one that no row sees
            if (j0 < lo_min || j0 + kTile > hi_max) {
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    const int t = j0 + VR * i + vrow;
                    if (t < lo_min || t > last) vr[i] = u32x4{};
                }
            }
#pragma unroll
            for (int i = 0; i < VN; ++i)
            {
                const int row = VR * i + vrow;
                *reinterpret_cast<u32x4*>(kt + row * (DH * 2) + (piece ^ k_swizzle<DH>(row)) * 16) = kr[i];
                *reinterpret_cast<u32x4*>(vt + row * (DH * 2) + v_piece<DH>(row, piece) * 16) = vr[i];
            }
            if (j0 + kStep < j_end) fetch(j0 + kStep);
            f32x4 sc[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                sc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
                const int row = 16 * x + col;
#pragma unroll
                for (int k = 0; k < KF; ++k) {
                    const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + row * (DH * 2) + ((4 * k + grp) ^ k_swizzle<DH>(row)) * 16);
                    sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[k], sc[x], 0, 0, 0);
                }
            }

            // ---- weights ------------------------------------------------------------
            float p[8];
            float top = minus_inf();
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int j = j0 + 16 * x + 4 * grp + v;
                    const float y = sc[x][v] * a.scale;
                    p[4 * x + v] = j >= lo && j < hi ? y : minus_inf();
                    top = fmaxf(top, p[4 * x + v]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m1 = fmaxf(m, top), zero = m1 == minus_inf() ? 0.f : m1;
            const bool same = m1 == m;                // rows that see nothing yet among them
            const float keep = exp2_(m - zero);
            m = m1;
            l *= keep;
            u32x4 pb;
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                p[v] = exp2_(p[v] - zero);
                l += p[v];
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) pb[v] = pack_bf16(p[2 * v], p[2 * v + 1]);
            if (!__all(same)) {
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= keep;
            }
            // ---- values ---------------------------------------------------------------
            if (__any(bad)) {
                // values that are not finite go to the rows that see them, key by
                // key, and count as zeros in the product
#pragma unroll 1
                for (int i = 0; i < kTile; ++i) {
                    uint32_t y = 0;       // key i lies in group (i / 4) % 4, element 4 (i / 16) + i % 4
#pragma unroll
                    for (int v = 0; v < 4; ++v) y = v == (i >> 4) * 2 + (i >> 1 & 1) ? pb[v] : y;
                    y = __shfl(y, (i & 12) * 4 + col);
                    const float w = from_bf16(i & 1 ? y >> 16 : y & 0xffffu);
                    const bool sees = j0 + i >= lo && j0 + i < hi;
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const int e = 16 * d + 4 * grp;
                        const uint16_t* q = reinterpret_cast<const uint16_t*>(vt + i * (DH * 2) + v_piece<DH>(i, e / 8) * 16) + e % 8;
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const float y = fmaf(w, from_bf16(q[v]), o[d][v]);
                            o[d][v] = sees && not_finite(q[v]) ? y : o[d][v];
                        }
                    }
                }
#pragma unroll 1
                for (int i = 0; i < kTile; ++i)
#pragma unroll 1
                    for (int e = lane; e < DH; e += 64) {
                        uint16_t* q = reinterpret_cast<uint16_t*>(vt + i * (DH * 2)) + e;
                        if (not_finite(*q)) *q = 0;
                    }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                s16x8 vf;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 16 * x + 4 * grp + (lane & 15) / 4, e = 16 * d + 4 * (lane & 3);
                    const unsigned char* q = vt + row * (DH * 2) + v_piece<DH>(row, e / 8) * 16 + (e % 8) * 2;
                    const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q);
#pragma unroll
                    for (int v = 0; v < 4; ++v) vf[4 * x + v] = t[v];
                }
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pb), o[d], 0, 0, 0);
            }
        }

        // ---- the four wavefronts' parts -------------------------------------------------
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        __syncthreads();
        float* red = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<f32x4*>(red + (wave * kRows + col) * PAD + 16 * d + 4 * grp) = o[d];
        if (grp == 0) {
            ml[wave][0][col] = m;
            ml[wave][1][col] = l;
        }
        __syncthreads();
        {
            constexpr int N = DH / 16;            // elements of a thread
            const int row = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * N;
            float top = minus_inf();
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w][0][row]);
            const float zero = top == minus_inf() ? 0.f : top;
            float sum = 0.f, acc[N] = {};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = exp2_(ml[w][0][row] - zero);
                sum = fmaf(ml[w][1][row], f, sum);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] = fmaf(red[(w * kRows + row) * PAD + e0 + e], f, acc[e]);
            }
            const uint32_t rr = (uint32_t)(rt * kRows + row);
            const int t = (int)divide(rr, a.by_group), hd = h * a.group + (int)(rr - (uint32_t)t * a.group);
            bool finish = whole;
            if (!whole) {
                constexpr int F = kPartFloats<DH, kRows>;
                const int64_t begin = pl.first + (int64_t)item * pl.steps;
                const Parts parts = parts_of(begin, begin + pl.steps, all.share);
                float* part = part_at<F>(a, parts, parts.mine);
                if (row < rows) {
#pragma unroll
                    for (int e = 0; e < N; e += 2) put2(part + row * DH + e0 + e, acc[e], acc[e + 1]);
                    if (e0 == 0) put2(part + kRows * DH + 2 * row, top, sum);
                }
                finish = last_to_arrive(a, parts, &flag);
                if (finish) {
                    // all parts in their order, eight of them on their way at a time
                    constexpr int U = N > 8 ? 4 : 8;
                    if (row < rows) {
                        top = minus_inf();
                        sum = 0.f;
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[e] = 0.f;
                        for (int i0 = 0; i0 < parts.count; i0 += U) {
                            float2 ml_i[U], v[U][N / 2];
#pragma unroll
                            for (int i = 0; i < U; ++i) {
                                const float* q = part_at<F>(a, parts, min(i0 + i, parts.count - 1));
                                ml_i[i] = get2(q + kRows * DH + 2 * row);
#pragma unroll
                                for (int e = 0; e < N; e += 2) v[i][e / 2] = get2(q + row * DH + e0 + e);
                            }
#pragma unroll
                            for (int i = 0; i < U; ++i) {
                                if (i0 + i >= parts.count) break;
                                const float m1 = fmaxf(top, ml_i[i].x), z = m1 == minus_inf() ? 0.f : m1;
                                const float f = exp2_(top - z), g = exp2_(ml_i[i].x - z);
                                top = m1;
                                sum = fmaf(ml_i[i].y, g, sum * f);
#pragma unroll
                                for (int e = 0; e < N; e += 2) {
                                    acc[e] = fmaf(v[i][e / 2].x, g, acc[e] * f);
                                    acc[e + 1] = fmaf(v[i][e / 2].y, g, acc[e + 1] * f);
                                }
                            }
                        }
                    }
                    joined(a, parts);
                }
            }
            if (finish && row < rows) finish_row<N>(a, s.q0 + t, hd, e0, acc, sum, top);
        }
        __syncthreads();
        u += step1 - step0;
    }
}

// ---- many rows ---------------------------------------------------------------------------
// A workgroup of NW wavefronts of 32 rows each over the same keys, in tiles of
// 64 that go from memory straight into shared memory, two tiles there at a time:
// one is loaded while the other is worked on.  Bound by the matrix instructions
// and by the softmax between them, which the two wavefronts of a SIMD overlap:
// a prompt of 18432 tokens of 32 heads of 128 takes 2.85-3.01 ms by the box
// (925-977 TFLOP/s; 42 % of the matrix units' cycles), eight chunks over long
// contexts 530-565 us (640-684: the last shares end unevenly, and their parts are
// joined).
//
// Shared memory rows are DH elements in pieces of 16 bytes; piece c of row r lies
// at piece c ^ f(r), which the loads bring about by each lane's choice of source
// (they fill shared memory in lane order).  f spreads the rows that one read of
// 16 (keys) or 4 (values) rows touches over all banks.
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

// PG16: pages of whole 16 tokens, below 2 GB: the rows that one wavefront's load
// fills lie in one page, whose address is the wavefront's.
template <int DH, int NW, int STEP, bool PG16, bool FULL>
__global__ __launch_bounds__(NW * 64, DH == 256 ? 1 : 2) void attend_many_kernel(AttendArgs a)
{
    constexpr int ROWS = NW * kManyRows, T = NW * 64;
    constexpr int KF = DH / 16, DT = DH / 32;               // fragments of keys, tiles of elements
    constexpr int PIECES = DH / 8, BYTES = kManyTile * DH * 2;
    constexpr int LR = T / PIECES, NI = kManyTile / LR;     // rows of one round of loads, rounds of a tile
    constexpr int WR = 64 / PIECES;                         // rows that a wavefront loads
    __shared__ __align__(16) unsigned char smem[4 * BYTES]; // stage 0: K, V; stage 1: K, V
    __shared__ int flag;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int lrow = threadIdx.x / PIECES, lpos = threadIdx.x % PIECES;

    const Shares all = shares_of<ROWS, STEP>(a, lane);
    const bool by_item = STEP == 0 || items_alone<ROWS, STEP>(a, all, lane);
    int64_t u, u_end = 0;
    if (by_item) {
        // whole items, the last ones (which see most) first
        u = (STEP == 0 ? all.total : shares_of<ROWS, 0>(a, lane).total) - 1 - (int64_t)blockIdx.x;
        if (u < 0) return;
    } else {
        u = (int64_t)blockIdx.x * all.share;
        u_end = min(u + all.share, all.total);
    }
    if constexpr (!FULL) {
        for (int i = threadIdx.x; i < 4 * BYTES / 16; i += T) reinterpret_cast<u32x4*>(smem)[i] = u32x4{};   // pieces past the head stay zero
        __syncthreads();
    }
    int from = 0;
    int64_t before = 0;
    while (by_item ? u >= 0 : u < u_end) {
        const Place pl = by_item ? place_of<ROWS, 0>(a, u, lane) : place_of<ROWS, STEP>(a, u, lane, from, before);
        from = pl.b;
        before = pl.first;
        const Sequence s = pl.s;
        const int64_t local = u - pl.first;
        const int item = (int)(local / pl.steps), step0 = (int)(local - (int64_t)item * pl.steps);
        const int step1 = by_item ? 1 : (int)min((int64_t)pl.steps, step0 + (u_end - u));
        const int rt = item / a.kv_heads, h = item - rt * a.kv_heads;
        const bool whole = by_item || (step0 == 0 && step1 == pl.steps);

        // ---- rows: this lane's, the wavefront's and the workgroup's -------------------
        const int rows = (int)min((int64_t)ROWS, (int64_t)s.n * a.group - (int64_t)rt * ROWS);
        const int wrow = wave * kManyRows, my = wrow + col;
        const bool live = my < rows;
        const uint32_t r = (uint32_t)rt * ROWS + my;
        const int tok = (int)divide(r, a.by_group), head = h * a.group + (int)(r - (uint32_t)tok * a.group);
        int lo = 0, hi = 0;
        if (live) seen_by(a, s, tok, lo, hi);
        auto bounds = [&](int r0, int r1, int& lo0, int& hi0, int& lo1, int& hi1) {    // of rows r0 .. r1 of the tile
            seen_by(a, s, (int)divide((uint32_t)rt * ROWS + r0, a.by_group), lo0, hi0);
            seen_by(a, s, (int)divide((uint32_t)rt * ROWS + r1, a.by_group), lo1, hi1);
        };
        int lo_min, hi_min, lo_max, hi_max, wlo_min = 0, whi_min = 0, wlo_max = 0, whi_max = 0;
        bounds(0, rows - 1, lo_min, hi_min, lo_max, hi_max);
        const bool works = wrow < rows;
        if (works) bounds(wrow, min(rows, wrow + kManyRows) - 1, wlo_min, whi_min, wlo_max, whi_max);
        const bool full_rows = wrow + kManyRows <= rows;

        bf16x8 qf[KF];
#pragma unroll
        for (int k = 0; k < KF; ++k) {
            u32x4 v{};
            if (live && (FULL || k * 16 + half * 8 < a.dim))
                v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q.p) + (s.q0 + tok) * a.q.token + (int64_t)head * a.q.head + k * 16 + half * 8);
            // scale < 0: that of -q; scale 0: scores of q = 0, NaN where it is not finite
            if (a.keep == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = ((v[i] & 0x7f80u) == 0x7f80u ? 0x7fc0u : 0u) | ((v[i] & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : 0u);
            }
            v ^= a.flip;
            qf[k] = __builtin_bit_cast(bf16x8, v);
        }
        f32x16 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
        float m = minus_inf(), l = 0.f;           // m: of the scores before their scale

        // ---- keys ---------------------------------------------------------------------
        const int base = s.begin & ~(kAlign - 1);
        int j0 = base + step0 * STEP;
        if (lo_min > j0) j0 += (lo_min - j0) / kManyTile * kManyTile;   // tiles that no row sees are skipped
        const int j_end = by_item ? hi_max : min(hi_max, base + step1 * STEP);
        const int last = hi_max - 1;
        const int32_t* table = a.step.table + (int64_t)pl.b * a.step.table_stride;
        const uint16_t* kp = static_cast<const uint16_t*>(a.cache.k) + (int64_t)h * a.cache.head;
        const uint16_t* vp = static_cast<const uint16_t*>(a.cache.v) + (int64_t)h * a.cache.head;
        // Rows that no row of the tile sees are read as the nearest that one does.
        int page[NI], in[NI];
        auto pages = [&](int j) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if constexpr (PG16) {
                    const int t0 = min(max(j + i * LR + wave * WR, lo_min & ~15), last & ~15) & ~15;
                    const int slot = (int)divide((uint32_t)t0, a.by_page);
                    page[i] = table[slot];
                    in[i] = min(max(j + i * LR + lrow, lo_min), last) - slot * a.cache.page_size;
                } else {
                    const int t = min(max(j + i * LR + lrow, lo_min), last);
                    const int slot = (int)divide((uint32_t)t, a.by_page);
                    page[i] = table[slot];
                    in[i] = t - slot * a.cache.page_size;
                }
            }
        };
        auto load = [&](int stage) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int row = i * LR + lrow;
                const int kc = (lpos ^ k_swizzle<DH>(row)) * 8, vc = (lpos ^ v_swizzle<DH>(row)) * 8;
                const uint32_t to = lds0 + stage * 2 * BYTES + (i * T + wave * 64) * 16;
                if constexpr (PG16) {
                    const int64_t at = (int64_t)min(max(__builtin_amdgcn_readfirstlane(page[i]), 0), a.cache.pages - 1) * a.cache.page;
                    const uint32_t off = (uint32_t)in[i] * (uint32_t)(a.cache.token * 2);
                    if (FULL || kc < a.dim) load_lds(to, kp + at, off + kc * 2);
                    if (FULL || vc < a.dim) load_lds(to + BYTES, vp + at, off + vc * 2);
                } else {
                    const int64_t at = (int64_t)min(max(page[i], 0), a.cache.pages - 1) * a.cache.page + (int64_t)in[i] * a.cache.token;
                    if (FULL || kc < a.dim) load_lds(to, kp + at + kc);
                    if (FULL || vc < a.dim) load_lds(to + BYTES, vp + at + vc);
                }
            }
        };
        if (j0 < j_end) {
            pages(j0);
            load(0);
            if (j0 + kManyTile < j_end) pages(j0 + kManyTile);
        }
        int stage = 0;
        for (; j0 < j_end; j0 += kManyTile, stage ^= 1) {
            wait_all_loads();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            if (j0 + kManyTile < j_end) {
                load(stage ^ 1);
                if (j0 + 2 * kManyTile < j_end) pages(j0 + 2 * kManyTile);
            }
            const unsigned char* kt = smem + stage * 2 * BYTES;
            unsigned char* vt = smem + stage * 2 * BYTES + BYTES;

            // a value that is not finite must not reach rows that do not see it, nor, by
            // the weight 0 of a key past the ends (which holds a seen one's value),
            // elements that are infinite
            bool bad = false;
            if (j0 < lo_max || j0 + kManyTile > hi_min) {
                bool mine = false;
                for (int i = threadIdx.x; i < BYTES / 16; i += T) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(vt + i * 16);
                    mine |= not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w);
                }
                bad = __syncthreads_or(mine);
            }
            const bool idle = !works || j0 >= whi_max || j0 + kManyTile <= wlo_min;
            if (idle && !bad) continue;

            f32x16 sc[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[x][v] = 0.f;
#pragma unroll
                for (int k = 0; k < KF; ++k) {
                    const int row = 32 * x + col;
                    const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + row * (DH * 2) + ((2 * k + half) ^ k_swizzle<DH>(row)) * 16);
                    sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[k], sc[x], 0, 0, 0);
                }
            }
            if (!full_rows || j0 < wlo_max || j0 + kManyTile > whi_min) {
                asm volatile("");      // a branch: most tiles need none of this
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int j = j0 + 32 * x + 8 * (v / 4) + 4 * half + v % 4;
                        sc[x][v] = j >= lo && j < hi ? sc[x][v] : minus_inf();
                    }
            }
            float top = minus_inf();
#pragma unroll
            for (int v = 0; v < 16; ++v) top = max3(top, sc[0][v], sc[1][v]);
            top = max_halves(top);
            // The maximum that a row's weights are relative to follows only when it is
            // left behind by 2^8: sums scaled by less than that lose nothing.
            const bool left = (top - m) * a.scale > 8.f;
            if (__any(left)) {
                const float keep = left ? exp2_((m - top) * a.scale) : 1.f;
                m = left ? top : m;
                l *= keep;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= keep;
            }
            const float zero = m == minus_inf() ? 0.f : m * a.scale;
            u32x4 pb[4];
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int v = 0; v < 16; v += 2) {
                    const float p = exp2_(fmaf(sc[x][v], a.scale, -zero)), q = exp2_(fmaf(sc[x][v + 1], a.scale, -zero));
                    sum[0] += p;
                    sum[1] += q;
                    pb[2 * x + v / 8][v / 2 % 4] = pack_bf16(p, q);
                }
            l += sum[0] + sum[1];
            if (bad) {
                // such values go to the rows that see them, key by key, and count as
                // zeros in the product
#pragma unroll 1
                for (int i = 0; i < kManyTile; ++i) {
                    // key i lies in half (i / 4) % 2, element 4 ((i / 8) % 2) + i % 4 of pb[i / 16]
                    uint32_t w = 0;
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int v = 0; v < 4; ++v) w = x == i >> 4 && v == (i >> 3 & 1) * 2 + (i >> 1 & 1) ? pb[x][v] : w;
                    w = __shfl(w, (i & 4) * 8 + col);
                    const float p = from_bf16(i & 1 ? w >> 16 : w & 0xffffu);
                    const bool sees = j0 + i >= lo && j0 + i < hi;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int e = 32 * d + 8 * v + 4 * half;
                            const uint16_t* q = reinterpret_cast<const uint16_t*>(vt + i * (DH * 2) + ((e / 8) ^ v_swizzle<DH>(i)) * 16) + e % 8;
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const float z = fmaf(p, from_bf16(q[y]), o[d][4 * v + y]);
                                o[d][4 * v + y] = sees && not_finite(q[y]) ? z : o[d][4 * v + y];
                            }
                        }
                }
                __syncthreads();
                for (int i = threadIdx.x; i < BYTES / 2; i += T) {
                    uint16_t* q = reinterpret_cast<uint16_t*>(vt) + i;
                    if (not_finite(*q)) *q = 0;
                }
                __syncthreads();
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    s16x8 vf;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int row = 16 * c + 8 * y + 4 * half + (lane & 15) / 4;
                        const int e = 32 * d + (lane & 16) + 4 * (lane & 3);
                        const unsigned char* q = vt + row * (DH * 2) + ((e / 8) ^ v_swizzle<DH>(row)) * 16 + (e % 8) * 2;
                        const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q);
#pragma unroll
                        for (int v = 0; v < 4; ++v) vf[4 * y + v] = t[v];
                    }
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pb[c]), o[d], 0, 0, 0);
                }
        }

        // ---- results: a lane holds 4 elements after another of its row -------------------
        l += __shfl_xor(l, 32);
        float top = m == minus_inf() ? m : m * a.scale;
        bool finish = whole;
        if (STEP != 0 && !whole) {
            // a part in the order of this kernel's registers, two floats of a lane at a
            // time beside those of its neighbours
            constexpr int F = kPartFloats<DH, ROWS>;
            const int64_t begin = pl.first + (int64_t)item * pl.steps;
            const Parts parts = parts_of(begin, begin + pl.steps, all.share);
            const int at = wave * kManyRows * DH + 2 * lane;
            finish = others_done(a, parts, &flag);
            if (!finish) {
                float* part = part_at<F>(a, parts, parts.mine);
                if (works) {
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int v = 0; v < 16; v += 2) put2(part + at + (d * 8 + v / 2) * 128, o[d][v], o[d][v + 1]);
                    if (half == 0) put2(part + ROWS * DH + 2 * my, top, l);
                }
                finish = last_to_arrive(a, parts, &flag);
            }
            if (finish) {
                if (works) {
                    // all parts in their order, this workgroup's from its registers
                    float most = top;
                    for (int i = 0; i < parts.count; ++i)
                        if (i != parts.mine) most = fmaxf(most, get2(part_at<F>(a, parts, i) + ROWS * DH + 2 * my).x);
                    const float z = most == minus_inf() ? 0.f : most;
                    float l_all = 0.f;
                    f32x16 o_all[DT];
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int v = 0; v < 16; ++v) o_all[d][v] = 0.f;
                    for (int i = 0; i < parts.count; ++i) {
                        const float* part = part_at<F>(a, parts, i);
                        if (i == parts.mine) {
                            const float f = exp2_(top - z);
                            l_all = fmaf(l, f, l_all);
#pragma unroll
                            for (int d = 0; d < DT; ++d)
#pragma unroll
                                for (int v = 0; v < 16; ++v) o_all[d][v] = fmaf(o[d][v], f, o_all[d][v]);
                        } else {
                            const float2 ml = get2(part + ROWS * DH + 2 * my);
                            const float f = exp2_(ml.x - z);
                            l_all = fmaf(ml.y, f, l_all);
#pragma unroll
                            for (int d = 0; d < DT; ++d)
#pragma unroll
                                for (int v = 0; v < 16; v += 2) {
                                    const float2 x = get2(part + at + (d * 8 + v / 2) * 128);
                                    o_all[d][v] = fmaf(x.x, f, o_all[d][v]);
                                    o_all[d][v + 1] = fmaf(x.y, f, o_all[d][v + 1]);
                                }
                        }
                    }
                    top = most;
                    l = l_all;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[d] = o_all[d];
                }
                joined(a, parts);
            }
        }
        if (finish && live) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float acc[4] = {o[d][4 * v], o[d][4 * v + 1], o[d][4 * v + 2], o[d][4 * v + 3]};
                    finish_row<4>(a, s.q0 + tok, head, 32 * d + 8 * v + 4 * half, acc, l, top);
                }
        }
        if constexpr (STEP == 0) return;
        __syncthreads();      // the tiles in shared memory are free
        u += by_item ? -(int64_t)gridDim.x : (int64_t)(step1 - step0);
    }
}

// ---- launches ------------------------------------------------------------------------------
Divisor divisor(uint32_t d)
{
    Divisor v;
    v.shift = 0;
    while ((1ull << v.shift) < d) ++v.shift;
    v.mul = (uint32_t)(((1ull << 32) * ((1ull << v.shift) - d)) / d + 1);
    return v;
}

// Whether 16 tokens from a multiple of 16 on lie in one page of less than 2 GB.
// Addressing them by the wavefront takes 64 single tokens over 8000 (pages of 64)
// from 178 to 173 us; a prompt of 8192 takes 599 either way.
bool in_halves(const AttendArgs& a)
{
    return a.cache.page_size % 16 == 0 && a.cache.token < INT32_MAX / 2 && a.cache.token * 2 * (int64_t)a.cache.page_size < INT32_MAX;
}

template <int DH>
hipError_t few(const AttendArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(kFewPerCu<DH> * a.cus));
    const bool pg16 = in_halves(a);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kFewThreads), 0, s, a);
        return hipGetLastError();
    };
    if (a.dim == DH) return pg16 ? launch(attend_few_kernel<DH, true, true>) : launch(attend_few_kernel<DH, false, true>);
    return pg16 ? launch(attend_few_kernel<DH, true, false>) : launch(attend_few_kernel<DH, false, false>);
}

// Wavefronts of a workgroup of the kernel for many rows, and its workgroups of a
// CU when items are shared.
template <int DH>
constexpr int kManyWaves = DH == 256 ? 4 : 8;
constexpr int kManyStep = 256;

template <int DH>
hipError_t many(const AttendArgs& a, hipStream_t s)
{
    constexpr int NW = kManyWaves<DH>, ROWS = NW * kManyRows;
    // no more items than this, whatever the sequences' lengths
    const int64_t items = ((a.tokens * a.group + ROWS - 1) / ROWS + a.step.seqs) * a.kv_heads;
    auto launch = [&](auto kernel, int64_t groups) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(NW * 64), 0, s, a);
        return hipGetLastError();
    };
    const bool pg16 = in_halves(a);
    // An item a workgroup where that makes two rounds at least, else a workgroup a CU
    // and shares of the steps (8 heads of keys of 128, a group of 4; 512 items of
    // chunks of 256 tokens over 4000: 349 us by items, 357 by shares; 1024: 639 and
    // 677; 128: 143 and 103; shares also keep a long context among short ones from
    // being one workgroup's).  A launch has fewer than 2^32 threads.
    if ((a.tokens * a.group / ROWS) * a.kv_heads >= 2 * a.cus && a.step.seqs <= kSearched && items * (NW * 64) <= (int64_t)UINT32_MAX) {
        if (a.dim == DH) return pg16 ? launch(attend_many_kernel<DH, NW, 0, true, true>, items) : launch(attend_many_kernel<DH, NW, 0, false, true>, items);
        return pg16 ? launch(attend_many_kernel<DH, NW, 0, true, false>, items) : launch(attend_many_kernel<DH, NW, 0, false, false>, items);
    }
    if (a.dim == DH)
        return pg16 ? launch(attend_many_kernel<DH, NW, kManyStep, true, true>, a.cus) : launch(attend_many_kernel<DH, NW, kManyStep, false, true>, a.cus);
    return pg16 ? launch(attend_many_kernel<DH, NW, kManyStep, true, false>, a.cus) : launch(attend_many_kernel<DH, NW, kManyStep, false, false>, a.cus);
}

template <int DH>
constexpr size_t kGroupFloats = 2 * std::max(kFewPerCu<DH> * kPartFloats<DH, kRows>, kPartFloats<DH, kManyWaves<DH> * kManyRows>);

template <int DH>
hipError_t attend(const AttendArgs& args, hipStream_t s)
{
    AttendArgs a = args;
    // By the rows of a sequence and key head, on average (28 and 4 heads of 128, 16
    // contexts of 8000): 28 rows take 98 us as few and 121 as many, 35 rows 137 and
    // 125; 64 contexts of 2000: 88 and 92, 132 and 95.
    if (a.tokens * a.group <= 32 * (int64_t)a.step.seqs) {
        a.scale = a.raw_scale * kLog2e;
        return few<DH>(a, s);
    }
    a.scale = fabsf(a.raw_scale) * kLog2e;
    a.flip = a.raw_scale < 0.f ? 0x80008000u : 0u;
    a.keep = a.scale > 0.f ? ~0u : 0u;
    if (!a.keep) a.scale = 1.f;
    return many<DH>(a, s);
}

}  // namespace

size_t attend_groups(int cus) { return (size_t)std::max({kFewPerCu<64>, kFewPerCu<128>, kFewPerCu<256>, 1}) * cus; }

size_t attend_part_floats(int dim, int cus)
{
    return (size_t)cus * (dim <= 64 ? kGroupFloats<64> : dim <= 128 ? kGroupFloats<128> : kGroupFloats<256>);
}

hipError_t launch_attend(const AttendArgs& args, hipStream_t s)
{
    AttendArgs a = args;
    a.group = a.heads / a.kv_heads;
    a.by_group = divisor((uint32_t)a.group);
    a.by_page = divisor((uint32_t)a.cache.page_size);
    a.most = (int32_t)std::min((int64_t)a.step.table_width * a.cache.page_size, (int64_t)INT32_MAX - 4096);
    return a.dim <= 64 ? attend<64>(a, s) : a.dim <= 128 ? attend<128>(a, s) : attend<256>(a, s);
}

}  // namespace tr
