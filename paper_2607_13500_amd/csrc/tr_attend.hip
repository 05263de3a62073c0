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
// unrounded): its operands have one type, and V is bf16.
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

// A value that is the same in all lanes, as a scalar.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
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
// workgroup's share can end inside an item, and then the item's parts are joined
// by join_kernel.  A workgroup's four wavefronts take tiles of 32 keys in turn,
// each with its own maximum and sums, and join them at the end of an item.
//
// Bound by the bytes of the cache: a wavefront has the next tile's keys and
// values in flight, in registers, while it works on one; 16 rows cost two
// matrix instructions of 16 cycles per 16 x 32 elements of keys.
constexpr int kRows = 16, kTile = 32, kStep = 128, kFewThreads = 256;

// Where a workgroup is in the row of all steps.
struct Place {
    int b;             // sequence
    Sequence s;
    int steps;         // of an item of it
    int tiles;         // of rows
    int64_t first;     // its first step in the row
};

__device__ __forceinline__ int steps_of(const Sequence& s)
{
    return max(1, (s.end - (s.begin & ~(kTile - 1)) + kStep - 1) / kStep);
}

__device__ __forceinline__ int64_t cost_of(const AttendArgs& a, int b)
{
    if (b >= a.step.seqs) return 0;
    const Sequence s = sequence_at(a, b);
    const int64_t tiles = ((int64_t)s.n * a.group + kRows - 1) / kRows;
    return tiles * steps_of(s) * a.kv_heads;
}

__device__ __forceinline__ int64_t wave_sum_i64(int64_t x)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    return x;
}

__device__ __forceinline__ int64_t all_steps(const AttendArgs& a, int lane)
{
    int64_t sum = 0;
    for (int b0 = 0; b0 < a.step.seqs; b0 += 64) sum += cost_of(a, b0 + lane);
    return uniform(wave_sum_i64(sum));
}

// The sequence that step u (< all_steps) lies in.
__device__ __forceinline__ Place place_of(const AttendArgs& a, int64_t u, int lane)
{
    Place p{};
    int64_t before = 0;
    for (int b0 = 0; b0 < a.step.seqs; b0 += 64) {
        const int64_t c = cost_of(a, b0 + lane);
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
    p.steps = steps_of(p.s);
    p.tiles = (int)(((int64_t)p.s.n * a.group + kRows - 1) / kRows);
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

// Floats of one part in the scratch: 16 rows of DH sums, their maxima and l.
template <int DH>
constexpr int kPartFloats = kRows * DH + 2 * kRows;

// Address swizzle of a row of V in shared memory, in pieces of 16 bytes: the 16
// rows that a transposing read touches spread over all banks.
template <int DH>
__device__ __forceinline__ int v_piece(int row, int piece)
{
    return piece ^ ((DH == 64 ? (row >> 1) & 3 : row & 7) << 1);
}

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
    constexpr int kLds = 4 * (kTile * DH * 2 > kRows * PAD * 4 ? kTile * DH * 2 : kRows * PAD * 4);
    __shared__ __align__(16) unsigned char smem[kLds];
    __shared__ float ml[4][2][kRows];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int vrow = lane / PIECES, piece = lane % PIECES;
    unsigned char* vt = smem + wave * (kTile * DH * 2);
    const int token_bytes = (int)(a.cache.token * 2);            // PG16
    const int k_lane = col * token_bytes + grp * 16, v_lane = vrow * token_bytes + piece * 16;

    const int64_t total = all_steps(a, lane);
    const int64_t share = max((int64_t)a.least, (total + gridDim.x - 1) / gridDim.x);
    int64_t u = (int64_t)blockIdx.x * share;
    const int64_t u_end = min(u + share, total);

    while (u < u_end) {
        const Place pl = place_of(a, u, lane);
        const Sequence s = pl.s;
        const int64_t local = u - pl.first;
        const int item = (int)(local / pl.steps), step0 = (int)(local - (int64_t)item * pl.steps);
        const int step1 = (int)min((int64_t)pl.steps, step0 + (u_end - u));
        const int h = item / pl.tiles, rt = item - h * pl.tiles;
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
        u32x4 kr[2][KF], vr[VN];
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
                    const char* kb = reinterpret_cast<const char*>(kp + off);
                    const char* vb = reinterpret_cast<const char*>(vp + off);
#pragma unroll
                    for (int k = 0; k < KF; ++k)
                        if (FULL || k * 32 + grp * 8 < a.dim) kr[x][k] = *reinterpret_cast<const u32x4*>(kb + k_lane + k * 64);
#pragma unroll
                    for (int i = 0; i < VN / 2; ++i)
                        if (FULL || piece * 8 < a.dim)
                            vr[x * (VN / 2) + i] = *reinterpret_cast<const u32x4*>(vb + i * VR * token_bytes + v_lane);
                }
            } else {
                int64_t koff[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int t = min(max(j + 16 * x + col, lo_min), last);
                    const int slot = (int)divide((uint32_t)t, a.by_page);
                    koff[x] = (int64_t)page_at(slot) * a.cache.page + (int64_t)(t - slot * a.cache.page_size) * a.cache.token;
#pragma unroll
                    for (int k = 0; k < KF; ++k)
                        if (FULL || k * 32 + grp * 8 < a.dim) kr[x][k] = *reinterpret_cast<const u32x4*>(kp + koff[x] + k * 32 + grp * 8);
                }
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    const int64_t off = __shfl(koff[VR * i / 16], (VR * i + vrow) & 15) + piece * 8;
                    if (FULL || piece * 8 < a.dim) vr[i] = *reinterpret_cast<const u32x4*>(vp + off);
                }
            }
        };
        if constexpr (!FULL) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int k = 0; k < KF; ++k) kr[x][k] = u32x4{};   // pieces past the head stay zero
        }
        if (j0 < j_end) fetch(j0);
        for (; j0 < j_end; j0 += kStep) {
            f32x4 sc[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                sc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KF; ++k)
                    sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[x][k]), qf[k], sc[x], 0, 0, 0);
            }
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
                *reinterpret_cast<u32x4*>(vt + (VR * i + vrow) * (DH * 2) + v_piece<DH>(VR * i + vrow, piece) * 16) = vr[i];
            if (j0 + kStep < j_end) fetch(j0 + kStep);

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
            const float keep = exp2_(m - zero);
            m = m1;
            l *= keep;
            s16x8 pb;
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                p[v] = exp2_(p[v] - zero);
                l += p[v];
                pb[v] = (short)to_bf16(p[v]);
            }
            if (!__all(keep == 1.f)) {
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= keep;
            }
            // ---- values ---------------------------------------------------------------
            if (__any(bad)) {
                // values that are not finite go to the rows that see them, key by
                // key, and count as zeros in the product
#pragma unroll 1
                for (int i = 0; i < kTile; ++i) {
                    const uint32_t w01 = i & 1 ? (uint16_t)pb[1] : (uint16_t)pb[0], w23 = i & 1 ? (uint16_t)pb[3] : (uint16_t)pb[2];
                    const uint32_t w45 = i & 1 ? (uint16_t)pb[5] : (uint16_t)pb[4], w67 = i & 1 ? (uint16_t)pb[7] : (uint16_t)pb[6];
                    const float w = from_bf16(__shfl(i & 16 ? (i & 2 ? w67 : w45) : (i & 2 ? w23 : w01), (i & 12) * 4 + col));
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
            if (row < rows) {
                if (whole) {
                    const uint32_t rr = (uint32_t)(rt * kRows + row);
                    const int t = (int)divide(rr, a.by_group), hd = h * a.group + (int)(rr - (uint32_t)t * a.group);
                    finish_row<N>(a, s.q0 + t, hd, e0, acc, sum, top);
                } else {
                    float* part = a.part + ((int64_t)blockIdx.x * 2 + (step0 == 0)) * kPartFloats<DH>;
#pragma unroll
                    for (int e = 0; e < N; ++e) part[row * DH + e0 + e] = acc[e];
                    if (e0 == 0) {
                        part[kRows * DH + row] = top;
                        part[kRows * DH + kRows + row] = sum;
                    }
                }
            }
        }
        __syncthreads();
        u += step1 - step0;
    }
}

// Joins the parts of each item that several workgroups worked on: workgroup i
// does the item that began in attend_few_kernel's workgroup i and went on past
// it, whose later parts are the first ones of the workgroups after i.  One
// wavefront a row.
template <int DH>
__global__ __launch_bounds__(1024) void join_kernel(AttendArgs a)
{
    constexpr int N = DH / 64;
    const int lane = threadIdx.x & 63, row = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t total = all_steps(a, lane);
    const int64_t share = max((int64_t)a.least, (total + gridDim.x - 1) / gridDim.x);
    const int64_t u0 = (int64_t)blockIdx.x * share, u1 = u0 + share;
    if (u1 >= total) return;                          // nothing goes on past the last share
    const Place pl = place_of(a, u1 - 1, lane);
    const int64_t local = u1 - 1 - pl.first;
    const int item = (int)(local / pl.steps);
    const int64_t begin = pl.first + (int64_t)item * pl.steps, end = begin + pl.steps;
    if (begin < u0 || end <= u1) return;              // not begun here, or done here
    const int h = item / pl.tiles, rt = item - h * pl.tiles;
    const int rows = (int)min((int64_t)kRows, (int64_t)pl.s.n * a.group - (int64_t)rt * kRows);
    if (row >= rows) return;
    const int parts = (int)((end - 1) / share - (int64_t)blockIdx.x) + 1;
    // part 0 is this workgroup's second, the others are the first of theirs
    auto part = [&](int i) { return a.part + (((int64_t)blockIdx.x + i) * 2 + (i == 0)) * kPartFloats<DH>; };
    float top = minus_inf();
    for (int i = lane; i < parts; i += 64) top = fmaxf(top, part(i)[kRows * DH + row]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float zero = top == minus_inf() ? 0.f : top;
    float sum = 0.f, acc[N] = {};
    for (int i = 0; i < parts; ++i) {
        const float* p = part(i);
        const float f = exp2_(p[kRows * DH + row] - zero);
        sum = fmaf(p[kRows * DH + kRows + row], f, sum);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = fmaf(p[row * DH + lane * N + e], f, acc[e]);
    }
    const uint32_t r = (uint32_t)(rt * kRows + row);
    const int t = (int)divide(r, a.by_group), head = h * a.group + (int)(r - (uint32_t)t * a.group);
    // a lane's N elements as two or more: neighbours' are fetched where N is 1
    if constexpr (N == 1) {
        const float next = __shfl_down(acc[0], 1);
        const float two[2] = {acc[0], next};
        if ((lane & 1) == 0) finish_row<2>(a, pl.s.q0 + t, head, lane, two, sum, top);
    } else {
        finish_row<N>(a, pl.s.q0 + t, head, lane * N, acc, sum, top);
    }
}

Divisor divisor(uint32_t d)
{
    Divisor v;
    v.shift = 0;
    while ((1ull << v.shift) < d) ++v.shift;
    v.mul = (uint32_t)(((1ull << 32) * ((1ull << v.shift) - d)) / d + 1);
    return v;
}

template <int DH>
hipError_t few(const AttendArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(kFewPerCu<DH> * a.cus));
    const bool pg16 = a.cache.page_size % 16 == 0 && a.cache.token * 2 * (int64_t)a.cache.page_size < INT32_MAX;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kFewThreads), 0, s, a);
        return hipGetLastError();
    };
    hipError_t e = a.dim == DH ? (pg16 ? launch(attend_few_kernel<DH, true, true>) : launch(attend_few_kernel<DH, false, true>))
                               : (pg16 ? launch(attend_few_kernel<DH, true, false>) : launch(attend_few_kernel<DH, false, false>));
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(join_kernel<DH>, grid, dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace

size_t attend_part_floats(int dim, int cus)
{
    const size_t groups = (size_t)2 * cus;            // two parts for each workgroup of a CU
    return groups * (dim <= 64 ? kFewPerCu<64> * kPartFloats<64> : dim <= 128 ? kFewPerCu<128> * kPartFloats<128>
                                                                           : kFewPerCu<256> * kPartFloats<256>);
}

hipError_t launch_attend(const AttendArgs& args, hipStream_t s)
{
    AttendArgs a = args;
    a.group = a.heads / a.kv_heads;
    a.by_group = divisor((uint32_t)a.group);
    a.by_page = divisor((uint32_t)a.cache.page_size);
    a.most = (int32_t)std::min((int64_t)a.step.table_width * a.cache.page_size, (int64_t)INT32_MAX - 4096);
    a.scale *= kLog2e;
    a.least = 1;
    return a.dim <= 64 ? few<64>(a, s) : a.dim <= 128 ? few<128>(a, s) : few<256>(a, s);
}

}  // namespace tr
