// Attention of packed new tokens over a paged cache of 8-bit values with a scale for
// each block of tokens and key head:
//   out = sum_j softmax_j(scale ks_j q . k8_j) vs_j v8_j  over the tokens j that a row sees,
// in one pass over the keys with a running maximum and sum, both products transposed
// (tr_attend.hip).
//
// An e4m3 value is a bf16 value, so keys and values are widened without loss, two by
// one instruction, and the products are bf16's.  Their scales never touch them: a
// key's multiplies its scores, together with the softmax's scale, and a value's its
// weights, in fp32, before these are rounded to bf16.
#include <algorithm>

#include "tr_attend_work.h"

namespace tr {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// Eight e4m3 values as bf16.
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    struct {
        bf16x2 v[4];
    } r;
    r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false);
    r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false);
    r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return __builtin_bit_cast(bf16x8, r);
}

// Whether a word holds an e4m3 that is NaN (there are no infinities).
__device__ __forceinline__ bool has_nan8(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }
__device__ __forceinline__ bool is_nan8(uint8_t v) { return (v & 0x7f) == 0x7f; }

// Where the 16 bytes `piece` of a row lie in shared memory: the rows that one read
// touches (16 of keys, 32 of values) spread over all banks.
template <int DH>
__device__ __forceinline__ int piece8(int row, int piece)
{
    return piece ^ (DH == 64 ? (row >> 1) & 3 : row & 7);
}

// ---- few rows over many keys -----------------------------------------------------------
// Items are RT tiles of 16 rows, steps kStep keys; the four wavefronts take tiles of 32
// keys in turn, as in the bf16 kernel, and what is widened of a tile serves all its rows.
constexpr int kTile = 32, kStep = 128;

template <int DH, int RT>
constexpr int kFewPerCu8 = DH == 256 ? 1 : RT == 4 ? 1 : 2;

// PG16: pages and blocks of whole halves of a tile (multiples of 16 tokens, pages below
// 2 GB), so that a half's page and scales are the wavefront's.  FULL: head_dim is DH.
template <int DH, int RT, bool PG16, bool FULL>
__global__ __launch_bounds__(kFewThreads, (kFewPerCu8<DH, RT>)) void attend8_few_kernel(Attend8Args a)
{
    constexpr int ROWS = 16 * RT;
    constexpr int KF = DH / 32, DT = DH / 16;          // fragments of keys, tiles of elements
    constexpr int PIECES = DH / 16, VR = 64 / PIECES, VN = kTile / VR;   // pieces of a row, rows of a load, loads of a tile
    constexpr int PAD = DH + 4;
    constexpr int BYTES = kTile * DH;
    constexpr int kLds = 4 * std::max(2 * BYTES, 16 * PAD * 4);
    __shared__ __align__(16) unsigned char smem[kLds];
    __shared__ float ml[4][2][16];
    __shared__ int flag;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int vrow = lane / PIECES, piece = lane % PIECES;
    unsigned char* kt = smem + wave * 2 * BYTES;                 // the wavefront's tile
    unsigned char* vt = kt + BYTES;
    const int token_bytes = (int)a.cache8.token;                 // PG16
    const int in_lane = vrow * token_bytes + piece * 16;

    const Shares all = shares_of<ROWS, kStep>(a, lane);
    int64_t u = (int64_t)blockIdx.x * all.share;
    const int64_t u_end = min(u + all.share, all.total);

    int from = 0;
    int64_t before = 0;
    while (u < u_end) {
        const Place pl = place_of<ROWS, kStep>(a, u, lane, from, before);
        from = pl.b;
        before = pl.first;
        const Sequence s = pl.s;
        const int64_t local = u - pl.first;
        const int item = (int)(local / pl.steps), step0 = (int)(local - (int64_t)item * pl.steps);
        const int step1 = (int)min((int64_t)pl.steps, step0 + (u_end - u));
        const int rt = item / a.kv_heads, h = item - rt * a.kv_heads;
        const bool whole = step0 == 0 && step1 == pl.steps;

        // ---- this lane's rows, one of each tile ---------------------------------------
        const int rows = (int)min((int64_t)ROWS, (int64_t)s.n * a.group - (int64_t)rt * ROWS);
        int lo[RT], hi[RT];
        bf16x8 qf[RT][KF];
        f32x4 o[RT][DT];
        float m[RT], l[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const uint32_t r = (uint32_t)(rt * ROWS + 16 * i + col);
            const int tok = (int)divide(r, a.by_group), head = h * a.group + (int)(r - (uint32_t)tok * a.group);
            const bool live = 16 * i + col < rows;
            lo[i] = hi[i] = 0;
            if (live) seen_by(a, s, tok, lo[i], hi[i]);
            // elements in the order in which widened keys have them: 16 of a lane's group
            // after another, 8 to a fragment
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                const int e = (k / 2) * 64 + grp * 16 + (k % 2) * 8;
                u32x4 v{};
                if (live && e < a.dim)
                    v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q.p) + (s.q0 + tok) * a.q.token + (int64_t)head * a.q.head + e);
                qf[i][k] = __builtin_bit_cast(bf16x8, v);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) o[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[i] = minus_inf();
            l[i] = 0.f;
        }
        int lo_min, lo_max, hi_min, hi_max;       // over all rows
        {
            const int t0 = (int)divide((uint32_t)rt * ROWS, a.by_group), t1 = (int)divide((uint32_t)(rt * ROWS + rows - 1), a.by_group);
            seen_by(a, s, t0, lo_min, hi_min);
            seen_by(a, s, t1, lo_max, hi_max);
        }

        // ---- keys -------------------------------------------------------------------
        const int base = s.begin & ~(kTile - 1);
        const int j_end = min(hi_max, base + step1 * kStep);
        const int first = base + step0 * kStep + wave * kTile;
        // tiles before any row's range are skipped
        int j0 = first;
        if (j0 + kTile <= lo_min) j0 += ((lo_min - j0) / kStep) * kStep;
        if (j0 + kTile <= lo_min) j0 += kStep;
        const int32_t* table = a.step.table + (int64_t)pl.b * a.step.table_stride;
        const uint8_t* kp = static_cast<const uint8_t*>(a.cache8.k) + (int64_t)h * a.cache8.head;
        const uint8_t* vp = static_cast<const uint8_t*>(a.cache8.v) + (int64_t)h * a.cache8.head;
        const float* ksp = a.cache8.k_scale + (int64_t)h * a.cache8.scale_head;
        const float* vsp = a.cache8.v_scale + (int64_t)h * a.cache8.scale_head;
        const int last = hi_max - 1;              // tokens past it (and before lo_min) are read as it (as lo_min)

        auto page_at = [&](int slot) { return min(max(table[slot], 0), a.cache8.pages - 1); };
        u32x4 kr[VN], vr[VN];
        float ks[2], vs[2];                       // PG16: of the tile's halves, else of this lane's token of each
        auto fetch = [&](int j) {
            if constexpr (PG16) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    // rows of a half that no row sees are read all the same (they are in
                    // the page), a half without any in the place of the nearest one
                    const int half = min(max(j + 16 * x, lo_min & ~15), last & ~15);
                    const int slot = (int)divide((uint32_t)half, a.by_page), in = half - slot * a.cache8.page_size;
                    const int page = __builtin_amdgcn_readfirstlane(page_at(slot));
                    const int64_t off = uniform((int64_t)page * a.cache8.page + (int64_t)in * a.cache8.token);
                    const int64_t scale = uniform((int64_t)page * a.cache8.scale_page + (int64_t)divide((uint32_t)in, a.by_block) * a.cache8.scale_block);
                    ks[x] = ksp[scale];
                    vs[x] = vsp[scale];
                    const unsigned char* kb = kp + off + in_lane;
                    const unsigned char* vb = vp + off + in_lane;
                    constexpr int HALF = VN >= 2 ? VN / 2 : 1;
#pragma unroll
                    for (int i = 0; i < HALF; ++i)
                        if (FULL || piece * 16 < a.dim) {
                            kr[x * HALF + i] = read_once(kb + i * VR * token_bytes);
                            vr[x * HALF + i] = read_once(vb + i * VR * token_bytes);
                        }
                }
            } else {
                int64_t koff[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int t = min(max(j + 16 * x + col, lo_min), last);
                    const int slot = (int)divide((uint32_t)t, a.by_page), in = t - slot * a.cache8.page_size, page = page_at(slot);
                    koff[x] = (int64_t)page * a.cache8.page + (int64_t)in * a.cache8.token;
                    const int64_t scale = (int64_t)page * a.cache8.scale_page + (int64_t)divide((uint32_t)in, a.by_block) * a.cache8.scale_block;
                    ks[x] = ksp[scale];
                    vs[x] = vsp[scale];
                }
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    const int64_t off = __shfl(koff[VR * i / 16], (VR * i + vrow) & 15) + piece * 16;
                    if (FULL || piece * 16 < a.dim) {
                        kr[i] = read_once(kp + off);
                        vr[i] = read_once(vp + off);
                    }
                }
            }
        };
        if constexpr (!FULL) {
#pragma unroll
            for (int i = 0; i < VN; ++i) kr[i] = vr[i] = u32x4{};   // pieces past the head stay zero
        }
        if (j0 < j_end) fetch(j0);
        for (; j0 < j_end; j0 += kStep) {
            // rows that see different tokens of this tile: a NaN must not reach the rows
            // that do not see it
            const bool mixed = lo_max > max(j0, lo_min) || hi_min < min(j0 + kTile, hi_max);
            // nor one that no row sees
            if (j0 < lo_min || j0 + kTile > hi_max) {
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    const int t = j0 + VR * i + vrow;
                    if (t < lo_min || t > last) vr[i] = u32x4{};
                }
            }
            bool bad = false;
            if (mixed) {
#pragma unroll
                for (int i = 0; i < VN; ++i) bad |= has_nan8(vr[i].x) || has_nan8(vr[i].y) || has_nan8(vr[i].z) || has_nan8(vr[i].w);
            }
#pragma unroll
            for (int i = 0; i < VN; ++i) {
                const int row = VR * i + vrow;
                *reinterpret_cast<u32x4*>(kt + row * DH + piece8<DH>(row, piece) * 16) = kr[i];
                *reinterpret_cast<u32x4*>(vt + row * DH + piece8<DH>(row, piece) * 16) = vr[i];
            }
            const float ks0[2] = {ks[0], ks[1]}, vs0[2] = {vs[0], vs[1]};
            if (j0 + kStep < j_end) fetch(j0 + kStep);
            f32x4 sc[RT][2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int i = 0; i < RT; ++i) sc[i][x] = f32x4{0.f, 0.f, 0.f, 0.f};
                const int row = 16 * x + col;
#pragma unroll
                for (int k = 0; k < KF; k += 2) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(kt + row * DH + piece8<DH>(row, 2 * k + grp) * 16);
                    const bf16x8 k0 = widen8(w.x, w.y), k1 = widen8(w.z, w.w);
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        sc[i][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[i][k], sc[i][x], 0, 0, 0);
                        sc[i][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[i][k + 1], sc[i][x], 0, 0, 0);
                    }
                }
            }

            // ---- weights ------------------------------------------------------------
            float kf[8], vf[8];                   // scales of this lane's keys
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    kf[4 * x + v] = (PG16 ? ks0[x] : __shfl(ks0[x], 4 * grp + v)) * a.scale;
                    vf[4 * x + v] = PG16 ? vs0[x] : __shfl(vs0[x], 4 * grp + v);
                }
            u32x4 pb[RT];
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float p[8];
                float top = minus_inf();
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int j = j0 + 16 * x + 4 * grp + v;
                        const float y = sc[i][x][v] * kf[4 * x + v];
                        p[4 * x + v] = j >= lo[i] && j < hi[i] ? y : minus_inf();
                        top = fmaxf(top, p[4 * x + v]);
                    }
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float m1 = fmaxf(m[i], top), zero = m1 == minus_inf() ? 0.f : m1;
                const bool same = m1 == m[i];             // rows that see nothing yet among them
                const float keep = exp2_(m[i] - zero);
                m[i] = m1;
                l[i] *= keep;
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    p[v] = exp2_(p[v] - zero);
                    l[i] += p[v];
                    p[v] = p[v] == 0.f ? 0.f : p[v] * vf[v];      // a token that is not seen may have any scale
                }
#pragma unroll
                for (int v = 0; v < 4; ++v) pb[i][v] = pack_bf16(p[2 * v], p[2 * v + 1]);
                if (!__all(same)) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[i][d] *= keep;
                }
            }
            // ---- values ---------------------------------------------------------------
            if (__any(bad)) {
                // elements of rows that see a NaN are NaN, which counts as zero in the product
#pragma unroll 1
                for (int t = 0; t < kTile; ++t) {
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        const bool sees = j0 + t >= lo[i] && j0 + t < hi[i];
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const unsigned char* q = vt + t * DH + piece8<DH>(t, d) * 16 + 4 * grp;
#pragma unroll
                            for (int v = 0; v < 4; ++v) o[i][d][v] = sees && is_nan8(q[v]) ? __builtin_nanf("") : o[i][d][v];
                        }
                    }
                }
#pragma unroll 1
                for (int t = 0; t < kTile; ++t)
#pragma unroll 1
                    for (int e = lane; e < DH; e += 64)
                        if (is_nan8(vt[t * DH + e])) vt[t * DH + e] = 0;
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                // eight keys of an element to a lane: those of its weights
                const int n = (lane & 15) >> 1, row = 4 * grp + (n & 3) + 16 * (n >> 2);
                const unsigned char* q = vt + row * DH + piece8<DH>(row, d) * 16 + (lane & 1) * 8;
                const i32x2 t = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)q);
                const bf16x8 w = widen8((uint32_t)t.x, (uint32_t)t.y);
#pragma unroll
                for (int i = 0; i < RT; ++i)
                    o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, pb[i]), o[i][d], 0, 0, 0);
            }
        }

        // ---- the four wavefronts' parts, a tile of rows after another --------------------
        constexpr int F = kPartFloats<DH, ROWS>;
        constexpr int N = DH / 16;                // elements of a thread
        const int row = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * N;
        const int64_t begin = pl.first + (int64_t)item * pl.steps;
        const Parts parts = parts_of(begin, begin + pl.steps, all.share);
        float* red = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            l[i] += __shfl_xor(l[i], 16);
            l[i] += __shfl_xor(l[i], 32);
            __syncthreads();
#pragma unroll
            for (int d = 0; d < DT; ++d)
                *reinterpret_cast<f32x4*>(red + (wave * 16 + col) * PAD + 16 * d + 4 * grp) = o[i][d];
            if (grp == 0) {
                ml[wave][0][col] = m[i];
                ml[wave][1][col] = l[i];
            }
            __syncthreads();
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
                for (int e = 0; e < N; ++e) acc[e] = fmaf(red[(w * 16 + row) * PAD + e0 + e], f, acc[e]);
            }
            const int mine = 16 * i + row;        // of the item's rows
            if (mine >= rows) continue;
            if (whole) {
                const uint32_t r = (uint32_t)(rt * ROWS + mine);
                const int t = (int)divide(r, a.by_group);
                finish_row<N>(a, s.q0 + t, h * a.group + (int)(r - (uint32_t)t * a.group), e0, acc, sum, top);
            } else {
                float* part = part_at<F>(a, parts, parts.mine);
#pragma unroll
                for (int e = 0; e < N; e += 2) put2(part + mine * DH + e0 + e, acc[e], acc[e + 1]);
                if (e0 == 0) put2(part + ROWS * DH + 2 * mine, top, sum);
            }
        }
        if (!whole && last_to_arrive(a, parts, &flag)) {
            // all parts in their order, eight of them on their way at a time
            constexpr int U = N > 8 ? 4 : 8;
            for (int mine = row; mine < rows; mine += 16) {
                float top = minus_inf(), sum = 0.f, acc[N] = {};
                for (int i0 = 0; i0 < parts.count; i0 += U) {
                    float2 ml_i[U], v[U][N / 2];
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        const float* q = part_at<F>(a, parts, min(i0 + i, parts.count - 1));
                        ml_i[i] = get2(q + ROWS * DH + 2 * mine);
#pragma unroll
                        for (int e = 0; e < N; e += 2) v[i][e / 2] = get2(q + mine * DH + e0 + e);
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
                const uint32_t r = (uint32_t)(rt * ROWS + mine);
                const int t = (int)divide(r, a.by_group);
                finish_row<N>(a, s.q0 + t, h * a.group + (int)(r - (uint32_t)t * a.group), e0, acc, sum, top);
            }
            joined(a, parts);
        }
        __syncthreads();
        u += step1 - step0;
    }
}

// ---- launches ------------------------------------------------------------------------------
// Whether 16 tokens from a multiple of 16 on lie in one page and block, a page below 2 GB.
bool in_halves(const Attend8Args& a)
{
    return a.cache8.page_size % 16 == 0 && a.cache8.block % 16 == 0 && a.cache8.token < INT32_MAX &&
           a.cache8.token * (int64_t)a.cache8.page_size < INT32_MAX;
}

template <int DH, int RT>
hipError_t few(const Attend8Args& a, hipStream_t s)
{
    const dim3 grid((unsigned)(kFewPerCu8<DH, RT> * a.cus));
    const bool pg16 = in_halves(a);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kFewThreads), 0, s, a);
        return hipGetLastError();
    };
    if (a.dim == DH) return pg16 ? launch(attend8_few_kernel<DH, RT, true, true>) : launch(attend8_few_kernel<DH, RT, false, true>);
    return pg16 ? launch(attend8_few_kernel<DH, RT, true, false>) : launch(attend8_few_kernel<DH, RT, false, false>);
}

template <int DH>
hipError_t attend8(const Attend8Args& args, hipStream_t s)
{
    Attend8Args a = args;
    a.scale = a.raw_scale * kLog2e;
    const int64_t rows = a.tokens * a.group;
    if (rows <= 16 * (int64_t)a.step.seqs) return few<DH, 1>(a, s);
    return few<DH, DH == 256 ? 2 : 4>(a, s);
}

}  // namespace

hipError_t launch_attend8(const Attend8Args& args, hipStream_t s)
{
    Attend8Args a = args;
    a.group = a.heads / a.kv_heads;
    a.by_group = divisor((uint32_t)a.group);
    a.by_page = divisor((uint32_t)a.cache8.page_size);
    a.by_block = divisor((uint32_t)a.cache8.block);
    a.most = (int32_t)std::min((int64_t)a.step.table_width * a.cache8.page_size, (int64_t)INT32_MAX - 4096);
    return a.dim <= 64 ? attend8<64>(a, s) : a.dim <= 128 ? attend8<128>(a, s) : attend8<256>(a, s);
}

}  // namespace tr
