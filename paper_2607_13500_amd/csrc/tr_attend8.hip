// Attention of packed new tokens over a paged cache of 8-bit values with a scale for
// each block of tokens and key head:
//   out = sum_j softmax_j(scale ks_j q . k8_j) vs_j v8_j  over the tokens j that a row sees,
// in one pass over the keys with a running maximum and sum, both products transposed
// (tr_attend.hip).
//
// An e4m3 value is a bf16 value, so keys and values are widened without loss, two by
// one instruction, and the products are bf16's.  A key's scale multiplies its scores in
// fp32, together with the softmax's scale.  A value's goes into that widening where it is
// a power of two, not above kLargeScale, which is exact, and else multiplies its weights in
// fp32, before these are rounded to bf16.
#include <algorithm>
#include <type_traits>

#include "tr_attend_work.h"

namespace tr {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

__device__ __forceinline__ float lane_of(float x, int i) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), i)); }

__device__ __forceinline__ int64_t lane_of(int64_t x, int i)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, i));
}

// Eight e4m3 values as bf16, four and four times a power of two.
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float by_a = 1.f, float by_b = 1.f)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    struct {
        bf16x2 v[4];
    } r;
    r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, by_a, false);
    r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, by_a, true);
    r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, by_b, false);
    r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, by_b, true);
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

// Sums have up to 2^31 products of a weight, which is 2^8 at most, and a value: finite
// while values' scales are no larger than this (448 < 2^8.9).  Where a tile has a larger
// one its rows' weights, and so all that their sums hold, are relative to 2^kRaise times
// their largest, 2^-40 at most: products with scales of up to 2^128 and their sums are finite
// then too.  What the sums lose at their small end are values below 2^-70 beside such a scale.
constexpr float kLargeScale = 0x1p80f, kRaise = 48.f;

// Whether a scale is a power of two by which widening is exact (no value leaves bf16's
// normal range) and not a large one.
__device__ __forceinline__ bool is_power(float s)
{
    const uint32_t w = __float_as_uint(s);
    return (w & 0x807fffffu) == 0 && w - (10u << 23) <= (197u << 23);       // 2^-117 .. 2^80
}

// Queries whose scores are for scale > 0: of -q for scale < 0, of q = 0 for scale 0, NaN
// where it is not finite.
__device__ __forceinline__ bf16x8 signed_query(const AttendArgs& a, u32x4 v)
{
    if (a.keep == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = ((v[i] & 0x7f80u) == 0x7f80u ? 0x7fc0u : 0u) | ((v[i] & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : 0u);
    }
    return __builtin_bit_cast(bf16x8, v ^ a.flip);
}

// A factor of scores.  Those of keys that no row sees may be anything; 0 would make NaN
// of -inf, which the smallest normal number does not.
__device__ __forceinline__ float factor(float x) { return fmaxf(x, 0x1p-126f); }

// The largest over the four groups of 16 lanes.
__device__ __forceinline__ float max_groups(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = max3(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return max3(__uint_as_float(q[0]), __uint_as_float(q[1]), __uint_as_float(q[1]));
}

// ---- few rows over many keys -----------------------------------------------------------
// Items are RT tiles of 16 rows, in steps of kStep keys, and what is widened of a tile
// of keys serves all its rows.  A workgroup's four wavefronts either take tiles of kTile
// keys of one key head in turn and join their sums at an item's end (HW = 1), or have a key
// head each (HW = 4, items then are those of four heads), for heads of 64, whose rows are
// half a line of memory: read at the same time side by side they come faster (32
// requests with 2 to 8 tokens each 100 us instead of 148; 64 requests with one 139
// instead of 211; heads of 128 are no faster so).
//
// Bound by the bytes of the cache, in calls of single tokens by the latency of what
// waits for one another (lengths, table, keys, the join of parts).  A wavefront has the
// next tile's 8 KB on their way into registers while it works on one.  One workgroup
// of a CU reads as fast as several, and there are fewer parts to join (64 requests
// over 256 to 16384 tokens, 4 heads of 128: 109 us, 5.65 TB/s; 118 with two, 129 with
// three; with tiles of 64 keys 119).
template <int DH>
constexpr int kFewTile = DH == 64 ? 64 : 32;

// PG16: pages and blocks of whole halves of a tile (multiples of 16 tokens, pages below
// 2 GB), so that a half's page and scales are the wavefront's (pages of 40 in blocks of 8:
// the 64 requests 118 us, the 32 119).  FULL: head_dim is DH.
// kv_heads counts groups of HW heads here.
template <int DH, int HW, int RT, bool PG16, bool FULL>
__global__ __launch_bounds__(kFewThreads, 1) void attend8_few_kernel(Attend8Args a)
{
    constexpr int ROWS = 16 * RT, kTile = kFewTile<DH>, kStep = 4 / HW * kTile;
    constexpr int X = kTile / 16, C = kTile / 32;      // sixteens of keys and fragments of weights of a tile
    constexpr int KF = DH / 32, DT = DH / 16;          // fragments of keys, tiles of elements
    constexpr int PIECES = DH / 16, VR = 64 / PIECES, VN = kTile / VR;   // pieces of a row, rows of a load, loads of a tile
    constexpr int PAD = DH + 4;
    constexpr int BYTES = kTile * DH;
    constexpr int kLds = 4 * (HW == 1 ? std::max(2 * BYTES, 16 * PAD * 4) : 2 * BYTES);
    __shared__ __align__(16) unsigned char smem[kLds];
    [[maybe_unused]] __shared__ float ml[4][2][16];
    __shared__ int flag;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int vrow = lane / PIECES, piece = lane % PIECES;
    unsigned char* kt = smem + wave * 2 * BYTES;                 // the wavefront's tile
    unsigned char* vt = kt + BYTES;
    const int token_bytes = (int)a.cache8.token;                 // PG16
    const uint32_t in_lane = (uint32_t)(vrow * token_bytes + piece * 16);

    Place pl;
    const Shares all = first_place<ROWS, kStep, HW>(a, lane, pl);
    int64_t u = (int64_t)blockIdx.x * all.share;
    const int64_t u_end = min(u + all.share, all.total);

    for (bool first_item = true; u < u_end; first_item = false) {
        if (!first_item) pl = place_of<ROWS, kStep>(a, u, lane, pl.b, pl.first, all.extra);
        const Sequence s = pl.s;
        const int64_t local = u - pl.first;
        const int item = (int)(local / pl.steps), part0 = (int)(local - (int64_t)item * pl.steps);
        const int part1 = (int)min((int64_t)pl.steps, part0 + (u_end - u));
        const int step0 = max(0, part0 - all.extra), step1 = max(0, part1 - all.extra);
        const int rt = item / a.kv_heads, h = (item - rt * a.kv_heads) * HW + wave % HW;
        const bool whole = part0 == 0 && part1 == pl.steps;

        // ---- the rows' bounds: this lane's, one of each tile, and all rows' -----------
        const int rows = (int)min((int64_t)ROWS, (int64_t)s.n * a.group - (int64_t)rt * ROWS);     // of each head
        int lo[RT], hi[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            lo[i] = hi[i] = 0;
            if (16 * i + col < rows) seen_by(a, s, (int)divide((uint32_t)(rt * ROWS + 16 * i + col), a.by_group), lo[i], hi[i]);
        }
        int lo_min, lo_max, hi_min, hi_max;
        {
            const int t0 = (int)divide((uint32_t)rt * ROWS, a.by_group), t1 = (int)divide((uint32_t)(rt * ROWS + rows - 1), a.by_group);
            seen_by(a, s, t0, lo_min, hi_min);
            seen_by(a, s, t1, lo_max, hi_max);
        }

        // ---- keys -------------------------------------------------------------------
        const int base = s.begin & ~(kAlign - 1);
        const int j_end = min(hi_max, base + step1 * kStep);
        const int first = base + step0 * kStep + wave / HW * kTile;
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

        u32x4 kr[VN], vr[VN];
        // PG16: each lane looks up sixteen keys, all lanes those of the next BT tiles, of
        // which a tile's are the wavefront's when its turn comes.  Rows of a sixteen that no row
        // sees are read all the same (they are in the page), one without any in the
        // place of the nearest one.
        // Else a lane looks up a key of one tile, a tile ahead.
        constexpr int BT = 64 / X;
        int page = 0, in = 0, ahead = 0, at = 0;  // ahead: tiles that are looked up and not fetched; at: the fetched tile's first lane
        int64_t off = 0;
        float ks = 0.f, vs = 0.f;
        auto look = [&](int j) {
            const int t = PG16 ? min(max(j + (lane / X) * kStep + (lane % X) * 16, lo_min & ~15), last & ~15)
                               : min(max(j + (lane & (kTile - 1)), lo_min), last);
            const int slot = (int)divide((uint32_t)t, a.by_page);
            page = table[slot];
            in = t - slot * a.cache8.page_size;
        };
        auto find = [&] {
            const int g = min(max(page, 0), a.cache8.pages - 1);
            off = (int64_t)g * a.cache8.page + (int64_t)in * a.cache8.token;
            const int64_t scale = (int64_t)g * a.cache8.scale_page + (int64_t)divide((uint32_t)in, a.by_block) * a.cache8.scale_block;
            ks = ksp[scale];
            vs = vsp[scale];
        };
        auto fetch = [&](int j) {
            if constexpr (PG16) {
                if (ahead == 0) {
                    look(j);
                    find();
                    ahead = BT;
                }
                at = (BT - ahead) * X;
                --ahead;
                constexpr int EACH = VN / X;
#pragma unroll
                for (int x = 0; x < X; ++x) {
                    const int64_t o = lane_of(off, at + x);
#pragma unroll
                    for (int i = 0; i < EACH; ++i) {
                        const uint8_t* kb = kp + o + (int64_t)i * VR * token_bytes;      // the wavefront's
                        const uint8_t* vb = vp + o + (int64_t)i * VR * token_bytes;
                        if (FULL || piece * 16 < a.dim) {
                            kr[x * EACH + i] = read_once(kb + in_lane);
                            vr[x * EACH + i] = read_once(vb + in_lane);
                        }
                    }
                }
            } else {
                find();
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    const int64_t o = __shfl(off, VR * i + vrow) + piece * 16;
                    if (FULL || piece * 16 < a.dim) {
                        kr[i] = read_once(kp + o);
                        vr[i] = read_once(vp + o);
                    }
                }
                if (j + kStep < j_end) look(j + kStep);
            }
        };
        if constexpr (!FULL) {
#pragma unroll
            for (int i = 0; i < VN; ++i) kr[i] = vr[i] = u32x4{};   // pieces past the head stay zero
        }
        if (j0 < j_end) {
            if constexpr (!PG16) look(j0);
            fetch(j0);
        }

        bf16x8 qf[RT][KF];
        f32x4 o[RT][DT];
        float m[RT], l[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const uint32_t r = (uint32_t)(rt * ROWS + 16 * i + col);
            const int tok = (int)divide(r, a.by_group), head = h * a.group + (int)(r - (uint32_t)tok * a.group);
            // elements in the order in which widened keys have them: 16 of a lane's group
            // after another, 8 to a fragment
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                const int e = (k / 2) * 64 + grp * 16 + (k % 2) * 8;
                u32x4 v{};
                if (16 * i + col < rows && e < a.dim)
                    v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q.p) + (s.q0 + tok) * a.q.token + (int64_t)head * a.q.head + e);
                qf[i][k] = signed_query(a, v);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) o[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[i] = minus_inf();
            l[i] = 0.f;
        }
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
            // the tile's scales: of its sixteens, or of this lane's key
            float ks_tile[X], vs_tile[X];
#pragma unroll
            for (int x = 0; x < X; ++x) {
                ks_tile[x] = PG16 ? lane_of(ks, at + x) : 0.f;
                vs_tile[x] = PG16 ? lane_of(vs, at + x) : 0.f;
            }
            const float ks_lane = ks, vs_lane = vs;
            if (j0 + kStep < j_end) fetch(j0 + kStep);
            f32x4 sc[RT][X];
#pragma unroll
            for (int x = 0; x < X; ++x) {
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
            // Factors of the scores, of sixteen keys each (else in the scores already), and
            // the values' scales: powers of two are for the widening, others for the weights.
            float f[X];
            bool folded = PG16, large = !PG16 && __any(vs_lane > kLargeScale);
#pragma unroll
            for (int x = 0; x < X; ++x) {
                if constexpr (PG16) {
                    f[x] = factor(ks_tile[x] * a.scale);
                    folded = folded && is_power(vs_tile[x]);
                    large = large || vs_tile[x] > kLargeScale;
                } else {
                    f[x] = 1.f;
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float z = factor(__shfl(ks_lane, 16 * x + 4 * grp + v) * a.scale);
#pragma unroll
                        for (int i = 0; i < RT; ++i) sc[i][x][v] *= z;
                    }
                }
            }
            const bool edge = j0 < lo_max || j0 + kTile > hi_min;     // rows past the last are nobody's
            // No branch lies between a matrix instruction and a reader of its result, but for
            // those that skip what all of a tile's rows would do: where several ways lead to a
            // reader the compiler did not count its wait on all of them
            // (tests/test_matrix_waits.py walks all of the built kernels' ways).
            u32x4 pb[RT][C];
            float top[RT];
            bool left[RT], any = false;
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                if (edge) {
                    asm volatile("");      // a branch: most tiles need none of this
#pragma unroll
                    for (int x = 0; x < X; ++x)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int j = j0 + 16 * x + 4 * grp + v;
                            sc[i][x][v] = j >= lo[i] && j < hi[i] ? sc[i][x][v] : minus_inf();
                        }
                }
                top[i] = minus_inf();
#pragma unroll
                for (int x = 0; x < X; ++x) {
                    const f32x4 z = sc[i][x];
                    const float t = max3(z[0], z[1], max3(z[2], z[3], z[3]));
                    top[i] = max3(top[i], t * f[x], top[i]);
                }
                top[i] = max_groups(top[i]) + (large ? kRaise : 0.f);
                // The maximum that a row's weights are relative to follows only when it is
                // left behind by 2^8: sums scaled by less than that lose nothing.
                left[i] = top[i] - m[i] > 8.f;
                any = any || left[i];
            }
            if (__any(any)) {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const float keep = left[i] ? exp2_(m[i] - top[i]) : 1.f;
                    m[i] = left[i] ? top[i] : m[i];
                    l[i] *= keep;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[i][d] *= keep;
                }
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const float zero = m[i] == minus_inf() ? 0.f : m[i];
                float p[4 * X], sum = 0.f;
#pragma unroll
                for (int x = 0; x < X; ++x)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        p[4 * x + v] = exp2_(fmaf(sc[i][x][v], f[x], -zero));
                        sum += p[4 * x + v];
                    }
                l[i] += sum;
                if (!folded) {
#pragma unroll
                    for (int x = 0; x < X; ++x)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            // a token that is not seen may have any scale
                            const float z = PG16 ? vs_tile[x] : __shfl(vs_lane, 16 * x + 4 * grp + v);
                            p[4 * x + v] = p[4 * x + v] == 0.f ? 0.f : p[4 * x + v] * z;
                        }
                }
#pragma unroll
                for (int v = 0; v < 2 * X; ++v) pb[i][v / 4][v % 4] = pack_bf16(p[2 * v], p[2 * v + 1]);
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
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    // eight keys of an element to a lane: those of its weights
                    const int n = (lane & 15) >> 1, row = 32 * c + 4 * grp + (n & 3) + 16 * (n >> 2);
                    const unsigned char* q = vt + row * DH + piece8<DH>(row, d) * 16 + (lane & 1) * 8;
                    const i32x2 t = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)q);
                    const bf16x8 w = widen8((uint32_t)t.x, (uint32_t)t.y, folded ? vs_tile[2 * c] : 1.f, folded ? vs_tile[2 * c + 1] : 1.f);
#pragma unroll
                    for (int i = 0; i < RT; ++i)
                        o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, pb[i][c]), o[i][d], 0, 0, 0);
                }
        }

        constexpr int F = kPartFloats<DH, ROWS * HW>;
        const int64_t begin = pl.first + (int64_t)item * pl.steps;
        const Parts parts = parts_of(begin, begin + pl.steps, all.share);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            l[i] += __shfl_xor(l[i], 16);
            l[i] += __shfl_xor(l[i], 32);
        }
        if constexpr (HW > 1) {
            // ---- each wavefront's rows: a lane has four elements after another of its row -----
            // A part lies in the order of these registers, two floats of a lane beside those
            // of its neighbours.
            bool finish = whole;
            if (!whole) {
                constexpr int MINE = ROWS * DH, ML = HW * MINE;
                const int at0 = wave * MINE + 2 * lane, at_ml = ML + wave * 2 * ROWS;
                float* part = part_at<F>(a, parts, parts.mine);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int v = 0; v < 4; v += 2) put2(part + at0 + ((i * DT + d) * 2 + v / 2) * 128, o[i][d][v], o[i][d][v + 1]);
                    if (grp == 0) put2(part + at_ml + 2 * (16 * i + col), m[i], l[i]);
                }
                finish = last_to_arrive(a, parts, &flag);
                if (finish) {
                    // all parts in their order, some of them on their way at a time
#pragma unroll 1
                    for (int i = 0; i < RT; ++i) {
                        constexpr int U = 4;
                        float top = minus_inf(), sum = 0.f;
                        f32x4 acc[DT];
#pragma unroll
                        for (int d = 0; d < DT; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
                        for (int n0 = 0; n0 < parts.count; n0 += U) {
                            float2 ml_n[U], v[U][DT][2];
#pragma unroll
                            for (int n = 0; n < U; ++n) {
                                const float* q = part_at<F>(a, parts, min(n0 + n, parts.count - 1));
                                ml_n[n] = get2(q + at_ml + 2 * (16 * i + col));
#pragma unroll
                                for (int d = 0; d < DT; ++d) {
                                    v[n][d][0] = get2(q + at0 + (i * DT + d) * 256);
                                    v[n][d][1] = get2(q + at0 + (i * DT + d) * 256 + 128);
                                }
                            }
#pragma unroll
                            for (int n = 0; n < U; ++n) {
                                if (n0 + n >= parts.count) break;
                                const float m1 = fmaxf(top, ml_n[n].x), z = m1 == minus_inf() ? 0.f : m1;
                                const float g0 = exp2_(top - z), g = exp2_(ml_n[n].x - z);
                                top = m1;
                                sum = fmaf(ml_n[n].y, g, sum * g0);
#pragma unroll
                                for (int d = 0; d < DT; ++d)
#pragma unroll
                                    for (int e = 0; e < 4; ++e) acc[d][e] = fmaf(e & 1 ? v[n][d][e / 2].y : v[n][d][e / 2].x, g, acc[d][e] * g0);
                            }
                        }
                        const uint32_t r = (uint32_t)(rt * ROWS + 16 * i + col);
                        const int tok = (int)divide(r, a.by_group);
                        if (16 * i + col < rows) {
#pragma unroll
                            for (int d = 0; d < DT; ++d) {
                                const float e[4] = {acc[d][0], acc[d][1], acc[d][2], acc[d][3]};
                                finish_row<4>(a, s.q0 + tok, h * a.group + (int)(r - (uint32_t)tok * a.group), 16 * d + 4 * grp, e, sum, top);
                            }
                        }
                    }
                    joined(a, parts);
                }
            } else {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const uint32_t r = (uint32_t)(rt * ROWS + 16 * i + col);
                    const int tok = (int)divide(r, a.by_group);
                    if (16 * i + col < rows) {
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const float e[4] = {o[i][d][0], o[i][d][1], o[i][d][2], o[i][d][3]};
                            finish_row<4>(a, s.q0 + tok, h * a.group + (int)(r - (uint32_t)tok * a.group), 16 * d + 4 * grp, e, l[i], m[i]);
                        }
                    }
                }
            }
        } else {
            // ---- the four wavefronts' parts, a tile of rows after another --------------------
            constexpr int N = DH / 16;                // elements of a thread
            float* red = reinterpret_cast<float*>(smem);
            auto row_of = [&](int mine, int& t, int& head) {     // whether there is one, its token and head
                const uint32_t r = (uint32_t)(rt * ROWS + mine);
                t = (int)divide(r, a.by_group);
                head = h * a.group + (int)(r - (uint32_t)t * a.group);
                return mine < rows;
            };
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int row = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * N;
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
                    const float g = exp2_(ml[w][0][row] - zero);
                    sum = fmaf(ml[w][1][row], g, sum);
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[e] = fmaf(red[(w * 16 + row) * PAD + e0 + e], g, acc[e]);
                }
                int t, head;
                if (!row_of(16 * i + row, t, head)) continue;
                if (whole) {
                    finish_row<N>(a, s.q0 + t, head, e0, acc, sum, top);
                } else {
                    float* part = part_at<F>(a, parts, parts.mine);
#pragma unroll
                    for (int e = 0; e < N; e += 2) put2(part + (16 * i + row) * DH + e0 + e, acc[e], acc[e + 1]);
                    if (e0 == 0) put2(part + ROWS * DH + 2 * (16 * i + row), top, sum);
                }
            }
            if (!whole && last_to_arrive(a, parts, &flag)) {
                // all parts in their order, eight of them on their way at a time; a thread has
                // four elements of a row
                constexpr int U = 8;
                for (int n = threadIdx.x; n < ROWS * (DH / 4); n += kFewThreads) {
                    const int mine = n / (DH / 4), e0 = n % (DH / 4) * 4;
                    int t, head;
                    if (!row_of(mine, t, head)) continue;
                    float top = minus_inf(), sum = 0.f, acc[4] = {};
                    for (int i0 = 0; i0 < parts.count; i0 += U) {
                        float2 ml_i[U], v[U][2];
#pragma unroll
                        for (int i = 0; i < U; ++i) {
                            const float* q = part_at<F>(a, parts, min(i0 + i, parts.count - 1));
                            ml_i[i] = get2(q + ROWS * DH + 2 * mine);
                            v[i][0] = get2(q + mine * DH + e0);
                            v[i][1] = get2(q + mine * DH + e0 + 2);
                        }
#pragma unroll
                        for (int i = 0; i < U; ++i) {
                            if (i0 + i >= parts.count) break;
                            const float m1 = fmaxf(top, ml_i[i].x), z = m1 == minus_inf() ? 0.f : m1;
                            const float f0 = exp2_(top - z), g = exp2_(ml_i[i].x - z);
                            top = m1;
                            sum = fmaf(ml_i[i].y, g, sum * f0);
                            acc[0] = fmaf(v[i][0].x, g, acc[0] * f0);
                            acc[1] = fmaf(v[i][0].y, g, acc[1] * f0);
                            acc[2] = fmaf(v[i][1].x, g, acc[2] * f0);
                            acc[3] = fmaf(v[i][1].y, g, acc[3] * f0);
                        }
                    }
                    finish_row<4>(a, s.q0 + t, head, e0, acc, sum, top);
                }
                joined(a, parts);
            }
        }
        __syncthreads();
        u += part1 - part0;
    }
}

// ---- many rows ---------------------------------------------------------------------------
// A workgroup of NW wavefronts of 32 rows each over the same keys, in tiles of 64 that
// are widened on their way into shared memory, two tiles there at a time: of the next
// one the bytes are in registers, of the one after it on their way there.  Widening in
// the stage is shared by all wavefronts; from there on a tile is the bf16 kernel's, whose
// bounds (matrix instructions and the softmax between them) are this one's (a prompt of
// 18432 tokens, 32 query and 8 key heads of 128: 2.82-2.91 ms, 955-985 TFLOP/s; the kernel for
// few rows, 16 rows an item: 19.2 ms).
//
// Values' scales that are powers of two go into the widening, which is exact, else
// they multiply the weights.  Keys' scales multiply scores, in the multiply-add that
// takes the maximum off.
// UNI: pages and blocks of whole 16 tokens, so that a scale is that of 16 keys; else each
// score is multiplied by its own key's (pages of 40 in blocks of 8: the prompt 4.20 ms, chunks
// of 8 requests 774 us and not 533).
template <int DH, int NW, int STEP, bool UNI, bool FULL>
__global__ __launch_bounds__(NW * 64, DH == 256 ? 1 : 2) void attend8_many_kernel(Attend8Args a)
{
    constexpr int ROWS = NW * kManyRows, T = NW * 64;
    constexpr int KF = DH / 16, DT = DH / 32;               // fragments of keys, tiles of elements
    constexpr int BYTES = kManyTile * DH * 2;               // of a widened tile
    constexpr int PIECES = DH / 16, NP = kManyTile * PIECES;   // pieces of a row and of a tile, 16 bytes each
    constexpr int NI = 2 * NP / T;                          // of a thread, keys' before values'
    // Items by themselves widen the next tile's pieces between the first product's
    // instructions (a prompt of 8192 tokens, 8 heads of 64: 435 us, before it 442; 4 of 256:
    // 2936 and 3276; 18432 tokens, 8 of 128: 2835 and 2890).  Shares widen them before it:
    // between, chunks of 8 requests with 4 heads of 128 take 546 us and not 533.
    constexpr bool kBetween = STEP == 0;
    __shared__ __align__(16) unsigned char smem[4 * BYTES]; // stage 0: K, V; stage 1: K, V
    __shared__ int flag;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;

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
            qf[k] = signed_query(a, v);
        }
        f32x16 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
        float m = minus_inf(), l = 0.f;           // m: of the scores in powers of two

        // ---- keys ---------------------------------------------------------------------
        const int base = s.begin & ~(kAlign - 1);
        int j0 = base + step0 * STEP;
        if (lo_min > j0) j0 += (lo_min - j0) / kManyTile * kManyTile;   // tiles that no row sees are skipped
        const int j_end = by_item ? hi_max : min(hi_max, base + step1 * STEP);
        const int last = hi_max - 1;
        const int32_t* table = a.step.table + (int64_t)pl.b * a.step.table_stride;
        const uint8_t* kp = static_cast<const uint8_t*>(a.cache8.k) + (int64_t)h * a.cache8.head;
        const uint8_t* vp = static_cast<const uint8_t*>(a.cache8.v) + (int64_t)h * a.cache8.head;
        const float* ksp = a.cache8.k_scale + (int64_t)h * a.cache8.scale_head;
        const float* vsp = a.cache8.v_scale + (int64_t)h * a.cache8.scale_head;
        // Each lane looks one key of a tile up.  Those that no row of the tile sees are
        // read as the nearest that one does.
        int page = 0, in = 0;
        auto look = [&](int j) {
            const int t = min(max(j + lane, lo_min), last);
            const int slot = (int)divide((uint32_t)t, a.by_page);
            page = table[slot];
            in = t - slot * a.cache8.page_size;
        };
        u32x4 raw[NI];
        float ks_next = 0.f, vs_next = 0.f;       // of this lane's key
        auto fetch = [&] {
            const int g = min(max(page, 0), a.cache8.pages - 1);
            const int64_t at = (int64_t)g * a.cache8.page + (int64_t)in * a.cache8.token;
            const int64_t scale = (int64_t)g * a.cache8.scale_page + (int64_t)divide((uint32_t)in, a.by_block) * a.cache8.scale_block;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int n = i * T + (int)threadIdx.x, p = n & (NP - 1);
                const uint8_t* from = n < NP ? kp : vp;
                raw[i] = u32x4{};
                const int64_t off = __shfl(at, p / PIECES);
                if (FULL || (p % PIECES) * 16 < a.dim) raw[i] = *reinterpret_cast<const u32x4*>(from + off + (p % PIECES) * 16);
            }
            ks_next = ksp[scale];
            vs_next = vsp[scale];
        };
        auto store = [&](int i, int stage, bool folded) {      // piece i of the tile in registers, into a stage
            const int n = i * T + (int)threadIdx.x, p = n & (NP - 1), row = p / PIECES, piece = 2 * (p % PIECES);
            const bool value = n >= NP;
            const float f = __shfl(vs_next, row);
            const float by = value && folded ? f : 1.f;
            const int turn = value ? v_swizzle<DH>(row) : k_swizzle<DH>(row);
            unsigned char* to = smem + stage * 2 * BYTES + (value ? BYTES : 0) + row * (DH * 2);
            *reinterpret_cast<bf16x8*>(to + (piece ^ turn) * 16) = widen8(raw[i].x, raw[i].y, by, by);
            *reinterpret_cast<bf16x8*>(to + ((piece + 1) ^ turn) * 16) = widen8(raw[i].z, raw[i].w, by, by);
        };
        float ks = 0.f, vs = 0.f;                 // of the stage that is read
        bool folded = false;
        if (j0 < j_end) {
            look(j0);
            fetch();
            if (j0 + kManyTile < j_end) look(j0 + kManyTile);
            ks = ks_next;
            vs = vs_next;
            folded = __all(is_power(vs)) != 0;
#pragma unroll
            for (int i = 0; i < NI; ++i) store(i, 0, folded);
            if (j0 + kManyTile < j_end) {
                fetch();
                if (j0 + 2 * kManyTile < j_end) look(j0 + 2 * kManyTile);
            }
        }
        int stage = 0;
        for (; j0 < j_end; j0 += kManyTile, stage ^= 1) {
            __syncthreads();
            const float ks_then = ks_next, vs_then = vs_next;       // of the stage that is filled
            const bool folded_then = __all(is_power(vs_then)) != 0;
            auto ahead = [&] {                    // past the last tile: its keys again
                fetch();
                look(j0 + 3 * kManyTile);
            };
            if (!kBetween && j0 + kManyTile < j_end) {
#pragma unroll
                for (int i = 0; i < NI; ++i) store(i, stage ^ 1, folded_then);
                if (j0 + 2 * kManyTile < j_end) ahead();
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
            if (!idle || bad) {
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
                        constexpr int EACH = 2 * KF / NI;
                        if (kBetween && (x * KF + k) % EACH == EACH - 1) store((x * KF + k) / EACH, stage ^ 1, folded_then);
                    }
                }
                if constexpr (kBetween) ahead();
                const float by = factor(ks * a.scale);
                float f[4];
                if constexpr (UNI) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) f[g] = lane_of(by, 16 * g);
                } else {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int v = 0; v < 16; ++v) sc[x][v] *= __shfl(by, 32 * x + 8 * (v / 4) + 4 * half + v % 4);
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
                for (int g = 0; g < 4; ++g) {
                    const f32x16& y = sc[g / 2];
                    const int v = 8 * (g % 2);
                    float t = max3(y[v], y[v + 1], y[v + 2]);
                    t = max3(t, y[v + 3], y[v + 4]);
                    t = max3(t, y[v + 5], max3(y[v + 6], y[v + 7], y[v + 7]));
                    top = max3(top, UNI ? t * f[g] : t, top);
                }
                top = max_halves(top);
                float up = 0.f;
                if (!folded) {
                    asm volatile("");      // a branch: append's scales need none of this
                    up = __any(vs > kLargeScale) ? kRaise : 0.f;
                }
                // The maximum that a row's weights are relative to follows only when it is
                // left behind by 2^8: sums scaled by less than that lose nothing.
                const bool left = top - m > 8.f - up;
                if (__any(left)) {
                    const float keep = left ? exp2_(m - (top + up)) : 1.f;
                    m = left ? top + up : m;
                    l *= keep;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[d] *= keep;
                }
                const float zero = m == minus_inf() ? 0.f : m;
                u32x4 pb[4];
                float sum[2] = {0.f, 0.f};
                auto weights = [&](auto scaled) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int v = 0; v < 16; v += 2) {
                            const int g = 2 * x + v / 8;
                            float p = exp2_(UNI ? fmaf(sc[x][v], f[g], -zero) : sc[x][v] - zero);
                            float q = exp2_(UNI ? fmaf(sc[x][v + 1], f[g], -zero) : sc[x][v + 1] - zero);
                            sum[0] += p;
                            sum[1] += q;
                            if constexpr (decltype(scaled)::value) {
                                // a key that is not seen may have any scale
                                const int key = 32 * x + 8 * (v / 4) + 4 * half + v % 4;
                                const float fp = UNI ? lane_of(vs, 16 * g) : __shfl(vs, key), fq = UNI ? fp : __shfl(vs, key + 1);
                                p = p == 0.f ? 0.f : p * fp;
                                q = q == 0.f ? 0.f : q * fq;
                            }
                            pb[2 * x + v / 8][v / 2 % 4] = pack_bf16(p, q);
                        }
                };
                if (folded) weights(std::false_type{});
                else weights(std::true_type{});
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
            } else if constexpr (kBetween) {
#pragma unroll
                for (int i = 0; i < NI; ++i) store(i, stage ^ 1, folded_then);
                ahead();
            }
            ks = ks_then;
            vs = vs_then;
            folded = folded_then;
        }

        // ---- results: a lane holds 4 elements after another of its row -------------------
        l += __shfl_xor(l, 32);
        float top = m;
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
// Whether 16 tokens from a multiple of 16 on lie in one page and block, a page below 2 GB.
bool in_halves(const Attend8Args& a)
{
    return a.cache8.page_size % 16 == 0 && a.cache8.block % 16 == 0 && a.cache8.token < INT32_MAX &&
           a.cache8.token * (int64_t)a.cache8.page_size < INT32_MAX;
}

template <int DH, int HW, int RT>
hipError_t few(const Attend8Args& args, hipStream_t s)
{
    static_assert(kPartsFit<DH, 16 * RT * HW>, "the parts' scratch is too small");
    Attend8Args a = args;
    a.kv_heads /= HW;
    const bool pg16 = in_halves(a);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.cus), dim3(kFewThreads), 0, s, a);
        return hipGetLastError();
    };
    if (a.dim == DH) return pg16 ? launch(attend8_few_kernel<DH, HW, RT, true, true>) : launch(attend8_few_kernel<DH, HW, RT, false, true>);
    return pg16 ? launch(attend8_few_kernel<DH, HW, RT, true, false>) : launch(attend8_few_kernel<DH, HW, RT, false, false>);
}

// Four heads to a workgroup where their rows are shorter than memory's lines and lie
// side by side, and there are enough of them that a workgroup need not begin and end
// many (one request of 32 heads of 64 over 1216 tokens: 12 us and 21).
template <int DH, int RT>
hipError_t few(const Attend8Args& a, hipStream_t s)
{
    if constexpr (DH == 64) {
        if (a.kv_heads % 4 == 0 && a.cache8.head < 128 && a.step.seqs * (a.kv_heads / 4) >= a.cus / 8) return few<DH, 4, RT>(a, s);
    }
    return few<DH, 1, RT>(a, s);
}

// Wavefronts of a workgroup of the kernel for many rows.
template <int DH>
constexpr int kManyWaves = DH == 256 ? 4 : 8;
constexpr int kManyStep = 256;

template <int DH>
hipError_t many(const Attend8Args& a, hipStream_t s)
{
    constexpr int NW = kManyWaves<DH>, ROWS = NW * kManyRows;
    static_assert(kPartsFit<DH, ROWS>, "the parts' scratch is too small");
    // no more items than this, whatever the sequences' lengths
    const int64_t items = ((a.tokens * a.group + ROWS - 1) / ROWS + a.step.seqs) * a.kv_heads;
    auto launch = [&](auto kernel, int64_t groups) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(NW * 64), 0, s, a);
        return hipGetLastError();
    };
    const bool uni = a.cache8.page_size % 16 == 0 && a.cache8.block % 16 == 0;
    // An item a workgroup where that makes two rounds at least, else a workgroup a CU
    // and shares of the steps, as in the bf16 kernel.  A launch has fewer than 2^32
    // threads.
    if ((a.tokens * a.group / ROWS) * a.kv_heads >= 2 * a.cus && a.step.seqs <= kSearched && items * (NW * 64) <= (int64_t)UINT32_MAX) {
        if (a.dim == DH) return uni ? launch(attend8_many_kernel<DH, NW, 0, true, true>, items) : launch(attend8_many_kernel<DH, NW, 0, false, true>, items);
        return uni ? launch(attend8_many_kernel<DH, NW, 0, true, false>, items) : launch(attend8_many_kernel<DH, NW, 0, false, false>, items);
    }
    if (a.dim == DH)
        return uni ? launch(attend8_many_kernel<DH, NW, kManyStep, true, true>, a.cus) : launch(attend8_many_kernel<DH, NW, kManyStep, false, true>, a.cus);
    return uni ? launch(attend8_many_kernel<DH, NW, kManyStep, true, false>, a.cus) : launch(attend8_many_kernel<DH, NW, kManyStep, false, false>, a.cus);
}

template <int DH>
hipError_t attend8(const Attend8Args& args, hipStream_t s)
{
    Attend8Args a = args;
    const int64_t rows = a.tokens * a.group;
    a.scale = fabsf(a.raw_scale) * kLog2e;
    a.flip = a.raw_scale < 0.f ? 0x80008000u : 0u;
    a.keep = a.scale > 0.f ? ~0u : 0u;
    if (!a.keep) a.scale = 1.f;
    // By the rows of a sequence and key head, on average (16 requests with 5 to 9 tokens,
    // groups of 8, heads of 128: 79 us with four tiles of rows, 166 as many; 64 with 2 to 4,
    // groups of 7: 140 with two, 193 with four).
    const int64_t seqs = a.step.seqs;
    if (rows <= 16 * seqs) return few<DH, 1>(a, s);
    if (rows <= 32 * seqs) return few<DH, 2>(a, s);
    if constexpr (DH < 256) {
        if (rows <= 64 * seqs) return few<DH, 4>(a, s);
    }
    return many<DH>(a, s);
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
