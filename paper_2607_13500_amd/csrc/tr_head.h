// Heads on the device, for the kernels that norm and rotate them: the turns of a
// position, elements, where a token's keys and values go in the cache, and a head
// as one wavefront's elements or as pieces of a few lanes'.
#pragma once

#include <type_traits>

#include "tr_attn.h"
#include "tr_row.h"
#include "tr_wave.h"

namespace tr {
namespace {

// ---- angles --------------------------------------------------------------------
struct Turn {
    float c, s;
};

// Cosine and sine of the fp32 angle pos * freq.
__device__ __forceinline__ Turn turn_of(int32_t pos, float freq)
{
    const double angle = (float)pos * freq;
    // turns: the angle times 1 / 2 pi in two parts, whole turns taken out of the
    // first product as it is before its rounding
    constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;
    double z = fma(angle, lo, fma(angle, hi, -rint(angle * hi)));
    z = (z - rint(z)) * 4.0;                          // quarters, [-2, 2]
    const double near = rint(z);
    const float x = (float)(z - near) * 1.57079632679f;
    const int quarter = (int)near;
    const float x2 = x * x;
    float s = fmaf(x2, 2.75573192e-6f, -1.98412698e-4f);
    s = fmaf(x2, s, 8.33333333e-3f);
    s = fmaf(x2, s, -1.66666667e-1f);
    s = fmaf(x2 * x, s, x);
    float c = fmaf(x2, -2.75573192e-7f, 2.48015873e-5f);
    c = fmaf(x2, c, -1.38888889e-3f);
    c = fmaf(x2, c, 4.16666667e-2f);
    c = fmaf(x2, c, -0.5f);
    c = fmaf(x2, c, 1.f);
    const bool odd = quarter & 1;
    const float cc = odd ? s : c, ss = odd ? c : s;
    Turn r;
    r.c = (quarter + 1) & 2 ? -cc : cc;   // quarters 1 and 2
    r.s = quarter & 2 ? -ss : ss;         // quarters 2 and 3
    return r;
}

// ---- elements --------------------------------------------------------------------
template <typename E>
__device__ __forceinline__ float widen(E v)
{
    if constexpr (std::is_same<E, uint16_t>::value) return __uint_as_float((uint32_t)v << 16);
    else return v;
}

template <typename E>
__device__ __forceinline__ E narrow(float v)
{
    if constexpr (std::is_same<E, uint16_t>::value) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return v;
}

// ---- where a token's keys and values go ----------------------------------------
// Element offset of token t's row in the cache, -1 where it has none (kNoRow),
// -2 where the token belongs to no sequence.
constexpr int64_t kNoRow = -1, kNoToken = -2;

__device__ __forceinline__ int64_t cache_row(const tr_step& st, const tr_cache& c, int64_t t, int lane)
{
    if (st.seqs < 1 || t >= (int64_t)st.q_start[st.seqs] || t < (int64_t)st.q_start[0]) return kNoToken;
    const int b = sequence_of(st.q_start, st.seqs, t, lane);
    const int64_t p = (int64_t)st.kv_len[b] - ((int64_t)st.q_start[b + 1] - t);
    if (p < 0 || p >= (int64_t)st.table_width * c.page_size) return kNoRow;
    const int32_t slot = (int32_t)(p / c.page_size), in = (int32_t)(p - (int64_t)slot * c.page_size);
    const int32_t g = st.table[(int64_t)b * st.table_stride + slot];
    if (g < 0 || g >= c.pages) return kNoRow;
    return uniform((int64_t)g * c.page + (int64_t)in * c.token);
}

// Sum over the 64 lanes, the same bits in every lane.
__device__ __forceinline__ float sum64(float x)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    return x;
}

// Heads whose mean square plus eps (v) leaves the range in which their fp32 squares
// are right are taken again times a power of two: of squares past the largest fp32
// times 2^-80, of tiny ones beside a tiny or no eps times 2^100.  v is then that of
// the scaled head, and what is left of the scale goes into the gradient at its end.
__device__ __forceinline__ bool in_range(float v) { return v >= 0x1p-100f && v <= 0x1.fffffep127f; }
__device__ __forceinline__ float scale_for(float v) { return in_range(v) ? 1.f : v < 1.f ? 0x1p100f : 0x1p-80f; }

// ---- any head: one wavefront a head, element by element -------------------------
// Lane l holds pairs l and l + 64 (rot / 2 <= 128) and of the rest elements
// rot + l + 64 j.
constexpr int kPairs = 2, kRest = 4;

template <typename E>
struct AnyHead {
    float a[kPairs], b[kPairs], r[kRest];

    __device__ __forceinline__ static void at(const RotateArgs& g, int i, int& ia, int& ib)
    {
        ia = g.adjacent ? 2 * i : i;
        ib = g.adjacent ? 2 * i + 1 : i + g.rot / 2;
    }
    __device__ __forceinline__ void load(const RotateArgs& g, const E* p, int lane)
    {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const int i = lane + 64 * j;
            a[j] = b[j] = 0.f;
            if (i < g.rot / 2) {
                int ia, ib;
                at(g, i, ia, ib);
                a[j] = widen<E>(p[ia]);
                b[j] = widen<E>(p[ib]);
            }
        }
#pragma unroll
        for (int j = 0; j < kRest; ++j) {
            const int i = g.rot + lane + 64 * j;
            r[j] = i < g.dim ? widen<E>(p[i]) : 0.f;
        }
    }
    __device__ __forceinline__ void store(const RotateArgs& g, E* p, int lane) const
    {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const int i = lane + 64 * j;
            if (i < g.rot / 2) {
                int ia, ib;
                at(g, i, ia, ib);
                p[ia] = narrow<E>(a[j]);
                p[ib] = narrow<E>(b[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < kRest; ++j) {
            const int i = g.rot + lane + 64 * j;
            if (i < g.dim) p[i] = narrow<E>(r[j]);
        }
    }
    __device__ __forceinline__ float dot(const AnyHead& o) const
    {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) s = fmaf(a[j], o.a[j], fmaf(b[j], o.b[j], s));
#pragma unroll
        for (int j = 0; j < kRest; ++j) s = fmaf(r[j], o.r[j], s);
        return sum64(s);
    }
    template <typename F>
    __device__ __forceinline__ void each(const AnyHead& o, F f)
    {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            a[j] = f(a[j], o.a[j]);
            b[j] = f(b[j], o.b[j]);
        }
#pragma unroll
        for (int j = 0; j < kRest; ++j) r[j] = f(r[j], o.r[j]);
    }
    // Takes the head times z, which scale_for chooses; 1 / sqrt(mean square + eps) of it.
    __device__ __forceinline__ float inverse(const RotateArgs& g, float& z)
    {
        float v = dot(*this) / (float)g.dim + g.eps;
        z = scale_for(v);
        if (z != 1.f) {        // the whole wavefront's
            const float f = z;
            each(*this, [&](float p, float) { return p * f; });
            v = dot(*this) / (float)g.dim + g.eps * f * f;
        }
        return 1.f / sqrtf(v);
    }
    __device__ __forceinline__ void fill(float v)
    {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) a[j] = b[j] = v;
#pragma unroll
        for (int j = 0; j < kRest; ++j) r[j] = v;
    }
    __device__ __forceinline__ void rotate(const RotateArgs& g, int64_t t, int lane, bool back)
    {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const int i = lane + 64 * j;
            if (i < g.rot / 2) {
                const Turn z = turn_of(g.pos[(int64_t)g.pair_axis[i] * g.ldpos + t], g.freq[i]);
                const float s = back ? -z.s : z.s, x = a[j], y = b[j];
                a[j] = fmaf(x, z.c, -(y * s));
                b[j] = fmaf(y, z.c, x * s);
            }
        }
    }
};

// ---- heads of whole pieces: LP lanes a head ----------------------------------------
// Lane j of the LP that share a head holds two pieces of four elements: the first
// and the second elements of four pairs (or, where pairs are adjacent, four pairs
// one after another), and past the rotated part any two pieces.  All the lanes of
// a group keep their sines and cosines while the wavefront walks over a token's
// heads, 64 / LP at a time, with DEPTH rounds of loads in flight.  Pieces of eight
// bf16 elements need twice the registers (fewer wavefronts) and, as each group
// works all angles out, twice the sines: 36864 tokens of 40 bf16 heads of 128
// took 190 us.
constexpr int kPiece = 4;

template <typename E>
using Raw = uint32_t __attribute__((ext_vector_type(sizeof(E))));   // a piece as it lies in memory

struct Piece {
    float a[kPiece], b[kPiece];   // of pair i: a[i], b[i]; past the rotated part: the two pieces
};

template <typename E, bool ADJ>
__device__ __forceinline__ Piece unpack(Raw<E> x, Raw<E> y)
{
    Piece p;
    float v[2 * kPiece];
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        if constexpr (sizeof(E) == 2) {
            v[i] = __uint_as_float(i & 1 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16);
            v[kPiece + i] = __uint_as_float(i & 1 ? y[i / 2] & 0xffff0000u : y[i / 2] << 16);
        } else {
            v[i] = __uint_as_float(x[i]);
            v[kPiece + i] = __uint_as_float(y[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        p.a[i] = ADJ ? v[2 * i] : v[i];
        p.b[i] = ADJ ? v[2 * i + 1] : v[kPiece + i];
    }
    return p;
}

template <typename E, bool ADJ>
__device__ __forceinline__ void pack(const Piece& p, Raw<E>& x, Raw<E>& y)
{
    float v[2 * kPiece];
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        v[ADJ ? 2 * i : i] = p.a[i];
        v[ADJ ? 2 * i + 1 : kPiece + i] = p.b[i];
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(E); ++i) {
        if constexpr (sizeof(E) == 2) {
            x[i] = (uint32_t)narrow<E>(v[2 * i]) | (uint32_t)narrow<E>(v[2 * i + 1]) << 16;
            y[i] = (uint32_t)narrow<E>(v[kPiece + 2 * i]) | (uint32_t)narrow<E>(v[kPiece + 2 * i + 1]) << 16;
        } else {
            x[i] = __float_as_uint(v[i]);
            y[i] = __float_as_uint(v[kPiece + i]);
        }
    }
}

template <typename E>
__device__ __forceinline__ Raw<E> load(const E* p) { return *reinterpret_cast<const Raw<E>*>(p); }

// Sum over each group of LP lanes, the same bits in all of them.
template <int LP>
__device__ __forceinline__ float group_sum(float x)
{
    auto add = [&](auto ctrl) {
        x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    add(std::integral_constant<int, 0xB1>{});                             // lane ^ 1
    add(std::integral_constant<int, 0x4E>{});                             // lane ^ 2
    if constexpr (LP > 4) add(std::integral_constant<int, 0x141>{});      // 7 - lane of eight
    if constexpr (LP > 8) add(std::integral_constant<int, 0x140>{});      // 15 - lane of sixteen
    if constexpr (LP > 16) x += __shfl_xor(x, 16);
    return x;
}

// Where lane j's two pieces begin in a head, and whether they rotate.
struct Spot {
    int e0, e1;
    bool on, turns;
};

template <bool ADJ>
__device__ __forceinline__ Spot spot_of(int j, int dim, int rot)
{
    constexpr int C = kPiece;
    Spot s;
    s.on = j < dim / (2 * C);
    s.turns = j < rot / (2 * C);
    s.e0 = s.turns && !ADJ ? C * j : 2 * C * j;
    s.e1 = s.turns && !ADJ ? rot / 2 + C * j : 2 * C * j + C;
    return s;
}

// What lane j's pairs turn by: their frequencies, and two bits of axis each.
struct Spin {
    float freq[kPiece];
    uint32_t axes;
};

__device__ __forceinline__ Spin spin_of(const RotateArgs& g, int j, bool turns)
{
    Spin s;
    s.axes = 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        s.freq[i] = turns ? g.freq[kPiece * j + i] : 0.f;
        s.axes |= turns ? (uint32_t)g.pair_axis[kPiece * j + i] << (2 * i) : 0u;
    }
    return s;
}

// A lane's turns for token t (none: cosine 1, sine 0).
__device__ __forceinline__ void turns_of(const RotateArgs& g, const Spin& spin, int64_t t, Turn (&z)[kPiece])
{
    static_assert(kMaxAxes == 4, "an axis is two bits");
    int32_t at[kMaxAxes];
#pragma unroll
    for (int x = 0; x < kMaxAxes; ++x) at[x] = x < g.axes && g.rot ? g.pos[(int64_t)x * g.ldpos + t] : 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        const int32_t lo = spin.axes >> (2 * i) & 1u ? at[1] : at[0], hi = spin.axes >> (2 * i) & 1u ? at[3] : at[2];
        z[i] = turn_of(spin.axes >> (2 * i) & 2u ? hi : lo, spin.freq[i]);
    }
}

template <typename E, bool ADJ>
__device__ __forceinline__ Piece load_weight(const void* w, const Spot& sp)
{
    Piece p;
    if (w && sp.on) {
        const E* q = static_cast<const E*>(w);
        return unpack<E, ADJ>(load(q + sp.e0), load(q + sp.e1));
    }
#pragma unroll
    for (int i = 0; i < kPiece; ++i) p.a[i] = p.b[i] = 1.f;
    return p;
}

// 1 / sqrt(x), to within an ulp, for x of at least 2^-126 (in_range).
__device__ __forceinline__ float rsqrt_(float x) { return __builtin_amdgcn_rsqf(x); }

// Norms a lane's piece of a head by the head's mean square and w.
template <int LP>
__device__ __forceinline__ void norm_piece(const RotateArgs& g, Piece& x, const Piece& w, bool live, float mean)
{
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < kPiece; ++e) q = fmaf(x.a[e], x.a[e], fmaf(x.b[e], x.b[e], q));
    q = group_sum<LP>(live ? q : 0.f);
    float v = fmaf(q, mean, g.eps);
    if (__any(live && !in_range(v))) {
        const float f = scale_for(v);
        q = 0.f;
#pragma unroll
        for (int e = 0; e < kPiece; ++e) {
            x.a[e] *= f;
            x.b[e] *= f;
            q = fmaf(x.a[e], x.a[e], fmaf(x.b[e], x.b[e], q));
        }
        v = fmaf(group_sum<LP>(live ? q : 0.f), mean, g.eps * f * f);
    }
    const float m = rsqrt_(v);
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        x.a[e] = x.a[e] * m * w.a[e];
        x.b[e] = x.b[e] * m * w.b[e];
    }
}

// Turns it.
__device__ __forceinline__ Piece turned(const Piece& x, const Turn (&z)[kPiece])
{
    Piece y;
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        y.a[e] = fmaf(x.a[e], z[e].c, -(x.b[e] * z[e].s));
        y.b[e] = fmaf(x.b[e], z[e].c, x.a[e] * z[e].s);
    }
    return y;
}

// Stores that nothing near reads again: past what the caches hold they are
// streamed (36864 tokens of 40 bf16 heads of 128 180 -> 170 us, 8 prompts
// appended 45 -> 38 us).
template <bool STREAM, typename E>
__device__ __forceinline__ void put(E* p, Raw<E> v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<Raw<E>*>(p));
    else *reinterpret_cast<Raw<E>*>(p) = v;
}

// Wavefront u: `per` rounds of one token, a round being 64 / LP heads of one side:
// queries, keys, then values.  A head's address is the round's (the wavefront's) and 32
// bits of a lane's.
template <typename E, int LP, bool ADJ, bool APPEND, bool STREAM>
__device__ __forceinline__ void rotate_wave(const RotateArgs& g, int per, int chunks, uint32_t u)
{
    constexpr int R = 64 / LP, DEPTH = 2;
    const int lane = threadIdx.x & 63, j = lane & (LP - 1), hl = lane / LP;
    const uint32_t t = u / (uint32_t)chunks;
    if (t >= g.tokens) return;
    const int n0 = (g.heads[0] + R - 1) / R, n1 = n0 + (g.heads[1] + R - 1) / R, all = n1 + (g.heads[2] + R - 1) / R;
    const int begin = (int)(u - t * (uint32_t)chunks) * per, end = min(all, begin + per);   // the wavefront's rounds
    const Spot sp = spot_of<ADJ>(j, g.dim, g.rot);

    Raw<E> x0[DEPTH], x1[DEPTH];
    auto fetch = [&](int d, int i) {
        if (i >= end) return;
        const int kind = i < n0 ? 0 : i < n1 ? 1 : 2;
        const int h = (i - (kind == 0 ? 0 : kind == 1 ? n0 : n1)) * R;
        const tr_heads in = g.in[kind];
        if (h + hl < g.heads[kind] && sp.on) {
            const char* p = static_cast<const char*>(in.p) + ((int64_t)t * in.token + (int64_t)h * in.head) * (int)sizeof(E);
            const uint32_t at = (uint32_t)hl * ((uint32_t)in.head * (uint32_t)sizeof(E));
            x0[d] = load(reinterpret_cast<const E*>(p + (at + sp.e0 * (uint32_t)sizeof(E))));
            x1[d] = load(reinterpret_cast<const E*>(p + (at + sp.e1 * (uint32_t)sizeof(E))));
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(d, begin + d);
    int64_t row = 0;
    if constexpr (APPEND) {
        row = cache_row(g.step, g.cache, t, lane);
        if (row == kNoToken) return;
    }
    Turn z[kPiece];
    turns_of(g, spin_of(g, j, sp.turns), t, z);
    Piece wq, wk;
    if (g.norm) {
        wq = load_weight<E, ADJ>(g.w[0], sp);
        wk = load_weight<E, ADJ>(g.w[1], sp);
    }
    const float mean = 1.f / (float)g.dim;
    for (int i0 = begin; i0 < end; i0 += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int i = i0 + d;
            if (i >= end) break;
            const int kind = i < n0 ? 0 : i < n1 ? 1 : 2;
            const int h = (i - (kind == 0 ? 0 : kind == 1 ? n0 : n1)) * R;
            const bool live = h + hl < g.heads[kind] && sp.on;
            Raw<E> y0 = x0[d], y1 = x1[d];
            fetch(d, i + DEPTH);
            if (!APPEND || kind < 2) {
                Piece x = unpack<E, ADJ>(y0, y1);
                if (g.norm) norm_piece<LP>(g, x, kind ? wk : wq, live, mean);
                const Piece y = sp.turns ? turned(x, z) : x;
                pack<E, ADJ>(y, y0, y1);
            }
            const bool to_cache = APPEND && kind > 0;
            if (to_cache && row == kNoRow) continue;
            const int64_t step = to_cache ? g.cache.head : g.out[kind].head;
            char* p = static_cast<char*>(to_cache ? (kind == 1 ? g.cache.k : g.cache.v) : g.out[kind].p) +
                      ((to_cache ? row : (int64_t)t * g.out[kind].token) + (int64_t)h * step) * (int)sizeof(E);
            const uint32_t at = (uint32_t)hl * ((uint32_t)step * (uint32_t)sizeof(E));
            if (live) {
                put<STREAM>(reinterpret_cast<E*>(p + (at + sp.e0 * (uint32_t)sizeof(E))), y0);
                put<STREAM>(reinterpret_cast<E*>(p + (at + sp.e1 * (uint32_t)sizeof(E))), y1);
            }
        }
    }
}

}  // namespace
}  // namespace tr
