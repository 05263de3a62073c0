// Positions of kept tokens, and norm, rotation and appending of heads:
//   y = R(pos) (x * w / sqrt(mean x^2 + eps))   for every head of every token,
// R turning pair i of the head by the angle pos[axis_i] * freq_i, and its
// gradient  dx = r (gw - u mean(gw u)),  dw = sum g u,  with g = R^T dy,
// r = 1 / sqrt(mean x^2 + eps), u = x r, gw = g w.
//
// Angles are formed as models form them, as the fp32 product of a position and a
// frequency.  That angle's fraction of a turn is taken in fp64 with 1 / 2 pi to
// 107 bits (below 2^-28 of a turn off at angles to 2^64), split into the nearest
// quarter and a rest of at most an eighth, where the Taylor series of sine and
// cosine to x^9 and x^10 are below 2e-9 off.
//
// All of it is bound by memory: heads are read once and written once.  Measured:
// 36864 tokens of 40 bf16 heads of 128 in 132-138 us (5.5-5.7 TB/s read and
// written; a library copy of 2 GiB 5.0), 8 prompts appended (9000 tokens) in 37 us
// (5.2), gradients of 16384 tokens in 93 us (5.4) and the sum of dw in 5 more.
// Small calls are bound by their launch: 64 tokens appended 5.6 us, 577 fp32 tokens
// 6.1, positions of 64 clips 2.6.
#include <algorithm>
#include <type_traits>

#include "tr_attn.h"
#include "tr_row.h"
#include "tr_wave.h"

namespace tr {
namespace {

// ---- positions -----------------------------------------------------------------
__global__ __launch_bounds__(256) void positions_kernel(PosArgs a)
{
    const PosImage im = a.image[blockIdx.y];
    const uint32_t i = blockIdx.x * blockDim.x + threadIdx.x;   // the last workgroup's may pass 2^31
    if (i >= (uint32_t)im.count) return;
    const int32_t n = a.idx[im.src + i];
    const int32_t t = n / im.hw, in = n - t * im.hw;
    const int32_t h = in / im.w, w = in - h * im.w;
    int32_t* p = a.pos + im.dst + i;
    p[0] = im.start[0] + t;
    p[a.ldpos] = im.start[1] + h;
    p[2 * a.ldpos] = im.start[2] + w;
}

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

template <typename E>
__global__ __launch_bounds__(256) void rotate_any_kernel(RotateArgs g, int64_t first)
{
    const int lane = threadIdx.x & 63;
    const int rows = g.heads[0] + g.heads[1] + g.heads[2];
    const int64_t u = first + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (u >= g.tokens * rows) return;
    const int64_t t = u / rows;
    int h = (int)(u - t * rows), kind = 0;
    while (h >= g.heads[kind]) h -= g.heads[kind++];
    E* dst = static_cast<E*>(g.out[kind].p) + t * g.out[kind].token + (int64_t)h * g.out[kind].head;
    if (g.append) {
        const int64_t row = cache_row(g.step, g.cache, t, lane);
        if (row == kNoToken || (kind > 0 && row == kNoRow)) return;
        if (kind > 0) dst = static_cast<E*>(kind == 1 ? g.cache.k : g.cache.v) + row + (int64_t)h * g.cache.head;
    }
    AnyHead<E> x;
    x.load(g, static_cast<const E*>(g.in[kind].p) + t * g.in[kind].token + (int64_t)h * g.in[kind].head, lane);
    if (kind < 2) {
        if (g.norm) {
            AnyHead<E> w;
            if (g.w[kind]) w.load(g, static_cast<const E*>(g.w[kind]), lane);
            else w.fill(1.f);
            float z;
            const float r = x.inverse(g, z);
            x.each(w, [&](float v, float m) { return v * r * m; });
        }
        x.rotate(g, t, lane, false);
    }
    x.store(g, dst, lane);
}

// Each wavefront walks heads u, u + waves, ... of one side (blockIdx.y) and
// keeps their share of dw; a workgroup's four shares go to `part`, whose rows
// sum_parts_kernel adds in order.
template <typename E>
__global__ __launch_bounds__(256) void rotate_back_any_kernel(RotateArgs g)
{
    __shared__ float red[4][kMaxHeadDim];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kind = blockIdx.y;
    const int rows = g.heads[kind];
    const int64_t waves = (int64_t)gridDim.x * 4;
    AnyHead<E> w, dw;
    w.fill(1.f);
    dw.fill(0.f);
    if (g.w[kind]) w.load(g, static_cast<const E*>(g.w[kind]), lane);
    for (int64_t u = (int64_t)blockIdx.x * 4 + wave; u < g.tokens * rows; u += waves) {
        const int64_t t = u / rows;
        const int64_t h = u - t * rows;
        AnyHead<E> y, x;
        y.load(g, static_cast<const E*>(g.grad[kind].p) + t * g.grad[kind].token + h * g.grad[kind].head, lane);
        if (g.norm) x.load(g, static_cast<const E*>(g.in[kind].p) + t * g.in[kind].token + h * g.in[kind].head, lane);
        y.rotate(g, t, lane, true);
        if (g.norm) {
            float z;
            const float r = x.inverse(g, z);
            x.each(x, [&](float v, float) { return v * r; });
            AnyHead<E> d = y;
            d.each(x, [](float p, float q) { return p * q; });
            dw.each(d, [](float p, float q) { return p + q; });
            y.each(w, [](float p, float q) { return p * q; });
            const float m = y.dot(x) / (float)g.dim;
            y.each(x, [&](float p, float q) { return r * fmaf(-q, m, p) * z; });
        }
        y.store(g, static_cast<E*>(g.out[kind].p) + t * g.out[kind].token + h * g.out[kind].head, lane);
    }
    if (!g.dw[kind]) return;   // the whole grid row leaves together
    AnyHead<float> share;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        share.a[j] = dw.a[j];
        share.b[j] = dw.b[j];
    }
#pragma unroll
    for (int j = 0; j < kRest; ++j) share.r[j] = dw.r[j];
    share.store(g, red[wave], lane);
    __syncthreads();
    for (int j = threadIdx.x; j < g.dim; j += 256)
        g.part[((int64_t)kind * gridDim.x + blockIdx.x) * g.dim + j] = (red[0][j] + red[1][j]) + (red[2][j] + red[3][j]);
}

// dw[kind][j] = sum over the workgroups' rows of `part`: 32 columns to a
// workgroup, 32 threads to a column, joined in a fixed order.
__global__ __launch_bounds__(1024) void sum_parts_kernel(RotateArgs g, int parts)
{
    __shared__ float red[32][33];
    const int kind = blockIdx.y, col = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int j = blockIdx.x * 32 + col;
    if (!g.dw[kind]) return;   // the whole workgroup leaves together
    constexpr int U = 8;                     // rows of a column on their way at a time
    float s = 0.f;
    for (int i0 = row; i0 < parts; i0 += 32 * U) {
        float v[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = i0 + 32 * k;
            v[k] = i < parts && j < g.dim ? g.part[((int64_t)kind * parts + i) * g.dim + j] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < U; ++k) s += v[k];
    }
    red[row][col] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) v += red[i][col];
        if (j < g.dim) g.dw[kind][j] = v;
    }
}

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

// Stores that nothing near reads again: past what the caches hold they are
// streamed (36864 tokens of 40 bf16 heads of 128 180 -> 170 us, 8 prompts
// appended 45 -> 38 us).
template <bool STREAM, typename E>
__device__ __forceinline__ void put(E* p, Raw<E> v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<Raw<E>*>(p));
    else *reinterpret_cast<Raw<E>*>(p) = v;
}

// Wavefront `first` and those after it: each takes `per` rounds of one token, a
// round being 64 / LP heads of one side: queries, keys, then values.  A head's address is the round's (the
// wavefront's) and 32 bits of a lane's.
template <typename E, int LP, bool ADJ, bool APPEND, bool STREAM>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs g, int per, int chunks, uint32_t first)
{
    constexpr int R = 64 / LP, DEPTH = 2;
    const int lane = threadIdx.x & 63, j = lane & (LP - 1), hl = lane / LP;
    const uint32_t u = first + blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
                if (g.norm) {
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
                    const Piece& w = kind ? wk : wq;
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) {
                        x.a[e] = x.a[e] * m * w.a[e];
                        x.b[e] = x.b[e] * m * w.b[e];
                    }
                }
                Piece y = x;
                if (sp.turns) {
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) {
                        y.a[e] = fmaf(x.a[e], z[e].c, -(x.b[e] * z[e].s));
                        y.b[e] = fmaf(x.b[e], z[e].c, x.a[e] * z[e].s);
                    }
                }
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

// Gradients of one side (blockIdx.y): a wavefront walks over tokens t, t +
// waves, ... and their heads, and keeps its lanes' share of dw, which a
// workgroup joins into its row of `part`.
template <typename E, int LP, bool ADJ, bool STREAM>
__global__ __launch_bounds__(256) void rotate_back_kernel(RotateArgs g)
{
    constexpr int R = 64 / LP, DEPTH = 2;
    __shared__ float red[4][kMaxHeadDim];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & (LP - 1), hl = lane / LP,
              kind = blockIdx.y;
    const int rows = g.heads[kind];
    const int64_t waves = (int64_t)gridDim.x * 4;
    const Spot sp = spot_of<ADJ>(j, g.dim, g.rot);
    const uint32_t b0 = sp.e0 * (uint32_t)sizeof(E), b1 = sp.e1 * (uint32_t)sizeof(E);
    const tr_heads hg = g.grad[kind], hx = g.in[kind], ho = g.out[kind];
    const Spin spin = spin_of(g, j, sp.turns);
    const float mean = 1.f / (float)g.dim;
    Piece w, dw;
    if (g.norm) w = load_weight<E, ADJ>(g.w[kind], sp);
#pragma unroll
    for (int e = 0; e < kPiece; ++e) dw.a[e] = dw.b[e] = 0.f;
    for (int64_t t = (int64_t)blockIdx.x * 4 + wave; t < g.tokens; t += waves) {
        Raw<E> g0[DEPTH], g1[DEPTH], x0[DEPTH], x1[DEPTH];
        auto fetch = [&](int d, int h) {              // heads h .. h + R - 1
            if (h + hl < rows && sp.on) {
                const char* p = static_cast<const char*>(hg.p) + (t * hg.token + (int64_t)h * hg.head) * (int)sizeof(E);
                const uint32_t at = (uint32_t)hl * ((uint32_t)hg.head * (uint32_t)sizeof(E));
                g0[d] = load(reinterpret_cast<const E*>(p + (at + b0)));
                g1[d] = load(reinterpret_cast<const E*>(p + (at + b1)));
                if (g.norm) {
                    const char* q = static_cast<const char*>(hx.p) + (t * hx.token + (int64_t)h * hx.head) * (int)sizeof(E);
                    const uint32_t ax = (uint32_t)hl * ((uint32_t)hx.head * (uint32_t)sizeof(E));
                    x0[d] = load(reinterpret_cast<const E*>(q + (ax + b0)));
                    x1[d] = load(reinterpret_cast<const E*>(q + (ax + b1)));
                }
            }
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fetch(d, d * R);
        Turn z[kPiece];
        turns_of(g, spin, t, z);
        for (int h0 = 0; h0 < rows; h0 += DEPTH * R) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int h = h0 + d * R;
                if (h >= rows) break;
                const bool live = h + hl < rows && sp.on;
                Piece y = unpack<E, ADJ>(g0[d], g1[d]);
                [[maybe_unused]] Piece x;
                if (g.norm) x = unpack<E, ADJ>(x0[d], x1[d]);
                fetch(d, h + DEPTH * R);
                if (sp.turns) {
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) {
                        const float a = y.a[e], b = y.b[e];
                        y.a[e] = fmaf(a, z[e].c, b * z[e].s);
                        y.b[e] = fmaf(b, z[e].c, -(a * z[e].s));
                    }
                }
                if (g.norm) {
                    float q = 0.f, m = 0.f;
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) {
                        q = fmaf(x.a[e], x.a[e], fmaf(x.b[e], x.b[e], q));
                        m = fmaf(y.a[e] * w.a[e], x.a[e], fmaf(y.b[e] * w.b[e], x.b[e], m));
                    }
                    q = group_sum<LP>(live ? q : 0.f);
                    m = group_sum<LP>(live ? m : 0.f);
                    float v = fmaf(q, mean, g.eps), f = 1.f;
                    const bool scaled = __any(live && !in_range(v));
                    if (scaled) {
                        f = scale_for(v);
                        q = m = 0.f;
#pragma unroll
                        for (int e = 0; e < kPiece; ++e) {
                            x.a[e] *= f;
                            x.b[e] *= f;
                            q = fmaf(x.a[e], x.a[e], fmaf(x.b[e], x.b[e], q));
                            m = fmaf(y.a[e] * w.a[e], x.a[e], fmaf(y.b[e] * w.b[e], x.b[e], m));
                        }
                        v = fmaf(group_sum<LP>(live ? q : 0.f), mean, g.eps * f * f);
                        m = group_sum<LP>(live ? m : 0.f);
                    }
                    const float n = rsqrt_(v);
                    m = m * n * mean;
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) {
                        const float ua = x.a[e] * n, ub = x.b[e] * n;
                        dw.a[e] += live ? y.a[e] * ua : 0.f;
                        dw.b[e] += live ? y.b[e] * ub : 0.f;
                        y.a[e] = n * fmaf(-ua, m, y.a[e] * w.a[e]);
                        y.b[e] = n * fmaf(-ub, m, y.b[e] * w.b[e]);
                    }
                    if (scaled) {
#pragma unroll
                        for (int e = 0; e < kPiece; ++e) {
                            y.a[e] *= f;
                            y.b[e] *= f;
                        }
                    }
                }
                if (live) {
                    Raw<E> y0, y1;
                    pack<E, ADJ>(y, y0, y1);
                    char* p = static_cast<char*>(ho.p) + (t * ho.token + (int64_t)h * ho.head) * (int)sizeof(E);
                    const uint32_t at = (uint32_t)hl * ((uint32_t)ho.head * (uint32_t)sizeof(E));
                    put<STREAM>(reinterpret_cast<E*>(p + (at + b0)), y0);
                    put<STREAM>(reinterpret_cast<E*>(p + (at + b1)), y1);
                }
            }
        }
    }
    if (!g.dw[kind]) return;   // the whole workgroup leaves together
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        float a = dw.a[e], b = dw.b[e];
#pragma unroll
        for (int m = LP; m < 64; m <<= 1) {
            a += __shfl_xor(a, m);
            b += __shfl_xor(b, m);
        }
        if (lane < LP && sp.on) {
            red[wave][ADJ ? sp.e0 + 2 * e : sp.e0 + e] = a;
            red[wave][ADJ ? sp.e0 + 2 * e + 1 : sp.e1 + e] = b;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < g.dim; i += 256)
        g.part[((int64_t)kind * gridDim.x + blockIdx.x) * g.dim + i] = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
}

// ---- launches ------------------------------------------------------------------------
// Workgroups of a side: with both sides' the chip is full at once, and each
// wavefront walks over many tokens (16384 tokens of 40 bf16 heads of 128: 102 us
// with two a CU, 112 with four, 121 with eight).
int back_groups(int cus) { return 2 * cus; }

bool whole(const tr_heads& h, int eb)
{
    if (h.head * eb > (int64_t)(INT32_MAX / 64)) return false;   // a round's heads lie within 2 GB
    return ((uintptr_t)h.p | (uintptr_t)(h.token * eb) | (uintptr_t)(h.head * eb)) % (kPiece * eb) == 0;
}

// Whether every head of the call is made of whole pieces: its address, its
// halves and its rotated part.
bool in_pieces(const RotateArgs& a, int eb, bool back)
{
    if (a.dim % (2 * kPiece) || a.rot % (2 * kPiece)) return false;
    for (int k = 0; k < 3; ++k) {
        if (!a.heads[k]) continue;
        const bool to_cache = a.append && k > 0;
        if (!whole(a.in[k], eb) && !(back && !a.norm)) return false;
        if (!to_cache && !whole(a.out[k], eb)) return false;
        if (back && !whole(a.grad[k], eb)) return false;
        if (k < 2 && (uintptr_t)a.w[k] % (kPiece * eb)) return false;
    }
    return !a.append || (a.cache.head * eb <= (int64_t)(INT32_MAX / 64) &&
                         ((uintptr_t)a.cache.k | (uintptr_t)a.cache.v) % (kPiece * eb) == 0 &&
                         (a.cache.page | a.cache.token | a.cache.head) % kPiece == 0);
}

// Launches f(first, workgroups) for n wavefronts, four to a workgroup: a launch
// has fewer than 2^32 threads.
template <typename F>
hipError_t in_launches(int64_t n, F f)
{
    constexpr int64_t kMost = int64_t(1) << 25;
    hipError_t e = hipSuccess;
    for (int64_t first = 0; first < n && e == hipSuccess; first += kMost) {
        f(first, (unsigned)((std::min(kMost, n - first) + 3) / 4));
        e = hipGetLastError();
    }
    return e;
}

// From what a call moves on its stores are streamed.
constexpr int64_t kStreamBytes = 32 << 20;

template <typename E, int LP>
hipError_t rotate_pieces(const RotateArgs& a, hipStream_t s)
{
    constexpr int R = 64 / LP;
    int rounds = 0, heads = 0;
    for (int k = 0; k < 3; ++k) {
        rounds += (a.heads[k] + R - 1) / R;
        heads += a.heads[k];
    }
    // All of a token's heads to a wavefront, which then works its angles out once,
    // where that leaves the chip full; else a round each.
    const int per = a.tokens >= 16 * (int64_t)a.cus ? rounds : 1;
    const int chunks = (rounds + per - 1) / per;
    const bool stream = a.tokens * heads * a.dim * (int64_t)sizeof(E) >= kStreamBytes;
    auto launch = [&](auto kernel) {
        return in_launches(a.tokens * chunks, [&](int64_t first, unsigned groups) {
            hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), 0, s, a, per, chunks, (uint32_t)first);
        });
    };
    auto pick = [&](auto adj, auto append) {
        constexpr bool A = decltype(adj)::value, P = decltype(append)::value;
        return stream ? launch(rotate_kernel<E, LP, A, P, true>) : launch(rotate_kernel<E, LP, A, P, false>);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    if (a.append) return a.adjacent ? pick(Yes{}, Yes{}) : pick(No{}, Yes{});
    return a.adjacent ? pick(Yes{}, No{}) : pick(No{}, No{});
}

template <typename E, int LP>
hipError_t back_pieces(const RotateArgs& a, int groups, hipStream_t s)
{
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups, 2), dim3(256), 0, s, a);
        return hipGetLastError();
    };
    const bool stream = a.tokens * (a.heads[0] + a.heads[1]) * a.dim * (int64_t)sizeof(E) >= kStreamBytes;
    if (stream) return a.adjacent ? launch(rotate_back_kernel<E, LP, true, true>) : launch(rotate_back_kernel<E, LP, false, true>);
    return a.adjacent ? launch(rotate_back_kernel<E, LP, true, false>) : launch(rotate_back_kernel<E, LP, false, false>);
}

template <typename E>
hipError_t rotate_typed(const RotateArgs& a, hipStream_t s)
{
    if (!in_pieces(a, (int)sizeof(E), false)) {
        return in_launches(a.tokens * (a.heads[0] + a.heads[1] + a.heads[2]), [&](int64_t first, unsigned groups) {
            hipLaunchKernelGGL(rotate_any_kernel<E>, dim3(groups), dim3(256), 0, s, a, first);
        });
    }
    const int lanes = a.dim / (2 * kPiece);
    if (lanes <= 4) return rotate_pieces<E, 4>(a, s);
    if (lanes <= 8) return rotate_pieces<E, 8>(a, s);
    if (lanes <= 16) return rotate_pieces<E, 16>(a, s);
    return rotate_pieces<E, 32>(a, s);
}

template <typename E>
hipError_t back_typed(const RotateArgs& a, hipStream_t s)
{
    const bool pieces = in_pieces(a, (int)sizeof(E), true);
    const int64_t units = pieces ? a.tokens : a.tokens * (a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1]);
    const int groups = (int)std::max((int64_t)1, std::min((int64_t)back_groups(a.cus), (units + 3) / 4));
    hipError_t e;
    if (!pieces) {
        hipLaunchKernelGGL(rotate_back_any_kernel<E>, dim3((unsigned)groups, 2), dim3(256), 0, s, a);
        e = hipGetLastError();
    } else {
        const int lanes = a.dim / (2 * kPiece);
        e = lanes <= 4 ? back_pieces<E, 4>(a, groups, s) : lanes <= 8 ? back_pieces<E, 8>(a, groups, s)
            : lanes <= 16 ? back_pieces<E, 16>(a, groups, s) : back_pieces<E, 32>(a, groups, s);
    }
    if (e == hipSuccess && (a.dw[0] || a.dw[1])) {
        hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)(a.dim + 31) / 32, 2), dim3(1024), 0, s, a, groups);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

hipError_t launch_positions(const PosArgs& a, int images, int most, hipStream_t s)
{
    if (images < 1 || most < 1) return hipSuccess;
    hipLaunchKernelGGL(positions_kernel, dim3(((unsigned)most + 255u) / 256u, (unsigned)images), dim3(256), 0, s, a);
    return hipGetLastError();
}

size_t rotate_part_floats(int dim, int cus) { return (size_t)2 * back_groups(cus) * dim; }

hipError_t launch_rotate(const RotateArgs& a, bool bf16, hipStream_t s)
{
    return bf16 ? rotate_typed<uint16_t>(a, s) : rotate_typed<float>(a, s);
}

hipError_t launch_rotate_backward(const RotateArgs& a, bool bf16, hipStream_t s)
{
    return bf16 ? back_typed<uint16_t>(a, s) : back_typed<float>(a, s);
}

}  // namespace tr
