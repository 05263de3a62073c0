// Positions of kept tokens, and norm, rotation and appending of heads:
//   y = R(pos) (x * w / sqrt(mean x^2 + eps))   for every head of every token,
// R turning pair i of the head by the angle pos[axis_i] * freq_i, and its
// gradient  dx = r (gw - u mean(gw u)),  dw = sum g u,  with g = R^T dy,
// r = 1 / sqrt(mean x^2 + eps), u = x r, gw = g w.
//
// Angles.  A frequency is kept as the fraction of a turn per position in 64
// bits; the product with the position, modulo 2^64, is the exact fraction of
// that frequency's turn at any int32 position.  Its upper 32 bits give the
// quarter and a rest of at most an eighth of a turn, where the Taylor series of
// sine and cosine to x^9 and x^10 are below 2e-9 off.
//
// All of it is bound by memory: heads are read once and written once.
#include <type_traits>

#include "tr_attn.h"
#include "tr_row.h"
#include "tr_wave.h"

namespace tr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---- positions -----------------------------------------------------------------
__global__ __launch_bounds__(256) void positions_kernel(PosArgs a)
{
    const PosImage im = a.image[blockIdx.y];
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= im.count) return;
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

// Cosine and sine of pos * turn / 2^64 of a turn.
__device__ __forceinline__ Turn turn_of(int32_t pos, uint64_t turn)
{
    const uint64_t z = (uint64_t)(int64_t)pos * turn;
    const uint32_t f = (uint32_t)(z >> 32);
    const uint32_t quarter = (f + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(f - (quarter << 30)) * 0x1.921fb6p-30f;   // 2 pi / 2^32
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
    const bool odd = quarter & 1u;
    const float cc = odd ? s : c, ss = odd ? c : s;
    Turn r;
    r.c = (quarter + 1u) & 2u ? -cc : cc;   // quarters 1 and 2
    r.s = quarter & 2u ? -ss : ss;          // quarters 2 and 3
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
    return (int64_t)g * c.page + (int64_t)in * c.token;
}

// Sum over the 64 lanes, the same bits in every lane.
__device__ __forceinline__ float sum64(float x)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    return x;
}

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
                const Turn z = turn_of(g.pos[(int64_t)g.pair_axis[i] * g.ldpos + t], g.turn[i]);
                const float s = back ? -z.s : z.s, x = a[j], y = b[j];
                a[j] = fmaf(x, z.c, -(y * s));
                b[j] = fmaf(y, z.c, x * s);
            }
        }
    }
};

template <typename E>
__global__ __launch_bounds__(256) void rotate_any_kernel(RotateArgs g)
{
    const int lane = threadIdx.x & 63;
    const int rows = g.heads[0] + g.heads[1] + g.heads[2];
    const int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
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
            const float r = 1.f / sqrtf(x.dot(x) / (float)g.dim + g.eps);
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
            const float r = 1.f / sqrtf(x.dot(x) / (float)g.dim + g.eps);
            x.each(x, [&](float v, float) { return v * r; });
            AnyHead<E> d = y;
            d.each(x, [](float p, float q) { return p * q; });
            dw.each(d, [](float p, float q) { return p + q; });
            y.each(w, [](float p, float q) { return p * q; });
            const float m = y.dot(x) / (float)g.dim;
            y.each(x, [&](float p, float q) { return r * fmaf(-q, m, p); });
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

// dw[kind][j] = sum over the workgroups' rows, in order: one wavefront an element.
__global__ __launch_bounds__(64) void sum_parts_kernel(RotateArgs g, int parts)
{
    const int kind = blockIdx.y, j = blockIdx.x;
    if (!g.dw[kind]) return;
    float s = 0.f;
    for (int i = threadIdx.x; i < parts; i += 64) s += g.part[((int64_t)kind * parts + i) * g.dim + j];
    s = sum64(s);
    if (threadIdx.x == 0) g.dw[kind][j] = s;
}

int back_groups(int cus) { return 4 * cus; }

template <typename E>
hipError_t rotate_any(const RotateArgs& a, hipStream_t s)
{
    const int64_t rows = a.tokens * (a.heads[0] + a.heads[1] + a.heads[2]);
    hipLaunchKernelGGL(rotate_any_kernel<E>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename E>
hipError_t back_any(const RotateArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL(rotate_back_any_kernel<E>, dim3((unsigned)back_groups(a.cus), 2), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && (a.dw[0] || a.dw[1])) {
        hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)a.dim, 2), dim3(64), 0, s, a, back_groups(a.cus));
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

hipError_t launch_positions(const PosArgs& a, int images, int most, hipStream_t s)
{
    if (images < 1 || most < 1) return hipSuccess;
    hipLaunchKernelGGL(positions_kernel, dim3((unsigned)((most + 255) / 256), (unsigned)images), dim3(256), 0, s, a);
    return hipGetLastError();
}

size_t rotate_part_floats(int dim, int cus) { return (size_t)2 * back_groups(cus) * dim; }

hipError_t launch_rotate(const RotateArgs& a, bool bf16, hipStream_t s)
{
    return bf16 ? rotate_any<uint16_t>(a, s) : rotate_any<float>(a, s);
}

hipError_t launch_rotate_backward(const RotateArgs& a, bool bf16, hipStream_t s)
{
    return bf16 ? back_any<uint16_t>(a, s) : back_any<float>(a, s);
}

}  // namespace tr
