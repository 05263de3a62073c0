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

#include "tr_head.h"

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

// Wavefront `first` and those after it (rotate_wave).
template <typename E, int LP, bool ADJ, bool APPEND, bool STREAM>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs g, int per, int chunks, uint32_t first)
{
    rotate_wave<E, LP, ADJ, APPEND, STREAM>(g, per, chunks, first + blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
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
