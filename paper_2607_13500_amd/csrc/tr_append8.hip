// New keys and values on their way into a paged cache of 8-bit values: norm and
// rotation as in the rotation kernels, then per block of tokens and head the scale
// that its largest element asks for, and e4m3.
//
// Scales are powers of two: an e4m3 value has its own exponent, so a finer scale
// gains at most one binade at the small end, and dividing by one, or changing it for a
// block whose largest element grows, is exact but for values that leave the normal
// range.  Elements stay fp32 from the inputs to that one rounding.
//
// Work.  A segment is a sequence's new tokens within one block.  How many there are is
// on the device only: sequence b is dealt the candidates from q_start[b] / block + 2 b
// on, no fewer than its segments, so that a candidate's sequence is found by a search
// and nothing is counted first.  Bound by memory as the rotation is.
#include <algorithm>

#include "tr_head.h"

namespace tr {
namespace {

constexpr float kTop = 448.f;
constexpr int kLeast = -117, kMost = 120;   // exponents of a scale

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.40282347e38f; }

// The smallest scale 2^e with top <= 448 2^e, 448 = 1.75 2^8.
__device__ __forceinline__ float scale_for_top(float top)
{
    const uint32_t w = __float_as_uint(top);
    const int e = (int)(w >> 23) - 127 - ((w & 0x7fffffu) > 0x600000u ? 7 : 8);
    return __uint_as_float((uint32_t)(min(max(e, kLeast), kMost) + 127) << 23);
}

// x / scale for values on their way to e4m3: the product with the exact inverse for
// powers of two.
struct Quotient {
    float scale, inverse;
    bool power;
    __device__ __forceinline__ explicit Quotient(float s) : scale(s), inverse(1.f / s), power((__float_as_uint(s) & 0x7fffffu) == 0) {}
    __device__ __forceinline__ float operator()(float x) const { return power ? x * inverse : x / scale; }
};

// Four values to e4m3, the first one lowest.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

__device__ __forceinline__ uint8_t to_e4m3(float a) { return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, a, 0, false); }

constexpr uint32_t kNan8 = 0x7f;

// ---- segments --------------------------------------------------------------------------
struct Segment {
    int64_t row;       // packed row of its first token
    int32_t count;     // tokens; 0: none
    int32_t before;    // older rows of the block
    int64_t at;        // element offset of the block's first row in the cache, head 0
    int64_t scale;     // offset of its scale, head 0
};

__device__ __forceinline__ int64_t candidate_of(const Append8Args& a, int b) { return (int64_t)a.step.q_start[b] / a.cache8.block + 2 * (int64_t)b; }

// Candidate c's segment, by a whole wavefront.
__device__ __forceinline__ Segment segment_of(const Append8Args& a, int64_t c, int lane)
{
    Segment s{};
    // the last sequence whose candidates begin at or before c, 64 probes a step
    int lo = 0, hi = a.step.seqs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const bool le = at < hi && candidate_of(a, at) <= c;
        const int n = __builtin_popcountll(__ballot(le));
        if (n == 0) break;
        hi = min(hi, lo + n * step);
        lo += (n - 1) * step;
    }
    const int b = __builtin_amdgcn_readfirstlane(lo);
    const int64_t i = c - candidate_of(a, b);
    const int64_t q0 = min(max((int64_t)a.step.q_start[b], (int64_t)0), a.tokens);
    const int64_t q1 = min(max((int64_t)a.step.q_start[b + 1], q0), a.tokens);
    const int64_t kv = a.step.kv_len[b], p0 = max(kv - (q1 - q0), (int64_t)0);
    const int64_t block = a.cache8.block, number = p0 / block + i;
    const int64_t first = max(p0, number * block), last = min(kv, (number + 1) * block);
    if (i < 0 || q1 == q0 || first >= last || first >= (int64_t)a.step.table_width * a.cache8.page_size) return s;
    const int32_t slot = (int32_t)(first / a.cache8.page_size);
    const int32_t page = a.step.table[(int64_t)b * a.step.table_stride + slot];
    if (page < 0 || page >= a.cache8.pages) return s;
    const int32_t row = (int32_t)(number * block - (int64_t)slot * a.cache8.page_size);      // of the page
    s.row = uniform(q1 - (kv - first));
    s.count = __builtin_amdgcn_readfirstlane((int)(last - first));
    s.before = __builtin_amdgcn_readfirstlane((int)(first - number * block));
    s.at = uniform((int64_t)page * a.cache8.page + (int64_t)row * a.cache8.token);
    s.scale = uniform((int64_t)page * a.cache8.scale_page + (int64_t)(row / a.cache8.block) * a.cache8.scale_block);
    return s;
}

// The block's scale from its new tokens' largest element and the older tokens' scale.
__device__ __forceinline__ float new_scale(float top, bool older, float old)
{
    return older && top <= kTop * old ? old : scale_for_top(top);
}

// ---- any head: a wavefront a segment, head and side, element by element ------------------
template <typename E>
__device__ __forceinline__ void load_any(const Append8Args& a, AnyHead<E>& x, int kind, int64_t t, int h, int lane)
{
    x.load(a, static_cast<const E*>(a.in[kind].p) + t * a.in[kind].token + (int64_t)h * a.in[kind].head, lane);
    if (kind == 2) return;
    if (a.norm) {
        AnyHead<E> w;
        if (a.w[1]) w.load(a, static_cast<const E*>(a.w[1]), lane);
        else w.fill(1.f);
        float z;
        const float r = x.inverse(a, z);
        x.each(w, [&](float v, float m) { return v * r * m; });
    }
    x.rotate(a, t, lane, false);
}

template <typename E>
__global__ __launch_bounds__(256) void append8_any_kernel(Append8Args a, int64_t first)
{
    const int lane = threadIdx.x & 63, units = 2 * a.heads[1];
    const int64_t u = first + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (u >= a.candidates * units) return;
    const int64_t c = u / units;
    const int in = (int)(u - c * units), kind = 1 + in % 2, h = in / 2;
    const Segment s = segment_of(a, c, lane);
    if (!s.count) return;
    uint8_t* cell = static_cast<uint8_t*>(kind == 1 ? a.cache8.k : a.cache8.v) + s.at + (int64_t)h * a.cache8.head;
    float* scale = (kind == 1 ? a.cache8.k_scale : a.cache8.v_scale) + s.scale + (int64_t)h * a.cache8.scale_head;
    const float old = *scale;
    float top = 0.f;
    for (int i = 0; i < s.count; ++i) {
        AnyHead<E> x;
        load_any(a, x, kind, s.row + i, h, lane);
        x.each(x, [&](float v, float) {
            if (finite(v)) top = fmaxf(top, fabsf(v));
            return v;
        });
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    const float now = new_scale(top, s.before > 0, old);
    if (lane == 0) *scale = now;
    if (s.before > 0 && now != old) {
        const float f = old / now;
        for (int r = 0; r < s.before; ++r)
            for (int e = lane; e < a.dim; e += 64) {
                uint8_t* p = cell + (int64_t)r * a.cache8.token + e;
                *p = to_e4m3(__builtin_amdgcn_cvt_f32_fp8(*p, 0) * f);
            }
    }
    const Quotient by(now);
    for (int i = 0; i < s.count; ++i) {
        AnyHead<E> x;
        load_any(a, x, kind, s.row + i, h, lane);
        uint8_t* p = cell + (int64_t)(s.before + i) * a.cache8.token;
        auto put = [&](int e, float v) { p[e] = finite(v) ? to_e4m3(by(v)) : (uint8_t)kNan8; };
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const int n = lane + 64 * j;
            if (n < a.rot / 2) {
                int ia, ib;
                AnyHead<E>::at(a, n, ia, ib);
                put(ia, x.a[j]);
                put(ib, x.b[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < kRest; ++j) {
            const int n = a.rot + lane + 64 * j;
            if (n < a.dim) put(n, x.r[j]);
        }
    }
}

template <typename E>
hipError_t append8(const Append8Args& a, hipStream_t s)
{
    constexpr int64_t kMostWaves = int64_t(1) << 25;
    const int64_t n = a.candidates * 2 * a.heads[1];
    hipError_t e = hipSuccess;
    for (int64_t first = 0; first < n && e == hipSuccess; first += kMostWaves) {
        hipLaunchKernelGGL(append8_any_kernel<E>, dim3((unsigned)((std::min(kMostWaves, n - first) + 3) / 4)), dim3(256), 0, s, a, first);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

hipError_t launch_append8(const Append8Args& args, bool bf16, hipStream_t s)
{
    Append8Args a = args;
    a.candidates = a.tokens / a.cache8.block + 2 * (int64_t)a.step.seqs;
    if (a.heads[0]) {
        RotateArgs q = a;
        q.heads[1] = q.heads[2] = 0;
        const hipError_t e = launch_rotate(q, bf16, s);
        if (e != hipSuccess) return e;
    }
    return bf16 ? append8<uint16_t>(a, s) : append8<float>(a, s);
}

}  // namespace tr
