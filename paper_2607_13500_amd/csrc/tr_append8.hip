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
    int32_t in_page;   // the block's first row in its page
    const int32_t* page;
};

__device__ __forceinline__ int64_t candidate_of(const Append8Args& a, int32_t start, int b) { return start / a.cache8.block + 2 * (int64_t)b; }

// Candidate c's segment, by a whole wavefront.
__device__ __forceinline__ Segment segment_of(const Append8Args& a, int64_t c, int lane)
{
    // the last sequence whose candidates begin at or before c, 64 probes a step; in the
    // last step each lane has what its sequence says
    int lo = 0, hi = a.step.seqs;
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const bool le = at < hi && candidate_of(a, a.step.q_start[at], at) <= c;
        const int n = __builtin_popcountll(__ballot(le));
        if (n == 0) break;
        hi = min(hi, lo + n * step);
        lo += (n - 1) * step;
    }
    const int at = min(lo + lane, a.step.seqs - 1);
    const int32_t start = a.step.q_start[at], next = a.step.q_start[at + 1], length = a.step.kv_len[at];
    const int n = __builtin_popcountll(__ballot(lo + lane < hi && candidate_of(a, start, at) <= c));
    const int from = max(n - 1, 0), b = lo + from;
    const int32_t first_row = __builtin_amdgcn_readlane(start, from), kv = __builtin_amdgcn_readlane(length, from);
    const int64_t q0 = min(max((int64_t)first_row, (int64_t)0), a.tokens);
    const int64_t q1 = min(max((int64_t)__builtin_amdgcn_readlane(next, from), q0), a.tokens);
    const int64_t i = c - candidate_of(a, first_row, b), p0 = max(kv - (q1 - q0), (int64_t)0);
    const int64_t block = a.cache8.block, number = p0 / block + i;
    const int64_t first = max(p0, number * block), last = min((int64_t)kv, (number + 1) * block);
    Segment s{};
    if (i < 0 || q1 == q0 || first >= last || first >= (int64_t)a.step.table_width * a.cache8.page_size) return s;
    const int32_t slot = (int32_t)(first / a.cache8.page_size);
    s.row = q1 - (kv - first);
    s.count = (int32_t)(last - first);
    s.before = (int32_t)(first - number * block);
    s.in_page = (int32_t)(number * block - (int64_t)slot * a.cache8.page_size);
    s.page = a.step.table + (int64_t)b * a.step.table_stride + slot;
    return s;
}

// Where it goes: element offset of the block's first row in the cache and offset of its
// scale, of head 0.
struct Target {
    int64_t at, scale;
};

__device__ __forceinline__ Target target_of(const Append8Args& a, const Segment& s, int32_t page)
{
    return {(int64_t)page * a.cache8.page + (int64_t)s.in_page * a.cache8.token,
            (int64_t)page * a.cache8.scale_page + (int64_t)(s.in_page / a.cache8.block) * a.cache8.scale_block};
}

// The block's scale from its new tokens' largest element and the older tokens' scale.
__device__ __forceinline__ float new_scale(float top, bool older, float old)
{
    return older && top <= kTop * old ? old : scale_for_top(top);
}

// ---- any head: a wavefront a segment, head and side, element by element ------------------
// Heads that are not whole pieces, and blocks that do not fit the registers of four
// wavefronts: the tokens one after another, twice.  Bound by the latency of that walk: 8
// prompts with 8 key heads of 100 in blocks of 32 take 244 us (of 104, in pieces, 40), of 128
// in blocks of 512 1.36 ms (of 256, in pieces, 57 us); 64 single tokens 16.
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
    const int32_t page = *s.page;
    if (page < 0 || page >= a.cache8.pages) return;
    const Target to = target_of(a, s, page);
    uint8_t* cell = static_cast<uint8_t*>(kind == 1 ? a.cache8.k : a.cache8.v) + to.at + (int64_t)h * a.cache8.head;
    float* scale = (kind == 1 ? a.cache8.k_scale : a.cache8.v_scale) + to.scale + (int64_t)h * a.cache8.scale_head;
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

// ---- heads of whole pieces ---------------------------------------------------------------
// A unit is a segment, head and side; LP lanes hold a token's head (see Piece), so that a
// wavefront takes 64 / LP tokens a round.  NW wavefronts share a unit's tokens and keep
// all their rounds in registers from the loads to the stores.  Its time is that of the
// loads that wait for one another (starts and lengths, elements beside the page, the old
// scale), so that many small units are better than few that walk over the heads with
// their angles kept (8 prompts, 9007 tokens together, 32 query and 8 key heads of 128:
// 49 us and 62).  Queries are the rotation kernel's work, done by workgroups of the same
// launch in turn with the units': they are bound by memory, the units by their latency
// and their angles (the same prompts 40 us, 4.4 TB/s; 50 with all queries first; 64
// tokens 6.6 us).  fp32 contexts, which move nearly twice the bytes: the prompts 73 us a
// call, bf16 44 to 47; 64 tokens 14 and 12.
// Sizes are compared as bits, in which what is not finite lies above all that is.
constexpr uint32_t kInfinite = 0x7f800000u;

__device__ __forceinline__ uint32_t size_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// A lane's elements in e4m3; `odd`: some of the unit are not finite.
template <bool ADJ>
__device__ __forceinline__ void words_of(const Piece& x, const Quotient& by, bool odd, uint32_t& w0, uint32_t& w1)
{
    float v[2 * kPiece];
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        v[ADJ ? 2 * e : e] = x.a[e];
        v[ADJ ? 2 * e + 1 : kPiece + e] = x.b[e];
    }
    w0 = to_e4m3(by(v[0]), by(v[1]), by(v[2]), by(v[3]));
    w1 = to_e4m3(by(v[4]), by(v[5]), by(v[6]), by(v[7]));
    if (odd) {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) {
            const uint32_t mask = 0xffu << (8 * e), nan = kNan8 << (8 * e);
            if (!finite(v[e])) w0 = (w0 & ~mask) | nan;
            if (!finite(v[kPiece + e])) w1 = (w1 & ~mask) | nan;
        }
    }
}

// Four e4m3 values times f, rounded again.
__device__ __forceinline__ uint32_t again(uint32_t w, float f)
{
    return to_e4m3(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * f, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * f,
                   __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * f, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * f);
}

// Of a launch's workgroups: those for queries and those for units, in turn as their
// numbers are to one another.
struct Turns {
    uint32_t queries, units;
};

__device__ __forceinline__ bool queries_turn(const Turns& t, uint32_t& at)
{
    const bool more = t.units >= t.queries;                      // units
    const uint32_t fewer = more ? t.queries : t.units;
    if (fewer == 0) return !more;
    const uint32_t each = (more ? t.units : t.queries) / fewer + 1, n = at / each;
    if (n >= fewer) {
        at -= fewer;
        return !more;
    }
    const bool its = at - n * each == 0;                         // the fewer ones' turn
    at = its ? n : at - n - 1;
    return its == more;
}

template <typename E, int LP, bool ADJ, int NW, int ROUNDS>
__global__ __launch_bounds__(256) void append8_kernel(Append8Args a, Turns all, int per, int chunks, bool stream, int64_t first)
{
    constexpr int R = 64 / LP;
    __shared__ uint32_t tops[4], some[4];
    const int lane = threadIdx.x & 63, j = lane & (LP - 1), hl = lane / LP;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t group = blockIdx.x;
    if (queries_turn(all, group)) {
        RotateArgs q = a;
        q.heads[1] = q.heads[2] = 0;
        if (stream) rotate_wave<E, LP, ADJ, true, true>(q, per, chunks, group * 4 + wave);
        else rotate_wave<E, LP, ADJ, true, false>(q, per, chunks, group * 4 + wave);
        return;
    }
    const int units = 2 * a.heads[1];
    const int64_t u = first + (NW == 1 ? (int64_t)group * 4 + wave : (int64_t)group);
    const int64_t c = u / units;
    if (c >= a.candidates) return;
    const int in = (int)(u - c * units), kind = 1 + in % 2, h = in / 2;
    const Segment s = segment_of(a, c, lane);
    if (!s.count) return;                     // the whole unit leaves together
    const int mine = NW == 1 ? 0 : wave;      // of the unit's wavefronts
    const Spot sp = spot_of<ADJ>(j, a.dim, a.rot);
    const char* from = static_cast<const char*>(a.in[kind].p) + (s.row * a.in[kind].token + (int64_t)h * a.in[kind].head) * (int)sizeof(E);
    const int64_t row_bytes = a.in[kind].token * (int)sizeof(E);
    Raw<E> x0[ROUNDS], x1[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i0 = (r * NW + mine) * R;
        if (i0 + hl < s.count && sp.on) {
            const char* p = from + (int64_t)i0 * row_bytes;
            const uint32_t at = (uint32_t)hl * (uint32_t)row_bytes;
            x0[r] = load(reinterpret_cast<const E*>(p + (at + sp.e0 * (uint32_t)sizeof(E))));
            x1[r] = load(reinterpret_cast<const E*>(p + (at + sp.e1 * (uint32_t)sizeof(E))));
        }
    }
    const int32_t page = *s.page;
    const Spin spin = spin_of(a, j, sp.turns && kind == 1);
    Piece w;
    if (a.norm && kind == 1) w = load_weight<E, ADJ>(a.w[1], sp);
    if (page < 0 || page >= a.cache8.pages) return;
    const Target to = target_of(a, s, page);
    uint8_t* cell = static_cast<uint8_t*>(kind == 1 ? a.cache8.k : a.cache8.v) + to.at + (int64_t)h * a.cache8.head;
    float* scale = (kind == 1 ? a.cache8.k_scale : a.cache8.v_scale) + to.scale + (int64_t)h * a.cache8.scale_head;
    const float old = *scale;
    const float mean = 1.f / (float)a.dim;
    Piece x[ROUNDS];
    uint32_t most = 0;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i0 = (r * NW + mine) * R;
        if (i0 >= s.count) break;
        const bool live = i0 + hl < s.count && sp.on;
        x[r] = unpack<E, ADJ>(x0[r], x1[r]);
        if (kind == 1) {
            if (a.norm) norm_piece<LP>(a, x[r], w, live, mean);
            if (sp.turns) {
                Turn z[kPiece];
                turns_of(a, spin, s.row + min(i0 + hl, s.count - 1), z);
                x[r] = turned(x[r], z);
            }
        }
        if (live) {
#pragma unroll
            for (int e = 0; e < kPiece; ++e) most = max(most, max(size_bits(x[r].a[e]), size_bits(x[r].b[e])));
        }
    }
    auto over_unit = [&](uint32_t v, uint32_t (&shared)[4]) {      // the largest
        v = wave_max_u32(v);
        if constexpr (NW > 1) {
            if (lane == 0) shared[wave] = v;
            __syncthreads();
            v = max(max(shared[0], shared[1]), max(shared[2], shared[3]));
        }
        return v;
    };
    most = over_unit(most, tops);
    const bool odd = most >= kInfinite;
    if (odd) {                                // again, of the finite ones
        most = 0;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int i0 = (r * NW + mine) * R;
            if (i0 >= s.count) break;
            if (i0 + hl < s.count && sp.on) {
#pragma unroll
                for (int e = 0; e < kPiece; ++e) {
                    if (finite(x[r].a[e])) most = max(most, size_bits(x[r].a[e]));
                    if (finite(x[r].b[e])) most = max(most, size_bits(x[r].b[e]));
                }
            }
        }
        most = over_unit(most, some);
    }
    const float top = __uint_as_float(most);
    const float now = new_scale(top, s.before > 0, old);
    if (lane == 0 && mine == 0) *scale = now;
    if (s.before > 0 && now != old && sp.on) {
        const float f = old / now;
        for (int i = mine * R + hl; i < s.before; i += NW * R) {
            uint8_t* p = cell + (int64_t)i * a.cache8.token;
            uint32_t* p0 = reinterpret_cast<uint32_t*>(p + sp.e0);
            uint32_t* p1 = reinterpret_cast<uint32_t*>(p + sp.e1);
            const uint32_t w0 = *p0, w1 = *p1;
            *p0 = again(w0, f);
            *p1 = again(w1, f);
        }
    }
    const Quotient by(now);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i0 = (r * NW + mine) * R;
        if (i0 >= s.count) break;
        if (i0 + hl < s.count && sp.on) {
            uint32_t w0, w1;
            words_of<ADJ>(x[r], by, odd, w0, w1);
            uint8_t* p = cell + (int64_t)(s.before + i0 + hl) * a.cache8.token;
            *reinterpret_cast<uint32_t*>(p + sp.e0) = w0;
            *reinterpret_cast<uint32_t*>(p + sp.e1) = w1;
        }
    }
}

// ---- launches ------------------------------------------------------------------------------
constexpr int64_t kMostGroups = int64_t(1) << 22;      // of a launch, which has fewer than 2^32 threads

template <typename E>
hipError_t append8_any(const Append8Args& a, hipStream_t s)
{
    const int64_t n = a.candidates * 2 * a.heads[1];
    hipError_t e = hipSuccess;
    for (int64_t first = 0; first < n && e == hipSuccess; first += 4 * kMostGroups) {
        hipLaunchKernelGGL(append8_any_kernel<E>, dim3((unsigned)((std::min(4 * kMostGroups, n - first) + 3) / 4)), dim3(256), 0, s, a, first);
        e = hipGetLastError();
    }
    return e;
}

template <typename E, int LP, int NW, int ROUNDS>
hipError_t append8_pieces(const Append8Args& a, bool with_queries, hipStream_t s)
{
    constexpr int R = 64 / LP;
    const int rounds = (a.heads[0] + R - 1) / R;
    const int per = a.tokens >= 16 * (int64_t)a.cus ? rounds : 1;               // as the rotation has it
    const int chunks = rounds ? (rounds + per - 1) / per : 0;
    const int64_t queries = with_queries ? (a.tokens * chunks + 3) / 4 : 0;
    const bool stream = a.tokens * a.heads[0] * a.dim * (int64_t)sizeof(E) >= (32 << 20);
    const int64_t units = a.candidates * 2 * a.heads[1], groups = NW == 1 ? (units + 3) / 4 : units;
    auto launch = [&](auto kernel) {
        hipError_t e = hipSuccess;
        for (int64_t at = 0; at < groups && e == hipSuccess; at += kMostGroups) {
            const Turns all{at == 0 ? (uint32_t)queries : 0u, (uint32_t)std::min(kMostGroups, groups - at)};
            hipLaunchKernelGGL(kernel, dim3(all.queries + all.units), dim3(256), 0, s, a, all, per, chunks, stream, at * (NW == 1 ? 4 : 1));
            e = hipGetLastError();
        }
        return e;
    };
    return a.adjacent ? launch(append8_kernel<E, LP, true, NW, ROUNDS>) : launch(append8_kernel<E, LP, false, NW, ROUNDS>);
}

// By the tokens of a block: one wavefront a unit, four, four with more in their registers.
template <typename E, int LP>
hipError_t append8_lanes(const Append8Args& a, bool with_queries, hipStream_t s)
{
    constexpr int R = 64 / LP;
    if (a.cache8.block <= 4 * R) return append8_pieces<E, LP, 1, 4>(a, with_queries, s);
    if (a.cache8.block <= 16 * R) return append8_pieces<E, LP, 4, 4>(a, with_queries, s);
    return append8_pieces<E, LP, 4, 16>(a, with_queries, s);
}

// Whether a round's tokens of a side lie within 2 GB and its pieces are whole.
template <typename E>
bool in_pieces(const tr_heads& x)
{
    return x.token * (int64_t)sizeof(E) <= INT32_MAX / 64 && x.head * (int64_t)sizeof(E) <= INT32_MAX / 64 &&
           ((uintptr_t)x.p | (uintptr_t)(x.token * (int64_t)sizeof(E)) | (uintptr_t)(x.head * (int64_t)sizeof(E))) % (kPiece * sizeof(E)) == 0;
}

template <typename E>
hipError_t append8(const Append8Args& a, hipStream_t s)
{
    const int lanes = a.dim / (2 * kPiece), most = lanes <= 8 ? 512 : lanes <= 16 ? 256 : 128;
    const bool pieces = a.dim % (2 * kPiece) == 0 && a.rot % (2 * kPiece) == 0 && a.cache8.block <= most && in_pieces<E>(a.in[1]) &&
                        in_pieces<E>(a.in[2]) && (uintptr_t)a.w[1] % (kPiece * sizeof(E)) == 0 &&
                        ((uintptr_t)a.cache8.k | (uintptr_t)a.cache8.v) % 4 == 0 && (a.cache8.page | a.cache8.token | a.cache8.head) % 4 == 0;
    const bool with = pieces && a.heads[0] && in_pieces<E>(a.in[0]) && in_pieces<E>(a.out[0]) && (uintptr_t)a.w[0] % (kPiece * sizeof(E)) == 0 &&
                      a.tokens * a.heads[0] < 4 * kMostGroups;
    if (a.heads[0] && !with) {
        RotateArgs q = a;
        q.heads[1] = q.heads[2] = 0;
        const hipError_t e = launch_rotate(q, sizeof(E) == 2, s);
        if (e != hipSuccess) return e;
    }
    if (!pieces) return append8_any<E>(a, s);
    return lanes <= 8 ? append8_lanes<E, 8>(a, with, s) : lanes <= 16 ? append8_lanes<E, 16>(a, with, s) : append8_lanes<E, 32>(a, with, s);
}

}  // namespace

hipError_t launch_append8(const Append8Args& args, bool bf16, hipStream_t s)
{
    Append8Args a = args;
    a.candidates = a.tokens / a.cache8.block + 2 * (int64_t)a.step.seqs;
    return bf16 ? append8<uint16_t>(a, s) : append8<float>(a, s);
}

}  // namespace tr
