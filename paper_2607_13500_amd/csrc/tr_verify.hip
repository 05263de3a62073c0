// Verification of drafted tokens: how many of a sequence's drafts are accepted, and the
// token drawn behind them by the inverse of the weights' sums.
//
// Of all rows only one of each sequence is read whole, the one that is drawn from:
// the drafts before it cost two numbers each.  Its slices go to the wavefronts of several
// workgroups, which each add some up (and find out the row for themselves); in a
// second launch a wavefront a sequence adds up the slices and looks through the one in
// which the sum passes its mark.  Sums are in 64 bits: the drawn token is the one whose
// interval the mark falls into, and those of a large vocabulary are as small as the
// rounding of an fp32 sum.  Bound by the bytes of the row (of the target and of the
// draft).
#include "tr_step.h"
#include "tr_wave.h"

namespace tr {
namespace {

constexpr int kWaves = 4;                        // of a workgroup of the first launch
constexpr int kRun = 4;                          // slices of a wavefront, one after another
constexpr int kGroups = kSlices / (kWaves * kRun);   // workgroups of a sequence
constexpr int kAhead = 4;                        // steps of a slice whose loads are on their way at a time

// 16 bytes from any address that an element can have.
template <typename E>
struct __attribute__((packed, aligned(sizeof(E)))) Raw16 {
    uint32_t w[4];
};

template <typename E>
__device__ __forceinline__ float widen(E v)
{
    if constexpr (sizeof(E) == 2) return __uint_as_float((uint32_t)v << 16);
    else return v;
}

// What counts as a probability: positive and finite, else 0.
__device__ __forceinline__ float proper(float p) { return p > 0.f && p <= 3.40282347e38f ? p : 0.f; }

// The row that a sequence's token is drawn from, and what is subtracted from it: a row
// of the draft, one element, or nothing.
template <typename E>
struct Drawn {
    int64_t q0;
    int drafts;        // of the sequence
    int accepted;
    const E* p;        // nullptr: the sequence has no rows
    const E* q;        // or nullptr
    int certain;       // a token that the draft was sure of, or -1
};

// With so many drafts accepted.
template <typename E>
__device__ __forceinline__ Drawn<E> drawn_from(const VerifyArgs& a, int b, int accepted)
{
    Drawn<E> d{};
    d.certain = -1;
    const int64_t q0 = min(max((int64_t)a.q_start[b], (int64_t)0), a.rows);
    const int64_t q1 = min(max((int64_t)a.q_start[b + 1], q0), a.rows);
    d.q0 = q0;
    if (q1 == q0) return d;
    d.drafts = (int)(q1 - q0 - 1);
    d.accepted = __builtin_amdgcn_readfirstlane(accepted);
    const int64_t r = q0 + d.accepted;
    d.p = static_cast<const E*>(a.target) + r * a.ld_target;
    if (d.accepted < min(d.drafts, a.width - 1)) {
        if (a.draft) d.q = static_cast<const E*>(a.draft) + r * a.ld_draft;
        else d.certain = a.ids[r + 1];
    }
    return d;
}

// The same after looking at the drafts, by a whole wavefront.
template <typename E>
__device__ __forceinline__ Drawn<E> drawn_of(const VerifyArgs& a, int b, int lane)
{
    const int64_t q0 = min(max((int64_t)a.q_start[b], (int64_t)0), a.rows);
    const int64_t q1 = min(max((int64_t)a.q_start[b + 1], q0), a.rows);
    const E* target = static_cast<const E*>(a.target);
    const E* draft = static_cast<const E*>(a.draft);
    const int most = (int)min(q1 - q0, (int64_t)a.width) - 1;
    int accepted = max(most, 0);
    for (int i0 = 0; i0 < most; i0 += 64) {
        const int i = i0 + lane;
        bool right = true;
        if (i < most) {
            const int64_t r = q0 + i;
            const int x = a.ids[r + 1];
            const bool in = x >= 0 && x < a.vocab;
            const float p = in ? proper(widen<E>(target[r * a.ld_target + x])) : 0.f;
            const float q = !in ? 0.f : draft ? proper(widen<E>(draft[r * a.ld_draft + x])) : 1.f;
            right = (double)a.accept[r] * (double)q < (double)p;
        }
        const uint64_t wrong = __ballot(!right);
        if (wrong) {
            accepted = i0 + __builtin_ctzll(wrong);
            break;
        }
    }
    return drawn_from<E>(a, b, accepted);
}

// Elements e .. e + N - 1 of the row as weights (those from `end` on are 0), and as
// the target's probabilities.
template <typename E>
constexpr int kVec = 16 / (int)sizeof(E);

template <typename E>
__device__ __forceinline__ void weights_at(const Drawn<E>& d, int e, int end, double (&w)[kVec<E>], double (&p)[kVec<E>])
{
    constexpr int N = kVec<E>;
    E x[N], y[N];
    if (e + N <= end) {
        const Raw16<E> v = *reinterpret_cast<const Raw16<E>*>(d.p + e);
        __builtin_memcpy(x, &v, 16);
        if (d.q) {
            const Raw16<E> u = *reinterpret_cast<const Raw16<E>*>(d.q + e);
            __builtin_memcpy(y, &u, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = e + i < end ? d.p[e + i] : E(0);
            y[i] = d.q && e + i < end ? d.q[e + i] : E(0);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = (double)proper(widen<E>(x[i]));
        const double q = d.q ? (double)proper(widen<E>(y[i])) : e + i == d.certain ? 1.0 : 0.0;
        w[i] = fmax(p[i] - q, 0.0);
    }
}

// Elements of a slice: whole pieces of 16 elements, so that aligned rows stay aligned.
__device__ __forceinline__ int slice_size(int vocab) { return ((vocab + kSlices - 1) / kSlices + 15) & ~15; }

// Sums over the wavefront's lanes up to each one.
__device__ __forceinline__ double dpp(double x, int m)
{
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)dpp_u32((uint32_t)(v >> 32), m) << 32 | dpp_u32((uint32_t)v, m));
}

__device__ __forceinline__ double upto(double x)
{
    x += dpp(x, 1);
    x += dpp(x, 2);
    x += dpp(x, 4);
    x += dpp(x, 8);
    x += dpp(x, 15);
    x += dpp(x, 31);
    return x;
}

__device__ __forceinline__ double lane_of(double x, int i)
{
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 |
                                          (uint32_t)__builtin_amdgcn_readlane((int)v, i));
}

__device__ __forceinline__ int last_of(uint64_t lanes) { return 63 - __builtin_clzll(lanes); }

template <typename E>
__global__ __launch_bounds__(kWaves * 64) void verify_sum_kernel(VerifyArgs a)
{
    constexpr int N = kVec<E>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / kGroups, slice0 = ((blockIdx.x % kGroups) * kWaves + wave) * kRun;
    const Drawn<E> d = drawn_of<E>(a, b, lane);
    if (slice0 == 0 && lane == 0) a.accepted[b] = d.accepted;
    if (!d.p) return;
    const int size = slice_size(a.vocab);
    double sw[kRun] = {}, sp[kRun] = {};
    for (int at = lane * N; at < size; at += 64 * N) {
        double w[kRun][N], p[kRun][N];
#pragma unroll
        for (int r = 0; r < kRun; ++r) {
            const int begin = (slice0 + r) * size;
            weights_at<E>(d, begin + at, min(begin + size, a.vocab), w[r], p[r]);
        }
#pragma unroll
        for (int r = 0; r < kRun; ++r)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sw[r] += w[r][i];
                sp[r] += p[r][i];
            }
    }
#pragma unroll
    for (int r = 0; r < kRun; ++r) {
        sw[r] = lane_of(upto(sw[r]), 63);
        sp[r] = lane_of(upto(sp[r]), 63);
    }
    double2* part = reinterpret_cast<double2*>(a.part) + (int64_t)b * kSlices + slice0;
#pragma unroll
    for (int r = 0; r < kRun; ++r)
        if (lane == r) part[r] = double2{sw[r], sp[r]};
}

// A wavefront a sequence; each lane has the sums of kPer slices after another.
constexpr int kPer = kSlices / 64;

template <typename E>
__global__ __launch_bounds__(64) void verify_draw_kernel(VerifyArgs a)
{
    constexpr int N = kVec<E>;
    const int lane = threadIdx.x, b = blockIdx.x;
    double2 part[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) part[i] = reinterpret_cast<const double2*>(a.part)[(int64_t)b * kSlices + lane * kPer + i];
    const float u = a.draw[b];
    const Drawn<E> d = drawn_from<E>(a, b, a.accepted[b]);
    int32_t* tokens = a.tokens + (int64_t)b * a.width;
    int word = 0;
    if (d.p) {
        double w = 0.0, p = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            w += part[i].x;
            p += part[i].y;
        }
        const double all_w = upto(w), all_p = upto(p);
        const bool whole = !(lane_of(all_w, 63) > 0.0);  // nothing is left: drawn from the target itself
        const double own = whole ? p : w, end = whole ? all_p : all_w, total = lane_of(end, 63);
        const double mark = (double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f) * total;
        // The first lane, slice, and in the end token, at whose end the sum is past the
        // mark.  Sums are rounded, each by its own order of additions: where none is past it
        // (of a part whose end was), it is the last with a weight.
        const uint64_t some = __ballot(own > 0.0), past = __ballot(own > 0.0 && end > mark);
        if (some) {
            const int at = past ? __builtin_ctzll(past) : last_of(some);
            double sum = lane_of(end, at) - lane_of(own, at);
            int slice = 0;
            double before = sum;
            bool found = false;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const double v = lane_of(whole ? part[i].y : part[i].x, at);
                if (v > 0.0 && !found) {
                    slice = i;
                    before = sum;
                    found = sum + v > mark;
                }
                sum += v;
            }
            const int size = slice_size(a.vocab), begin = (at * kPer + slice) * size, limit = min(begin + size, a.vocab);
            sum = before;
            int last = -1;                               // of the slice's tokens with a weight
            word = -1;
            for (int e0 = begin; e0 < limit && word < 0; e0 += 64 * N * kAhead) {
                double x[kAhead][N];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    double y[N];
                    weights_at<E>(d, e0 + (k * 64 + lane) * N, limit, x[k], y);
#pragma unroll
                    for (int i = 0; i < N; ++i) x[k][i] = whole ? y[i] : x[k][i];
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int e = e0 + (k * 64 + lane) * N;
                    double mine = 0.0;
                    int top = -1;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        mine += x[k][i];
                        if (x[k][i] > 0.0) top = e + i;
                    }
                    const double ends = sum + upto(mine);
                    const uint64_t over = __ballot(mine > 0.0 && ends > mark), any = __ballot(top >= 0);
                    if (over && word < 0) {
                        double s = ends - mine;
                        int found = top;
#pragma unroll
                        for (int i = N - 1; i >= 0; --i) {
                            double t = s;
#pragma unroll
                            for (int j = 0; j <= i; ++j) t += x[k][j];
                            if (x[k][i] > 0.0 && t > mark) found = e + i;
                        }
                        word = __builtin_amdgcn_readlane(found, __builtin_ctzll(over));
                    }
                    if (any) last = __builtin_amdgcn_readlane(top, last_of(any));
                    sum = lane_of(ends, 63);
                }
            }
            if (word < 0) word = max(last, 0);
        }
    }
    const bool any = d.p != nullptr;
    for (int i = lane; i < a.width; i += 64)
        tokens[i] = !any ? -1 : i < d.accepted ? a.ids[d.q0 + 1 + i] : i == d.accepted ? word : -1;
    if (lane == 0) a.change[b] = any ? d.accepted - d.drafts : 0;
}

template <typename E>
hipError_t verify(const VerifyArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL(verify_sum_kernel<E>, dim3((unsigned)a.seqs * kGroups), dim3(kWaves * 64), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_draw_kernel<E>, dim3((unsigned)a.seqs), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, bool bf16, hipStream_t s) { return bf16 ? verify<uint16_t>(a, s) : verify<float>(a, s); }

}  // namespace tr
