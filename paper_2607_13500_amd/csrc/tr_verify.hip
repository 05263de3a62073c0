// Verification of drafted tokens: how many of a sequence's drafts are accepted, and the
// token drawn behind them by the inverse of the weights' sums.
//
// Of all rows only one of each sequence is read whole, the one that is drawn from:
// the drafts before it cost two numbers each.  Its 64 slices go to the wavefronts of
// several workgroups, which each add one up (and find out the row for themselves); a
// second launch adds up the slices, and one wavefront walks through the slice in
// which the sum passes its mark.  Sums are in 64 bits: the drawn token is the one whose
// interval the mark falls into, and those of a large vocabulary are as small as the
// rounding of an fp32 sum.  Bound by the bytes of the row (of the target and of the
// draft).
#include "tr_step.h"
#include "tr_wave.h"

namespace tr {
namespace {

constexpr int kWaves = 4;                        // of a workgroup of the first launch
constexpr int kGroups = kSlices / kWaves;        // workgroups of a sequence

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

// By a whole wavefront, the same in all its lanes.
template <typename E>
__device__ __forceinline__ Drawn<E> drawn_of(const VerifyArgs& a, int b, int lane)
{
    Drawn<E> d{};
    d.certain = -1;
    const int64_t q0 = min(max((int64_t)a.q_start[b], (int64_t)0), a.rows);
    const int64_t q1 = min(max((int64_t)a.q_start[b + 1], q0), a.rows);
    d.q0 = q0;
    if (q1 == q0) return d;
    const E* target = static_cast<const E*>(a.target);
    const E* draft = static_cast<const E*>(a.draft);
    d.drafts = (int)(q1 - q0 - 1);
    const int most = min(d.drafts, a.width - 1);
    d.accepted = most;
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
            d.accepted = i0 + __builtin_ctzll(wrong);
            break;
        }
    }
    d.accepted = __builtin_amdgcn_readfirstlane(d.accepted);
    const int64_t r = q0 + d.accepted;
    d.p = target + r * a.ld_target;
    if (d.accepted < most) {
        if (draft) d.q = draft + r * a.ld_draft;
        else d.certain = a.ids[r + 1];
    }
    return d;
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

template <typename E>
__global__ __launch_bounds__(kWaves * 64) void verify_sum_kernel(VerifyArgs a)
{
    constexpr int N = kVec<E>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / kGroups, slice = (blockIdx.x % kGroups) * kWaves + wave;
    const Drawn<E> d = drawn_of<E>(a, b, lane);
    if (!d.p) return;
    const int size = slice_size(a.vocab), begin = min((int64_t)slice * size, (int64_t)a.vocab), end = min((int64_t)begin + size, (int64_t)a.vocab);
    double sw = 0.0, sp = 0.0;
    for (int e = begin + lane * N; e < end; e += 64 * N) {
        double w[N], p[N];
        weights_at<E>(d, e, end, w, p);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            sw += w[i];
            sp += p[i];
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        sw += __shfl_xor(sw, m);
        sp += __shfl_xor(sp, m);
    }
    if (lane == 0) {
        double* part = a.part + ((int64_t)b * kSlices + slice) * 2;
        part[0] = sw;
        part[1] = sp;
    }
}

__device__ __forceinline__ double lane_of(double x, int i)
{
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 |
                                          (uint32_t)__builtin_amdgcn_readlane((int)v, i));
}

// A wavefront a sequence.
template <typename E>
__global__ __launch_bounds__(64) void verify_draw_kernel(VerifyArgs a)
{
    constexpr int N = kVec<E>;
    const int lane = threadIdx.x, b = blockIdx.x;
    const Drawn<E> d = drawn_of<E>(a, b, lane);
    int32_t* tokens = a.tokens + (int64_t)b * a.width;
    int word = 0;
    if (d.p) {
        // the sums up to each slice, one after another: what the next one adds is above 0
        // where its own sum is
        const double* part = a.part + ((int64_t)b * kSlices + lane) * 2;
        double w = part[0], p = part[1];
        double sw = 0.0, sp = 0.0, before_w = 0.0, before_p = 0.0;
        for (int i = 0; i < kSlices; ++i) {
            if (lane == i) {
                before_w = sw;
                before_p = sp;
            }
            sw += lane_of(w, i);
            sp += lane_of(p, i);
        }
        const bool whole = !(sw > 0.0);                  // nothing is left: drawn from the target itself
        const double total = whole ? sp : sw, before = whole ? before_p : before_w, mine = whole ? p : w;
        const double mark = (double)fminf(fmaxf(a.draw[b], 0.f), 0x1.fffffep-1f) * total;
        const uint64_t past = __ballot(before + mine > mark);
        if (past) {
            const int slice = __builtin_ctzll(past), size = slice_size(a.vocab);
            const int begin = slice * size, end = min(begin + size, a.vocab);
            double sum = __shfl(before, slice);
            int last = -1;                               // of the slice's tokens with a weight
            word = -1;
            for (int e0 = begin; e0 < end && word < 0; e0 += 64 * N) {
                double x[N], y[N];
                weights_at<E>(d, e0 + lane * N, end, x, y);
                double own = 0.0;
                int top = -1;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (whole) x[i] = y[i];
                    own += x[i];
                    if (x[i] > 0.0) top = e0 + lane * N + i;
                }
                double upto = own;
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) {
                    const double o = __shfl_up(upto, m);
                    if (lane >= m) upto += o;
                }
                const uint64_t over = __ballot(sum + upto > mark && own > 0.0);
                if (over) {
                    const int at = __builtin_ctzll(over);
                    double s = sum + (upto - own);
                    int found = top;
#pragma unroll
                    for (int i = N - 1; i >= 0; --i) {
                        double upto_i = s;
#pragma unroll
                        for (int j = 0; j <= i; ++j) upto_i += x[j];
                        if (x[i] > 0.0 && upto_i > mark) found = e0 + lane * N + i;
                    }
                    word = __shfl(found, at);
                }
                const uint64_t some = __ballot(top >= 0);
                if (some) last = __shfl(top, 63 - __builtin_clzll(some));
                sum += __shfl(upto, 63);
            }
            if (word < 0) word = max(last, 0);           // the sums' roundings: the last one before the mark
        }
    }
    const bool any = d.p != nullptr;
    for (int i = lane; i < a.width; i += 64)
        tokens[i] = !any ? -1 : i < d.accepted ? a.ids[d.q0 + 1 + i] : i == d.accepted ? word : -1;
    if (lane == 0) {
        a.accepted[b] = any ? d.accepted : 0;
        a.change[b] = any ? d.accepted - d.drafts : 0;
    }
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
