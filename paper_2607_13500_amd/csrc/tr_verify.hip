// Verification of drafted tokens: how many of a sequence's drafts are accepted, and the
// token drawn behind them by the inverse of the weights' sums.
//
// Of all rows only one of each sequence is read whole, the one that is drawn from:
// the drafts before it cost two numbers each.  Its slices go to the wavefronts of several
// workgroups, which each add some up (and find out the row for themselves); in a
// second launch a wavefront a sequence adds up the slices and looks through the one in
// which the sum passes its mark.  Sums are in 64 bits: the drawn token is the one whose
// interval the mark falls into, and those of a large vocabulary are as small as the
// rounding of an fp32 sum.  Bound by the bytes of the row, of the target and of the
// draft (64 sequences, 128000 fp32 words: 65.5 MB in 13.6 us, 4.8 TB/s, and the second
// launch 4.8 us).
#include "tr_step.h"
#include "tr_wave.h"

namespace tr {
namespace {

constexpr int kWaves = 4;                        // of a workgroup of the first launch
constexpr int kRun = 4;                          // slices of a wavefront, one after another
constexpr int kGroups = kSlices / (kWaves * kRun);   // workgroups of a sequence

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
__device__ __forceinline__ float proper(float p)
{
    constexpr int kSubnormal = 1 << 7, kNormal = 1 << 8;     // positive ones
    return __builtin_amdgcn_classf(p, kSubnormal | kNormal) ? p : 0.f;
}

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

template <typename E>
constexpr int kVec = 16 / (int)sizeof(E);
template <typename E>
constexpr int kAhead = 2 * (int)sizeof(E);       // steps whose loads are on their way at a time


// A lane's elements e .. e + N - 1 of the row, as they lie in memory; those from `end` on
// are 0.  `whole`: the target's alone.
struct Elements {
    uint32_t p[4], q[4];
};

template <typename E>
__device__ __forceinline__ void load16(const E* from, int e, int end, uint32_t (&w)[4])
{
    if (e + kVec<E> <= end) {
        const Raw16<E> v = *reinterpret_cast<const Raw16<E>*>(from + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v.w[i];
    } else {
        constexpr int EACH = kVec<E> / 4;    // elements of a word
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = 0;
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (e + i * EACH + k < end) w[i] |= __float_as_uint(widen<E>(from[e + i * EACH + k])) >> (EACH == 2 && k == 0 ? 16 : 0);
        }
    }
}

template <typename E>
__device__ __forceinline__ void load(const Drawn<E>& d, int e, int end, bool whole, Elements& x)
{
    load16(d.p, e, end, x.p);
    if (d.q && !whole) load16(d.q, e, end, x.q);
}

// Element i of those words as fp32.
template <typename E>
__device__ __forceinline__ float element(const uint32_t (&w)[4], int i)
{
    if constexpr (sizeof(E) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else return __uint_as_float(w[i]);
}

// Their weights, max(p - q, 0) = p - min(p, q): the minimum costs nothing in 64 bits.
template <typename E>
__device__ __forceinline__ void weigh(const Drawn<E>& d, int e, bool whole, const Elements& x, double (&w)[kVec<E>])
{
    constexpr int N = kVec<E>;
    if (d.q && !whole) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = proper(element<E>(x.p, i)), q = proper(element<E>(x.q, i));
            w[i] = (double)p - (double)fminf(p, q);
        }
    } else {
        const int certain = whole ? -1 : d.certain;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = proper(element<E>(x.p, i));
            w[i] = (double)p - (e + i == certain ? (double)fminf(p, 1.f) : 0.0);
        }
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

// The sum of a slice's weights, by a whole wavefront.
template <typename E>
__device__ __forceinline__ double sum_of(const Drawn<E>& d, int begin, int limit, bool whole, int lane)
{
    constexpr int N = kVec<E>;
    double sum = 0.0;
    for (int e0 = begin + lane * N; e0 < limit; e0 += 64 * N * kAhead<E>) {
        Elements x[kAhead<E>];
#pragma unroll
        for (int k = 0; k < kAhead<E>; ++k) load(d, e0 + k * 64 * N, limit, whole, x[k]);
#pragma unroll
        for (int k = 0; k < kAhead<E>; ++k) {
            double w[N];
            weigh(d, e0 + k * 64 * N, whole, x[k], w);
#pragma unroll
            for (int i = 0; i < N; ++i) sum += w[i];
        }
    }
    return lane_of(upto(sum), 63);
}

// The token of a slice, some of which have a weight, at which the sum passes the mark,
// `sum` being that of what is before the slice; by a whole wavefront.
template <typename E>
__device__ __forceinline__ int word_in(const Drawn<E>& d, int begin, int limit, double sum, double mark, bool whole, int lane)
{
    constexpr int N = kVec<E>;
    int last = 0;                            // of the tokens with a weight
    for (int e0 = begin; e0 < limit; e0 += 64 * N * kAhead<E>) {
        Elements y[kAhead<E>];
#pragma unroll
        for (int k = 0; k < kAhead<E>; ++k) load(d, e0 + (k * 64 + lane) * N, limit, whole, y[k]);
#pragma unroll
        for (int k = 0; k < kAhead<E>; ++k) {
            const int e = e0 + (k * 64 + lane) * N;
            double x[N], mine = 0.0;
            weigh(d, e, whole, y[k], x);
            int top = -1;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                mine += x[i];
                if (x[i] > 0.0) top = e + i;
            }
            const double ends = sum + upto(mine);
            const uint64_t over = __ballot(mine > 0.0 && ends > mark), any = __ballot(top >= 0);
            if (over) {
                const double s = ends - mine;
                int found = top;
#pragma unroll
                for (int i = N - 1; i >= 0; --i) {
                    double t = s;
#pragma unroll
                    for (int j = 0; j <= i; ++j) t += x[j];
                    if (x[i] > 0.0 && t > mark) found = e + i;
                }
                return __builtin_amdgcn_readlane(found, __builtin_ctzll(over));
            }
            if (any) last = __builtin_amdgcn_readlane(top, last_of(any));
            sum = lane_of(ends, 63);
        }
    }
    return last;
}

__device__ __forceinline__ double mark_of(float u, double total) { return (double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f) * total; }

// A sequence's results, by a wavefront.
template <typename E>
__device__ __forceinline__ void write_results(const VerifyArgs& a, const Drawn<E>& d, int b, int word, int lane)
{
    const bool any = d.p != nullptr;
    int32_t* tokens = a.tokens + (int64_t)b * a.width;
    for (int i = lane; i < a.width; i += 64)
        tokens[i] = !any ? -1 : i < d.accepted ? a.ids[d.q0 + 1 + i] : i == d.accepted ? word : -1;
    if (lane == 0) {
        a.accepted[b] = any ? d.accepted : 0;
        a.change[b] = any ? d.accepted - d.drafts : 0;
    }
}

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
    // weights, and the target's probabilities of slices without any: only they are asked
    // for where no slice has one
    double sw[kRun] = {}, sp[kRun] = {};
    for (int at = lane * N; at < size; at += 64 * N) {
        Elements x[kRun];
#pragma unroll
        for (int r = 0; r < kRun; ++r) load(d, (slice0 + r) * size + at, min((slice0 + r + 1) * size, a.vocab), false, x[r]);
#pragma unroll
        for (int r = 0; r < kRun; ++r) {
            double w[N];
            weigh(d, (slice0 + r) * size + at, false, x[r], w);
#pragma unroll
            for (int i = 0; i < N; ++i) sw[r] += w[i];
        }
    }
#pragma unroll
    for (int r = 0; r < kRun; ++r) {
        sw[r] = lane_of(upto(sw[r]), 63);
        const int begin = (slice0 + r) * size;
        if (!(sw[r] > 0.0)) sp[r] = sum_of<E>(d, begin, min(begin + size, a.vocab), true, lane);
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
    const int lane = threadIdx.x, b = blockIdx.x;
    double2 part[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) part[i] = reinterpret_cast<const double2*>(a.part)[(int64_t)b * kSlices + lane * kPer + i];
    const float u = a.draw[b];
    const Drawn<E> d = drawn_from<E>(a, b, a.accepted[b]);
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
        const double mark = mark_of(u, total);
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
            const int size = slice_size(a.vocab), begin = (at * kPer + slice) * size;
            word = word_in<E>(d, begin, min(begin + size, a.vocab), before, mark, whole, lane);
        }
    }
    write_results(a, d, b, word, lane);
}

// Rows of at most kOneWords: a workgroup a sequence, in one launch.  Each wavefront has
// one slice, of whose sums all wavefronts see where the mark falls.  Bound by one CU's
// 64-bit additions (a call of 1 to 64 sequences and a draft's words: 32000
// fp32 or bf16 words 13.3 us, 16.0 in two launches; 40000 words 15 to 18.4, and 16.0; 64000
// fp32 words 14.2 with one sequence, 16.9 with 16, 19.5 with 64, and 15.8.  256 sequences of
// 40000 words: 24.1 and 23.5 fp32, 19.1 and 33.8 bf16).
constexpr int kOneWaves = 16;
constexpr int kOneWords = 40000;

template <typename E>
__global__ __launch_bounds__(kOneWaves * 64) void verify_one_kernel(VerifyArgs a)
{
    __shared__ double sums[2][kOneWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = blockIdx.x;
    const float u = a.draw[b];
    const Drawn<E> d = drawn_of<E>(a, b, lane);
    if (!d.p) {                               // the whole workgroup leaves together
        if (wave == 0) write_results(a, d, b, 0, lane);
        return;
    }
    const int size = ((a.vocab + kOneWaves - 1) / kOneWaves + 15) & ~15, begin = min(wave * size, a.vocab), limit = min(begin + size, a.vocab);
    double own = 0.0, end = 0.0, total = 0.0;        // lane i: of slice i, and up to its end
    bool whole = false;
    for (;; whole = true) {
        const double sum = sum_of<E>(d, begin, limit, whole, lane);
        if (lane == 0) sums[whole][wave] = sum;
        __syncthreads();
        own = lane < kOneWaves ? sums[whole][lane & (kOneWaves - 1)] : 0.0;
        end = upto(own);
        total = lane_of(end, kOneWaves - 1);
        if (whole || total > 0.0) break;             // nothing is left: drawn from the target itself
    }
    const double mark = mark_of(u, total);
    // The first slice whose end is past the mark; where, by the sums' roundings, none
    // is, the last with a weight.
    const uint64_t some = __ballot(own > 0.0), past = __ballot(own > 0.0 && end > mark);
    const int at = past ? __builtin_ctzll(past) : some ? last_of(some) : 0;
    if (wave != at) return;
    const int word = some ? word_in<E>(d, begin, limit, lane_of(end, at) - lane_of(own, at), mark, whole, lane) : 0;
    write_results(a, d, b, word, lane);
}

template <typename E>
hipError_t verify(const VerifyArgs& a, hipStream_t s)
{
    if (a.vocab <= kOneWords) {
        hipLaunchKernelGGL(verify_one_kernel<E>, dim3((unsigned)a.seqs), dim3(kOneWaves * 64), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(verify_sum_kernel<E>, dim3((unsigned)a.seqs * kGroups), dim3(kWaves * 64), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_draw_kernel<E>, dim3((unsigned)a.seqs), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, bool bf16, hipStream_t s) { return bf16 ? verify<uint16_t>(a, s) : verify<float>(a, s); }

}  // namespace tr
