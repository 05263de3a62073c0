// Internal declarations of the language model's side: positions, rotated
// heads, the paged cache and attention over it.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tr.h"
#include "tr_divide.h"

namespace tr {

constexpr int kMaxHeadDim = 256;
constexpr int kMaxAxes = 4;

// ---- positions of kept tokens ------------------------------------------------
constexpr int kPosImages = 64;   // images of one launch (their descriptors are kernel arguments)

struct PosImage {
    int64_t src;       // first kept token of the image in idx
    int64_t dst;       // its column of pos
    int32_t count;
    int32_t hw, w;     // tokens of a frame and of a row of it
    int32_t start[3];
};

struct PosArgs {
    const int32_t* idx;
    int32_t* pos;
    int64_t ldpos;
    PosImage image[kPosImages];
};

hipError_t launch_positions(const PosArgs& a, int images, int most, hipStream_t s);

// ---- norm and rotation of heads ----------------------------------------------
struct RotateArgs {
    int64_t tokens;
    int32_t heads[3];          // query, key and value heads of a token (0: left out)
    int32_t dim, rot;
    int32_t axes;
    bool adjacent, norm;
    float eps;
    tr_heads in[3];            // queries, keys, values (backward: the inputs q, k)
    tr_heads out[3];           // where they go; in an append call keys and values go to the cache
    tr_heads grad[2];          // backward: gradients of the outputs
    const void* w[2];          // norm weights of queries and keys, or nullptr: 1
    const int32_t* pos;        // [axes, ldpos]
    int64_t ldpos;
    const float* freq;         // [rot / 2] angle per position
    const int32_t* pair_axis;  // [rot / 2]
    float* part;               // backward: partial sums of dw
    float* dw[2];              // backward: sums, or nullptr
    int32_t cus;
    bool append;
    tr_cache cache;
    tr_step step;
};

// An append call on a cache of 8-bit values.  `cache` has no memory: its pages and rows
// say which queries belong to a sequence.
struct Append8Args : RotateArgs {
    tr_cache8 cache8;
    int64_t candidates;        // of segments; filled in by the launch
};

hipError_t launch_append8(const Append8Args& a, bool bf16, hipStream_t s);

// Floats of RotateArgs::part for head_dim dim on a device of cus compute units.
size_t rotate_part_floats(int dim, int cus);
hipError_t launch_rotate(const RotateArgs& a, bool bf16, hipStream_t s);
hipError_t launch_rotate_backward(const RotateArgs& a, bool bf16, hipStream_t s);

// ---- attention ---------------------------------------------------------------
struct AttendArgs {
    int64_t tokens;
    int32_t heads, kv_heads, dim;
    int32_t group;             // heads / kv_heads
    Divisor by_group, by_page;
    int32_t most;              // tokens that a row of the table has pages for
    float* part;               // attend_part_floats of scratch
    int32_t* arrived;          // attend_groups counts, zero between calls
    tr_heads q, out;
    tr_cache cache;
    tr_step step;
    float raw_scale;           // of the scores
    float scale;               // the same in powers of two
    uint32_t keep, flip;       // 0: scale is 0, q counts as 0; bits of q to flip, where scale has to be > 0
    int32_t causal, window;
    float* lse;                // [tokens, heads] or nullptr
    int32_t cus;
};

// Over a cache of 8-bit values.  `cache` has no memory: its pages and their size say
// where tokens lie.
struct Attend8Args : AttendArgs {
    tr_cache8 cache8;
    Divisor by_block;
};

// group, the divisors, most, scale, keep and flip are filled in by the launch.
size_t attend_part_floats(int dim, int cus);
size_t attend_groups(int cus);
hipError_t launch_attend(const AttendArgs& a, hipStream_t s);
hipError_t launch_attend8(const Attend8Args& a, hipStream_t s);

// ---- device helpers ------------------------------------------------------------
// A value that is the same in all lanes, as a scalar.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// Sequence of packed row t: the last b with q_start[b] <= t, clamped to
// [0, seqs - 1], by one wavefront (64 probes a step).
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int seqs, int64_t t, int lane)
{
    int lo = 0, hi = seqs;   // the answer's first index past it lies in (lo, hi]
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64;
        const int at = lo + lane * step;
        const bool le = at < hi && (int64_t)q_start[at] <= t;
        const int n = __builtin_popcountll(__ballot(le));
        if (n == 0) return lo;
        hi = min(hi, lo + n * step);
        lo += (n - 1) * step;
    }
    const int at = lo + lane;
    const bool le = at < hi && (int64_t)q_start[at] <= t;
    const int n = __builtin_popcountll(__ballot(le));
    return n ? lo + n - 1 : lo;
}

}  // namespace tr
