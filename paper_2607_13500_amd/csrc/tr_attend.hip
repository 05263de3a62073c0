// Attention of packed new tokens over a paged cache:
//   out = sum_j softmax_j(scale q . k_j) v_j  over the tokens that a row sees,
// in one pass over the keys with a running maximum m and sum l:  a block's
// weights are exp(s - m'), and what was summed before is scaled by exp(m - m').
#include "tr_attn.h"
#include "tr_wave.h"

namespace tr {
namespace {

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t narrow(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// One wavefront a (token, head): 64 keys at a time, one a lane, then the
// lane's elements of the head summed over them.
__global__ __launch_bounds__(64) void attend_simple_kernel(AttendArgs a)
{
    __shared__ float q[kMaxHeadDim];
    __shared__ float p[64];
    __shared__ int64_t row[64];
    const int lane = threadIdx.x;
    const int64_t t = blockIdx.x;
    const int h = blockIdx.y, g = h / (a.heads / a.kv_heads);
    const tr_step& st = a.step;
    if (st.seqs < 1 || t >= (int64_t)st.q_start[st.seqs] || t < (int64_t)st.q_start[0]) return;
    const int b = sequence_of(st.q_start, st.seqs, t, lane);
    const int64_t most = (int64_t)st.table_width * a.cache.page_size;
    const int64_t kv = min((int64_t)st.kv_len[b], most);
    const int64_t pos = (int64_t)st.kv_len[b] - ((int64_t)st.q_start[b + 1] - t);
    const int64_t end = a.causal ? min(kv, pos + 1) : kv;
    const int64_t begin = a.window > 0 ? max((int64_t)0, pos - a.window + 1) : 0;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q.p) + t * a.q.token + (int64_t)h * a.q.head;
    for (int j = lane; j < a.dim; j += 64) q[j] = widen(qp[j]) * a.scale;
    __syncthreads();
    float m = -__builtin_huge_valf(), l = 0.f;
    float o[kMaxHeadDim / 64] = {};
    for (int64_t j0 = begin; j0 < end; j0 += 64) {
        const int64_t j = j0 + lane;
        float s = -__builtin_huge_valf();
        int64_t at = 0;
        if (j < end) {
            const int64_t slot = j / a.cache.page_size;
            int32_t page = st.table[(int64_t)b * st.table_stride + slot];
            page = min(max(page, 0), a.cache.pages - 1);
            at = (int64_t)page * a.cache.page + (j - slot * a.cache.page_size) * a.cache.token + (int64_t)g * a.cache.head;
            const uint16_t* k = static_cast<const uint16_t*>(a.cache.k) + at;
            s = 0.f;
            for (int d = 0; d < a.dim; ++d) s = fmaf(q[d], widen(k[d]), s);
        }
        float top = s;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float m1 = fmaxf(m, top), base = m1 == -__builtin_huge_valf() ? 0.f : m1;
        const float w = expf(s - base), keep = expf(m - base);
        float sum = w;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
        m = m1;
        l = l * keep + sum;
        p[lane] = w;
        row[lane] = at;
        __syncthreads();
        const int n = (int)min((int64_t)64, end - j0);
#pragma unroll
        for (int i = 0; i < kMaxHeadDim / 64; ++i) {
            const int d = lane + 64 * i;
            if (d < a.dim) {
                o[i] *= keep;
                for (int u = 0; u < n; ++u) o[i] = fmaf(p[u], widen(static_cast<const uint16_t*>(a.cache.v)[row[u] + d]), o[i]);
            }
        }
        __syncthreads();
    }
    uint16_t* op = static_cast<uint16_t*>(a.out.p) + t * a.out.token + (int64_t)h * a.out.head;
#pragma unroll
    for (int i = 0; i < kMaxHeadDim / 64; ++i)
        if (lane + 64 * i < a.dim) op[lane + 64 * i] = narrow(l > 0.f || l != l ? o[i] / l : 0.f);
    if (a.lse && lane == 0) a.lse[t * a.heads + h] = l > 0.f || l != l ? m + logf(l) : -__builtin_huge_valf();
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, hipStream_t s)
{
    if (a.tokens < 1) return hipSuccess;
    hipLaunchKernelGGL(attend_simple_kernel, dim3((unsigned)a.tokens, (unsigned)a.heads), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace tr
