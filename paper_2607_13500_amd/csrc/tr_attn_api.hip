// The language model's side of the C ABI of include/tr.h: validation, the
// rotation's tables, scratch ownership and launches.
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <new>
#include <utility>

#include "tr.h"
#include "tr_attn.h"
#include "tr_host.h"

using tr::aligned16;
using tr::clear_error;
using tr::CtxAlloc;
using tr::DeviceGuard;
using tr::elem_bytes;
using tr::fail;
using tr::hip_fail;
using tr::log_line;
using tr::Range;

struct tr_attn {
    tr_attn_params p{};
    int device = 0;
    int eb = 4;
    int cus = 256;
    float* freq = nullptr;          // [rot_dim / 2], see RotateArgs
    int32_t* pair_axis = nullptr;   // [rot_dim / 2]
    float* part = nullptr;          // partial sums of dw
    float* parts = nullptr;         // parts of rows that several workgroups attend for (bf16)
    int32_t* arrived = nullptr;     // and how many of an item's are there
};

namespace {

constexpr int64_t kMaxTokens = INT32_MAX;

tr_status check_attn_params(const tr_attn_params* p)
{
    if (!p) return fail(TR_EINVAL, "params is NULL");
    if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads)
        return fail(TR_EINVAL, "heads must be a positive multiple of kv_heads (got %d and %d)", p->heads, p->kv_heads);
    if (p->heads > 65535) return fail(TR_EINVAL, "heads must be at most 65535 (got %d)", p->heads);
    if (p->head_dim < 1 || p->head_dim > tr::kMaxHeadDim)
        return fail(TR_EINVAL, "head_dim must be in [1, %d] (got %d)", tr::kMaxHeadDim, p->head_dim);
    if (p->rot_dim < 0 || p->rot_dim > p->head_dim || p->rot_dim % 2)
        return fail(TR_EINVAL, "rot_dim must be even and in [0, head_dim] (got %d)", p->rot_dim);
    if (p->axes < 1 || p->axes > tr::kMaxAxes)
        return fail(TR_EINVAL, "axes must be in [1, %d] (got %d)", tr::kMaxAxes, p->axes);
    if (p->adjacent != 0 && p->adjacent != 1) return fail(TR_EINVAL, "adjacent must be 0 or 1 (got %d)", p->adjacent);
    if (p->norm != 0 && p->norm != 1) return fail(TR_EINVAL, "norm must be 0 or 1 (got %d)", p->norm);
    if (p->dtype != TR_FP32 && p->dtype != TR_BF16)
        return fail(TR_EINVAL, "dtype must be TR_FP32 or TR_BF16 (got %d)", p->dtype);
    if (p->norm && !(p->eps >= 0.0 && isfinite(p->eps))) return fail(TR_EINVAL, "eps must be finite and >= 0 (got %g)", p->eps);
    if (!p->inv_freq && p->rot_dim && !(p->base > 0.0 && isfinite(p->base)))
        return fail(TR_EINVAL, "base must be finite and > 0 (got %g)", p->base);
    for (int i = 0; i < p->rot_dim / 2; ++i) {
        if (p->inv_freq && !isfinite((float)p->inv_freq[i]))
            return fail(TR_EINVAL, "inv_freq[%d] is not finite in fp32", i);
        if (p->pair_axis && (p->pair_axis[i] < 0 || p->pair_axis[i] >= p->axes))
            return fail(TR_EINVAL, "pair_axis[%d] = %d must be in [0, %d)", i, p->pair_axis[i], p->axes);
    }
    return TR_OK;
}

// Whether rows of dim elements at the given strides (each with its count)
// can overlap: sorted by stride, each must step over all that lies below it.
bool rows_overlap(std::initializer_list<std::pair<int64_t, int64_t>> strides, int64_t dim)
{
    std::pair<int64_t, int64_t> v[3];
    int n = 0;
    for (const auto& s : strides)
        if (s.second > 1) v[n++] = s;
    std::sort(v, v + n);
    __int128 extent = dim;
    for (int i = 0; i < n; ++i) {
        if (v[i].first < extent) return true;
        extent += (__int128)v[i].first * (v[i].second - 1);
    }
    return false;
}

// An input's heads.  Strides of 0 (a broadcast input) are fine.
tr_status check_heads(const char* name, const tr_heads& x, int eb, int64_t T, int heads)
{
    if (!x.p) return fail(TR_EINVAL, "%s must be non-NULL", name);
    if ((uintptr_t)x.p & (uintptr_t)(eb - 1))
        return fail(TR_EUNSUPPORTED, "%s must be aligned to the element size (%d bytes)", name, eb);
    if ((heads > 1 && x.head < 0) || (T > 1 && x.token < 0)) return fail(TR_EINVAL, "%s has a negative stride", name);
    return TR_OK;
}

tr_status check_out_heads(const char* name, const tr_heads& x, int eb, int64_t T, int heads, int dim)
{
    tr_status st = check_heads(name, x, eb, T, heads);
    if (st != TR_OK) return st;
    if (rows_overlap({{x.token, T}, {x.head, heads}}, dim))
        return fail(TR_EINVAL, "%s has rows that overlap (strides %lld and %lld, rows of %d elements)", name,
                    (long long)x.token, (long long)x.head, dim);
    return TR_OK;
}

tr_status check_positions(const tr_attn* a, const int32_t* pos, int64_t ldpos)
{
    if (!a->p.rot_dim) return TR_OK;
    if (!pos) return fail(TR_EINVAL, "pos must be non-NULL");
    if ((uintptr_t)pos & 3u) return fail(TR_EUNSUPPORTED, "pos must be 4-byte aligned");
    if (a->p.axes > 1 && ldpos < 0) return fail(TR_EINVAL, "ldpos must be >= 0 (got %lld)", (long long)ldpos);
    return TR_OK;
}

tr_status check_weights(const tr_attn* a, const void* wq, const void* wk)
{
    if (!a->p.norm && (wq || wk)) return fail(TR_EINVAL, "norm weights need a context with norm");
    if (((uintptr_t)wq | (uintptr_t)wk) & (uintptr_t)(a->eb - 1))
        return fail(TR_EUNSUPPORTED, "wq and wk must be aligned to the element size (%d bytes)", a->eb);
    return TR_OK;
}

tr_status check_tokens(const tr_attn* a, int64_t T)
{
    if (!a) return fail(TR_EINVAL, "attn is NULL");
    if (T < 0 || T > kMaxTokens) return fail(TR_EINVAL, "T must be in [0, 2^31 - 1] (got %lld)", (long long)T);
    if (T * (a->p.heads + 2 * (int64_t)a->p.kv_heads) > kMaxTokens - 65536)
        return fail(TR_EUNSUPPORTED, "T = %lld tokens have more than 2^31 - 65536 heads", (long long)T);
    return TR_OK;
}

tr_status check_cache(const tr_attn* a, const tr_cache* c, const tr_step* s)
{
    if (!c || !s) return fail(TR_EINVAL, "cache and step must be non-NULL");
    if (c->pages < 1 || c->page_size < 1)
        return fail(TR_EINVAL, "the cache needs pages >= 1 and page_size >= 1 (got %d and %d)", c->pages, c->page_size);
    if (!c->k || !c->v) return fail(TR_EINVAL, "the cache's k and v must be non-NULL");
    if (((uintptr_t)c->k | (uintptr_t)c->v) & (uintptr_t)(a->eb - 1))
        return fail(TR_EUNSUPPORTED, "the cache must be aligned to the element size (%d bytes)", a->eb);
    const int64_t dim = a->p.head_dim;
    if (rows_overlap({{c->page, c->pages}, {c->token, c->page_size}, {c->head, a->p.kv_heads}}, dim))
        return fail(TR_EINVAL, "the cache has rows that overlap (strides %lld, %lld and %lld, rows of %lld elements)",
                    (long long)c->page, (long long)c->token, (long long)c->head, (long long)dim);
    if (s->seqs < 1) return fail(TR_EINVAL, "seqs must be >= 1 where there are tokens (got %d)", s->seqs);
    if (s->table_width < 0 || s->table_stride < 0)
        return fail(TR_EINVAL, "table_width = %d and table_stride = %lld must be >= 0", s->table_width,
                    (long long)s->table_stride);
    if (!s->q_start || !s->kv_len || (!s->table && s->table_width))
        return fail(TR_EINVAL, "q_start, kv_len and table must be non-NULL");
    if (((uintptr_t)s->q_start | (uintptr_t)s->kv_len | (uintptr_t)s->table) & 3u)
        return fail(TR_EUNSUPPORTED, "q_start, kv_len and table must be 4-byte aligned");
    return TR_OK;
}

// The fields that every call on heads shares.
tr::RotateArgs rotate_args(const tr_attn* a, int64_t T, const void* wq, const void* wk, const int32_t* pos, int64_t ldpos)
{
    tr::RotateArgs r{};
    r.tokens = T;
    r.dim = a->p.head_dim;
    r.rot = a->p.rot_dim;
    r.axes = a->p.axes;
    r.adjacent = a->p.adjacent != 0;
    r.norm = a->p.norm != 0;
    r.eps = (float)a->p.eps;
    r.w[0] = wq;
    r.w[1] = wk;
    r.pos = pos;
    r.ldpos = ldpos;
    r.freq = a->freq;
    r.pair_axis = a->pair_axis;
    r.part = a->part;
    r.cus = a->cus;
    return r;
}

}  // namespace

extern "C" {

tr_status tr_attn_create(const tr_attn_params* p, tr_attn** out)
{
    clear_error();
    if (!out) return fail(TR_EINVAL, "out is NULL");
    *out = nullptr;
    tr_status st = check_attn_params(p);
    if (st != TR_OK) return st;
    float freq[tr::kMaxHeadDim / 2] = {};
    int32_t axis[tr::kMaxHeadDim / 2] = {};
    const int pairs = p->rot_dim / 2;
    for (int i = 0; i < pairs; ++i) {
        freq[i] = (float)(p->inv_freq ? p->inv_freq[i] : pow(p->base, -(double)(2 * i) / (double)p->rot_dim));
        axis[i] = p->pair_axis ? p->pair_axis[i] : 0;
    }
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    tr_attn* a = new (std::nothrow) tr_attn;
    if (!a) return fail(TR_ENOMEM, "host allocation failed");
    a->p = *p;
    a->p.inv_freq = nullptr;    // the caller's arrays are read here only
    a->p.pair_axis = nullptr;
    a->device = dev;
    a->eb = elem_bytes(p->dtype);
    if ((e = hipDeviceGetAttribute(&a->cus, hipDeviceAttributeMultiprocessorCount, dev)) != hipSuccess) {
        tr_attn_destroy(a);
        return hip_fail(e, "hipDeviceGetAttribute");
    }
    CtxAlloc al;
    if ((e = al(&a->freq, sizeof freq)) != hipSuccess || (e = al(&a->pair_axis, sizeof axis)) != hipSuccess ||
        (e = al(&a->part, tr::rotate_part_floats(p->head_dim, a->cus) * sizeof(float))) != hipSuccess) {
        tr_attn_destroy(a);
        return fail(TR_ENOMEM, "hipMalloc of a layer's tables failed: %s", hipGetErrorString(e));
    }
    if (p->dtype == TR_BF16 && p->head_dim % 8 == 0 &&
        ((e = al(&a->parts, tr::attend_part_floats(p->head_dim, a->cus) * sizeof(float))) != hipSuccess ||
         (e = al(&a->arrived, tr::attend_groups(a->cus) * sizeof(int32_t))) != hipSuccess)) {
        tr_attn_destroy(a);
        return fail(TR_ENOMEM, "hipMalloc of a layer's scratch failed: %s", hipGetErrorString(e));
    }
    if ((e = hipMemcpy(a->freq, freq, sizeof freq, hipMemcpyHostToDevice)) != hipSuccess ||
        (e = hipMemcpy(a->pair_axis, axis, sizeof axis, hipMemcpyHostToDevice)) != hipSuccess ||
        (a->arrived && (e = hipMemset(a->arrived, 0, tr::attend_groups(a->cus) * sizeof(int32_t))) != hipSuccess) ||
        (e = hipDeviceSynchronize()) != hipSuccess) {
        tr_attn_destroy(a);
        return hip_fail(e, "scratch initialisation");
    }
    log_line("attention context on device %d: %d query and %d key heads of %d, %d rotated over %d axes, %s%s", dev,
             p->heads, p->kv_heads, p->head_dim, p->rot_dim, p->axes, p->dtype == TR_BF16 ? "bf16" : "fp32",
             p->norm ? ", normed" : "");
    *out = a;
    return TR_OK;
}

void tr_attn_destroy(tr_attn* a)
{
    if (!a) return;
    DeviceGuard g(a->device);
    if (a->freq) (void)hipFree(a->freq);
    if (a->pair_axis) (void)hipFree(a->pair_axis);
    if (a->part) (void)hipFree(a->part);
    if (a->parts) (void)hipFree(a->parts);
    if (a->arrived) (void)hipFree(a->arrived);
    delete a;
}

tr_status tr_kept_positions(const int32_t* idx, int32_t B, const int32_t* K, const int32_t* grid, const int32_t* start,
                            const int64_t* dst, int32_t* pos, int64_t ldpos, void* stream)
{
    clear_error();
    Range range("tr_kept_positions");
    if (B < 0) return fail(TR_EINVAL, "B must be >= 0 (got %d)", B);
    if (B == 0) return TR_OK;
    if (!K || !grid || !start) return fail(TR_EINVAL, "K, grid and start must be non-NULL");
    int64_t rows = 0;
    for (int32_t b = 0; b < B; ++b) {
        const int32_t* d = grid + 3 * (int64_t)b;
        if (K[b] < 0) return fail(TR_EINVAL, "K[%d] = %d must be >= 0", b, K[b]);
        if (d[0] < 1 || d[1] < 1 || d[2] < 1 || (int64_t)d[1] * d[2] > INT32_MAX ||
            (int64_t)d[1] * d[2] * d[0] > INT32_MAX)
            return fail(TR_EINVAL, "grid[%d] = (%d, %d, %d) must be positive and of at most 2^31 - 1 tokens", b, d[0], d[1], d[2]);
        const int64_t at = dst ? dst[b] : rows;
        if (at < 0 || at + K[b] > ldpos)
            return fail(TR_EINVAL, "columns %lld .. %lld of image %d lie outside [0, ldpos = %lld)", (long long)at,
                        (long long)(at + K[b]), b, (long long)ldpos);
        rows += K[b];
    }
    if (rows == 0) return TR_OK;
    if (!idx || !pos) return fail(TR_EINVAL, "idx and pos must be non-NULL");
    if (((uintptr_t)idx | (uintptr_t)pos) & 3u) return fail(TR_EUNSUPPORTED, "idx and pos must be 4-byte aligned");
    tr::PosArgs a{};
    a.idx = idx;
    a.pos = pos;
    a.ldpos = ldpos;
    int64_t src = 0;
    for (int32_t b0 = 0; b0 < B; b0 += tr::kPosImages) {
        const int n = std::min(B - b0, tr::kPosImages);
        int most = 0;
        for (int i = 0; i < n; ++i) {
            const int32_t b = b0 + i;
            tr::PosImage& im = a.image[i];
            im.src = src;
            im.dst = dst ? dst[b] : src;
            im.count = K[b];
            im.hw = grid[3 * (int64_t)b + 1] * grid[3 * (int64_t)b + 2];
            im.w = grid[3 * (int64_t)b + 2];
            for (int x = 0; x < 3; ++x) im.start[x] = start[3 * (int64_t)b + x];
            src += K[b];
            most = std::max(most, K[b]);
        }
        hipError_t e = tr::launch_positions(a, n, most, static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return hip_fail(e, "position kernel launch");
    }
    return TR_OK;
}

tr_status tr_rotate(tr_attn* a, int64_t T, tr_heads q, tr_heads k, const void* wq, const void* wk, const int32_t* pos,
                    int64_t ldpos, tr_heads q_out, tr_heads k_out, void* stream)
{
    clear_error();
    Range range("tr_rotate");
    tr_status st = check_tokens(a, T);
    if (st != TR_OK || T == 0) return st;
    if (!q.p && !k.p) return fail(TR_EINVAL, "nothing to rotate: q and k are NULL");
    const int dim = a->p.head_dim;
    if (q.p && ((st = check_heads("q", q, a->eb, T, a->p.heads)) != TR_OK ||
                (st = check_out_heads("q_out", q_out, a->eb, T, a->p.heads, dim)) != TR_OK))
        return st;
    if (k.p && ((st = check_heads("k", k, a->eb, T, a->p.kv_heads)) != TR_OK ||
                (st = check_out_heads("k_out", k_out, a->eb, T, a->p.kv_heads, dim)) != TR_OK))
        return st;
    if ((st = check_weights(a, wq, wk)) != TR_OK || (st = check_positions(a, pos, ldpos)) != TR_OK) return st;
    DeviceGuard g(a->device);
    if (!g.ok) return fail(TR_EDEVICE, "hipSetDevice(%d) failed", a->device);
    tr::RotateArgs r = rotate_args(a, T, wq, wk, pos, ldpos);
    r.heads[0] = q.p ? a->p.heads : 0;
    r.heads[1] = k.p ? a->p.kv_heads : 0;
    r.in[0] = q;
    r.in[1] = k;
    r.out[0] = q_out;
    r.out[1] = k_out;
    hipError_t e = tr::launch_rotate(r, a->p.dtype == TR_BF16, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "rotation kernel launch");
    return TR_OK;
}

tr_status tr_rotate_backward(tr_attn* a, int64_t T, tr_heads gq, tr_heads gk, tr_heads q, tr_heads k, const void* wq,
                             const void* wk, const int32_t* pos, int64_t ldpos, tr_heads dq, tr_heads dk, float* dwq,
                             float* dwk, void* stream)
{
    clear_error();
    Range range("tr_rotate_backward");
    tr_status st = check_tokens(a, T);
    if (st != TR_OK) return st;
    if (!a->p.norm && (dwq || dwk)) return fail(TR_EINVAL, "dwq and dwk need a context with norm");
    if (((uintptr_t)dwq | (uintptr_t)dwk) & 3u) return fail(TR_EUNSUPPORTED, "dwq and dwk must be 4-byte aligned");
    if (T > 0) {
        if (!gq.p && !gk.p) return fail(TR_EINVAL, "nothing to compute: gq and gk are NULL");
        if ((!gq.p && dwq) || (!gk.p && dwk)) return fail(TR_EINVAL, "dwq needs gq, and dwk needs gk");
        const tr_heads* side[2][3] = {{&gq, &q, &dq}, {&gk, &k, &dk}};
        const char* name[2][3] = {{"gq", "q", "dq"}, {"gk", "k", "dk"}};
        for (int i = 0; i < 2; ++i) {
            const int heads = i ? a->p.kv_heads : a->p.heads;
            if (!side[i][0]->p) continue;
            if ((st = check_heads(name[i][0], *side[i][0], a->eb, T, heads)) != TR_OK ||
                (a->p.norm && (st = check_heads(name[i][1], *side[i][1], a->eb, T, heads)) != TR_OK) ||
                (st = check_out_heads(name[i][2], *side[i][2], a->eb, T, heads, a->p.head_dim)) != TR_OK)
                return st;
        }
        if ((st = check_weights(a, wq, wk)) != TR_OK || (st = check_positions(a, pos, ldpos)) != TR_OK) return st;
    }
    if (T == 0 && !dwq && !dwk) return TR_OK;
    DeviceGuard g(a->device);
    if (!g.ok) return fail(TR_EDEVICE, "hipSetDevice(%d) failed", a->device);
    tr::RotateArgs r = rotate_args(a, T, wq, wk, pos, ldpos);
    r.heads[0] = gq.p ? a->p.heads : 0;
    r.heads[1] = gk.p ? a->p.kv_heads : 0;
    r.grad[0] = gq;
    r.grad[1] = gk;
    r.in[0] = q;
    r.in[1] = k;
    r.out[0] = dq;
    r.out[1] = dk;
    r.dw[0] = dwq;
    r.dw[1] = dwk;
    hipError_t e = tr::launch_rotate_backward(r, a->p.dtype == TR_BF16, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "rotation gradient launch");
    return TR_OK;
}

tr_status tr_append(tr_attn* a, int64_t T, tr_heads q, tr_heads k, tr_heads v, const void* wq, const void* wk,
                    const int32_t* pos, int64_t ldpos, tr_heads q_out, const tr_cache* c, const tr_step* s, void* stream)
{
    clear_error();
    Range range("tr_append");
    tr_status st = check_tokens(a, T);
    if (st != TR_OK || T == 0) return st;
    const int dim = a->p.head_dim;
    if ((st = check_cache(a, c, s)) != TR_OK || (st = check_heads("k", k, a->eb, T, a->p.kv_heads)) != TR_OK ||
        (st = check_heads("v", v, a->eb, T, a->p.kv_heads)) != TR_OK)
        return st;
    if (q.p && ((st = check_heads("q", q, a->eb, T, a->p.heads)) != TR_OK ||
                (st = check_out_heads("q_out", q_out, a->eb, T, a->p.heads, dim)) != TR_OK))
        return st;
    if ((st = check_weights(a, wq, wk)) != TR_OK || (st = check_positions(a, pos, ldpos)) != TR_OK) return st;
    DeviceGuard g(a->device);
    if (!g.ok) return fail(TR_EDEVICE, "hipSetDevice(%d) failed", a->device);
    tr::RotateArgs r = rotate_args(a, T, wq, wk, pos, ldpos);
    r.heads[0] = q.p ? a->p.heads : 0;
    r.heads[1] = r.heads[2] = a->p.kv_heads;
    r.in[0] = q;
    r.in[1] = k;
    r.in[2] = v;
    r.out[0] = q_out;
    r.append = true;
    r.cache = *c;
    r.step = *s;
    hipError_t e = tr::launch_rotate(r, a->p.dtype == TR_BF16, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "append kernel launch");
    return TR_OK;
}

tr_status tr_attend(tr_attn* a, int64_t T, tr_heads q, const tr_cache* c, const tr_step* s, double scale, int32_t causal,
                    int32_t window, tr_heads out, float* lse, void* stream)
{
    clear_error();
    Range range("tr_attend");
    tr_status st = check_tokens(a, T);
    if (st != TR_OK) return st;
    if (a->p.dtype != TR_BF16) return fail(TR_EUNSUPPORTED, "tr_attend needs a bf16 context");
    if (a->p.head_dim % 8) return fail(TR_EUNSUPPORTED, "tr_attend needs head_dim %% 8 == 0 (got %d)", a->p.head_dim);
    if (!isfinite((float)scale)) return fail(TR_EINVAL, "scale must be finite in fp32 (got %g)", scale);
    if (causal != 0 && causal != 1) return fail(TR_EINVAL, "causal must be 0 or 1 (got %d)", causal);
    if (window < 0 || (window > 0 && !causal))
        return fail(TR_EINVAL, "window must be >= 0, and 0 without causal (got %d)", window);
    if (T == 0) return TR_OK;
    const int dim = a->p.head_dim;
    if ((st = check_cache(a, c, s)) != TR_OK || (st = check_heads("q", q, a->eb, T, a->p.heads)) != TR_OK ||
        (st = check_out_heads("out", out, a->eb, T, a->p.heads, dim)) != TR_OK)
        return st;
    if (!aligned16(q.p) || !aligned16(out.p) || !aligned16(c->k) || !aligned16(c->v) ||
        (q.token | q.head | out.token | out.head | c->page | c->token | c->head) % 8)
        return fail(TR_EUNSUPPORTED, "q, out and the cache need bases and strides of 16 bytes");
    if ((uintptr_t)lse & 3u) return fail(TR_EUNSUPPORTED, "lse must be 4-byte aligned");
    DeviceGuard g(a->device);
    if (!g.ok) return fail(TR_EDEVICE, "hipSetDevice(%d) failed", a->device);
    tr::AttendArgs r{};
    r.tokens = T;
    r.heads = a->p.heads;
    r.kv_heads = a->p.kv_heads;
    r.dim = dim;
    r.q = q;
    r.out = out;
    r.cache = *c;
    r.step = *s;
    r.raw_scale = (float)scale;
    r.causal = causal;
    r.window = window;
    r.lse = lse;
    r.part = a->parts;
    r.arrived = a->arrived;
    r.cus = a->cus;
    hipError_t e = tr::launch_attend(r, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "attention kernel launch");
    return TR_OK;
}

}  // extern "C"
