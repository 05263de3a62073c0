// A step's tables and its drafts' verification in the C ABI of include/tr.h:
// validation and launches.
#include "tr.h"
#include "tr_host.h"
#include "tr_step.h"

using tr::clear_error;
using tr::elem_bytes;
using tr::fail;
using tr::hip_fail;
using tr::Range;

namespace {

// Whether two arrays of so many bytes share some without being the same.
bool crosses(const void* a, const void* b, int64_t bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x != y && x < y + (uintptr_t)bytes && y < x + (uintptr_t)bytes;
}

}  // namespace

extern "C" {

tr_status tr_update_pages(int32_t seqs, const int32_t* change, const int32_t* kv_len, int32_t* kv_out, int32_t* table,
                          int32_t table_width, int64_t table_stride, int32_t page_size, const tr_pool* pool, int32_t* q_start,
                          int64_t rows, int64_t* slots, int32_t* pos, int32_t* short_of, void* stream)
{
    clear_error();
    Range range("tr_update_pages");
    if (seqs < 0) return fail(TR_EINVAL, "seqs must be >= 0 (got %d)", seqs);
    if (!pool) return fail(TR_EINVAL, "pool must be non-NULL");
    if (rows < 0 || rows > INT32_MAX) return fail(TR_EINVAL, "rows must be in [0, 2^31 - 1] (got %lld)", (long long)rows);
    if (page_size < 1) return fail(TR_EINVAL, "page_size must be >= 1 (got %d)", page_size);
    if (table_width < 0) return fail(TR_EINVAL, "table_width must be >= 0 (got %d)", table_width);
    if (seqs > 1 && table_width > 0 && table_stride < table_width)
        return fail(TR_EINVAL, "the table has rows that overlap (stride %lld, rows of %d)", (long long)table_stride, table_width);
    if (pool->pages < 1) return fail(TR_EINVAL, "the pool needs pages >= 1 (got %d)", pool->pages);
    if (!pool->ring || !pool->state || !pool->state_out) return fail(TR_EINVAL, "the pool's ring, state and state_out must be non-NULL");
    if (!q_start || !short_of) return fail(TR_EINVAL, "q_start and short_of must be non-NULL");
    if (seqs && (!change || !kv_len || !kv_out || (!table && table_width)))
        return fail(TR_EINVAL, "change, kv_len, kv_out and table must be non-NULL");
    const uintptr_t words = (uintptr_t)change | (uintptr_t)kv_len | (uintptr_t)kv_out | (uintptr_t)table | (uintptr_t)pool->ring |
                            (uintptr_t)pool->state | (uintptr_t)pool->state_out | (uintptr_t)q_start | (uintptr_t)pos | (uintptr_t)short_of;
    if ((words & 3u) || ((uintptr_t)slots & 7u))
        return fail(TR_EUNSUPPORTED, "int32 arrays must be 4-byte and slots 8-byte aligned");
    if (crosses(kv_len, kv_out, 4 * (int64_t)seqs) || crosses(pool->state, pool->state_out, 8))
        return fail(TR_EINVAL, "kv_out and state_out must be kv_len and state themselves or apart from them");
    if (crosses(change, kv_out, 4 * (int64_t)seqs) || (seqs && change == kv_out && kv_out != kv_len))
        return fail(TR_EINVAL, "kv_out must not share memory with change");
    tr::PagesArgs a{};
    a.seqs = seqs;
    a.change = change;
    a.kv_len = kv_len;
    a.kv_out = kv_out;
    a.table = table;
    a.table_width = table_width;
    a.table_stride = table_stride;
    a.page_size = page_size;
    a.pages = pool->pages;
    a.ring = pool->ring;
    a.state = pool->state;
    a.state_out = pool->state_out;
    a.q_start = q_start;
    a.rows = rows;
    a.slots = slots;
    a.pos = pos;
    a.short_of = short_of;
    const hipError_t e = tr::launch_pages(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "page table kernel launch");
    return TR_OK;
}

size_t tr_verify_scratch(int32_t seqs) { return seqs > 0 ? (size_t)seqs * tr::kSlices * 2 * sizeof(double) : 0; }

tr_status tr_verify_drafts(int64_t T, int32_t vocab, int32_t dtype, const void* target, int64_t ld_target, const void* draft,
                           int64_t ld_draft, const int32_t* ids, int32_t seqs, const int32_t* q_start, const float* accept,
                           const float* draw, int32_t width, int32_t* tokens, int32_t* accepted, int32_t* change, void* scratch,
                           void* stream)
{
    clear_error();
    Range range("tr_verify_drafts");
    if (T < 0 || T > INT32_MAX) return fail(TR_EINVAL, "T must be in [0, 2^31 - 1] (got %lld)", (long long)T);
    if (seqs < 0 || seqs >= 1 << 20) return fail(TR_EINVAL, "seqs must be in [0, 2^20 - 1] (got %d)", seqs);
    if (vocab < 1 || vocab > 1 << 30) return fail(TR_EINVAL, "vocab must be in [1, 2^30] (got %d)", vocab);
    if (width < 1) return fail(TR_EINVAL, "width must be >= 1 (got %d)", width);
    if (dtype != TR_FP32 && dtype != TR_BF16) return fail(TR_EINVAL, "dtype must be TR_FP32 or TR_BF16 (got %d)", dtype);
    if (seqs == 0) return TR_OK;
    if (!q_start || !draw || !tokens || !accepted || !change || !scratch)
        return fail(TR_EINVAL, "q_start, draw, tokens, accepted, change and scratch must be non-NULL");
    if (T && (!target || !ids || !accept)) return fail(TR_EINVAL, "target, ids and accept must be non-NULL");
    if ((T > 1 && ld_target < vocab) || (draft && T > 1 && ld_draft < vocab))
        return fail(TR_EINVAL, "rows of probabilities overlap (ld %lld and %lld, vocab %d)", (long long)ld_target, (long long)ld_draft, vocab);
    const uintptr_t element = (uintptr_t)(elem_bytes(dtype) - 1);
    if (((uintptr_t)target | (uintptr_t)draft) & element)
        return fail(TR_EUNSUPPORTED, "target and draft must be aligned to the element size (%d bytes)", elem_bytes(dtype));
    const uintptr_t words = (uintptr_t)ids | (uintptr_t)q_start | (uintptr_t)accept | (uintptr_t)draw | (uintptr_t)tokens |
                            (uintptr_t)accepted | (uintptr_t)change;
    if ((words & 3u) || ((uintptr_t)scratch & 15u))
        return fail(TR_EUNSUPPORTED, "int32 and float arrays must be 4-byte and scratch 16-byte aligned");
    tr::VerifyArgs a{};
    a.rows = T;
    a.vocab = vocab;
    a.target = target;
    a.draft = draft;
    a.ld_target = ld_target;
    a.ld_draft = ld_draft;
    a.ids = ids;
    a.seqs = seqs;
    a.q_start = q_start;
    a.accept = accept;
    a.draw = draw;
    a.width = width;
    a.tokens = tokens;
    a.accepted = accepted;
    a.change = change;
    a.part = static_cast<double*>(scratch);
    const hipError_t e = tr::launch_verify(a, dtype == TR_BF16, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "verification kernel launch");
    return TR_OK;
}

}  // extern "C"
