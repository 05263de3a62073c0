"""Attention over the paged cache against its definition in 64 bits (attn_ref).

Tolerance, from the arithmetic: the weights are rounded to bf16 for their product
with v (2^-8 of each), the result is rounded to bf16 (2^-8 of itself).  Scores are
fp32 sums of at most 256 products (off by less than 2e-5 of sum |q k| scale, which
stays below 60 in these inputs: 1.2e-3 of a weight), the exponentials and sums are
below 1e-5.  So |got - want| <= 2^-8 |want| + (2^-8 + 1.5e-3) sum_j w_j |v_j|, and
lse is off by less than 1.2e-3 at worst, in truth by far less: 2e-5 (1 + |largest
score|) is asked for."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2607_13500_amd as tr
from test_gpu_rotate import BF, DEV, F32, caches, gen, on_device, say, step_of

pytestmark = pytest.mark.gpu


def queries(g, tokens, heads, dim, size=1.0):
    return (size * torch.randn(tokens, heads, dim, generator=g)).to(BF)


def normal_caches(pages, page_size, kv_heads, dim, g, layout="rows"):
    c = caches(pages, page_size, kv_heads, dim, BF, g, layout)
    for t in c:
        t.copy_(torch.randn(t.shape, generator=g).to(BF))
    return c


def compare(a, q, cache, step, *, causal=True, window=0, scale=None, what=""):
    """attend against the definition; returns (out, lse)."""
    s = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    want, lse, mass, most = ref.attend(q.cpu(), cache.k.cpu(), cache.v.cpu(), step, s, causal, window)
    out, got_lse = a.attend(q.to(DEV), cache, on_device(step), scale=scale, causal=causal, window=window, want_lse=True)
    only, none = a.attend(q.to(DEV), cache, on_device(step), scale=scale, causal=causal, window=window)
    used = ~torch.isnan(lse)
    assert none is None and torch.equal(only[used.to(DEV)], out[used.to(DEV)])
    o, l = out.cpu().double(), got_lse.cpu().double()
    assert torch.isfinite(o[used]).all(), what
    over = ((o - want).abs() - 2.0 ** -8 * want.abs() - (2.0 ** -8 + 1.5e-3) * mass)[used]
    if over.numel():
        assert float(over.max()) <= 0.0, (what, float(over.max()))
    empty = used & torch.isinf(lse)
    assert (l[empty] == -math.inf).all() and (o[empty] == 0).all(), what
    some = used & ~empty
    off = ((l - lse).abs() - 2e-5 * (1.0 + most))[some]
    if off.numel():
        assert float(off.max()) <= 0.0, (what, float(off.max()))
    return out, got_lse


HEADS = [(1, 1), (4, 4), (8, 2), (7, 1), (28, 4), (16, 1), (33, 1)]


@pytest.mark.parametrize("dim", [64, 128, 80, 96, 8, 256, 136])
@pytest.mark.parametrize("heads,kv_heads", HEADS)
def test_single_tokens(dim, heads, kv_heads):
    """Decoding: one token a sequence, lengths from one to some tiles."""
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300, 1000]
    for page_size, layout in ((16, "rows"), (1, "heads"), (48, "joined")):
        say("single", dim, heads, kv_heads, page_size)
        g = gen(dim + heads)
        step, pages = step_of([1] * len(kv), kv, page_size, g)
        a = tr.Attention(heads, kv_heads, dim, BF)
        compare(a, queries(g, len(kv), heads, dim), normal_caches(pages, page_size, kv_heads, dim, g, layout), step, what=(dim, heads, page_size))
        a.close()


@pytest.mark.parametrize("dim", [64, 128, 80, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 2), (7, 1), (28, 4)])
def test_chunks(dim, heads, kv_heads):
    """Chunks of new tokens after none, some and many tokens in the cache."""
    new = [1, 5, 0, 32, 33, 100, 17, 64, 260]
    kv = [1, 5, 40, 32, 133, 117, 400, 1000, 261]
    for page_size, causal, window in ((16, True, 0), (48, True, 20), (64, False, 0), (7, True, 1), (256, True, 129)):
        say("chunks", dim, heads, kv_heads, page_size, causal, window)
        g = gen(dim + heads)
        step, pages = step_of(new, kv, page_size, g)
        a = tr.Attention(heads, kv_heads, dim, BF)
        compare(a, queries(g, sum(new), heads, dim), normal_caches(pages, page_size, kv_heads, dim, g), step, causal=causal, window=window,
                what=(dim, heads, page_size, causal, window))
        a.close()


def test_one_long_sequence():
    """Few rows over a long cache (work split along it), and a window far into it."""
    for new, kv, window in ((1, 40000, 0), (3, 33333, 0), (1, 40000, 1000), (2, 70000, 1), (150, 20000, 0), (40, 9000, 700)):
        say("long", new, kv, window)
        g = gen(kv)
        step, pages = step_of([new], [kv], 64, g)
        a = tr.Attention(7, 1, 128, BF)
        compare(a, queries(g, new, 7, 128, 1.5), normal_caches(pages, 64, 1, 128, g), step, window=window, what=(new, kv, window))


def test_many_sequences():
    """More sequences than one probe of the search, some without new tokens."""
    g = gen(77)
    new = [int(x) for x in torch.randint(0, 4, (700,), generator=g)]
    kv = [n + int(x) for n, x in zip(new, torch.randint(0, 60, (700,), generator=g))]
    say("many sequences", sum(new))
    step, pages = step_of(new, kv, 16, g)
    a = tr.Attention(4, 2, 64, BF)
    compare(a, queries(g, sum(new), 4, 64), normal_caches(pages, 16, 2, 64, g), step)


def test_mixed_lengths():
    """One long prompt and one long context among single tokens."""
    new = [1] * 20 + [300] + [1] * 11 + [0, 2]
    kv = [7 * i + 1 for i in range(20)] + [300] + [9000 if i == 5 else 30 for i in range(11)] + [50, 2]
    for heads, kv_heads in ((8, 2), (4, 4)):
        say("mixed", heads)
        g = gen(5)
        step, pages = step_of(new, kv, 32, g)
        a = tr.Attention(heads, kv_heads, 128, BF)
        compare(a, queries(g, sum(new), heads, 128), normal_caches(pages, 32, kv_heads, 128, g), step)


def test_rows_that_see_nothing():
    """Sequences of no tokens, and new tokens before a sequence's first one."""
    say("empty rows")
    g = gen(3)
    step = tr.Step(torch.tensor([0, 2, 7, 8], dtype=torch.int32), torch.tensor([0, 3, 0], dtype=torch.int32),
                   torch.tensor([[0], [1], [2]], dtype=torch.int32))
    a = tr.Attention(4, 2, 64, BF)
    cache = normal_caches(3, 16, 2, 64, g)
    out, lse = compare(a, queries(g, 8, 4, 64), cache, step)
    assert not out[:4].any() and (lse[:4] == -math.inf).all() and not out[7].any()
    none = tr.Step(step.q_start, step.kv_len, torch.empty(3, 0, dtype=torch.int32))    # no page at all
    out, lse = a.attend(queries(g, 8, 4, 64).to(DEV), cache, on_device(none), want_lse=True)
    assert not out.any() and (lse == -math.inf).all()


def test_rows_of_no_sequence_stay():
    say("rows of none")
    g = gen(4)
    step = tr.Step(torch.tensor([2, 3, 5], dtype=torch.int32), torch.tensor([9, 17], dtype=torch.int32), torch.tensor([[0, -1], [1, 2]], dtype=torch.int32))
    for heads in (2, 8):
        a = tr.Attention(heads, 2, 128, BF)
        cache = normal_caches(3, 16, 2, 128, g)
        q = queries(g, 9, heads, 128)
        out = torch.full((9, heads, 128), 7.0, dtype=BF, device=DEV)
        a.attend(q.to(DEV), cache, on_device(step), out=out)
        assert (out[[0, 1, 5, 6, 7, 8]] == 7.0).all()
        want, _, mass, _ = ref.attend(q, cache.k.cpu(), cache.v.cpu(), step, 128 ** -0.5, True, 0)
        o = out.cpu().double()[2:5]
        assert ((o - want[2:5]).abs() <= 2.0 ** -8 * want[2:5].abs() + (2.0 ** -8 + 1.5e-3) * mass[2:5]).all()


@pytest.mark.parametrize("new,kv", [(1, 200), (1, 3000), (40, 300), (300, 300), (130, 4000)])
def test_hidden_elements_change_nothing(new, kv):
    """NaN and infinities past the sequence's end, in pages of none, before the
    window and in tokens later than the row: the same bits as with zeros there."""
    for heads, kv_heads, window in ((4, 4, 0), (8, 1, 0), (8, 2, 37), (7, 7, 64)):
        say("hidden", new, kv, heads, window)
        g = gen(kv + new)
        step, pages = step_of([new], [kv], 16, g)
        a = tr.Attention(heads, kv_heads, 128, BF)
        cache = normal_caches(pages, 16, kv_heads, 128, g)
        used = torch.zeros(pages, 16, dtype=torch.bool)
        for j in range(max(0, kv - new - window + 1) if window else 0, kv):
            page, row = ref.place(step, 0, j, 16)
            used[page, row] = True
        q = queries(g, new, heads, 128)
        for t in cache:
            t[~used.to(DEV)] = 0.0
        clean, clean_lse = compare(a, q, cache, step, window=window, what=(new, kv, window))
        for bad in (math.nan, math.inf, -math.inf):
            for t in cache:
                t[~used.to(DEV)] = bad
            out, lse = a.attend(q.to(DEV), cache, on_device(step), window=window, want_lse=True)
            assert torch.equal(out, clean) and torch.equal(lse, clean_lse), bad
        # a later token of the chunk is not finite: the rows before it do not see it
        if new > 1:
            for t in cache:
                t[~used.to(DEV)] = 0.0
            for bad in (math.nan, math.inf):
                late = new // 2
                page, row = ref.place(step, 0, kv - new + late, 16)
                kept = [t[page, row].clone() for t in cache]
                cache.k[page, row, :, 3:7] = bad
                cache.v[page, row, :, 5:9] = bad
                out, lse = a.attend(q.to(DEV), cache, on_device(step), window=window, want_lse=True)
                assert torch.equal(out[:late], clean[:late]) and torch.equal(lse[:late], clean_lse[:late]), bad
                if window:      # and the rows that have left it behind
                    assert torch.equal(out[late + window:], clean[late + window:])
                cache.k[page, row], cache.v[page, row] = kept
        a.close()


def test_not_finite_values_that_are_seen():
    """A NaN key makes its row NaN; a value's NaN or infinity stays in its element."""
    g = gen(6)
    step, pages = step_of([2], [50], 16, g)
    a = tr.Attention(2, 2, 64, BF)
    cache = normal_caches(pages, 16, 2, 64, g)
    page, row = ref.place(step, 0, 10, 16)
    cache.v[page, row, 1, 5] = math.inf
    cache.v[page, row, 0, 9] = math.nan
    out, _ = a.attend(queries(g, 2, 2, 64).to(DEV), cache, on_device(step))
    assert (out[:, 1, 5] == math.inf).all() and torch.isnan(out[:, 0, 9]).all()
    out[:, 1, 5] = out[:, 0, 9] = 0.0
    assert torch.isfinite(out).all()


def test_scores_of_every_size():
    """Scores far apart, far from zero, and all alike: the running maximum."""
    g = gen(12)
    step, pages = step_of([3], [700], 16, g)
    a = tr.Attention(4, 2, 64, BF)
    cache = normal_caches(pages, 16, 2, 64, g)
    q = queries(g, 3, 4, 64)
    for scale in (0.0, -0.125, 1e-3):
        compare(a, q, cache, step, scale=scale, what=scale)
    # one key far above the others: its value comes back
    page, row = ref.place(step, 0, 400, 16)
    cache.k[page, row] = 30.0
    one = torch.full((3, 4, 64), 4.0, dtype=BF)
    out, lse = a.attend(one.to(DEV), cache, on_device(step), want_lse=True)
    assert torch.equal(out, cache.v[page, row].repeat_interleave(2, 0).expand(3, 4, 64))
    assert torch.allclose(lse, torch.full_like(lse, 4.0 * 30.0 * 64 / 8.0))
    # scores of -3000 and less, all rows: the maximum is far below zero
    cache.k.copy_(-cache.k.abs() - 20.0)
    compare(a, (20.0 + 0.01 * queries(g, 3, 4, 64)).to(BF), cache, step, scale=0.125 / 400, what="below zero")


def test_views_and_outputs():
    """Queries and outputs as slices of wider tensors and head-major."""
    g = gen(21)
    new, kv = [5, 1, 70], [20, 300, 70]
    step, pages = step_of(new, kv, 16, g)
    a = tr.Attention(8, 2, 64, BF)
    cache = normal_caches(pages, 16, 2, 64, g, "joined")
    q = queries(g, 76, 8, 64)
    want, _ = compare(a, q, cache, step)
    wide = torch.randn(76, 12, 72, generator=g).to(BF).to(DEV)
    wide[:, 2:10, :64] = q.to(DEV)
    out = torch.zeros(8, 76, 64, dtype=BF, device=DEV)
    got, _ = a.attend(wide[:, 2:10, :64], cache, on_device(step), out=out.transpose(0, 1))
    assert torch.equal(got, want) and torch.equal(out.transpose(0, 1), want)
    inplace = q.to(DEV)
    a.attend(inplace, cache, on_device(step), out=inplace)
    assert torch.equal(inplace, want)


def test_far_pages():
    """Element offsets beyond 2^32 in the cache."""
    say("far pages")
    dim, kv_heads, page_size, pages = 128, 8, 1024, 4200
    k_cache, v_cache = (torch.zeros(pages, page_size, kv_heads, dim, dtype=BF, device=DEV) for _ in range(2))
    g = gen(31)
    small = normal_caches(2, page_size, kv_heads, dim, g)
    for new, kv in ((1, 1500), (200, 1500)):
        a = tr.Attention(16, kv_heads, dim, BF)
        q = queries(g, new, 16, dim).to(DEV)
        near, far = (tr.Step(*(torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, new], [kv], t))) for t in ([[0, 1]], [[4199, 4101]]))
        for c, s in ((k_cache, small.k), (v_cache, small.v)):
            c[4199], c[4101] = s[0], s[1]
        want, _ = a.attend(q, small, near)
        got, _ = a.attend(q, tr.KVCache(k_cache, v_cache), far)
        assert torch.equal(got, want)


def test_shared_pages():
    """Two sequences that begin with the same pages."""
    g = gen(13)
    table = torch.tensor([[3, 1, 0], [3, 1, 2]], dtype=torch.int32)
    step = tr.Step(torch.tensor([0, 1, 2], dtype=torch.int32), torch.tensor([40, 45], dtype=torch.int32), table)
    a = tr.Attention(4, 2, 64, BF)
    compare(a, queries(g, 2, 4, 64), normal_caches(4, 16, 2, 64, g), step)


def test_calls_repeat_bit_for_bit():
    g = gen(14)
    new, kv = [1] * 9 + [70], [3000 + 700 * i for i in range(9)] + [5000]
    step, pages = step_of(new, kv, 32, g)
    a = tr.Attention(28, 4, 128, BF)
    cache, s = normal_caches(pages, 32, 4, 128, g), on_device(step)
    q = queries(g, sum(new), 28, 128).to(DEV)
    first, lse = a.attend(q, cache, s, want_lse=True)
    for _ in range(20):
        out, l = a.attend(q, cache, s, want_lse=True)
        assert torch.equal(out, first) and torch.equal(l, lse)


def test_a_context_serves_calls_of_every_shape():
    """One context, calls of different kinds in turn: scratch that one leaves does not reach the next."""
    g = gen(15)
    a = tr.Attention(8, 2, 128, BF)
    runs = []
    for new, kv in (([1], [30000]), ([1] * 64, [500 + 13 * i for i in range(64)]), ([300], [300]), ([2, 90], [20000, 90]), ([1], [5])):
        step, pages = step_of(new, kv, 64, g)
        runs.append((queries(g, sum(new), 8, 128).to(DEV), normal_caches(pages, 64, 2, 128, g), on_device(step)))
    alone = []
    for q, c, s in runs:
        b = tr.Attention(8, 2, 128, BF)
        alone.append(b.attend(q, c, s)[0])
        b.close()
    for order in ([0, 1, 2, 3, 4], [4, 3, 2, 1, 0], [0, 0, 3, 1, 3, 0]):
        for i in order:
            q, c, s = runs[i]
            assert torch.equal(a.attend(q, c, s)[0], alone[i]), (order, i)


def test_step_replays_from_a_graph():
    """Append and attend recorded once, replayed with other tokens and lengths."""
    g = gen(16)
    seqs, dim, page_size = 6, 128, 16
    a = tr.Attention(8, 2, dim, BF, norm=True)
    x = torch.zeros(seqs, 12, dim, dtype=BF, device=DEV)
    pos = torch.zeros(1, seqs, dtype=torch.int32, device=DEV)
    table = torch.randperm(seqs * 256, generator=g).to(torch.int32).view(seqs, 256).to(DEV)
    step = tr.Step(torch.arange(seqs + 1, dtype=torch.int32, device=DEV), torch.ones(seqs, dtype=torch.int32, device=DEV), table)
    cache = normal_caches(seqs * 256, page_size, 2, dim, g)
    out = torch.empty(seqs, 8, dim, dtype=BF, device=DEV)

    def call(c, o):
        q = a.append(x[:, :8], x[:, 8:10], x[:, 10:], pos, c, step)
        a.attend(q, c, step, out=o)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(cache, out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(cache, out)
    for most in (4096, 30, 2000, 700, 4096, 1):
        x.copy_(torch.randn(seqs, 12, dim, generator=g).to(BF))
        step.kv_len.copy_(torch.randint(1, most + 1, (seqs,), generator=g).to(torch.int32))
        pos.copy_(torch.randint(0, 999, (1, seqs), generator=g).to(torch.int32))
        want = torch.empty_like(out)
        call(tr.KVCache(*(c.clone() for c in cache)), want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), most


def test_refusals():
    a = tr.Attention(4, 2, 64, BF)
    g = gen(1)
    step, pages = step_of([3], [40], 16, g)
    cache, s, q = normal_caches(pages, 16, 2, 64, g), on_device(step), queries(g, 3, 4, 64).to(DEV)
    bad = [lambda: a.attend(q.float(), cache, s), lambda: a.attend(q[:, :2], cache, s), lambda: a.attend(q, cache, s, window=-1),
           lambda: a.attend(q, cache, s, causal=False, window=4), lambda: a.attend(q, cache, s, scale=math.nan),
           lambda: a.attend(q, cache, s, out=q[:2]), lambda: a.attend(q, cache, s, out=q[:, :1].expand(3, 4, 64)),
           lambda: a.attend(q, tr.KVCache(cache.k, cache.v[:1]), s),
           lambda: a.attend(torch.zeros(3, 4, 68, dtype=BF, device=DEV)[..., 4:], cache, s),        # 8-byte aligned
           lambda: a.attend(torch.zeros(3, 4, 68, dtype=BF, device=DEV)[..., :64], cache, s),       # strides of 136 bytes
           lambda: a.attend(q, cache, s._replace(table=s.table.long())), lambda: a.attend(q, cache, s._replace(q_start=s.q_start[:1])),
           lambda: tr.Attention(4, 2, 64, F32).attend(q.float(), tr.KVCache(*(c.float() for c in cache)), s),
           lambda: tr.Attention(4, 2, 60, BF).attend(torch.zeros(3, 4, 60, dtype=BF, device=DEV),
                                                     tr.KVCache(*(torch.zeros(9, 16, 2, 60, dtype=BF, device=DEV) for _ in range(2))), s)]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, tr.TRError)):
            f()
            print("not refused:", i)
    out, lse = a.attend(q[:0], cache, tr.Step(s.q_start[:1] * 0, s.kv_len[:0], s.table[:0]), want_lse=True)    # no tokens: nothing to do
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
