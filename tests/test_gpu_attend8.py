"""Attention over the paged cache of 8-bit values against its definition in 64 bits
(attn_ref on the values that the cache stands for).

Tolerance, from the arithmetic, as for the bf16 cache: keys and values are widened
without loss; a weight times its value's scale is rounded to fp32 (2^-24 of itself) and
then to bf16 (2^-8), the result to bf16 (2^-8).  Scores are fp32 sums of at most 256
products and two fp32 products more (off by less than 2e-5 of sum |q k| scale, below 60
here: 1.2e-3 of a weight), the exponentials and sums are below 1e-5.  So
|got - want| <= 2^-8 |want| + (2^-8 + 1.5e-3) sum_j w_j |v_j|, and lse is off by less
than 2e-5 (1 + |largest score|)."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2607_13500_amd as tr
from test_gpu_attend import queries
from test_gpu_rotate import BF, DEV, F32, gen, on_device, say, step_of

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def cache8(pages, page_size, kv_heads, dim, g, block=None, layout="rows", powers=True):
    """Values of about 1 in a KVCache8 of any layout, scales from 2^-9 to 2^-5 (times
    1 .. 1.5 where they are no powers of two)."""
    block = block or page_size
    n = page_size // block
    scale = torch.exp2(torch.randint(-9, -4, (2, pages, n, kv_heads), generator=g).float())
    if not powers:
        scale *= 1.0 + 0.5 * torch.rand(scale.shape, generator=g)
    x = torch.randn(2, pages, n, block, kv_heads, dim, generator=g) * torch.exp(0.3 * torch.randn(2, pages, n, 1, kv_heads, 1, generator=g))
    codes = (x / scale[:, :, :, None, :, None]).clamp(-448, 448).to(E4M3).view(2, pages, page_size, kv_heads, dim).to(DEV)
    scale = scale.to(DEV)
    if layout == "heads":            # a page's heads one after another, scales likewise
        k, v = (c.transpose(1, 2).contiguous().transpose(1, 2) for c in codes)
        ks, vs = (s.transpose(1, 2).contiguous().transpose(1, 2) for s in scale)
    elif layout == "joined":         # keys and values side by side in one tensor
        both = torch.zeros(pages, page_size, kv_heads, 2, dim + 16, dtype=torch.uint8, device=DEV).view(E4M3)
        k, v = both[..., 0, :dim], both[..., 1, :dim]
        k.copy_(codes[0])
        v.copy_(codes[1])
        scales = torch.zeros(pages, n, kv_heads, 2, device=DEV)
        ks, vs = scales[..., 0], scales[..., 1]
        ks.copy_(scale[0])
        vs.copy_(scale[1])
    else:
        (k, v), (ks, vs) = codes, scale
    return tr.KVCache8(k, v, ks, vs)


def stands_for(cache):
    """(k, v) in 64 bits on the CPU."""
    out = []
    for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        block = c.shape[1] // s.shape[1]
        out.append(c.float().cpu().double() * s.cpu().double().repeat_interleave(block, 1)[..., None])
    return out


def compare(a, q, cache, step, *, causal=True, window=0, scale=None, what=""):
    """attend against the definition; returns (out, lse)."""
    s = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    want, lse, mass, most = ref.attend(q.cpu(), *stands_for(cache), step, s, causal, window)
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
    off = ((l - lse).abs() - 2e-5 * (1.0 + most))[used & ~empty]
    if off.numel():
        assert float(off.max()) <= 0.0, (what, float(off.max()))
    return out, got_lse


def test_every_code():
    """All e4m3 values come back as they are: one key, its value the row's result."""
    codes = torch.arange(256, dtype=torch.uint8)
    codes = codes[(codes & 0x7f) != 0x7f].repeat(2)[:256].view(4, 64)
    cache = tr.KVCache8(*(torch.zeros(4, 16, 1, 64, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)),
                        *(torch.ones(4, 1, 1, device=DEV) for _ in range(2)))
    cache.v.view(torch.uint8)[:, 0, 0] = codes.to(DEV)
    step = tr.Step(*(torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 1, 2, 3, 4], [1] * 4, [[0], [1], [2], [3]])))
    a = tr.Attention(1, 1, 64, BF)
    out, lse = a.attend(torch.ones(4, 1, 64, dtype=BF, device=DEV), cache, step, want_lse=True)
    assert torch.equal(out[:, 0], cache.v[:, 0, 0].to(BF)) and not lse.any()


HEADS = [(1, 1), (4, 4), (8, 2), (7, 1), (28, 4), (16, 1), (33, 1)]


@pytest.mark.parametrize("dim", [64, 128, 80, 96, 16, 256, 144])
@pytest.mark.parametrize("heads,kv_heads", HEADS)
def test_single_tokens(dim, heads, kv_heads):
    """Decoding: one token a sequence, lengths from one to some tiles."""
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300, 1000]
    for page_size, block, layout in ((16, 16, "rows"), (1, 1, "heads"), (48, 16, "joined"), (64, 4, "rows")):
        say("single", dim, heads, kv_heads, page_size, block)
        g = gen(dim + heads)
        step, pages = step_of([1] * len(kv), kv, page_size, g)
        a = tr.Attention(heads, kv_heads, dim, BF)
        compare(a, queries(g, len(kv), heads, dim), cache8(pages, page_size, kv_heads, dim, g, block, layout), step, what=(dim, heads, page_size))
        a.close()


@pytest.mark.parametrize("dim", [64, 128, 80, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 2), (7, 1), (28, 4)])
def test_chunks(dim, heads, kv_heads):
    """Drafts and chunks of new tokens after none, some and many tokens in the cache."""
    sets = [([1, 5, 0, 32, 33, 100, 17, 64, 260], [1, 5, 40, 32, 133, 117, 400, 1000, 261]),
            ([2, 3, 8, 1, 5], [300, 3, 700, 90, 1000]), ([4, 9, 12], [9, 500, 333])]
    for page_size, block, causal, window in ((16, 16, True, 0), (48, 48, True, 20), (64, 32, False, 0), (7, 7, True, 1), (256, 64, True, 129)):
        for new, kv in sets:
            say("chunks", dim, heads, kv_heads, page_size, block, causal, window, new)
            g = gen(dim + heads)
            step, pages = step_of(new, kv, page_size, g)
            a = tr.Attention(heads, kv_heads, dim, BF)
            compare(a, queries(g, sum(new), heads, dim), cache8(pages, page_size, kv_heads, dim, g, block, powers=page_size != 48), step,
                    causal=causal, window=window, what=(dim, heads, page_size, causal, window))
            a.close()


def test_one_long_sequence():
    """Few rows over a long cache (work split along it), and a window far into it."""
    for new, kv, window in ((1, 40000, 0), (3, 33333, 0), (8, 30000, 0), (1, 40000, 1000), (2, 70000, 1), (150, 20000, 0), (40, 9000, 700)):
        say("long", new, kv, window)
        g = gen(kv)
        step, pages = step_of([new], [kv], 64, g)
        a = tr.Attention(7, 1, 128, BF)
        compare(a, queries(g, new, 7, 128, 1.5), cache8(pages, 64, 1, 128, g, 32), step, window=window, what=(new, kv, window))


def test_many_sequences():
    """More sequences than one probe of the search, some without new tokens."""
    g = gen(77)
    new = [int(x) for x in torch.randint(0, 4, (700,), generator=g)]
    kv = [n + int(x) for n, x in zip(new, torch.randint(0, 60, (700,), generator=g))]
    say("many sequences", sum(new))
    step, pages = step_of(new, kv, 16, g)
    a = tr.Attention(4, 2, 64, BF)
    compare(a, queries(g, sum(new), 4, 64), cache8(pages, 16, 2, 64, g), step)


def test_mixed_lengths():
    """One long prompt and one long context among single tokens."""
    new = [1] * 20 + [300] + [1] * 11 + [0, 2]
    kv = [7 * i + 1 for i in range(20)] + [300] + [9000 if i == 5 else 30 for i in range(11)] + [50, 2]
    for heads, kv_heads in ((8, 2), (4, 4)):
        say("mixed", heads)
        g = gen(5)
        step, pages = step_of(new, kv, 32, g)
        a = tr.Attention(heads, kv_heads, 128, BF)
        compare(a, queries(g, sum(new), heads, 128), cache8(pages, 32, kv_heads, 128, g), step)


def test_rows_that_see_nothing():
    """Sequences of no tokens, and new tokens before a sequence's first one."""
    say("empty rows")
    g = gen(3)
    step = tr.Step(torch.tensor([0, 2, 7, 8], dtype=torch.int32), torch.tensor([0, 3, 0], dtype=torch.int32),
                   torch.tensor([[0], [1], [2]], dtype=torch.int32))
    for heads in (4, 40):
        a = tr.Attention(heads, 2, 64, BF)
        cache = cache8(3, 16, 2, 64, g)
        out, lse = compare(a, queries(g, 8, heads, 64), cache, step)
        assert not out[:4].any() and (lse[:4] == -math.inf).all() and not out[7].any()
        none = tr.Step(step.q_start, step.kv_len, torch.empty(3, 0, dtype=torch.int32))    # no page at all
        out, lse = a.attend(queries(g, 8, heads, 64).to(DEV), cache, on_device(none), want_lse=True)
        assert not out.any() and (lse == -math.inf).all()


def test_rows_of_no_sequence_stay():
    say("rows of none")
    g = gen(4)
    step = tr.Step(torch.tensor([2, 3, 5], dtype=torch.int32), torch.tensor([9, 17], dtype=torch.int32), torch.tensor([[0, -1], [1, 2]], dtype=torch.int32))
    for heads in (2, 8, 64):
        a = tr.Attention(heads, 2, 128, BF)
        cache = cache8(3, 16, 2, 128, g)
        q = queries(g, 9, heads, 128)
        out = torch.full((9, heads, 128), 7.0, dtype=BF, device=DEV)
        a.attend(q.to(DEV), cache, on_device(step), out=out)
        assert (out[[0, 1, 5, 6, 7, 8]] == 7.0).all()
        want, _, mass, _ = ref.attend(q, *stands_for(cache), step, 128 ** -0.5, True, 0)
        o = out.cpu().double()[2:5]
        assert ((o - want[2:5]).abs() <= 2.0 ** -8 * want[2:5].abs() + (2.0 ** -8 + 1.5e-3) * mass[2:5]).all()


@pytest.mark.parametrize("dim", [64, 48, 16])
@pytest.mark.parametrize("most", [1, 4, 9])
def test_heads_side_by_side(dim, most):
    """Enough sequences that a workgroup takes four heads at a time, of one to some tiles
    of rows; layouts in which they do and do not lie side by side."""
    for kv_heads, page_size, block, layout, window, powers in ((4, 16, 16, "rows", 0, True), (8, 64, 32, "rows", 50, False), (4, 24, 8, "rows", 0, False),
                                                               (4, 32, 16, "heads", 0, True), (8, 16, 16, "joined", 7, True)):
        say("side by side", dim, most, kv_heads, page_size, layout)
        g = gen(dim + most + kv_heads)
        new = [1 + i % most for i in range(40)]
        kv = [n + int(x) for n, x in zip(new, torch.randint(0, 300, (40,), generator=g))]
        kv[3], kv[17] = 5000, new[17]
        new[9] = 0
        step, pages = step_of(new, kv, page_size, g)
        a = tr.Attention(4 * kv_heads, kv_heads, dim, BF)
        compare(a, queries(g, sum(new), 4 * kv_heads, dim), cache8(pages, page_size, kv_heads, dim, g, block, layout, powers), step, window=window,
                what=(dim, most, kv_heads, layout))
        a.close()


# new tokens, lengths, heads, key heads, causal: each kernel and its ways of dealing the work
KERNELS = {"four": ([1] * 33 + [2], [40 + 9 * i for i in range(34)], 12, 4, True), "four_of_two": ([6] * 34, [70 + 9 * i for i in range(34)], 16, 4, True),
           "four_of_four": ([13] * 34, [70 + 19 * i for i in range(34)], 16, 4, False),
           "single": ([1, 1], [700, 90], 4, 2, True), "drafts": ([3, 8], [700, 90], 4, 2, True), "shares": ([70, 130], [701, 300], 4, 2, False),
           "in_turn": ([1200], [1200], 80, 80, True), "items": ([2048], [2050], 64, 64, True)}


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dim", [64, 128])
def test_hidden_elements_change_nothing(kernel, dim):
    """NaN past the sequences' ends and in pages of none, in keys, values and their
    scales, and infinite scales: the same bits as with zeros there; and NaN in a late
    token leaves the rows before it."""
    new, kv, heads, kv_heads, causal = KERNELS[kernel]
    for page_size, block in ((16, 16), (24, 8), (64, 1)):
        say("hidden", kernel, dim, page_size, block)
        g = gen(dim)
        step, pages = step_of(new, kv, page_size, g)
        a = tr.Attention(heads, kv_heads, dim, BF)
        cache = cache8(pages, page_size, kv_heads, dim, g, block)
        k8, v8 = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
        used = torch.zeros(pages, page_size, dtype=torch.bool)
        for b, n in enumerate(kv):
            j = torch.arange(n)
            used[step.table[b][j // page_size].long(), j % page_size] = True
        hidden, idle = ~used.to(DEV), ~used.view(pages, -1, block).any(2).to(DEV)
        q = queries(g, sum(new), heads, dim).to(DEV)
        for t in (k8, v8):
            t[hidden] = 0
        clean, lse = a.attend(q, cache, on_device(step), causal=causal, want_lse=True)
        for bad in (0x7f, 0xff):
            for t in (k8, v8):
                t[hidden] = bad
            for s in (cache.k_scale, cache.v_scale):
                s[idle] = math.nan if bad == 0x7f else math.inf
            out, l = a.attend(q, cache, on_device(step), causal=causal, want_lse=True)
            assert torch.equal(out, clean) and torch.equal(l, lse), (kernel, bad)
        if causal:                               # a late token of the last sequence
            late, t0 = new[-1] // 2, sum(new[:-1])
            page, row = ref.place(step, len(kv) - 1, kv[-1] - new[-1] + late, page_size)
            k8[page, row, :, 3:7] = 0x7f
            v8[page, row, :, 5:9] = 0xff
            out, l = a.attend(q, cache, on_device(step), want_lse=True)
            assert torch.equal(out[:t0 + late], clean[:t0 + late]) and torch.equal(l[:t0 + late], lse[:t0 + late])
            assert torch.isnan(out[t0 + late:]).any(2).all()
        a.close()


@pytest.mark.parametrize("kernel", KERNELS)
def test_nan_values_that_are_seen(kernel):
    """A value's NaN stays in its element, of the rows that see it and of its head."""
    new, kv, heads, kv_heads, causal = KERNELS[kernel]
    say("seen", kernel)
    g = gen(6)
    step, pages = step_of(new, kv, 16, g)
    a = tr.Attention(heads, kv_heads, 64, BF)
    cache = cache8(pages, 16, kv_heads, 64, g)
    q = queries(g, sum(new), heads, 64).to(DEV)
    clean, _ = a.attend(q, cache, on_device(step), causal=causal)
    t0, at = sum(new[:-1]), kv[-1] - (new[-1] + 1) // 2
    page, row = ref.place(step, len(kv) - 1, at, 16)
    cache.v.view(torch.uint8)[page, row, kv_heads - 1, 9] = 0x7f
    # the product has that element as 0 then: compare with the value 0 there
    out, _ = a.attend(q, cache, on_device(step), causal=causal)
    first = t0 + (max(0, at - (kv[-1] - new[-1])) if causal else 0)
    group = heads // kv_heads
    hit = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
    hit[first:, heads - group:, 9] = True
    assert torch.equal(torch.isnan(out), hit)
    assert torch.equal(out[~hit], clean[~hit])
    a.close()


@pytest.mark.parametrize("kernel", KERNELS)
def test_scores_of_every_size(kernel):
    """Scales of both signs and zero, scales of keys and values from tiny to large, one
    key far above the others, scores all far below zero."""
    new, kv, heads, kv_heads, causal = KERNELS[kernel]
    say("scores", kernel)
    g = gen(12)
    step, pages = step_of(new, kv, 16, g)
    a = tr.Attention(heads, kv_heads, 64, BF)
    cache = cache8(pages, 16, kv_heads, 64, g)
    q = queries(g, sum(new), heads, 64).to(DEV)
    from test_gpu_attend_edges import definition

    def held(scale):
        got, lse = a.attend(q, cache, on_device(step), scale=scale, causal=causal, want_lse=True)
        wide = tr.KVCache(*(t.to(DEV) for t in stands_for(cache)))
        want, want_lse, mass, most = definition(q, wide, step, scale, causal)
        assert float(((got.double() - want).abs() - 2.0 ** -8 * want.abs() - (2.0 ** -8 + 1.5e-3) * mass).max()) <= 0.0, scale
        assert float(((lse.double() - want_lse).abs() - 2e-5 * (1.0 + most)).max()) <= 0.0, scale

    for scale in (0.0, -0.125, 1e-3, -1e-30):
        held(scale)
    cache.k_scale.mul_(2.0 ** -100)
    cache.v_scale.mul_(2.0 ** 90)
    held(2.0 ** 97)
    cache.k_scale.mul_(2.0 ** 100)
    cache.v_scale.mul_(2.0 ** -190)
    held(0.125)
    cache.v_scale.mul_(2.0 ** 100)
    # scores of -1000 and less, all rows: the maximum is far below zero
    cache.k.copy_((-(cache.k.float().abs() + 200.0).clamp(max=448.0)).to(E4M3))
    q.copy_(20.0 + 0.01 * q)
    held(0.125 / 40)
    a.close()


def test_queries_that_are_not_finite():
    """A NaN or infinite query makes its own row and head NaN, at scale 0 too."""
    for kernel, (new, kv, heads, kv_heads, causal) in KERNELS.items():
        say("queries", kernel)
        g = gen(8)
        step, pages = step_of(new, kv, 16, g)
        a = tr.Attention(heads, kv_heads, 64, BF)
        cache, q = cache8(pages, 16, kv_heads, 64, g), queries(g, sum(new), heads, 64).to(DEV)
        for scale in (0.125, 0.0):
            bad = q.clone()
            bad[-1, 0, 3] = math.nan
            bad[0, heads - 1, 7] = math.inf
            beside = cache.k.view(torch.uint8)[:, :, :, 7]
            beside[(beside & 0x7f) == 0] = 0x08                   # no zero key beside the infinity
            clean, _ = a.attend(q, cache, on_device(step), scale=scale, causal=causal)
            out, _ = a.attend(bad, cache, on_device(step), scale=scale, causal=causal)
            assert torch.isnan(out[-1, 0]).all()
            keep = torch.ones(out.shape[:2], dtype=torch.bool, device=DEV)
            keep[-1, 0] = keep[0, heads - 1] = False
            assert torch.equal(out[keep], clean[keep])
            if scale == 0.0:
                assert torch.isnan(out[0, heads - 1]).all()
        a.close()


def test_views_and_outputs():
    """Queries and outputs as slices of wider tensors and head-major."""
    g = gen(21)
    new, kv = [5, 1, 70], [20, 300, 70]
    step, pages = step_of(new, kv, 16, g)
    for heads in (8, 2):
        a = tr.Attention(heads, 2, 64, BF)
        cache = cache8(pages, 16, 2, 64, g, layout="joined")
        q = queries(g, 76, heads, 64)
        want, _ = compare(a, q, cache, step)
        wide = torch.randn(76, heads + 4, 72, generator=g).to(BF).to(DEV)
        wide[:, 2:heads + 2, :64] = q.to(DEV)
        out = torch.zeros(heads, 76, 64, dtype=BF, device=DEV)
        got, _ = a.attend(wide[:, 2:heads + 2, :64], cache, on_device(step), out=out.transpose(0, 1))
        assert torch.equal(got, want) and torch.equal(out.transpose(0, 1), want)
        inplace = q.to(DEV)
        a.attend(inplace, cache, on_device(step), out=inplace)
        assert torch.equal(inplace, want)


def test_far_pages():
    """Element offsets beyond 2^32 in the cache."""
    say("far pages")
    dim, kv_heads, page_size, pages = 128, 8, 1024, 8400
    far8 = tr.KVCache8(*(torch.zeros(pages, page_size, kv_heads, dim, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)),
                       *(torch.zeros(pages, 64, kv_heads, device=DEV) for _ in range(2)))
    g = gen(31)
    small = cache8(2, page_size, kv_heads, dim, g, 16)
    for new, kv in ((1, 1500), (6, 1500), (200, 1500)):
        a = tr.Attention(16, kv_heads, dim, BF)
        q = queries(g, new, 16, dim).to(DEV)
        near, far = (tr.Step(*(torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, new], [kv], t))) for t in ([[0, 1]], [[8399, 8201]]))
        for c, s in zip(far8, small):
            c, s = (t.view(torch.uint8) if t.dtype == E4M3 else t for t in (c, s))
            c[8399], c[8201] = s[0], s[1]
        want, _ = a.attend(q, small, near)
        got, _ = a.attend(q, far8, far)
        assert torch.equal(got, want)


def test_shared_pages():
    """Two sequences that begin with the same pages."""
    g = gen(13)
    table = torch.tensor([[3, 1, 0], [3, 1, 2]], dtype=torch.int32)
    step = tr.Step(torch.tensor([0, 1, 2], dtype=torch.int32), torch.tensor([40, 45], dtype=torch.int32), table)
    a = tr.Attention(4, 2, 64, BF)
    compare(a, queries(g, 2, 4, 64), cache8(4, 16, 2, 64, g), step)


def test_calls_of_both_caches_repeat_bit_for_bit():
    """One context, calls of different kinds over caches of both types in turn: scratch
    that one leaves does not reach the next."""
    g = gen(15)
    a = tr.Attention(8, 2, 128, BF)
    runs = []
    for new, kv in (([1], [30000]), ([1] * 64, [500 + 13 * i for i in range(64)]), ([300], [300]), ([2, 90], [20000, 90]), ([1], [5]),
                    ([6] * 9, [3000 + 700 * i for i in range(9)])):
        step, pages = step_of(new, kv, 64, g)
        cache = cache8(pages, 64, 2, 128, g)
        q, s = queries(g, sum(new), 8, 128).to(DEV), on_device(step)
        runs += [(q, cache, s), (q, tr.KVCache(*(t.to(BF).to(DEV) for t in stands_for(cache))), s)]
    alone = []
    for q, c, s in runs:
        b = tr.Attention(8, 2, 128, BF)
        alone.append(b.attend(q, c, s)[0])
        b.close()
    for order in (list(range(12)), list(range(11, -1, -1)), [0, 0, 3, 1, 7, 0, 10, 10, 11]):
        for i in order:
            q, c, s = runs[i]
            assert torch.equal(a.attend(q, c, s)[0], alone[i]), (order, i)


def test_refusals():
    a = tr.Attention(4, 2, 64, BF)
    g = gen(1)
    step, pages = step_of([3], [40], 16, g)
    cache, s, q = cache8(pages, 16, 2, 64, g), on_device(step), queries(g, 3, 4, 64).to(DEV)
    wide = torch.zeros(pages, 16, 2, 72, dtype=torch.uint8, device=DEV).view(E4M3)
    bad = [lambda: a.attend(q.float(), cache, s), lambda: a.attend(q[:, :2], cache, s), lambda: a.attend(q, cache, s, window=-1),
           lambda: a.attend(q, cache, s, causal=False, window=4), lambda: a.attend(q, cache, s, scale=math.nan),
           lambda: a.attend(q, cache, s, out=q[:2]),
           lambda: a.attend(q, cache._replace(v=cache.v[:1]), s), lambda: a.attend(q, cache._replace(k=cache.k.view(torch.uint8)), s),
           lambda: a.attend(q, cache._replace(k=cache.k.to(BF), v=cache.v.to(BF)), s),
           lambda: a.attend(q, cache._replace(k_scale=cache.k_scale[:1]), s), lambda: a.attend(q, cache._replace(v_scale=cache.v_scale.double()), s),
           lambda: a.attend(q, cache._replace(k_scale=cache.k_scale[..., :1], v_scale=cache.v_scale[..., :1]), s),
           lambda: a.attend(q, cache._replace(k_scale=torch.ones(pages, 3, 2, device=DEV), v_scale=torch.ones(pages, 3, 2, device=DEV)), s),
           lambda: a.attend(q, cache._replace(k_scale=cache.k_scale[:, :0], v_scale=cache.v_scale[:, :0]), s),
           lambda: a.attend(q, cache._replace(k_scale=cache.k_scale[:1].expand(pages, 1, 2), v_scale=cache.v_scale[:1].expand(pages, 1, 2)), s),
           lambda: a.attend(q, tr.KVCache8(wide[..., 8:], wide[..., 8:], *cache[2:]), s),               # 8-byte aligned
           lambda: a.attend(q, tr.KVCache8(wide[..., :64], wide[..., :64], *cache[2:]), s),             # strides of 72 bytes
           lambda: a.attend(q, cache, s._replace(table=s.table.long())),
           lambda: tr.Attention(4, 2, 64, F32).attend(q.float(), cache, s),
           lambda: tr.Attention(4, 2, 72, BF).attend(torch.zeros(3, 4, 72, dtype=BF, device=DEV), tr.KVCache8(wide, wide, *cache[2:]), s)]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, tr.TRError)):
            f()
            print("not refused:", i)
    out, lse = a.attend(q[:0], cache, tr.Step(s.q_start[:1] * 0, s.kv_len[:0], s.table[:0]), want_lse=True)    # no tokens: nothing to do
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
