"""New keys and values rounded into a paged cache of 8-bit values, against the
definitions in 64 bits (attn_ref for norm and rotation).

Tolerances, from the arithmetic: an element is off by less than 3e-6 of the length of
the pair that it turns in before it is rounded (test_gpu_rotate), and e4m3 rounds by at
most 2^-4 of it, or by 2^-10 scales where it is below the normal range: |got - want| <=
2^-4 |want| + 2^-10 scale + 3.2e-6 length (the 2^-4 of what the first error adds
included).  Values are not normed or turned: their one rounding is exactly that of the
definition.  A scale is right where the largest element is further than 3e-6 of its
pair's length from a border between two scales, else either of the two.  Old rows that
are rounded again are compared bit for bit: their factor is a power of two."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2607_13500_amd as tr
from test_gpu_attend8 import E4M3, cache8
from test_gpu_rotate import BF, DEV, F32, gen, inputs, on_device, positions, say, side64, step_of, weights

pytestmark = pytest.mark.gpu

EPS = 1e-6


def least_scale(top):
    """The smallest 2^e, -117 <= e <= 120, with top <= 448 2^e."""
    if top == 0.0:
        return 2.0 ** -117
    e = math.frexp(top)[1] - 9
    if top > 448.0 * 2.0 ** e:
        e += 1
    elif top <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** min(max(e, -117), 120)


def rounded(x):
    """fp64 values to e4m3, ties to even, NaN where they are not finite."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    step = torch.where(x.abs() >= 16 * step, 2 * step, step)         # log2's rounding
    return torch.where(torch.isfinite(x), torch.round(x / step) * step, torch.full_like(x, math.nan))


def blocks_of(step, page_size, block):
    """(page, number of the block in it, rows of the block, their packed rows, older rows)."""
    for b, t0, n, kv in ref.sequences(step):
        done = kv - n
        while done < kv:
            upto = min(kv, (done // block + 1) * block)
            at = ref.place(step, b, done, page_size)
            if at is not None:
                page, row = at
                yield page, row // block, list(range(row % block, row % block + upto - done)), list(range(t0 + done - kv + n, t0 + upto - kv + n)), row % block
            done = upto


def check_side(got, got_scale, old, old_scale, want, length, step, block, exact, what):
    """One side of the cache after an append: codes as float64, scales."""
    pages, page_size = got.shape[:2]
    expect_same = torch.ones(got.shape[:3], dtype=torch.bool)
    scale_same = torch.ones(got_scale.shape, dtype=torch.bool)
    for page, number, rows, packed, before in blocks_of(step, page_size, block):
        first = number * block
        at = [first + r for r in rows]
        expect_same[page, at] = False
        for h in range(got.shape[2]):
            x = want[packed, h]
            finite = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
            top, slack = float(finite.abs().max()), 0.0 if exact else float(3e-6 * length[packed, h].max())
            s0, s = float(old_scale[page, number, h]), float(got_scale[page, number, h])
            allowed = set()
            for t in (top - slack, top + slack):
                allowed.add(s0 if before and t <= 448.0 * s0 else least_scale(max(t, 0.0)))
            assert s in allowed, (what, page, number, h, s, allowed)
            scale_same[page, number, h] = False
            y = got[page, at, h]
            if exact:
                assert torch.equal(torch.nan_to_num(y, nan=1e9), torch.nan_to_num(rounded(x / s), nan=1e9)), (what, page, number, h)
            else:
                over = (y * s - x).abs() - (2.0 ** -4 * x.abs() + 2.0 ** -10 * s + 3.2e-6 * length[packed, h])
                assert float(over.max()) <= 0.0, (what, page, number, h, float(over.max()))
            if before:
                older = list(range(first, first + before))
                expect_same[page, older, h] = False
                was = old[page, older, h]
                assert torch.equal(got[page, older, h], was if s == s0 else rounded(was * (s0 / s))), (what, page, number, h)
    assert torch.equal(got_scale[scale_same], old_scale[scale_same]), what
    assert torch.equal(got[expect_same], old[expect_same]), what


def wide(cache):
    return [cache.k.float().cpu().double(), cache.v.float().cpu().double(), cache.k_scale.cpu().double(), cache.v_scale.cpu().double()]


def check(a, q, k, v, pos, cache, step, wq, wk, sections, adjacent, what, block):
    k0, v0, ks0, vs0 = wide(cache)
    got = a.append(q, k, v, pos.to(DEV), cache, on_device(step), wq=wq, wk=wk)
    k1, v1, ks1, vs1 = wide(cache)
    want, length, _, _ = side64(k, wk, pos, a.head_dim, a.rot_dim, sections, adjacent, a.norm, EPS)
    check_side(k1, ks1, k0, ks0, want, length, step, block, False, (what, "k"))
    x = v.cpu().double()
    check_side(v1, vs1, v0, vs0, x, x.abs(), step, block, True, (what, "v"))
    if q is not None:
        assert torch.equal(got, a.rotate(q, None, pos.to(DEV), wq=wq)[0])       # the same arithmetic: the same bits
    else:
        assert got is None


STEPS = [([1], [1], 16, 16), ([3, 0, 5, 1], [3, 7, 9, 33], 8, 4), ([1] * 70, [1 + 3 * i for i in range(70)], 16, 16),
         ([200, 17], [201, 17], 48, 16), ([40], [41], 1, 1), ([130, 5, 1], [190, 300, 65], 64, 64), ([300, 2], [333, 129], 256, 256),
         ([9, 31], [12, 40], 50, 25), ([600], [1200], 512, 512)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim,rot,sections", [(128, 128, (16, 24, 24)), (64, 32, (16,)), (80, 80, (20, 20)), (256, 256, (128,)), (16, 16, (8,)),
                                              (10, 6, (3,)), (136, 136, (68,)), (33, 0, ())])
@pytest.mark.parametrize("layout", ["rows", "heads"])
def test_append(dim, rot, sections, dtype, layout):
    for n, (new, kv, page_size, block) in enumerate(STEPS):
        heads, kv_heads, how, normed, adjacent = [(4, 4, "packed", True, False), (8, 2, "own", True, True), (7, 1, "own", False, False),
                                                  (2, 2, "odd", True, False), (6, 3, "head_major", True, True)][n % 5]
        say("append8", dim, dtype, layout, len(new), page_size, block, how)
        g = gen(dim + 7 * n)
        step, pages = step_of(new, kv, page_size, g)
        tokens = sum(new)
        a = tr.Attention(heads, kv_heads, dim, dtype, rot_dim=rot, sections=sections or None, norm=normed, adjacent=adjacent, eps=EPS)
        q, k = inputs(dim, dtype, tokens, heads, kv_heads, how, g)
        _, v = inputs(dim, dtype, tokens, heads, kv_heads, how, g)
        wq, wk = weights(dim, dtype, g, normed)
        pos = positions(max(1, len(sections)), tokens, g)
        cache = cache8(pages, page_size, kv_heads, dim, g, block, layout)
        check(a, q, k, v, pos, cache, step, wq, wk, sections, adjacent, (dim, n), block)
        check(a, None, k, v, pos, cache, step, None, wk, sections, adjacent, (dim, n, "again"), block)     # over what is there now
        a.close()


def test_tokens_one_by_one():
    """A block filled token by token, whose elements grow and shrink: the scale only
    grows, older rows are rounded again with it, a new block begins anew."""
    g = gen(5)
    for dim in (64, 128, 20):
        a = tr.Attention(2, 2, dim, F32, rot_dim=0)
        cache = cache8(4, 16, 2, dim, g)
        table = torch.tensor([[2, 0, 3]], dtype=torch.int32)
        sizes = [1.0, 0.3, 7.0, 1e-3, 600.0, 2.0, 0.0, 1e5, 1.0, 1e-20, 3e5, 1.0, 5.0, 1e30, 1.0, 2.0, 1e-4, 2e-4, 5.0]
        for i, size in enumerate(sizes):
            say("token", dim, i)
            step = tr.Step(torch.tensor([0, 1], dtype=torch.int32), torch.tensor([i + 1], dtype=torch.int32), table)
            q, k, v = (size * torch.randn(1, 2, dim, generator=g).to(DEV) for _ in range(3))
            check(a, q, k, v, torch.zeros(1, 1, dtype=torch.int32), cache, step, None, None, (), False, (dim, i), 16)
        a.close()


def test_elements_of_every_size():
    """Zeros, the smallest and the largest fp32 values, borders between two scales,
    ties between two e4m3 values, and elements that are not finite."""
    say("sizes")
    dim, block = 64, 4
    top = float(torch.finfo(F32).max)
    rows = [torch.zeros(dim), torch.full((dim,), 448.0), torch.full((dim,), 448.0 + 2.0 ** -15), torch.full((dim,), 1e-45),
            torch.full((dim,), 2.0 ** -126), torch.full((dim,), top), torch.tensor([math.nan, math.inf, -math.inf, 1.0] * 16),
            torch.full((dim,), math.nan), torch.tensor([448.0, 17.0, 19.0, 18.5, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 1.5 * 2.0 ** -10] * 8),
            torch.tensor([464.0, 272.0, 304.0, -272.0] * 16)]
    for dt in (F32, BF):
        a = tr.Attention(1, 1, dim, dt, rot_dim=0)
        for i, row in enumerate(rows):
            x = row.to(dt).view(1, 1, dim).to(DEV)
            cache = cache8(2, block, 1, dim, gen(i), block)
            k0, v0, ks0, vs0 = wide(cache)
            step = tr.Step(torch.tensor([0, 1], dtype=torch.int32), torch.tensor([1], dtype=torch.int32), torch.tensor([[1]], dtype=torch.int32))
            a.append(None, x, x, torch.zeros(1, 1, dtype=torch.int32, device=DEV), cache, on_device(step))
            k1, v1, ks1, vs1 = wide(cache)
            for new, old, scale, old_scale in ((k1, k0, ks1, ks0), (v1, v0, vs1, vs0)):
                check_side(new, scale, old, old_scale, x.cpu().double(), x.cpu().double(), step, block, True, (dt, i))
        a.close()


def test_leaves_what_is_not_its_own():
    """Rows of no sequence, tokens whose page is out of range or past the table, and
    tokens before a sequence's first: no key, value or scale is written for them."""
    say("not its own")
    g = gen(9)
    for dim in (128, 12):
        a = tr.Attention(4, 2, dim, BF)
        step = tr.Step(torch.tensor([2, 7, 9, 12, 13], dtype=torch.int32), torch.tensor([5, 18, 40, -3], dtype=torch.int32),
                       torch.tensor([[3, 1], [0, 99], [2, 4], [-1, -1]], dtype=torch.int32))
        cache = cache8(5, 16, 2, dim, g)
        q, k, v = (torch.randn(16, n, dim, generator=g).to(BF).to(DEV) for n in (4, 2, 2))
        pos = positions(1, 16, g)
        before = wide(cache)
        out = torch.full((16, 4, dim), 7.0, dtype=BF, device=DEV)
        a.append(q, k, v, pos.to(DEV), cache, on_device(step), q_out=out)
        after = wide(cache)
        own = torch.zeros(5, 16, dtype=torch.bool)
        own[3, :5] = True                        # sequence 0: its five tokens; the others' are out of the table or their pages out of the cache
        for x, y in zip(before[:2], after[:2]):
            assert torch.equal(x[~own], y[~own]) and not torch.equal(x[own], y[own])
        for x, y in zip(before[2:], after[2:]):
            assert torch.equal(x[[0, 1, 2, 4]], y[[0, 1, 2, 4]])
        assert (out[[0, 1, 13, 14, 15]] == 7.0).all() and (out[2:13] != 7.0).any(2).all()
        a.close()


def test_far_pages():
    """Element offsets beyond 2^32 in the cache."""
    say("far pages")
    dim, kv_heads, page_size, pages = 128, 8, 1024, 4300
    k, v = (torch.zeros(pages, page_size, kv_heads, dim, dtype=torch.uint8, device=DEV) for _ in range(2))
    scales = [torch.full((pages, 64, kv_heads), 7.0, device=DEV) for _ in range(2)]
    far = tr.KVCache8(k.view(E4M3), v.view(E4M3), *scales)
    g = gen(3)
    a = tr.Attention(8, kv_heads, dim, BF)
    x = torch.randn(40, 24, dim, generator=g).to(BF).to(DEV)
    near = tr.KVCache8(*(torch.zeros(2, page_size, kv_heads, dim, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)),
                       *(torch.full((2, 64, kv_heads), 7.0, device=DEV) for _ in range(2)))
    pos = positions(1, 40, g).to(DEV)
    for cache, table in ((near, [[0, 1]]), (far, [[4299, 4200]])):
        step = tr.Step(*(torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([0, 40], [1050], table)))
        a.append(x[:, :8], x[:, 8:16], x[:, 16:], pos, cache, step)
    for c, n in zip(far, near):
        c, n = (t.view(torch.uint8) if t.dtype == E4M3 else t for t in (c, n))
        assert torch.equal(c[4299], n[0]) and torch.equal(c[4200], n[1])
    assert int(k.count_nonzero()) == int(near.k.view(torch.uint8).count_nonzero())


def test_other_scales_of_older_tokens():
    """Older tokens' scales that are no powers of two: kept where they are large enough."""
    say("other scales")
    g = gen(17)
    dim = 64
    a = tr.Attention(1, 1, dim, F32, rot_dim=0)
    for s0, size in ((0.3, 1.0), (0.3, 134.0), (0.3, 1000.0), (1e-3, 0.4), (1e-3, 7.0)):
        cache = cache8(1, 16, 1, dim, g)
        cache.k_scale.fill_(s0)
        cache.v_scale.fill_(s0)
        _, v0, _, vs0 = wide(cache)
        x = size * (0.5 + 0.5 * torch.rand(1, 1, dim, generator=g)).to(DEV)
        step = tr.Step(*(torch.tensor(t, dtype=torch.int32) for t in ([0, 1], [6], [[0]])))
        a.append(None, x, x, torch.zeros(1, 1, dtype=torch.int32, device=DEV), cache, on_device(step))
        _, v1, _, vs1 = wide(cache)
        s, old = float(vs1[0, 0, 0]), float(vs0[0, 0, 0])
        top = float(x.abs().max())
        assert s == (old if top <= 448.0 * old else least_scale(top))
        # quotients and products are fp32: an e4m3 half step and 2^-23 of the value, twice
        for got, want in ((v1[0, 5, 0] * s, x[0, 0].cpu().double()), (v1[0, :5, 0] * s, v0[0, :5, 0] * old)):
            assert ((got - want).abs() <= (2.0 ** -4 + 2.0 ** -22) * want.abs() + 2.0 ** -10 * s).all()
        assert torch.equal(v1[0, 6:], v0[0, 6:])


def test_step_replays_from_a_graph():
    """Append and attend recorded once, replayed with other tokens and lengths."""
    g = gen(16)
    seqs, dim, page_size = 6, 128, 16
    a = tr.Attention(8, 2, dim, BF, norm=True)
    x = torch.zeros(seqs, 12, dim, dtype=BF, device=DEV)
    pos = torch.zeros(1, seqs, dtype=torch.int32, device=DEV)
    table = torch.randperm(seqs * 256, generator=g).to(torch.int32).view(seqs, 256).to(DEV)
    step = tr.Step(torch.arange(seqs + 1, dtype=torch.int32, device=DEV), torch.ones(seqs, dtype=torch.int32, device=DEV), table)
    cache = cache8(seqs * 256, page_size, 2, dim, g)
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
        other = tr.KVCache8(*(c.clone() for c in cache))
        call(other, want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), most
        for c, o in zip(cache, other):
            assert torch.equal(c.view(torch.uint8), o.view(torch.uint8)), most


def test_refusals():
    g = gen(1)
    a = tr.Attention(4, 2, 64, BF)
    step, pages = step_of([3], [40], 16, g)
    cache, s = cache8(pages, 16, 2, 64, g), on_device(step)
    q, k = (torch.zeros(3, n, 64, dtype=BF, device=DEV) for n in (4, 2))
    pos = torch.zeros(1, 3, dtype=torch.int32, device=DEV)
    w = torch.ones(64, dtype=BF, device=DEV)
    bad = [lambda: a.append(q, k.float(), k, pos, cache, s), lambda: a.append(q, k, k[:2], pos, cache, s),
           lambda: a.append(q, k, k, pos, cache, s, wk=w), lambda: a.append(q, k, k, pos[:, :2], cache, s),
           lambda: a.append(q, k, k, pos, cache._replace(k=cache.k[:, :8]), s),
           lambda: a.append(q, k, k, pos, cache._replace(k_scale=cache.k_scale.to(BF)), s),
           lambda: a.append(q, k, k, pos, cache._replace(k=cache.k.cpu()), s),
           lambda: a.append(q, k, k, pos, cache._replace(k=cache.k[:1].expand(pages, 16, 2, 64), v=cache.v[:1].expand(pages, 16, 2, 64)), s),
           lambda: a.append(q, k, k, pos, cache, s._replace(kv_len=s.kv_len.long())),
           lambda: a.append(q, k, k, pos, cache, s, q_out=q[:, :2])]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, tr.TRError)):
            f()
            print("not refused:", i)
    none = torch.zeros(0, 2, 64, dtype=BF, device=DEV)
    assert a.append(None, none, none, pos[:, :0], cache, s) is None
