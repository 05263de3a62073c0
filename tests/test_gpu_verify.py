"""Verification of drafted tokens against its definition: whole numbers, all equal.

The oracle adds the weights up exactly (as fractions).  The library's sums are in 64
bits: off by less than 2^-40 of the whole, so a drawn number that lies so near a
border between two tokens could fall on either side; the tests ask that none of
theirs does before they compare."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_rotate import BF, DEV, F32, gen, say

pytestmark = pytest.mark.gpu

I32 = torch.int32


def proper(x):
    return x if math.isfinite(x) and x > 0.0 else 0.0


def plain(target, ids, q_start, accept, draw, width, draft):
    """(tokens, accepted, change) as lists; the nearest that a mark comes to a border."""
    vocab, tokens, accepted, change, near = target.shape[1], [], [], [], 1.0
    for b, (t0, t1) in enumerate(zip(q_start, q_start[1:])):
        if t0 == t1:
            tokens.append([-1] * width)
            accepted.append(0)
            change.append(0)
            continue
        most, n, rejected = min(t1 - t0, width) - 1, 0, False
        while n < most and not rejected:
            r, x = t0 + n, ids[t0 + n + 1]
            p = q = 0.0
            if 0 <= x < vocab:
                p = proper(float(target[r, x]))
                q = 1.0 if draft is None else proper(float(draft[r, x]))
            if Fraction(accept[r]) * Fraction(q) < Fraction(p):
                n += 1
            else:
                rejected = True
        r = t0 + n
        p = torch.tensor([proper(v) for v in target[r].double().tolist()], dtype=torch.float64)
        w = p
        if rejected:
            if draft is None:
                w = p.clone()
                x = ids[r + 1]
                if 0 <= x < vocab:
                    w[x] = max(float(p[x]) - 1.0, 0.0)
            else:
                w = (p - torch.tensor([proper(v) for v in draft[r].double().tolist()], dtype=torch.float64)).clamp(min=0)
            if not w.any():
                w = p
        parts = [Fraction(v) for v in w.tolist()]
        total = sum(parts)
        mark, upto, word = Fraction(min(max(draw[b], 0.0), 1.0 - 2.0 ** -24)) * total, Fraction(0), 0
        for i, v in enumerate(parts):
            upto += v
            if total:
                near = min(near, abs(float((upto - mark) / total)) if v else 1.0)
            if upto > mark:
                word = i
                break
        tokens.append(([ids[t0 + 1 + i] for i in range(n)] + [word] + [-1] * width)[:width])
        accepted.append(n)
        change.append(n - (t1 - t0 - 1))
    return tokens, accepted, change, near


def check(target, ids, rows, accept, draw, width, draft=None, what=""):
    q_start = [sum(rows[:b]) for b in range(len(rows) + 1)]
    tokens, accepted, change, near = plain(target, ids.tolist(), q_start, accept.tolist(), draw.tolist(), width, draft)
    assert near > 2.0 ** -40 or not draw.any(), (what, near)
    dev = lambda t: None if t is None else t.to(DEV)
    v = tr.verify_drafts(dev(target), dev(ids), torch.tensor(q_start, dtype=I32, device=DEV), dev(accept), dev(draw), width, draft=dev(draft))
    assert v.tokens.dtype == v.accepted.dtype == v.change.dtype == I32 and v.tokens.shape == (len(rows), width)
    assert v.accepted.tolist() == accepted, what
    assert v.change.tolist() == change, what
    assert v.tokens.tolist() == tokens, what
    return v


def inputs(g, rows, vocab, dtype, with_draft, spread=3.0):
    """Distributions, and drafts that were drawn from those near them."""
    total = sum(rows)
    logits = spread * torch.randn(total, vocab, generator=g)
    target = torch.softmax(logits, 1).to(dtype)
    draft = torch.softmax(logits + 0.7 * torch.randn(total, vocab, generator=g), 1).to(dtype) if with_draft else None
    words = torch.multinomial((draft if with_draft else target).float(), 1, generator=g)[:, 0] if total else torch.zeros(0, dtype=torch.int64)
    ids = torch.randint(0, vocab, (total,), generator=g)
    ids[1:] = words[:-1]
    return target, ids.to(I32), torch.rand(total, generator=g), torch.rand(len(rows), generator=g), draft


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 15, 16, 17, 63, 64, 65, 255, 1000, 1025, 5000])
def test_drafts(vocab, with_draft, dtype):
    """Sequences of no rows, one row, some and many drafts; vocabularies from one word on."""
    say("verify", vocab, with_draft, dtype)
    g = gen(vocab)
    rows = [1, 0, 2, 5, 9, 1, 3, 0, 4]
    check(*(lambda t, i, a, d, q: (t, i, rows, a, d, 9, q))(*inputs(g, rows, vocab, dtype, with_draft)), what=vocab)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("with_draft", [True, False])
def test_large_vocabularies(with_draft, dtype):
    for vocab in (32000, 50001, 128000):
        say("large", vocab)
        g = gen(vocab)
        rows = [5, 1, 2]
        t, i, a, d, q = inputs(g, rows, vocab, dtype, with_draft)
        check(t, i, rows, a, d, 5, q, what=vocab)


def test_many_sequences_and_drafts():
    say("many")
    g = gen(8)
    rows = [int(x) for x in torch.randint(0, 4, (700,), generator=g)]
    t, i, a, d, q = inputs(g, rows, 50, F32, True)
    check(t, i, rows, a, d, 3, q)
    rows = [200, 1, 70, 66]                                            # more drafts than a wavefront has lanes, all accepted or nearly
    t, i, a, d, q = inputs(g, rows, 40, F32, True)
    v = check(t, i, rows, a * 1e-3, d, 200, t.clone())
    assert v.accepted.tolist() == [199, 0, 69, 65]
    a = a * 1e-3
    a[150], a[201 + 64] = 0.999999, 0.999999                            # rejected behind the first 64
    t2 = t.clone()
    t2[150, i[151]] *= 0.5
    t2[265, i[266]] *= 0.5
    v = check(t2, i, rows, a, d, 200, t)
    assert v.accepted.tolist() == [150, 0, 64, 65]


def test_width_cuts_drafts_off():
    """At most width - 1 drafts are looked at; those past them are given up."""
    say("width")
    g = gen(3)
    rows = [6, 2, 4, 1]
    for width in (1, 2, 3, 9):
        t, i, a, d, q = inputs(g, rows, 30, F32, True)
        v = check(t, i, rows, a * 0.0, d, width, q)
        assert v.accepted.tolist() == [min(n, width) - 1 for n in rows]


SMALL_AND_LARGE = pytest.mark.parametrize("vocab", [300, 41003])      # one launch, and two


@SMALL_AND_LARGE
def test_borders(vocab):
    """Numbers at the ends of their range and out of it, weights of 0 at both ends, all
    mass on one word, equal distributions, none at all."""
    say("borders", vocab)
    one = torch.zeros(1, vocab)
    cases = []
    for first, last in ((0, vocab - 1), (7, 7), (vocab - 1, vocab - 1), (0, 0), (100, 200), (vocab - 150, vocab - 1)):
        p = one.clone()
        p[0, first:last + 1] = 0.25
        for u, want in ((0.0, first), (1.0 - 2.0 ** -24, last), (1.0, last), (5.0, last), (-1.0, first), (math.nan, first)):
            cases.append((p, u, want))
    for p, u, want in cases:
        v = tr.verify_drafts(p.to(DEV), torch.zeros(1, dtype=I32, device=DEV), torch.tensor([0, 1], dtype=I32, device=DEV),
                             torch.zeros(1, device=DEV), torch.tensor([u], device=DEV), 1)
        assert v.tokens.tolist() == [[want]], (u, want)
    g = gen(1)
    t, i, a, d, q = inputs(g, [2, 2, 2], vocab, F32, True)
    near1 = torch.full_like(a, 1.0 - 2.0 ** -24)
    check(t, i, [2, 2, 2], near1, d, 2, t.clone())                      # u q < p with q = p: accepted
    half = t * 0.5
    v = check(half, i, [2, 2, 2], near1, d, 2, t)                       # rejected, and nothing is left over: the target itself
    assert v.accepted.tolist() == [0, 0, 0]
    nothing = torch.zeros_like(t)
    v = check(nothing, i, [2, 2, 2], a, d, 2, t)
    assert v.tokens.tolist() == [[0, -1]] * 3
    # a mark exactly on a border belongs to the next word
    p = torch.full((1, 4), 0.25)
    for u, want in ((0.25, 1), (0.5, 2), (0.75, 3), (0.25 - 2.0 ** -26, 0)):
        v = tr.verify_drafts(p.to(DEV), torch.zeros(1, dtype=I32, device=DEV), torch.tensor([0, 1], dtype=I32, device=DEV),
                             torch.zeros(1, device=DEV), torch.tensor([u], device=DEV), 1)
        assert v.tokens.tolist() == [[want]]


@SMALL_AND_LARGE
def test_improper_probabilities(vocab):
    """NaN, negative and infinite ones count as 0, drafts that are no words are rejected."""
    say("improper", vocab)
    g = gen(9)
    rows = [3, 4, 2]
    for dtype in (F32, BF):
        for with_draft in (True, False):
            t, i, a, d, q = inputs(g, rows, vocab, dtype, with_draft)
            for n, bad in enumerate((math.nan, -0.5, math.inf, -math.inf)):
                t[:, 5 + n] = bad
                if with_draft:
                    q[:, 6 + n] = bad
            i[1], i[4], i[8] = -1, vocab, 5
            check(t, i, rows, a, d, 4, q)
            t.fill_(math.nan)
            v = check(t, i, rows, a, d, 4, q)
            assert (v.tokens[:, 0] == 0).all()


def test_rows_anywhere():
    """Rows of wider tensors, one element off alignment, rows of no sequence."""
    say("rows")
    g = gen(10)
    rows = [3, 2, 5]
    for dtype in (F32, BF):
        for vocab in (64, 333, 41005):
            t, i, a, d, q = inputs(g, rows, vocab, dtype, True)
            want = check(t, i, rows, a, d, 5, q)
            wide = torch.full((13, vocab + 5), math.nan, dtype=dtype, device=DEV)
            other = torch.full((13 * (vocab + 1) + 1,), math.nan, dtype=dtype, device=DEV)[1:].view(13, vocab + 1)
            wide[:10, 3:vocab + 3], other[:10, :vocab] = t.to(DEV), q.to(DEV)
            pad = lambda x: torch.cat([x, x[:3]]).to(DEV)
            v = tr.verify_drafts(wide[:, 3:vocab + 3], pad(i), torch.tensor([0, 3, 5, 10], dtype=I32, device=DEV), pad(a), d.to(DEV), 5, draft=other[:, :vocab])
            assert all(torch.equal(x, y) for x, y in zip(v, want))


def test_row_starts_out_of_range():
    """Starts outside the rows are cut down to them: no memory beyond them is read."""
    say("starts")
    g = gen(12)
    t, i, a, d, q = inputs(g, [4, 4], 50, F32, True)
    start = torch.tensor([-5, 4, 99], dtype=I32, device=DEV)
    v = tr.verify_drafts(t.to(DEV), i.to(DEV), start, a.to(DEV), d.to(DEV), 4, draft=q.to(DEV))
    want = check(t, i, [4, 4], a, d, 4, q)
    assert all(torch.equal(x, y) for x, y in zip(v, want))
    v = tr.verify_drafts(t[:0].to(DEV), i[:0].to(DEV), start, a[:0].to(DEV), d.to(DEV), 4)
    assert (v.tokens == -1).all() and not v.accepted.any() and not v.change.any()


@SMALL_AND_LARGE
def test_replays_from_a_graph(vocab):
    g = gen(13)
    rows = [3, 1, 4]
    t, i, a, d, q = (x.to(DEV) for x in inputs(g, rows, vocab, F32, True))
    start = torch.tensor([0, 3, 4, 8], dtype=I32, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        tr.verify_drafts(t, i, start, a, d, 4, draft=q)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        v = tr.verify_drafts(t, i, start, a, d, 4, draft=q)
    for n in range(5):
        new = inputs(g, rows, vocab, F32, True)
        for old, x in zip((t, i, a, d, q), new):
            old.copy_(x)
        want = check(*(new[0], new[1], rows, new[2], new[3], 4, new[4]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(v, want)), n


def test_draws_follow_the_target():
    """Over many given numbers, evenly spread: the first token's distribution is the
    target's, whatever the draft's.  With u and v on grids of n points each word's share
    is off by at most its borders' grid cells: 2 / n for the accepted and (words + 2) / n
    for the drawn."""
    say("distribution")
    g = gen(14)
    words, n = 6, 400
    target, draft = (torch.softmax(torch.randn(1, words, generator=g), 1) for _ in range(2))
    grid = (torch.arange(n) + 0.5) / n
    share = torch.zeros(words, dtype=torch.float64)
    for x in range(words):
        rows = torch.arange(n * n + 1, dtype=I32, device=DEV) * 2
        u, v = grid.repeat_interleave(n), grid.repeat(n)
        ids = torch.tensor([0, x], dtype=I32).repeat(n * n)
        r = tr.verify_drafts(target.expand(2 * n * n, words).contiguous().to(DEV), ids.to(DEV), rows, u.repeat_interleave(2).contiguous().to(DEV), v.to(DEV), 2,
                             draft=draft.expand(2 * n * n, words).contiguous().to(DEV))
        first = torch.bincount(r.tokens[:, 0].cpu().long(), minlength=words).double() / (n * n)
        share += float(draft[0, x]) * first
    assert float((share - target[0].double()).abs().max()) <= (words + 4) / n


def test_refusals():
    t = torch.rand(4, 10, device=DEV)
    i, s, a, d = torch.zeros(4, dtype=I32, device=DEV), torch.tensor([0, 4], dtype=I32, device=DEV), torch.zeros(4, device=DEV), torch.zeros(1, device=DEV)
    bad = [lambda: tr.verify_drafts(t.double(), i, s, a, d, 4), lambda: tr.verify_drafts(t.cpu(), i, s, a, d, 4), lambda: tr.verify_drafts(t, i.long(), s, a, d, 4),
           lambda: tr.verify_drafts(t, i[:3], s, a, d, 4), lambda: tr.verify_drafts(t, i, s.long(), a, d, 4), lambda: tr.verify_drafts(t, i, s[:0], a, d, 4),
           lambda: tr.verify_drafts(t, i, s, a.double(), d, 4), lambda: tr.verify_drafts(t, i, s, a, a, 4), lambda: tr.verify_drafts(t, i, s, a, d, 0), lambda: tr.verify_drafts(t, i, s, a, d, (1 << 32) + 1),
           lambda: tr.verify_drafts(t, i, s, a, d, 4, draft=t[:, :9]), lambda: tr.verify_drafts(t, i, s, a, d, 4, draft=t.to(BF)),
           lambda: tr.verify_drafts(t.t(), i, s, a, d, 4), lambda: tr.verify_drafts(t[:1].expand(4, 10), i, s, a, d, 4), lambda: tr.verify_drafts(t[:, :0], i, s, a, d, 4)]
    for n, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, tr.TRError)):
            f()
            print("not refused:", n)
    v = tr.verify_drafts(t, i, s[:1], a, d[:0], 4)
    assert v.tokens.shape == (0, 4) and v.accepted.shape == (0,)
