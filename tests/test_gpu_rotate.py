"""Positions of kept tokens, norm and rotation of heads, their gradients and the
append to a paged cache, against the definitions in 64 bits (attn_ref).

Tolerances, from the arithmetic: results are rounded once to their type (2^-8 of
the value in bf16, 2^-24 in fp32).  Before that all is fp32: a head's mean of at
most 256 squares is off by less than 2e-6 of itself (its square root by half of
that), sines and cosines by less than 3e-7, the products by 2^-23 each: together
below 3e-6 of the length of the pair that an element turns in.  A gradient has
one more mean over the head, whose rounding is below 3e-6 of the root mean square
of the terms.  dw adds fp32 terms, at most a few hundred to a lane before they
are joined: 5e-5 of the sum of their magnitudes."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2607_13500_amd as tr

pytestmark = pytest.mark.gpu

DEV = "cuda"
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[case]", *a, flush=True)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def values(g, *shape, dtype):
    return (torch.randn(*shape, generator=g) * torch.exp(0.5 * torch.randn(shape[0], *([1] * (len(shape) - 1)), generator=g))).to(dtype)


def freqs(rot_dim, base=10000.0):
    return [base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]


def close(got, want, unit, scale, rel, what):
    """|got - want| <= unit |want| + rel scale, everywhere."""
    got = got.detach().cpu().double()
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - (unit * want.abs() + rel * scale)
    if over.numel():
        assert float(over.max()) <= 0.0, (what, float(over.max()), int(over.argmax()))


# ---- positions -------------------------------------------------------------------
@pytest.mark.parametrize("images", [1, 3, 64, 65, 130])
def test_positions(images):
    g = gen(images)
    K, grid, start, idx = [], [], [], []
    for b in range(images):
        T, H, W = (int(torch.randint(1, n, (1,), generator=g)) for n in (9, 30, 30))
        k = int(torch.randint(0, min(300, T * H * W) + 1, (1,), generator=g))
        idx += sorted(torch.randperm(T * H * W, generator=g)[:k].tolist())
        K.append(k)
        grid.append((T, H, W))
        start.append(tuple(int(x) for x in torch.randint(-5, 100000, (3,), generator=g)))
    idx = torch.tensor(idx, dtype=torch.int32)
    say("positions", images, len(idx))
    want = ref.kept_positions(idx, K, grid, start)
    got = tr.kept_positions(idx.to(DEV), K, grid, start)
    assert got.dtype == torch.int32 and torch.equal(got.cpu().long(), want)
    # with other columns between the images', which stay
    gaps = [5 * b + 2 for b in range(images)]
    dst = [sum(K[:b]) + gaps[b] for b in range(images)]
    out = torch.full((3, sum(K) + 5 * images + 9), -7, dtype=torch.int32, device=DEV)
    full = torch.full(out.shape, -7, dtype=torch.int64)
    r = 0
    for k, d in zip(K, dst):
        full[:, d:d + k] = want[:, r:r + k]
        r += k
    tr.kept_positions(idx.to(DEV), K, grid, start, dst=dst, out=out)
    assert torch.equal(out.cpu().long(), full)


def test_positions_refusals():
    idx = torch.zeros(4, dtype=torch.int32, device=DEV)
    for bad in (dict(K=[5]), dict(grid=[(1, 0, 4)]), dict(grid=[(1 << 20, 1 << 10, 1 << 10)]), dict(K=[-1, 5], grid=[(1, 2, 2)] * 2, start=[(0, 0, 0)] * 2),
                dict(start=[]), dict(dst=[3], out=torch.zeros(3, 6, dtype=torch.int32, device=DEV)), dict(dst=[0]),
                dict(out=torch.zeros(3, 3, dtype=torch.int32, device=DEV)), dict(out=torch.zeros(3, 4, device=DEV)),
                dict(idx=idx.long()), dict(idx=idx.cpu())):
        args = dict(idx=idx, K=[4], grid=[(1, 2, 2)], start=[(0, 0, 0)])
        args.update(bad)
        i = args.pop("idx")
        with pytest.raises((ValueError, tr.TRError)):
            tr.kept_positions(i, args.pop("K"), args.pop("grid"), args.pop("start"), **args)


# ---- rotation ----------------------------------------------------------------------
# (head_dim, rot_dim, sections): whole and partly rotated heads, widths that are
# and are not multiples of 16 bytes, one axis to four, axes without pairs
GEOMETRY = [(128, 128, (16, 24, 24)), (64, 64, (32,)), (128, 64, (8, 0, 24)), (80, 80, (10, 30)), (96, 48, (8, 8, 8)),
            (256, 256, (128,)), (256, 128, (16, 16, 16, 16)), (6, 4, (1, 1)), (130, 130, (65,)), (40, 36, (18,)),
            (1, 0, ()), (2, 2, (1,)), (16, 0, ()), (72, 72, (12, 12, 12))]


def inputs(dim, dtype, tokens, heads, kv_heads, how, g):
    """q and k as slices of one projection, as tensors of their own, head-major,
    or one element off 16-byte alignment."""
    if how == "packed":
        x = values(g, tokens, heads + 2 * kv_heads, dim, dtype=dtype).to(DEV)
        return x[:, :heads], x[:, heads:heads + kv_heads]
    if how == "head_major":
        return tuple(values(g, h, tokens, dim, dtype=dtype).to(DEV).transpose(0, 1) for h in (heads, kv_heads))
    if how == "odd":
        out = []
        for h in (heads, kv_heads):
            flat = torch.zeros(1 + tokens * h * (dim + 3), dtype=dtype, device=DEV)
            v = flat[1:].view(tokens, h, dim + 3)[..., :dim]
            v.copy_(values(g, tokens, h, dim, dtype=dtype))
            out.append(v)
        return tuple(out)
    return tuple(values(g, tokens, h, dim, dtype=dtype).to(DEV) for h in (heads, kv_heads))


def weights(dim, dtype, g, on):
    if not on:
        return None, None
    return tuple((1.0 + 0.3 * torch.randn(dim, generator=g)).to(dtype).to(DEV) for _ in range(2))


def positions(axes, tokens, g, most=40000):
    return torch.randint(-most // 8, most, (axes, tokens), generator=g).to(torch.int32)


def side64(x, w, pos, dim, rot, sections, adjacent, normed, eps):
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    ang = ref.angles(pos, freqs(rot), axis) if rot else torch.zeros(pos.shape[1], 0)
    v = x.detach().cpu().double()
    w64 = None if w is None else w.detach().cpu().double()
    if normed:
        v = ref.norm(v, w64, eps)
    return ref.turn(v, ang, rot, adjacent), ref.pair_norm(v, rot, adjacent), ang, w64


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("geometry", GEOMETRY)
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotate(geometry, dtype, adjacent):
    dim, rot, sections = geometry
    for n, (tokens, heads, kv_heads, how, normed, weighted) in enumerate([
            (1, 1, 1, "own", True, True), (3, 28, 4, "packed", True, True), (37, 6, 2, "odd", True, False),
            (19, 8, 8, "head_major", False, False), (65, 5, 5, "packed", False, False), (130, 3, 1, "own", True, True)]):
        say("rotate", geometry, dtype, adjacent, tokens, heads, kv_heads, how, normed)
        g = gen(dim * 31 + n)
        axes = max(1, len(sections))
        a = tr.Attention(heads, kv_heads, dim, dtype, rot_dim=rot, sections=sections if rot else None, adjacent=adjacent, norm=normed, eps=1e-6)
        q, k = inputs(dim, dtype, tokens, heads, kv_heads, how, g)
        wq, wk = weights(dim, dtype, g, weighted)
        pos = positions(axes, tokens, g)
        q0, k0 = q.clone(), k.clone()
        qo, ko = a.rotate(q, k, pos.to(DEV), wq=wq, wk=wk)
        assert torch.equal(q, q0) and torch.equal(k, k0)
        for x, w, got in ((q, wq, qo), (k, wk, ko)):
            want, scale, _, _ = side64(x, w, pos, dim, rot, sections, adjacent, normed, 1e-6)
            close(got, want, UNIT[dtype], scale, 3e-6, (geometry, how))
        # one side alone, and in place: the same bits
        q1, none = a.rotate(q, None, pos.to(DEV), wq=wq)
        assert none is None and torch.equal(q1, qo)
        none, k1 = a.rotate(None, k, pos.to(DEV), wk=wk)
        assert none is None and torch.equal(k1, ko)
        a.rotate(q, k, pos.to(DEV), wq=wq, wk=wk, q_out=q, k_out=k)
        assert torch.equal(q, qo) and torch.equal(k, ko)
        a.close()


def test_rotate_many_tokens():
    """More tokens than a launch has wavefronts, both types; a few rows checked."""
    for dtype in (BF, F32):
        tokens, heads, kv_heads, dim, sections = 20011, 28, 4, 128, (16, 24, 24)
        say("rotate many", dtype)
        a = tr.Attention(heads, kv_heads, dim, dtype, sections=sections, norm=True)
        g = gen(5)
        q, k = inputs(dim, dtype, tokens, heads, kv_heads, "packed", g)
        wq, wk = weights(dim, dtype, g, True)
        pos = positions(3, tokens, g)
        qo, ko = a.rotate(q, k, pos.to(DEV), wq=wq, wk=wk)
        some = torch.cat([torch.arange(0, tokens, 397), torch.arange(tokens - 40, tokens)])
        for x, w, got in ((q, wq, qo), (k, wk, ko)):
            want, scale, _, _ = side64(x[some.to(DEV)], w, pos[:, some], dim, dim, sections, False, True, 1e-6)
            close(got[some.to(DEV)], want, UNIT[dtype], scale, 3e-6, dtype)


def test_rotate_at_every_position():
    """Sines and cosines are right for positions up to the ends of int32."""
    dim = 128
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, 1 << 24, (1 << 24) + 1, 99999999, 123456789]], dtype=torch.int32)
    a = tr.Attention(2, 1, dim, F32)
    g = gen(9)
    q, k = inputs(dim, F32, pos.shape[1], 2, 1, "own", g)
    qo, ko = a.rotate(q, k, pos.to(DEV))
    # 1 / 2 pi in 53 bits, times an angle of 2^31: below 2^-24 of a turn, 3.8e-7
    for x, got in ((q, qo), (k, ko)):
        want, scale, _, _ = side64(x, None, pos, dim, dim, (64,), False, False, 0.0)
        close(got, want, UNIT[F32], scale, 3e-6, "positions")


def test_rotate_given_frequencies():
    """inv_freq and pair_axis of the caller's own: negative, zero and whole turns."""
    dim, pairs = 16, 8
    inv = [0.0, -1.0, 2 * math.pi, 100.0, 1e-9, 0.5, -3e-3, 1.0]
    axis = [1, 0, 2, 2, 1, 0, 1, 2]
    a = tr.Attention(3, 3, dim, F32, inv_freq=inv, pair_axis=axis, adjacent=True)
    assert a.axes == 3
    g = gen(4)
    q, k = inputs(dim, F32, 50, 3, 3, "own", g)
    pos = positions(3, 50, g, most=3000)
    qo, _ = a.rotate(q, k, pos.to(DEV))
    x = q.cpu().double()
    want, scale = ref.turn(x, ref.angles(pos, inv, axis), dim, True), ref.pair_norm(x, dim, True)
    close(qo, want, UNIT[F32], scale, 3e-6, "given")


def test_rotate_rows_of_zeros_and_eps():
    a = tr.Attention(2, 2, 64, F32, norm=True, eps=1e-6)
    q = torch.zeros(3, 2, 64, device=DEV)
    q[1] = 1e-20            # far below eps
    pos = torch.arange(3, dtype=torch.int32, device=DEV)
    qo, ko = a.rotate(q, q, pos)
    assert not qo[0].any() and not qo[2].any() and torch.isfinite(qo).all()
    want, scale, _, _ = side64(q, None, pos.cpu()[None], 64, 64, (32,), False, True, 1e-6)
    close(qo, want, UNIT[F32], scale, 3e-6, "eps")
    z = tr.Attention(2, 2, 64, F32, norm=True, eps=0.0)
    qo, _ = z.rotate(q, q, pos)
    assert torch.isnan(qo[0]).all()      # 0 / 0, as the formula


# ---- gradients ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("geometry", GEOMETRY)
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotate_backward(geometry, dtype, adjacent):
    dim, rot, sections = geometry
    for n, (tokens, heads, kv_heads, how, normed, weighted) in enumerate([
            (1, 1, 1, "own", True, True), (7, 28, 4, "packed", True, True), (37, 6, 2, "odd", True, False),
            (19, 8, 8, "head_major", False, False), (130, 3, 1, "own", True, True)]):
        say("rotate_backward", geometry, dtype, adjacent, tokens, heads, kv_heads, how, normed)
        g = gen(dim * 37 + n)
        axes = max(1, len(sections))
        a = tr.Attention(heads, kv_heads, dim, dtype, rot_dim=rot, sections=sections if rot else None, adjacent=adjacent, norm=normed, eps=1e-6)
        q, k = inputs(dim, dtype, tokens, heads, kv_heads, how, g)
        gq, gk = inputs(dim, dtype, tokens, heads, kv_heads, "own", g)
        wq, wk = weights(dim, dtype, g, weighted)
        pos = positions(axes, tokens, g)
        got = a.rotate_backward(gq, gk, q, k, pos.to(DEV), wq=wq, wk=wk)
        again = a.rotate_backward(gq, gk, q, k, pos.to(DEV), wq=wq, wk=wk)
        for u, v in zip(got, again):     # one order of the sums
            assert (u is None) == (v is None) and (u is None or torch.equal(u, v))
        for x, gr, w, dx, dw in ((q, gq, wq, got[0], got[2]), (k, gk, wk, got[1], got[3])):
            _, _, ang, w64 = side64(x, w, pos, dim, rot, sections, adjacent, normed, 1e-6)
            x64, g64 = x.cpu().double(), gr.cpu().double()
            want, want_w, mass = ref.backward(g64, x64, w64, ang, rot, adjacent, 1e-6, normed)
            if not normed:
                assert dw is None
                close(dx, want, UNIT[dtype], ref.pair_norm(g64, rot, adjacent), 3e-6, geometry)
                continue
            r = 1.0 / torch.sqrt((x64 * x64).mean(-1, keepdim=True) + 1e-6)
            gw = ref.turn(g64, -ang, rot, adjacent) * (1.0 if w64 is None else w64)
            # the terms of an element: its pair's gradient, and u times the mean
            scale = r * (ref.pair_norm(g64, rot, adjacent) * (1.0 if w64 is None else w64.abs())
                         + (x64 * r).abs() * (gw * x64 * r).pow(2).mean(-1, keepdim=True).sqrt())
            close(dx, want, UNIT[dtype], scale, 6e-6, geometry)
            assert dw.dtype == torch.float32
            close(dw, want_w, 0.0, mass + 1e-30, 5e-5, geometry)
        # one side alone and in place
        dq, none, dwq, nonew = a.rotate_backward(gq, None, q, None, pos.to(DEV), wq=wq)
        assert none is None and nonew is None and torch.equal(dq, got[0]) and (dwq is None or torch.equal(dwq, got[2]))
        dq, dk, _, _ = a.rotate_backward(gq, gk, q, k, pos.to(DEV), wq=wq, wk=wk, dq=gq, dk=gk)
        assert dq is gq and torch.equal(gq, got[0]) and torch.equal(gk, got[1])
        a.close()


def test_rotate_backward_many_tokens():
    """dw over more tokens than one pass of the launch, against float64 on the device."""
    for dtype in (BF, F32):
        tokens, heads, kv_heads, dim = 9001, 28, 4, 128
        say("rotate_backward many", dtype)
        a = tr.Attention(heads, kv_heads, dim, dtype, rot_dim=64, norm=True)
        g = gen(3)
        q, k = inputs(dim, dtype, tokens, heads, kv_heads, "packed", g)
        gq, gk = inputs(dim, dtype, tokens, heads, kv_heads, "own", g)
        wq, wk = weights(dim, dtype, g, True)
        pos = torch.arange(tokens, dtype=torch.int32)[None]
        dq, dk, dwq, dwk = a.rotate_backward(gq, gk, q, k, pos.to(DEV), wq=wq, wk=wk)
        _, _, ang, _ = side64(q[:, :1, :], wq, pos, dim, 64, (32,), False, True, 1e-6)
        for x, gr, w, dx, dw in ((q, gq, wq, dq, dwq), (k, gk, wk, dk, dwk)):
            want, want_w, mass = ref.backward(gr.cpu().double(), x.cpu().double(), w.cpu().double(), ang, 64, False, 1e-6, True)
            close(dw, want_w, 0.0, mass, 5e-5, dtype)


def test_rotate_backward_matches_differences():
    """<dx, d> and <dw, e> against central differences of the forward definition in 64 bits."""
    dim, rot, sections, tokens, heads = 24, 16, (3, 5), 6, 4
    g = gen(11)
    a = tr.Attention(heads, 2, dim, F32, rot_dim=rot, sections=sections, norm=True, eps=1e-6)
    q, k = inputs(dim, F32, tokens, heads, 2, "own", g)
    gq, gk = inputs(dim, F32, tokens, heads, 2, "own", g)
    wq, wk = weights(dim, F32, g, True)
    pos = positions(2, tokens, g)
    got = a.rotate_backward(gq, gk, q, k, pos.to(DEV), wq=wq, wk=wk)
    axis = [0] * 3 + [1] * 5
    ang = ref.angles(pos, freqs(rot), axis)
    for x, gr, w, dx, dw in ((q, gq, wq, got[0], got[2]), (k, gk, wk, got[1], got[3])):
        x, gr, w = (t.cpu().double() for t in (x, gr, w))
        f = lambda x, w: float((ref.turn(ref.norm(x, w, 1e-6), ang, rot, False) * gr).sum())
        h = 1e-5
        for _ in range(4):
            d, e = torch.randn(x.shape, generator=g).double(), torch.randn(w.shape, generator=g).double()
            # third derivatives times h^2, and 2^-52 of f over h: both below 1e-8 of the sums
            num = (f(x + h * d, w) - f(x - h * d, w)) / (2 * h)
            prod = dx.cpu().double() * d
            assert abs(num - float(prod.sum())) <= 1e-5 * float(prod.abs().sum())
            num = (f(x, w + h * e) - f(x, w - h * e)) / (2 * h)
            prod = dw.cpu().double() * e
            assert abs(num - float(prod.sum())) <= 1e-4 * float(prod.abs().sum())


def test_no_tokens():
    a = tr.Attention(4, 2, 32, F32, norm=True)
    e4, e2 = torch.empty(0, 4, 32, device=DEV), torch.empty(0, 2, 32, device=DEV)
    pos = torch.empty(1, 0, dtype=torch.int32, device=DEV)
    q, k = a.rotate(e4, e2, pos)
    assert q.shape == e4.shape and k.shape == e2.shape
    dq, dk, dwq, dwk = a.rotate_backward(e4, e2, e4, e2, pos)
    assert dq.shape == e4.shape and not dwq.any() and not dwk.any()


# ---- append ------------------------------------------------------------------------
def step_of(new, kv, page_size, g, spare_pages=3, width=None):
    counts = [(n + page_size - 1) // page_size for n in kv]
    pages = sum(counts) + spare_pages
    order = torch.randperm(pages, generator=g).to(torch.int32)
    width = max(counts + [1]) if width is None else width
    table = torch.full((len(kv), width), -1, dtype=torch.int32)
    r = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[r:r + c]
        r += c
    q_start = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32)
    return tr.Step(q_start, torch.tensor(kv, dtype=torch.int32), table), pages


def on_device(step):
    return tr.Step(*(t.to(DEV) for t in step))


def caches(pages, page_size, kv_heads, dim, dtype, g, layout="rows"):
    def one():
        if layout == "heads":         # [pages, kv_heads, page_size, dim] in memory
            return values(g, pages, kv_heads, page_size, dim, dtype=dtype).to(DEV).transpose(1, 2)
        return values(g, pages, page_size, kv_heads, dim, dtype=dtype).to(DEV)
    if layout == "joined":            # keys and values side by side
        both = values(g, pages, page_size, 2, kv_heads, dim, dtype=dtype).to(DEV)
        return tr.KVCache(both[:, :, 0], both[:, :, 1])
    return tr.KVCache(one(), one())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim,rot,sections", [(128, 128, (16, 24, 24)), (64, 32, (16,)), (80, 80, (20, 20)), (10, 6, (3,))])
@pytest.mark.parametrize("layout", ["rows", "heads", "joined"])
def test_append(dim, rot, sections, dtype, layout):
    for n, (new, kv, page_size, heads, kv_heads, how, normed) in enumerate([
            ([1], [1], 16, 4, 4, "packed", True), ([3, 0, 5, 1], [3, 7, 9, 33], 4, 8, 2, "packed", True),
            ([1] * 70, [1 + 3 * i for i in range(70)], 16, 7, 1, "own", False), ([200, 17], [201, 17], 48, 2, 2, "odd", True),
            ([40], [41], 1, 3, 3, "own", False)]):
        say("append", dim, dtype, layout, len(new), page_size, how)
        g = gen(dim + 7 * n)
        step, pages = step_of(new, kv, page_size, g)
        tokens = sum(new)
        a = tr.Attention(heads, kv_heads, dim, dtype, rot_dim=rot, sections=sections, norm=normed)
        q, k = inputs(dim, dtype, tokens, heads, kv_heads, how, g)
        _, v = inputs(dim, dtype, tokens, heads, kv_heads, how, g)
        wq, wk = weights(dim, dtype, g, normed)
        pos = positions(len(sections), tokens, g)
        cache = caches(pages, page_size, kv_heads, dim, dtype, g, layout)
        kept = [c.clone() for c in cache]
        want_q, want_k = a.rotate(q, k, pos.to(DEV), wq=wq, wk=wk)
        got = a.append(q, k, v, pos.to(DEV), cache, on_device(step), wq=wq, wk=wk)
        assert torch.equal(got, want_q)           # the same arithmetic: the same bits
        for b, t0, m, length in ref.sequences(step):
            for i in range(m):
                page, row = ref.place(step, b, length - m + i, page_size)
                kept[0][page, row], kept[1][page, row] = want_k[t0 + i], v[t0 + i]
        assert torch.equal(cache.k, kept[0]) and torch.equal(cache.v, kept[1])
        # keys and values alone
        cache.k.zero_()
        cache.v.zero_()
        assert a.append(None, k, v, pos.to(DEV), cache, on_device(step), wk=wk) is None
        for b, t0, m, length in ref.sequences(step):
            for i in range(m):
                page, row = ref.place(step, b, length - m + i, page_size)
                assert torch.equal(cache.k[page, row], want_k[t0 + i]) and torch.equal(cache.v[page, row], v[t0 + i])
        a.close()


def test_append_leaves_what_is_not_its_own():
    """Rows of no sequence, tokens before the sequence's first or past the table,
    and pages out of range: nothing is written for them."""
    say("append bounds")
    g = gen(2)
    dim, page_size = 32, 4
    a = tr.Attention(4, 2, dim, F32)
    cache = caches(6, page_size, 2, dim, F32, g)
    before = [c.clone() for c in cache]
    # packed rows: 1 of none; seq 0: 5 new of a length of 3 (two come before its first token);
    # seq 1: 2 new, its second page out of range; seq 2: past the table; 2 rows of none at the end
    step = tr.Step(torch.tensor([1, 6, 8, 10], dtype=torch.int32), torch.tensor([3, 5, 12], dtype=torch.int32),
                   torch.tensor([[0, 1], [2, 6], [4, -1]], dtype=torch.int32))
    tokens = 12
    q, k = inputs(dim, F32, tokens, 4, 2, "own", g)
    v = values(g, tokens, 2, dim, dtype=F32).to(DEV)
    pos = torch.arange(tokens, dtype=torch.int32, device=DEV)
    q_out = torch.full((tokens, 4, dim), 7.0, device=DEV)
    want_q, want_k = a.rotate(q, k, pos)
    a.append(q, k, v, pos, cache, on_device(step), q_out=q_out)
    assert (q_out[[0, 10, 11]] == 7.0).all() and torch.equal(q_out[1:10], want_q[1:10])
    for t, page, row in ((3, 0, 0), (4, 0, 1), (5, 0, 2), (6, 2, 3)):
        before[0][page, row], before[1][page, row] = want_k[t], v[t]
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])


def test_append_far_pages():
    """Element offsets beyond 2^32 in a cache of more than 8 GB a side."""
    say("append far")
    dim, kv_heads, page_size = 128, 8, 1024
    pages = 4200                                   # 4200 * 2^20 elements
    k_cache, v_cache = (torch.zeros(pages, page_size, kv_heads, dim, dtype=BF, device=DEV) for _ in range(2))
    a = tr.Attention(8, 8, dim, BF)
    g = gen(1)
    q, k = inputs(dim, BF, 2, 8, 8, "own", g)
    v = values(g, 2, 8, dim, dtype=BF).to(DEV)
    step = tr.Step(*(torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 2], [1025], [[4199, 4100]])))
    pos = torch.arange(2, dtype=torch.int32, device=DEV)
    _, want_k = a.rotate(q, k, pos)
    a.append(q, k, v, pos, tr.KVCache(k_cache, v_cache), step)
    assert torch.equal(k_cache[4199, 1023], want_k[0]) and torch.equal(k_cache[4100, 0], want_k[1])
    assert torch.equal(v_cache[4199, 1023], v[0]) and torch.equal(v_cache[4100, 0], v[1])
    assert not k_cache[:4100].any()


# ---- refusals ----------------------------------------------------------------------
def test_create_refusals():
    for bad in (dict(heads=6, kv_heads=4), dict(heads=0), dict(head_dim=257), dict(head_dim=0), dict(rot_dim=3), dict(rot_dim=66),
                dict(sections=(1, 2)), dict(sections=(33, -1)), dict(sections=(8, 8, 8, 4, 4)), dict(pair_axis=[0] * 31), dict(pair_axis=[5] + [0] * 31),
                dict(inv_freq=[1.0]), dict(inv_freq=[math.nan] * 32), dict(base=0.0), dict(base=math.inf), dict(norm=True, eps=-1.0),
                dict(norm=True, eps=math.nan), dict(sections=(32,), pair_axis=[0] * 32)):
        args = dict(heads=4, kv_heads=2, head_dim=64, dtype=BF)
        args.update(bad)
        with pytest.raises((ValueError, tr.TRError)):
            tr.Attention(args.pop("heads"), args.pop("kv_heads"), args.pop("head_dim"), args.pop("dtype"), **args)
    with pytest.raises(TypeError):
        tr.Attention(4, 2, 64, torch.float16)


def test_call_refusals():
    a = tr.Attention(4, 2, 64, F32)
    n = tr.Attention(4, 2, 64, F32, norm=True)
    T = 3
    q, k = torch.zeros(T, 4, 64, device=DEV), torch.zeros(T, 2, 64, device=DEV)
    pos = torch.zeros(1, T, dtype=torch.int32, device=DEV)
    w = torch.ones(64, device=DEV)
    bad = [lambda: a.rotate(None, None, pos), lambda: a.rotate(q.bfloat16(), k, pos), lambda: a.rotate(q.cpu(), k, pos),
           lambda: a.rotate(k, q, pos), lambda: a.rotate(q, k[:2], pos), lambda: a.rotate(q, k, pos.long()),
           lambda: a.rotate(q, k, pos[:, :2]), lambda: a.rotate(q, k, pos.expand(2, T)), lambda: a.rotate(q, k, pos, wq=w),
           lambda: n.rotate(q, k, pos, wq=w[:32]), lambda: n.rotate(q, k, pos, wq=w.bfloat16()),
           lambda: a.rotate(q, k, pos, q_out=torch.zeros(T, 1, 64, device=DEV).expand(T, 4, 64)),
           lambda: a.rotate(q.transpose(1, 2).contiguous().transpose(1, 2), k, pos),
           lambda: n.rotate_backward(q, k, None, k, pos), lambda: n.rotate_backward(None, None, q, k, pos)]
    cache = tr.KVCache(*(torch.zeros(3, 4, 2, 64, device=DEV) for _ in range(2)))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    step = tr.Step(i32([0, 3]), i32([3]), i32([[0]]))
    bad += [lambda: a.append(q, k, k[:2], pos, cache, step), lambda: a.append(q, k, k, pos, cache._replace(v=cache.v[:2]), step),
            lambda: a.append(q, k, k, pos, cache._replace(v=cache.v.transpose(0, 1).contiguous().transpose(0, 1)), step),
            lambda: a.append(q, k, k, pos, tr.KVCache(*(c[:0] for c in cache)), step),
            lambda: a.append(q, k, k, pos, tr.KVCache(*(c[:1].expand(3, 4, 2, 64) for c in cache)), step),
            lambda: a.append(q, k, k, pos, cache, step._replace(q_start=i32([0, 1, 3]))),
            lambda: a.append(q, k, k, pos, cache, step._replace(kv_len=torch.tensor([3], device=DEV))),
            lambda: a.append(q, k, k, pos, cache, tr.Step(i32([0]), i32([]), i32([[]]).view(0, 1)))]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, AttributeError, tr.TRError)):
            f()
            print("not refused:", i)
    qo, ko = a.rotate(q, k[:, :1].expand(T, 2, 64), pos)      # broadcast inputs are fine
    assert ko.shape == (T, 2, 64)


# ---- streams and graphs ----------------------------------------------------------------
def test_calls_are_ordered_on_their_stream():
    """Inputs made on a stream of their own right before the call on it."""
    a = tr.Attention(28, 4, 128, BF, norm=True)
    side = torch.cuda.Stream()
    pos = torch.arange(4000, dtype=torch.int32, device=DEV)
    x = torch.zeros(4000, 32, 128, dtype=BF, device=DEV)
    y = torch.randn(4000, 32, 128, device=DEV).to(BF)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            x.copy_(y)
            x.mul_(0.5)
        x.copy_(y)
    q, k = a.rotate(x[:, :28], x[:, 28:], pos, stream=side)
    side.synchronize()
    q1, k1 = a.rotate(y[:, :28], y[:, 28:], pos)
    assert torch.equal(q, q1) and torch.equal(k, k1)


def test_append_replays_from_a_graph():
    """A recorded step replays with the lengths, tables and tokens it finds then."""
    g = gen(8)
    dim, page_size, seqs = 64, 8, 5
    a = tr.Attention(6, 2, dim, BF, norm=True)
    x = torch.zeros(seqs, 10, dim, dtype=BF, device=DEV)
    pos = torch.zeros(1, seqs, dtype=torch.int32, device=DEV)
    table = torch.randperm(40, generator=g).to(torch.int32).view(seqs, 8).to(DEV)
    step = tr.Step(torch.arange(seqs + 1, dtype=torch.int32, device=DEV), torch.zeros(seqs, dtype=torch.int32, device=DEV), table)
    cache = tr.KVCache(*(torch.zeros(40, page_size, 2, dim, dtype=BF, device=DEV) for _ in range(2)))
    q_out = torch.empty(seqs, 6, dim, dtype=BF, device=DEV)
    call = lambda c, o: a.append(x[:, :6], x[:, 6:8], x[:, 8:], pos, c, step, q_out=o)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(cache, q_out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(cache, q_out)
    for i in range(5):
        x.copy_(values(g, seqs, 10, dim, dtype=BF))
        step.kv_len.copy_(torch.randint(1, 64, (seqs,), generator=g).to(torch.int32))
        pos.copy_(torch.randint(0, 999, (1, seqs), generator=g).to(torch.int32))
        other, q1 = tr.KVCache(*(c.clone() for c in cache)), torch.empty_like(q_out)
        call(other, q1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, q1) and torch.equal(cache.k, other.k) and torch.equal(cache.v, other.v)
