"""Sizes and values at the ends of what the rotation takes."""
import pytest
import torch

import attn_ref as ref
import paper_2607_13500_amd as tr
from test_gpu_rotate import BF, DEV, F32, UNIT, close, freqs, gen, inputs, positions, say, side64, values, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,heads,dim", [(4200007, 16, 6), (67200003, 1, 8)])
def test_more_heads_than_a_launch_has_threads_for(tokens, heads, dim):
    """2^26 wavefronts and more of 64 threads: heads of any kind, and tokens of heads of
    whole pieces.  The same bits as the two halves by themselves."""
    say("large", tokens, heads, dim)
    g = torch.Generator(device=DEV).manual_seed(1)
    a = tr.Attention(heads, heads, dim, BF, norm=True)
    q = torch.randn(tokens, heads, dim, generator=g, device=DEV, dtype=BF)
    pos = torch.randint(0, 1000, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    out, _ = a.rotate(q, None, pos)
    half = tokens // 2
    for part in (slice(0, half), slice(half, tokens)):
        want, _ = a.rotate(q[part], None, pos[part])
        assert torch.equal(out[part], want)
    a.close()


def test_positions_of_as_many_tokens_as_an_index_counts():
    """2^31 - 1 kept tokens: the launch's last threads have no token."""
    kept = 2 ** 31 - 1
    say("positions", kept)
    idx = torch.zeros(kept, dtype=torch.int32, device=DEV)
    T, H, W = 3, 17, 42107522
    idx[-1] = T * H * W - 1
    pos = tr.kept_positions(idx, [kept], [(T, H, W)], [(5, -6, 7)])
    assert pos[:, -1].tolist() == [5 + T - 1, H - 1 - 6, 7 + W - 1]
    for row, first in zip(pos, (5, -6, 7)):
        assert (row[:-1] == first).all()


def test_one_row_of_positions_for_all_axes():
    """Text counts alike on every axis: an expanded row of positions."""
    a = tr.Attention(4, 2, 64, BF, sections=(16, 8, 8), norm=True)
    g = torch.Generator(device=DEV).manual_seed(2)
    q, k = (torch.randn(50, h, 64, generator=g, device=DEV, dtype=BF) for h in (4, 2))
    text = torch.arange(50, dtype=torch.int32, device=DEV)
    whole, shared = text.expand(3, 50).contiguous(), text.expand(3, 50)
    for want, got in zip(a.rotate(q, k, whole), a.rotate(q, k, shared)):
        assert torch.equal(want, got)
    for want, got in zip(a.rotate_backward(q, k, q, k, whole), a.rotate_backward(q, k, q, k, shared)):
        assert torch.equal(want, got)
    # and rows that overlap, as windows of one range do
    windows = torch.arange(60, dtype=torch.int32, device=DEV).unfold(0, 50, 5)
    for want, got in zip(a.rotate(q, k, windows.contiguous()), a.rotate(q, k, windows)):
        assert torch.equal(want, got)


def test_angles_up_to_2_to_the_64():
    """Frequencies far above 1: fractions of a turn of angles that fp64 holds only to
    whole turns."""
    dim, inv = 32, [1.0, 3.7, 1e3, 12345.678, 1e5, 2.0 ** 20, 1e7, 1e8, 2.0 ** 30 + 1e3, 5e9, 8.5e9, -8.5e9, -1e6, 3e-9, 0.25, 7e9]
    pos = torch.tensor([[1, -1, 2 ** 31 - 1, -2 ** 31, 123456789, 2 ** 30 + 12345, 1 << 24, 7, 99, 2000000011]], dtype=torch.int32)
    a = tr.Attention(2, 2, dim, F32, inv_freq=inv)
    q = values(gen(5), pos.shape[1], 2, dim, dtype=F32).to(DEV)
    got, _ = a.rotate(q, None, pos.to(DEV))
    x = q.cpu().double()
    want = ref.turn(x, ref.angles(pos, inv, [0] * len(inv)), dim, False)
    close(got, want, UNIT[F32], ref.pair_norm(x, dim, False), 3e-6, "large angles")


def test_angles_are_those_of_positions_and_frequencies():
    """The fp32 product stands for position times frequency: the position, the
    frequency and the product are rounded by 2^-24 each, so the angle is off by less
    than 3 * 2^-24 of itself, and an element by that of its pair's length."""
    dim, rot = 64, 64
    inv = freqs(rot)
    pos = torch.cat([torch.arange(0, 40000, 37), torch.tensor([131071, 262143, 1048575])]).to(torch.int32)[None]
    a = tr.Attention(1, 1, dim, F32)
    q = values(gen(6), pos.shape[1], 1, dim, dtype=F32).to(DEV)
    got, _ = a.rotate(q, None, pos.to(DEV))
    x = q.cpu().double()
    angle = pos[0].double()[:, None] * torch.tensor(inv, dtype=torch.float64)      # below 2^20: its 2^-53 are nothing here
    want, length = ref.turn(x, angle, rot, False), ref.pair_norm(x, rot, False)
    off = 3 * 2.0 ** -24 * torch.cat([angle, angle], 1)[:, None]
    over = (got.cpu().double() - want).abs() - 2.0 ** -24 * want.abs() - (3e-6 + off) * length
    assert float(over.max()) <= 0.0


# ---- heads far from 1: squares beyond fp32, and below it -------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("how", ["own", "odd"])
@pytest.mark.parametrize("dim,adjacent", [(128, False), (64, True), (24, False), (256, True)])
def test_norm_of_heads_of_every_size(dim, adjacent, how, dtype):
    """Tolerances as in test_gpu_rotate: the norm does not depend on a head's size."""
    sizes = torch.tensor([1.0, 1e-36, 1e25, 1e-19, 1e30, 1e-25, 3e18, 3e37, 1e-15, 1e19, 0.1])
    for eps in (0.0, 1e-6, 1e-33):
        say("sizes", dim, adjacent, how, dtype, eps)
        g = gen(dim)
        tokens, heads, kv_heads = len(sizes), 6, 2
        a = tr.Attention(heads, kv_heads, dim, dtype, adjacent=adjacent, norm=True, eps=eps)
        q, k = inputs(dim, dtype, tokens, heads, kv_heads, how, g)
        order = torch.stack([sizes.roll(h) for h in range(heads)], 1)[..., None].to(DEV)      # other sizes beside each other
        for x in (q, k):
            x.copy_((torch.randn(x.shape, generator=g).clamp(-4, 4).to(DEV) * order[:, :x.shape[1]]).to(dtype))
        wq, wk = weights(dim, dtype, g, True)
        pos = positions(1, tokens, g)
        for x, w, got in zip((q, k), (wq, wk), a.rotate(q, k, pos.to(DEV), wq=wq, wk=wk)):
            want, _, ang, w64 = side64(x, w, pos, dim, dim, (dim // 2,), adjacent, True, eps)
            unit = ref.norm(x.cpu().double(), w64, eps)
            close(got, want, UNIT[dtype], ref.pair_norm(unit, dim, adjacent), 3e-6, eps)
        # gradients, of heads whose own stay in the type's range
        for x in (q, k):
            size = order[:, :x.shape[1]].expand(x.shape)
            x[(size < 1e-30) | (size > 2e30)] = 0.5
        gq, gk = inputs(dim, dtype, tokens, heads, kv_heads, "own", g)
        got = a.rotate_backward(gq, gk, q, k, pos.to(DEV), wq=wq, wk=wk)
        for x, gr, w, dx, dw in ((q, gq, wq, got[0], got[2]), (k, gk, wk, got[1], got[3])):
            _, _, ang, w64 = side64(x, w, pos, dim, dim, (dim // 2,), adjacent, True, eps)
            x64, g64 = x.cpu().double(), gr.cpu().double()
            want, want_w, mass = ref.backward(g64, x64, w64, ang, dim, adjacent, eps, True)
            r = 1.0 / torch.sqrt((x64 * x64).mean(-1, keepdim=True) + eps)
            gw = ref.turn(g64, -ang, dim, adjacent) * w64
            scale = r * (ref.pair_norm(g64, dim, adjacent) * w64.abs() + (x64 * r).abs() * (gw * x64 * r).pow(2).mean(-1, keepdim=True).sqrt())
            close(dx, want, UNIT[dtype], scale, 6e-6, eps)
            close(dw, want_w, 0.0, mass, 5e-5, eps)
        a.close()
