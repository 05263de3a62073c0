"""Attention over 8-bit values whose scales are among fp32's largest: results are finite
where the definition's are, sums of many keys and of keys whose weights come after the
running maximum included.  Tolerances are those of test_gpu_attend8."""
import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_attend import queries
from test_gpu_attend8 import E4M3, KERNELS, cache8, stands_for
from test_gpu_attend_edges import definition
from test_gpu_rotate import BF, DEV, gen, on_device, say, step_of

pytestmark = pytest.mark.gpu

TOP = 2.0 ** 127                     # of the values; bf16's largest is close to 2^128
SCALES = (2.0 ** 119, 2.0 ** 120, 1.5 * 2.0 ** 119, 2.0 ** 127)


def held(a, q, cache, step, causal, what, scale=None):
    s = q.shape[2] ** -0.5 if scale is None else scale
    got, lse = a.attend(q, cache, on_device(step), scale=s, causal=causal, want_lse=True)
    want, want_lse, mass, most = definition(q, tr.KVCache(*(t.to(DEV) for t in stands_for(cache))), step, s, causal)
    assert torch.isfinite(want).all() and torch.isfinite(got).all(), what
    assert float(((got.double() - want).abs() - 2.0 ** -8 * want.abs() - (2.0 ** -8 + 1.5e-3) * mass).max()) <= 0.0, what
    assert float(((lse.double() - want_lse).abs() - 2e-5 * (1.0 + most)).max()) <= 0.0, what


def large(t, scale, g, signs):
    """Codes that stand for values up to TOP, from its half on where all are positive."""
    x = torch.rand(t.shape, generator=g)
    x = 2.0 * x - 1.0 if signs else 0.5 + 0.5 * x
    t.copy_((x * (TOP / scale)).clamp(-448, 448).to(E4M3))


@pytest.mark.parametrize("page_size,block", [(16, 16), (24, 8)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kernel", KERNELS)
def test_large_values(kernel, dim, page_size, block):
    new, kv, heads, kv_heads, causal = KERNELS[kernel]
    g = gen(dim + block)
    step, pages = step_of(new, kv, page_size, g)
    a = tr.Attention(heads, kv_heads, dim, BF)
    cache = cache8(pages, page_size, kv_heads, dim, g, block)
    q = queries(g, sum(new), heads, dim).to(DEV)
    for scale in SCALES if kernel not in ("in_turn", "items") else SCALES[1:3]:
        say("large", kernel, dim, page_size, scale)
        cache.v_scale.fill_(scale)
        large(cache.v, scale, g, True)
        held(a, q, cache, step, causal, ("random", scale))
        # equal weights of many keys
        keys = cache.k.clone()
        cache.k.zero_()
        large(cache.v, scale, g, False)
        held(a, q, cache, step, causal, ("equal", scale))
        # then a late key whose weight is 2^7.2 times the others'
        cache.k_scale.fill_(1.0)
        for b, (n, length) in enumerate(zip(new, kv)):
            if n:
                at = length - n
                cache.k[step.table[b][at // page_size].long(), at % page_size] = 0.5
        held(a, torch.ones_like(q), cache, step, causal, ("late", scale), scale=10.0 / dim)
        cache.k.copy_(keys)
        cache.k_scale.fill_(2.0 ** -7)
    a.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kernel", [k for k in KERNELS if k not in ("in_turn", "items")])
def test_large_blocks_among_ordinary_ones(kernel, dim):
    """One block of a large scale: the rows that see it, and those that do not; and with
    values of zero, where the ordinary ones are the result."""
    new, kv, heads, kv_heads, causal = KERNELS[kernel]
    g = gen(dim)
    for page_size, block in ((16, 16), (24, 8)):
        say("among", kernel, dim, page_size)
        step, pages = step_of(new, kv, page_size, g)
        a = tr.Attention(heads, kv_heads, dim, BF)
        cache = cache8(pages, page_size, kv_heads, dim, g, block)
        q = queries(g, sum(new), heads, dim).to(DEV)
        for scale in (2.0 ** 80, 2.0 ** 81, 1.25 * 2.0 ** 90, 2.0 ** 119):
            for b, (n, length) in enumerate(zip(new, kv)):
                at = (length - n, length - 1 - n // 2, 0)[b % 3] if n else 0
                page, row = step.table[b][at // page_size].long(), at % page_size
                cache.v_scale[page, row // block, b % kv_heads] = scale
            held(a, q, cache, step, causal, scale)
            where = cache.v_scale.repeat_interleave(block, 1) > 1e20
            kept = cache.v.clone()
            cache.v.view(torch.uint8)[where] = 0
            held(a, q, cache, step, causal, (scale, "zeros"))
            cache.v.copy_(kept)
        a.close()
