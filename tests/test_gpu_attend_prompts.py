"""Prompts whose tiles see only part of their sequence: the workgroups take whole
items in turn.  Tolerances as in test_gpu_attend."""
import math

import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_attend import normal_caches, queries
from test_gpu_rotate import BF, DEV, gen, on_device, say, step_of

pytestmark = pytest.mark.gpu


def definition(q, cache, step, window):
    """(out, lse, sum w |v|, largest |score|) in 64 bits, a head of a sequence at a time."""
    page, group = cache.k.shape[1], q.shape[1] // cache.k.shape[2]
    out, mass = (torch.zeros(q.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    lse, most = (torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV) for _ in range(2))
    for b, kv in enumerate(step.kv_len.tolist()):
        t0, t1 = step.q_start[b].item(), step.q_start[b + 1].item()
        j = torch.arange(kv, device=DEV)
        rows = step.table[b].to(DEV).long()[j // page] * page + j % page
        behind = torch.arange(kv - (t1 - t0), kv, device=DEV)[:, None] - j
        hide = (behind < 0) | (behind >= window) if window else behind < 0
        for h in range(q.shape[1]):
            k, v = (c.flatten(0, 1)[rows, h // group].double() for c in cache)
            s = torch.matmul(q[t0:t1, h].double(), k.t().contiguous()) / math.sqrt(q.shape[2])
            most[t0:t1, h] = s.masked_fill(hide, 0.0).abs().amax(1)
            s = s.masked_fill(hide, -math.inf)
            lse[t0:t1, h] = torch.logsumexp(s, 1)
            w = torch.exp(s - lse[t0:t1, h, None])
            out[t0:t1, h], mass[t0:t1, h] = torch.matmul(w, v), torch.matmul(w, v.abs())
    return out, lse, mass, most


@pytest.mark.parametrize("new,kv,heads,kv_heads,dim,window,page_size", [
    ([1200], [1200], 80, 80, 64, 0, 64), ([1500], [3000], 16, 16, 64, 100, 16), ([3000], [3000], 32, 8, 128, 0, 48),
    ([700, 1, 0, 900], [700, 300, 20, 1000], 40, 20, 80, 0, 64), ([2000, 33], [2100, 4000], 16, 8, 128, 1, 7),
    ([1500, 64], [1500, 2000], 14, 14, 256, 300, 64)])
def test_prompts(new, kv, heads, kv_heads, dim, window, page_size):
    say("prompts", new, kv, heads, kv_heads, dim, window, page_size)
    g = gen(sum(kv) + dim)
    step, pages = step_of(new, kv, page_size, g)
    cache = normal_caches(pages, page_size, kv_heads, dim, g)
    q = queries(g, sum(new), heads, dim).to(DEV)
    a = tr.Attention(heads, kv_heads, dim, BF)
    got, got_lse = a.attend(q, cache, on_device(step), window=window, want_lse=True)
    again, _ = a.attend(q, cache, on_device(step), window=window)
    assert torch.equal(got, again)
    want, lse, mass, most = definition(q, cache, step, window)
    assert float(((got.double() - want).abs() - 2.0 ** -8 * want.abs() - (2.0 ** -8 + 1.5e-3) * mass).max()) <= 0.0
    assert float(((got_lse.double() - lse).abs() - 2e-5 * (1.0 + most)).max()) <= 0.0


def test_numbers_beyond_fp32_are_refused():
    with pytest.raises(tr.TRError):
        tr.Attention(4, 2, 64, BF, inv_freq=[1e300] * 32)
    a = tr.Attention(4, 2, 64, BF)
    g = gen(2)
    step, pages = step_of([3], [40], 16, g)
    with pytest.raises(tr.TRError):
        a.attend(queries(g, 3, 4, 64).to(DEV), normal_caches(pages, 16, 2, 64, g), on_device(step), scale=1e300)
