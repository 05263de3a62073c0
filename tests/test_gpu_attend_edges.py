"""Attention's edges in each of its kernels: the one for few rows, and the one for
many by shares of all steps, by whole items in turn, and by an item a workgroup.
Tolerances as in test_gpu_attend."""
import math

import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_attend import normal_caches
from test_gpu_rotate import BF, DEV, gen, on_device, say, step_of

pytestmark = pytest.mark.gpu

# new tokens, lengths, heads, key heads, causal
KERNELS = {"few": ([3, 1], [700, 90], 4, 2, True), "shares": ([70, 130], [701, 300], 4, 2, False),
           "in_turn": ([1200], [1200], 80, 80, True), "items": ([2048], [2050], 64, 64, True)}


def definition(q, cache, step, scale, causal, window=0):
    """(out, lse, sum w |v|, largest |score|) in 64 bits, a head of a sequence at a time."""
    page, group = cache.k.shape[1], q.shape[1] // cache.k.shape[2]
    out, mass = (torch.zeros(q.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    lse, most = (torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV) for _ in range(2))
    for b, kv in enumerate(step.kv_len.tolist()):
        t0, t1 = step.q_start[b].item(), step.q_start[b + 1].item()
        j = torch.arange(kv, device=DEV)
        rows = step.table[b].to(DEV).long()[j // page] * page + j % page
        behind = torch.arange(kv - (t1 - t0), kv, device=DEV)[:, None] - j
        hide = (behind < 0) & causal
        if window:
            hide = hide | (behind >= window)
        for h in range(q.shape[1]):
            k, v = (c.flatten(0, 1)[rows, h // group].double() for c in cache)
            s = torch.matmul(q[t0:t1, h].double(), k.t().contiguous()) * scale
            most[t0:t1, h] = s.masked_fill(hide, 0.0).abs().amax(1)
            s = s.masked_fill(hide, -math.inf)
            lse[t0:t1, h] = torch.logsumexp(s, 1)
            w = torch.exp(s - lse[t0:t1, h, None])
            out[t0:t1, h], mass[t0:t1, h] = torch.matmul(w, v), torch.matmul(w, v.abs())
    return out, lse, mass, most


def compare(a, q, cache, step, scale, causal):
    got, got_lse = a.attend(q, cache, on_device(step), scale=scale, causal=causal, want_lse=True)
    again, _ = a.attend(q, cache, on_device(step), scale=scale, causal=causal)
    assert torch.equal(got, again)
    want, lse, mass, most = definition(q, cache, step, scale, causal)
    assert torch.isfinite(got).all() and torch.isfinite(got_lse).all()
    assert float(((got.double() - want).abs() - 2.0 ** -8 * want.abs() - (2.0 ** -8 + 1.5e-3) * mass).max()) <= 0.0
    assert float(((got_lse.double() - lse).abs() - 2e-5 * (1.0 + most)).max()) <= 0.0


def inputs(kernel, dim, page_size, g):
    new, kv, heads, kv_heads, causal = KERNELS[kernel]
    step, pages = step_of(new, kv, page_size, g)
    return (torch.randn(sum(new), heads, dim, generator=g).to(BF), normal_caches(pages, page_size, kv_heads, dim, g), step,
            tr.Attention(heads, kv_heads, dim, BF), causal)


@pytest.mark.parametrize("dim", [64, 128, 80, 256])
@pytest.mark.parametrize("kernel", KERNELS)
def test_partial_sums_that_cancel(kernel, dim):
    """Scores of ordinary size whose sums over the first elements of a head are
    thousands: the last elements take them back.  All elements are multiples of 1/8
    of at most 16, so every partial sum (below 2^13, a multiple of 2^-6) is exact."""
    say("cancel", kernel, dim)
    g = gen(dim)
    q, cache, step, a, causal = inputs(kernel, dim, 16, g)
    eighths = lambda t: (8.0 * t.float()).round().clamp(-24, 24) / 8.0
    for sign in (1.0, -1.0):          # the partial sums far above, and far below
        q = eighths(q).to(BF)
        q[..., :16] = q[..., dim - 16:] = 16.0
        cache.k.copy_(eighths(cache.k))
        cache.k[..., :16], cache.k[..., dim - 16:] = 16.0 * sign, -16.0 * sign
        compare(a, q.to(DEV), cache, step, 1.0 / math.sqrt(dim), causal)
    a.close()


@pytest.mark.parametrize("new,kv,heads,kv_heads,causal,window", [
    ([64], [50], 2, 2, False, 0), ([70, 90], [64, 129], 4, 2, False, 0), ([1], [90], 33, 1, True, 20), ([1, 1], [65, 700], 40, 1, True, 0),
    ([2048], [70], 64, 64, False, 0), ([2], [50], 2, 2, False, 0)])
def test_infinite_values_at_the_ends_of_what_is_seen(new, kv, heads, kv_heads, causal, window):
    """All rows see the same keys, whose first and last values are infinite: those
    elements are infinite, all others as they are without."""
    for dim, page_size in ((64, 16), (128, 48), (80, 7), (256, 16)):
        say("ends", new, kv, heads, causal, window, dim)
        g = gen(dim + heads)
        step, pages = step_of(new, kv, page_size, g)
        cache = normal_caches(pages, page_size, kv_heads, dim, g)
        q = torch.randn(sum(new), heads, dim, generator=g).to(BF).to(DEV)
        a = tr.Attention(heads, kv_heads, dim, BF)
        ends = []
        for b, n in enumerate(kv):
            for j in (max(0, n - window) if window else 0, n - 1):
                ends.append((int(step.table[b, j // page_size]), j % page_size))
        for e, (page, row) in zip((3, 40, 5, 6), ends):
            cache.v[page, row, :, e] = 0.0
        clean, lse = a.attend(q, cache, on_device(step), causal=causal, window=window, want_lse=True)
        want = clean.clone()
        for i, (e, (page, row)) in enumerate(zip((3, 40, 5, 6), ends)):
            sign = -1.0 if i % 2 else 1.0
            cache.v[page, row, :, e] = sign * math.inf
            first = sum(new[:i // 2])
            want[first:first + new[i // 2], :, e] = sign * math.inf
        got, got_lse = a.attend(q, cache, on_device(step), causal=causal, window=window, want_lse=True)
        assert torch.equal(got, want) and torch.equal(got_lse, lse)
        a.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kernel", KERNELS)
def test_scores_of_every_size(kernel, dim):
    """Scales of both signs and zero, a running maximum that rises all the way, one
    key far above the others, scores all far below zero."""
    say("scores", kernel, dim)
    g = gen(dim + 1)
    q, cache, step, a, causal = inputs(kernel, dim, 16, g)
    q = q.to(DEV)
    for scale in (0.0, -0.125, 1e-3, -1e-30):
        compare(a, q, cache, step, scale, causal)
    kept = cache.k.clone()
    most = max(step.kv_len.tolist())
    # of equal elements: sums over a head are exact.  Up, then down
    fours = torch.full_like(q, 4.0)
    rise = torch.arange(most, dtype=torch.float32) * 0.004
    for b, kv in enumerate(step.kv_len.tolist()):
        j = torch.arange(kv)
        cache.k[step.table[b].long()[j // 16].to(DEV), (j % 16).to(DEV)] = rise[:kv].to(BF).to(DEV)[:, None, None]
    for scale in (1.0 / math.sqrt(dim), -1.0 / math.sqrt(dim)):
        compare(a, fours, cache, step, scale, causal)
    cache.k.copy_(kept)
    for b, kv in enumerate(step.kv_len.tolist()):
        cache.k[int(step.table[b, (kv * 3 // 4) // 16]), (kv * 3 // 4) % 16] = 30.0
    compare(a, fours, cache, step, 1.0 / math.sqrt(dim), causal)
    cache.k.copy_(-kept.abs() - 20.0)
    compare(a, (20.0 + 0.01 * q.float()).to(BF), cache, step, 0.125 / 400, causal)
    a.close()


@pytest.mark.parametrize("kernel", KERNELS)
def test_not_finite_values_that_are_seen(kernel):
    """A NaN key makes the rows NaN that see it; a value's NaN or infinity stays in
    its element, of the rows that see it."""
    say("seen", kernel)
    dim, at = 64, 41
    new, kv, _, kv_heads, causal = KERNELS[kernel]
    q, cache, step, a, causal = inputs(kernel, dim, 16, gen(3))
    q, group = q.to(DEV), a.heads // kv_heads
    clean, lse = a.attend(q, cache, on_device(step), causal=causal, want_lse=True)
    page, row = int(step.table[0, at // 16]), at % 16
    sees = torch.zeros(sum(new), dtype=torch.bool, device=DEV)
    sees[:new[0]] = torch.arange(new[0], device=DEV) + kv[0] - new[0] >= at if causal else True
    cache.v[page, row, 1, 5], cache.v[page, row, 0, 9], cache.v[page, row, 1, 63] = math.inf, math.nan, -math.inf
    out, out_lse = a.attend(q, cache, on_device(step), causal=causal, want_lse=True)
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(out_lse, lse)
    first, second = slice(0, group), slice(group, 2 * group)
    assert (out[sees, second, 5] == math.inf).all() and (out[sees, second, 63] == -math.inf).all() and torch.isnan(out[sees, first, 9]).all()
    out[sees, second, 5] = out[sees, second, 63] = out[sees, first, 9] = 0.0
    cache.v[page, row, 1, 5], cache.v[page, row, 0, 9], cache.v[page, row, 1, 63] = 0.0, 0.0, 0.0
    want, _ = a.attend(q, cache, on_device(step), causal=causal)
    want[sees, second, 5] = want[sees, second, 63] = want[sees, first, 9] = 0.0
    assert torch.equal(out, want)
    cache.k[page, row, 1, 7] = math.nan
    out, out_lse = a.attend(q, cache, on_device(step), causal=causal, want_lse=True)
    assert torch.isnan(out[sees][:, second]).all() and torch.isnan(out_lse[sees][:, second]).all()
    others = torch.ones(a.heads, dtype=torch.bool, device=DEV)
    others[second] = False
    assert torch.equal(out_lse[:, others], lse[:, others]) and torch.equal(out_lse[~sees], lse[~sees])
    a.close()


@pytest.mark.parametrize("kernel", KERNELS)
def test_scale_zero_of_queries_that_are_not_finite(kernel):
    """0 times a sum that is not finite is NaN, and so is its row; the others are means."""
    say("scale 0", kernel)
    q, cache, step, a, causal = inputs(kernel, 64, 16, gen(8))
    q = q.to(DEV)
    clean, lse = a.attend(q, cache, on_device(step), scale=0.0, causal=causal, want_lse=True)
    q[1, 0, 7], q[2, 3, 8], q[2, 1, 63] = math.nan, math.inf, -math.inf
    out, out_lse = a.attend(q, cache, on_device(step), scale=0.0, causal=causal, want_lse=True)
    for t, h in ((1, 0), (2, 3), (2, 1)):
        assert torch.isnan(out[t, h]).all() and torch.isnan(out_lse[t, h])
        out[t, h], out_lse[t, h] = clean[t, h], lse[t, h]
    assert torch.equal(out, clean) and torch.equal(out_lse, lse)
    a.close()


@pytest.mark.parametrize("seqs,kv_heads,tokens", [(1000, 1, 32766), (128, 65535, 4200)])
def test_more_items_than_a_launch_has_threads_for(seqs, kv_heads, tokens):
    """2^23 tiles of 256 rows and more, of 512 threads each.  Keys of zeros and equal
    values, so that every row of a sequence is its value exactly."""
    heads, dim, page_size = 65535, 8, 16
    say("large", seqs, heads, kv_heads, tokens)
    a = tr.Attention(heads, kv_heads, dim, BF)
    assert (tokens * heads // kv_heads + seqs * 256) * kv_heads * 2 >= 2 ** 32
    value = (torch.arange(seqs, device=DEV) % 200 + 1).to(BF)
    shape = (seqs, page_size, kv_heads, dim)
    cache = tr.KVCache(torch.zeros(shape, dtype=BF, device=DEV), value[:, None, None, None].expand(shape).contiguous())
    q_start = (torch.arange(seqs + 1, device=DEV) * tokens // seqs).to(torch.int32)
    step = tr.Step(q_start, torch.full((seqs,), 11, dtype=torch.int32, device=DEV), torch.arange(seqs, dtype=torch.int32, device=DEV)[:, None])
    q = torch.ones(1, 1, dim, dtype=BF, device=DEV).expand(tokens, heads, dim)
    out = torch.zeros(tokens, heads, dim, dtype=BF, device=DEV)
    a.attend(q, cache, step, causal=False, out=out)
    want = torch.repeat_interleave(value, (q_start[1:] - q_start[:-1]).long())
    for t in range(0, tokens, 4096):
        assert (out[t:t + 4096] == want[t:t + 4096, None, None]).all()
    a.close()


def test_one_row_of_the_table_for_all_sequences():
    """Sequences that read the same pages: an expanded row, which is only read."""
    g = gen(9)
    for heads, kv_heads, new in ((4, 2, [1, 1, 1]), (8, 1, [20, 3, 9])):
        table = torch.tensor([[2, 0, 3]], dtype=torch.int32)
        whole = tr.Step(torch.tensor([0] + [sum(new[:b + 1]) for b in range(3)], dtype=torch.int32),
                        torch.tensor([40, 33, 45], dtype=torch.int32), table.expand(3, 3).contiguous())
        cache, q = normal_caches(4, 16, kv_heads, 64, g), torch.randn(sum(new), heads, 64, generator=g).to(BF).to(DEV)
        a = tr.Attention(heads, kv_heads, 64, BF)
        want, _ = a.attend(q, cache, on_device(whole))
        shared = on_device(whole)._replace(table=table.to(DEV).expand(3, 3))
        assert shared.table.stride(0) == 0 and torch.equal(a.attend(q, cache, shared)[0], want)
        a.close()


def singles(seqs, new, g, heads=4, kv_heads=2, dim=64, page_size=16, kv=16):
    """`seqs` sequences of `new` tokens at the end of a page of their own."""
    cache = tr.KVCache(*(torch.randn(seqs, page_size, kv_heads, dim, generator=g, device=DEV, dtype=BF) for _ in range(2)))
    step = tr.Step(torch.arange(seqs + 1, dtype=torch.int32, device=DEV) * new, torch.full((seqs,), kv, dtype=torch.int32, device=DEV),
                   torch.randperm(seqs, device=DEV, generator=g).to(torch.int32)[:, None])
    return torch.randn(seqs * new, heads, dim, generator=g, device=DEV, dtype=BF), cache, step


def least_time(call):
    least = math.inf
    for _ in range(5):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        call()
        end.record()
        torch.cuda.synchronize()
        least = min(least, begin.elapsed_time(end))
    return least


@pytest.mark.parametrize("new", [1, 16])
def test_thousands_of_sequences(new):
    """Every workgroup walks over the sequences once: the time of a call grows with
    their number, not with its square (four times as many: 4, not 16 times)."""
    g = torch.Generator(device=DEV).manual_seed(new)
    heads, kv_heads, dim = (4, 2, 64) if new == 1 else (16, 2, 64)
    times = []
    for seqs in (5003, 20012):
        say("sequences", seqs, new)
        q, cache, step = singles(seqs, new, g, heads, kv_heads, dim)
        a = tr.Attention(heads, kv_heads, dim, BF)
        out, _ = a.attend(q, cache, step)
        k, v = (c[step.table[:, 0].long()].double().repeat_interleave(heads // kv_heads, 2) for c in cache)      # [seqs, 16, heads, dim]
        for i in range(new):
            s = (q[i::new].double()[:, None] * k).sum(-1) / math.sqrt(dim)
            s[:, 16 - new + i + 1:] = -math.inf
            w = torch.softmax(s, 1)[..., None]
            want, mass = (w * v).sum(1), (w * v.abs()).sum(1)
            assert float(((out[i::new].double() - want).abs() - 2.0 ** -8 * want.abs() - (2.0 ** -8 + 1.5e-3) * mass).max()) <= 0.0
        times.append(least_time(lambda: a.attend(q, cache, step, out=out)))
        a.close()
    assert times[1] < 9 * times[0], times


def test_a_long_sequence_without_new_tokens():
    """A slot that waits, however long its context, takes nothing from the others: the
    same rows, and their work still goes to all workgroups."""
    say("waiting")
    g = gen(10)
    kv, waiting, page_size = 20000, 1 << 20, 64
    cache, q = normal_caches(320, page_size, 8, 128, g), torch.randn(1, 8, 128, generator=g).to(BF).to(DEV)
    table = torch.zeros(2, waiting // page_size, dtype=torch.int32)
    table[0, :320] = torch.randperm(320, generator=g)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    alone = tr.Step(i32([0, 1]), i32([kv]), table[:1].to(DEV))
    both = tr.Step(i32([0, 1, 1]), i32([kv, waiting]), table.to(DEV))
    a = tr.Attention(8, 8, 128, BF)
    want, _ = a.attend(q, cache, alone)
    got, _ = a.attend(q, cache, both)
    # other parts, other roundings: each is within its bound of the definition
    ref_out, _, mass, _ = definition(q, cache, tr.Step(*(t.cpu() for t in alone)), 128 ** -0.5, True)
    for out in (want, got):
        assert float(((out.double() - ref_out).abs() - 2.0 ** -8 * ref_out.abs() - (2.0 ** -8 + 1.5e-3) * mass).max()) <= 0.0
    assert least_time(lambda: a.attend(q, cache, both)) < 3 * least_time(lambda: a.attend(q, cache, alone))
    a.close()
