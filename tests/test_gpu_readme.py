"""README's calls of the language model's side, run as they are written there."""
import math
import os
from types import SimpleNamespace

import pytest
import torch

import attn_ref as ref
import paper_2607_13500_amd as tr
import test_gpu_verify as verify_
from conftest import ROOT
from test_gpu_attend8 import cache8, stands_for
from test_gpu_rotate import BF, DEV, gen, say, step_of, on_device

pytestmark = pytest.mark.gpu

I32 = torch.int32


def parts():
    """(calls over a bf16 cache, a server's step) of README's block."""
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    lines = text[text.index("    attn = tr.Attention("):].split("\n")
    block = []
    for line in lines:
        if line.strip() and not line.startswith("    "):
            break
        block.append(line[4:])
    first, _, second = "\n".join(block).partition("# a server's step")
    assert first.strip() and "verify_drafts" in second
    return first, "#" + second


def heads_of(g, rows):
    return torch.randn(rows, 48, 128, generator=g).to(BF).to(DEV).split([32, 8, 8], 1)


def weights(g):
    return [(1 + 0.2 * torch.randn(128, generator=g)).to(BF).to(DEV) for _ in range(2)]


def close(out, q, cache, step):
    """attend against the definition, as test_gpu_attend8 has it."""
    rows = int(step.q_start[-1])
    kv = stands_for(cache) if isinstance(cache, tr.KVCache8) else [t.cpu().double() for t in cache]
    want, _, mass, _ = ref.attend(q.cpu()[:rows], *kv, tr.Step(*(t.cpu() for t in step)), 128 ** -0.5, True, 0)
    assert ((out.cpu().double()[:rows] - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 1.5e-3) * mass).all()


def test_calls_over_a_bf16_cache():
    say("bf16 cache")
    g = gen(1)
    K, grid, start = [5, 3], [(1, 6, 6), (1, 4, 9)], [(0, 0, 0), (2, 2, 2)]
    step, pages = step_of(K, K, 16, g)
    q, k, v = heads_of(g, 8)
    wq, wk = weights(g)
    cache = tr.KVCache(*(torch.zeros(pages, 16, 8, 128, dtype=BF, device=DEV) for _ in range(2)))
    names = dict(torch=torch, tr=tr, res=SimpleNamespace(idx=torch.tensor([0, 7, 8, 20, 35, 3, 9, 35], dtype=I32, device=DEV)), K=K, grid=grid,
                 start=start, q=q, k=k, v=v, wq=wq, wk=wk, cache=cache, step=on_device(step))
    exec(parts()[0], names)
    assert names["pos"].tolist() == [[0] * 5 + [2] * 3, [0, 1, 1, 3, 5, 2, 3, 5], [0, 1, 2, 2, 5, 5, 2, 10]]
    close(names["out"], names["q"], cache, step)


def test_a_servers_step():
    """Three prompts, two with an image's kept tokens, whose text then goes on three axes
    ahead of (or behind) its places; steps of drafts."""
    g = gen(2)
    seqs, page_size, pages, vocab, width, most = 3, 16, 40, 300, 4, 4
    kept, side, before = [6, 0, 40], [24, 0, 24], [4, 7, 9]
    lengths = [b + k + 1 for b, k in zip(before, kept)]
    shift = [s - k for s, k in zip(side, kept)]
    a = tr.Attention(32, 8, 128, sections=(16, 24, 24), norm=True)
    wq, wk = weights(g)
    c = cache8(pages, page_size, 8, 128, g)
    names = dict(torch=torch, tr=tr, attn=a, wq=wq, wk=wk, k8=c.k, v8=c.v, k_scale=c.k_scale, v_scale=c.v_scale, page_size=page_size, width=width,
                 kv_len=torch.zeros(seqs, dtype=I32, device=DEV), table=torch.full((seqs, 8), -1, dtype=I32, device=DEV),
                 pool=tr.PagePool(torch.randperm(pages, generator=g).to(I32).to(DEV), torch.tensor([0, pages], dtype=I32, device=DEV)),
                 ahead=torch.tensor(shift, dtype=I32, device=DEV))
    # the prompts: words, kept tokens, a word
    u = tr.update_pages(torch.tensor(lengths, dtype=I32, device=DEV), names["kv_len"], names["table"], names["pool"], page_size, sum(lengths), in_place=True)
    pos = torch.zeros(3, sum(lengths), dtype=I32)
    at = 0
    for b, k, s in zip(before, kept, side):
        pos[:, at:at + b] = torch.arange(b, dtype=I32)
        pos[:, at + b:at + b + k] = b + torch.randint(0, max(s, 1), (3, k), generator=g, dtype=I32)
        pos[:, at + b + k] = b + s
        at += b + k + 1
    q, k, v = heads_of(g, sum(lengths))
    a.append(q, k, v, pos.to(DEV), c, u.step, wq=wq, wk=wk)
    second = parts()[1]
    for n in range(5):
        say("step", n)
        counts = [int(x) for x in torch.randint(1, most + 1, (seqs,), generator=g)]
        rows = sum(counts) + 2
        q, k, v = heads_of(g, rows)
        target, ids, accept, draw, draft = verify_.inputs(g, counts, vocab, torch.float32, True)
        names.update(change=torch.tensor(counts, dtype=I32, device=DEV), rows=rows, q=q, k=k, v=v, target=target.to(DEV), ids=ids.to(DEV),
                     accept=accept.to(DEV), draw=draw.to(DEV), draft=draft.to(DEV))
        exec(second, names)
        want = [length + s + i for length, s, m in zip(lengths, shift, counts) for i in range(m)]
        assert names["pos"].shape == (3, rows) and names["pos"][:, :rows - 2].tolist() == [want] * 3
        # the step as it was before its rejected drafts left
        step = names["u"].step._replace(kv_len=torch.tensor([x + y for x, y in zip(lengths, counts)], dtype=I32))
        close(names["out"], names["q"], c, step)
        rk = a.rotate(None, k[:rows - 2], torch.tensor([want] * 3, dtype=I32, device=DEV), wk=wk)[1].float()
        slots = names["u"].slots[:rows - 2]
        newest = stands_for(c)[0].flatten(0, 1).to(DEV)[slots].float()
        scale = c.k_scale.repeat_interleave(page_size // c.k_scale.shape[1], 1).flatten(0, 1)[slots]
        assert ((newest - rk).abs() <= (2.0 ** -4 + 2.0 ** -8) * rk.abs() + 2.0 ** -10 * scale[..., None] + 1e-5).all()
        accepted = names["d"].accepted.tolist()
        assert names["d"].change.tolist() == [x - (m - 1) for x, m in zip(accepted, counts)]
        lengths = [length + 1 + x for length, x in zip(lengths, accepted)]
        assert names["kv_len"].tolist() == lengths and names["u"].short.tolist() == [0]
        held = [p for r, x in zip(names["table"].tolist(), lengths) for p in r[:math.ceil(x / page_size)]]
        first, free = names["pool"].state.tolist()
        assert sorted(held + [names["pool"].ring.tolist()[(first + i) % pages] for i in range(free)]) == list(range(pages))
