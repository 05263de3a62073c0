"""examples/answer.py: the operators together, as a model calls them."""
import importlib.util
import os

import pytest
import torch

import paper_2607_13500_amd as tr
from conftest import ROOT

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("answer_example", os.path.join(ROOT, "examples", "answer.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def test_runs():
    print("answer", flush=True)
    said, losses = example.main(["--images", "3", "--tokens", "5"])
    assert said.shape == (5, 3) and (said >= 0).all() and (said < 1000).all()
    assert losses[2] < losses[1] < losses[0]
    again, _ = example.main(["--images", "3", "--tokens", "5"])
    assert torch.equal(said, again)


def test_prompt_positions():
    K, before = [3, 2], 4
    idx = torch.tensor([0, 25, 575, 1, 30], dtype=torch.int32, device="cuda")
    kept = torch.arange(5.0, device="cuda")[:, None].expand(5, 8).contiguous()
    words = -1.0 - torch.arange(9.0, device="cuda")[:, None].expand(9, 8)
    x, pos, lengths = example.prompts(kept, idx, K, (1, 24, 24), before, words)
    assert lengths == [8, 7]
    assert x[:, 0].tolist() == [-1, -2, -3, -4, 0, 1, 2, -5, -1, -2, -3, -4, 3, 4, -5]
    assert pos.tolist() == [[0, 1, 2, 3, 4, 4, 4, 28, 0, 1, 2, 3, 4, 4, 28],
                            [0, 1, 2, 3, 4, 5, 27, 28, 0, 1, 2, 3, 4, 5, 28],
                            [0, 1, 2, 3, 4, 5, 27, 28, 0, 1, 2, 3, 5, 10, 28]]


def test_a_prompt_at_once_and_token_by_token():
    """The same rows attended in one call (tiles of many rows) and one by one.  Each
    is within 2^-8 |want| + (2^-8 + 1.5e-3) sum w |v| of the definition, and both
    sums of weights times |v| are at most the largest |v|."""
    print("prompt and tokens", flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    a = tr.Attention(8, 2, 128, torch.bfloat16, sections=(16, 24, 24), norm=True)
    n = 150
    pages = (n + example.PAGE - 1) // example.PAGE
    whole, single = (example.Layer(a, 256, pages, torch.Generator(device="cuda").manual_seed(2)) for _ in range(2))
    x = torch.randn(n, 256, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 500, (3, n), generator=g, device="cuda", dtype=torch.int32)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    q, k, v = whole.split(x)
    step = lambda new, kv: tr.Step(torch.tensor([0, new], dtype=torch.int32, device="cuda"), torch.tensor([kv], dtype=torch.int32, device="cuda"), table)
    together = whole.attend(q, k, v, pos, step(n, n))
    one = torch.cat([single.attend(q[i:i + 1], k[i:i + 1], v[i:i + 1], pos[:, i:i + 1].contiguous(), step(1, i + 1)) for i in range(n)])
    assert torch.equal(whole.cache.k, single.cache.k) and torch.equal(whole.cache.v, single.cache.v)
    bound = 2 * (2 * 2.0 ** -8 + 1.5e-3) * float(v.float().abs().max())
    assert float((together.float() - one.float()).abs().max()) <= bound
