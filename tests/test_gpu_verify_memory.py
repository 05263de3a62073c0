"""What verification's results keep of the device's memory: themselves."""
import pytest
import torch

import paper_2607_13500_amd as tr
import test_gpu_verify as verify_
from test_gpu_rotate import DEV, gen, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [300, 50001])
def test_results_do_not_keep_the_scratch(vocab):
    counts, width = [4] * 64, 5
    say("memory", vocab)
    target, ids, accept, draw, draft = (t.to(DEV) for t in verify_.inputs(gen(vocab), counts, vocab, torch.float32, True))
    q_start = torch.arange(0, 4 * 64 + 1, 4, dtype=torch.int32, device=DEV)
    kept = tr.verify_drafts(target, ids, q_start, accept, draw, width, draft=draft)
    results = sum(t.numel() * t.element_size() for t in kept)
    assert sum({t.untyped_storage().data_ptr(): t.untyped_storage().nbytes() for t in kept}.values()) <= results
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    more = [tr.verify_drafts(target, ids, q_start, accept, draw, width, draft=draft) for _ in range(20)]
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before <= 20 * (results + 511) and all(torch.equal(a, b) for v in more for a, b in zip(v, kept))
