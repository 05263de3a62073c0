"""Sizes and values at the ends of what the rotation takes."""
import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_rotate import BF, DEV, say

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
