"""Appends of thousands of sequences, whose segments are found by a search of several
rounds: the bits that calls on a few sequences each leave."""
import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_attend8 import cache8
from test_gpu_rotate import BF, DEV, F32, gen, on_device, say, step_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,dtype", [(64, BF), (10, F32)])
@pytest.mark.parametrize("seqs,most,page_size,block", [(4097, 3, 16, 16), (9000, 1, 4, 2), (5000, 40, 48, 16)])
def test_many_sequences(seqs, most, page_size, block, dim, dtype):
    say("append8 many", seqs, most, dim)
    g = gen(seqs + dim)
    new = torch.randint(0, most + 1, (seqs,), generator=g)
    new[:70] = 0                                          # none at all in the first ones, and many after another
    new[3000:3300] = 0
    new = new.tolist()
    kv = [n + int(x) for n, x in zip(new, torch.randint(0, 2 * page_size, (seqs,), generator=g))]
    step, pages = step_of(new, kv, page_size, g)
    a = tr.Attention(4, 2, dim, dtype, norm=True)
    x = torch.randn(sum(new), 8, dim, generator=g).to(dtype).to(DEV)
    q, k, v = x.split([4, 2, 2], 1)
    pos = torch.randint(0, 5000, (sum(new),), generator=g, dtype=torch.int32).to(DEV)
    whole, parts = (cache8(pages, page_size, 2, dim, gen(1), block) for _ in range(2))
    got = a.append(q, k, v, pos, whole, on_device(step))
    for b in range(0, seqs, 50):
        t0, t1 = int(step.q_start[b]), int(step.q_start[min(b + 50, seqs)])
        if t0 < t1:
            some = tr.Step(step.q_start[b:b + 51] - t0, step.kv_len[b:b + 50], step.table[b:b + 50])
            assert torch.equal(got[t0:t1], a.append(q[t0:t1], k[t0:t1], v[t0:t1], pos[t0:t1], parts, on_device(some)))
    for one, other in zip(whole, parts):
        assert torch.equal(one.view(torch.uint8), other.view(torch.uint8))
    a.close()
