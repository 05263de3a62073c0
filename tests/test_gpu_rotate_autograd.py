"""Attention.rotate where autograd records: the gradients of rotate_backward, which
test_gpu_rotate compares with their definition."""
import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_rotate import BF, DEV, F32, gen, inputs, positions, weights

pytestmark = pytest.mark.gpu


def case(dtype, norm, how="packed"):
    g = gen(17)
    a = tr.Attention(6, 2, 64, dtype, sections=(16, 16), norm=norm)
    q, k = inputs(64, dtype, 33, 6, 2, how, g)
    gq, gk = inputs(64, dtype, 33, 6, 2, "own", g)
    wq, wk = weights(64, dtype, g, norm)
    return a, q, k, gq, gk, wq, wk, positions(2, 33, g).to(DEV)


def asking(*tensors):
    return [None if t is None else t.detach().requires_grad_(True) for t in tensors]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("norm", [True, False])
def test_gradients_reach_every_input(dtype, norm):
    a, q, k, gq, gk, wq, wk, pos = case(dtype, norm)
    plain = a.rotate(q, k, pos, wq=wq, wk=wk)
    dq, dk, dwq, dwk = a.rotate_backward(gq, gk, q, k, pos, wq=wq, wk=wk)
    q, k, wq, wk = asking(q, k, wq, wk)
    qo, ko = a.rotate(q, k, pos, wq=wq, wk=wk)
    assert torch.equal(qo, plain[0]) and torch.equal(ko, plain[1])
    torch.autograd.backward([qo, ko], [gq, gk])
    assert torch.equal(q.grad, dq) and torch.equal(k.grad, dk)
    if norm:
        assert torch.equal(wq.grad, dwq.to(dtype)) and torch.equal(wk.grad, dwk.to(dtype))


def test_gradients_of_some():
    """Inputs and outputs without a gradient are left out."""
    a, q, k, gq, gk, wq, wk, pos = case(BF, True)
    dq, dk, dwq, dwk = a.rotate_backward(gq, gk, q, k, pos, wq=wq, wk=wk)
    w, = asking(wk)
    qo, ko = a.rotate(q, k, pos, wq=wq, wk=w)
    torch.autograd.backward([qo, ko], [gq, gk])
    assert torch.equal(w.grad, dwk.to(BF)) and q.grad is None
    x, y = asking(q, k)
    qo, ko = a.rotate(x, y, pos, wq=wq, wk=wk)
    qo.backward(gq)                       # the keys are not used
    assert torch.equal(x.grad, dq) and y.grad is None
    x, = asking(q)
    qo, none = a.rotate(x, None, pos, wq=wq)
    qo.backward(gq)
    assert none is None and torch.equal(x.grad, dq)


def test_gradient_of_a_sum():
    """An expanded gradient of ones, through slices of one projection."""
    a, q, k, *_, wq, wk, pos = case(F32, True, "own")
    both = torch.cat([q, k], 1).requires_grad_(True)
    qo, ko = a.rotate(both[:, :6], both[:, 6:], pos, wq=wq, wk=wk)
    (qo.sum() + ko.sum()).backward()
    dq, dk, _, _ = a.rotate_backward(torch.ones_like(q), torch.ones_like(k), q, k, pos, wq=wq, wk=wk)
    assert torch.equal(both.grad, torch.cat([dq, dk], 1))


def test_streams_recording_and_outputs():
    a, q, k, gq, gk, wq, wk, pos = case(BF, True)
    dq, dk, _, _ = a.rotate_backward(gq, gk, q, k, pos, wq=wq, wk=wk)
    x, y = asking(q, k)
    with torch.no_grad():
        qo, ko = a.rotate(x, y, pos, wq=wq, wk=wk, q_out=q.clone(), k_out=k.clone())
    assert not qo.requires_grad and not ko.requires_grad
    with pytest.raises(RuntimeError):
        a.rotate(x, y, pos, wq=wq, wk=wk, q_out=q.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    qo, ko = a.rotate(x, y, pos, wq=wq, wk=wk, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.autograd.backward([qo, ko], [gq, gk])
    torch.cuda.synchronize()
    assert torch.equal(x.grad, dq) and torch.equal(y.grad, dk)
