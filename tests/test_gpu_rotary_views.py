"""Rotary positions of dense views that begin anywhere in a larger buffer: as Q, as K, and as a gradient."""
import pytest
import torch

from paper_2603_02170_amd.autograd import sage_rotary

pytestmark = pytest.mark.gpu


def _at(offset, shape, g):
    """A dense tensor that begins `offset` elements into its storage."""
    n = torch.Size(shape).numel()
    t = torch.randn(n + offset, generator=g).to(torch.bfloat16).cuda()[offset:].view(shape)
    assert t.is_contiguous() and t.storage_offset() == offset
    return t


@pytest.mark.parametrize("offset", [1, 3, 4, 7, 8, 12])
@pytest.mark.parametrize("shape,token_major", [((9, 2, 64), True), ((2, 5, 3, 128), True), ((2, 3, 5, 128), False), ((1, 1, 64), True)])
def test_dense_views_off_16_bytes(offset, shape, token_major):
    g = torch.Generator().manual_seed(offset)
    N = shape[0] if len(shape) == 3 else shape[1 if token_major else 2]
    pos, f = torch.arange(N, device="cuda"), torch.rand(shape[-1] // 2, generator=g).cuda()
    Q, K = _at(offset, shape, g), _at(offset + 1, shape, g)
    turn = lambda q, k: sage_rotary(q, k, pos, f, token_major=token_major)  # noqa: E731
    want = turn(Q.clone(), K.clone())
    for got in (turn(Q, K), turn(Q, K.clone()), turn(Q.clone(), K)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(turn(Q, None)[0], want[0])


def test_a_gradient_that_is_a_view_off_16_bytes():
    """torch.cat of a tensor of odd size and the turned ones hands each a slice of one gradient."""
    g = torch.Generator().manual_seed(2)
    Q, K = (torch.randn((6, h, 64), generator=g).to(torch.bfloat16).cuda().requires_grad_() for h in (3, 1))
    pos, f, odd = torch.arange(6, device="cuda"), torch.rand(32, generator=g).cuda(), torch.zeros(5, dtype=torch.bfloat16, device="cuda")
    q, k = sage_rotary(Q, K, pos, f)
    w = torch.randn(5 + q.numel() + 1 + k.numel(), generator=g).to(torch.bfloat16).cuda()
    torch.cat([odd, q.flatten(), odd[:1], k.flatten()]).backward(w)
    dQ, dK = w[5:5 + q.numel()].view_as(q), w[6 + q.numel():].view_as(k)
    want = sage_rotary(dQ.clone(), dK.clone(), pos, f, inverse=True)
    assert torch.equal(Q.grad, want[0]) and torch.equal(K.grad, want[1])
    (only,) = torch.autograd.grad(torch.cat([odd, sage_rotary(Q, K, pos, f)[1].flatten()]), [K], w[:5 + k.numel()])
    assert torch.equal(only, sage_rotary(w[5:5 + k.numel()].view_as(k).clone(), None, pos, f, inverse=True)[0])
