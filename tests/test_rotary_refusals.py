"""What sage_rotary has no derivative or rule for is refused, whichever argument brings it, on the host and before any other check."""
import os

import pytest
import torch
import torch.autograd.forward_ad as fwAD

from paper_2603_02170_amd import build
from paper_2603_02170_amd.autograd import sage_rotary


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(build.HOST):
        build.build(verbose=False)


def _inputs():
    return torch.randn(4, 2, 64).to(torch.bfloat16), torch.randn(4, 1, 64).to(torch.bfloat16), torch.arange(4), torch.rand(32)


@pytest.mark.parametrize("which", [0, 1, 3])
def test_a_tangent_of_any_argument_is_refused(which):
    """A tangent that is dropped reads as a zero derivative."""
    with fwAD.dual_level():
        args = list(_inputs())
        args[which] = fwAD.make_dual(args[which], torch.ones_like(args[which]))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            sage_rotary(*args)
        args[which] = fwAD.unpack_dual(args[which]).primal
        with pytest.raises(ValueError, match="Q: need cuda"):          # (goes on to the next check)
            sage_rotary(*args)


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_a_batch_of_any_argument_is_refused(which):
    args = list(_inputs())
    args[which] = torch.stack([args[which]] * 2)

    def one(x):
        return sage_rotary(*args[:which], x, *args[which + 1:])[0]
    with pytest.raises(NotImplementedError, match="vmap"):
        torch.func.vmap(one)(args[which])


def test_a_functional_derivative_of_the_frequencies_is_refused():
    Q, K, pos, f = _inputs()
    with pytest.raises(NotImplementedError):
        torch.func.jvp(lambda x: sage_rotary(Q, K, pos, x)[0].float(), (f,), (torch.ones_like(f),))
    with pytest.raises(NotImplementedError):
        torch.func.grad(lambda x: sage_rotary(Q, K, pos, x)[0].float().sum())(f)


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1])
def test_a_tangent_of_a_gradient_is_refused(which):
    Q, K, pos, f = (t.cuda() for t in _inputs())
    Q.requires_grad_(), K.requires_grad_()
    out = sage_rotary(Q, K, pos, f)
    plain = [torch.ones_like(t) for t in out]
    want = torch.autograd.grad(out, [Q, K], plain, retain_graph=True)
    with fwAD.dual_level():
        grads = list(plain)
        grads[which] = fwAD.make_dual(plain[which], torch.ones_like(plain[which]))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            torch.autograd.grad(out, [Q, K], grads, retain_graph=True)
    # the graph still serves a gradient without one
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, [Q, K], plain, retain_graph=True), want))
    with pytest.raises(NotImplementedError, match="vmap"):
        torch.autograd.grad(out, [Q, K], [g.expand(2, *g.shape).contiguous() for g in plain], is_grads_batched=True)
