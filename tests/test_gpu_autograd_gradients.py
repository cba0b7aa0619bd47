"""Gradients that the attention's backward has no rule for: one with a forward-mode tangent, a batched one."""
import pytest
import torch
import torch.autograd.forward_ad as fwAD

from paper_2603_02170_amd.autograd import sage_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("share", [False, True])
def test_a_tangent_of_the_gradient_is_refused(share):
    x = [torch.randn(1, 2, 70, 64, device="cuda").to(torch.bfloat16).requires_grad_() for _ in range(3)]
    O = sage_attention(*x, share_quantized=share)
    dO = torch.randn_like(O)
    with fwAD.dual_level():
        with pytest.raises(NotImplementedError, match="forward-mode"):
            torch.autograd.grad(O, x, fwAD.make_dual(dO, torch.ones_like(dO)), retain_graph=True)
    with pytest.raises(NotImplementedError, match="vmap"):
        torch.autograd.grad(O, x, torch.stack([dO, dO]), is_grads_batched=True, retain_graph=True)
    # the graph still serves a gradient without one
    want = torch.autograd.grad(sage_attention(*x), x, dO)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(O, x, dO), want))
