"""autograd.distill_loss: what makes the loss require a gradient, the same in both forms."""
import pytest
import torch

import paper_2507_19766_amd as ulorl
from test_gpu_distill import F, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("which", ["teacher_logp", "weights", "both"])
def test_a_target_that_requires_a_gradient_makes_a_node_and_gets_none(which, fused):
    z, ids, logp, w = problem(20, 3000, 10, F, 6)
    if which != "weights":
        logp = logp.requires_grad_(True)
    if which != "teacher_logp":
        w = w.requires_grad_(True)
    loss = ulorl.autograd.distill_loss(z, ids, logp, w, fused=fused)
    assert loss.requires_grad
    loss.backward()
    assert logp.grad is None and w.grad is None and z.grad is None
    leaf = z.clone().requires_grad_(True)
    ulorl.autograd.distill_loss(leaf, ids, logp, w, fused=fused).backward()
    plain = z.clone().requires_grad_(True)
    ulorl.autograd.distill_loss(plain, ids, logp.detach(), w.detach(), fused=fused).backward()
    assert torch.equal(leaf.grad, plain.grad) and logp.grad is None and w.grad is None
    with torch.no_grad():
        assert not ulorl.autograd.distill_loss(leaf, ids, logp, w, fused=fused).requires_grad
    assert not ulorl.autograd.distill_loss(z, ids, logp.detach(), w.detach(), fused=fused).requires_grad
    assert not ulorl.autograd.distill_loss(z, ids, logp.detach(), None, fused=fused).requires_grad
