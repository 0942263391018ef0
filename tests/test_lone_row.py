"""A lone row has no stride: token_topk and the distillation calls take it whatever its tensor says of one."""
import pytest
import torch

import paper_2507_19766_amd as ulorl
from test_distill_host import forward, p_, params, topk

DEV = "cuda:0"
STRIDES = [0, 1, 999, 1001, 2 ** 40 + 3, -8]


@pytest.mark.parametrize("stride", STRIDES)
def test_the_stride_of_a_lone_row_is_not_looked_at(stride):
    """The temperature is checked after the stride, and refused: nothing is launched."""
    assert topk(N=1, stride=stride, T=0.0) == -5
    for both in (False, True):
        assert forward(N=1, stride=stride, p=params(T=0.0), both=both) == -5
    assert ulorl.load_library().ulorl_distill_bwd(p_(0x1000), 1, 1, 1000, stride, p_(0x2000), 8, 0.0, p_(0x7000), p_(0x8000), p_(0x9000), 1.0, None,
                                                  p_(0xa000), None) == -5
    assert topk(N=1, V=0, stride=stride) == -2 and topk(N=1, V=1 << 31, stride=stride) == -2 and topk(N=1, V=2 ** 63 - 1, stride=stride) == -2
    assert topk(N=2, stride=min(stride, 999)) == -2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 1001, 151936])
def test_a_column_taken_as_a_row(V, dtype):
    column = torch.randn(V, 1, device=DEV).to(dtype)
    z, same = column.t(), column.reshape(1, V)
    assert z.stride() == (1, 1) or V == 1
    k = min(V, 20)
    a, b = ulorl.token_topk(z, k), ulorl.token_topk(same, k)
    assert torch.equal(a.top_ids, b.top_ids) and torch.equal(a.top_logp, b.top_logp) and torch.equal(a.entropy, b.entropy)
    r, d = ulorl.distill_fwd_bwd(z, b.top_ids, b.top_logp)
    want, dw = ulorl.distill_fwd_bwd(same, b.top_ids, b.top_logp)
    assert torch.equal(r.loss, want.loss) and torch.equal(d, dw) and d.stride() == z.stride()
    assert torch.equal(ulorl.distill_bwd(z, b.top_ids, ulorl.distill_fwd(z, b.top_ids, b.top_logp)),
                       ulorl.distill_bwd(same, b.top_ids, ulorl.distill_fwd(same, b.top_ids, b.top_logp)))
    leaf = z.detach().requires_grad_(True)
    ulorl.autograd.distill_loss(leaf, b.top_ids, b.top_logp).backward()
    assert (leaf.grad.float() - dw.float()).abs().max() <= 2.0 ** -7 * dw.float().abs().max() + 1e-9
