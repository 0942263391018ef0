"""What token_topk returns when it writes to an earlier result."""
import pytest
import torch

import paper_2507_19766_amd as ulorl
from test_gpu_topk import F, rows, tokens

pytestmark = pytest.mark.gpu


def test_without_a_token_there_is_no_log_prob_of_one():
    a, b, y = rows(9, 5000, F, 1), rows(9, 5000, F, 2), tokens(9, 5000)
    first = ulorl.token_topk(a, 4, y)
    logp = first.logp.clone()
    second = ulorl.token_topk(b, 4, out=first)
    assert second.logp is None and torch.equal(first.logp, logp)            # a's, not passed on as b's
    assert second.lse.data_ptr() == first.lse.data_ptr() and torch.equal(second.top_ids, ulorl.token_topk(b, 4).top_ids)
    third = ulorl.token_topk(b, 4, y, out=first)
    assert third.logp.data_ptr() == first.logp.data_ptr() and torch.equal(third.logp, ulorl.token_topk(b, 4, y).logp)
