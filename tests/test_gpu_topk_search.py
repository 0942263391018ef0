"""token_topk on rows that overflow its lists, whose K-th largest is found by the exact search: in workgroups of four waves and, where
few long rows are split, of eight; at lengths of an odd and of an even number of bits."""
import math

import pytest
import torch

from test_gpu_topk import BF, DEV, F, check, rows, tokens

pytestmark = pytest.mark.gpu


def overflowing(n, V, dtype, seed):
    z = rows(n, V, dtype, seed)
    col = torch.arange(V, device=DEV)
    z[0] = 1.5                                                  # one value only
    z[1] = (z[1] * 0.4).round()                                 # a handful of values
    z[2] = (col % 5).to(dtype)                                  # each one spread over the row
    z[3] = -(col // max(1, V // 3)).to(dtype)                   # and side by side
    z[4, V // 2:] = -math.inf
    z[4, :V // 2] = -4.0
    return z


# elements / groups of 1000 bf16 (125 groups) to 4099 fp32 (1025): bits of the one, the other or both odd
@pytest.mark.parametrize("V,dtype", [(1000, BF), (1000, F), (2000, BF), (4096, BF), (4099, F), (5000, BF), (16384, F), (20000, F), (32003, BF), (50257, BF)])
@pytest.mark.parametrize("k", [1, 100, 128])
def test_four_waves(V, dtype, k):
    for n in (5, 7):
        z = overflowing(n, V, dtype, k)
        first = check(z, k, 1.0, tokens(n, V))
        again = check(z, k, 1.0, tokens(n, V))
        assert torch.equal(first.top_ids, again.top_ids) and torch.equal(first.top_logp, again.top_logp)


@pytest.mark.parametrize("V,dtype", [(70001, BF), (128256, BF), (151936, BF), (32003, F), (128256, F), (400000, BF)])
@pytest.mark.parametrize("k", [1, 100, 128])
def test_eight_waves(V, dtype, k):
    z = overflowing(6, V, dtype, k)
    first = check(z, k, 1.0, tokens(6, V))
    again = check(z, k, 1.0, tokens(6, V))
    assert torch.equal(first.top_ids, again.top_ids) and torch.equal(first.top_logp, again.top_logp)
