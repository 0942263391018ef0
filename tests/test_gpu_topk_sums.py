"""token_topk's sums over rows whose terms are alike, so that the roundings of a long sum add up instead of averaging out."""
import pytest
import torch

import paper_2507_19766_amd as ulorl
from test_gpu_topk import BF, DEV, EPS, F

pytestmark = pytest.mark.gpu


def expected(z, T):
    """Entropy and log-sum-exp in 64 bits, and how far the call's may be off whatever the row's length.  With X = (largest - z) / T:
    a term e^-X is off by a unit of exp2 for itself, its lane and its wave, and by the roundings of its argument and of the differences of
    largest logits, EPS (4 + 2 X) in all, which moves the entropy by p (1 + |X - mean|) of it and ln sum by p.  A batch's terms take
    up to six half-steps on their way into the sum and twelve into the weighted one; the sums over batches carry what they round off.  So
    the mean of X is off by 9 EPS of itself and ln sum by 3 EPS, and each result is rounded once."""
    x = (z.double() - z.double().amax(1, keepdim=True)) / T
    p = torch.softmax(x, 1)
    ln_s, mean = torch.logsumexp(x, 1), (p * -x).sum(1)
    term = EPS * p * (4 - 2 * x)
    lse = z.double().amax(1) / T + ln_s
    return dict(entropy=(ln_s + mean, (term * (1 + (-x - mean[:, None]).abs())).sum(1) + EPS * (3 + 9 * mean + ln_s + mean)),
                lse=(lse, term.sum(1) + EPS * (3 + lse.abs())))


def rows_of_few_values(n, V, dtype):
    vec = 8 if dtype == BF else 4
    z = torch.zeros(n, V + -V % vec, dtype=dtype, device=DEV)[:, :V]
    third = V // 3
    for r in range(n):
        low = -(1.0, 5.0, 9.6875, 0.3125, 2.5)[r % 5]
        z[r] = low
        if r % 4 == 0:
            z[r, V // 2] = 0.0                                  # the largest amid the row
        elif r % 4 == 1:
            z[r, third:2 * third], z[r, 2 * third:] = low + 0.25, low + 0.5      # rising
            z[r, V - 1] = 0.0
        elif r % 4 == 2:
            z[r, ::257] = 0.0                                   # a sum's largest early in each lane
        else:
            z[r, ::3], z[r, 0] = 2 * low, 0.0
    return z


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,V", [(20, 151936), (201, 151936), (20, 32003), (1100, 5000), (4, 1 << 24), (300, 400003)])
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_sums_of_terms_that_are_alike(n, V, dtype, T):
    distinct = min(n, 20)
    z = rows_of_few_values(distinct, V, dtype)
    whole = z if n == distinct else torch.zeros(n, z.stride(0), dtype=dtype, device=DEV)[:, :V]
    for a in range(0, n, distinct) if whole is not z else ():
        whole[a:a + distinct] = z[:min(distinct, n - a)]
    r = ulorl.token_topk(whole, 3, temperature=T)
    for name, (want, tol) in expected(z, float(torch.tensor(T, dtype=F))).items():
        got = getattr(r, name)
        off = (got[:distinct].double() - want).abs() / tol
        assert off.max() <= 1, (name, int(off.argmax()), float(off.max()))
        for a in range(0, n, distinct):                         # the same row, the same bits
            assert torch.equal(got[a:a + distinct], got[:min(distinct, n - a)])
