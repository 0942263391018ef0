"""The loss of a distillation whose logits lie beyond 2^31 elements, from either path."""
import pytest
import torch

import paper_2507_19766_amd as ulorl
from test_gpu_distill import BF, DEV, EPS, compare, reference

pytestmark = pytest.mark.gpu


def test_the_loss_of_rows_beyond_32_bits_of_offset():
    n, V, K = 14200, 151936, 8                                  # 2.16e9 logits
    z = torch.empty(n, V, dtype=BF, device=DEV)
    z.normal_(0, 3, generator=torch.Generator(device=DEV).manual_seed(1))
    ids = torch.randint(0, V // K, (n, K), device=DEV, dtype=torch.int32) * K + torch.arange(K, device=DEV, dtype=torch.int32)
    logp = torch.full((n, K), -3.0, device=DEV)
    one, d = ulorl.distill_fwd_bwd(z, ids, logp)
    two = ulorl.distill_fwd(z, ids, logp)
    d2 = ulorl.distill_bwd(z, ids, two)
    picked = torch.cat([torch.arange(4), torch.arange(n - 80, n, 9), torch.tensor([14133, 14134, 14135])]).unique().to(DEV)    # 2^31 / V is 14134.2
    ref, tol = reference(z[picked], ids[picked], logp[picked], None, ulorl.DistillParams(denominator=n))
    for r, got in ((one, d), (two, d2)):
        part = r.kl[picked].double().sum() / n
        compare(dict(kl=r.kl[picked], lse=r.lse[picked], loss=part, dlogits=got[picked]), ref,
                dict(tol, loss=tol["loss"] + EPS * part.abs()), BF)
        # the loss is the 64-bit mean of the divergences, which are rounded to 32 bits apart from it
        kl = r.kl.double()
        assert (r.loss.double() - kl.sum() / n).abs() <= EPS * (kl.abs().sum() / n)
        assert r.counters.tolist() == [n, 0, 0, 0]
        assert (kl > 1).all()                                   # every row has been looked at: random tokens as a teacher
