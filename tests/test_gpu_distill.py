"""distill_fwd, distill_bwd, distill_fwd_bwd and autograd.distill_loss against their definition in 64 bits: every output of every
row, at the lengths, lists, masks and weights where they can go wrong."""
import math

import pytest
import torch

import paper_2507_19766_amd as ulorl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
EPS = 2.0 ** -23
HALF_STEP = {BF: 2.0 ** -8, F: 2.0 ** -24}
MASKED = -9e29
TAILS = [ulorl.TAIL_BUCKET, ulorl.TAIL_RENORM, ulorl.TAIL_DROP]


def reference(z, ids, logp, w, p, grad_out=1.0):
    """Outputs in 64 bits, and how far the calls' may be off.

    The calls sum e^x over the unlisted tokens in 32 bits: a term (x <= 0 relative to the largest) is off by the rounding of its
    argument and a unit of exp2, EPS (1 + |x|), and by up to nine roundings on its way through the sums.  ``off`` is what that
    makes of ln sum; everything after it is in 64 bits, except the coefficient of the unlisted tokens' gradient (eight roundings
    of its two terms) and a last exp2 per token.  A listed token's gradient is the difference of two numbers of up to 1.25 that take four
    roundings of 64 bits each, at most 1.4e-16: 1e-15 of g where they cancel."""
    n, V, T = z.shape[0], z.shape[1], float(torch.tensor(p.temperature, dtype=F))
    D = p.denominator if p.denominator > 0 else n
    z = z.double()
    z = torch.where(z <= MASKED, -math.inf, z)
    top = z.amax(1, keepdim=True)               # x relative to it: lse of hundreds (low temperatures) would cost digits
    x = (z - top) / T
    here = ids >= 0
    w = torch.ones(n, dtype=torch.float64, device=z.device) if w is None else w.double()
    t = torch.where(here, logp.double(), -math.inf)
    some = here.any(1)
    if p.tail == ulorl.TAIL_RENORM:
        some = some & (t > -math.inf).any(1)
        t = torch.log_softmax(t, 1)
    rows, cols = (here & some[:, None]).nonzero(as_tuple=True)
    at = ids[rows, cols].long()
    q = torch.zeros_like(x)
    q[rows, at] = t[rows, cols].exp()
    listed = torch.zeros_like(x, dtype=torch.bool)
    listed[rows, at] = True
    lse = torch.logsumexp(x, 1)
    lp = x - lse[:, None]
    prob = lp.exp()
    rest = torch.where(listed, -math.inf, x)
    m_rest = rest.amax(1, keepdim=True)
    soft_rest = torch.softmax(rest, 1).nan_to_num(nan=0.0)
    lse_rest = torch.logsumexp(rest, 1)
    p_rest = (lse_rest - lse).exp()
    q_sum = q.sum(1)
    q_rest = torch.zeros_like(q_sum)
    if p.tail == ulorl.TAIL_BUCKET:
        q_rest = torch.where(m_rest[:, 0] > -math.inf, (1 - q_sum).clamp(min=0), 0.0)
    mass = q_sum + q_rest
    kl = torch.where(q > 0, q * (q.log() - lp), 0.0).sum(1)
    kl = kl + torch.where(q_rest > 0, q_rest * (q_rest.log() - (lse_rest - lse)), 0.0)
    on = some & (w != 0)
    g = torch.where(on, w, 0.0) / (D * T) * grad_out
    rest_part = (mass * p_rest - q_rest)[:, None] * soft_rest
    d = g[:, None] * torch.where(listed, prob * mass[:, None] - q, rest_part)
    ref = dict(kl=torch.where(on, kl, 0.0), lse=torch.where(on, lse + top[:, 0] / T, 0.0), loss=(w * torch.where(on, kl, 0.0)).sum() / D, dlogits=d)

    X = torch.where(soft_rest > 0, m_rest - rest, 0.0)
    eta = EPS * (10 + X)
    off = (soft_rest * eta).sum(1)
    tol_kl = (mass * p_rest - q_rest).abs() * off + EPS * ref["kl"].abs() + 1e-13
    size = (torch.where(q > 0, q * (q.log().abs() + lp.abs()), 0.0)).sum(1) * 1e-14
    tol = dict(kl=tol_kl + size, lse=p_rest * off + EPS * ref["lse"].abs())
    tol["loss"] = (w.abs() * torch.where(on, tol["kl"], 0.0)).sum() / D + EPS * ref["loss"].abs()
    unlisted = rest_part.abs() * (2 * eta + off[:, None] + 4 * EPS) + soft_rest * ((mass * p_rest + q_rest) * 8 * EPS + mass * p_rest * off)[:, None]
    on_list = prob * (mass * p_rest * off)[:, None] + EPS * (prob * mass[:, None] - q).abs()
    tol["dlogits"] = g.abs()[:, None] * torch.where(listed, on_list + 1e-15, unlisted)
    ref["on"] = on
    return ref, tol


def compare(got, ref, tol, dtype=F):
    for name in ("kl", "lse", "loss"):
        a, b = got[name].double().reshape(ref[name].shape), ref[name]
        off = (a - b).abs() / (tol[name] + 1e-300)
        assert off.max() <= 1, (name, float(off.max()), int(off.argmax()))
    if "dlogits" in got:
        t = tol["dlogits"] + HALF_STEP[dtype] * (ref["dlogits"].abs() + tol["dlogits"]) + 1.2e-38      # below it the storage has fewer digits
        off = (got["dlogits"].double() - ref["dlogits"]).abs() / t
        assert off.max() <= 1, ("dlogits", float(off.max()), divmod(int(off.argmax()), off.shape[1]))


def buffer(n, V, dtype, pad=None):
    vec = 8 if dtype == BF else 4
    return torch.zeros(n, V + (-V % vec if pad is None else pad), dtype=dtype, device=DEV)[:, :V]


def problem(n, V, K, dtype=BF, seed=0, T=1.0, std=3.0, noise=0.7, ragged=False, tail=ulorl.TAIL_BUCKET):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = buffer(n, V, dtype)
    z.copy_(torch.randn(n, V, generator=g, device=DEV) * std)
    t = torch.log_softmax((z.float() + noise * torch.randn(n, V, generator=g, device=DEV)) / T, 1)
    k = min(K, V)
    best = t.topk(k, dim=1)
    ids = torch.full((n, K), -1, dtype=torch.int32, device=DEV)
    logp = torch.full((n, K), -math.inf, device=DEV)
    ids[:, :k], logp[:, :k] = best.indices, best.values
    order = torch.rand(n, K, generator=g, device=DEV).argsort(1)          # entries, missing ones among them, in any order
    ids, logp = ids.gather(1, order), logp.gather(1, order)
    if tail == ulorl.TAIL_RENORM:
        logp += 5.0
    if ragged:
        out = torch.rand(n, K, generator=g, device=DEV) < torch.rand(n, 1, generator=g, device=DEV) * 1.3
        ids = torch.where(out, torch.randint(-9, 0, (n, K), generator=g, device=DEV, dtype=torch.int32), ids)
        logp = torch.where(out, math.nan, logp)                           # of a missing entry nothing is looked at
    w = torch.rand(n, generator=g, device=DEV) * 2 - 0.5
    return z, ids.contiguous(), logp.contiguous(), w


def check(z, ids, logp, w, p, paths=("one", "two", "autograd"), launch=None):
    ref, tol = reference(z, ids, logp, w, p)
    found = {}
    for path in paths:
        before = z.clone()
        if path == "one":
            r, d = ulorl.distill_fwd_bwd(z, ids, logp, w, p, launch=launch)
        elif path == "two":
            r = ulorl.distill_fwd(z, ids, logp, w, p)
            d = ulorl.distill_bwd(z, ids, r, p)
        else:
            leaf = z.detach().requires_grad_(True)
            got = []
            loss = ulorl.autograd.distill_loss(leaf, ids, logp, w, p, results=got)
            r, d = got[0], torch.autograd.grad(loss, leaf)[0]
        assert torch.equal(before.view(torch.int16 if z.dtype == BF else torch.int32), z.view(torch.int16 if z.dtype == BF else torch.int32))
        compare(dict(kl=r.kl, lse=r.lse, loss=r.loss, dlogits=d), ref, tol, z.dtype)
        weightless = int((w == 0).sum()) if w is not None else 0
        assert r.counters.tolist() == [int(ref["on"].sum()), weightless, z.shape[0] - int(ref["on"].sum()) - weightless, 0]
        found[path] = (r, d)
    return found


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("tail", TAILS)
@pytest.mark.parametrize("T", [1.0, 0.5, 2.0])
def test_tails_and_temperatures(tail, T, dtype):
    p = ulorl.DistillParams(temperature=T, tail=tail)
    for n, V, K in [(9, 5000, 20), (5, 32003, 128)]:
        z, ids, logp, w = problem(n, V, K, dtype, n, T, tail=tail)
        check(z, ids, logp, w, p)
        check(z, ids, logp, None, p, ("one",))


@pytest.mark.parametrize("tail", TAILS)
@pytest.mark.parametrize("T", [0.001, 0.05, 0.2, 5.0, 30.0, 1000.0])
def test_peaked_and_flat_distributions(tail, T):
    """From one token that has everything to a divergence of 1e-11 beside logarithms of 12: what is in 64 bits is as good as 64 bits."""
    p = ulorl.DistillParams(temperature=T, tail=tail)
    for n, V, dtype in [(2, 151936, F), (2100, 1000, F), (2, 151936, BF), (300, 20000, BF)]:
        z, ids, logp, w = problem(n, V, 20, dtype, 3, T, tail=tail)
        check(z, ids, logp, w, p, ("one", "two"))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("mean,std", [(1e4, 3.0), (-1e4, 3.0), (1e6, 3.0), (-3e7, 100.0), (0.0, 1e5), (50.0, 0.0)])
def test_logits_of_any_size(mean, std, dtype):
    for n, V in [(3, 32003), (2100, 1000), (300, 20000)]:
        z, ids, logp, w = problem(n, V, 20, dtype, 3)
        z.copy_((z.float() / 3 * std + mean).to(dtype))
        check(z, ids, logp, w, ulorl.DistillParams(), ("one", "two"))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 255, 2047, 2048, 2049, 8192, 15359, 15360, 15361, 16385, 30719, 30720, 30721, 61439, 61441, 100003])
def test_lengths_of_rows(V, dtype):
    for n, K, tail in [(1, 1, ulorl.TAIL_BUCKET), (3, 64, ulorl.TAIL_BUCKET), (2, 128, ulorl.TAIL_DROP), (4, 5, ulorl.TAIL_RENORM)]:
        z, ids, logp, w = problem(n, V, K, dtype, V, tail=tail)
        if V > 300 and K > 8:       # the ends of the row and of what threads hold
            edge = torch.tensor([0, V - 1, V - 2, 7, 8, 2047, 2048, V // 2], device=DEV, dtype=torch.int32)
            edge = edge[edge < V].unique()
            free = (ids[:, :, None] == edge).any(2)
            ids[free] = -1
            for row in ids:
                row[:len(edge)] = edge
            logp[:, :len(edge)] = -7.0
            logp[ids < 0] = -math.inf
        check(z, ids, logp, w, ulorl.DistillParams(tail=tail), ("one", "two"))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("K", [1, 2, 63, 64, 65, 127, 128])
def test_lists(K, dtype):
    for tail in TAILS:
        z, ids, logp, w = problem(33, 20011, K, dtype, K, ragged=True, tail=tail)
        ids[3], logp[3] = -1, 0.0                               # nothing listed
        logp[5] = torch.where(ids[5] >= 0, -math.inf, logp[5])  # listed, of no probability
        w[7] = 0.0
        check(z, ids, logp, w, ulorl.DistillParams(tail=tail, denominator=17.5), ("one", "two"))


@pytest.mark.parametrize("n,V,K,dtype", [(1, 151936, 64, BF), (37, 151936, 128, BF), (11, 151936, 16, F), (130, 50257, 32, BF), (300, 4096, 8, F),
                                         (1, 1000003, 20, BF), (1, 500001, 20, F), (2, 2000003, 64, BF), (1, 1000001, 64, F)])
def test_large_vocabularies(n, V, K, dtype):
    z, ids, logp, w = problem(n, V, K, dtype, 3)
    check(z, ids, logp, w, ulorl.DistillParams())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [1, 7, 129, 1000, 1024, 1025, 2047, 2048, 2049, 4096, 4097])
def test_many_short_rows(V, dtype):
    for n, K, tail in [(2047, 9, ulorl.TAIL_BUCKET), (2048, 64, ulorl.TAIL_BUCKET), (2049, 65, ulorl.TAIL_DROP), (2500, 128, ulorl.TAIL_RENORM)]:
        z, ids, logp, w = problem(n, V, K, dtype, V + K, ragged=True, tail=tail)
        w[n // 2], w[n - 1] = 0.0, 0.0
        check(z, ids, logp, w, ulorl.DistillParams(tail=tail), ("one", "two"))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [600, 2000, 4096])
def test_many_short_rows_that_do_not_count(V, dtype):
    n, K = 2050, 100
    z, ids, logp, w = problem(n, V, K, dtype, 1)
    w = w.abs() + 0.1
    z[1, 17] = math.nan
    z[20, ids[20, 4].long()] = math.nan
    z[300, V - 1] = math.inf
    z[401, ids[401, 99].long()] = math.inf
    z[555] = -math.inf
    z[666, ids[666, 70].long()] = -math.inf                     # masked, and the teacher wants it
    ids[777, 2] = V
    ids[888, 3] = ids[888, 67]                                  # an id twice, and by the same thread of a wave
    ids[889, 99] = ids[889, 98]
    ids[2049, 64] = ids[2049, 0]
    logp[1000, 5] = math.nan
    w[1200] = math.nan
    w[2000] = 0.0
    z[2000], ids[2000], logp[2000] = math.nan, V + 5, math.nan  # padding: not looked at
    bad = [1, 20, 300, 401, 555, 666, 777, 888, 889, 2049, 1000, 1200, 2000]
    good = torch.ones(n, dtype=torch.bool, device=DEV)
    good[bad] = False
    ref, tol = reference(z[good], ids[good], logp[good], w[good], ulorl.DistillParams(denominator=n))
    def look(r, d):
        assert r.counters.tolist() == [n - len(bad), 1, 0, 1 | 2 | 16]
        assert (r.kl[bad] == 0).all() and (d[bad] == 0).all() and (r.top_grad[bad] == 0).all() and (r.rest_coef[bad] == 0).all()
        compare(dict(kl=r.kl[good], lse=r.lse[good], loss=r.loss, dlogits=d[good]), ref, tol, dtype)
    p = ulorl.DistillParams()
    look(*ulorl.distill_fwd_bwd(z, ids, logp, w, p))
    r = ulorl.distill_fwd(z, ids, logp, w, p)
    look(r, ulorl.distill_bwd(z, ids, r, p))
    look(*ulorl.distill_fwd_bwd(z, ids, logp, w, p, inplace=True))


@pytest.mark.parametrize("n", [2, 3, 4, 5, 63, 257, 4095, 4097, 20001])
def test_numbers_of_rows(n):
    z, ids, logp, w = problem(n, 1003, 9, BF, n)
    w[n // 2] = 0.0
    check(z, ids, logp, w, ulorl.DistillParams(), ("one", "two"))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("mask", [-math.inf, "lowest", -1e30])
def test_masked_logits(mask, dtype):
    value = torch.finfo(dtype).min if mask == "lowest" else mask
    V, K = 20003, 40
    z, ids, logp, w = problem(6, V, K, dtype, 5)
    w = w.abs() + 0.1
    unlisted = torch.ones(6, V, dtype=torch.bool, device=DEV).scatter_(1, ids.long(), False)
    z[0, (torch.rand(V, device=DEV) < 0.9) & unlisted[0]] = value
    z[1, unlisted[1]] = value                                   # nothing unlisted is left: no bucket
    z[2, V - 300:] = torch.where(unlisted[2, V - 300:], value, z[2, V - 300:])
    only = unlisted[3].float().argmax()
    z[3, unlisted[3]] = value
    z[3, only] = 1.0                                            # one token is left
    for j in (4, 5):                                            # masked tokens that the teacher lists with probability 0
        z[j, ids[j, 3].long()] = z[j, ids[j, 30].long()] = value
        logp[j, 3] = logp[j, 30] = -math.inf
    for tail in TAILS:
        check(z, ids, logp, w, ulorl.DistillParams(tail=tail), ("one", "two"))


def test_every_token_listed():
    for V, dtype in [(5, F), (64, BF), (128, F)]:
        z, ids, logp, w = problem(7, V, 128, dtype, V)
        for tail in TAILS:
            check(z, ids, logp, w, ulorl.DistillParams(tail=tail))


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_sure_student(dtype):
    """Nearly all of the student's mass is on the list: what is left to the others is summed, not subtracted."""
    z, ids, logp, w = problem(8, 151936, 16, dtype, 8)
    for r, up in enumerate([10., 15., 20., 25., 30., 40., 60., 90.]):
        z[r, ids[r, 3].long()] = up
    check(z, ids, logp, w.abs() + 0.5, ulorl.DistillParams())


def test_student_is_teacher():
    z, _, _, _ = problem(12, 50000, 1, F, 2)
    record = ulorl.token_topk(z, 64)
    r, d = ulorl.distill_fwd_bwd(z, record.top_ids, record.top_logp)
    assert r.kl.abs().max() < 1e-6 and d.abs().max() < 1e-7


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [3000, 151936])
def test_rows_that_do_not_count(V, dtype):
    n, K = 16, 24
    z, ids, logp, w = problem(n, V, K, dtype, 1)
    w = w.abs() + 0.1
    p = ulorl.DistillParams()
    good = [0, 8]
    ref, tol = reference(z[good], ids[good], logp[good], w[good], ulorl.DistillParams(denominator=n))
    z[1, 17] = math.nan
    z[2, ids[2, 4].long()] = math.nan
    z[3, V - 1] = math.inf
    z[4, ids[4, 23].long()] = math.inf
    z[5] = -math.inf
    z[6, ids[6, 0].long()] = -math.inf                          # masked, and the teacher wants it
    ids[7, 2] = V
    ids[9, 3] = ids[9, 20]                                      # an id twice
    logp[10, 5] = math.nan
    logp[11, 6] = math.inf
    w[12] = math.nan
    w[13] = math.inf
    logp[15] = logp[15] + 3.0                                   # probabilities of 20: logits, say
    w[14] = 0.0
    z[14], ids[14], logp[14] = math.nan, V + 5, math.nan        # padding: not looked at
    def look(r, d):
        assert r.counters.tolist() == [2, 1, 0, 1 | 2 | 16]
        bad = [i for i in range(n) if i not in good]
        assert (r.kl[bad] == 0).all() and (d[bad] == 0).all() and (r.top_grad[bad] == 0).all() and (r.rest_coef[bad] == 0).all()
        compare(dict(kl=r.kl[good], lse=r.lse[good], loss=r.loss, dlogits=d[good]), ref, tol, dtype)
    look(*ulorl.distill_fwd_bwd(z, ids, logp, w, p))
    r = ulorl.distill_fwd(z, ids, logp, w, p)
    look(r, ulorl.distill_bwd(z, ids, r, p))
    r, d = ulorl.distill_fwd_bwd(z, ids, logp, w, p, inplace=True)
    assert d.data_ptr() == z.data_ptr()
    look(r, d)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [60, 900])
def test_ids_listed_twice_in_any_piece(n, dtype):
    V, K = 50003, 70
    z, ids, logp, w = problem(n, V, K, dtype, 4)
    w = w.abs() + 0.1
    bad = list(range(0, n, 7))
    for i, r in enumerate(bad):
        ids[r, (5 * i) % 60] = ids[r, 60 + i % 10] = (i * 4001) % V         # in every piece of a row
    assert (ids[bad].long().sort(1).values.diff(dim=1) == 0).any(1).all()
    w[n - 1] = 0.0
    good = torch.ones(n, dtype=torch.bool, device=DEV)
    good[bad] = good[n - 1] = False
    ref, tol = reference(z[good], ids[good], logp[good], w[good], ulorl.DistillParams(denominator=n))
    def look(r, d):
        assert r.counters.tolist() == [int(good.sum()), 1 if n - 1 not in bad else 0, 0, 16]
        assert (r.kl[~good] == 0).all() and (d[~good] == 0).all() and (r.top_grad[~good] == 0).all()
        compare(dict(kl=r.kl[good], lse=r.lse[good], loss=r.loss, dlogits=d[good]), ref, tol, dtype)
    look(*ulorl.distill_fwd_bwd(z, ids, logp, w))
    r = ulorl.distill_fwd(z, ids, logp, w)
    look(r, ulorl.distill_bwd(z, ids, r))
    look(*ulorl.distill_fwd_bwd(z, ids, logp, w, launch=ulorl.Launch(per_row=True)))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("between", [math.nan, math.inf, 1e4])
def test_what_lies_between_rows_is_left_alone(between, dtype):
    vec = 8 if dtype == BF else 4
    for n, V in [(2100, 1001), (2100, 130), (700, 5003), (3, 32003), (70, 151931), (5, 3)]:
        base = torch.full((n + 1, V + (-V % vec) + vec), between, dtype=dtype, device=DEV)
        z = base[:n, :V]
        given, ids, logp, w = problem(n, V, 20, dtype, 3)
        z.copy_(given)
        check(z, ids, logp, w, ulorl.DistillParams(), ("one", "two"))
        before = base.clone()
        ulorl.distill_fwd_bwd(z, ids, logp, w, inplace=True)
        outside = torch.ones_like(base, dtype=torch.bool)
        outside[:n, :V] = False
        assert torch.equal(before[outside].view(torch.int16 if dtype == BF else torch.int32),
                           base[outside].view(torch.int16 if dtype == BF else torch.int32))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,V", [(5, 4096), (70, 151936), (300, 32003)])
def test_in_place_and_strided(n, V, dtype):
    """Over the logits the same bits; what lies between the rows is left alone; the same call twice gives the same bits."""
    z, ids, logp, w = problem(n, V, 30, dtype, 7)
    w[1] = 0.0
    p = ulorl.DistillParams(temperature=0.8)
    r, d = ulorl.distill_fwd_bwd(z, ids, logp, w, p, grad_out=0.5)
    again, d2 = ulorl.distill_fwd_bwd(z, ids, logp, w, p, grad_out=0.5)
    for name in ("loss", "kl", "lse", "rest_max", "rest_coef", "top_grad", "counters"):
        assert torch.equal(getattr(r, name), getattr(again, name)), name
    assert torch.equal(d, d2)
    vec = 8 if dtype == BF else 4
    wide = torch.full((n, V + 3 * vec + (-V % vec)), 77.0, dtype=dtype, device=DEV)
    view = wide[:, :V]
    view.copy_(z)
    r3, d3 = ulorl.distill_fwd_bwd(view, ids, logp, w, p, grad_out=0.5, inplace=True)
    assert d3.data_ptr() == wide.data_ptr() and torch.equal(view, d) and (wide[:, V:] == 77.0).all() and torch.equal(r3.kl, r.kl)
    view.copy_(z)
    r4 = ulorl.distill_fwd(view, ids, logp, w, p)
    d4 = ulorl.distill_bwd(view, ids, r4, p, grad_out=0.5, inplace=True)
    assert (wide[:, V:] == 77.0).all()
    ref, tol = reference(z, ids, logp, w, p, 0.5)
    for got in (d, d4):
        compare(dict(kl=r4.kl, lse=r4.lse, loss=r4.loss, dlogits=got), ref, tol, dtype)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,V", [(3, 40000), (40, 151936), (700, 32003)])
def test_pieces_whose_wait_expires(n, V, dtype):
    """A wait of one poll: what a workgroup leaves undone is written by the kernel that finishes the rows, in place too."""
    z, ids, logp, w = problem(n, V, 40, dtype, 7, ragged=True)
    w[0] = 0.0
    p = ulorl.DistillParams()
    short = ulorl.Launch(sync_spins=1)
    check(z, ids, logp, w, p, ("one",), launch=short)
    r, d = ulorl.distill_fwd_bwd(z, ids, logp, w, p)
    r2, d2 = ulorl.distill_fwd_bwd(z, ids, logp, w, p, inplace=True, launch=short)
    assert torch.equal(r.kl, r2.kl) and torch.equal(r.top_grad, r2.top_grad)
    assert (d.float() - d2.float()).abs().max() <= 4 * HALF_STEP[dtype] * d.float().abs().max()


@pytest.mark.parametrize("dtype", [BF, F])
def test_two_passes_on_request(dtype):
    z, ids, logp, w = problem(30, 70001, 40, dtype, 7)
    check(z, ids, logp, w, ulorl.DistillParams(), ("one",), launch=ulorl.Launch(per_row=True))
    r = ulorl.distill_fwd(z, ids, logp, w)
    r2, d2 = ulorl.distill_fwd_bwd(z, ids, logp, w, launch=ulorl.Launch(per_row=True))
    assert torch.equal(d2, ulorl.distill_bwd(z, ids, r)) and torch.equal(r.loss, r2.loss)


def test_the_gradient_against_differences():
    """Along random directions u, |u| <= 1: (kl(z + h u) - kl(z - h u)) / 2h is off by h^2 / 6 times a third cumulant of u (at
    most 8, in each of two terms of mass at most 1) and by the rounding of the two divergences over 2h."""
    h = 0.02
    for tail in TAILS:
        z, ids, logp, _ = problem(40, 777, 12, F, 4, tail=tail)
        p = ulorl.DistillParams(tail=tail, denominator=1.0)
        r, d = ulorl.distill_fwd_bwd(z, ids, logp, None, p)
        u = torch.rand(z.shape, device=DEV) * 2 - 1
        shifted = []
        for s in (h, -h):
            zs = buffer(*z.shape, F)
            zs.copy_(z + s * u)
            shifted.append(ulorl.distill_fwd(zs, ids, logp, None, p).kl.double())
        slope = (shifted[0] - shifted[1]) / (2 * h)
        along = (d.double() * u).sum(1)
        assert ((slope - along).abs() <= h * h / 6 * 16 + 4 * EPS * (1 + r.kl) * 20 / (2 * h)).all()


def test_autograd_scales_and_repeats():
    z, ids, logp, w = problem(20, 3000, 10, F, 6)
    p = ulorl.DistillParams(temperature=1.5)
    _, d = ulorl.distill_fwd_bwd(z, ids, logp, w, p)
    leaf = z.clone().requires_grad_(True)
    loss = ulorl.autograd.distill_loss(leaf, ids, logp, w, p)
    a = torch.autograd.grad(loss * 4.0, leaf, retain_graph=True)[0]
    b = torch.autograd.grad(loss, leaf)[0]
    assert torch.equal(a, 4.0 * b)
    ref, tol = reference(z, ids, logp, w, p)
    compare(dict(kl=ref["kl"], lse=ref["lse"], loss=loss.detach(), dlogits=b), ref, tol)
    fused = ulorl.autograd.distill_loss(leaf, ids, logp, w, p, fused=True)
    fused.backward()
    assert torch.equal(leaf.grad, d)
    with pytest.raises(RuntimeError, match="upstream"):
        (2 * ulorl.autograd.distill_loss(leaf, ids, logp, w, p, fused=True)).backward()
    with pytest.raises(ValueError, match="in_place"):
        ulorl.autograd.distill_loss(leaf, ids, logp, w, p, in_place=True)
    assert not ulorl.autograd.distill_loss(z, ids, logp, w, p).requires_grad


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("up", [math.nan, math.inf, -math.inf])
def test_an_upstream_gradient_that_is_not_finite(up, dtype):
    """Not hidden: rows that count are not finite (a bucket's tokens have a gradient each), the others' gradient stays 0."""
    for n, V in [(40, 3000), (30, 40003), (2100, 600)]:
        z, ids, logp, w = problem(n, V, 10, dtype, 6)
        w = w.abs() + 0.1
        w[3], w[n - 1] = 0.0, 0.0
        z[7, 5] = math.nan
        z[8, 11] = -math.inf
        ids[9, 2] = V
        off = torch.zeros(n, dtype=torch.bool, device=DEV)
        off[[3, n - 1, 7, 9]] = True
        r = ulorl.distill_fwd(z, ids, logp, w)
        scale = torch.tensor(up, device=DEV)
        leaf = z.detach().requires_grad_(True)
        (ulorl.autograd.distill_loss(leaf, ids, logp, w) * up).backward()
        for d in (ulorl.distill_bwd(z, ids, r, grad_scale=scale), ulorl.distill_bwd(z, ids, r, grad_out=up),
                  ulorl.distill_fwd_bwd(z, ids, logp, w, grad_out=up)[1],
                  ulorl.distill_fwd_bwd(z, ids, logp, w, grad_out=up, launch=ulorl.Launch(sync_spins=1))[1], leaf.grad):
            assert (d[off] == 0).all()
            assert (~d[~off].isfinite()).any(1).all()


def test_a_fused_gradient_is_given_once():
    z, ids, logp, w = problem(20, 3000, 10, F, 6)
    loss = ulorl.autograd.distill_loss(z.clone().requires_grad_(True), ids, logp, w, fused=True)
    loss.backward(retain_graph=True)
    with pytest.raises(RuntimeError, match="earlier backward"):
        loss.backward()


def test_beside_the_token_loss():
    """The two objectives on the same logits: the gradient of their sum is the sum of their gradients."""
    z, ids, logp, w = problem(64, 5000, 10, F, 9)
    y = torch.randint(0, 5000, (64,), device=DEV, dtype=torch.int32)
    cu = torch.tensor([0, 40, 64], device=DEV, dtype=torch.int32)
    adv = torch.randn(64, device=DEV)
    old = ulorl.row_stats(z, y).logp + 0.05
    leaf = z.clone().requires_grad_(True)
    a = ulorl.autograd.token_loss(leaf, y, cu, adv, old)
    b = ulorl.autograd.distill_loss(leaf, ids, logp, w)
    both = torch.autograd.grad(a + 0.3 * b, leaf, retain_graph=True)[0]
    one, two = torch.autograd.grad(a, leaf)[0], torch.autograd.grad(b, leaf)[0]
    assert (both - (one + 0.3 * two)).abs().max() <= 4 * EPS * (one.abs() + two.abs()).max()


def test_record_then_distil():
    """As they are used together: a teacher's logits recorded, a student's distilled from the record, alone and in a graph that is
    replayed on new logits with other work in between."""
    n, V, K = 48, 50257, 32
    teacher, student = buffer(n, V, BF), buffer(n, V, BF)
    w = torch.ones(n, device=DEV)
    w[5] = 0.0
    p = ulorl.DistillParams()

    def fill(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        student.copy_(torch.randn(n, V, generator=g, device=DEV) * 3)
        teacher.copy_(student.float() + 0.5 * torch.randn(n, V, generator=g, device=DEV))

    def step(record, out, d, ws_a, ws_b):
        ulorl.token_topk(teacher, K, out=record, workspace=ws_a)
        ulorl.distill_fwd_bwd(student, record.top_ids, record.top_logp, w, p, out=out, dlogits=d, workspace=ws_b)

    fill(0)
    record = ulorl.token_topk(teacher, K)
    out, d = ulorl.distill_fwd_bwd(student, record.top_ids, record.top_logp, w, p)
    ref, tol = reference(student, record.top_ids, record.top_logp, w, p)
    compare(dict(kl=out.kl, lse=out.lse, loss=out.loss, dlogits=d), ref, tol, BF)
    ws_a = torch.empty(ulorl.token_topk_workspace_bytes(n, V), dtype=torch.uint8, device=DEV)
    ws_b = torch.empty(ulorl.distill_workspace_bytes(n, V), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(record, out, d, ws_a, ws_b)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(record, out, d, ws_a, ws_b)
    for seed in range(1, 5):
        fill(seed)
        ws_a.fill_(255)
        ws_b.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = ulorl.token_topk(teacher, K)
        want, dw = ulorl.distill_fwd_bwd(student, eager.top_ids, eager.top_logp, w, p)
        assert torch.equal(record.top_ids, eager.top_ids) and torch.equal(record.top_logp, eager.top_logp)
        for name in ("loss", "kl", "lse", "rest_max", "rest_coef", "top_grad", "counters"):
            assert torch.equal(getattr(out, name), getattr(want, name)), name
        assert torch.equal(d, dw)


def test_autograd_in_a_graph():
    """Forward and backward captured together; the upstream gradient stays on the device and may change between replays."""
    z, ids, logp, w = problem(24, 32003, 16, BF, 2)
    p = ulorl.DistillParams(temperature=1.3)
    leaf = z.detach().requires_grad_(True)
    scale = torch.ones((), device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(ulorl.autograd.distill_loss(leaf, ids, logp, w, p) * scale, leaf)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = ulorl.autograd.distill_loss(leaf, ids, logp, w, p)
        grad = torch.autograd.grad(loss * scale, leaf)[0]
    for seed in range(3):
        new, new_ids, new_logp, _ = problem(24, 32003, 16, BF, 30 + seed)
        with torch.no_grad():
            leaf.copy_(new)
        ids.copy_(new_ids)
        logp.copy_(new_logp)
        scale.fill_(0.5 + seed)
        graph.replay()
        torch.cuda.synchronize()
        r = ulorl.distill_fwd(new, ids, logp, w, p)
        want = ulorl.distill_bwd(new, ids, r, p, grad_scale=scale)
        assert torch.equal(loss.reshape(1), r.loss) and torch.equal(grad, want)


def test_two_graphs_and_two_streams():
    """Graphs that share a workspace, replayed in turn; calls on two streams at once, each with its own."""
    problems = [problem(40, 70001, 16, BF, 1), problem(20, 4099, 60, BF, 2)]
    shared = torch.empty(max(ulorl.distill_workspace_bytes(z.shape[0], z.shape[1]) for z, _, _, _ in problems), dtype=torch.uint8, device=DEV)
    want = [ulorl.distill_fwd_bwd(z, ids, logp, w) for z, ids, logp, w in problems]
    made = []
    for z, ids, logp, w in problems:
        out, d = ulorl.distill_fwd_bwd(z, ids, logp, w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ulorl.distill_fwd_bwd(z, ids, logp, w, out=out, dlogits=d, workspace=shared)
        made.append((graph, out, d))
    for turn in range(6):
        graph, out, d = made[turn % 2]
        for t in (out.kl, out.top_grad, d):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        r, dw = want[turn % 2]
        assert torch.equal(out.kl, r.kl) and torch.equal(out.top_grad, r.top_grad) and torch.equal(d, dw) and torch.equal(out.loss, r.loss)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for turn in range(4):
        with torch.cuda.stream(streams[turn % 2]):
            z, ids, logp, w = problems[turn % 2]
            got.append(ulorl.distill_fwd_bwd(z, ids, logp, w))
    torch.cuda.synchronize()
    for turn, (r, d) in enumerate(got):
        assert torch.equal(r.kl, want[turn % 2][0].kl) and torch.equal(d, want[turn % 2][1])


def test_on_a_stream_of_its_own():
    z, ids, logp, w = problem(40, 151936, 20, BF, 3)
    want, dw = ulorl.distill_fwd_bwd(z, ids, logp, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r, d = ulorl.distill_fwd_bwd(z, ids, logp, w)
        leaf = z.detach().requires_grad_(True)
        g = torch.autograd.grad(ulorl.autograd.distill_loss(leaf, ids, logp, w), leaf)[0]
    side.synchronize()
    assert torch.equal(d, dw) and torch.equal(r.loss, want.loss)
    ref, tol = reference(z, ids, logp, w, ulorl.DistillParams())
    compare(dict(kl=want.kl, lse=want.lse, loss=want.loss, dlogits=g), ref, tol, BF)


def test_rows_beyond_32_bits_of_offset():
    n, V, K = 14200, 151936, 8                                  # 2.16e9 logits
    z = torch.empty(n, V, dtype=BF, device=DEV)
    z.normal_(0, 3, generator=torch.Generator(device=DEV).manual_seed(1))
    last = slice(n - 8, n)
    ids = torch.randint(0, V // K, (n, K), device=DEV, dtype=torch.int32) * K + torch.arange(K, device=DEV, dtype=torch.int32)
    logp = torch.full((n, K), -3.0, device=DEV)
    p = ulorl.DistillParams()
    top = ulorl.token_topk(z, 4)
    few = ulorl.token_topk(z[last], 4)
    assert torch.equal(top.top_ids[last], few.top_ids)
    ref, tol = reference(z[last], ids[last], logp[last], None, ulorl.DistillParams(denominator=n))
    r, d = ulorl.distill_fwd_bwd(z, ids, logp, None, p)
    for got in (d, ulorl.distill_bwd(z, ids, ulorl.distill_fwd(z, ids, logp, None, p), p)):
        compare(dict(kl=r.kl[last], lse=r.lse[last], loss=ref["loss"], dlogits=got[last]), ref, tol, BF)


def test_results_are_written_or_refused():
    z, ids, logp, w = problem(6, 1000, 5, F, 1)
    r = ulorl.distill_fwd(z, ids, logp, w)
    keep = {name: getattr(r, name).clone() for name in ("loss", "kl", "lse", "rest_max", "rest_coef", "top_grad", "counters")}
    for name in keep:
        getattr(r, name).zero_()
    same = ulorl.distill_fwd(z, ids, logp, w, out=r)
    for name, t in keep.items():
        assert getattr(same, name).data_ptr() == getattr(r, name).data_ptr() and torch.equal(getattr(r, name), t)
    for name in keep:
        bad = ulorl.DistillResult(**{k: getattr(r, k) for k in keep})
        setattr(bad, name, getattr(r, name)[:-1])
        with pytest.raises(ValueError):
            ulorl.distill_fwd(z, ids, logp, w, out=bad)
        setattr(bad, name, None)
        with pytest.raises(ValueError):
            ulorl.distill_fwd_bwd(z, ids, logp, w, out=bad)


def test_refusals():
    z, ids, logp, w = problem(6, 1000, 5, F, 1)
    r = ulorl.distill_fwd(z, ids, logp, w)
    for call in (lambda *a: ulorl.distill_fwd(*a), lambda *a: ulorl.distill_fwd_bwd(*a), lambda *a: ulorl.autograd.distill_loss(*a)):
        with pytest.raises(ValueError):
            call(z, ids.long(), logp, w)
        with pytest.raises(ValueError):
            call(z, ids[:, :4], logp, w)
        with pytest.raises(ValueError):
            call(z, ids[:5], logp[:5], w)
        with pytest.raises(ValueError):
            call(z, ids[0], logp[0], w)
        with pytest.raises(ValueError):
            call(z, ids, logp.double(), w)
        with pytest.raises(ValueError):
            call(z, ids, logp, w[:5])
        with pytest.raises(ValueError):
            call(z, ids.cpu(), logp, w)
        with pytest.raises(ValueError):
            call(z, torch.zeros(6, 129, dtype=torch.int32, device=DEV), torch.zeros(6, 129, device=DEV), w)
        with pytest.raises(TypeError):
            call(z.half(), ids, logp, w)
        for bad in (dict(temperature=0.0), dict(temperature=math.nan), dict(tail=3), dict(tail=-1), dict(denominator=math.nan)):
            with pytest.raises(ulorl.UlorlError) as e:
                call(z, ids, logp, w, ulorl.DistillParams(**bad))
            assert e.value.status == -5
        with pytest.raises(ulorl.UlorlError) as e:
            call(torch.zeros(6, 1001, device=DEV), ids, logp, w)
        assert e.value.status == -4
    with pytest.raises(ulorl.UlorlError) as e:
        ulorl.distill_fwd(z, ids, logp, w, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == -6
    with pytest.raises(ValueError):
        ulorl.distill_fwd_bwd(z, ids, logp, w, dlogits=torch.empty(6, 1008, device=DEV)[:, :1000])
    with pytest.raises(ValueError):
        ulorl.distill_bwd(z, ids[:, :4].contiguous(), r)
    with pytest.raises(ValueError):
        ulorl.distill_bwd(z, ids, r, grad_scale=torch.ones(2, device=DEV))
