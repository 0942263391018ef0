"""Distillation next to the token loss, as cases to be timed and compared: what a teacher's logits are recorded as, and the
loss and gradient of a student against the record.

  topk      ``token_topk``: log-prob of each row's token, entropy, and the k likeliest tokens with their log-probs
  forward   ``distill_fwd``: the divergence of each row from its teacher's record, for a validation set
  one_call  ``distill_fwd_bwd``: loss and gradient of the student's logits in one pass (the trainer's step)
  two_call  ``autograd.distill_loss`` and ``backward()``: the same inside a torch training script
  chain     ``token_topk`` on a teacher's logits, then ``distill_fwd_bwd`` of a student's on what it recorded

Shapes: vocabularies from 1000 to 151 936 and odd ones, from one row (a decode step) to 16 384, 1 to 128 recorded tokens a row.

Values: Gaussian logits with a share of peaked rows; the last ``dead`` columns are padding of the vocabulary at -infinity;
``allowed`` keeps a few tokens a row and masks the others (a decode step under a grammar).  A teacher is the student with noise
added.  A record may be ragged (rows with fewer entries, some with none: id -1), and rows may have weight 0 (prompt tokens).

``run`` computes the plain form in 32 bits on tensors [rows, vocabulary]; with ``own`` set it makes this package's calls.
"""
import math

import torch

own = False

DEV = "cuda"
MASKED = -9e29          # a logit at or below it has probability 0 and is never an alternative
BUCKET, RENORM, DROP = "bucket", "renorm", "drop"


def listed():
    return [
        # one sequence being decoded: the next token's alternatives, as an answer's log-probs show them
        dict(name="topk_one_row", kind="topk", rows=1, V=151936, pad=0, dtype="bf16", k=20, T=1.0, dead=267, allowed=0),
        # a decode batch under a grammar that leaves fewer tokens than are asked for, at the sampling temperature
        dict(name="topk_grammar_64_rows", kind="topk", rows=64, V=151936, pad=0, dtype="bf16", k=8, T=0.7, dead=0, allowed=6),
        # fp32 logits of a small vocabulary
        dict(name="topk_small_f32", kind="topk", rows=512, V=4096, pad=0, dtype="f32", k=5, T=1.0, dead=0, allowed=0),
        # odd everything: a vocabulary that is no multiple of a vector, padded rows, an odd number of alternatives
        dict(name="topk_odd_vocab", kind="topk", rows=1777, V=32003, pad=5, dtype="bf16", k=33, T=1.3, dead=3, allowed=0),
        # one finished 16k segment as its teacher saw it, recorded for distillation
        dict(name="topk_16384_rows", kind="topk", rows=16384, V=151936, pad=0, dtype="bf16", k=64, T=1.0, dead=267, allowed=0),
        # a toy run or a unit test: launches are all it costs
        dict(name="one_call_tiny_f32", kind="one_call", rows=256, V=4096, pad=0, dtype="f32", k=8, T=1.0, tail=BUCKET,
             ragged=False, prompt=0.0, dead=0),
        # one short micro-batch of a large vocabulary
        dict(name="one_call_584_rows", kind="one_call", rows=584, V=151936, pad=0, dtype="bf16", k=64, T=1.0, tail=BUCKET,
             ragged=False, prompt=0.1, dead=267),
        # the ordinary step: a quarter of the rows are prompt
        dict(name="one_call_16384_rows", kind="one_call", rows=16384, V=151936, pad=0, dtype="bf16", k=64, T=1.0, tail=BUCKET,
             ragged=False, prompt=0.25, dead=267),
        # odd everything, ragged records of a softened teacher renormalised over what is listed
        dict(name="one_call_odd_vocab", kind="one_call", rows=3001, V=32003, pad=5, dtype="bf16", k=100, T=2.0, tail=RENORM,
             ragged=True, prompt=0.1, dead=3),
        # fp32 logits (a trainer that upcasts) through autograd, forward and backward apart
        dict(name="two_call_wide_f32", kind="two_call", rows=2048, V=151936, pad=0, dtype="f32", k=16, T=1.0, tail=DROP,
             ragged=False, prompt=0.0, dead=0),
        # validation: divergence only, the longest records
        dict(name="forward_4096_rows", kind="forward", rows=4096, V=151936, pad=0, dtype="bf16", k=128, T=1.0, tail=BUCKET,
             ragged=True, prompt=0.0, dead=267),
        # teacher and student in one step: what the first call records is what the second one reads
        dict(name="chain_4096_rows", kind="chain", rows=4096, V=128256, pad=0, dtype="bf16", k=32, T=1.0, tail=BUCKET,
             ragged=False, prompt=0.0, dead=0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["topk", "topk", "one_call", "one_call", "two_call", "forward", "chain"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    vec = 8 if dtype == "bf16" else 4
    V = rng.choice([151936, _log_uniform(rng, 1000, 151936), _log_uniform(rng, 1000, 151936)])
    rows = _log_uniform(rng, 1, max(2, min(8192, 1_200_000_000 // (V * (16 // vec)))))
    case = dict(kind=kind, rows=rows, V=V, pad=-V % vec, dtype=dtype, k=_log_uniform(rng, 1, 128), T=rng.choice([1.0, 1.0, 0.6, 2.0]),
                dead=rng.choice([0, V // 500]))
    if kind == "topk":
        return dict(case, allowed=rng.choice([0, 0, _log_uniform(rng, 1, 200)]))
    return dict(case, tail=rng.choice([BUCKET, BUCKET, RENORM, DROP]), ragged=kind != "chain" and rng.choice([False, True]),
                prompt=rng.choice([0.0, 0.3]))


# ------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, V, k = case["rows"], case["V"], case["k"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def rand(*size):
        return torch.rand(size, generator=g, device=DEV)

    def ints(hi, *size):
        return torch.randint(0, hi, size, generator=g, device=DEV)

    def buffer():
        return torch.zeros(n, V + case["pad"], dtype=dt, device=DEV)[:, :V]

    logits, teacher = buffer(), buffer() if case["kind"] == "chain" else None
    token_ids = torch.empty(n, dtype=torch.int32, device=DEV)
    ids = torch.empty(n, k, dtype=torch.int32, device=DEV)
    logp = torch.empty(n, k, device=DEV)
    std, boost = (2.0, 12.0) if V < 16384 else (3.0, 15.0)
    live = V - case["dead"]
    step = max(1, 400_000_000 // V)
    for a in range(0, n, step):
        b = min(n, a + step)
        z = torch.randn(b - a, V, generator=g, device=DEV).mul_(std)
        z[torch.arange(b - a, device=DEV), ints(live, b - a)] += boost * (rand(b - a) < 0.4)
        z[:, live:] = -math.inf
        if case.get("allowed"):
            few = torch.full_like(z, -math.inf)
            at = ints(live, b - a, case["allowed"])
            z = few.scatter_(1, at, z.gather(1, at))
        logits[a:b] = z
        if case["kind"] == "topk":
            z.sub_(rand(b - a, V).clamp_(1e-20, 1 - 1e-7).log_().neg_().log_())
            token_ids[a:b] = z.argmax(1)
            continue
        z.add_(torch.randn(z.shape, generator=g, device=DEV), alpha=0.7)
        if teacher is not None:
            teacher[a:b] = z
            continue
        z.div_(case["T"])
        best = z.topk(min(k, live), dim=1)
        ids[a:b], logp[a:b] = -1, -math.inf
        ids[a:b, :best.values.shape[1]] = best.indices
        logp[a:b, :best.values.shape[1]] = best.values if case["tail"] == RENORM else best.values - torch.logsumexp(z, 1, keepdim=True)
    del z
    s = dict(case=case, logits=logits)
    if case["kind"] == "topk":
        return dict(s, token_ids=token_ids)
    s["weights"] = (rand(n) >= case["prompt"]).float() * (0.5 + rand(n)) if case["prompt"] > 0 else None
    if teacher is not None:
        return dict(s, teacher=teacher)
    if case["ragged"]:
        short = torch.arange(k, device=DEV)[None, :] >= ints(k + 1, n, 1)
        ids[short], logp[short] = -1, -math.inf
    if case["kind"] == "two_call":
        s["logits"].requires_grad_(True)
    return dict(s, ids=ids, logp=logp)


# ------------------------------------------------------------------------------------------- the plain form

def _topk(z, k, T, y=None):
    """Log-softmax of z / T at y, entropy, and the k largest logits (ties: the lowest index) with their log-probs."""
    z = z.float()
    z = torch.where(z <= MASKED, -math.inf, z)
    m = z.amax(1, keepdim=True)
    x = (z - m) / T
    e = x.exp()
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    weighted = (e * x.clamp(min=-1e4)).sum(1, keepdim=True, dtype=torch.float64)
    out = dict(lse=(m.double() / T + total.log())[:, 0].float(), entropy=(total.log() - weighted / total)[:, 0].float())
    if y is not None:
        out["logp"] = (x.gather(1, y.long()[:, None]) - total.log())[:, 0].float()
    bits = (z + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7fffffff)).long()
    column = torch.arange(z.shape[1], device=z.device)
    best = ((order << 32) | (0x7fffffff - column)).topk(min(k, z.shape[1]), dim=1).values
    ids = 0x7fffffff - (best & 0x7fffffff)
    logp = (x.gather(1, ids) - total.log()).float()
    ids = torch.where(logp == -math.inf, -1, ids).int()
    more = k - ids.shape[1]
    out["top_ids"] = torch.nn.functional.pad(ids, (0, more), value=-1)
    out["top_logp"] = torch.nn.functional.pad(logp, (0, more), value=-math.inf)
    return out


def _distill(z, ids, logp, weights, case, gradient):
    """Loss, divergences and (wanted) the gradient to z, of the dtype of z.  A divergence is a small sum of larger terms, so
    what goes into it, the listed tokens and the sums over the vocabulary, is in 64 bits."""
    n, V, T = z.shape[0], z.shape[1], case["T"]
    z32 = z.detach().float()
    z32 = torch.where(z32 <= MASKED, -math.inf, z32)
    m = z32.amax(1, keepdim=True)
    here = ids >= 0
    q = torch.where(here, logp, -math.inf).double()
    if case["tail"] == RENORM:
        q = q - q.amax(1, keepdim=True).clamp(min=-1e30)
        q = q - q.exp().sum(1, keepdim=True).clamp(min=1e-30).log()
    lnq, q = q, q.exp()
    some = here.any(1)
    at = torch.where(here, ids, V).long()
    padded = torch.nn.functional.pad(z32, (0, 1))
    top = (padded.gather(1, at).double() - m) / T
    rest = padded.scatter_(1, at, -math.inf)[:, :V]
    m_rest = rest.amax(1, keepdim=True).clamp(min=-1e30)
    rest = (rest - m_rest) / T
    lse_rest = rest.exp().sum(1, keepdim=True, dtype=torch.float64).log()
    to_max = (m_rest.double() - m) / T
    total = torch.logaddexp(lse_rest + to_max, torch.where(here, top, -math.inf).exp().sum(1, keepdim=True).log())
    lse = (m.double() / T + total)[:, 0]
    top = torch.where(here, top - total, 0.0)
    ln_rest = (lse_rest + to_max - total)[:, 0]
    p_rest = ln_rest.exp()
    q_rest = (1 - q.sum(1)).clamp(min=0) if case["tail"] == BUCKET else torch.zeros_like(ln_rest)
    q_rest = torch.where(ln_rest > -math.inf, q_rest, 0.0)
    w = torch.ones(n, device=z.device) if weights is None else weights
    on = some & (w != 0)
    kl = torch.where(q > 0, q * (lnq - top), 0.0).sum(1) + torch.where(q_rest > 0, q_rest * (q_rest.log() - ln_rest), 0.0)
    kl = torch.where(on, kl, 0.0)
    out = dict(loss=((w * kl).sum() / n).float(), kl=kl.float(), lse=torch.where(on, lse, 0.0).float(),
               counters=torch.stack([on.sum(), (w == 0).sum(), (~some & (w != 0)).sum(), torch.zeros_like(on.sum())]))
    if gradient:
        scale = torch.where(on, w, 0.0) / (n * T)
        mass = q.sum(1) + q_rest
        d = (rest - lse_rest.clamp(min=-1e30).float()).exp()
        d *= (scale * (mass * p_rest - q_rest)).float()[:, None]
        listed_d = (scale[:, None] * (torch.where(here, top.exp(), 0.0) * mass[:, None] - q)).float()
        d = torch.nn.functional.pad(d, (0, 1)).scatter_(1, at, listed_d)[:, :V]
        out["dlogits"] = d.to(z.dtype)
    return out


# ------------------------------------------------------------------------------------------- the calls

def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind == "topk":
            return _topk(s["logits"], case["k"], case["T"], s["token_ids"])
        if kind == "chain":
            record = _topk(s["teacher"], case["k"], case["T"])
            out = _distill(s["logits"], record["top_ids"], record["top_logp"], s["weights"], case, True)
            return dict(out, top_ids=record["top_ids"], top_logp=record["top_logp"])
        return _distill(s["logits"], s["ids"], s["logp"], s["weights"], case, kind != "forward")

    import paper_2507_19766_amd as ulorl
    if kind == "topk":
        r = ulorl.token_topk(s["logits"], case["k"], s["token_ids"], temperature=case["T"])
        return dict(top_ids=r.top_ids, top_logp=r.top_logp, logp=r.logp, entropy=r.entropy, lse=r.lse)
    tail = {BUCKET: ulorl.TAIL_BUCKET, RENORM: ulorl.TAIL_RENORM, DROP: ulorl.TAIL_DROP}[case["tail"]]
    params = ulorl.DistillParams(temperature=case["T"], tail=tail)
    out = {}
    if kind == "chain":
        r = ulorl.token_topk(s["teacher"], case["k"], temperature=case["T"])
        ids, logp = out["top_ids"], out["top_logp"] = r.top_ids, r.top_logp
    else:
        ids, logp = s["ids"], s["logp"]
    if kind == "forward":
        r = ulorl.distill_fwd(s["logits"], ids, logp, s["weights"], params)
    elif kind == "two_call":
        got = []
        s["logits"].grad = None
        ulorl.autograd.distill_loss(s["logits"], ids, logp, s["weights"], params, results=got).backward()
        r, out["dlogits"] = got[0], s["logits"].grad
    else:
        r, out["dlogits"] = ulorl.distill_fwd_bwd(s["logits"], ids, logp, s["weights"], params)
    return dict(out, loss=r.loss.reshape(()), kl=r.kl, lse=r.lse, counters=r.counters)


# ------------------------------------------------------------------------------------------- work, 64-bit results

def work(case):
    n, V, k = case["rows"], case["V"], case["k"]
    b = 4.0 if case["dtype"] == "f32" else 2.0
    topk = {"bytes": n * (V * b + 8 * k + 16), "flops": 6.0 * n * V}
    if case["kind"] == "topk":
        return topk
    if case["kind"] == "forward":
        return {"bytes": n * (V * b + 8 * k + 12), "flops": 5.0 * n * V}
    step = {"bytes": n * (2 * V * b + 8 * k + 12), "flops": 8.0 * n * V}
    return {key: step[key] + topk[key] for key in step} if case["kind"] == "chain" else step


def exact(case, seed):
    """Row by row of the definition in 64 bits: a distribution over listed tokens and one bucket for the others."""
    s = prepare(case, seed)
    n, V, k, T = case["rows"], case["V"], case["k"], case["T"]
    f64 = dict(dtype=torch.float64, device=DEV)
    step = max(1, 150_000_000 // V)
    out = {}
    if case["kind"] in ("topk", "chain"):
        lse, ent, at_y = (torch.empty(n, **f64) for _ in range(3))
        top = torch.full((n, k), -math.inf, **f64)
        ids = torch.full((n, k), -1, dtype=torch.int64, device=DEV)
        source = s["teacher" if case["kind"] == "chain" else "logits"]
        for a in range(0, n, step):
            b = min(n, a + step)
            x = source[a:b].double() / T
            lse[a:b] = torch.logsumexp(x, 1)
            lp = x - lse[a:b, None]
            ent[a:b] = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(1)
            if case["kind"] == "topk":
                at_y[a:b] = lp.gather(1, s["token_ids"][a:b].long()[:, None])[:, 0]
                top[a:b, :min(k, V)] = lp.topk(min(k, V), dim=1).values
            else:                                          # whose tokens a tie goes to matters for what follows
                best = lp.sort(dim=1, descending=True, stable=True)
                top[a:b, :min(k, V)], ids[a:b, :min(k, V)] = best.values[:, :k], best.indices[:, :k]
        if case["kind"] == "topk":
            return dict(top_ids=None, top_logp=top, logp=at_y, entropy=ent, lse=lse)
        ids[top == -math.inf] = -1
        s["ids"], s["logp"] = ids, top
        out.update(top_ids=None, top_logp=top)
    w = torch.ones(n, **f64) if s["weights"] is None else s["weights"].double()
    kl, lse = torch.zeros(n, **f64), torch.zeros(n, **f64)
    d = None if case["kind"] == "forward" else torch.zeros(n, V, **f64)
    for a in range(0, n, step):
        b = min(n, a + step)
        x = s["logits"].detach()[a:b].double() / T
        lp = torch.log_softmax(x, 1)
        ids, t = s["ids"][a:b].long(), s["logp"][a:b].double()
        rows, cols = (ids >= 0).nonzero(as_tuple=True)
        t = t.masked_fill(ids < 0, -math.inf)
        if case["tail"] == RENORM:
            t = torch.log_softmax(t, 1).nan_to_num(nan=-math.inf)
        target = torch.zeros_like(x)                       # the teacher's mass of each listed token
        target[rows, ids[rows, cols]] = t[rows, cols].exp()
        outside = torch.ones_like(x, dtype=torch.bool)
        outside[rows, ids[rows, cols]] = False
        p = lp.exp()
        p_rest = torch.where(outside, p, 0.0).sum(1)
        q_rest = (1 - target.sum(1)).clamp(min=0) if case["tail"] == BUCKET else torch.zeros(b - a, **f64)
        q_rest = torch.where(p_rest > 0, q_rest, 0.0)
        on = (ids >= 0).any(1) & (w[a:b] != 0)
        terms = torch.where(target > 0, target * (target.log() - lp), 0.0).sum(1)
        terms += torch.where(q_rest > 0, q_rest * (q_rest / p_rest).log(), 0.0)
        kl[a:b] = torch.where(on, terms, 0.0)
        lse[a:b] = torch.where(on, torch.logsumexp(x, 1), 0.0)
        if d is not None:
            mass = target.sum(1) + q_rest
            share = torch.where(p_rest > 0, q_rest / p_rest, 0.0)
            per_row = torch.where(on, w[a:b], 0.0) / (n * T)
            d[a:b] = per_row[:, None] * (p * mass[:, None] - torch.where(outside, p * share[:, None], target))
    out.update(loss=(w * kl).sum() / n, kl=kl, lse=lse, counters=None)
    return out if d is None else dict(out, dlogits=d)
