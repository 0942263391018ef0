"""Arguments that token_topk and the distillation calls refuse, without a GPU: every call below fails on the host, before
anything is launched."""
import ctypes
import math

import pytest
import torch

import paper_2507_19766_amd as ulorl

vp = ctypes.c_void_p


def topk(logits=0x1000, dt=1, N=4, V=1000, stride=1000, y=0x2000, K=8, T=1.0, ids=0x3000, logps=0x4000, logp=0x5000, ent=0x6000, lse=0x7000,
         ws=None, size=0):
    return ulorl.load_library().ulorl_token_topk(vp(logits) if logits else None, dt, N, V, stride, vp(y) if y else None, K, T,
                                                 vp(ids) if ids else None, vp(logps) if logps else None, vp(logp) if logp else None,
                                                 vp(ent) if ent else None, vp(lse) if lse else None, vp(ws) if ws else None, size, None)


def test_topk_refuses_before_anything_is_launched():
    assert topk(logits=0) == -1 and topk(ids=0) == -1 and topk(logps=0) == -1 and topk(ent=0) == -1 and topk(lse=0) == -1
    assert topk(logp=0) == -1                                  # a token's log-prob is asked for
    assert topk(dt=2) == -3
    assert topk(N=0) == -2 and topk(V=0) == -2 and topk(stride=999) == -2 and topk(K=0) == -2 and topk(K=129) == -2
    assert topk(N=1 << 31) == -2 and topk(V=1 << 31, stride=1 << 31) == -2
    assert topk(logits=0x1008) == -4 and topk(V=999, stride=1001) == -4
    for T in (0.0, -1.0, math.nan, math.inf, 1e-4, 1e4):
        assert topk(T=T) == -5
    assert topk(ws=0x8001, size=1 << 30) == -6 and topk(ws=0x8000, size=1) == -6


def test_topk_workspace_query():
    assert ulorl.token_topk_workspace_bytes(0, 100) == 0 and ulorl.token_topk_workspace_bytes(4, 0) == 0
    assert ulorl.token_topk_workspace_bytes(4, 1 << 31) == 0
    assert 0 < ulorl.token_topk_workspace_bytes(1, 151936) < 1 << 20
    assert ulorl.token_topk_workspace_bytes(100000, 151936) < 1 << 24


def test_topk_needs_a_gpu_tensor():
    with pytest.raises(RuntimeError, match="GPU"):
        ulorl.token_topk(torch.zeros(2, 16), 4)




def params(T=1.0, tail=0, D=0.0, reserved=0):
    return ulorl.binding._CDistillParams(T, tail, D, (ctypes.c_int32 * 2)(0, reserved))


def p_(x):
    return vp(x) if x else None


def forward(logits=0x1000, dt=1, N=4, V=1000, stride=1000, ids=0x2000, teacher=0x3000, K=8, w=0, p=params(), loss=0x4000, kl=0x5000, lse=0x6000,
            rmax=0x7000, rcoef=0x8000, top=0x9000, counters=0, dlogits=0xa000, ws=0x100000, size=1 << 30, both=False):
    lib = ulorl.load_library()
    head = [p_(logits), dt, N, V, stride, p_(ids), p_(teacher), K, p_(w), ctypes.byref(p) if p else None]
    tail = [p_(x) for x in (loss, kl, lse, rmax, rcoef, top, counters)]
    if both:
        return lib.ulorl_distill_fwd_bwd(*head, 1.0, *tail, p_(dlogits), p_(ws), size, None, None)
    return lib.ulorl_distill_fwd(*head, *tail, p_(ws), size, None)


@pytest.mark.parametrize("both", [False, True])
def test_distill_refuses_before_anything_is_launched(both):
    for name in ("logits", "ids", "teacher", "loss", "kl", "lse", "rmax", "rcoef", "top", "p"):
        assert forward(**{name: 0, "both": both}) == -1, name
    assert forward(dt=7, both=both) == -3
    for bad in (dict(N=0), dict(V=0), dict(stride=992), dict(K=0), dict(K=129), dict(N=(1 << 24) + 1), dict(V=1 << 31, stride=1 << 31)):
        assert forward(both=both, **bad) == -2, bad
    assert forward(logits=0x1004, both=both) == -4 and forward(V=1001, stride=1001, both=both) == -4
    for bad in (params(T=0.0), params(T=-1.0), params(T=math.nan), params(T=math.inf), params(tail=3), params(tail=-1), params(D=math.nan),
                params(reserved=1)):
        assert forward(p=bad, both=both) == -5
    assert forward(ws=0, both=both) == -6 and forward(ws=0x100010, both=both) == -6 and forward(size=64, both=both) == -6
    if both:
        assert forward(dlogits=0, both=True) == -1 and forward(dlogits=0xa004, both=True) == -4


def test_distill_backward_refuses_before_anything_is_launched():
    lib = ulorl.load_library()

    def bwd(logits=0x1000, dt=1, N=4, V=1000, stride=1000, ids=0x2000, K=8, T=1.0, rmax=0x7000, rcoef=0x8000, top=0x9000, d=0xa000):
        return lib.ulorl_distill_bwd(p_(logits), dt, N, V, stride, p_(ids), K, T, p_(rmax), p_(rcoef), p_(top), 1.0, None, p_(d), None)
    for name in ("logits", "ids", "rmax", "rcoef", "top", "d"):
        assert bwd(**{name: 0}) == -1, name
    assert bwd(dt=2) == -3 and bwd(N=0) == -2 and bwd(K=129) == -2 and bwd(stride=900) == -2 and bwd(d=0xa008) == -4 and bwd(T=0.0) == -5


def test_distill_workspace_query():
    size = ulorl.distill_workspace_bytes
    assert size(0, 100) == 0 and size(4, 0) == 0 and size((1 << 24) + 1, 100) == 0 and size(4, 1 << 31) == 0
    for dtype in (torch.bfloat16, torch.float32):
        sizes = [size(n, 151936, dtype) for n in (1, 2, 100, 1000, 16384, 131072)]
        assert sizes == sorted(sizes) and sizes[0] > 0 and sizes[-1] < 131072 * 256 and all(s % 256 == 0 for s in sizes)


def test_distill_needs_a_gpu_tensor():
    ids, logp = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 4)
    for call in (ulorl.distill_fwd, ulorl.distill_fwd_bwd, ulorl.autograd.distill_loss):
        with pytest.raises(RuntimeError, match="GPU"):
            call(torch.zeros(2, 16), ids, logp)
