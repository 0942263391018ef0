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
