"""token_topk where few long rows are split over workgroups, which is what its workspace is for: whatever the workspace holds, shared by
two shapes, in graphs, and without one."""
import ctypes

import pytest
import torch

import paper_2507_19766_amd as ulorl
from test_gpu_distill import compare, problem, reference
from test_gpu_topk import BF, DEV, F, check, rows, tokens
from test_gpu_topk import reference as topk_reference

pytestmark = pytest.mark.gpu
FIELDS = ("top_ids", "top_logp", "logp", "entropy", "lse")


def workspace(n, V):
    return torch.empty(ulorl.token_topk_workspace_bytes(n, V), dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("n,V,dtype", [(1, 151936, BF), (40, 70001, BF), (200, 57352, BF), (40, 32003, F)])
def test_split_rows_in_a_graph(n, V, dtype):
    """Replays read the logits of the moment, with other work between them and garbage in the workspace before each."""
    z, y, ws = rows(n, V, dtype, 4), tokens(n, V), workspace(n, V)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = ulorl.token_topk(z, 12, y)
    with torch.cuda.stream(side):
        ulorl.token_topk(z, 12, y, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ulorl.token_topk(z, 12, y, out=out, workspace=ws)
    for seed in range(4):
        z.copy_(rows(n, V, dtype, 20 + seed))
        ws.fill_((255, 0, 127, 128)[seed])
        for name in FIELDS:
            getattr(out, name).zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = check(z, 12, 1.0, y)
        for name in FIELDS:
            assert torch.equal(getattr(out, name), getattr(eager, name)), name


def test_a_workspace_shared_by_two_shapes():
    a, b = rows(40, 151936, BF, 1), rows(7, 70001, F, 2)
    want = [ulorl.token_topk(a, 33), ulorl.token_topk(b, 128)]
    ws, graphs, outs = workspace(40, 151936), [], []
    for z, k in ((a, 33), (b, 128)):
        out, graph = ulorl.token_topk(z, k, workspace=ws), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ulorl.token_topk(z, k, out=out, workspace=ws)
        graphs.append(graph)
        outs.append(out)
    for turn in range(6):
        out, r = outs[turn % 2], want[turn % 2]
        for name in ("top_ids", "top_logp", "entropy", "lse"):
            getattr(out, name).zero_()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        for name in ("top_ids", "top_logp", "entropy", "lse"):
            assert torch.equal(getattr(out, name), getattr(r, name)), name


@pytest.mark.parametrize("n,V,dtype", [(1, 151936, BF), (64, 151936, BF), (200, 57352, BF), (3, 70001, F), (5, 32003, BF)])
def test_without_a_workspace_the_ids_are_the_same(n, V, dtype):
    z, y, k = rows(n, V, dtype, 3), tokens(n, V), 40
    z[0] = (z[0] * 0.4).round()                                 # equal logits too
    split = check(z, k, 1.0, y)
    r = ulorl.TopkResult(*(torch.empty_like(getattr(split, name)) for name in FIELDS))

    def at(t):
        return ctypes.c_void_p(t.data_ptr())
    rc = ulorl.load_library().ulorl_token_topk(at(z), ulorl.BF16 if dtype == BF else ulorl.F32, n, V, z.stride(0), at(y), k, 1.0, at(r.top_ids),
                                               at(r.top_logp), at(r.logp), at(r.entropy), at(r.lse), None, 0,
                                               ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    assert torch.equal(r.top_ids, split.top_ids)
    want, tol = topk_reference(z, k, 1.0, y)
    for name, t in tol.items():
        assert ((getattr(r, name).double() - want[name]).abs() <= t).all(), name


def test_split_rows_recorded_and_distilled_in_a_graph():
    n, V, K = 48, 70001, 32
    teacher, w, p = rows(n, V, BF, 1), torch.ones(n, device=DEV), ulorl.DistillParams()
    student = problem(n, V, K, BF, 2)[0]
    w[5] = 0.0
    ws_a, ws_b = workspace(n, V), torch.empty(ulorl.distill_workspace_bytes(n, V), dtype=torch.uint8, device=DEV)
    record = ulorl.token_topk(teacher, K, workspace=ws_a)
    out, d = ulorl.distill_fwd_bwd(student, record.top_ids, record.top_logp, w, p, workspace=ws_b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ulorl.token_topk(teacher, K, out=record, workspace=ws_a)
        ulorl.distill_fwd_bwd(student, record.top_ids, record.top_logp, w, p, out=out, dlogits=d, workspace=ws_b)
    for seed in range(3):
        teacher.copy_(rows(n, V, BF, 30 + seed))
        student.copy_(rows(n, V, BF, 40 + seed))
        ws_a.fill_(255)
        ws_b.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(record.top_ids, ulorl.token_topk(teacher, K).top_ids)
        ref, tol = reference(student, record.top_ids, record.top_logp, w, p)
        compare(dict(kl=out.kl, lse=out.lse, loss=out.loss, dlogits=d), ref, tol, BF)
