"""The RMS norm of the streams' sum against its 64-bit form."""
import pytest
import torch

import op_refs as R
from paper_2607_14530_gb300 import synth
from paper_2607_14530_gb300.xhc import SumNorm, XhcError
from xhc_cases import Guarded

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
SHAPES = [(1, 1, 8), (1, 16, 4096), (3, 32, 16384), (5, 7, 264), (17, 1, 2056), (24, 16, 4096), (31, 2, 248), (64, 1, 256),
          (100, 8, 1024), (129, 9, 520), (700, 4, 264), (1000, 1, 16384), (2500, 1, 4096), (5003, 1, 2056), (3001, 16, 512)]


def run(op, X, w, dy, accumulate=False, start=None):
    T = dy.shape[0]
    saved, ws = op.alloc_saved(T), op.alloc_workspace(T)
    saved.fill_(0xFF)
    ws.fill_(0xFF)
    y, dX = Guarded(torch.full((T, op.C), float("nan"), dtype=BF)), Guarded(torch.full(X.shape, float("nan"), dtype=BF))
    dw = Guarded(torch.full((op.C,), float("nan")) if start is None else start)
    op.forward(w, X, y=y.t, saved=saved)
    op.backward(w, X if op.N == 1 else None, dy, dw.t, saved, ws, dX=dX.t, accumulate=accumulate)
    torch.cuda.synchronize()
    assert y.intact() and dX.intact() and dw.intact()
    return {"y": y.t, "dX": dX.t, "dw": dw.t}


def inputs(T, N, C, seed):
    return (synth.normal_bf16((T, N, C), seed).cuda(), (1 + 0.2 * synth.normal_bf16((C,), seed + 1).float()).cuda(),
            synth.normal_bf16((T, C), seed + 2).cuda())


@pytest.mark.parametrize("T,N,C", SHAPES)
def test_forward_and_backward(T, N, C):
    X, w, dy = inputs(T, N, C, T)
    op = SumNorm(N, C)
    got = run(op, X, w, dy)
    R.assert_within(got, R.sum_norm(X, w, op.eps, dy))
    assert torch.equal(op.forward(w, X), got["y"])        # nothing kept: the same bits
    start = torch.randn(C, generator=torch.Generator().manual_seed(1))
    assert torch.equal(run(op, X, w, dy, True, start)["dw"], got["dw"] + start.cuda())


def test_hidden_vector_without_a_stream_axis():
    X, w, dy = inputs(40, 1, 256, 5)
    op = SumNorm(1, 256)
    a, b = run(op, X, w, dy), run(op, X[:, 0].contiguous(), w, dy)
    assert torch.equal(a["y"], b["y"]) and torch.equal(a["dX"][:, 0], b["dX"]) and torch.equal(a["dw"], b["dw"])


@pytest.mark.parametrize("N", [1, 4])
def test_magnitudes(N):
    """Zero tokens (the norm is eps alone), tiny and large ones, and a token with NaN beside them."""
    X, w, dy = inputs(6, N, 512, 7)
    X[0] = 0
    X[1] *= 2.0 ** -40
    X[2] *= 2.0 ** 40
    op = SumNorm(N, 512)
    got = run(op, X, w, dy)
    assert bool((got["y"][0] == 0).all())
    ref = R.sum_norm(X, w, op.eps, dy)
    R.assert_within(got, ref, ("y", "dX"))
    X[4, 0, 9] = float("nan")
    bad = run(op, X, w, dy)
    assert bool(bad["y"][4].isnan().all())
    for t in (0, 1, 2, 3, 5):
        assert torch.equal(bad["y"][t], got["y"][t]) and torch.equal(bad["dX"][t], got["dX"][t])


@pytest.mark.parametrize("T,N,C", [(24, 16, 1024), (3000, 1, 2056)])
def test_streams_repeats_and_graphs(T, N, C):
    X, w, dy = inputs(T, N, C, 3)
    op = SumNorm(N, C)
    want = run(op, X, w, dy)
    saved, ws = op.alloc_saved(T), op.alloc_workspace(T)
    y, dX, dw = torch.empty(T, C, dtype=BF, device="cuda"), torch.empty_like(X), torch.empty_like(w)
    side = torch.cuda.Stream()

    def step():
        op.forward(w, X, y=y, saved=saved)
        op.backward(w, X, dy, dw, saved, ws, dX=dX)

    def same():
        torch.cuda.synchronize()
        return torch.equal(y, want["y"]) and torch.equal(dX, want["dX"]) and torch.equal(dw, want["dw"])

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            step()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, dX, dw):
        t.fill_(float("nan"))
    graph.replay()
    assert same()


def test_refusals():
    X, w, dy = inputs(4, 2, 64, 1)
    op = SumNorm(2, 64)
    saved, ws = op.alloc_saved(4), op.alloc_workspace(4)
    with pytest.raises(XhcError, match="X must be"):
        op.forward(w, X.float())
    with pytest.raises(XhcError, match="shape"):
        op.forward(w, X[:, :1].contiguous())
    with pytest.raises(XhcError, match="w must be"):
        op.forward(w.to(BF), X)
    with pytest.raises(XhcError, match="bytes"):
        op.forward(w, X, saved=saved[:16])
    with pytest.raises(XhcError, match="X is needed"):
        SumNorm(1, 64).backward(w, None, dy, torch.empty_like(w), saved, ws)
    with pytest.raises(XhcError, match="invalid"):
        op.forward(w, X[:0])
