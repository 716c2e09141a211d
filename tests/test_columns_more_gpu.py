"""More of the learned columns on the GPU: fits that drop features on the same rows."""
from __future__ import annotations

import pytest

from paper_2606_28565_amd import fit
from tests.test_columns_fit_gpu import data

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ fits that drop features
def test_two_fits_on_the_same_rows():
    """Two captured steps on the same Measurements, replayed on two streams at a time: each
    as on rows of its own."""
    import torch
    n = 40_000
    shared, kw = data(n, 0), dict(in_dim=16, hidden=32, feature_dropout=0.3)
    alone = [(fit.GatedFit(seed=s, **kw), data(n, 0)) for s in (1, 2)]
    both = [fit.GatedFit(seed=s, **kw) for s in (1, 2)]
    for ft in both:
        ft.step(shared)
    for ft, rows in alone:
        ft.step(rows)
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in both]
    for ft in both:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ft.step(shared)
        graphs.append(g)
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (ft, rows), other in zip(alone, both):
            ft.step(rows)
            assert torch.equal(ft.loss, other.loss) and all(torch.equal(ft.param[k], other.param[k]) for k in ft.param)


def test_a_capture_needs_the_rows_first():
    """Without workspace() a step that drops features cannot be captured; with it, replays and
    eager steps go on from each other."""
    import torch
    d, ft, other = data(500, 0), fit.GatedFit(16, 16, seed=3, feature_dropout=0.2), fit.GatedFit(16, 16, seed=3, feature_dropout=0.2)
    zero = torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="workspace"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            zero.zero_()
            ft.step(d)
    assert int(ft.count) == 0
    ft.workspace(d)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ft.step(d)
    for i in range(3):
        ft.step(d)   # (before the first replay too)
        g.replay()
        other.step(d)
        other.step(d)
        torch.cuda.synchronize()
        assert torch.equal(ft.loss, other.loss) and all(torch.equal(ft.param[k], other.param[k]) for k in ft.param), i
        assert (d.noisy[:, 15] == 1).all()
