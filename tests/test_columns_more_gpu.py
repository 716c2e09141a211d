"""More of the learned columns on the GPU against the fp64 oracle: launches that begin inside a
row, digits of ten bits, three digits, what is not finite beside what is, widths whose blocks do not
divide a workgroup, the loss at far z, and fits that drop features on the same rows."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import ks_columns as o
from paper_2606_28565_amd import fit
from tests.test_columns_fit_gpu import data
from tests.test_columns_gpu import (SEED, check_back, check_eta, columns, f64, family_split, make_ids, rnd, run_back,
                                    run_dropout, run_embed, run_eta, run_order, untouched)

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


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_what_is_not_finite_beside_what_is(t):
    """Rows of numbers between rows of infinities and NaN keep their values."""
    import torch
    x = rnd(64, 23, 23, 0, t)
    x[::3] = float("nan")
    x[1::3] = float("inf")
    buf, y = columns(64, 23, 29, 1, t)
    run_dropout(x, y, 0.5)
    k = o.keep(np.arange(64), 23, 0.5, SEED, 1, 5)[0]
    got, want = f64(y), f64(x)
    assert (got[2::3][k[2::3]] == 2 * want[2::3][k[2::3]]).all() and (got[~k] == 0).all()
    assert np.isnan(got[::3][k[::3]]).all() and (got[1::3][k[1::3]] == np.inf).all()
    assert untouched(buf, y)


def test_a_launch_that_begins_inside_a_row():
    """Three blocks a row: a launch's 2^28 blocks (2^29 of a lookup of bfloat16) end inside
    one, and the next launch's begin there."""
    import torch
    seam = (1 << 28) // 3
    x = torch.ones(seam + 50_000, 17, dtype=torch.bfloat16, device="cuda")
    run_dropout(x, x, 0.5)
    for lo in (0, seam - 30_000, seam + 40_000):
        rows = np.arange(lo, min(lo + 60_000, len(x)))
        assert (f64(x[lo:lo + 60_000]) == 2.0 * o.keep(rows, 17, 0.5, SEED, 1, 5)[0]).all()
    share = sum(int((c != 0).sum()) for c in x.split(1 << 24)) / x.numel()
    assert abs(share - 0.5) < 5 * 0.5 / np.sqrt(x.numel())
    del x
    seam = (1 << 29) // 3
    table = rnd(7, 17, 17, 0, "bf16")
    ids = torch.arange(seam + 50_000, dtype=torch.int32, device="cuda").remainder_(9)   # (7 and 8: none)
    y = torch.full((seam + 50_000, 17), -77.0, dtype=torch.bfloat16, device="cuda")
    run_embed(table, 1.0, ids, y)
    far = torch.cat([table, torch.zeros_like(table[:2])])
    for lo in range(0, len(y), 1 << 24):
        assert torch.equal(y[lo:lo + (1 << 24)], far[ids[lo:lo + (1 << 24)].long()]), lo
    run_embed(table, 1.0, ids, y, (0.5, SEED, 1, 5))
    for lo in (0, seam - 30_000, seam + 40_000):
        rows = np.arange(lo, min(lo + 60_000, len(y)))
        assert (f64(y[lo:lo + 60_000]) == 2.0 * f64(far)[rows % 9] * o.keep(rows, 17, 0.5, SEED, 1, 5)[0]).all()


# ------------------------------------------------------------------ order of ids
def check_order(ids, v):
    import torch
    got = run_order(ids, v)
    key = torch.where((ids < 0) | (ids >= v), v, ids)
    want, row = torch.sort(key, stable=True)
    assert (got.t["row"].long() == row).all() and (got.t["id"] == want).all()
    for lo in range(0, v + 1, 1 << 24):
        at = torch.arange(lo, min(lo + (1 << 24), v + 1), dtype=torch.int32, device="cuda")
        assert torch.equal(got.t["off"][lo:lo + (1 << 24)], torch.searchsorted(want, at, out_int32=True)), lo
    return got


@pytest.mark.parametrize("v", [1 << 18, 300_007, (1 << 20) - 2, (1 << 20) - 1, (1 << 24) + 1, (1 << 27) + 5])
@pytest.mark.parametrize("n", [1, 4096, 4097, 8192, 8193, 16_384, 16_385, 70_001, 1_100_003])
def test_order_of_wide_digits(n, v):
    """Two digits of ten bits, within and in passes; three of nine and ten."""
    for kind in ("skew", "one", "all"):
        check_order(make_ids(n, v, n % 1000, kind), v)


# ------------------------------------------------------------------ the table's gradient
def test_zeros_that_begin_inside_a_row():
    """Three quads of columns a row, over 2^30 in all: the second launch's zeros begin inside
    a row; all ids' rows and nothing else."""
    import torch
    v, dim, n = (1 << 30) // 3 + 100_000, 10, 5000
    ids = (torch.rand(n, generator=torch.Generator("cuda").manual_seed(4), device="cuda", dtype=torch.float64) * v).int()
    ids[:40] = (1 << 30) // 3 - 20 + torch.arange(40, device="cuda")   # (about where it begins)
    ids[40:43] = torch.tensor([0, v - 1, v], device="cuda")
    dy = rnd(n, dim, dim, 0, "f32")
    order = check_order(ids, v)
    grad = torch.full((v, dim), float("nan"), device="cuda")
    run_back(order, dy, grad)
    known = ids < v
    want = torch.zeros(n, dim, dtype=torch.float64, device="cuda")   # an id's sum, where it first stands
    seen, to = torch.unique(ids[known].long(), return_inverse=True)
    want = want[:len(seen)].index_add_(0, to, dy[known].double())
    size = torch.zeros_like(want).index_add_(0, to, dy[known].double().abs())
    assert int(torch.bincount(to).max()) <= 64   # (so that an id's additions are its rows' alone)
    assert ((grad[seen].double() - want).abs() <= (torch.bincount(to).max() + 1) * o.EPS * size).all()
    grad[seen] = 0.0
    assert all(bool((c == 0).all()) for c in grad.split(1 << 24))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [696, 1032, 1040, 1536, 2047, 2049, 2304])
def test_gradient_of_widths_off_the_workgroup(t, dim):
    """Blocks that leave lanes without work, and a last tile of few."""
    for n, v, kind in ((3, 5, "all"), (2500, 40, "skew"), (4001, 1, "one")):
        check_back(n, v, dim, t, 3, 1, 0.7, (0.2, SEED, 3, 4), kind)


@pytest.mark.parametrize("dim", [1024, 2048, 4096])
def test_gradient_of_one_id_and_wide_rows(dim):
    """All rows are one id's: its sum goes on through every workgroup."""
    check_back(9001, 3, dim, "bf16", kind="one", positive=True)


# ------------------------------------------------------------------ the loss at given z
@pytest.mark.parametrize("n", [5000, 60_001])
@pytest.mark.parametrize("huber", [0.3, 1e3, float("inf")])
@pytest.mark.parametrize("around", [0, 20, 45, 70])
def test_dz_of_far_z(n, huber, around):
    """sigma(-z) down to 1e-32 keeps its precision, whatever its size; eta near and far from
    what z says."""
    import torch
    g = torch.Generator().manual_seed(around + n)
    z = around + 5 * torch.rand(n, generator=g)
    z = torch.where(torch.rand(n, generator=g) < 0.1, -z, z)
    eta = torch.exp(torch.rand(n, generator=g) * torch.tensor([1e-3, 1.0, 30.0])[torch.randint(0, 3, (n,), generator=g)])
    weight = 0.5 + torch.rand(n, generator=g)
    z, eta, weight = z.cuda(), eta.cuda(), weight.cuda()
    off = family_split(n)
    check_eta(z, eta, weight, off, huber, run_eta(z, eta, weight, off, huber))
    check_eta(z, eta, None, off, huber, run_eta(z, eta, None, off, huber))
