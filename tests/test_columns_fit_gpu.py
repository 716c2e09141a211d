"""A fit with learned columns and dropout as a whole: its gradients against the fp64 oracle,
captured steps, changed ids, and the heads of one category in the evaluation."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import ks_columns as oc
from oracle import ks_fit as of
from paper_2606_28565_amd import abi, fit
from tests.test_columns_gpu import f64, family_split, make_eta, make_ids
from tests.test_gated_eval_gpu import REL, REL_BF16, gated_oracle
from workload import gen

pytestmark = pytest.mark.gpu
NFAM = abi.NFAM
EPS = of.EPS


def data(n, categories, prec="f32", seed=3, huber=0.5, kind="mixed"):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.rand(n, 16, generator=g)
    x[:, 15] = 1.0
    x = x.to(torch.bfloat16 if prec == "bf16" else torch.float32).cuda()
    _, eta, weight = make_eta(n)
    ids = make_ids(n, categories, seed) if categories else None
    return fit.Measurements(x, family_split(n, kind), eta, weight, huber, ids, categories)


def noisy(d, ft, prec):
    """The rows that a step's heads see, as the oracle forms them (fp64; bf16 rounded)."""
    x, count = f64(d.x)[:, :16], int(ft.count)
    def low(v):   # what a row's type makes of a number
        import torch
        return torch.from_numpy(v).to(torch.bfloat16 if prec == "bf16" else torch.float32).double().numpy()
    if ft.feature_drop is not None:
        x = np.concatenate([low(oc.drop(x[:, :15], ft.feature_drop.p, ft.feature_drop.seed, 0, count)), x[:, 15:]], 1)
    drop = None if ft.drop is None else (ft.drop.p, ft.drop.seed, 1, count)
    e = oc.embed(f64(ft.weights["table"]), 1.0, d.ids.cpu().numpy(), drop)
    return np.concatenate([x, low(e)], 1), drop


@pytest.mark.parametrize("prec,hid", [("f32", 48), ("f32", 64), ("bf16", 64), ("bf16", 130)])
@pytest.mark.parametrize("dropout,feature_dropout", [(0.0, 0.0), (0.3, 0.0), (0.2, 0.1)])
def test_gradients_of_a_step(prec, hid, dropout, feature_dropout):
    """Loss and gradients of the second step, against the oracle's chain; bounds as of the
    parts: dz carries z's error, the rows' gradients dz's, the table's theirs."""
    n, c = 3000, 9
    d = data(n, c, prec)
    ft = fit.GatedFit(hidden=hid, precision=prec, seed=5, categories=c, dropout=dropout, feature_dropout=feature_dropout)
    ft.step(d)
    x, drop = noisy(d, ft, prec)
    w = {k: f64(v) for k, v in ft.weights.items()}
    loss = f64(ft.gradients(d))
    # the rows are within a rounding (bf16's is part of the rows' definition; its borders may
    # fall either way after fp32's two roundings) of the oracle's: take theirs
    seen = f64(ft_rows(d, ft))
    assert (np.abs(seen - x) <= (3 * EPS + (2.0 ** -7 if prec == "bf16" else 0)) * np.abs(x)).all()
    x = seen
    off, eta, weight = list(d.rows.fam_off), f64(d.eta), f64(d.weight)
    dx, edx = np.zeros((n, 32)), np.zeros((n, 32))
    for f in range(NFAM):
        r = slice(off[f], off[f + 1])
        if r.start == r.stop:
            continue
        z, k = of.block(x[r], w["w1"][f], w["w2"][f], w["w3"][f], w["b3"][f])
        want, dz = of.eta_loss(z, eta[r], weight[r], 0.5)
        b, b_dz = oc.eta_bounds(z, eta[r], weight[r], 0.5, want, dz)
        wt = of.counted(eta[r], weight[r])
        share = wt / wt.sum()
        ez = np.where(wt > 0, k["err"]["z"], 0)
        assert abs(loss[f] - want) <= b + (share * np.minimum(0.5, 20) * ez).sum() + 4 * EPS * want
        # drho/dz = slope sigma(-z): its derivative by z is at most sigma^2 + slope sigma (1 - sigma) < 1.2
        edz = b_dz + share * 1.2 * ez
        val, err = of.gradients(x[r], w["w1"][f], w["w2"][f], w["w3"][f], dz, k, 16 + n // 128)
        t = np.abs(k["s"] + k["a"] * (1 - k["s"])) * np.abs(k["u"]) * np.abs(w["w3"][f])
        a3 = np.abs(k["a"] * w["w3"][f])
        more = {"w1": (edz[:, None] * t).T @ np.abs(x[r]), "w2": (edz[:, None] * a3).T @ np.abs(x[r]),
                "w3": (edz[:, None] * np.abs(k["y"])).sum(0), "b3": edz.sum()}
        for key, m in more.items():
            got = f64(ft.grad[key])[f]
            assert (np.abs(got - val[key]) <= 1.01 * (err[key] + m) + 2 * EPS * np.abs(val[key])).all(), (key, f)
        dx[r] = val["x"]
        edx[r] = err["x"] + edz[:, None] * (t @ np.abs(w["w1"][f]) + a3 @ np.abs(w["w2"][f]))
        if prec == "bf16":
            edx[r] += 2.0 ** -8 * (np.abs(dx[r]) + edx[r])
    want, b = oc.embed_back(d.ids.cpu().numpy(), c, dx[:, 16:], 1.0, drop)
    spread, _ = oc.embed_back(d.ids.cpu().numpy(), c, edx[:, 16:], 1.0, drop)
    assert (np.abs(f64(ft.grad["table"]) - want) <= 1.01 * (b + spread) + 4 * EPS * spread).all()


def ft_rows(d, ft):
    return d.noisy if ft.feature_drop is not None else d.x


def test_feature_dropout_without_categories():
    """ks_gated_loss on the dropped rows: the same call by hand, bit for bit."""
    import torch
    n = 2000
    d = data(n, 0)
    ft = fit.GatedFit(16, 32, seed=5, feature_dropout=0.25)
    ft.step(d)
    loss = ft.gradients(d).clone()
    want = oc.drop(f64(d.x[:, :15]), 0.25, 5, 0, 1)
    assert (np.abs(f64(d.noisy[:, :15]) - want) <= 3 * EPS * np.abs(want)).all() and (d.noisy[:, 15] == 1).all()
    by_hand = fit.Measurements(d.noisy, list(d.rows.fam_off), d.eta, d.weight, 0.5)
    plain = fit.GatedFit(16, 32, seed=5)
    for k in plain.param:
        plain.param[k].copy_(ft.param[k])
    assert torch.equal(plain.gradients(by_hand), loss) and all(torch.equal(plain.grad[k], ft.grad[k]) for k in ft.grad)


@pytest.mark.parametrize("prec,bits", [("f32", 32), ("bf16", 8)])
def test_captured_steps_are_the_eager_ones(prec, bits):
    """Parameters and loss after every replay, bit for bit; each replay drops anew; eager work
    of another fit between the replays."""
    import torch
    n, c = 5000, 11
    make = lambda: fit.GatedFit(hidden=40, precision=prec, seed=7, state_bits=bits, categories=c, dropout=0.2, feature_dropout=0.1)
    a, b, da, db = make(), make(), data(n, c, prec), data(n, c, prec)
    b.workspace(db)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.step(db)
    torch.cuda.current_stream().wait_stream(s)
    a.step(da)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step(db)
    masks = []
    for i in range(4):
        g.replay()
        torch.cuda.synchronize()
        a.step(da)
        torch.cuda.synchronize()
        assert torch.equal(a.loss, b.loss) and all(torch.equal(a.param[k], b.param[k]) for k in a.param), i
        assert torch.equal(da.noisy, db.noisy)
        masks.append(da.noisy[:, 16:] == 0)
    assert int(b.count) == 5
    assert not any(torch.equal(masks[i], masks[i + 1]) for i in range(3))


def test_changed_ids():
    """A minibatch in the same tensors: after sort() as with rows made for it."""
    import torch
    n, c = 1500, 30
    d = data(n, c)
    ft, other = fit.GatedFit(hidden=16, categories=c), fit.GatedFit(hidden=16, categories=c)
    ft.gradients(d)
    d.ids.copy_(make_ids(n, c, 77))
    d.sort()
    fresh = data(n, c)
    fresh.ids.copy_(make_ids(n, c, 77))
    fresh.sort()
    assert torch.equal(ft.gradients(d), other.gradients(fresh)) and torch.equal(ft.grad["table"], other.grad["table"])


@pytest.mark.parametrize("n", [0, 1, 7])
def test_few_rows(n):
    d = data(n, 3)
    ft = fit.GatedFit(hidden=8, categories=3, dropout=0.5)
    ft.step(d)
    import torch
    torch.cuda.synchronize()
    assert all(torch.isfinite(v).all() for v in ft.param.values()) and torch.isfinite(ft.loss).all()
    if n == 0:
        assert (ft.grad["table"] == 0).all() and (ft.loss == 0).all()


def test_rows_without_a_category_train_the_heads_alone():
    import torch
    n, c = 900, 4
    d = data(n, c)
    d.ids.fill_(-1)
    d.sort()
    ft = fit.GatedFit(hidden=24, categories=c)
    ft.gradients(d)
    assert (d.x[:, 16:] == 0).all() and (ft.grad["table"] == 0).all() and (ft.grad["w1"][:, :, :16] != 0).any()
    torch.cuda.synchronize()


# ------------------------------------------------------------------ one category's heads
@pytest.mark.parametrize("prec,hid", [("f32", 64), ("bf16", 100)])
@pytest.mark.parametrize("category", [None, 0, 3])
def test_heads_of_a_category(prec, hid, category):
    """z of rows of that category is z of the 16 features through its heads; 16 products and
    the addition to column 15 are rounded (bf16: the column once more)."""
    import torch
    c, n = 4, 400
    d = data(n, c, prec, kind="one")
    ft = fit.GatedFit(hidden=hid, precision=prec, seed=9, categories=c)
    for _ in range(3):
        ft.step(d)
    d.ids.fill_(-1 if category is None else category)
    d.sort()
    ft.gradients(d)
    h = ft.heads_for(category)
    z = torch.empty(n, device="cuda")
    x16 = d.x[:, :16]
    abi.ks_gated_forward(h, abi.feature_rows(x16, list(d.rows.fam_off)), z.data_ptr(), abi.current_stream())
    torch.cuda.synchronize()
    f = 4
    w = {k: f64(v)[f] for k, v in ft.weights.items() if k != "table"}
    want, k = of.block(f64(d.x), w["w1"], w["w2"], w["w3"], w["b3"])
    folded = {k_: f64(v)[f] for k_, v in h.weights.items()}
    z16, k16 = of.block(f64(x16), folded["w1"], folded["w2"], folded["w3"], folded["b3"])
    assert (np.abs(f64(z) - z16) <= k16["err"]["z"]).all()
    e = np.abs(f64(d.x[:, 16:]))
    def moved(name):
        sums = e @ np.abs(w[name][:, 16:]).T + np.abs(w[name][:, 15])
        return (18 * EPS + (2.0 ** -8 if prec == "bf16" else 0)) * sums
    by = (1.1 * moved("w1") * np.abs(k["u"]) + moved("w2") * (np.abs(k["a"]) + 1.1 * moved("w1"))) @ np.abs(w["w3"])
    assert (np.abs(z16 - want) <= 1.01 * by + 1e-14).all()


@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_a_category_in_the_evaluation(prec):
    """Feature rows of records for two spec vectors, each a category; a fit on them; records
    priced with each category's heads: the oracle's evaluation with those weights."""
    import torch
    wl = gen.config1(0, 20)
    di = abi.DeviceInputs(wl, n_specs=2)
    rows = fit.feature_rows_of(di, 16, prec)
    n = rows.x.shape[0]
    # within a family the rows come spec by spec
    ids = torch.empty(n, dtype=torch.int32)
    for f in range(NFAM):
        lo, hi = rows.fam_off[f], rows.fam_off[f + 1]
        ids[lo:hi] = (torch.arange(hi - lo) >= (hi - lo) // 2).to(torch.int32)
    _, eta, _ = make_eta(n)
    d = fit.Measurements(rows.x, rows.fam_off, eta, ids=ids.cuda(), categories=2)
    ft = fit.GatedFit(hidden=64, precision=prec, categories=2, dropout=0.1)
    for _ in range(3):
        ft.step(d)
    for category in (0, 1, None):
        h = ft.heads_for(category)
        o, so = abi.kernel_outputs(wl.desc.n_rows, 2)
        abi.ks_eval_kernels(di.desc, di.specs_ptr, 2, h, so, di.ws_ptr, di.ws_bytes, abi.current_stream())
        torch.cuda.synchronize()
        want = gated_oracle(wl, {k: f64(v) for k, v in h.weights.items()}, 16, prec == "bf16", 2)
        for s in range(2):
            rel = np.abs(o["t_kernel"][s].double().cpu().numpy() - want["t"][s]) / want["t"][s]
            assert rel.max() <= (REL_BF16 if prec == "bf16" else REL), (category, s, rel.max())


def test_categories_priced_with_their_own_heads_differ():
    """The learned columns do reach the price (a category's heads are not another's)."""
    c = 3
    d = data(2000, c)
    ft = fit.GatedFit(hidden=32, categories=c)
    ft.step(d)
    w = [ft.heads_for(i).weights["w1"] for i in (None, 0, 1, 2)]
    assert all((w[0][:, :, :15] == v[:, :, :15]).all() for v in w)
    assert all((w[i][:, :, 15] != w[j][:, :, 15]).any() for i in range(4) for j in range(i))
