"""Gated heads where the framework uses them: feature rows (ks_features), the
evaluation (ks_eval_kernels, ks_eval_steps, ks_simulate in mode KS_ETA_GATED), and
a fit from measured times to priced steps."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import ks_fit as of
from oracle import ks_oracle as o
from paper_2606_28565_amd import abi, fit
from tests import gpu_helpers as g
from workload import gen

pytestmark = pytest.mark.gpu
NFAM = abi.NFAM
REL, REL_BF16 = 1e-5, 1e-2      # the evaluation's own tolerances (fp32 and bf16 heads)


def weights(prec, inp, hid, seed=11):
    import torch
    r = torch.Generator().manual_seed(seed)
    w = {"w1": torch.randn(NFAM, hid, inp, generator=r) * 0.3, "w2": torch.randn(NFAM, hid, inp, generator=r) * 0.3,
         "w3": torch.randn(NFAM, hid, generator=r) * 0.1, "b3": torch.randn(NFAM, generator=r) * 0.3}
    w = {k: v.to(torch.bfloat16 if prec == "bf16" else torch.float32) for k, v in w.items()}
    return {k: v.cuda() for k, v in w.items()}, {k: v.double().numpy() for k, v in w.items()}


def gated_oracle(wl, w, inp, bf16, n_specs, bounded=None, grid=None):
    """The oracle's evaluation with the gated block as the head of every family."""
    base = o.eval_kernels(wl.desc, wl.specs, None, eta_one=True, spec_ids=range(n_specs), bounded=bounded, grid=grid)
    fam = wl.desc.family()
    cnt = o.kernel_counts(wl.desc)
    eta = base["eta"].copy()
    for s in range(n_specs):
        sp = o.spec_at(wl.specs, s)
        rf = o.roofline(cnt["F"], cnt["Bt"], cnt["B"], sp)
        x = o.features(cnt, wl.desc.n, o.effective_k(wl.desc, np.arange(wl.desc.n_rows)), rf, sp, inp)
        if bf16:
            x = o.round_bf16(x)
        for f in np.unique(fam):
            sel = (fam == f) & ~base["routed"][s]
            if bounded is not None and (bounded.mask >> f) & 1:
                continue
            z, _ = of.block(x[sel], w["w1"][f], w["w2"][f], w["w3"][f], w["b3"][f])
            eta[s, sel] = 1 + np.exp(-z)
    t0 = wl.specs["t0"][:n_specs, None]
    return dict(base, eta=eta, t=np.maximum(base["t_roof"] * eta, t0))


def evaluate(wl, d, n_specs, steps=True, per_pair=True, bounded=None, grid=None):
    import torch
    di = abi.DeviceInputs(wl, n_specs=n_specs)
    hd = abi.gated_heads(d["w1"], d["w2"], d["w3"], d["b3"])
    if bounded is not None or grid is not None:
        m = di.make_heads("f32", 16, 64, abi.KS_ETA_GATED, bounded, grid)
        for k in ("in_dim", "hidden", "precision", "w1", "w2", "w3", "b3"):
            setattr(m, k, getattr(hd, k))
        m.b2 = None
        hd = m
    so_t, so = abi.step_outputs(wl.desc.n_steps, n_specs)
    ko_t, ko = abi.kernel_outputs(wl.desc.n_rows, n_specs, counts=False) if per_pair else ({}, None)
    if steps:
        abi.ks_eval_steps(di.desc, di.steps, di.specs_ptr, n_specs, hd, di.host, so, ko, di.ws_ptr, di.ws_bytes,
                          abi.current_stream())
    else:
        abi.ks_eval_kernels(di.desc, di.specs_ptr, n_specs, hd, ko, di.ws_ptr, di.ws_bytes, abi.current_stream())
    torch.cuda.synchronize()
    abi.ks_device_status(di.ws_ptr, di.ws_bytes, abi.current_stream())
    uniq = abi.ks_different_families(di.desc, n_specs, hd, ko, di.ws_bytes)
    return {k: v.cpu().numpy() for k, v in {**(so_t if steps else {}), **ko_t}.items()}, uniq


@pytest.fixture(scope="module")
def small():
    return gen.config1(0, 8)


@pytest.mark.parametrize("prec", ["f32", "bf16"])
@pytest.mark.parametrize("inp", [16, 32])
@pytest.mark.parametrize("hid", [1, 64, 100, 256])
def test_evaluation(small, prec, inp, hid):
    d, w = weights(prec, inp, hid)
    ns = len(small.specs["peak_flops"])
    ref = gated_oracle(small, w, inp, prec == "bf16", ns)
    rs = o.eval_steps(small.desc, small.steps, small.specs, small.host, spec_ids=range(ns), kern=ref)
    got, _ = evaluate(small, d, ns)
    tol = REL_BF16 if prec == "bf16" else REL
    assert g.rel_err(got["eta"], ref["eta"]).max() <= tol
    assert g.rel_err(got["t_kernel"], ref["t"]).max() <= tol
    assert g.rel_err(got["t_step"], rs["t_step"]).max() <= tol
    alone, _ = evaluate(small, d, ns, steps=False)
    assert (alone["t_kernel"] == got["t_kernel"]).all()


@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_evaluation_of_the_different_records(prec):
    """A trace whose records recur: evaluated once each, with the same steps."""
    wl = gen.config1(0, 1000)
    d, w = weights(prec, 16, 256)
    ns = len(wl.specs["peak_flops"])
    ref = gated_oracle(wl, w, 16, prec == "bf16", ns)
    rs = o.eval_steps(wl.desc, wl.steps, wl.specs, wl.host, spec_ids=range(ns), kern=ref)
    got, uniq = evaluate(wl, d, ns, per_pair=False)
    assert uniq != 0
    tol = REL_BF16 if prec == "bf16" else REL
    for k in ("t_body", "t_step"):
        assert g.rel_err(got[k], rs[k]).max() <= tol, k
    got, _ = evaluate(wl, d, ns)
    assert g.rel_err(got["t_kernel"], ref["t"]).max() <= tol


def test_beside_the_bounded_head_and_grids(small):
    bounded = gen.make_bounded(0b1000010010)
    d, w = weights("f32", 16, 96)
    ns = len(small.specs["peak_flops"])
    ref = gated_oracle(small, w, 16, False, ns, bounded=bounded)
    got, _ = evaluate(small, d, ns, bounded=bounded)
    assert g.rel_err(got["eta"], ref["eta"]).max() <= REL
    grid = gen.make_grid((1 << NFAM) - 1)
    ref = gated_oracle(small, w, 16, False, ns, grid=grid)
    got, _ = evaluate(small, d, ns, grid=grid)
    off = g.rel_err(got["eta"], ref["eta"])
    # (a query within rounding of the box or of a cell face may be routed either way)
    assert (off <= 1e-4).mean() >= 0.999


@pytest.mark.parametrize("prec", ["f32", "bf16"])
@pytest.mark.parametrize("inp", [16, 32])
@pytest.mark.parametrize("which", ["dense", "moe"])
def test_feature_rows(prec, inp, which):
    """Every pair's features and roofline in the documented order; fp32 features
    within 2^-20 of size 1 (a few units of the hardware's logarithms and
    reciprocals), bf16 ones within half a step more."""
    import torch
    wl = gen.config1(0, 8) if which == "dense" else gen.config3(0, 3)
    di = abi.DeviceInputs(wl)
    r = fit.feature_rows_of(di, inp, prec)
    torch.cuda.synchronize()
    abi.ks_device_status(di.ws_ptr, di.ws_bytes, abi.current_stream())
    cnt = o.kernel_counts(wl.desc)
    ks = o.effective_k(wl.desc, np.arange(wl.desc.n_rows))
    x, roof = r.x.double().cpu().numpy(), r.t_roof.double().cpu().numpy()
    off = [int(v) for v in wl.desc.fam_off]
    assert r.fam_off == [di.n_specs * v for v in off]
    for s in range(di.n_specs):
        sp = o.spec_at(wl.specs, s)
        rf = o.roofline(cnt["F"], cnt["Bt"], cnt["B"], sp)
        want = o.features(cnt, wl.desc.n, ks, rf, sp, inp)
        for f in range(NFAM):
            n = off[f + 1] - off[f]
            at = slice(di.n_specs * off[f] + s * n, di.n_specs * off[f] + (s + 1) * n)
            rec = slice(off[f], off[f + 1])
            half = 2.0 ** -8 if prec == "bf16" else 0.0
            assert (np.abs(x[at] - want[rec]) <= 2.0 ** -20 + half * np.abs(want[rec])).all(), (s, f)
            if n:
                assert g.rel_err(roof[at], rf["t_roof"][rec]).max() <= 1e-6


@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_feature_rows_stride(prec):
    """A row stride that leaves rows unaligned: the same values, nothing between."""
    import torch
    wl = gen.config1(0, 2)
    di = abi.DeviceInputs(wl)
    want = fit.feature_rows_of(di, 16, prec)
    n = di.n_specs * wl.desc.n_rows
    x = torch.full((n, 19), -5.0, dtype=want.x.dtype, device="cuda")
    abi.ks_features(di.desc, di.specs_ptr, di.n_specs, 16, abi.KS_BF16 if prec == "bf16" else abi.KS_F32, x.data_ptr(), 19,
                    None, di.ws_ptr, di.ws_bytes, abi.current_stream())
    torch.cuda.synchronize()
    assert (x[:, :16] == want.x).all() and (x[:, 16:].float() == -5).all()


def test_feature_rows_of_bad_records():
    """A record whose step is out of range gets zeros and raises the flag."""
    import torch
    wl = gen.config1(0, 4)
    di = abi.DeviceInputs(wl)
    want = fit.feature_rows_of(di, 16)
    last = int(wl.desc.fam_off[1]) - 1
    di.t["step"][last] = 1 << 20
    got = fit.feature_rows_of(di, 16)
    torch.cuda.synchronize()
    with pytest.raises(abi.KsError):
        abi.ks_device_status(di.ws_ptr, di.ws_bytes, abi.current_stream())
    n = int(wl.desc.fam_off[1])
    bad = torch.zeros(len(want.x), dtype=torch.bool, device="cuda")
    bad[[s * n + last for s in range(di.n_specs)]] = True
    assert (got.x[bad] == 0).all() and (got.t_roof[bad] == 0).all()
    assert (got.x[~bad] == want.x[~bad]).all()


def test_empty_records():
    import torch
    wl = gen.config1(0, 2)
    di = abi.DeviceInputs(wl)
    for f in range(NFAM + 1):
        di.desc.fam_off[f] = 0
    di.desc.n_rows = 0
    abi.ks_features(di.desc, di.specs_ptr, di.n_specs, 16, 0, None, 16, None, di.ws_ptr, di.ws_bytes, abi.current_stream())
    torch.cuda.synchronize()


@pytest.mark.parametrize("prec,bits", [("f32", 32), ("bf16", 8)])
def test_from_measured_times_to_priced_steps(prec, bits):
    """Feature rows, loss, gradients and AdamW as a fit uses them, then the
    evaluation with the fitted heads: each step's loss and gradients are the oracle's
    for the parameters it started from, the parameters move as the oracle moves them,
    and the evaluation's eta is the fitted block's on the same rows.  A tenth of the
    kernels was never measured."""
    import torch
    wl = gen.config1(0, 6)
    di = abi.DeviceInputs(wl)
    r = fit.feature_rows_of(di, 16, prec)
    rng = torch.Generator().manual_seed(3)
    t = r.t_roof * (1 + torch.exp(0.5 * torch.randn(len(r.t_roof), generator=rng)).cuda())
    eta = t / r.t_roof
    eta[::10] = float("nan")
    data = fit.Measurements(r.x, r.fam_off, eta, None, 1.0)
    ft = fit.GatedFit(16, 64, prec, seed=4, state_bits=bits, weight_decay=0.01)
    x, e = r.x.double().cpu().numpy(), eta.double().cpu().numpy()
    for step in range(1, 4):
        before = {k: v.double().cpu().numpy() for k, v in ft.param.items()}
        read = {k: v.double().cpu().numpy() for k, v in ft.weights.items()}
        old = {}
        for k, st in ft.state.items():
            flat = {n: st[n].float().cpu().numpy().reshape(-1).astype(np.float64) for n in ("m", "v")}
            if bits == 8:
                flat = {n: of.decode(flat[n], st[n + "_exp"].cpu().numpy(), len(flat[n])) for n in ("m", "v")}
            old[k] = flat
        loss = ft.step(data).double().cpu().numpy()
        torch.cuda.synchronize()
        grad = {k: v.double().cpu().numpy() for k, v in ft.grad.items()}
        for f in range(NFAM):
            rr = slice(r.fam_off[f], r.fam_off[f + 1])
            if rr.start == rr.stop:
                continue
            z, k = of.block(x[rr], read["w1"][f], read["w2"][f], read["w3"][f], read["b3"][f])
            want, dz = of.eta_loss(z, e[rr], None, 1.0)
            val, _ = of.gradients(x[rr], read["w1"][f], read["w2"][f], read["w3"][f], dz, k, 64)
            assert abs(loss[f] - want) <= 1e-5 * want
            for key in ("w1", "w2", "w3", "b3"):
                assert np.linalg.norm(grad[key][f] - val[key]) <= 2e-5 * np.linalg.norm(val[key]), (step, f, key)
        for key, p0 in before.items():
            m, v = of.moments32(old[key]["m"], old[key]["v"], grad[key].reshape(-1), 1.0, 0.9, 0.999)
            want = of.step(p0.reshape(-1), m, v, 3e-3, 0.01 if key in ("w1", "w2") else 0.0, 0.9, 0.999, 1e-8, step)
            got = ft.param[key].double().cpu().numpy().reshape(-1)
            assert np.abs(got - want).max() <= 1e-6
            if prec == "bf16":
                assert (ft.weights[key] == ft.param[key].bfloat16()).all()
    # the evaluation reads the weights the fit moved
    ko_t, ko = abi.kernel_outputs(wl.desc.n_rows, di.n_specs, counts=False)
    abi.ks_eval_kernels(di.desc, di.specs_ptr, di.n_specs, ft.heads, ko, di.ws_ptr, di.ws_bytes, abi.current_stream())
    z = torch.empty(len(r.x), device="cuda")
    abi.ks_gated_forward(ft.heads, data.rows, z.data_ptr(), abi.current_stream())
    torch.cuda.synchronize()
    off = [int(v) for v in wl.desc.fam_off]
    zs = torch.cat([z[r.fam_off[f]:r.fam_off[f + 1]].view(di.n_specs, -1) for f in range(NFAM)], 1)
    want = 1 + torch.exp(-zs.double())
    assert (((ko_t["eta"].double() - want) / want).abs().max().item()) <= 1e-6
    assert off[-1] == wl.desc.n_rows


def test_captured_fit():
    """A captured step replayed trains on: the same parameters as eager steps."""
    import torch
    wl = gen.config1(0, 4)
    di = abi.DeviceInputs(wl)
    r = fit.feature_rows_of(di, 16)
    eta = 1 + torch.rand(len(r.x), generator=torch.Generator().manual_seed(3)).cuda()
    data = fit.Measurements(r.x, r.fam_off, eta)
    eager, graphed = fit.GatedFit(16, 64, seed=2), fit.GatedFit(16, 64, seed=2)
    eager.step(data)
    graphed.step(data)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        graphed.step(data)
    for i in range(5):
        eager.step(data)
        gr.replay()
        torch.cuda.synchronize()
        for k in eager.param:
            assert (eager.param[k] == graphed.param[k]).all(), (i, k)
    assert int(graphed.count) == 6


def test_captured_fit_beside_larger_rows():
    """A captured step keeps its workspace when the same fit then takes more rows:
    replays in turn with eager steps on the larger set train as eager steps do."""
    import torch
    few, many = (abi.DeviceInputs(gen.config1(0, n)) for n in (2, 12))
    sets = []
    for i, di in enumerate((few, many)):
        r = fit.feature_rows_of(di, 16)
        eta = 1 + torch.rand(len(r.x), generator=torch.Generator().manual_seed(i)).cuda()
        sets.append(fit.Measurements(r.x, r.fam_off, eta))
    eager, graphed = fit.GatedFit(16, 64, seed=2), fit.GatedFit(16, 64, seed=2)
    eager.step(sets[0])
    graphed.step(sets[0])
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        graphed.step(sets[0])
    first = graphed.ws.data_ptr()
    for i in range(4):
        eager.step(sets[1])
        graphed.step(sets[1])
        assert graphed.ws.data_ptr() != first
        other = torch.full((len(sets[0].x), 64), float("nan"), device="cuda")   # takes memory that is free
        eager.step(sets[0])
        gr.replay()
        torch.cuda.synchronize()
        assert other.isnan().all()
        for k in eager.param:
            assert (eager.param[k] == graphed.param[k]).all(), (i, k)


def test_fit_refuses_rows_of_another_kind():
    import torch
    ft = fit.GatedFit(16, 32, "bf16")
    off = [0] + [6] * NFAM
    eta = torch.ones(6, device="cuda")
    for x in (torch.zeros(6, 16, device="cuda"), torch.zeros(6, 40, device="cuda").bfloat16()[:, :32]):
        with pytest.raises(ValueError):
            ft.step(fit.Measurements(x, off, eta))
    with pytest.raises(ValueError):
        fit.Measurements(torch.zeros(6, 16, device="cuda"), off, eta.cpu())
    assert int(ft.count) == 0


def test_simulation_with_gated_heads():
    """The serving simulation takes gated heads like any others: its first step's
    latency is the evaluation's."""
    import torch
    d, _ = weights("f32", 16, 64)
    hd = abi.gated_heads(d["w1"], d["w2"], d["w3"], d["b3"])
    host = abi.ks_host(4e-6, 1.5e-3, 2.5e-3, 3e-4, 1.04)
    sched = abi.ks_sched(16, 2048, 16, 0, 4000)
    spec = {k: v[0] for k, v in gen.config1(0, 1).specs.items()}
    req = {"arrival": np.zeros(5), "prompt": np.array([100, 200, 300, 50, 7]), "output": np.array([3, 1, 4, 2, 5])}
    res = abi.simulate(gen.LLAMA7B, spec, hd, host, sched, req)
    again = abi.simulate(gen.LLAMA7B, spec, hd, host, sched, req)
    torch.cuda.synchronize()
    assert (res["state"] == 2).all() and res["n_steps"] == again["n_steps"]
    np.testing.assert_array_equal(res["step_latency"], again["step_latency"])
    assert (res["step_latency"] > 0).all()


def test_allocation_free_evaluation(small):
    """ks_eval_steps_static takes gated heads: the results of ks_eval_steps."""
    import torch
    d, _ = weights("bf16", 32, 200)
    ns = len(small.specs["peak_flops"])
    want, _ = evaluate(small, d, ns, per_pair=False)
    di = abi.DeviceInputs(small)
    so_t, so = abi.step_outputs(small.desc.n_steps, ns)
    flags = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    abi.ks_eval_steps_static(di.desc, di.steps, di.specs_ptr, ns, abi.gated_heads(d["w1"], d["w2"], d["w3"], d["b3"]),
                             di.host, so, None, flags.data_ptr(), abi.current_stream())
    torch.cuda.synchronize()
    assert int(flags) == 0
    for k in ("t_body", "t_step"):
        np.testing.assert_array_equal(so_t[k].cpu().numpy(), want[k])
