"""Gated fp32 heads at the top of fp32 (GPU): 3.4e38 lies above the largest bfloat16 and
below the largest fp32 number, so its leading piece may not be the nearest bfloat16,
which is infinity.  Tolerances are the oracle's bounds on fp32 arithmetic."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import ks_oracle as o
from tests import gpu_helpers as g
from tests.test_gated_eval_gpu import REL, evaluate, gated_oracle, weights
from tests.test_gated_gpu import backward, check_forward, check_grads, forward, make
from workload import gen

pytestmark = pytest.mark.gpu
TOP = 3.4e38


@pytest.mark.parametrize("inp,hid", [(16, 70), (32, 40), (32, 160)])
@pytest.mark.parametrize("which", ["rows", "weights"])
def test_largest_finite_numbers(inp, hid, which):
    """Features or weights of 3.4e38, the other factor near 2^-100: z is finite in fp32, and
    so are the gradients for a dz of 2^-60."""
    import torch
    d, h, off = make(300, "f32", inp, hid)
    sign = torch.where(torch.arange(300) % 3 == 0, -1.0, 1.0)
    if which == "rows":
        d["x"][:, 3] = TOP * sign.cuda()
        for k in ("w1", "w2"):
            d[k][:, :, 3] *= 2.0 ** -100
    else:
        d["x"][:, 3] *= 2.0 ** -100 * sign.cuda()
        for k in ("w1", "w2"):
            d[k][:, :, 3] = torch.where(d[k][:, :, 3] < 0, -TOP, TOP)
    for k in ("x", "w1", "w2"):
        h[k] = d[k].double().cpu().numpy()
    z = forward(d, off)
    assert np.isfinite(z).all()
    check_forward(d, h, off, z)
    dz = torch.randn(300, generator=torch.Generator().manual_seed(5))
    if which == "rows":
        got = backward(d, off, (dz * 2.0 ** -60).cuda())
        assert all(np.isfinite(v).all() for v in got.values())
        check_grads(h, off, (dz * 2.0 ** -60).numpy(), got, "f32")
        return
    # The weights' gradients are sums of dz x: 2^-60 2^-100 is below fp32, where they are
    # not promised (from 2^-102 up), so they are taken for a dz of 1, where the rows' are
    # past fp32 (2^28 3.4e38); the rows' for a dz of 2^-60.
    got = backward(d, off, dz.cuda(), dx=False)
    check_grads(h, off, dz.numpy(), got, "f32", dx=False)
    got["x"] = backward(d, off, (dz * 2.0 ** -60).cuda())["x"]
    assert all(np.isfinite(v).all() for v in got.values())
    small = {k: v * 2.0 ** -60 for k, v in got.items() if k != "x"}   # (exact)
    check_grads(h, off, (dz * 2.0 ** -60).numpy(), {**small, "x": got["x"]}, "f32")


def test_evaluation_with_the_largest_finite_weight():
    """(A z that is no number gave eta = NaN and the floor as latency.)"""
    wl = gen.config1(0, 4)
    d, _ = weights("f32", 16, 64)
    d["w1"][:, 0, :] = 0.0
    d["w1"][:, 0, 15] = TOP       # (feature 15 is 1)
    d["w2"][:, 0, :] *= 2.0 ** -100
    d["w3"][:, 0] *= 2.0 ** -28
    w = {k: v.double().cpu().numpy() for k, v in d.items()}
    ns = len(wl.specs["peak_flops"])
    ref = gated_oracle(wl, w, 16, False, ns)
    assert np.isfinite(ref["eta"]).all()
    got, _ = evaluate(wl, d, ns)
    assert g.rel_err(got["eta"], ref["eta"]).max() <= REL
    assert g.rel_err(got["t_kernel"], ref["t"]).max() <= REL
    rs = o.eval_steps(wl.desc, wl.steps, wl.specs, wl.host, spec_ids=range(ns), kern=ref)
    assert g.rel_err(got["t_step"], rs["t_step"]).max() <= REL
