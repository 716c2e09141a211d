"""Calls with gated heads that the documentation allows: rows and their gradients as
columns of one buffer, the serving simulation priced by the gated block."""
from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import pytest

from oracle import ks_expand as ox
from oracle import ks_oracle as o
from oracle import ks_sim as osim
from paper_2606_28565_amd import abi
from tests import gpu_helpers as g
from tests.test_gated_eval_gpu import REL, REL_BF16, gated_oracle, weights
from tests.test_gated_gpu import NFAM, check_grads, heads_of, make
from tests.test_sim_gpu import gpu_steps, host_struct, one_spec, replay, sched_struct, spec_row, u32
from workload import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec,inp,ld", [("f32", 16, 32), ("f32", 32, 67), ("bf16", 16, 40), ("bf16", 32, 65)])
def test_rows_and_gradients_as_columns_of_one_buffer(prec, inp, ld):
    """The gradients right behind the rows, up to the next one, vector stores or not."""
    import torch
    n, hid = 700, 40
    d, h, off = make(n, prec, inp, hid)
    buf = torch.full((n, ld), -77.0, dtype=d["x"].dtype, device="cuda")
    x, gx = buf[:, :inp], buf[:, ld - inp:]
    x.copy_(d["x"])
    dz = torch.randn(n, generator=torch.Generator().manual_seed(5))
    dz_d = dz.cuda()
    hd, rows = heads_of(d), abi.feature_rows(x, off)
    out = {k: torch.empty(d[k].shape, device="cuda") for k in ("w1", "w2", "w3", "b3")}
    ws = torch.empty(abi.ks_gated_workspace_bytes(hd, rows), dtype=torch.uint8, device="cuda")
    abi.ks_gated_backward(hd, rows, dz_d.data_ptr(), abi.gated_grad(**out, x=gx), ws.data_ptr(), ws.numel(),
                          abi.current_stream())
    torch.cuda.synchronize()
    assert (x == d["x"]).all() and (buf[:, inp:ld - inp].float() == -77).all()
    got = {k: v.double().cpu().numpy() for k, v in out.items()}
    check_grads(h, off, dz.numpy(), {**got, "x": gx.double().cpu().numpy()}, prec)


def latency(shape, w, inp, bf16):
    """The oracle's latency of a batch's step, every family priced by the gated block."""
    def f(batch, prefill):
        q, hist = [b[0] for b in batch], [b[1] for b in batch]
        e = ox.expand(shape, [0, len(q)], q, [prefill], homogeneous=True)
        d = gen.Desc(e["fam_off"], *(u32(e[k]) for k in ("step", "m", "n", "k", "a", "b")),
                     u32([0, len(q)]), u32(q), u32(hist), u32([]), 2, u32(e["mult"]))
        rec = gen.StepRec(*(u32(e[k]) for k in ("layers", "hidden", "tp", "n_launch")))
        kern = gated_oracle(SimpleNamespace(desc=d, specs=one_spec()), w, inp, bf16, 1)
        return float(o.eval_steps(d, rec, one_spec(), gen.HostConsts(), spec_ids=range(1), kern=kern)["t_step"][0, 0])
    return f


@pytest.mark.parametrize("prec,inp,hid", [("f32", 16, 64), ("bf16", 32, 200)])
def test_simulated_steps_are_the_gated_heads(prec, inp, hid):
    """The batches are those the oracle's scheduler forms, and each step's latency is the
    oracle's of that batch with the gated block in every family."""
    d, w = weights(prec, inp, hid)
    hd = abi.gated_heads(d["w1"], d["w2"], d["w3"], d["b3"])
    cfg = osim.SchedCfg(max_num_seqs=16, max_batched_tokens=1024, block_tokens=16, kv_blocks=4000)
    reqs = gen.make_requests(12, rate=200.0, seed=7, prompt_median=200, output_median=8)
    res = abi.simulate(gen.LLAMA7B, spec_row(), hd, host_struct(), sched_struct(cfg), reqs)
    replay(reqs, cfg, res)
    want = latency(gen.LLAMA7B, w, inp, prec == "bf16")
    tol = REL_BF16 if prec == "bf16" else REL
    assert res["n_steps"] > 5
    for i, step in enumerate(gpu_steps(res)):
        lat = want([(q, hist) for _, q, hist in step], bool(res["step_prefill"][i]))
        assert abs(res["step_latency"][i] - lat) <= tol * lat, i


def test_gated_heads_beside_the_bounded_head_and_grids():
    """Built by gated_heads alone: families on the bounded head or a grid take it, the
    others the gated block, as the oracle has them."""
    import torch
    wl = gen.config1(0, 8)
    ns = len(wl.specs["peak_flops"])
    d, w = weights("f32", 16, 96)
    di = abi.DeviceInputs(wl)
    for bounded, grid, share in ((gen.make_bounded(0b1000010010), None, 1.0), (None, gen.make_grid((1 << NFAM) - 1), 0.999)):
        ref = gated_oracle(wl, w, 16, False, ns, bounded=bounded, grid=grid)
        hd = abi.gated_heads(d["w1"], d["w2"], d["w3"], d["b3"], bounded, grid)
        ko_t, ko = abi.kernel_outputs(wl.desc.n_rows, ns, counts=False)
        abi.ks_eval_kernels(di.desc, di.specs_ptr, ns, hd, ko, di.ws_ptr, di.ws_bytes, abi.current_stream())
        torch.cuda.synchronize()
        off = g.rel_err(ko_t["eta"].cpu().numpy(), ref["eta"])
        # (a grid's query within rounding of the box or of a cell face may go either way)
        assert (off <= (REL if grid is None else 1e-4)).mean() >= share
