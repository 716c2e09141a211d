"""Learned columns without a GPU: the oracle against published vectors, differences and
counts; struct layouts; refused calls (fake device addresses: nothing is read)."""
from __future__ import annotations

import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import ks_columns as o
from oracle import ks_fit as of
from paper_2606_28565_amd import abi

NFAM = abi.NFAM
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = "/opt/rocm/include"
A = 0x100000          # fake device addresses, 1 GiB apart
GIB = 1 << 30


def at(i, shift=0):
    return A + i * GIB + shift


# ------------------------------------------------------------------ the oracle
@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((o.M32,) * 4, (o.M32,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_philox_gives_the_published_words(counter, key, want):
    assert tuple(o.philox(counter, key)) == want


def test_many_blocks_are_each_ones():
    rng = np.random.default_rng(1)
    block = [0, 1, 7, (1 << 32) - 1, 1 << 32, (1 << 51) + 12345]
    seed, step, site = int(rng.integers(1 << 62)), 77, 3
    got = o.philox_many(block, step, site, seed)
    for i, b in enumerate(block):
        assert tuple(got[i]) == tuple(o.philox((b & o.M32, b >> 32, step, site), (seed & o.M32, seed >> 32)))


@pytest.mark.parametrize("p", [0.0, 0.1, 0.25, 0.9, 1.0])
def test_share_dropped(p):
    """Within five deviations of p's step of 2^-16; the rest is lifted to the same mean."""
    n, cols = 2000, 41
    k, up = o.keep(np.arange(n), cols, p, 5)
    t = o.least(p) / 65536
    assert abs(k.mean() - (1 - t)) <= 5 * np.sqrt(t * (1 - t) / (n * cols))
    assert p == 1.0 or up * (1 - t) == 1.0


def test_a_row_drops_the_same_in_any_matrix_of_its_width():
    whole = o.keep(np.arange(50), 19, 0.5, 9, 2, 4)[0]
    assert (o.keep([7, 30], 19, 0.5, 9, 2, 4)[0] == whole[[7, 30]]).all()
    assert (o.keep(np.arange(50), 24, 0.5, 9, 2, 4)[0][:, :19] == whole).all()


@pytest.mark.parametrize("dropout", [None, (0.3, 11, 1, 2)])
def test_gradient_against_differences(dropout):
    """The lookup is linear in the table, so differences are exact up to rounding."""
    rng = np.random.default_rng(3)
    ids = np.array([2, 0, 2, -1, 3, 2, 9, 0])
    table, dy = rng.standard_normal((5, 11)), rng.standard_normal((8, 11))
    grad, bound = o.embed_back(ids, 5, dy, 1.5, dropout)
    for v in range(5):
        for c in range(11):
            up, down = table.copy(), table.copy()
            up[v, c] += 0.5
            down[v, c] -= 0.5
            diff = (dy * (o.embed(up, 1.5, ids, dropout) - o.embed(down, 1.5, ids, dropout))).sum()
            assert abs(diff - grad[v, c]) < 1e-13
    assert (bound[1] == 0).all() and (grad[1] == 0).all() and (grad[4] == 0).all()


def test_order():
    row, ids, off = o.order([3, 1, -1, 3, 0, 4, 1], 4)
    assert row.tolist() == [4, 1, 6, 0, 3, 2, 5] and ids.tolist() == [0, 1, 1, 3, 3, 4, 4] and off.tolist() == [0, 1, 3, 3, 5]


@pytest.mark.parametrize("huber", [float("inf"), 0.3])
def test_dz_against_differences(huber):
    rng = np.random.default_rng(5)
    z, eta = rng.standard_normal(20), 1 + np.exp(rng.standard_normal(20))
    eta[3], eta[4] = np.nan, 0.0
    w = rng.random(20) + 0.5
    w[5] = 0
    _, dz = of.eta_loss(z, eta, w, huber)
    for i in range(20):
        h = 1e-6
        up, down = z.copy(), z.copy()
        up[i] += h
        down[i] -= h
        diff = (of.eta_loss(up, eta, w, huber)[0] - of.eta_loss(down, eta, w, huber)[0]) / (2 * h)
        assert abs(diff - dz[i]) < 1e-8
    assert (dz[[3, 4, 5]] == 0).all()


# ------------------------------------------------------------------ layouts
def test_struct_layout_matches_header(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ is not available")
    structs = {"ks_matrix": abi.ks_matrix, "ks_drop": abi.ks_drop, "ks_id_order": abi.ks_id_order}
    lines = ["#include <cstddef>", "#include <cstdio>", '#include "ks.h"', "int main() {"]
    for name, s in structs.items():
        lines.append(f'std::printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'std::printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in s._fields_]
    src = tmp_path / "layout.cpp"
    src.write_text("\n".join(lines + ["}"]))
    exe = str(tmp_path / "layout")
    subprocess.run(["g++", "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I", f"{ROOT}/include", str(src), "-o", exe], check=True)
    got = dict(line.split() for line in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, s in structs.items():
        assert int(got[name]) == C.sizeof(s)
        for f, _ in s._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(s, f).offset


# ------------------------------------------------------------------ refused calls
BIG = 1 << 40


def mat(p=at(0), n_rows=100, n_cols=20, ld=24, type=abi.KS_F32):
    return abi.ks_matrix(p, n_rows, n_cols, ld, type)


def dropping(p=0.1, step_dev=None):
    return abi.ks_drop(p, 1, 2, 3, step_dev)


def sorted_ids(n_rows=100, n_ids=50, row=at(4), id=at(5), off=at(6)):
    return abi.ks_id_order(n_rows, n_ids, row, id, off)


def target(eta=at(10), weight=None, huber=1.0):
    return abi.ks_eta_target(eta, weight, huber)


def offsets(n=100):
    return abi.family_offsets([0] * 4 + [n] * (NFAM - 3))


def dropout(drop=dropping(), x=mat(), y=mat(at(1))):
    return abi.ks_dropout(drop, x, y, None, check=False)


def embed(table=mat(n_rows=50), scale=1.0, ids=at(2), drop=None, y=mat(at(1))):
    return abi.ks_embed(table, scale, ids, drop, y, None, check=False)


def sort(ids=at(2), order=sorted_ids(), ws=at(7), size=BIG):
    return abi.ks_embed_sort(ids, order, ws, size, None, check=False)


def backward(order=sorted_ids(), scale=1.0, dy=mat(), drop=None, grad=mat(at(1), 50), ws=at(7), size=BIG):
    return abi.ks_embed_backward(order, scale, dy, drop, grad, ws, size, None, check=False)


def eta_loss(off=offsets(), z=at(8), t=target(), loss=at(11), dz=at(12), ws=at(13), size=BIG):
    return abi.ks_eta_loss(off, z, t, loss, dz, ws, size, None, check=False)


BAD_MATRIX = [(dict(type=2), abi.KS_EINVAL), (dict(n_rows=-1), abi.KS_ERANGE), (dict(n_rows=1 << 31), abi.KS_ERANGE),
              (dict(n_cols=0), abi.KS_ERANGE), (dict(n_cols=-1), abi.KS_ERANGE), (dict(n_cols=(1 << 20) + 1, ld=1 << 21), abi.KS_ERANGE),
              (dict(ld=19), abi.KS_EINVAL), (dict(ld=(1 << 20) + 1), abi.KS_EINVAL), (dict(p=None), abi.KS_EINVAL),
              (dict(p=at(0, 2)), abi.KS_EINVAL), (dict(type=abi.KS_BF16, p=at(0, 1)), abi.KS_EINVAL)]


@pytest.mark.parametrize("bad,status", BAD_MATRIX)
def test_bad_matrices(bad, status):
    got = [dropout(x=mat(**bad)), dropout(y=mat(**bad)), embed(table=mat(**bad)), embed(y=mat(**bad)),
           backward(dy=mat(**bad)), backward(grad=mat(**bad))]
    assert got == [status] * 6
    assert abi.ks_last_error()


@pytest.mark.parametrize("p", [-0.1, 1.0001, float("nan"), float("inf")])
def test_bad_share(p):
    assert [dropout(drop=dropping(p)), embed(drop=dropping(p)), backward(drop=dropping(p))] == [abi.KS_EINVAL] * 3


def test_bad_counter():
    d = dropping(step_dev=at(9, 2))
    assert [dropout(drop=d), embed(drop=d), backward(drop=d)] == [abi.KS_EINVAL] * 3


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), 1e39])
def test_bad_scale(scale):
    assert [embed(scale=scale), backward(scale=scale)] == [abi.KS_EINVAL] * 2


def test_scale_that_overflows_with_dropout():
    assert [f(scale=2e38, drop=dropping(0.5)) for f in (embed, backward)] == [abi.KS_EINVAL] * 2


def test_shapes_that_do_not_go_together():
    assert dropout(drop=None) == abi.KS_EINVAL
    for other in (dict(n_rows=99), dict(n_cols=21), dict(type=abi.KS_BF16)):
        assert dropout(y=mat(at(1), **other)) == abi.KS_EINVAL
    assert embed(y=mat(at(1), n_cols=21)) == abi.KS_EINVAL
    for bad in (dict(dy=mat(n_rows=99)), dict(dy=mat(n_cols=21)), dict(grad=mat(at(1), 51)), dict(grad=mat(at(1), 50, 19)),
                dict(grad=mat(at(1), 50, type=abi.KS_BF16))):
        assert backward(**bad) == abi.KS_EINVAL


@pytest.mark.parametrize("ids", [None, at(2, 2)])
def test_bad_ids(ids):
    assert [embed(ids=ids), sort(ids=ids)] == [abi.KS_EINVAL] * 2


BAD_ORDER = [(dict(n_rows=-1), abi.KS_ERANGE), (dict(n_rows=1 << 31), abi.KS_ERANGE), (dict(n_ids=0), abi.KS_ERANGE),
             (dict(n_ids=1 << 31), abi.KS_ERANGE), (dict(row=None), abi.KS_EINVAL), (dict(id=None), abi.KS_EINVAL),
             (dict(off=None), abi.KS_EINVAL), (dict(row=at(4, 2)), abi.KS_EINVAL), (dict(off=at(6, 1)), abi.KS_EINVAL)]


@pytest.mark.parametrize("bad,status", BAD_ORDER)
def test_bad_orders(bad, status):
    assert [sort(order=sorted_ids(**bad)), backward(order=sorted_ids(**bad))] == [status] * 2
    if "n_rows" in bad or "n_ids" in bad:
        assert abi.ks_embed_sort_workspace_bytes(sorted_ids(**bad)) == 0
        assert abi.ks_embed_backward_workspace_bytes(sorted_ids(**bad), mat()) == 0


def test_workspaces():
    """Sizes alone are read; a smaller, missing or misaligned workspace is refused."""
    bare = abi.ks_id_order(100, 50, None, None, None)
    need = abi.ks_embed_sort_workspace_bytes(bare)
    assert need > 0 and need % 256 == 0
    assert sort(size=need - 1) == sort(ws=None) == sort(ws=at(7, 128)) == abi.KS_EWORKSPACE
    need = abi.ks_embed_backward_workspace_bytes(bare, mat(None))
    assert need > 0 and need % 256 == 0
    assert backward(size=need - 1) == backward(ws=None) == backward(ws=at(7, 128)) == abi.KS_EWORKSPACE
    assert abi.ks_embed_backward_workspace_bytes(bare, mat(type=5)) == 0
    need = abi.ks_eta_loss_workspace_bytes(offsets())
    assert need > 0 and need % 256 == 0
    assert eta_loss(size=need - 1) == eta_loss(ws=None) == eta_loss(ws=at(13, 128)) == abi.KS_EWORKSPACE
    lib = abi.load()
    assert lib.ks_embed_sort_workspace_bytes(None) == lib.ks_embed_backward_workspace_bytes(None, C.byref(mat())) == 0
    assert lib.ks_embed_backward_workspace_bytes(C.byref(bare), None) == lib.ks_eta_loss_workspace_bytes(None) == 0


@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (129, 1, 1), (2_000_003, 67, 16), (1 << 24, 1 << 20, 67), ((1 << 31) - 1, (1 << 31) - 1, 16)])
def test_workspaces_stay_small(n, v, d):
    """The order's by its keys and their digits' counts, the gradient's by an eighth of dy's
    elements."""
    order = abi.ks_id_order(n, v, None, None, None)
    assert abi.ks_embed_sort_workspace_bytes(order) <= 8 * n + 4 * 1024 * (4096 + 2) + 1024
    assert abi.ks_embed_backward_workspace_bytes(order, mat(n_rows=n, n_cols=d, ld=d)) <= 2 * 4 * (8 * -(-d // 8)) * (n / 64 + 1) + 512


def test_null_structs():
    lib = abi.load()
    m, s, d = C.byref(mat()), C.byref(sorted_ids()), C.byref(dropping())
    assert lib.ks_dropout(d, None, m, None) == lib.ks_dropout(d, m, None, None) == abi.KS_EINVAL
    assert lib.ks_embed(None, 1.0, at(2), None, m, None) == lib.ks_embed(m, 1.0, at(2), None, None, None) == abi.KS_EINVAL
    assert lib.ks_embed_sort(at(2), None, at(7), BIG, None) == abi.KS_EINVAL
    assert lib.ks_embed_backward(None, 1.0, m, None, m, at(7), BIG, None) == abi.KS_EINVAL
    assert lib.ks_embed_backward(s, 1.0, None, None, m, at(7), BIG, None) == abi.KS_EINVAL
    assert lib.ks_embed_backward(s, 1.0, m, None, None, at(7), BIG, None) == abi.KS_EINVAL
    assert lib.ks_eta_loss(None, at(8), C.byref(target()), at(11), at(12), at(13), BIG, None) == abi.KS_EINVAL
    assert lib.ks_eta_loss(offsets(), at(8), None, at(11), at(12), at(13), BIG, None) == abi.KS_EINVAL


def test_empty_calls_need_nothing():
    assert dropout(x=mat(None, 0), y=mat(None, 0)) == abi.KS_OK
    assert embed(ids=None, y=mat(None, 0)) == abi.KS_OK
    assert embed(table=mat(None, 0), ids=None, y=mat(None, 0)) == abi.KS_OK


def test_what_is_written_may_not_lie_over_what_is_read():
    # the last element of 100 rows of 20 every 24 ends at 4 (99 * 24 + 20)
    end = 4 * (99 * 24 + 20)
    assert dropout(y=mat(at(0, 4))) == dropout(y=mat(at(0, 4 * 23))) == dropout(y=mat(at(0), ld=25)) == abi.KS_EINVAL
    assert dropout(y=mat(at(0, -end + 4))) == abi.KS_EINVAL
    # columns of one buffer that meet in the next row
    assert dropout(x=mat(n_cols=8), y=mat(at(0, 4 * 20), n_cols=8)) == abi.KS_EINVAL
    assert dropout(drop=dropping(step_dev=at(1, 40))) == abi.KS_EINVAL
    assert embed(table=mat(at(1, 96), 50)) == embed(ids=at(1, end - 4)) == embed(ids=at(1, -396)) == abi.KS_EINVAL
    assert embed(drop=dropping(step_dev=at(1, 40))) == abi.KS_EINVAL
    for bad in (dict(ids=at(4)), dict(ids=at(6, 4 * 50)), dict(ws=at(2)), dict(ws=at(5)), dict(order=sorted_ids(id=at(4, 396))),
                dict(order=sorted_ids(off=at(5, -200)))):
        assert sort(**bad) == abi.KS_EINVAL, bad
    for bad in (dict(grad=mat(at(0, 4), 50)), dict(grad=mat(at(4), 50)), dict(grad=mat(at(5), 50)), dict(grad=mat(at(6), 50)),
                dict(drop=dropping(step_dev=at(1)))):
        assert backward(**bad) == abi.KS_EINVAL, bad
    many = dict(order=sorted_ids(5000), dy=mat(n_rows=5000))   # (a workspace that is used)
    for ws in (at(0), at(1), at(4), at(5), at(6)):
        assert backward(ws=ws, **many) == abi.KS_EINVAL, ws
    for bad in (dict(dz=at(8, 4)), dict(dz=at(10)), dict(loss=at(8)), dict(loss=at(12)), dict(ws=at(8)), dict(ws=at(10)), dict(ws=at(12)),
                dict(ws=at(11)), dict(t=target(weight=at(12)))):
        assert eta_loss(**bad) == abi.KS_EINVAL, bad


@pytest.mark.parametrize("off", [[1] + [100] * NFAM, [0, 5, 4] + [100] * (NFAM - 2), [0] * NFAM + [-1]])
def test_bad_offsets(off):
    assert eta_loss(off=abi.family_offsets(off)) == abi.KS_EINVAL
    assert abi.ks_eta_loss_workspace_bytes(abi.family_offsets(off)) == 0


def test_bad_losses():
    assert eta_loss(off=offsets(1 << 31)) == abi.KS_ERANGE
    for bad in (dict(z=None), dict(loss=None), dict(dz=None), dict(z=at(8, 2)), dict(dz=at(12, 1)), dict(loss=at(11, 2)),
                dict(t=target(None)), dict(t=target(at(10, 2))), dict(t=target(weight=at(3, 2))), dict(t=target(huber=0.0)),
                dict(t=target(huber=-1.0)), dict(t=target(huber=float("nan"))), dict(t=target(huber=1e-60))):
        assert eta_loss(**bad) == abi.KS_EINVAL, bad


# ------------------------------------------------------------------ the binding
def test_binding_refuses_what_it_cannot_describe():
    import torch
    x = torch.zeros(6, 8)
    with pytest.raises(ValueError):
        abi.matrix(x.double())
    with pytest.raises(ValueError):
        abi.matrix(x.t())
    with pytest.raises(ValueError):
        abi.matrix(x[0])
    with pytest.raises(ValueError):
        abi.matrix(x[:1].expand(6, 8))
    with pytest.raises(ValueError):
        abi.drop(0.1, 1, step_dev=torch.zeros(1))
    with pytest.raises(ValueError):
        abi.ks_eta_loss(offsets(7), at(8), abi.eta_target(torch.ones(6)), at(11), at(12), at(13), BIG, None)


def test_tensors_on_the_cpu():
    import torch
    m, s = abi.matrix(torch.zeros(6, 8)), abi.id_order(6, 4, "cpu")
    for call in (lambda: abi.ks_dropout(dropping(), m, m, None), lambda: abi.ks_embed(m, 1.0, at(2), None, mat(), None),
                 lambda: abi.ks_embed_sort(at(2), s, at(7), BIG, None),
                 lambda: abi.ks_embed_backward(sorted_ids(), 1.0, m, None, mat(), at(7), BIG, None),
                 lambda: abi.ks_dropout(abi.drop(0.1, 1, step_dev=torch.zeros(1, dtype=torch.int32)), mat(), mat(), None)):
        with pytest.raises(ValueError):
            call()


def test_matrices_of_views():
    import torch
    buf = torch.zeros(5, 32)
    m = abi.matrix(buf[:, 16:])
    assert (m.p, m.n_rows, m.n_cols, m.ld, m.type) == (buf.data_ptr() + 64, 5, 16, 32, abi.KS_F32)
    m = abi.matrix(buf[::2, 3:7].bfloat16())
    assert (m.n_rows, m.n_cols, m.ld, m.type) == (3, 4, 4, abi.KS_BF16)
    m = abi.matrix(buf[::2, 3:7])
    assert (m.n_rows, m.n_cols, m.ld) == (3, 4, 64)
    assert abi.matrix(buf[:0]).p is None and abi.matrix(buf[1:2, :4]).ld == 4


# ------------------------------------------------------------------ the fit's refusals and its chain
def test_fit_refuses_rows_that_do_not_go_together():
    import torch
    from paper_2606_28565_amd import fit
    x, eta = torch.zeros(6, 16), torch.ones(6)
    off = [0] * NFAM + [6]
    ids = torch.zeros(6, dtype=torch.int32)
    for bad in (dict(ids=ids.long(), categories=2), dict(ids=ids[:5], categories=2), dict(ids=ids, categories=0),
                dict(ids=torch.zeros(12, dtype=torch.int32)[::2], categories=2)):
        with pytest.raises(ValueError):
            fit.Measurements(x, off, eta, **bad)
    with pytest.raises(ValueError):
        fit.Measurements(torch.zeros(6, 32), off, eta, ids=ids, categories=2)
    for bad in (dict(dropout=0.1), dict(categories=-1), dict(categories=2, dropout=1.0), dict(feature_dropout=-0.1)):
        with pytest.raises(ValueError):
            fit.GatedFit(16, 8, device="cpu", **bad)
    plain, learned = fit.GatedFit(32, 8, device="cpu"), fit.GatedFit(16, 8, device="cpu", categories=2)
    assert learned.block.in_dim == 32 and plain.heads is plain.block
    with pytest.raises(ValueError):
        learned.heads
    with pytest.raises(ValueError):
        learned.workspace(fit.Measurements(torch.zeros(6, 32), off, eta))
    with pytest.raises(ValueError):
        plain.heads_for(0)
    for category in (-1, 2):
        with pytest.raises(ValueError):
            learned.heads_for(category)


def test_heads_of_a_category_on_the_cpu():
    """W[:, 16:] e goes to column 15, None leaves the 16 features' weights."""
    import torch
    from paper_2606_28565_amd import fit
    ft = fit.GatedFit(16, 8, device="cpu", categories=3, precision="bf16")
    h = ft.heads_for(1)
    w, e = ft.weights["w2"].float(), ft.weights["table"][1].float()
    want = w[:, :, 15] + (w[:, :, 16:] * e).sum(-1)
    assert torch.equal(h.weights["w2"][:, :, 15], want.bfloat16()) and torch.equal(h.weights["w2"][:, :, :15], ft.weights["w2"][:, :, :15])
    assert torch.equal(ft.heads_for().weights["w1"], ft.weights["w1"][:, :, :16]) and (h.hidden, h.in_dim) == (8, 16)


def test_the_chain_against_differences():
    """The loss by one element of the table at a time, through dropout, lookup, block and
    loss: the gradients that a fit's step goes through."""
    rng = np.random.default_rng(8)
    n, c, hid = 12, 3, 5
    x16, table = rng.random((n, 16)), rng.standard_normal((c, 16)) * 0.3
    w1, w2, w3 = (rng.standard_normal(s) * 0.3 for s in ((hid, 32), (hid, 32), (hid,)))
    ids = rng.integers(-1, c, n)
    eta = 1 + np.exp(rng.standard_normal(n))
    drop = (0.3, 99, 1, 4)

    def chain(table):
        x = np.concatenate([oc_drop, o.embed(table, 1.0, ids, drop)], 1)
        z, k = of.block(x, w1, w2, w3, 0.1)
        loss, dz = of.eta_loss(z, eta, None, 0.4)
        return loss, x, dz, k
    oc_drop = np.concatenate([o.drop(x16[:, :15], 0.2, 99, 0, 4), x16[:, 15:]], 1)
    loss, x, dz, k = chain(table)
    dx = of.gradients(x, w1, w2, w3, dz, k, 1)[0]["x"]
    grad = o.embed_back(ids, c, dx[:, 16:], 1.0, drop)[0]
    for v in range(c):
        for j in range(16):
            up, down = table.copy(), table.copy()
            up[v, j] += 1e-5
            down[v, j] -= 1e-5
            assert abs((chain(up)[0] - chain(down)[0]) / 2e-5 - grad[v, j]) < 1e-8
