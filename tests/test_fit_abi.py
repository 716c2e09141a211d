"""Fitting entry points, CPU only: struct layouts, refusals before any launch, and
the oracle's gradients against differences and its 8-bit rounding against torch's."""
from __future__ import annotations

import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from oracle import ks_fit as o
from paper_2606_28565_amd import abi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NFAM = abi.NFAM
A = 1 << 20      # an address that is never read: every call here is refused on the host


def test_struct_layout_matches_header(tmp_path):
    structs = {"ks_rows": abi.ks_rows, "ks_gated_grad": abi.ks_gated_grad, "ks_eta_target": abi.ks_eta_target,
               "ks_tensor": abi.ks_tensor, "ks_adamw_config": abi.ks_adamw_config}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ks.h"', "int main(void){"]
    for s, cls in structs.items():
        lines.append(f'printf("{s} size %zu\\n", sizeof({s}));')
        lines += [f'printf("{s} {f} %zu\\n", offsetof({s}, {f}));' for f, _ in cls._fields_]
    lines.append('printf("mode x %d\\n", KS_ETA_GATED); return 0;}')
    c, exe = tmp_path / "probe.c", tmp_path / "probe"
    c.write_text("\n".join(lines))
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    str(c), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        s, f, n = line.split()
        want = abi.KS_ETA_GATED if s == "mode" else C.sizeof(structs[s]) if f == "size" else getattr(structs[s], f).offset
        assert int(n) == want, line


def heads(**kw):
    h = abi.ks_heads()
    h.in_dim, h.hidden, h.precision, h.mode = 16, 64, abi.KS_F32, abi.KS_ETA_GATED
    h.w1 = h.w2 = h.w3 = h.b3 = A
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def rows(n=20, **kw):
    r = abi.ks_rows()
    r.n_rows, r.x, r.ldx = n, A, 16
    for f in range(NFAM + 1):
        r.fam_off[f] = n * f // NFAM
    for k, v in kw.items():
        if k.startswith("off"):
            r.fam_off[int(k[3:])] = v
        else:
            setattr(r, k, v)
    return r


BAD_HEADS = [dict(mode=abi.KS_ETA_MLP), dict(mode=abi.KS_ETA_ONE), dict(mode=3), dict(in_dim=8), dict(in_dim=17),
             dict(in_dim=64), dict(hidden=0), dict(hidden=-1), dict(hidden=257), dict(precision=2), dict(w1=None),
             dict(w2=None), dict(w3=None), dict(b3=None), dict(w1=A + 2), dict(w3=A + 1), dict(precision=abi.KS_BF16, b3=A + 1)]
BAD_ROWS = [(dict(n_rows=-1), abi.KS_ERANGE), (dict(n_rows=1 << 31), abi.KS_ERANGE), (dict(off0=1), abi.KS_EINVAL),
            (dict(off4=3), abi.KS_EINVAL), (dict(off10=21), abi.KS_EINVAL), (dict(ldx=15), abi.KS_EINVAL),
            (dict(ldx=(1 << 31) + 1), abi.KS_EINVAL), (dict(x=None), abi.KS_EINVAL), (dict(x=A + 2), abi.KS_EINVAL)]


def calls(h, r):
    """Each row entry point's status on these heads and rows, all else valid."""
    t, g = abi.ks_eta_target(A, None, 1.0), abi.ks_gated_grad(A, A, A, A, None, 0)
    big = 1 << 40
    return [abi.ks_gated_forward(h, r, A, None, check=False),
            abi.ks_gated_backward(h, r, A, g, A, big, None, check=False),
            abi.ks_gated_loss(h, r, t, A, None, g, A, big, None, check=False)]


@pytest.mark.parametrize("bad", BAD_HEADS)
def test_bad_heads(bad):
    assert calls(heads(**bad), rows()) == [abi.KS_EINVAL] * 3
    assert abi.ks_last_error()


@pytest.mark.parametrize("bad,status", BAD_ROWS)
def test_bad_rows(bad, status):
    assert calls(heads(), rows(**bad)) == [status] * 3
    assert abi.ks_last_error()


def test_null_structs():
    lib = abi.load()
    h, r = heads(), rows()
    assert lib.ks_gated_forward(None, C.byref(r), A, None) == abi.KS_EINVAL
    assert lib.ks_gated_forward(C.byref(h), None, A, None) == abi.KS_EINVAL
    assert lib.ks_gated_backward(C.byref(h), C.byref(r), A, None, A, 1 << 40, None) == abi.KS_EINVAL
    assert lib.ks_gated_loss(C.byref(h), C.byref(r), None, A, None, None, A, 1 << 40, None) == abi.KS_EINVAL
    assert lib.ks_gated_workspace_bytes(None, C.byref(r)) == 0
    assert lib.ks_gated_workspace_bytes(C.byref(h), None) == 0
    assert lib.ks_adamw(None, None, 0, None) == abi.KS_EINVAL
    assert abi.ks_gated_forward(h, r, None, None, check=False) == abi.KS_EINVAL
    assert abi.ks_gated_forward(h, r, A + 2, None, check=False) == abi.KS_EINVAL


def test_empty_forward_needs_nothing():
    assert abi.ks_gated_forward(heads(), rows(0, x=None), None, None) == abi.KS_OK


def test_workspace():
    """Sizes alone are read; the room grows with rows and widths, and a smaller,
    missing or misaligned one is refused."""
    h, r = heads(), rows(5000)
    need = abi.ks_gated_workspace_bytes(h, r)
    assert need > 0 and need % 256 == 0
    bare = abi.ks_heads()
    bare.in_dim, bare.hidden, bare.mode = 16, 64, abi.KS_ETA_GATED
    assert abi.ks_gated_workspace_bytes(bare, rows(5000, x=None)) == need
    assert abi.ks_gated_workspace_bytes(heads(hidden=256, in_dim=32), rows(5000, ldx=32)) > need
    assert abi.ks_gated_workspace_bytes(h, rows(0)) > 0
    for bad in (dict(hidden=300), dict(in_dim=20), dict(mode=abi.KS_ETA_MLP)):
        assert abi.ks_gated_workspace_bytes(heads(**bad), r) == 0
    assert abi.ks_gated_workspace_bytes(h, rows(off3=0)) == 0
    t, g = abi.ks_eta_target(A, None, 1.0), abi.ks_gated_grad(A, A, A, A, None, 0)
    for ws, size in ((None, need), (A, need - 1), (A + 128, need)):
        assert abi.ks_gated_backward(h, r, A, g, ws, size, None, check=False) == abi.KS_EWORKSPACE
        assert abi.ks_gated_loss(h, r, t, A, None, g, ws, size, None, check=False) == abi.KS_EWORKSPACE


@pytest.mark.parametrize("prec", [abi.KS_F32, abi.KS_BF16])
@pytest.mark.parametrize("hid,inp", [(1, 16), (96, 32), (129, 32), (256, 16)])
def test_workspace_of_any_split(prec, hid, inp):
    """Rows over the families in any way, up to the most there may be: the room is
    that of at most 512 workgroups' sums (1024 of the forward pass), and each row's dz."""
    h = heads(hidden=hid, in_dim=inp, precision=prec)
    part = 4 * ((hid + 31) // 32 * 32 * 2 * inp + 1)
    rng = np.random.default_rng(5)
    for n in (0, 1, 9, 127, 128, 129, 5120, 65536, 65537, 131072, 10**6, (1 << 31) - 1):
        for k in range(4):
            r = rows(n, ldx=inp)
            cut = np.sort(rng.integers(0, n + 1, NFAM - 1)) if k < 2 else np.full(NFAM - 1, n if k == 2 else 0)
            for f in range(1, NFAM):
                r.fam_off[f] = int(cut[f - 1])
            r.fam_off[NFAM] = n
            need = abi.ks_gated_workspace_bytes(h, r)
            assert 4 * n <= need - (256 if n == 0 else 0) <= 512 * part + 1024 * 16 + 4 * n + 3 * 256, (n, k)


def test_bad_gradients():
    h, r, big = heads(), rows(), 1 << 40

    def back(*g):
        return abi.ks_gated_backward(h, r, A, abi.ks_gated_grad(*g), A, big, None, check=False)

    assert back(A, None, A, A, None, 0) == abi.KS_EINVAL
    assert back(A, A, A, A + 1, None, 0) == abi.KS_EINVAL
    far = A + (1 << 16)
    assert back(A, A, A, A, far, 15) == abi.KS_EINVAL            # a row does not fit its stride
    assert back(A, A, A, A, far + 2, 16) == abi.KS_EINVAL        # not aligned to its type
    assert back(A, A, A, A, far, (1 << 20) + 1) == abi.KS_EINVAL
    assert back(A, A, A, A, A, 16) == abi.KS_EINVAL              # over the rows themselves
    assert back(A, A, A, A, A + 16 * 4 * 19, 16) == abi.KS_EINVAL   # over the last of them
    assert abi.ks_gated_backward(h, r, None, abi.ks_gated_grad(A, A, A, A, None, 0), A, big, None, check=False) == abi.KS_EINVAL
    t = abi.ks_eta_target(A, None, 1.0)
    assert abi.ks_gated_loss(h, r, t, A, None, abi.ks_gated_grad(A, A, A, A, far, 16), A, big, None, check=False) == abi.KS_EINVAL


@pytest.mark.parametrize("huber", [0.0, -1.0, float("nan"), 1e-60])
def test_bad_huber(huber):
    t = abi.ks_eta_target(A, None, huber)
    assert abi.ks_gated_loss(heads(), rows(), t, A, None, None, A, 1 << 40, None, check=False) == abi.KS_EINVAL


def test_bad_targets():
    h, r = heads(), rows()

    def loss(t, out=A, z=None):
        return abi.ks_gated_loss(h, r, t, out, z, None, A, 1 << 40, None, check=False)

    assert loss(abi.ks_eta_target(None, None, 1.0)) == abi.KS_EINVAL
    assert loss(abi.ks_eta_target(A + 1, None, 1.0)) == abi.KS_EINVAL
    assert loss(abi.ks_eta_target(A, A + 2, 1.0)) == abi.KS_EINVAL
    assert loss(abi.ks_eta_target(A, None, 1.0), None) == abi.KS_EINVAL
    assert loss(abi.ks_eta_target(A, None, 1.0), A, A + 3) == abi.KS_EINVAL


def desc(n=20):
    d = abi.ks_desc()
    d.n_rows, d.n_steps, d.elem_bytes = n, 1, 2
    for f in range(NFAM + 1):
        d.fam_off[f] = n * f // NFAM
    d.step = d.m = d.n = d.k = d.a = d.b = d.req_off = A
    return d


def test_bad_features():
    d, big = desc(), 1 << 40

    def call(desc_=d, specs=A, ns=2, inp=16, prec=0, x=A, ldx=16, roof=None, ws=A, wsb=big):
        return abi.ks_features(desc_, specs, ns, inp, prec, x, ldx, roof, ws, wsb, None, check=False)

    for kw in (dict(inp=8), dict(inp=31), dict(prec=2), dict(x=None), dict(x=A + 2), dict(ldx=15), dict(inp=32, ldx=16),
               dict(roof=A + 1), dict(specs=None), dict(ns=0), dict(ns=-3)):
        assert call(**kw) == abi.KS_EINVAL, kw
    assert call(ws=None) == abi.KS_EWORKSPACE
    assert call(wsb=16) == abi.KS_EWORKSPACE
    assert call(ws=A + 16) == abi.KS_EWORKSPACE
    assert call(desc_=desc(1 << 30), ns=2) == abi.KS_ERANGE
    bad = desc()
    bad.fam_off[3] = 0
    assert call(desc_=bad) == abi.KS_EINVAL
    assert abi.load().ks_features(None, A, 1, 16, 0, A, 16, None, A, big, None) == abi.KS_EINVAL


def test_bad_adamw():
    def tensor(**kw):
        t = abi.ks_tensor(10, A, A, A, A, None, None, None, 0.0, abi.KS_F32)
        for k, v in kw.items():
            setattr(t, k, v)
        return t

    def call(cfg, *tensors):
        return abi.ks_adamw(cfg, (abi.ks_tensor * len(tensors))(*tensors), None, check=False)

    good = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=1.0, state_bits=32, step=1)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(lr=1e39), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan),
               dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-60), dict(eps=inf), dict(grad_scale=nan), dict(grad_scale=1e300),
               dict(state_bits=16), dict(state_bits=0), dict(step=0)):
        assert call(abi.adamw_config(**{**good, **kw}), tensor()) == abi.KS_EINVAL, kw
    cfg, cfg8 = abi.adamw_config(**good), abi.adamw_config(**{**good, "state_bits": 8})
    for kw in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(grad_type=2), dict(weight_decay=nan),
               dict(weight_decay=inf),
               dict(param=A + 2), dict(grad=A + 2), dict(m=A + 1), dict(v=A + 2), dict(copy=A + 1), dict(m_exp=A)):
        assert call(cfg, tensor(param=A + 4096), tensor(**kw)) == abi.KS_EINVAL, kw
    for n in (-1, (1 << 35) + 1):
        assert call(cfg, tensor(n=n)) == abi.KS_ERANGE
    assert call(cfg8, tensor()) == abi.KS_EINVAL
    assert call(cfg8, tensor(m_exp=A)) == abi.KS_EINVAL
    assert call(cfg, tensor(), tensor()) == abi.KS_EINVAL         # the same parameter twice
    assert "share" in abi.ks_last_error()
    assert call(cfg, tensor(param=A + 36), tensor()) == abi.KS_EINVAL   # ... its last element
    assert "share" in abi.ks_last_error()
    assert abi.load().ks_adamw(C.byref(cfg), None, 2, None) == abi.KS_EINVAL
    assert abi.load().ks_adamw(C.byref(cfg), None, -1, None) == abi.KS_EINVAL


def test_binding_refuses_what_it_cannot_describe():
    import torch
    z = torch.zeros
    w = (z(NFAM, 64, 16), z(NFAM, 64, 16), z(NFAM, 64), z(NFAM))
    assert abi.gated_heads(*w).hidden == 64
    with pytest.raises(ValueError):
        abi.gated_heads(w[0], z(NFAM, 32, 16), w[2], w[3])
    with pytest.raises(ValueError):
        abi.gated_heads(w[0], w[1].bfloat16(), w[2], w[3])
    with pytest.raises(ValueError):
        abi.gated_heads(z(NFAM, 16, 64).transpose(1, 2), w[1], w[2], w[3])
    with pytest.raises(ValueError):
        abi.feature_rows(z(16, 30).t(), [0] * 11)
    for x in (z(16).expand(30, 16), z(64).as_strided((10, 16), (4, 1))):   # rows over one another
        with pytest.raises(ValueError):
            abi.feature_rows(x, [0] * 11)
        with pytest.raises(ValueError):
            abi.gated_grad(x=x)
    assert abi.feature_rows(z(16).expand(1, 16), [0] * 11).ldx == 16
    with pytest.raises(ValueError):
        abi.gated_grad(w1=w[0].bfloat16())
    with pytest.raises(ValueError):
        abi.eta_target(z(5), z(4))
    with pytest.raises(ValueError):
        abi.eta_target(z(5).double())
    t = {"param": z(70), "grad": z(70), "m": z(70), "v": z(70)}
    assert abi.adamw_tensors([t])[0].n == 70
    for bad in ({"grad": z(69)}, {"m": z(70).bfloat16()}, {"m_exp": torch.zeros(2, dtype=torch.uint8)},
                {"copy": z(70)}, {"param": z(70).double()}):
        with pytest.raises(ValueError):
            abi.adamw_tensors([{**t, **bad}])


# ------------------------------------------------------------------ the oracle itself
def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(2)
    n, D, H = 12, 16, 7
    x, w1, w2, w3, b3 = rng.random((n, D)), rng.normal(size=(H, D)), rng.normal(size=(H, D)), rng.normal(size=H), 0.3
    eta, wt = 1 + rng.random(n), rng.random(n)
    wt[3], eta[5] = 0.0, np.nan

    for huber in (np.inf, 0.4):
        def loss(p):
            z, _ = o.block(p["x"], p["w1"], p["w2"], p["w3"], p["b3"])
            return o.eta_loss(z, eta, wt, huber)[0]

        p = {"x": x, "w1": w1, "w2": w2, "w3": w3, "b3": b3}
        z, k = o.block(x, w1, w2, w3, b3)
        _, dz = o.eta_loss(z, eta, wt, huber)
        assert dz[3] == 0 and dz[5] == 0
        val, _ = o.gradients(x, w1, w2, w3, dz, k, n)
        for key in ("x", "w1", "w2", "w3"):
            for _ in range(20):
                i = tuple(rng.integers(0, s) for s in p[key].shape)
                up, dn = (dict(p, **{key: p[key].copy()}) for _ in range(2))
                h = 1e-5
                up[key][i] += h
                dn[key][i] -= h
                # the third derivative's h^2 / 6 beside the rounding of two losses, 1e-16 / h
                assert abs((loss(up) - loss(dn)) / (2 * h) - val[key][i]) <= 1e-8, (key, i)
        assert abs((loss(dict(p, b3=b3 + 1e-5)) - loss(dict(p, b3=b3 - 1e-5))) / 2e-5 - val["b3"]) <= 1e-8


@pytest.mark.parametrize("second", [False, True])
def test_oracle_8_bit_rounding_is_torchs(second):
    import torch
    v = torch.randn(4096, generator=torch.Generator().manual_seed(3)) * torch.logspace(-12, 3, 4096)
    v = (v * v if second else v).numpy()
    q, e = o.encode(v, second)
    inv = np.exp2(127.0 - e).repeat(64).astype(np.float32)
    want = (torch.from_numpy(v) * torch.from_numpy(inv)).to(torch.float8_e5m2 if second else torch.float8_e4m3fn).float().numpy()
    tiny = second & (v > 0) & (want == 0)
    assert np.array_equal(np.where(tiny, 2.0 ** -16, want), q)
    assert (np.abs(q).reshape(-1, 64).max(1) >= (2.0 ** 14 if second else 2.0 ** 7)).all()
    assert (np.abs(q).reshape(-1, 64).max(1) <= (2.0 ** 15 if second else 2.0 ** 8)).all()


def test_oracle_8_bit_edges():
    q, e = o.encode(np.array([0.0, 1e-45, 0.0]), True)
    assert e[0] == 1 and q[1] == 2.0 ** -16 and q[0] == 0
    q, e = o.encode(np.array([np.inf, -np.inf, np.nan, 1.0]), False)
    assert np.isnan(q[:3]).all() and q[3] == 128 and e[0] == 120
    q, _ = o.encode(np.array([np.inf, np.nan, 4.0]), True)
    assert q[0] == np.inf and np.isnan(q[1]) and q[2] == 2.0 ** 14
