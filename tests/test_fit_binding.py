"""The binding's structs of the fitting calls remember the shapes, types and devices they
were made for, and the calls refuse those that do not go together: the library sees
addresses only.  CPU only; nothing here reaches a launch."""
from __future__ import annotations

import pytest

from paper_2606_28565_amd import abi

NFAM = abi.NFAM
A = 1 << 20      # an address that is never read
OFF = [0] + [20] * NFAM


def tensors(hid=8, inp=16, dtype=None):
    import torch
    dt = dtype or torch.float32
    return [torch.zeros(s, dtype=dt) for s in ((NFAM, hid, inp), (NFAM, hid, inp), (NFAM, hid), (NFAM,))]


def made(what, place=None):
    """As if made from tensors of a GPU (None: of the caller's own addresses)."""
    what.place = place
    return what


def parts(n=20, hid=8, inp=16, place=0):
    import torch
    return [made(s, place) for s in (abi.gated_heads(*tensors(hid, inp)), abi.feature_rows(torch.zeros(n, inp), OFF),
                                     abi.gated_grad(*tensors(hid, inp)), abi.eta_target(torch.ones(n)))]


def refused(h, r, g, t):
    """How many of the row calls refuse to go on to the library."""
    n = 0
    for call in (lambda: abi.ks_gated_forward(h, r, None, None, check=False),
                 lambda: abi.ks_gated_backward(h, r, A, g, None, 0, None, check=False),
                 lambda: abi.ks_gated_loss(h, r, t, A, None, g, None, 0, None, check=False)):
        try:
            assert call() in (abi.KS_EINVAL, abi.KS_EWORKSPACE)      # (the library's own refusal: no z, no workspace)
        except ValueError:
            n += 1
    return n


def test_what_goes_together_is_taken():
    assert refused(*parts()) == 0
    assert refused(*parts(place=None)) == 0


def test_tensors_on_the_cpu():
    assert refused(*parts(place=-1)) == 3
    assert [s.place for s in (abi.gated_heads(*tensors()), abi.gated_grad(*tensors()))] == [-1, -1]


@pytest.mark.parametrize("which,calls", [(0, 3), (1, 3), (2, 2), (3, 1)])
def test_tensors_on_different_gpus(which, calls):
    p = parts()
    p[which].place = 1
    assert refused(*p) == calls


def test_rows_of_another_kind():
    import torch
    h, r, g, t = parts()
    for x in (torch.zeros(20, 16).bfloat16(), torch.zeros(20, 64)[:, :8]):
        assert refused(h, made(abi.feature_rows(x, OFF), 0), g, t) == 3
    assert refused(h, made(abi.feature_rows(torch.zeros(20, 40), OFF), 0), g, t) == 0    # (the first 16 are read)


def test_gradients_of_another_shape():
    import torch
    h, r, g, t = parts()
    for hid, inp in ((7, 16), (8, 32), (9, 16)):
        assert refused(h, r, made(abi.gated_grad(*tensors(hid, inp)), 0), t) == 2
    for x in (torch.zeros(19, 16), torch.zeros(20, 64)[:, :8], torch.zeros(20, 16).bfloat16()):
        assert refused(h, r, made(abi.gated_grad(x=x), 0), t) == 2
    assert refused(h, r, made(abi.gated_grad(x=torch.zeros(21, 40)), 0), t) == 0    # (room for more)
    w1, w2, w3, b3 = tensors()
    for bad in ((w1, w2[:, :7].contiguous(), w3, b3), (w1, w2, w3[:, :5].contiguous(), b3), (w1, w2, w3, b3[:3]),
                (w1[:, :, :15].contiguous(), w2, w3, b3), (w1, w2, w3[:0], b3)):
        with pytest.raises(ValueError):
            abi.gated_grad(*bad)
    flat = [v.reshape(-1) for v in (w1, w2, w3, b3)]      # (parts of one buffer, as an optimiser may keep them)
    assert refused(h, r, made(abi.gated_grad(*flat), 0), t) == 0
    assert refused(h, r, made(abi.gated_grad(*(v.reshape(-1) for v in tensors(16, 8))), 0), t) == 2


def test_targets_of_another_length():
    import torch
    h, r, g, _ = parts()
    for n, refusals in ((0, 1), (19, 1), (21, 0)):
        assert refused(h, r, g, made(abi.eta_target(torch.ones(n)), 0)) == refusals


def test_adamw():
    import torch
    z = torch.zeros
    arr = abi.adamw_tensors([{"param": z(70), "grad": z(70), "m": z(70), "v": z(70)}])
    count = z(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        abi.ks_adamw(abi.adamw_config(1e-3), arr, None)
    for tp, cp in ((0, -1), (0, 1)):
        with pytest.raises(ValueError):
            abi.ks_adamw(made(abi.adamw_config(1e-3, step_dev=count), cp), made(arr, tp), None)
    assert abi.ks_adamw(made(abi.adamw_config(-1.0, step_dev=count), 0), made(arr, 0), None, check=False) == abi.KS_EINVAL
    for bad in (z(1), z(0, dtype=torch.int32), z(1, dtype=torch.int16)):
        with pytest.raises(ValueError):
            abi.adamw_config(1e-3, step_dev=bad)


def test_gated_heads_beside_the_bounded_head_and_grids():
    """The fields that make_heads fills for MLP heads, with arrays that live as long as the
    struct."""
    import ctypes as C

    import numpy as np

    from workload import gen
    bounded, grid = gen.make_bounded(0b1000010010), gen.make_grid(0b0000100001)
    h = abi.gated_heads(*tensors(), bounded=bounded, grid=grid)
    m = abi.DeviceInputs(gen.config1(0, 1), device="cpu").make_heads("f32", 16, 64, abi.KS_ETA_GATED, bounded, grid)
    assert (h.mode, h.hidden, h.in_dim) == (abi.KS_ETA_GATED, 8, 16)
    for name in ("bounded_mask", "grid_mask"):
        assert getattr(h, name) == getattr(m, name) != 0
    for name in ("grid_axis", "grid_n", "grid_lo", "grid_hi"):
        assert list(getattr(h, name)) == list(getattr(m, name)), name
    for at, want in ((h.bounded, bounded.storage), (h.grid, grid.values)):
        got = np.frombuffer((C.c_float * want.size).from_address(at), np.float32)
        np.testing.assert_array_equal(got, np.asarray(want, np.float32).reshape(-1))
    plain = abi.gated_heads(*tensors())
    assert plain.bounded_mask == plain.grid_mask == 0 and plain.bounded is None and plain.grid is None
