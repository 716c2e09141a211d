"""The fit with learned columns and dropout without a GPU: what it refuses, and which rows it
works in."""
from __future__ import annotations

import pytest

from paper_2606_28565_amd import abi, fit

NFAM = abi.NFAM


def measurements(n=6, in_dim=16):
    import torch
    return fit.Measurements(torch.rand(n, in_dim), [0] * NFAM + [n], torch.ones(n))


@pytest.mark.parametrize("p", [0.25, 1e-9])
@pytest.mark.parametrize("precision", ["f32", "bf16"])
def test_features_beside_their_squares_are_not_dropped(p, precision):
    """Rows of 32 inputs are the 16 features and their squares: columns 15 and 31 are the
    constant, and no dropout keeps both a feature's expected value and its square's."""
    with pytest.raises(ValueError, match="squares"):
        fit.GatedFit(32, 8, precision, device="cpu", feature_dropout=p)
    assert fit.GatedFit(32, 8, precision, device="cpu").feature_drop is None
    for kind in (dict(in_dim=16), dict(in_dim=32, categories=2), dict(in_dim=16, categories=2)):
        assert fit.GatedFit(hidden=8, precision=precision, device="cpu", feature_dropout=p, **kind).feature_drop is not None


def test_the_constant_is_not_among_the_features_to_drop():
    d = measurements()
    fit.GatedFit(16, 8, device="cpu", feature_dropout=0.1).workspace(d)
    assert d.noisy.shape == d.x.shape and (d.noisy == d.x).all()


def test_each_fit_drops_features_in_rows_of_its_own():
    """Fits on the same rows may step at the same time, on streams or in graphs of their own:
    none writes what another one reads."""
    d, other = measurements(), measurements(9)
    a, b = (fit.GatedFit(16, 8, device="cpu", seed=s, feature_dropout=0.1) for s in (1, 2))
    seen = []
    for ft in (a, b):
        for data in (d, other):
            ft.workspace(data)
            seen.append(data.noisy)
    assert len({t.data_ptr() for t in seen + [d.x, other.x]}) == 6
    # ... and keeps them: a captured step goes on using them
    for ft, data, rows in zip((a, a, b, b), (d, other) * 2, seen):
        ft.workspace(data)
        assert data.noisy is rows
