"""The layers' 64-bit reference: gradients against differences, Philox against published answers."""
import numpy as np
import pytest

from oracle import layers as ref

ACTS = ["none", "relu", "silu", "gelu"]


def difference(f, a, h=1e-6):
    """Central differences of the number f() in every element of a."""
    g = np.zeros_like(a)
    for i in np.ndindex(a.shape):
        keep = a[i]
        a[i] = keep + h
        hi = f()
        a[i] = keep - h
        lo = f()
        a[i] = keep
        g[i] = (hi - lo) / (2 * h)
    return g


# Central differences at h = 1e-6 of values of size 1 in 64 bits: rounding 1e-16 / 1e-6 times the sum's terms
# (about 100), curvature h^2: both below 1e-7.
TOL = 1e-7


@pytest.mark.parametrize("name", ACTS)
def test_dense_gradients(name):
    rng = np.random.default_rng(1)
    x, w, b, dy = rng.normal(size=(3, 4)), rng.normal(size=(5, 4)), rng.normal(size=5), rng.normal(size=(3, 5))
    _, z = ref.dense(x, w, b, None, name)
    assert np.abs(z).min() > 1e-3                        # away from relu's corner
    dx, dw, db = ref.dense_back(x, w, dy, z, name)
    f = lambda: float((ref.dense(x, w, b, None, name)[0] * dy).sum())
    for got, a in ((dx, x), (dw, w), (db, b)):
        assert np.abs(got - difference(f, a)).max() < TOL


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("groups", [1, 2, 6])
def test_norm_gradients(name, groups):
    rng = np.random.default_rng(2)
    x, dy = rng.normal(size=(2, 3, 6)), rng.normal(size=(2, 3, 6))
    w, b = rng.normal(size=6), rng.normal(size=6)
    y, mean, rstd = ref.norm(x, groups, 1e-2, w, b, name)
    assert name != "relu" or np.abs(ref.norm(x, groups, 1e-2, w, b)[0]).min() > 1e-4
    dx, dw, db = ref.norm_back(x, groups, mean, rstd, dy, w, b, name)
    f = lambda: float((ref.norm(x, groups, 1e-2, w, b, name)[0] * dy).sum())
    for got, a in ((dx, x), (dw, w), (db, b)):
        assert np.abs(got - difference(f, a)).max() < TOL


def test_philox_known_answers():
    """The vectors that the generator's authors publish with it."""
    ones = 0xFFFFFFFF
    assert ref.philox4x32((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert ref.philox4x32((ones,) * 4, (ones,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert ref.philox4x32((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == [
        0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_dropout_mask_rates():
    """Kept shares: of n independent values within five standard deviations; a mask is its own at
    another site, step and seed."""
    rows, cols = range(64), 100
    for p in (0.1, 0.5, 0.9):
        keep, scale = ref.dropout_keep(rows, cols, p, 7, 1, 2)
        n = keep.size
        assert abs(keep.mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n)
        assert abs(scale * (1 - p) - 1) < 1e-4
    base = ref.dropout_keep(rows, cols, 0.5, 7, 1, 2)[0]
    for other in ((8, 1, 2), (7, 2, 2), (7, 1, 3), (7 + (1 << 40), 1, 2)):
        same = (ref.dropout_keep(rows, cols, 0.5, *other)[0] == base).mean()
        assert abs(same - 0.5) < 5 * np.sqrt(0.25 / base.size)
    assert ref.dropout_keep(rows, cols, 0.0, 7, 1, 2)[0].all()
    assert not ref.dropout_keep(rows, cols, 1.0, 7, 1, 2)[0].any()
