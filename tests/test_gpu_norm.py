"""Group norm with an activation against the 64-bit reference (tolerances: layer_checks, and below)."""
import numpy as np
import pytest
import torch

from layer_checks import DEV, U, close, half, host, like, padded, padding_kept, vector
from layer_sizes import NORM
from oracle import layers as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ACTS = ["none", "relu", "silu", "gelu"]
EPS = 1e-5


def norm(p, c, g, dtype, name="none", n=8, eps=EPS):
    import paper_2309_16743_amd as ot
    return ot.GroupNorm(c, g, positions=p, precision=ot.OT_BF16 if dtype == BF16 else ot.OT_FP32,
                        activation=ACTS.index(name), eps=eps, max_samples=n)


def problem(n, p, c, dtype, seed, extra=0, affine=True, level=3.0):
    rng = np.random.default_rng(seed)
    x = padded(rng.normal(size=(n, p, c)) * rng.uniform(0.2, 2, c) + rng.uniform(-level, level, c), dtype, extra)
    w, b = (vector(rng.uniform(0.5, 1.5, c)), vector(rng.uniform(-0.5, 0.5, c))) if affine else (None, None)
    return rng, x, w, b


def arrays(w, b, c):
    return (np.ones(c) if w is None else host(w)), (np.zeros(c) if b is None else host(b))


def stats_tol(x, groups, mean, rstd):
    """mean: rounded once, and sums of N differences (from the mean or a value of the group) of size
    sigma; rstd: half the relative error of a sum of N squares, and of its own steps."""
    n, p, c = x.shape
    N = p * c // groups
    sigma = 1 / rstd
    return 2 * U * np.abs(mean) + (4 * np.sqrt(N) + 8) * U * sigma, (4 * np.sqrt(N) + 8) * U * rstd


def spread(v, per):
    return np.repeat(v, per, axis=-1)[:, None, :]


def forward_tol(x, groups, mean, rstd, w, b, y, dtype):
    per = x.shape[2] // groups
    tm, tr = stats_tol(x, groups, mean, rstd)
    d = x - spread(mean, per)
    xh = np.abs(d * spread(rstd, per))
    t = spread(tm * rstd, per) + spread(tr / rstd, per) * xh + 4 * U * xh
    return 1.13 * (t * np.abs(w) + 2 * U * (xh * np.abs(w) + np.abs(b))) + 80 * U * np.abs(y) + half(dtype) * np.abs(y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(NORM)))
def test_forward(i, dtype):
    n, p, c, g = NORM[i]
    name, extra = ACTS[i % 4], 8 * (i % 3)
    _, x, w, b = problem(n, p, c, dtype, 10 + i, extra, affine=i % 5 != 0)
    y, stats = like((n, p, c), dtype, extra), torch.full((n, g, 2), 7.0, device=DEV)
    op = norm(p, c, g, dtype, name, n)
    op.forward(x, y, weight=w, bias=b, stats=stats)
    hx, (hw, hb) = host(x), arrays(w, b, c)
    want, mean, rstd = ref.norm(hx, g, EPS, hw, hb, name)
    tm, tr = stats_tol(hx, g, mean, rstd)
    close(stats[..., 0], mean, tm, "mean")
    close(stats[..., 1], rstd, tr, "rstd")
    close(y, want, forward_tol(hx, g, mean, rstd, hw, hb, want, dtype), "y")
    padding_kept(y, 7.0)
    again = x.clone() if extra == 0 and c % 8 == 0 else None
    if again is not None:                                  # in place, without statistics
        op.forward(again, again, weight=w, bias=b)
        assert torch.equal(again, y)
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(NORM)))
def test_backward(i, dtype):
    n, p, c, g = NORM[i]
    per = c // g
    name, extra = ACTS[(i + 1) % 4], 8 * (i % 3)
    rng, x, w, b = problem(n, p, c, dtype, 40 + i, extra, affine=i % 5 != 0)
    hx, (hw, hb) = host(x), arrays(w, b, c)
    mean, rstd = ref.moments(hx, g, EPS)
    stats = torch.from_numpy(np.stack((mean, rstd), -1).astype(np.float32)).to(DEV)
    mean, rstd = host(stats)[..., 0], host(stats)[..., 1]
    xh = (hx - spread(mean, per)) * spread(rstd, per)
    hd = rng.normal(size=(n, p, c))
    if name == "relu":                                     # nothing at the corner, where a rounding decides
        hd[np.abs(xh * hw + hb) < 1e-4] = 0
    dy = padded(hd, dtype, extra)
    hd = host(dy)
    dx, dw, db = like((n, p, c), dtype, extra), vector(np.full(c, 7.0)), vector(np.full(c, 7.0))
    op = norm(p, c, g, dtype, name, n)
    op.backward(x, stats, dy, weight=w, bias=b, dx=dx, dweight=dw, dbias=db)
    want = ref.norm_back(hx, g, mean, rstd, hd, hw, hb, name)
    # xh is off by 3 u, p by 4 u of its terms, dp by 45 u of dy plus the slope's change (second derivative at
    # most 0.8) with p
    ad = np.abs(hd) * (1.13 if name in ("silu", "gelu") else 1.0)
    e_dp = np.zeros_like(ad) if name in ("none", "relu") else ad * (45 * U + 0.8 * 6 * U * (np.abs(xh * hw) + np.abs(hb)))
    N, R = p * per, n * p
    mean_of = lambda v: spread(v.reshape(n, p, g, per).mean((1, 3)), per)
    t1 = mean_of(np.abs(hw) * (e_dp + (4 * np.sqrt(N) + 8) * U * ad))
    t2 = mean_of(np.abs(hw * xh) * (e_dp + (4 * np.sqrt(N) + 12) * U * ad))
    m2 = mean_of(np.abs(hw * xh) * ad)
    tol = spread(rstd, per) * (np.abs(hw) * e_dp + t1 + np.abs(xh) * t2
                               + 8 * U * (np.abs(hw) * ad + mean_of(np.abs(hw) * ad) + np.abs(xh) * m2))
    close(dx, want[0], tol + half(dtype) * np.abs(want[0]), "dx")
    s = 4 * np.sqrt(R) + 8
    close(dw, want[1], (np.abs(xh) * (e_dp + s * U * ad)).sum((0, 1)) + U * np.abs(want[1]), "dweight")
    close(db, want[2], (e_dp + s * U * ad).sum((0, 1)) + U * np.abs(want[2]), "dbias")
    padding_kept(dx, 7.0)
    for kind, whole in (("dx", dx), ("dweight", dw), ("dbias", db)):       # each alone has the same bits
        one = like((n, p, c), dtype) if kind == "dx" else vector(np.zeros(c))
        op.backward(x, stats, dy, weight=w, bias=b, **{kind: one})
        assert torch.equal(one, whole), kind
    if extra == 0 and c % 8 == 0:
        op.backward(x, stats, dy, weight=w, bias=b, dx=dy)                 # in place
        assert torch.equal(dy, dx)
    op.close()


@pytest.mark.parametrize("shape", [(2, 1, 64, 4), (2, 5000, 8, 2)])
@pytest.mark.parametrize("level", [1e3, -3e5])
def test_levels_far_above_the_spread(shape, level):
    """The variance of values far from zero keeps its digits (to what x itself holds)."""
    n, p, c, g = shape
    rng = np.random.default_rng(3)
    x = padded(level + rng.normal(size=(n, p, c)))
    y, stats = like((n, p, c)), torch.zeros(n, g, 2, device=DEV)
    op = norm(p, c, g, F32, "none", n)
    op.forward(x, y, stats=stats)
    want, mean, rstd = ref.norm(host(x), g, EPS)
    tm, tr = stats_tol(host(x), g, mean, rstd)
    close(stats[..., 0], mean, tm, "mean")
    # a mean that is off by 2 u of itself adds its square to the variance
    close(stats[..., 1], rstd, tr + rstd * (2 * U * np.abs(mean) * rstd) ** 2, "rstd")
    close(y, want, forward_tol(host(x), g, mean, rstd, np.ones(c), np.zeros(c), want, F32)
          + spread((2 * U * np.abs(mean) * rstd) ** 2, c // g) * np.abs(want), "y")
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(3, 1, 40, 4), (2, 30, 40, 4), (2, 3000, 16, 2)])
def test_constant_groups(dtype, shape):
    """Of values that are all alike the mean is their value, the variance 0, the result the bias."""
    n, p, c, g = shape
    value = 300.25 if dtype == F32 else 300.0
    x = padded(np.full((n, p, c), value), dtype)
    b = vector(np.linspace(-1, 1, c))
    y, stats = like((n, p, c), F32 if dtype == F32 else BF16), torch.zeros(n, g, 2, device=DEV)
    op = norm(p, c, g, dtype, "none", n)
    op.forward(x, y, bias=b, stats=stats)
    assert bool((stats[..., 0] == value).all())
    close(stats[..., 1], np.full((n, g), EPS ** -0.5), 4 * U * EPS ** -0.5)
    assert torch.equal(y, b.to(y.dtype).expand(n, p, c))
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(3, 1, 40, 4), (2, 30, 40, 4), (2, 3000, 16, 2)])
def test_a_nan_stays_in_its_group(dtype, shape):
    n, p, c, g = shape
    per = c // g
    _, x, w, b = problem(n, p, c, dtype, 5)
    y, clean = like((n, p, c), dtype), like((n, p, c), dtype)
    op = norm(p, c, g, dtype, "relu", n)
    op.forward(x, clean, weight=w, bias=b)
    x[1, p - 1, per] = float("nan")
    x[0, 0, 0] = float("inf")
    stats = torch.zeros(n, g, 2, device=DEV)
    op.forward(x, y, weight=w, bias=b, stats=stats)
    hit = torch.zeros(n, p, c, dtype=torch.bool, device=DEV)
    hit[1, :, per:2 * per] = True
    hit[0, :, :per] = True
    assert torch.equal(y[~hit], clean[~hit])
    assert bool(y[1, :, per:2 * per].isnan().all()) and bool(y[0, 0, 0].isnan())
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_samples_and_two_dimensions(dtype):
    op = norm(1, 24, 3, dtype, "silu", 0)
    op.forward(like((0, 24), dtype), like((0, 24), dtype))
    dw, db = vector(np.full(24, 7.0)), vector(np.full(24, 7.0))
    op.backward(like((0, 24), dtype), torch.zeros(0, 3, 2, device=DEV), like((0, 24), dtype), dweight=dw, dbias=db)
    assert not host(dw).any() and not host(db).any()
    _, x, w, b = problem(5, 1, 24, dtype, 6)
    y, y2 = like((5, 1, 24), dtype), like((5, 24), dtype)
    op.forward(x, y, weight=w, bias=b)
    op.forward(x[:, 0], y2, weight=w, bias=b)
    assert torch.equal(y[:, 0], y2)
    op.close()


def test_offsets_past_32_bits():
    """Rows 2^28 values apart."""
    ld = 1 << 28
    if torch.cuda.mem_get_info()[0] < 3 * 18 * ld * 2:
        pytest.skip("not enough memory")
    big = torch.empty(18 * ld, dtype=BF16, device=DEV)
    view = lambda at, n, p, c: torch.as_strided(big, (n, p, c), (p * ld, ld, 1), at)
    for n, p, c, g in ((2, 9, 16, 2), (1, 17, 1000, 1)):      # one of each form
        rng = np.random.default_rng(9)
        x, y, dy, dx = (view(at, n, p, c) for at in (0, 1024, 2048, 4096))
        x.copy_(torch.from_numpy(rng.normal(size=(n, p, c))))
        dy.copy_(torch.from_numpy(rng.normal(size=(n, p, c))))
        near = [t.clone() for t in (x, dy)]
        op = norm(p, c, g, BF16, "none", n)
        stats = torch.zeros(n, g, 2, device=DEV)
        y2, dx2 = torch.empty_like(near[0]), torch.empty_like(near[0])
        op.forward(x, y, stats=stats)
        op.forward(near[0], y2)
        assert torch.equal(y.clone(), y2)
        op.backward(x, stats, dy, dx=dx)
        op.backward(near[0], stats, near[1], dx=dx2)
        assert torch.equal(dx.clone(), dx2)
        op.close()
