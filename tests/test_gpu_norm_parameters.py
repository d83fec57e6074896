"""Group norm's parameters: values that are not finite stay in their group."""
import numpy as np
import pytest
import torch

from layer_checks import DEV, host, like, padded, vector

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def norm(p, c, g, dtype, n, act=0):
    import paper_2309_16743_amd as ot
    return ot.GroupNorm(c, g, positions=p, precision=ot.OT_BF16 if dtype == BF16 else ot.OT_FP32, activation=act,
                        max_samples=n)


# samples, positions, channels, groups: teams with idle lanes (groups of 3, 5, 9 and 75 vectors of 8 channels), teams
# without, slabs, split passes
SIZES = [(6, 1, 72, 3), (700, 1, 120, 3), (9, 1, 144, 2), (3, 1, 1800, 3), (5, 1, 64, 4), (4, 2, 48, 2), (3, 9, 12, 4),
         (2, 200, 24, 3), (2, 3000, 16, 2)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("n,p,c,g", SIZES)
def test_a_weight_that_is_not_finite_stays_in_its_group(n, p, c, g, bad, dtype):
    per = c // g
    rng = np.random.default_rng(21)
    x, dy = padded(rng.normal(size=(n, p, c)), dtype), padded(rng.normal(size=(n, p, c)), dtype)
    w, b = vector(rng.uniform(0.5, 1.5, c)), vector(rng.uniform(-0.5, 0.5, c))
    op = norm(p, c, g, dtype, n, act=1)
    got = []
    for first in (1.0, bad):
        w[0] = first
        y, dx = like((n, p, c), dtype), like((n, p, c), dtype)
        dw, db, stats = vector(np.zeros(c)), vector(np.zeros(c)), torch.zeros(n, g, 2, device=DEV)
        op.forward(x, y, weight=w, bias=b, stats=stats)
        op.backward(x, stats, dy, weight=w, bias=b, dx=dx, dweight=dw, dbias=db)
        got.append((y, dx, dw, db))
    (y, dx, dw, db), (y2, dx2, dw2, db2) = got
    assert torch.equal(y[..., 1:], y2[..., 1:])
    assert torch.equal(dx[..., per:], dx2[..., per:]) and bool(torch.isfinite(dx2[..., per:]).all())
    assert torch.equal(dw[1:], dw2[1:]) and torch.equal(db[1:], db2[1:])
    op.close()
