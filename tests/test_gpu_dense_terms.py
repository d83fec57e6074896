"""The input gradient of a bf16 layer takes dz = dy act'(pre) with all its 24 bits, however short its sums are.

Every row has one value of pre, so that act' is one number s, and two values of dy that are not 0: dx is
s (a w1 - b w2) for them, which cancels where (w1, w2) = (b, a).  dz is rounded to 24 bits (u of it, u = 2^-24), a
sum of two such products and its terms adds (4 sqrt 2 + 8) u of the absolute values, s itself is off by 40 u in all
products alike, and the result is rounded to bf16.  Two bf16 terms of dz would leave up to 64 u of each product."""
import numpy as np
import pytest
import torch

from layer_checks import DEV, U, close, half, like, padded
from oracle import layers as ref

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def between_1_and_2(rng, n):
    """bf16 values."""
    return 1 + rng.integers(0, 128, n) / 128


# rows, in, out, the two columns of dy that are not 0 (whole k tiles and the rest past them; every tile, split and not)
SIZES = [(64, 64, 2, 0, 1), (1, 9, 5, 1, 4), (64, 64, 96, 3, 70), (700, 900, 130, 0, 129), (70, 100, 4000, 17, 3999),
         (4000, 2000, 530, 64, 513), (4100, 2000, 130, 5, 128), (300, 260, 41000, 1, 40990)]


@pytest.mark.parametrize("name,z", [("silu", 0.703125), ("gelu", 0.703125), ("gelu", -0.40625)])
@pytest.mark.parametrize("n,n_in,n_out,j1,j2", SIZES)
def test_sums_that_cancel(n, n_in, n_out, j1, j2, name, z):
    import paper_2309_16743_amd as ot
    rng = np.random.default_rng(n + n_in)
    a, b = between_1_and_2(rng, max(n, n_in)), between_1_and_2(rng, max(n, n_in))
    dy = torch.zeros(n, (n_out + 7) // 8 * 8, dtype=BF16, device=DEV)
    dy[:, j1] = torch.from_numpy(a[:n]).to(DEV, BF16)
    dy[:, j2] = torch.from_numpy(-b[:n]).to(DEV, BF16)
    w = padded(rng.normal(size=(n_out, n_in)), BF16)
    w[j1] = torch.from_numpy(b[:n_in]).to(DEV, BF16)
    w[j2] = torch.from_numpy(a[:n_in]).to(DEV, BF16)
    pre = padded(np.full((n, n_out), z), BF16)
    dx = like((n, n_in), BF16)
    op = ot.DenseLayer(n_in, n_out, precision=ot.OT_BF16, activation={"silu": ot.OT_ACT_SILU, "gelu": ot.OT_ACT_GELU}[name],
                       max_rows=n)
    op.backward(None, w, dy[:, :n_out], pre=pre, dx=dx)
    s = float(ref.slope(np.array(z), name))
    ab, ba = np.outer(a[:n], b[:n_in]), np.outer(b[:n], a[:n_in])
    want = s * (ab - ba)
    assert not np.diagonal(want).any()
    close(dx, want, (4 * np.sqrt(2) + 9) * U * s * (ab + ba) + (40 * U + half(BF16)) * np.abs(want), "dx")
    op.close()
