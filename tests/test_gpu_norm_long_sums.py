"""Group norm's dweight and dbias over very many samples."""
import pytest
import torch

from layer_checks import DEV, U, close, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,p,c,g", [(131072, 16, 16, 2), (40000, 64, 24, 3)])
def test_equal_terms(n, p, c, g):
    """With the statistics 0 and 1 and x = 1 the terms of a channel are all its dy.  A chunk of 16 (64) positions sums
    them in powers of two, without rounding; what is left is the sum over n chunks, rounded once to fp32.  (Added one by
    one in fp32, 4096 equal terms would be off by up to 700 u of their sum.)"""
    import paper_2309_16743_amd as ot
    x = torch.ones(n, p, c, device=DEV)
    value = torch.linspace(0.1, 0.9, c, device=DEV)
    dy = value.expand(n, p, c).contiguous()
    stats = torch.zeros(n, g, 2, device=DEV)
    stats[..., 1] = 1.0
    want = n * p * host(value)
    op = ot.GroupNorm(c, g, positions=p, max_samples=n)
    for dx in (None, torch.empty_like(x)):
        dw, db = torch.zeros(c, device=DEV), torch.zeros(c, device=DEV)
        op.backward(x, stats, dy, dx=dx, dweight=dw, dbias=db)
        close(dw, want, 2 * U * want, "dweight")
        close(db, want, 2 * U * want, "dbias")
    op.close()
