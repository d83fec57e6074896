"""Dropout against the generator's published definition and the 64-bit values."""
import numpy as np
import pytest
import torch

from layer_checks import DEV, U, close, half, host, like, padded, padding_kept
from layer_sizes import DROPOUT
from oracle import layers as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def dropout(p, seed=0x123456789abcdef0, site=3, dtype=F32):
    import paper_2309_16743_amd as ot
    return ot.Dropout(p, seed, site=site, precision=ot.OT_BF16 if dtype == BF16 else ot.OT_FP32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(DROPOUT)))
def test_values(i, dtype):
    n, cols = DROPOUT[i]
    p, extra, step = (0.1, 0.5, 0.75, 0.25, 1e-3)[i % 5], 8 * (i % 3), (5, 2 ** 32 - 1, 0)[i % 3]
    rng = np.random.default_rng(i)
    x = padded(rng.normal(size=(n, cols)), dtype, extra)
    r = padded(rng.normal(size=(n, cols)), dtype, extra) if i % 2 else None
    y, dx = like((n, cols), dtype, extra), like((n, cols), dtype, extra)
    op = dropout(p, dtype=dtype)
    op.forward(x, y, step, residual=r)
    op.backward(x, dx, step)
    keep, scale = ref.dropout_keep(range(n), cols, p, op.seed, op.site, step)
    part = np.where(keep, host(x) * scale, 0.0)
    want = part + (0 if r is None else host(r))
    # the scale is rounded, the product and the sum once together
    close(y, want, 2 * U * np.abs(part) + half(dtype) * np.abs(want), "y")
    close(dx, part, 2 * U * np.abs(part) + half(dtype) * np.abs(part), "dx")
    for t in (y, dx):
        padding_kept(t, 7.0)
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_none_and_all(dtype):
    x = padded(np.random.default_rng(1).normal(size=(20, 33)), dtype)
    r = padded(np.random.default_rng(2).normal(size=(20, 33)), dtype)
    x[3, 4] = float("nan")
    y = like((20, 33), dtype)
    op = dropout(0.0, dtype=dtype)
    op.forward(x, y, 0)
    assert torch.equal(y.view(torch.int16 if dtype == BF16 else torch.int32)[x == x],
                       x.view(torch.int16 if dtype == BF16 else torch.int32)[x == x])
    op.close()
    op = dropout(1.0, dtype=dtype)
    op.forward(x, y, 0, residual=r)
    assert torch.equal(y, r)
    op.forward(x, y, 0)
    assert not host(y).any()
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropped_values_may_be_anything(dtype):
    x = padded(np.random.default_rng(1).normal(size=(50, 70)), dtype)
    op = dropout(0.5, dtype=dtype)
    keep = torch.from_numpy(ref.dropout_keep(range(50), 70, 0.5, op.seed, op.site, 9)[0]).to(DEV)
    y, y2 = like((50, 70), dtype), like((50, 70), dtype)
    op.forward(x, y, 9)
    x[~keep] = float("inf")
    op.forward(x, y2, 9)
    assert torch.equal(y, y2)
    x[~keep] = float("nan")
    op.forward(x, y2, 9, residual=y)
    assert torch.equal(y2[~keep], y[~keep])
    op.close()


def test_a_mask_is_of_rows_and_columns_alone():
    """Not of strides, types or the number of rows and columns: parts of a matrix that start at its first
    row and column have its mask."""
    x = padded(np.ones((40, 100)))
    whole = like((40, 100))
    op = dropout(0.5)
    op.forward(x, whole, 1)
    for n, cols, extra in ((40, 100, 24), (13, 100, 0), (40, 37, 8), (1, 3, 0)):
        part = like((n, cols), F32, extra)
        op.forward(x[:n, :cols], part, 1)
        assert torch.equal(part, whole[:n, :cols])
    b = dropout(0.5, dtype=BF16)
    y = like((40, 100), BF16)
    b.forward(padded(np.ones((40, 100)), BF16), y, 1)
    assert torch.equal(y.float(), whole)
    op.close()
    b.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(dtype):
    rng = np.random.default_rng(4)
    x, r = padded(rng.normal(size=(30, 50)), dtype), padded(rng.normal(size=(30, 50)), dtype)
    y = like((30, 50), dtype)
    op = dropout(0.25, dtype=dtype)
    op.forward(x, y, 2, residual=r)
    a, b = x.clone(), r.clone()
    a, b = padded(host(a), dtype), padded(host(b), dtype)
    op.forward(a, a, 2, residual=r)
    op.forward(x, b, 2, residual=b)
    assert torch.equal(a, y) and torch.equal(b, y)
    op.close()


def test_a_step_on_the_device():
    """The step is read when the kernel runs: replays of a captured call take masks of their own."""
    x = padded(np.ones((20, 40)))
    op = dropout(0.5)
    want = []
    for s in range(4):
        y = like((20, 40))
        op.forward(x, y, s)
        want.append(y)
    assert not torch.equal(want[0], want[1])
    step, y = torch.zeros(1, dtype=torch.int64, device=DEV), like((20, 40))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        op.forward(x, y, step)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            op.forward(x, y, step)
            step.add_(1)
    torch.cuda.synchronize()
    for s in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[s]), s
        assert int(step.item()) == s + 1
    step.fill_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want[2])
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rates(dtype):
    """Kept shares of a large matrix within five standard deviations, by row, by column and by place in a block."""
    n, cols = 4096, 512
    x, y = torch.ones(n, cols, dtype=dtype, device=DEV), torch.zeros(n, cols, dtype=dtype, device=DEV)
    for p in (0.1, 0.5):
        op = dropout(p, seed=11, dtype=dtype)
        op.forward(x, y, 0)
        kept = (y != 0).double()
        for share, m in ((kept.mean(), n * cols), (kept.mean(0), n), (kept.mean(1), cols),
                         (kept.reshape(n, -1, 8).mean((0, 1)), n * cols // 8)):
            # five deviations, and the 5.5 of the largest of 4096 shares
            assert float((share - (1 - p)).abs().max()) < 6.5 * np.sqrt(p * (1 - p) / m)
        op.close()
