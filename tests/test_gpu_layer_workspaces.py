"""A call is refused under capture (and replaces workspaces outside of it) only if it keeps more between its launches
than the object's workspace holds, whatever the number of its rows."""
import numpy as np
import pytest
import torch

from layer_checks import DEV, like, padded, vector

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ot():
    import paper_2309_16743_amd as ot
    return ot


def captured(call):
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        call()
    return graph


def replayed(call, outs, wants):
    """The captured call gives the eager one's bits at every replay, with eager work between them."""
    graph = captured(call)
    for _ in range(3):
        for t in outs:
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, want in zip(outs, wants):
            assert torch.equal(t, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("c,g", [(64, 8), (30, 3)])          # a team of lanes, a slab
def test_norm_input_gradients_alone(ot, c, g, dtype):
    """dx of groups that one launch holds keeps nothing."""
    n, prec = 50, ot.OT_BF16 if dtype == BF16 else ot.OT_FP32
    rng = np.random.default_rng(0)
    x, dy = padded(rng.normal(size=(n, c)), dtype), padded(rng.normal(size=(n, c)), dtype)
    y, stats, want, dx = like((n, c), dtype), torch.zeros(n, g, 2, device=DEV), like((n, c), dtype), like((n, c), dtype)
    whole, none = (ot.GroupNorm(c, g, precision=prec, max_samples=k) for k in (n, 0))
    whole.forward(x, y, stats=stats)
    whole.backward(x, stats, dy, dx=want)
    replayed(lambda: none.backward(x, stats, dy, dx=dx), [dx], [want])
    for op in (whole, none):
        op.close()


def test_norm_sums_of_many_samples(ot):
    """Sums over teams and slabs need no more from 1024 samples on."""
    n, c, g = 5000, 64, 8
    rng = np.random.default_rng(1)
    x, dy = padded(rng.normal(size=(n, c))), padded(rng.normal(size=(n, c)))
    stats = torch.zeros(n, g, 2, device=DEV)
    whole, part = (ot.GroupNorm(c, g, max_samples=k) for k in (n, 1024))
    whole.forward(x, like((n, c)), stats=stats)
    out, want = ([like((n, c)), vector(np.zeros(c)), vector(np.zeros(c))] for _ in range(2))
    back = lambda op, o: op.backward(x, stats, dy, dx=o[0], dweight=o[1], dbias=o[2])
    back(whole, want)
    replayed(lambda: back(part, out), out, want)
    for op in (whole, part):
        op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dense_gradients_that_keep_nothing(ot, dtype):
    """No activation and products that are not split."""
    n, n_in, n_out = 40, 64, 64
    prec = ot.OT_BF16 if dtype == BF16 else ot.OT_FP32
    rng = np.random.default_rng(2)
    x, w, dy = (padded(rng.normal(size=s), dtype) for s in ((n, n_in), (n_out, n_in), (n, n_out)))
    whole, none = (ot.DenseLayer(n_in, n_out, precision=prec, max_rows=k) for k in (n, 0))
    out, want = ([like((n, n_in), dtype), like((n_out, n_in))] for _ in range(2))
    back = lambda op, o: op.backward(x, w, dy, dx=o[0], dw=o[1])
    back(whole, want)
    replayed(lambda: back(none, out), out, want)
    for op in (whole, none):
        op.close()


def test_what_needs_more_is_refused(ot):
    """A split weight gradient, dz, and split norm passes beyond what the object holds: refused under capture, with the
    outputs as they were; the same calls run outside of it."""
    rng = np.random.default_rng(3)
    n, n_in, n_out = 3000, 64, 64
    x, w, dy = (padded(rng.normal(size=s)) for s in ((n, n_in), (n_out, n_in), (n, n_out)))
    dw, dx, y = like((n_out, n_in)), like((n, n_in)), like((2, 400, 48))
    maps = padded(rng.normal(size=(2, 400, 48)))
    plain, silu = ot.DenseLayer(n_in, n_out, max_rows=0), ot.DenseLayer(n_in, n_out, activation=ot.OT_ACT_SILU, max_rows=8)
    gn = ot.GroupNorm(48, 2, positions=400, max_samples=1)
    calls = (lambda: plain.backward(x, None, dy, dw=dw), lambda: silu.backward(None, w, dy, pre=dy, dx=dx),
             lambda: gn.forward(maps, y))

    def refuse():
        for call in calls:
            with pytest.raises(ot.OTError) as e:
                call()
            assert e.value.status == ot.OT_E_STATE
        mark.add_(1.0)                                       # (a graph with something in it)

    mark = torch.zeros(1, device=DEV)
    graph = captured(refuse)
    graph.replay()
    torch.cuda.synchronize()
    assert float(mark) == 1.0 and all(bool((t == 7.0).all()) for t in (dw, dx, y))
    for call in calls:
        call()
    torch.cuda.synchronize()
    assert not any(bool((t == 7.0).all()) for t in (dw, dx, y))
    for op in (plain, silu, gn):
        op.close()
