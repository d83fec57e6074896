"""The layers' calls refuse bad arguments without touching their outputs, and keep to the rules of
capture, streams and workspaces."""
import numpy as np
import pytest
import torch

from layer_checks import DEV, host, like, padded, vector

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ot():
    import paper_2309_16743_amd as ot
    return ot


def refused(ot, call, word):
    with pytest.raises((ot.OTError, ValueError), match=word):
        call()


def test_dense(ot):
    op = ot.DenseLayer(12, 20, activation=ot.OT_ACT_SILU, max_rows=8)
    x, w, y = padded(np.ones((4, 12))), padded(np.ones((20, 12))), like((4, 20))
    big = torch.zeros(4, 64, device=DEV)
    for bad, word in ((big[:, 1:13], "16-byte"), (big[:, :11], "x"), (torch.zeros(4, 13, device=DEV)[:, :12], "leading"),
                      (x[:1].expand(4, 12), "leading"), (x.to(BF16), "x"), (x.cpu(), "x"), (x.t(), "x")):
        refused(ot, lambda: op.forward(bad, w, y), word)
    refused(ot, lambda: op.forward(x, w[:19], y), "w")
    refused(ot, lambda: op.forward(x, w, y.half()), "y")
    refused(ot, lambda: op.forward(x, w, y, bias=vector(np.zeros(19))), "bias")
    refused(ot, lambda: op.forward(x, w, y, residual=y.to(BF16)), "residual")
    refused(ot, lambda: op.forward(x, w, y, pre=like((4, 20), BF16)), "pre")
    refused(ot, lambda: op.backward(x, w, y, dx=like((4, 12))), "pre")
    refused(ot, lambda: op.backward(None, w, y, pre=y, dw=like((20, 12))), "dw needs x")
    refused(ot, lambda: op.backward(x, None, y, pre=y, dx=like((4, 12))), "dx needs w")
    refused(ot, lambda: op.backward(x, w, y, pre=y, dw=like((20, 12), BF16)), "dw")
    refused(ot, lambda: op.backward(x, w, y, pre=y, dbias=vector(np.zeros(21))), "dbias")
    torch.cuda.synchronize()
    assert (host(y) == 7).all()
    op.close()


def test_norm(ot):
    op = ot.GroupNorm(24, 3, positions=5, max_samples=2)
    x, y, st = padded(np.ones((2, 5, 24))), like((2, 5, 24)), torch.zeros(2, 3, 2, device=DEV)
    for bad, word in ((x[:, :4], "x"), (x.reshape(10, 24), "x"), (x.to(BF16), "x"), (x.cpu(), "x"),
                      (torch.zeros(2, 6, 24, device=DEV)[:, :5], "follow"), (x[:1].expand(2, 5, 24), "follow"),
                      (torch.zeros(2, 5, 25, device=DEV)[..., :24], "leading"),
                      (torch.zeros(2, 5, 32, device=DEV)[..., 1:25], "16-byte")):
        refused(ot, lambda: op.forward(bad, y), word)
    refused(ot, lambda: op.forward(x, y, weight=vector(np.ones(23))), "weight")
    refused(ot, lambda: op.forward(x, y, stats=torch.zeros(2, 3, device=DEV)), "stats")
    refused(ot, lambda: op.forward(x, y, stats=torch.zeros(2, 3, 2, device=DEV, dtype=torch.float64)), "stats")
    refused(ot, lambda: op.forward(x, y[:1]), "y")
    refused(ot, lambda: op.backward(x, None, y, dx=like((2, 5, 24))), "stats")
    refused(ot, lambda: op.backward(x, st, y, dweight=vector(np.ones(5))), "dweight")
    torch.cuda.synchronize()
    assert (host(y) == 7).all()
    op.close()


def test_dropout(ot):
    op = ot.Dropout(0.5, 1)
    x, y = padded(np.ones((3, 10))), like((3, 10))
    refused(ot, lambda: op.forward(x, like((3, 9)), 0), "y")
    refused(ot, lambda: op.forward(x, like((3, 10), BF16), 0), "y")
    refused(ot, lambda: op.forward(x, y, -1), "step")
    refused(ot, lambda: op.forward(x, y, 1 << 32), "step")
    refused(ot, lambda: op.forward(x, y, torch.zeros(1, device=DEV)), "step")
    refused(ot, lambda: op.forward(x, y, torch.zeros(1, dtype=torch.int64)), "step")
    refused(ot, lambda: op.forward(x, y, 0, residual=like((2, 10))), "residual")
    refused(ot, lambda: op.backward(x[:, 1:], y[:, 1:], 0), "16-byte")
    refused(ot, lambda: ot.Dropout(0.5, -1), "seed")
    refused(ot, lambda: ot.Dropout(0.5, 1, site=1 << 32), "site")
    torch.cuda.synchronize()
    assert (host(y) == 7).all()
    op.close()


def capture(stream, call):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    return graph


def test_workspaces_under_capture(ot):
    """A captured call that needs larger workspaces is refused; one that has them replays right after the object
    has replaced them for a larger eager call; two graphs of one object share them."""
    rng = np.random.default_rng(0)
    op = ot.DenseLayer(40, 30, activation=ot.OT_ACT_GELU, precision=ot.OT_BF16, max_rows=16)
    gn = ot.GroupNorm(48, 1, positions=400, max_samples=1)
    make = lambda n: [padded(rng.normal(size=s), BF16) for s in ((n, 40), (30, 40), (n, 30), (n, 30))]
    small, large = make(16), make(400)
    out = lambda n: (like((n, 40), BF16), like((30, 40)), vector(np.zeros(30)))
    s_out, l_out, want = out(16), out(400), out(16)
    back = lambda t, o: op.backward(t[0], t[1], t[2], pre=t[3], dx=o[0], dw=o[1], dbias=o[2])
    x1, x3 = padded(rng.normal(size=(1, 400, 48))), padded(rng.normal(size=(3, 400, 48)))
    y1, y3, y_want = like((1, 400, 48)), like((3, 400, 48)), like((1, 400, 48))
    back(small, want)
    gn.forward(x1, y_want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        def refuse():
            for call in (lambda: back(large, l_out), lambda: gn.forward(x3, y3)):
                with pytest.raises(ot.OTError) as e:
                    call()
                assert e.value.status == ot.OT_E_STATE
            s_out[0].zero_()                               # (a graph with something in it)
        capture(stream, refuse)
        first = capture(stream, lambda: back(small, s_out))
        second = capture(stream, lambda: gn.forward(x1, y1))
        third = capture(stream, lambda: (back(small, s_out), gn.forward(x1, y1)))
    torch.cuda.synchronize()
    back(large, l_out)                                     # new workspaces; the graphs keep theirs
    gn.forward(x3, y3)
    junk = torch.full((1 << 22,), float("nan"), device=DEV)
    for graphs in ((first, second), (third,), (second, first, third)):
        for t in (*s_out, y1):
            t.fill_(3.0)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y1, y_want)
        for a, b in zip(s_out, want):
            assert torch.equal(a, b)
    del junk
    op.close()
    gn.close()


def test_another_stream(ot):
    """Calls run on the current stream, or on the one given."""
    rng = np.random.default_rng(1)
    op = ot.DenseLayer(64, 64, max_rows=0)
    x, w = padded(rng.normal(size=(32, 64))), padded(rng.normal(size=(64, 64)))
    want, y = like((32, 64)), like((32, 64))
    op.forward(x, w, want)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for how in ("current", "given"):
        y.fill_(7.0)
        late = torch.zeros_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)
            late.copy_(x)
            if how == "current":
                op.forward(late, w, y)
        if how == "given":
            op.forward(late, w, y, stream=stream)
        stream.synchronize()
        assert torch.equal(y, want), how
    op.close()


def test_rows_out_of_range(ot):
    """Numbers of rows that the headers exclude are refused before anything is read."""
    t = torch.zeros(16, device=DEV)
    p, st = t.data_ptr(), torch.cuda.current_stream().cuda_stream
    dense, norm, drop = ot.DenseLayer(2048, 8, max_rows=0), ot.GroupNorm(64, 2, positions=1 << 12, max_samples=0), ot.Dropout(0.5, 1)
    lib, e = ot.load(), ot.OT_E_INVAL
    for n, word in ((-1, b"n outside"), ((1 << 26) + 1, b"n outside"), (1 << 26, b"2^36")):
        assert lib.dense_forward(dense.handle, p, 2048, p, 2048, None, None, 0, n, p, 8, 0, None, 0, st) == e
        assert word in lib.ot_last_error()
        assert lib.dense_backward(dense.handle, p, 2048, p, 2048, n, p, 8, None, 0, p, 2048, None, 0, None, st) == e
        assert word in lib.ot_last_error()
        assert lib.norm_forward(norm.handle, p, 64, None, None, n, p, 64, None, st) == e
        assert word in lib.ot_last_error()
        assert lib.norm_backward(norm.handle, p, 64, None, None, n, p, p, 64, p, 64, None, None, st) == e
        assert word in lib.ot_last_error()
    for n, cols in ((-1, 4), (4, -1), (1 << 31, 4), (4, 1 << 31)):
        assert lib.dropout_forward(drop.handle, p, 4, None, 0, n, cols, p, 4, 0, None, st) == e
        assert lib.dropout_backward(drop.handle, p, 4, n, cols, p, 4, 0, None, st) == e
        assert b"outside" in lib.ot_last_error()
    for o in (dense, norm, drop):
        o.close()
