"""An AdapterTrainer used on other streams than the one it was made on: the same bits as on one stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
WIDTHS = (6, 40, 24, 100)
N = 64
SPIN = 40_000_000        # cycles, about 20 ms: inputs that are late on their stream


def batches(steps):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    out = []
    for _ in range(steps):
        x, u = torch.zeros(N, 8, device=DEV)[:, :6], torch.empty(N, 100, device=DEV)
        x.copy_(torch.rand(N, 6, generator=gen, device=DEV))
        u.uniform_(-1, 1, generator=gen)
        out.append((x, u, torch.randint(-1, 3, (N,), generator=gen, device=DEV).to(torch.int32)))
    torch.cuda.synchronize()
    return out


def trainer(**kw):
    from paper_2309_16743_amd import Surrogate
    from paper_2309_16743_amd.finetune import AdapterTrainer
    sur = Surrogate(WIDTHS, seed=3, max_batch=N)
    t = AdapterTrainer(sur, n_ensembles=3, rank=5, batch=N, lr=1e-2, seed=1, **kw)
    sur.close()
    torch.cuda.synchronize()
    return t


def state(t):
    return [p.clone() for p in t.params + t.m + t.v] + [t.loss.clone(), t.norm.clone()]


def plain_run(data):
    t = trainer()
    losses = []
    for b in data:
        t.train_step(*b)
        losses.append(t.loss.clone())
    y = torch.empty(N, 100, device=DEV)
    t.predict(data[0][0], data[0][2], y)
    torch.cuda.synchronize()
    out = state(t), losses, y
    t.close()
    return out


def late(b):
    """Copies of a batch that the current stream fills only after a while."""
    new = (torch.zeros(N, 8, device=DEV)[:, :6], torch.zeros(N, 100, device=DEV),
           torch.zeros(N, dtype=torch.int32, device=DEV))
    torch.cuda._sleep(SPIN)
    for a, c in zip(new, b):
        a.copy_(c)
    return new


@pytest.mark.parametrize("own_stream", [False, True])
def test_steps_follow_the_callers_stream(own_stream):
    """Inputs that the current stream makes late, results read on it, another stream for every step."""
    data = batches(5)
    want, losses, y_want = plain_run(data)
    t = trainer(stream=torch.cuda.Stream()) if own_stream else trainer()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got, keep = [], []
    for i, b in enumerate(data):
        with torch.cuda.stream(sides[i % 2]):
            keep.append(late(b))
            t.train_step(*keep[-1])
            got.append(t.loss.clone())
    with torch.cuda.stream(sides[0]):
        x, _, ids = late(data[0])
        y = torch.zeros(N, 100, device=DEV)
        t.predict(x, ids, y)
        y = y.clone()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, losses))
    assert all(torch.equal(a, b) for a, b in zip(state(t), want)) and torch.equal(y, y_want)
    t.close()


@pytest.mark.parametrize("own_stream", [False, True])
def test_freed_inputs_are_not_reused_while_a_step_reads_them(own_stream):
    """Inputs dropped right after the call and their memory filled anew on the caller's stream, behind work that
    keeps a trainer's own stream busy."""
    data = batches(4)
    want, _, _ = plain_run(data)
    t = trainer(stream=torch.cuda.Stream()) if own_stream else trainer()
    for b in data:
        new = [a.clone(memory_format=torch.preserve_format) for a in b[1:]]
        x = torch.zeros(N, 8, device=DEV)[:, :6]
        x.copy_(b[0])
        if own_stream:
            with torch.cuda.stream(t.stream):
                torch.cuda._sleep(SPIN)
        t.train_step(x, *new)
        del x, new
        for size in (N * 8, N * 100, N):
            torch.full((size,), float("nan"), device=DEV)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(state(t), want))
    t.close()


@pytest.mark.parametrize("own_stream", [False, True])
def test_a_captured_step(own_stream):
    """A step captured on the stream that torch captures on, replayed, eager steps on another stream between."""
    data = batches(5)
    want, losses, _ = plain_run(data)
    t = trainer(stream=torch.cuda.Stream()) if own_stream else trainer()
    cells = [a.clone(memory_format=torch.preserve_format) for a in data[0]]
    x = torch.zeros(N, 8, device=DEV)[:, :6]
    x.copy_(data[0][0])
    cells[0] = x
    t.train_step(*cells)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.train_step(*cells)
    side = torch.cuda.Stream()
    for i in range(1, 5):
        for a, b in zip(cells, data[i]):
            a.copy_(b)
        torch.cuda.synchronize()
        if i == 3:
            with torch.cuda.stream(side):
                t.train_step(*cells)
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t.loss, losses[i]), i
    assert all(torch.equal(a, b) for a, b in zip(state(t), want))
    t.close()


def test_a_captured_step_of_many_values():
    """Outputs whose loss takes more than one block's sum: eight replays against eager steps of a second trainer,
    eager work on other memory and synchronizations between them."""
    from paper_2309_16743_amd import Surrogate
    from paper_2309_16743_amd.finetune import AdapterTrainer
    n, widths = 256, (6, 32, 30_000)
    sur = Surrogate(widths, seed=3, max_batch=n)
    a, b = (AdapterTrainer(sur, n_ensembles=2, rank=3, batch=n, lr=1e-2, seed=1) for _ in range(2))
    sur.close()
    gen = torch.Generator(device=DEV)
    gen.manual_seed(6)
    x, u = torch.zeros(n, 8, device=DEV)[:, :6], torch.zeros(n, 30_000, device=DEV)
    ids = torch.zeros(n, dtype=torch.int32, device=DEV)
    for t in (a, b):
        t.train_step(x, u, ids)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.train_step(x, u, ids)
    other = torch.empty(1 << 22, device=DEV)
    for i in range(8):
        x.copy_(torch.rand(n, 6, generator=gen, device=DEV))
        u.uniform_(-1, 1, generator=gen)
        ids.copy_(torch.randint(-1, 2, (n,), generator=gen, device=DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        other.normal_(generator=gen).square_().sum()
        b.train_step(x, u, ids)
        torch.cuda.synchronize()
        assert torch.equal(a.loss, b.loss) and torch.equal(a.norm, b.norm), i
        assert all(torch.equal(p, q) for p, q in zip(a.params, b.params)), i
    a.close()
    b.close()
