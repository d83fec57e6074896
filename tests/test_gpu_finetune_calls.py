"""Calls of an AdapterTrainer that it refuses, before anything of it has changed."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


@pytest.fixture
def tuner():
    from paper_2309_16743_amd import Surrogate
    from paper_2309_16743_amd.finetune import AdapterTrainer
    sur = Surrogate((6, 16, 24), seed=3, max_batch=8)
    t = AdapterTrainer(sur, n_ensembles=2, rank=3, batch=8, seed=1)
    sur.close()
    yield t
    t.close()


def rows(n):
    return torch.zeros(n, 8, device=DEV)[:, :6], torch.zeros(n, 24, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)


def test_targets_of_another_shape(tuner):
    """Targets that torch would spread over the rows or columns, and others."""
    x, u, ids = rows(5)
    before = [p.clone() for p in tuner.params]
    for bad in (u[:1], u[:, :1], u[0], u[:4], torch.zeros(24, device=DEV), torch.zeros(1, device=DEV),
                torch.zeros(5, 5, 24, device=DEV)):
        with pytest.raises(ValueError, match="u: expected"):
            tuner.train_step(x, bad, ids)
    assert tuner.adam.get_steps() == 0 and all(torch.equal(a, b) for a, b in zip(before, tuner.params))
    tuner.train_step(x, u, ids)
    assert tuner.adam.get_steps() == 1


def test_numbers_of_rows(tuner):
    for n in (0, 9):
        with pytest.raises(ValueError, match="row"):
            tuner.train_step(*rows(n))
    assert tuner.adam.get_steps() == 0
    x, y, ids = rows(0)
    tuner.predict(x, ids, y)
    for n in (1, 8):
        tuner.train_step(*rows(n))
    torch.cuda.synchronize()
    assert tuner.adam.get_steps() == 2 and bool(torch.isfinite(tuner.loss).all())


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_a_trainer_holds_the_arrays_that_a_step_needs(precision):
    """Per hidden layer one array of activations and one of their gradients for the batch; per output its values and
    their gradient; weights, adapters, gradients and moments (a quarter above their sum for paddings and the rest)."""
    from paper_2309_16743_amd import OT_BF16, OT_FP32, Surrogate
    from paper_2309_16743_amd.finetune import AdapterTrainer
    widths, batch, e = (6, 16, 100_000, 16, 8), 1000, 2 if precision == "bf16" else 4
    sur = Surrogate(widths, seed=3, max_batch=8)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    t = AdapterTrainer(sur, n_ensembles=2, rank=3, batch=batch, precision=OT_BF16 if e == 2 else OT_FP32)
    held = torch.cuda.memory_allocated() - before
    hidden = sum(2 * e * batch * w for w in widths[1:-1])
    rest = sum(e * i * o + 2 * 3 * (i + o) * (16 + (2 if e == 2 else 0)) for i, o in zip(widths, widths[1:]))
    assert held < 1.25 * (hidden + rest) + (4 << 20)
    t.close()
    sur.close()
