"""Adapters of a whole surrogate trained on mixed batches against a 64-bit loop of the same steps, and the
adapted prediction against the merged weights W + s up^T down."""
import numpy as np
import pytest
import torch

from oracle import adapters as ref

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def padded(a, extra=0):
    n = a.shape[1]
    t = torch.zeros(a.shape[0], (n + 7) // 8 * 8, device=DEV)[:, :n]
    t.copy_(torch.from_numpy(a.astype(np.float32)))
    return t


def host(t):
    return t.double().cpu().numpy()


class Reference:
    def __init__(self, tuner, lr, max_norm):
        self.w = [host(w) for w in tuner.w]
        self.b = [host(b) for b in tuner.bias]
        self.scale = host(tuner.scale)
        self.p = [host(p[..., :n]) for p, n in zip(tuner.params, self.dims(tuner))]
        self.m = [np.zeros_like(p) for p in self.p]
        self.v = [np.zeros_like(p) for p in self.p]
        self.lr, self.max_norm, self.step_no = lr, max_norm, 0

    @staticmethod
    def dims(tuner):
        return [n for i, o in zip(tuner.widths, tuner.widths[1:]) for n in (i, o)]

    def forward(self, x, ids):
        acts, ts = [x], []
        for l in range(len(self.w)):
            y, t = ref.forward(acts[-1], self.w[l], self.b[l], self.p[2 * l], self.p[2 * l + 1], self.scale, ids,
                               relu=l + 1 < len(self.w))
            acts.append(y)
            ts.append(t)
        return acts, ts

    def step(self, x, u, ids):
        acts, ts = self.forward(x, ids)
        r = acts[-1] - u
        dy = 2.0 * r / r.size
        grads = [None] * len(self.p)
        for l in range(len(self.w) - 1, -1, -1):
            grads[2 * l], grads[2 * l + 1], dy = ref.backward(acts[l], self.w[l], self.p[2 * l], self.p[2 * l + 1],
                                                              self.scale, ids, dy, ts[l], relu_input=l > 0)
        norm, c = ref.clip(grads, self.max_norm)
        self.step_no += 1
        for p, m, v, g in zip(self.p, self.m, self.v, grads):
            m += 0.1 * (c * g - m)
            v += 0.001 * ((c * g) ** 2 - v)
            p -= self.lr * (m / (1 - 0.9 ** self.step_no)) / (np.sqrt(v / (1 - 0.999 ** self.step_no)) + 1e-8)
        return float(np.mean(r * r)), norm


def batch(rng, n, d, ensembles):
    x = rng.uniform(0, 1, (n, 6)).astype(np.float32)
    u = rng.uniform(-1, 1, (n, d)).astype(np.float32)
    return x, u, rng.integers(-1, ensembles, n).astype(np.int32)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("widths", [(6, 40, 24, 100), (6, 64, 96, 50, 333)])
def test_training_follows_the_reference(widths, precision):
    """Losses and norms of five steps (fp32: sums of at most 100 fp32 roundings, 1e-5; bf16: operands
    of 2^-9, 2e-2), the adapters after them by the length of the difference against the length of the way
    they went (Adam normalises each element, so elements with gradients near zero may differ)."""
    from paper_2309_16743_amd import OT_BF16, OT_FP32, Surrogate
    from paper_2309_16743_amd.finetune import AdapterTrainer
    tol = 1e-5 if precision == "fp32" else 2e-2
    sur = Surrogate(widths, seed=3, max_batch=64)
    tuner = AdapterTrainer(sur, n_ensembles=3, rank=5, batch=70, lr=1e-2, max_norm=0.05, seed=1,
                           precision=OT_BF16 if precision == "bf16" else OT_FP32)
    model = Reference(tuner, 1e-2, 0.05)
    start = [p.copy() for p in model.p]
    rng = np.random.default_rng(0)
    for i in range(5):
        x, u, ids = batch(rng, 70 if i % 2 else 33, widths[-1], 3)
        tuner.train_step(padded(x), padded(u), torch.from_numpy(ids).to(DEV))
        loss, norm = model.step(x.astype(np.float64), u.astype(np.float64), ids)
        torch.cuda.synchronize()
        assert abs(tuner.loss.item() - loss) < tol * loss and abs(tuner.norm.item() - norm) < 5 * tol * norm, i
    assert tuner.adam.get_steps() == 5
    for p, w, s, n in zip(tuner.params, model.p, start, Reference.dims(tuner)):
        assert np.linalg.norm(host(p[..., :n]) - w) < (0.02 if precision == "fp32" else 0.3) * np.linalg.norm(w - s)
        assert not p[..., n:].any()
    tuner.close()
    sur.close()


def test_prediction_is_the_merged_layers():
    """Each row through plain layers with its ensemble's merged weights (64 bits): 1e-5 of the largest value."""
    from paper_2309_16743_amd import Surrogate
    from paper_2309_16743_amd.finetune import AdapterTrainer
    widths = (6, 48, 80, 500)
    sur = Surrogate(widths, seed=5, max_batch=64)
    tuner = AdapterTrainer(sur, n_ensembles=4, rank=3, batch=64, lr=1e-2, seed=2)
    rng = np.random.default_rng(1)
    for _ in range(4):
        x, u, ids = batch(rng, 64, 500, 4)
        tuner.train_step(padded(x), padded(u), torch.from_numpy(ids).to(DEV))
    x, _, ids = batch(rng, 50, 500, 4)
    y = padded(np.zeros((50, 500)))
    tuner.predict(padded(x), torch.from_numpy(ids).to(DEV), y)
    plain = padded(np.zeros((50, 500)))
    sur.predict(padded(x), plain)
    torch.cuda.synchronize()
    got = host(y)
    for i in range(50):
        a = x[i].astype(np.float64)
        for l in range(3):
            w = host(tuner.w[l])
            if ids[i] >= 0:
                w = w + host(tuner.scale)[ids[i]] * host(tuner.up[l][ids[i]]).T @ host(tuner.down[l][ids[i]])
            a = w @ a + host(tuner.bias[l])
            a = np.maximum(a, 0) if l < 2 else a
        assert np.max(np.abs(got[i] - a)) < 1e-5 * max(1.0, np.max(np.abs(a)))
        if ids[i] < 0:
            assert np.max(np.abs(got[i] - host(plain[i]))) < 1e-5 * max(1.0, np.max(np.abs(a)))
    with pytest.raises(ValueError):
        tuner.predict(padded(np.zeros((65, 6))), torch.zeros(65, dtype=torch.int32, device=DEV), padded(np.zeros((65, 500))))
    tuner.close()
    sur.close()
