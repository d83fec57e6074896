"""The adapters' 64-bit reference against central differences of its own forward."""
import numpy as np
import pytest

from oracle import adapters


def problem(seed, n=7, n_in=6, n_out=9, r=3, g=4):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(n, n_in))
    return {"x": x, "w": rng.normal(size=(n_out, n_in)), "down": rng.normal(size=(g, r, n_in)),
            "up": rng.normal(size=(g, r, n_out)), "scale": rng.uniform(0.5, 2, g),
            "ids": np.array([2, -1, 0, 2, 9, 0, 2])[:n], "bias": rng.normal(size=n_out)}


@pytest.mark.parametrize("seed", range(3))
def test_gradients_match_differences(seed):
    """The forward is a polynomial of degree 2 in (down, up) along each of the directions below, so
    central differences with step 1e-3 are exact up to rounding: 1e-16 * |loss| / 1e-3."""
    p = problem(seed)
    rng = np.random.default_rng(100 + seed)
    target = rng.normal(size=(7, 9))

    def loss(x, down, up):
        return float(np.sum(adapters.forward(x, p["w"], p["bias"], down, up, p["scale"], p["ids"])[0] * target))

    _, t = adapters.forward(p["x"], p["w"], p["bias"], p["down"], p["up"], p["scale"], p["ids"])
    grads = adapters.backward(p["x"], p["w"], p["down"], p["up"], p["scale"], p["ids"], target, t)
    args = {"down": p["down"], "up": p["up"], "x": p["x"]}
    for name, grad in zip(("down", "up", "x"), grads):
        d = rng.normal(size=args[name].shape)
        hi, lo = dict(args), dict(args)
        hi[name], lo[name] = args[name] + 1e-3 * d, args[name] - 1e-3 * d
        diff = (loss(hi["x"], hi["down"], hi["up"]) - loss(lo["x"], lo["down"], lo["up"])) / 2e-3
        assert abs(diff - float(np.sum(grad * d))) < 1e-9 * (1 + abs(diff))


def test_rows_without_adapter_pass_the_layer_alone():
    p = problem(0)
    y, t = adapters.forward(p["x"], p["w"], p["bias"], p["down"], p["up"], p["scale"], p["ids"])
    assert np.allclose(y[[1, 4]], (p["x"] @ p["w"].T + p["bias"])[[1, 4]]) and not t[[1, 4]].any()


def test_clip():
    g = [np.array([3.0]), np.array([[4.0]])]
    assert adapters.clip(g, 1.0) == (5.0, 0.2) and adapters.clip(g, 6.0) == (5.0, 1.0)
    assert adapters.clip([np.zeros(3)], 1.0) == (0.0, 1.0)
    assert adapters.clip([np.array([np.inf])], 1.0)[1] == 1.0
