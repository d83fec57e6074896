"""Inputs, tolerances and comparisons of the layers' GPU tests.

With u = 2^-24 and S the same sum taken over absolute values, a sum of k products
rounded in fp32 is off by at most about 4 sqrt(k) u S (roundings that do not
conspire, four deviations wide) and a few u of S for joins.  A result of type t adds
eps(t) / 2 of its value.  Values of the activations and their slopes: exp and erfc of the
device are good to a few u; erfc(-z / sqrt 2) takes an argument rounded by u, which its
slope turns into at most (2 t^2 + 1) u of its value, t = |z| / sqrt 2: 37 u for |z| <= 6, so 80 u of
the value in all; slopes are at most 1.13 and off by at most 40 u."""
import numpy as np
import torch

DEV = torch.device("cuda:0")
U = 2.0 ** -24
TINY = 2.0 ** -120


def half(dtype):
    return torch.finfo(dtype).eps / 2


def padded(a, dtype=torch.float32, extra=0, fill=float("nan")):
    """Device tensor of a's values in rows padded to whole 16-byte pieces (and `extra` more), the padding NaN."""
    a = np.asarray(a, dtype=np.float32)
    n = a.shape[-1]
    full = torch.full(a.shape[:-1] + ((n + 7) // 8 * 8 + extra,), fill, dtype=dtype, device=DEV)
    full[..., :n] = torch.from_numpy(a).to(DEV).to(dtype)
    return full[..., :n]


def like(shape, dtype=torch.float32, extra=0, fill=7.0):
    return padded(np.full(shape, fill, np.float32), dtype, extra, fill)


def vector(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DEV)


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, want, tol, what=""):
    got = host(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape
    err = np.abs(got - want)
    bad = ~(err <= tol + TINY)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off, first at {i}: {got[i]!r} for {want[i]!r}, "
                             f"tolerance {np.broadcast_to(tol, err.shape)[i]!r}")


def padding_kept(t, fill):
    """The values between a row's end and its leading dimension are as they were."""
    base = t._base if t._base is not None else t
    rest = host(base)[..., t.shape[-1]:]
    assert np.array_equal(rest, np.full_like(rest, fill), equal_nan=True)
