"""The dense layer against the 64-bit reference (tolerances: layer_checks)."""
import numpy as np
import pytest
import torch

from layer_checks import DEV, U, close, half, host, like, padded, padding_kept, vector
from layer_sizes import DENSE
from oracle import layers as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ACTS = ["none", "relu", "silu", "gelu"]


def layer(n_in, n_out, dtype, name="none", max_rows=4096):
    import paper_2309_16743_amd as ot
    return ot.DenseLayer(n_in, n_out, precision=ot.OT_BF16 if dtype == BF16 else ot.OT_FP32,
                         activation=ACTS.index(name), max_rows=max_rows)


def problem(n, n_in, n_out, dtype, seed, extra=0):
    rng = np.random.default_rng(seed)
    x = padded(rng.normal(size=(n, n_in)), dtype, extra)
    w = padded(rng.normal(size=(n_out, n_in)) / np.sqrt(n_in), dtype, extra)
    return rng, x, w, vector(rng.uniform(-0.5, 0.5, n_out))


def forward_tol(x, w, b, r, y, y_type, k):
    """Of z: the sum's; of y: the same through a slope of at most 1.13, the activation's own, the residual's sum."""
    s = np.abs(x) @ np.abs(w).T + (0 if b is None else np.abs(b))
    z = (4 * np.sqrt(k) + 8) * U * s
    return z, 1.13 * z + 80 * U * (np.abs(y) + (0 if r is None else np.abs(r))) + half(y_type) * np.abs(y)


@pytest.mark.parametrize("dtype,y_type", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("i", range(len(DENSE)))
def test_forward(i, dtype, y_type):
    n, n_in, n_out = DENSE[i]
    name, extra = ACTS[i % 4], 8 * (i % 3)
    rng, x, w, b = problem(n, n_in, n_out, dtype, 10 + i, extra)
    b = b if i % 5 else None
    r = padded(rng.normal(size=(n, n_out)), y_type, extra) if i % 2 else None
    y = like((n, n_out), y_type, extra)
    pre = like((n, n_out), dtype, extra) if i % 3 else None
    op = layer(n_in, n_out, dtype, name, 0)
    op.forward(x, w, y, bias=b, residual=r, pre=pre)
    hx, hw = host(x), host(w)
    hb, hr = None if b is None else host(b), None if r is None else host(r)
    want, z = ref.dense(hx, hw, hb, hr, name)
    tz, ty = forward_tol(hx, hw, hb, hr, want, y_type, n_in)
    close(y, want, ty, "y")
    padding_kept(y, 7.0)
    if pre is not None:
        close(pre, z, tz + half(dtype) * np.abs(z), "pre")
        padding_kept(pre, 7.0)
    op.close()


def backward_tols(x, w, dy, pre, name, k_dx, k_dw, dtype=F32):
    """Sums over absolute values; dz is off by 40 u of dy and rounded by u.  A bf16 dx takes two bf16 terms of
    silu's and gelu's dz, which leave half a step of half a step of it: 2^-18 = 64 u."""
    a = np.abs(dy) if pre is None or name == "relu" else 1.13 * np.abs(dy)
    if name in ("silu", "gelu"):
        extra = 45
    else:
        extra = 0
    s_dx, s_dw, s_db = a @ np.abs(w), a.T @ np.abs(x), a.sum(0)
    f = lambda k: (4 * np.sqrt(k) + 8 + extra) * U
    return (f(k_dx) + (64 * U if extra and dtype == BF16 else 0)) * s_dx, f(k_dw) * s_dw, f(k_dw) * s_db


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(DENSE)))
def test_backward(i, dtype):
    n, n_in, n_out = DENSE[i]
    name, extra = ACTS[(i + 1) % 4], 8 * (i % 3)
    rng, x, w, _ = problem(n, n_in, n_out, dtype, 40 + i, extra)
    dy = padded(rng.normal(size=(n, n_out)), dtype, extra)
    pre = padded(rng.normal(size=(n, n_out)), dtype) if name != "none" else None
    dx, dw, db = like((n, n_in), dtype, extra), like((n_out, n_in), F32, extra), vector(np.full(n_out, 7.0))
    op = layer(n_in, n_out, dtype, name, n)
    op.backward(x, w, dy, pre=pre, dx=dx, dw=dw, dbias=db)
    hx, hw, hdy = host(x), host(w), host(dy)
    hp = None if pre is None else host(pre)
    want = ref.dense_back(hx, hw, hdy, hp, name)
    tol = backward_tols(hx, hw, hdy, hp, name, n_out, n, dtype)
    close(dx, want[0], tol[0] + half(dtype) * np.abs(want[0]), "dx")
    close(dw, want[1], tol[1] + U * np.abs(want[1]), "dw")
    close(db, want[2], tol[2] + U * np.abs(want[2]), "dbias")
    padding_kept(dx, 7.0)
    padding_kept(dw, 7.0)
    # each gradient alone has the same bits
    for kind in ("dx", "dw", "dbias"):
        one = {"dx": like((n, n_in), dtype), "dw": like((n_out, n_in)), "dbias": vector(np.zeros(n_out))}[kind]
        op.backward(x if kind == "dw" else None, w if kind == "dx" else None, dy, pre=pre, **{kind: one})
        assert torch.equal(one, {"dx": dx, "dw": dw, "dbias": db}[kind]), kind
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_training_pair_with_one_product(dtype):
    """forward's pre goes into backward: gradients of the whole function against the 64-bit ones and against
    differences of the function the device computes."""
    n, n_in, n_out, name = 12, 20, 9, "gelu"
    rng, x, w, b = problem(n, n_in, n_out, F32, 3)
    if dtype == BF16:
        x, w = padded(host(x), BF16), padded(host(w), BF16)
    dy = padded(rng.normal(size=(n, n_out)), dtype)
    op = layer(n_in, n_out, dtype, name)
    y, pre = like((n, n_out)), like((n, n_out), dtype)
    op.forward(x, w, y, bias=b, pre=pre)
    dw, db = like((n_out, n_in)), vector(np.zeros(n_out))
    op.backward(x, w, dy, pre=pre, dw=dw, dbias=db)
    hx, hw, hdy = host(x), host(w), host(dy)
    z = ref.dense(hx, hw, host(b), None, name)[1]
    # pre's rounding moves a slope by at most 0.8 (the largest second derivative of gelu) times half an eps of z
    dw_ref, db_ref = ref.dense_back(hx, hw, hdy, z, name)[1:]
    move = np.abs(hdy) * (0.8 * (half(dtype) + 40 * U) * np.abs(z) + 60 * U)
    close(dw, dw_ref, move.T @ np.abs(hx) + 1e-6, "dw")
    close(db, db_ref, move.sum(0) + 1e-6, "dbias")
    if dtype == F32:
        # a difference over 2 h: rounding of the outputs (1e-6 of values of size 1, summed with 108 weights of size
        # 1) over 2 h, and a curvature below 2 h^2 times the same sum
        h = 2.0 ** -6
        for at in ((0, 0), (4, 11), (8, 19)):
            vals = []
            for sign in (1, -1):
                moved = padded(hw)
                moved[at] += sign * h
                op.forward(x, moved, y, bias=b)
                vals.append((host(y) * hdy).sum())
            assert abs((vals[0] - vals[1]) / (2 * h) - host(dw)[at]) < 1e-6 * 108 / h + 2 * h * h * 108
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_in,n_out", [(77, 13), (1, 401), (2047, 1), (131, 9001)])
def test_one_row_with_any_leading_dimension(n_in, n_out, dtype):
    """One row may have a leading dimension that is no whole number of pieces: the same bits as padded ones."""
    rng, x, w, b = problem(1, n_in, n_out, dtype, 8)
    dy, pre = padded(rng.normal(size=(1, n_out)), dtype), padded(rng.normal(size=(1, n_out)), dtype)
    r = padded(rng.normal(size=(1, n_out)), dtype)
    op = layer(n_in, n_out, dtype, "silu", 1)
    got = []
    for odd in (False, True):
        f = (lambda t: t.contiguous().as_strided(t.shape, (3, 1)) if t.shape[0] == 1 else t) if odd else lambda t: t
        y, z, dx, dw = (f(like(s, t)) for s, t in (((1, n_out), dtype), ((1, n_out), dtype), ((1, n_in), dtype),
                                                  ((n_out, n_in), F32)))
        db = vector(np.zeros(n_out))
        op.forward(f(x), f(w), y, bias=b, residual=f(r), pre=z)
        op.backward(f(x), f(w), f(dy), pre=f(pre), dx=dx, dw=dw, dbias=db)
        got.append((y, z, dx, dw, db))
    for u, v in zip(*got):
        assert torch.equal(u, v)
    want, z = ref.dense(host(x), host(w), host(b), host(r), "silu")
    close(got[1][0], want, forward_tol(host(x), host(w), host(b), host(r), want, dtype, n_in)[1], "y")
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows(dtype):
    op = layer(5, 9, dtype, "silu", 4)
    x, w, y = like((0, 5), dtype), like((9, 5), dtype), like((0, 9), dtype)
    op.forward(x, w, y)
    dw, db = like((9, 5)), vector(np.full(9, 7.0))
    op.backward(x, w, y, pre=y, dx=like((0, 5), dtype), dw=dw, dbias=db)
    assert not host(dw).any() and not host(db).any()
    padding_kept(dw, 7.0)
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [3, 40, 300])
def test_the_residual_may_be_the_output(dtype, n):
    rng, x, w, b = problem(n, 70, 133, dtype, 5)
    h = padded(rng.normal(size=(n, 133)), dtype)
    y = like((n, 133), dtype)
    op = layer(70, 133, dtype, "gelu", 0)
    op.forward(x, w, y, bias=b, residual=h)
    op.forward(x, w, h, bias=b, residual=h)
    assert torch.equal(y, h)
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,n_out", [(12, 200), (70, 200), (700, 900)])
def test_rows_and_columns_keep_their_special_values(n, n_out, dtype):
    """An infinity or NaN in a row of x, a row of W, the bias or the residual reaches what the formula says and nothing
    else (finite parts keep to the tolerance); NaN passes relu."""
    n_in = 45
    for name in ("none", "relu"):
        rng, x, w, b = problem(n, n_in, n_out, dtype, 6)
        r = padded(rng.normal(size=(n, n_out)), dtype)
        x[3, 44] = float("inf")
        x[5, 0] = float("nan")
        w[7, 2] = float("-inf")
        b[11] = float("nan")
        r[9, 13] = float("inf")
        y = like((n, n_out), dtype)
        op = layer(n_in, n_out, dtype, name, 0)
        op.forward(x, w, y, bias=b, residual=r)
        with np.errstate(invalid="ignore"):
            want = ref.dense(host(x), host(w), host(b), host(r), name)[0]
        got = host(y)
        bad = ~np.isfinite(want)
        assert bad.any() and not bad.all()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(got[bad & ~np.isnan(want)], want[bad & ~np.isnan(want)])
        hx, hw = np.nan_to_num(host(x), posinf=0), np.nan_to_num(host(w), neginf=0)
        tol = forward_tol(hx, hw, np.nan_to_num(host(b)), None, np.where(bad, 0, want), dtype, n_in)[1]
        close(np.where(bad, 0, got), np.where(bad, 0, want), tol + 80 * U * np.abs(np.where(bad, 0, host(r))))
        op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_relu_drops_infinite_gradients(dtype):
    """dy that is not finite where relu is off reaches nothing."""
    n, n_in, n_out = 40, 33, 50
    rng, x, w, _ = problem(n, n_in, n_out, dtype, 7)
    hd, hp = rng.normal(size=(n, n_out)), rng.normal(size=(n, n_out))
    dy, pre = padded(hd, dtype), padded(hp, dtype)
    clean = padded(np.where(hp > 0, hd, 0), dtype)
    off = host(pre) <= 0
    dy[torch.from_numpy(off).to(DEV)] = float("inf")
    op = layer(n_in, n_out, dtype, "relu", n)
    out = []
    for g in (dy, clean):
        dx, dw, db = like((n, n_in), dtype), like((n_out, n_in)), vector(np.zeros(n_out))
        op.backward(x, w, g, pre=pre, dx=dx, dw=dw, dbias=db)
        out.append((dx, dw, db))
    for a, b in zip(*out):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_row_offsets_past_32_bits(dtype):
    """Rows of x, W and y that lie 2^29 values apart (slices of one wide array)."""
    e = 2 if dtype == BF16 else 4
    ld, n, n_in, n_out = 1 << 29, 5, 24, 6
    if torch.cuda.mem_get_info()[0] < 3 * 6 * ld * e:
        pytest.skip("not enough memory")
    rng = np.random.default_rng(8)
    big = torch.empty(6 * ld, dtype=dtype, device=DEV)
    view = lambda at, rows, cols: torch.as_strided(big, (rows, cols), (ld, 1), at)
    x, w, y, dx = view(0, n, n_in), view(64, n_out, n_in), view(128, n, n_out), view(192, n, n_in)
    hx, hw = rng.normal(size=(n, n_in)), rng.normal(size=(n_out, n_in))
    x.copy_(torch.from_numpy(hx))
    w.copy_(torch.from_numpy(hw))
    op = layer(n_in, n_out, dtype, "none", n)
    op.forward(x, w, y)
    want = ref.dense(host(x), host(w))[0]
    close(y, want, forward_tol(host(x), host(w), None, None, want, dtype, n_in)[1])
    dw = like((n_out, n_in))
    op.backward(x, w, y, dx=dx, dw=dw)
    hx, hw, hy = host(x), host(w), host(y)
    want = ref.dense_back(hx, hw, hy)
    tol = backward_tols(hx, hw, hy, None, "none", n_out, n)
    close(dx, want[0], tol[0] + half(dtype) * np.abs(want[0]))
    close(dw, want[1], tol[1] + U * np.abs(want[1]))
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_tiles_with_offsets_past_32_bits(dtype):
    """The tiled products and the activation's backward on matrices whose rows lie 2^23 values apart, among them
    whole k tiles past 2^32 values: the same bits as with rows that follow each other."""
    ld, n, n_in, n_out = 1 << 23, 600, 200, 1000
    e = 2 if dtype == BF16 else 4
    if torch.cuda.mem_get_info()[0] < 2 * n_out * ld * e:
        pytest.skip("not enough memory")
    rng, x, w, b = problem(n, n_in, n_out, dtype, 14)
    dy, r = padded(rng.normal(size=(n, n_out)), dtype), padded(rng.normal(size=(n, n_out)), dtype)
    big = torch.empty(n_out * ld, dtype=dtype, device=DEV)
    at = [0]

    def far(t, wanted=True):
        at[0] += 2048
        v = torch.as_strided(big, tuple(t.shape), (ld, 1), at[0])
        if wanted:
            v.copy_(t)
        return v

    op = layer(n_in, n_out, dtype, "silu", n)
    got = []
    for place in (lambda t, wanted=True: t, far):
        y, pre, dx = (place(like(s, dtype), False) for s in ((n, n_out), (n, n_out), (n, n_in)))
        dw, db = like((n_out, n_in)), vector(np.zeros(n_out))
        if place is far and dtype == F32:
            dw = far(dw, False)
        px, pw = place(x), place(w)
        op.forward(px, pw, y, bias=b, residual=place(r), pre=pre)
        op.backward(px, pw, place(dy), pre=pre, dx=dx, dw=dw, dbias=db)
        got.append([t.clone() for t in (y, pre, dx, dw, db)])
    for u, v in zip(*got):
        assert torch.equal(u, v)
    op.close()


@pytest.mark.parametrize("name", ACTS)
def test_activations_and_slopes(name):
    """A layer of one weight 1 is the activation itself, its input gradient the slope: over the range where gelu's
    lower tail is a normal number, at the corner, and where exp over- or underflows."""
    z = np.concatenate([np.linspace(-12.5, 12.5, 20001), [0.0, -0.0, 1e-30, -1e-30, 80, -80, 87.5, -87.5, 1e4, -1e4, 3e38]])
    x, one = padded(z[:, None]), padded(np.ones((1, 1)))
    hx = host(x)
    n = len(z)
    y, dx = like((n, 1)), like((n, 1))
    op = layer(1, 1, F32, name, n)
    op.forward(x, one, y)
    op.backward(x, one, padded(np.ones((n, 1))), pre=x, dx=dx)
    want, slope = ref.act(hx, name), ref.slope(hx, name)
    # Phi is off by 7 u of its value, the sigmoid by 4, the products by 2; a slope adds z phi(z), of size 0.25 and
    # off by 6 u, or z s (1 - s), where 1 - s is off by u.  Sigmoids and integrals below 2^-126, the smallest normal
    # number, are taken as 0 (the device's reciprocal and exp2 have no smaller results), times |z| in y and slope.
    none = np.minimum(np.abs(hx), 200) * 2.0 ** -126
    close(y, want, 10 * U * np.abs(want) + none, "y")
    close(dx, slope, 10 * U * (np.abs(slope) + 0.3) + none if name in ("silu", "gelu") else 0, "slope")
    # NaN, and infinities as the formula has them
    x = padded(np.array([[np.nan], [np.inf], [-np.inf]]))
    y = like((3, 1))
    op.forward(x, one, y)
    with np.errstate(invalid="ignore"):
        want = ref.act(host(x), name)
    got = host(y)
    assert np.isnan(got[0, 0]) and got[1, 0] == np.inf
    assert name in ("silu", "gelu") or got[2, 0] == want[2, 0]
    op.close()


@pytest.mark.parametrize("n,n_in,n_out", [(40, 33, 50), (700, 45, 900)])
def test_values_past_2_to_60(n, n_in, n_out):
    """fp32 values whose bf16 terms would overflow or lose themselves keep the tolerance."""
    rng, x, w, b = problem(n, n_in, n_out, F32, 11)
    x[3] *= 2.0 ** 70
    x[5, 7] = 3e37
    w[9] *= 2.0 ** -60
    dy = padded(rng.normal(size=(n, n_out)))
    dy[4] *= 2.0 ** 65
    op = layer(n_in, n_out, F32, "none", n)
    y, dx, dw, db = like((n, n_out)), like((n, n_in)), like((n_out, n_in)), vector(np.zeros(n_out))
    op.forward(x, w, y, bias=b)
    op.backward(x, w, dy, dx=dx, dw=dw, dbias=db)
    hx, hw, hdy, hb = host(x), host(w), host(dy), host(b)
    want = ref.dense(hx, hw, hb)[0]
    close(y, want, forward_tol(hx, hw, hb, None, want, F32, n_in)[1], "y")
    want = ref.dense_back(hx, hw, hdy)
    tol = backward_tols(hx, hw, hdy, None, "none", n_out, n)
    for got, v, t in zip((dx, dw, db), want, tol):
        close(got, v, t + U * np.abs(v))
    op.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("n,n_in,n_out", [(40, 33, 50), (700, 45, 900), (600, 300, 260)])
def test_a_gradient_that_is_not_finite_stays_in_its_row_and_column(n, n_in, n_out, name, dtype):
    """One NaN (and, where dz is whole, one infinity) of dy: its row of dx, its row of dw, its dbias."""
    rng, x, w, _ = problem(n, n_in, n_out, dtype, 12)
    hp = rng.normal(size=(n, n_out))
    hp[7, 11] = hp[9, 13] = 0.5
    dy, pre = padded(rng.normal(size=(n, n_out)), dtype), padded(hp, dtype)
    clean = padded(host(dy), dtype)
    dy[7, 11] = float("nan")
    whole = name in ("none", "relu") or dtype == F32
    if whole:
        dy[9, 13] = float("inf")
    op = layer(n_in, n_out, dtype, name, n)
    out = []
    for g in (dy, clean):
        dx, dw, db = like((n, n_in), dtype), like((n_out, n_in)), vector(np.zeros(n_out))
        op.backward(x, w, g, pre=None if name == "none" else pre, dx=dx, dw=dw, dbias=db)
        out.append([host(t) for t in (dx, dw, db)])
    rows, cols = np.zeros(n, bool), np.zeros(n_out, bool)
    rows[7] = cols[11] = True
    assert np.isnan(out[0][0][7]).all() and np.isnan(out[0][1][11]).all() and np.isnan(out[0][2][11])
    if whole:
        rows[9] = cols[13] = True
        with np.errstate(invalid="ignore"):
            assert np.array_equal(out[0][0][9], np.inf * np.sign(host(w)[13]))
            assert np.array_equal(out[0][1][13], np.inf * np.sign(host(x)[9]))
        assert out[0][2][13] == np.inf
    # the others' sums may be formed another way (fp32 tiles with such a value are summed again), within the tolerance
    hx, hw, hd = host(x), host(w), host(clean)
    tol = backward_tols(hx, hw, hd, None if name == "none" else host(pre), name, n_out, n, dtype)
    close(out[0][0][~rows], out[1][0][~rows], 2 * tol[0][~rows] + 2 * half(dtype) * np.abs(out[1][0][~rows]), "dx")
    close(out[0][1][~cols], out[1][1][~cols], 2 * tol[1][~cols], "dw")
    close(out[0][2][~cols], out[1][2][~cols], 2 * tol[2][~cols], "dbias")
    op.close()


@pytest.mark.parametrize("name", ["none", "relu", "gelu"])
@pytest.mark.parametrize("n,n_in,n_out", [(300, 260, 41000), (100, 1030, 40000), (257, 256, 131072)])
def test_long_weight_gradients(n, n_in, n_out, name):
    """bf16 weight gradients of several rounds of blocks (ragged tiles, k with and without a rest): right in every
    tile, and the same bits each time."""
    rng, x, _, _ = problem(n, n_in, n_out, BF16, 13)
    dy = padded(rng.normal(size=(n, n_out)), BF16)
    pre = None if name == "none" else padded(rng.normal(size=(n, n_out)), BF16)
    op = layer(n_in, n_out, BF16, name, n)
    dw = like((n_out, n_in))
    op.backward(x, None, dy, pre=pre, dw=dw)
    first = dw.clone()
    for _ in range(3):
        dw.fill_(7.0)
        op.backward(x, None, dy, pre=pre, dw=dw)
        assert torch.equal(dw, first)
    padding_kept(dw, 7.0)
    # the 64-bit reference, some columns at a time
    hx = host(x)
    for c in range(0, n_out, 8192):
        s = slice(c, min(n_out, c + 8192))
        hd, hp = host(dy[:, s]), None if pre is None else host(pre[:, s])
        want = ref.dense_back(hx, np.zeros((hd.shape[1], n_in)), hd, hp, name)[1]
        a = np.abs(hd) * (1.13 if name == "gelu" else 1)
        tol = (4 * np.sqrt(n) + 8 + (45 if name == "gelu" else 0)) * U * (a.T @ np.abs(hx))
        close(dw[s], want, tol + U * np.abs(want), "dw")
    op.close()
