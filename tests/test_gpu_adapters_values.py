"""Values of the adapters' products that an ordinary random test does not reach: low-rank values of more
bits than two bf16 terms hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
BF = torch.bfloat16

# rows, short side, long side, by the tile of the bf16 product that they take
FORWARD = [(5, 24, 40), (40, 24, 31_000), (200, 24, 15_400), (600, 24, 12_300), (150, 24, 61_500)]
GRADIENT = [(5, 24, 40), (40, 300, 4_200), (70, 7_700, 8_300), (300, 7_700, 8_300), (520, 20_500, 2_100)]


def bank_of(n_in, n_out, n):
    from paper_2309_16743_amd import OT_BF16, LowRankAdapters
    return LowRankAdapters(n_in, n_out, 2, 3, precision=OT_BF16, max_rows=n)


def zeros(*shape, dtype=BF):
    full = torch.zeros(*shape[:-1], (shape[-1] + 7) // 8 * 8, dtype=dtype, device=DEV)
    return full[..., :shape[-1]]


def set_long(x, down):
    """Rows x of (1, 2^-9, 2^-20) and down of (1, 1, 1), (1, 1, 0): low-rank values 1 + 2^-9 + 2^-20 and
    1 + 2^-9, which fp32 holds whole."""
    x[:, 0], x[:, 1], x[:, 2] = 1.0, 2.0 ** -9, 2.0 ** -20
    down[:, 0, :3] = 1.0
    down[:, 1, :2] = 1.0


@pytest.mark.parametrize("y_type", [BF, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,n_in,n_out", FORWARD)
def test_forward_takes_low_rank_values_whole(n, n_in, n_out, y_type):
    """W = 0 and up = (1, -1): y is the difference of the two low-rank values, 2^-20, which every
    intermediate sum holds in 24 bits; two bf16 terms of them differ by 0."""
    print(f"whole values, forward {n} {n_in} {n_out}", flush=True)
    bank = bank_of(n_in, n_out, n)
    x, w, down, up = zeros(n, n_in), zeros(n_out, n_in), zeros(3, 2, n_in), zeros(3, 2, n_out)
    set_long(x, down)
    up[:, 0], up[:, 1] = 1.0, -1.0
    ids = (torch.arange(n, device=DEV) % 3).to(torch.int32)
    y = zeros(n, n_out, dtype=y_type)
    bank.forward(x, w, down, up, ids, y)
    assert bool((y == 2.0 ** -20).all())
    bank.close()


@pytest.mark.parametrize("n,n_in,n_out", GRADIENT)
def test_input_gradient_takes_low_rank_values_whole(n, n_in, n_out):
    print(f"whole values, input gradient {n} {n_in} {n_out}", flush=True)
    bank = bank_of(n_in, n_out, n)
    x, w, down, up, dy = zeros(n, n_in), zeros(n_out, n_in), zeros(3, 2, n_in), zeros(3, 2, n_out), zeros(n, n_out)
    set_long(dy, up)
    down[:, 0], down[:, 1] = 1.0, -1.0
    ids = (torch.arange(n, device=DEV) % 3).to(torch.int32)
    dx, t = zeros(n, n_in), torch.zeros(n, 2, device=DEV)
    ddown, dup = zeros(3, 2, n_in, dtype=torch.float32), zeros(3, 2, n_out, dtype=torch.float32)
    bank.backward(x, w, down, up, ids, dy, t, ddown, dup, dx=dx)
    assert bool((dx == 2.0 ** -20).all())
    bank.close()


def special(gen, n, cols, dtype):
    """Values in (-1, 1) of which some are zero, and in rows 1, 4, 7, .. some infinities of either sign and NaN."""
    a = zeros(n, cols, dtype=dtype)
    a.uniform_(-1, 1, generator=gen)
    at = torch.rand(n, cols, generator=gen, device=DEV)
    a[at < 0.1] = 0.0
    odd = (torch.arange(n, device=DEV) % 3 == 1)[:, None]
    for lo, v in ((0.90, float("inf")), (0.93, float("-inf")), (0.96, float("nan"))):
        a[odd & (at >= lo) & (at < lo + 0.01)] = v
    return a


def outer(coef, src, ids, g):
    """sum over each adapter's rows of coef^T src in 64 bits, term by term (a matrix product may skip zeros)."""
    out = torch.zeros(g, coef.shape[1], src.shape[1], dtype=torch.float64, device=DEV)
    for i, k in enumerate(ids.tolist()):
        if 0 <= k < g:
            out[k] += coef[i].double()[:, None] * src[i].double()[None, :]
    return out


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,n_in,n_out,r,g", [(40, 33, 70, 3, 5), (200, 70, 130, 5, 1), (30, 40, 20_001, 17, 2),
                                              (300, 40, 17_000, 4, 2), (70, 20, 131_000, 40, 1)])
def test_infinities_in_the_gradients_of_a_bank(n, n_in, n_out, r, g, dtype):
    """dup where dy holds infinities and ddown where x does: infinite, NaN and finite where the formula's terms
    are, and the finite values within the bound of their sums (4 sqrt(n) of 2^-24 of the sum of absolute values)."""
    from paper_2309_16743_amd import OT_BF16, OT_FP32, LowRankAdapters
    print(f"infinities {n} {n_in} {n_out} {r} {g} {dtype}", flush=True)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    bank = LowRankAdapters(n_in, n_out, r, g, precision=OT_BF16 if dtype == BF else OT_FP32, max_rows=n)
    ids = torch.randint(-1 if g > 1 else 0, g, (n,), generator=gen, device=DEV).to(torch.int32)
    t = torch.empty(n, r, device=DEV).uniform_(-1, 1, generator=gen)
    t[::4, ::2] = 0.0
    t[2::4, ::2] = 0.5                                             # one term holds it, the others are zero
    up = zeros(g, r, n_out, dtype=dtype)
    up.uniform_(-1, 1, generator=gen)
    ddown, dup = (zeros(g, r, c, dtype=torch.float32) for c in (n_in, n_out))

    def check(got, coef, src):
        want, size = outer(coef, src, ids, g), outer(coef.abs(), src.abs(), ids, g)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        inf = torch.isinf(want)
        assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf].double(), want[inf])
        fine = torch.isfinite(want)
        assert bool(((got.double() - want).abs()[fine] <= (4 * n ** 0.5 + 16) * 2.0 ** -24 * size[fine] + 1e-30).all())
        assert bool(inf.any()) and bool(fine.any())

    x = zeros(n, n_in, dtype=dtype)
    x.uniform_(0, 1, generator=gen)
    dy = special(gen, n, n_out, dtype)
    bank.backward(x, None, None, up, ids, dy, t, ddown, dup)
    check(dup, t, dy)
    # dt of few bits, so that the 64-bit sums start from the kernel's own: dy and up of small whole numbers
    x = special(gen, n, n_in, dtype)
    dy, up = zeros(n, n_out, dtype=dtype), zeros(g, r, n_out, dtype=dtype)
    dy[:, :8] = torch.randint(-2, 3, (n, 8), generator=gen, device=DEV).to(dtype)
    up[..., :8] = torch.randint(-2, 3, (g, r, 8), generator=gen, device=DEV).to(dtype)
    bank.backward(x, None, None, up, ids, dy, t, ddown, dup)
    dt = torch.zeros(n, r, device=DEV)
    for i, k in enumerate(ids.tolist()):
        if k >= 0:
            dt[i] = (up[k].float() * dy[i].float()).sum(1)
    check(ddown, dt, x)
    bank.close()


def not_finite_banks(gen, inner, outer_, dtype):
    """Three adapters of rank 2: one whose first inner row holds an infinity (and one more infinity in its second),
    one of finite inner rows, one with infinities of both signs; every outer row cycles through infinities, NaN, zeros and
    ordinary values, the second row shifted."""
    a, b = zeros(3, 2, inner, dtype=dtype), zeros(3, 2, outer_, dtype=dtype)
    a.uniform_(0.1, 1, generator=gen)
    inf = float("inf")
    a[0, 0, 1] = inf
    a[2, 0, 0], a[2, 1, 1] = -inf, inf
    cycle = torch.tensor([1.0, 0.0, inf, -inf, float("nan"), -2.0, 0.5], device=DEV).to(dtype)
    at = torch.arange(outer_, device=DEV)
    b[:, 0] = cycle[at % 7]
    b[:, 1] = cycle[at // 7 % 7]
    return a, b


def adapted(src, w, inner, outer_, ids):
    """src w^T + sum_r (inner_r src) outer_r in 64 bits, term by term."""
    out = torch.empty(src.shape[0], w.shape[0], dtype=torch.float64, device=DEV)
    size = torch.empty_like(out)
    for i, k in enumerate(ids.tolist()):
        s = src[i].double()
        out[i], size[i] = w.double() @ s, w.double().abs() @ s.abs()
        if k >= 0:
            for r in range(2):
                t = (inner[k, r].double() * s).sum()
                out[i] += t * outer_[k, r].double()
                size[i] += (t * outer_[k, r].double()).abs()
    return out, size


def same_kind(got, want, size, k):
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf].double(), want[inf])
    fine = torch.isfinite(want)
    unit = 2.0 ** -8 if got.dtype == BF else 0.0
    bound = (4 * k ** 0.5 + 16) * 2.0 ** -24 * size + unit * want.abs()
    assert bool(((got.double() - want).abs()[fine] <= bound[fine]).all())
    assert bool(inf.any()) and bool(fine.any())


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,n_in,n_out", [(5, 24, 40), (50, 40, 31_000), (200, 24, 15_400), (150, 24, 61_500)])
def test_infinities_on_both_sides_of_an_adapter(n, n_in, n_out, dtype):
    """An adapter's low-rank value is infinite and its second matrix holds infinities, NaN and zeros: each result as
    the formula says (an infinity times an infinity is one, times zero NaN), the other rows finite."""
    from paper_2309_16743_amd import OT_BF16, OT_FP32, LowRankAdapters
    print(f"infinities on both sides {n} {n_in} {n_out} {dtype}", flush=True)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    bank = LowRankAdapters(n_in, n_out, 2, 3, precision=OT_BF16 if dtype == BF else OT_FP32, max_rows=n)
    ids = (torch.arange(n, device=DEV) % 4 - 1).to(torch.int32)
    w = zeros(n_out, n_in, dtype=dtype)
    w.uniform_(-1, 1, generator=gen)
    x, dy = zeros(n, n_in, dtype=dtype), zeros(n, n_out, dtype=dtype)
    x.uniform_(0.1, 1, generator=gen)
    down, up = not_finite_banks(gen, n_in, n_out, dtype)
    y = zeros(n, n_out, dtype=dtype)
    bank.forward(x, w, down, up, ids, y)
    same_kind(y, *adapted(x, w, down, up, ids), n_in)
    dy.uniform_(0.1, 1, generator=gen)
    up, down = not_finite_banks(gen, n_out, n_in, dtype)
    t, dx = torch.zeros(n, 2, device=DEV), zeros(n, n_in, dtype=dtype)
    ddown, dup = zeros(3, 2, n_in, dtype=torch.float32), zeros(3, 2, n_out, dtype=torch.float32)
    bank.backward(x, w, down, up, ids, dy, t, ddown, dup, dx=dx)
    same_kind(dx, *adapted(dy, w.t(), up, down, ids), n_out)
    bank.close()
