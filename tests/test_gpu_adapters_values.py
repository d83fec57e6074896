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
