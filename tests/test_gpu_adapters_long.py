"""Adapters of layers with long outputs (both low-rank products of dy in one launch, split
sums, large tiles), at sizes that end inside a piece, a round of rows or a tile; bounds as in
test_gpu_adapters."""
import pytest
import torch

from test_gpu_adapters import Problem, check_backward, check_forward

pytestmark = pytest.mark.gpu

SIZES = [   # rows, in, out, rank, adapters, ids
    (1, 24, 65_536, 1, 1, "one"),
    (70, 40, 70_001, 5, 3, "mixed"),
    (300, 24, 66_003, 20, 2, "one"),         # more rows than a round holds, an adapter without rows
    (130, 136, 65_543, 48, 4, "sorted"),
    (65, 33, 131_072, 64, 6, "random"),
    (40, 64, 100_004, 16, 9, "none"),
    (200, 260, 68_000, 8, 40, "mixed"),
    (129, 300, 30_007, 7, 3, "mixed"),       # forward on 256 x 256 tiles, split input gradient
    (600, 96, 20_001, 16, 5, "random"),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n,n_in,n_out,r,g,ids", SIZES)
def test_long_outputs(n, n_in, n_out, r, g, ids, dtype):
    print(f"long outputs {n} {n_in} {n_out} {r} {g} {ids} {dtype}", flush=True)
    p = Problem(n, n_in, n_out, r, g, dtype, ids, seed=n + r + 2)
    bank = p.bank()
    y, t = p.forward(bank, torch.float32)
    check_forward(p, y, t, False)
    check_backward(p, *p.backward(bank, relu_input=True), True)
    check_backward(p, *p.backward(bank, dx=False), False)
    bank.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_long_outputs_keep_values_apart(dtype):
    """NaN in one adapter's rows and infinities in its matrices leave the others' bits; repeated runs agree."""
    p = Problem(150, 48, 66_001, 6, 4, dtype, "random", seed=5)
    bank = p.bank()
    first = p.backward(bank)
    assert all(torch.equal(a, b) for a, b in zip(first, p.backward(bank)))
    rows = p.ids == 2
    p.dy[rows] = float("nan")
    p.up[2, :, 100:200] = float("inf")
    p.down[2].fill_(float("-inf"))
    got = p.backward(bank)
    for k in (0, 1, 3):
        assert torch.equal(first[0][k], got[0][k]) and torch.equal(first[1][k], got[1][k])
    assert torch.equal(first[2][~rows], got[2][~rows]) and torch.isnan(got[2][rows]).all()
    bank.close()
