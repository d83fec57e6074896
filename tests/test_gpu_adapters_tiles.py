"""Adapters at sizes that take every tile, split and launch that the plans can choose (adapter_sizes.py), in odd
sizes, every type of y with and without ReLU, against the 64-bit reference; bounds as in test_gpu_adapters."""
import pytest
import torch

from adapter_sizes import SIZES
from test_gpu_adapters import Problem, check_backward, check_forward

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.mark.parametrize("kind,n,n_in,n_out", SIZES)
def test_every_kernel(kind, n, n_in, n_out):
    print(f"every kernel {kind} {n} {n_in} {n_out}", flush=True)
    p = Problem(n, n_in, n_out, 13, 8, TYPES[kind], "mixed", seed=n + n_in)
    bank = p.bank()
    for y_type, relu in ((torch.float32, True), (torch.bfloat16, True), (torch.bfloat16, False)):
        y, t = p.forward(bank, y_type, relu)
        check_forward(p, y, t, relu)
    first = p.backward(bank, relu_input=True)
    check_backward(p, *first, True)
    assert all(torch.equal(a, b) for a, b in zip(first, p.backward(bank, relu_input=True)))
    check_backward(p, *p.backward(bank), False)
    bank.close()


@pytest.mark.parametrize("kind,n,n_in,n_out", [s for s in SIZES if s[0] == "fp32"])
def test_rows_of_large_values(kind, n, n_in, n_out):
    """fp32 rows past 2^60, which the three-term products sum again in fp32: right within the same bounds, and the
    other rows keep their bits."""
    print(f"large values {n} {n_in} {n_out}", flush=True)
    p = Problem(n, n_in, n_out, 13, 8, TYPES[kind], "random", seed=n + n_out)
    bank = p.bank()
    plain = p.forward(bank, torch.float32) + p.backward(bank, relu_input=True)[2:]
    big = [0, n // 2, n - 1]
    p.x[big] *= 2.0 ** 70
    y, t = p.forward(bank, torch.float32)
    check_forward(p, y, t, False)
    p.x[big] *= 2.0 ** -70                      # (2^65 dy times 2^70 x would pass fp32's range in ddown)
    p.dy[big] *= 2.0 ** 65
    got = p.backward(bank, relu_input=True)
    check_backward(p, *got, True)
    rest = [i for i in range(n) if i not in big]
    for a, b in zip(plain, (y, t, got[2])):
        assert torch.equal(a[rest], b[rest])
    bank.close()
