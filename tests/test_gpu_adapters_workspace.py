"""Workspaces of the adapters: device memory that a bank takes when it is made, and calls whose partial sums are
held to a bound."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("n_out,rank,g", [(1_000_000, 64, 1), (1 << 26, 64, 1), (1 << 26, 16, 8)])
def test_a_bank_of_many_rows_takes_little_memory(n_out, rank, g):
    """At most 1 GB for 4096 rows whatever the layer's length: a bank that only serves pays it too."""
    from paper_2309_16743_amd import OT_BF16, LowRankAdapters
    torch.zeros(1, device=DEV)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    bank = LowRankAdapters(64, n_out, rank, g, precision=OT_BF16, max_rows=4096)
    taken = before - torch.cuda.mem_get_info()[0]
    bank.close()
    assert taken < 1 << 30


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,n_out,rank,g", [(4096, 300_011, 64, 1), (4000, 70_001, 33, 2), (4097, 20_003, 5, 2),
                                            (5000, 16_384, 20, 3)])
def test_many_rows_of_a_long_gradient(n, n_out, rank, g, dtype):
    """Rows whose partial sums reach the bound (longer column ranges), and more rows than the pass takes (the two
    products apart): both gradients against 64 bits, tolerance as for the other sizes (4 sqrt(k) 2^-24 of the sum of
    absolute values)."""
    from paper_2309_16743_amd import OT_BF16, OT_FP32, LowRankAdapters
    print(f"many rows {n} {n_out} {rank} {g} {dtype}", flush=True)
    n_in = 24
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)

    def uniform(*shape, t=dtype):
        full = torch.empty(*shape[:-1], (shape[-1] + 7) // 8 * 8, dtype=t, device=DEV).uniform_(-1, 1, generator=gen)
        return full[..., :shape[-1]]

    x, dy, up = uniform(n, n_in), uniform(n, n_out), uniform(g, rank, n_out)
    t, ids = uniform(n, rank, t=torch.float32), torch.randint(-1, g, (n,), generator=gen, device=DEV).to(torch.int32)
    if g == 1:
        ids.zero_()
    ddown, dup = uniform(g, rank, n_in, t=torch.float32), uniform(g, rank, n_out, t=torch.float32)
    bank = LowRankAdapters(n_in, n_out, rank, g, precision=OT_BF16 if dtype == torch.bfloat16 else OT_FP32, max_rows=n)
    bank.backward(x, None, None, up, ids, dy, t, ddown, dup)
    torch.cuda.synchronize()
    for k in range(g):
        rows = torch.nonzero(ids == k)[:, 0]
        tk, xk = t[rows].double(), x[rows].double()
        dt, dt_size = 0, 0
        for c in range(0, n_out, 32_768):
            dyc, upc = dy[rows, c:c + 32_768].double(), up[k, :, c:c + 32_768].double()
            want, size = tk.t() @ dyc, tk.t().abs() @ dyc.abs()
            bound = (4 * len(rows) ** 0.5 + 16) * 2.0 ** -24 * size
            assert bool(((dup[k, :, c:c + 32_768].double() - want).abs() <= bound).all())
            dt, dt_size = dt + dyc @ upc.t(), dt_size + dyc.abs() @ upc.t().abs()
        bound = (4 * (n_out + n) ** 0.5 + 16) * 2.0 ** -24 * (dt_size.t() @ xk.abs())
        assert bool(((ddown[k].double() - dt.t() @ xk).abs() <= bound).all())
    bank.close()


def test_host_time_of_a_call_does_not_grow_with_its_rows():
    """A call needs the address of its partial sums, not their size (which looks at the plan of every group of 32
    rows): the host's time for 2^20 rows is that for 32 rows within 40 us (the shortest of 20 calls each)."""
    import time

    from paper_2309_16743_amd import LowRankAdapters
    n = 1 << 20
    x, w, y = (torch.zeros(r, 8, device=DEV) for r in (n, 8, n))
    down, up = torch.zeros(1, 1, 8, device=DEV), torch.zeros(1, 1, 8, device=DEV)
    ids = torch.zeros(n, dtype=torch.int32, device=DEV)
    bank = LowRankAdapters(8, 8, 1, 1, max_rows=n)

    def shortest(rows):
        best = 1.0
        for _ in range(20):
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            bank.forward(x[:rows], w, down, up, ids[:rows], y[:rows])
            best = min(best, time.perf_counter() - t0)
        return best

    few, many = shortest(32), shortest(n)
    torch.cuda.synchronize()
    print(f"host time of a call of 32 rows {few * 1e6:.0f} us, of 2^20 {many * 1e6:.0f} us", flush=True)
    bank.close()
    assert many < few + 40e-6
