"""The adapters' workspaces are sized once for all calls of up to so many rows (a captured call holds their
address), so the bound must cover every plan, and stay small enough to be had (CPU only).

Builds tests/host/adapter_plans.cpp against the library's own adapt_plan.h and runs it over sizes, ranks,
adapters and rows.  A second build bounds the partial sums of the pass over a long dy by its rows alone, which must
be seen to pass the limit."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRC = os.path.join(HERE, "host", "adapter_plans.cpp")


def build(folder, *flags):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not found")
    exe = os.path.join(str(folder), "adapter_plans")
    inc = os.path.join(ROOT, "paper_2309_16743_amd", "csrc")
    res = subprocess.run([gxx, "-std=c++17", "-O2", "-Wall", "-Werror", *flags, f"-I{inc}", SRC, "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return exe


def run(exe, *args):
    return subprocess.run([exe, *args], capture_output=True, text=True, timeout=120)


def test_workspace_covers_every_call_and_is_bounded(tmp_path):
    res = run(build(tmp_path), "bound")
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout[-2000:]


def test_rows_alone_do_not_bound_the_pass(tmp_path):
    res = run(build(tmp_path, "-DROWS_ONLY"), "bound")
    assert res.returncode == 1 and "values for" in res.stdout, res.stdout[-2000:]


def test_the_gpu_tests_run_every_kernel(tmp_path):
    """Each product kernel and each way of the low-rank products that some call takes is taken by one of the tested
    sizes (test_gpu_adapters_tiles)."""
    from adapter_sizes import SIZES
    exe = build(tmp_path)
    every = set(run(exe, "kernels").stdout.splitlines())
    assert len(every) > 20
    seen = set()
    for size in SIZES:
        seen |= set(run(exe, "of", *map(str, size)).stdout.splitlines())
    assert seen == every, sorted(every ^ seen)
