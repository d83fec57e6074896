"""The layers' workspaces are sized once for all calls of up to so many rows (a captured call holds their
address), so the bound must cover every plan; and the GPU tests' sizes must run every kernel that a plan can
choose (CPU only: builds tests/host/layer_plans.cpp against the library's own layer_plan.h and norm_plan.h)."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

from layer_sizes import DENSE, NORM

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRC = os.path.join(HERE, "host", "layer_plans.cpp")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not found")
    out = str(tmp_path_factory.mktemp("plans") / "layer_plans")
    inc = os.path.join(ROOT, "paper_2309_16743_amd", "csrc")
    res = subprocess.run([gxx, "-std=c++17", "-O2", "-Wall", "-Werror", f"-I{inc}", SRC, "-o", out],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return out


def run(exe, *args):
    return subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=120)


def test_workspaces_cover_every_call(exe):
    res = run(exe, "bound")
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout[-2000:]


def test_launches_of_the_largest_calls(exe):
    res = run(exe, "launches")
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout[-2000:]


@pytest.mark.parametrize("what,sizes", [("dense", DENSE), ("norm", NORM)])
def test_the_gpu_tests_run_every_kernel(exe, what, sizes):
    every = set(run(exe, what).stdout.splitlines())
    assert len(every) > 8
    seen = set()
    for size in sizes:
        seen |= set(run(exe, what + "-of", *size).stdout.splitlines())
    assert seen >= every, sorted(every - seen)
