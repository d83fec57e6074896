"""The layers' plans over sizes drawn from their whole range: the GPU tests' sizes run every kernel that any of them
takes, and workspaces keep to their bounds (CPU only: builds tests/host/layer_plan_sweep.cpp against the library's own
layer_plan.h)."""
from __future__ import annotations

import functools
import os
import shutil
import subprocess

import pytest

from layer_sizes import DENSE

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2309_16743_amd", "csrc")


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not found")

    @functools.cache
    def build(name):
        out = str(tmp_path_factory.mktemp("sweep") / name)
        res = subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", f"-I{CSRC}",
                              os.path.join(HERE, "host", name + ".cpp"), "-o", out], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr
        return out
    return build


def lines(*args):
    res = subprocess.run([*map(str, args)], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout[-2000:]
    return res.stdout.splitlines()


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_the_gpu_tests_run_every_kernel(built, seed):
    sweep, of = built("layer_plan_sweep"), built("layer_plans")
    every = dict(line.split("\t") for line in lines(sweep, "kernels", 300000, seed))
    assert len(every) >= 38
    seen = set()
    for size in DENSE:
        seen |= set(lines(of, "dense-of", *size))
    assert seen >= set(every), {k: every[k] for k in sorted(set(every) - seen)}


@pytest.mark.parametrize("seed", [1, 2])
def test_workspaces_keep_to_their_bounds(built, seed):
    assert lines(built("layer_plan_sweep"), "bound", 200000, seed) == ["ok"]
