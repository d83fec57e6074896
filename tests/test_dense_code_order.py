"""The dense layer's bf16 products read LDS by inline assembly too: the generated code of dense_bf16.hip is
followed along all paths as the adapters' is (test_adapters_code_order)."""
import os
import re
import subprocess

import pytest

from paper_2309_16743_amd import build
from test_adapters_code_order import early_uses, kernels

SOURCE = os.path.join(build.CSRC, "dense_bf16.hip")


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    try:
        compiler = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("code") / "dense_bf16.s"
    res = subprocess.run([compiler, *build.HIP_FLAGS, "-S", "--cuda-device-only", SOURCE, "-o", str(out)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return out.read_text()


def test_no_register_is_touched_before_its_read_arrives(listing):
    found = {k: code for k, code in kernels(listing).items() if any("s_endpgm" in line for line in code)}
    products = [k for k in found if "gemm_bf16" in k]
    assert len(products) >= 15
    early = {k: early_uses(code) for k, code in found.items()}
    assert not {k: v[:3] for k, v in early.items() if v}


def test_the_products_keep_their_sums_in_registers(listing):
    """No product spills (its accumulators would go through memory at every step)."""
    spills = dict(zip(re.findall(r"\.name:\s+(_Z\w+)", listing), re.findall(r"\.vgpr_spill_count:\s*(\d+)", listing)))
    assert len(spills) >= 15
    assert not {k: v for k, v in spills.items() if int(v)}
