"""The surrogate's pipelined bf16 products read LDS by inline assembly: the generated code of surrogate.hip is followed
along all paths as the adapters' is (test_adapters_code_order)."""
import os
import re
import subprocess

import pytest

from paper_2309_16743_amd import build
from test_adapters_code_order import early_uses, kernels

SOURCE = os.path.join(build.CSRC, "surrogate.hip")


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    try:
        compiler = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("code") / "surrogate.s"
    res = subprocess.run([compiler, *build.HIP_FLAGS, "-S", "--cuda-device-only", SOURCE, "-o", str(out)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return out.read_text()


def test_no_register_is_touched_before_its_read_arrives(listing):
    found = {k: code for k, code in kernels(listing).items() if any("s_endpgm" in line for line in code)}
    products = {k: code for k, code in found.items() if "gemm_bf16_pipe" in k or "gemm_bf16_pp" in k}
    assert len(products) >= 16
    assert all(any("ds_read_b64_tr" in x or "ds_read_b128" in x for x in code) for code in products.values())
    early = {k: early_uses(code) for k, code in found.items()}
    assert not {k: v[:3] for k, v in early.items() if v}


def test_the_pipelined_products_keep_their_sums_in_registers(listing):
    spills = dict(zip(re.findall(r"\.name:\s+(_Z\w+)", listing), re.findall(r"\.vgpr_spill_count:\s*(\d+)", listing)))
    products = {k: int(v) for k, v in spills.items() if "gemm_bf16_pipe" in k or "gemm_bf16_pp" in k}
    assert len(products) >= 16 and not {k: v for k, v in products.items() if v}
