"""The adapters' matrix products read LDS by inline assembly whose outputs arrive only at the wait that
follows (the compiler takes them as there at once).  Their generated code must touch no such register
between the read and the wait: checked on the gfx950 assembly of the source, in listing order."""
import os
import re
import subprocess

import pytest

from paper_2309_16743_amd import build

SOURCE = os.path.join(build.CSRC, "adapters.hip")


def registers(text):
    out = set()
    for kind, lo, hi, kind1, one in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        if kind:
            out |= {(kind, i) for i in range(int(lo), int(hi) + 1)}
        else:
            out.add((kind1, int(one)))
    return out


def early_uses(listing):
    """{kernel: [instructions that touch the target of an LDS read still under way]} of the bf16 products."""
    found, kernel, pending = {}, None, set()
    for line in listing.splitlines():
        m = re.match(r"(_Z\w+):", line)
        if m:
            kernel, pending = m.group(1), set()
            if "gemm_bf16" in kernel:
                found[kernel] = []
        code = line.split(";")[0].strip()
        if kernel not in found or not code or code.startswith(".") or code.endswith(":"):
            continue
        op, _, args = code.partition(" ")
        if op == "s_waitcnt" and "lgkmcnt" in args:
            pending = set()
        elif op.startswith("ds_read"):
            pending |= registers(args.split(",")[0])
        elif not op.startswith("s_") and registers(args) & pending:
            found[kernel].append(code)
    return found


def test_no_register_is_touched_before_its_read_arrives(tmp_path):
    try:
        compiler = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = tmp_path / "adapters.s"
    res = subprocess.run([compiler, *build.HIP_FLAGS, "-S", "--cuda-device-only", SOURCE, "-o", str(out)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    found = early_uses(out.read_text())
    assert len(found) >= 8
    assert not {k: v[:3] for k, v in found.items() if v}


def test_the_check_sees_an_early_use():
    text = "_Z9gemm_bf16x:\n\tds_read_b128 v[4:7], v1\n\tv_mov_b32 v9, v6\n\ts_waitcnt lgkmcnt(0)\n\tv_mov_b32 v9, v6\n"
    assert early_uses(text) == {"_Z9gemm_bf16x": ["v_mov_b32 v9, v6"]}
