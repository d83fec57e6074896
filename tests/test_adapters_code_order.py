"""The LDS reads that the adapters' products issue by inline assembly, followed through the generated code: along
every branch, loops included, no instruction may read or write the target of a read that is still under way, be it as
an operand, an address or the target of another read.  LDS operations complete in order, so a wait for
lgkmcnt(N) ends those with N or more LDS operations behind them (scalar loads count too, but may
end first, so they are not relied on)."""
import os
import re
import subprocess

import pytest

from paper_2309_16743_amd import build

SOURCE = os.path.join(build.CSRC, "adapters.hip")
MOST = 16                # lgkmcnt holds 4 bits


def registers(text):
    out = set()
    for kind, lo, hi, kind1, one in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        if kind:
            out |= {(kind, i) for i in range(int(lo), int(hi) + 1)}
        else:
            out.add((kind1, int(one)))
    return out


def blocks(code):
    """(instructions, indices of the blocks that may follow) of a kernel's lines."""
    starts, out, labels = [[]], [], {}
    for line in code:
        line = line.split(";")[0].strip()
        m = re.match(r"([.\w$]+):$", line)
        if m:
            starts.append([])
            labels[m.group(1)] = len(starts) - 1
        elif line and not line.startswith("."):
            starts[-1].append(line)
            if re.match(r"s_(c?branch|endpgm|setpc)", line):
                starts.append([])
    for i, b in enumerate(starts):
        last = b[-1] if b else ""
        m = re.match(r"s_c?branch\w*\s+([.\w$]+)", last)
        follow = [labels[m.group(1)]] if m else []
        if not re.match(r"s_(branch|endpgm|setpc)", last) and i + 1 < len(starts):
            follow.append(i + 1)
        out.append((b, follow))
    return out


def returns(op):
    return re.match(r"ds_(read|bpermute|permute|swizzle)", op) or "_rtn" in op


def step(line, pending, found):
    """pending: {register under way: LDS operations issued after its read}."""
    op, _, args = line.partition(" ")
    if op == "s_waitcnt":
        m = re.search(r"lgkmcnt\((\d+)\)", args)
        if m:
            return {r: k for r, k in pending.items() if k < int(m.group(1))}
        assert re.fullmatch(r"\s*((vmcnt|expcnt)\(\d+\)[\s&]*)*", args), line
        return pending
    if not op.startswith("s_") and registers(args) & pending.keys():
        found.add(line)
    if op.startswith("ds_"):
        pending = {r: min(MOST, k + 1) for r, k in pending.items()}
        if returns(op):
            pending.update(dict.fromkeys(registers(args.split(",")[0]), 0))
    return pending


def early_uses(code):
    """Instructions of a kernel that touch the target of an LDS read still under way on some path."""
    bs, found = blocks(code), set()
    at = [None] * len(bs)
    at[0], todo = {}, [0]
    while todo:
        i = todo.pop()
        state = at[i]
        for line in bs[i][0]:
            state = step(line, state, found)
        for j in bs[i][1]:
            if at[j] is None:
                at[j] = dict(state)
                todo.append(j)
                continue
            lower = {r: k for r, k in state.items() if k < at[j].get(r, MOST + 1)}      # the youngest read counts
            if lower:
                at[j].update(lower)
                todo.append(j)
    return sorted(found)


def kernels(listing):
    out, name = {}, None
    for line in listing.splitlines():
        m = re.match(r"(_Z\w+):", line)
        if m:
            name = m.group(1)
            out[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name:
            out[name].append(line)
    return out


def test_no_register_is_touched_before_its_read_arrives(tmp_path):
    try:
        compiler = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = tmp_path / "adapters.s"
    res = subprocess.run([compiler, *build.HIP_FLAGS, "-S", "--cuda-device-only", SOURCE, "-o", str(out)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    found = {k: code for k, code in kernels(out.read_text()).items() if any("s_endpgm" in line for line in code)}
    products = [k for k in found if "gemm_bf16" in k]
    assert len(products) >= 8 and all(any("ds_read_b64_tr" in x or "ds_read_b128" in x for x in found[k]) for k in products)
    early = {k: early_uses(code) for k, code in found.items()}
    assert not {k: v[:3] for k, v in early.items() if v}


READ = "\tds_read_b128 v[4:7], v1\n"
WAIT = "\ts_waitcnt lgkmcnt(0)\n"
USE = "\tv_mov_b32 v9, v6\n"
END = "\ts_endpgm\n"


@pytest.mark.parametrize("text,early", [
    (READ + WAIT + USE, False),
    (READ + USE + WAIT, True),
    (READ + "\ts_waitcnt vmcnt(0)\n" + USE, True),
    # a partial wait leaves the youngest reads under way
    (READ + "\tds_read_b128 v[10:13], v1\n\ts_waitcnt lgkmcnt(1)\n" + USE, False),
    ("\tds_read_b128 v[10:13], v1\n" + READ + "\ts_waitcnt lgkmcnt(1)\n" + USE, True),
    (READ + "\tds_write_b32 v1, v2\n\ts_waitcnt vmcnt(3) lgkmcnt(1)\n" + USE, False),
    (READ + "\ts_load_dword s4, s[0:1], 0x0\n\ts_waitcnt lgkmcnt(1)\n" + USE, True),
    # a pending address, a pending target, a pending value written to LDS or memory
    ("\tds_read_b32 v1, v2\n" + READ + WAIT, True),
    (READ + "\tds_read_b64 v[6:7], v2\n" + WAIT, True),
    (READ + "\tds_write_b32 v1, v5\n" + WAIT, True),
    (READ + "\tglobal_store_dword v1, v7, s[0:1]\n" + WAIT, True),
    # the next turn of a loop, and only one side of a branch
    (".LBB0_1:\n" + USE + READ + "\ts_cbranch_scc1 .LBB0_1\n" + WAIT, True),
    (".LBB0_1:\n" + WAIT + USE + READ + "\ts_cbranch_scc1 .LBB0_1\n" + WAIT, False),
    ("\ts_cbranch_scc0 .LBB0_2\n" + READ + ".LBB0_2:\n" + USE + WAIT, True),
    ("\ts_cbranch_scc0 .LBB0_2\n" + READ + WAIT + ".LBB0_2:\n" + USE, False),
    (READ + "\ts_branch .LBB0_3\n.LBB0_2:\n" + USE + END + ".LBB0_3:\n" + WAIT + "\ts_branch .LBB0_2\n", False),
])
def test_the_check_itself(text, early):
    assert bool(early_uses((text + END).splitlines())) == early
