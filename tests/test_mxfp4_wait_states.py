"""Matrix instructions of the MXFP4 attention kernels and the vector instructions that take their results.

A result may be read or overwritten by a vector instruction eight wait states after the matrix instruction was issued, and the
hardware does not wait.  The compiler inserts what is missing, but has left it out across branches (scores read one state after
their product: NaN in some rows of some launches).  The assembly built here is followed along every branch."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2605_10195_amd import build

STATES = 8  # products of 16 x 16 rows and columns


def registers(operand):
    out = set()
    for kind, first, last, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operand):
        base = 0 if kind == "v" else 1000
        out |= {base + int(one)} if one else set(range(base + int(first), base + int(last) + 1))
    return out


def functions(text):
    for part in re.split(r"\n(?=_Z\w+:)", text):
        code, labels = [], {}
        for line in part.split("\n")[1:]:
            label = re.match(r"^(\.LBB\w+):", line)
            if label:
                labels[label.group(1)] = len(code)
                continue
            line = line.split(";")[0].strip()
            if line and line[0] != "." and not line.endswith(":"):
                code.append(line)
        yield part.split(":")[0], code, labels


def too_soon(code, labels):
    """(product, instruction that comes too soon) of every product, along every path."""
    found = []
    for i, line in enumerate(code):
        if not line.startswith(("v_mfma_", "v_smfmac_")):
            continue
        ways, seen = [(i + 1, 0, frozenset(registers(line.split(None, 1)[1].split(",")[0])))], set()
        while ways:
            at, states, live = ways.pop()
            if at >= len(code) or states >= STATES or not live or (at, states) in seen:
                continue
            seen.add((at, states))
            name, _, rest = code[at].partition(" ")
            if name == "s_nop":
                ways.append((at + 1, states + int(rest) + 1, live))
            elif name.startswith(("s_cbranch", "s_branch")):
                if rest.strip() in labels:
                    ways.append((labels[rest.strip()], states + 1, live))
                if name != "s_branch":
                    ways.append((at + 1, states + 1, live))
            elif name == "s_endpgm":
                continue
            elif name.startswith(("v_mfma_", "v_smfmac_")):  # between products the hardware waits itself
                ways.append((at + 1, states + 1, live - registers(rest.split(",")[0])))
            elif name.startswith(("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")) and registers(rest) & live:
                found.append((line, code[at], states))
            else:
                ways.append((at + 1, states + 1, live))
    return found


def test_the_check_itself():
    code = ["v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[0:3], 0", "s_cbranch_scc1 .LBB0_1", "s_nop 7", "v_max_f32_e32 v1, v4, v5", "s_nop 6",
            "v_max_f32_e32 v2, v6, v7", "s_endpgm"]
    assert not too_soon(code, {})
    assert [f[1] for f in too_soon(code, {".LBB0_1": 4})] == []
    assert [f[1] for f in too_soon(code, {".LBB0_1": 5})] == ["v_max_f32_e32 v2, v6, v7"]
    assert [f[1] for f in too_soon(code[:2] + code[3:], {})] == ["v_max_f32_e32 v1, v4, v5"]


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_results_of_products_are_waited_for(tmp_path):
    out = str(tmp_path / "attention.s")
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    made = subprocess.run([hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                           "-x", "hip", "-fno-honor-nans", "-S", "--offload-device-only", os.path.join(build.CSRC, "mxfp4_attention.hip"), "-o", out],
                          capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    products = 0
    with open(out) as f:
        for name, code, labels in functions(f.read()):
            products += sum(line.startswith(("v_mfma_", "v_smfmac_")) for line in code)
            assert not too_soon(code, labels), (name, too_soon(code, labels)[:4])
    assert products > 1000
