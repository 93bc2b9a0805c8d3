"""Which kernels decode attention over MXFP4 pools runs by itself, and that a path of a million tokens comes out the same of either."""

import os
import shutil
import subprocess

import pytest
import torch

import paper_2605_10195_amd as spex
from test_host_sanitizers import CSRC, HERE, build_with_sanitizers


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_choices_under_sanitizers(tmp_path):
    exe = str(tmp_path / "mxfp4_route")
    build_with_sanitizers(exe, [os.path.join(HERE, "mxfp4_route.cpp"), os.path.join(CSRC, "planner.cpp"), os.path.join(CSRC, "page_table.cpp")])
    run = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and run.stdout == "ok\n", (run.stdout[-2000:], run.stderr[-4000:])


@pytest.mark.gpu
@pytest.mark.parametrize("heads,walk", [((4, 1, 64), False), ((4, 2, 64), True)])
def test_a_million_tokens(heads, walk):
    """Values are constant in each stretch of 2^16 tokens and keys zero, so that the output is the mean of the stretches' values; then one
    token behind them, which takes all of the weight."""
    hq, hkv, dim = heads
    tokens = 16 << 16
    tree = spex.SpexTree(*heads, 16, "bf16", "mxfp4", num_pages=tokens // 16 + 8)
    (root,) = tree.fork(-1, 1)
    k = torch.zeros((1 << 16, hkv, dim), dtype=torch.bfloat16, device="cuda")
    for i in range(16):
        tree.append_step(root, k, torch.full_like(k, float(1 + i % 4)), quantize=True)
    q = torch.ones((1, hq, dim), dtype=torch.bfloat16, device="cuda")
    out, lse = tree.decode_attention([root], None, q, 1.0)
    assert (tree.last_launch_info()["walk_row_tiles"] != 0) == walk
    # sums of 2^20 equal weights and of their products with small numbers: an exact power of two, 10 times 2^18
    assert (out - 2.5).abs().max() <= 2.5 * 2.0 ** -20 and (lse - 20 * 0.6931471805599453).abs().max() <= 2.0 ** -17
    (leaf,) = tree.fork(root, 1)
    tree.append_step(leaf, torch.full_like(k[:1], 1.0), torch.full_like(k[:1], -6.0), quantize=True)
    out, lse = tree.decode_attention([leaf], None, q, 1.0)
    assert (tree.last_launch_info()["walk_row_tiles"] != 0) == walk
    # a score of 64 against 2^20 of zero: e^-64 2^20 is nothing in fp32
    assert (out + 6.0).abs().max() <= 6 * 2.0 ** -22 and (lse - 64.0).abs().max() <= 2.0 ** -15
    tree.close()
