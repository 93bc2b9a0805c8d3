"""The workgroups of the tree walk over MXFP4 pools: their lists on the host, and attention through every kind of them."""

import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2605_10195_amd as spex
from mxfp4_common import quantised
from test_host_sanitizers import CSRC, HERE, build_with_sanitizers
from test_mxfp4_attention import Forest


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_lists_of_pieces_under_sanitizers(tmp_path):
    exe = str(tmp_path / "mxfp4_pieces")
    build_with_sanitizers(exe, [os.path.join(HERE, "mxfp4_pieces.cpp"), os.path.join(CSRC, "planner.cpp"), os.path.join(CSRC, "page_table.cpp")])
    run = subprocess.run([exe, "120"], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0, (run.stdout[-2000:], run.stderr[-4000:])
    assert run.stdout == "ok\n", run.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(4, 2, 32), (8, 1, 64), (6, 2, 96), (8, 2, 128), (2, 1, 160), (3, 1, 192), (4, 1, 224), (4, 1, 256), (40, 1, 128)])
@pytest.mark.parametrize("tiles", [0, 2])
def test_long_paths_in_pieces(heads, tiles):
    """Few requests on long paths: their states are merged by a second launch."""
    f = Forest(heads, [(-1, 5003), (0, 70), (0, 1), (-1, 4100), (-1, 9)], seed=heads[2] + tiles, kernel_mode=3, walk_row_tiles=tiles)
    if tiles and heads[0] // heads[1] > 16 * tiles:  # a token's rows stay together
        with pytest.raises(spex.SpexError, match="UNSUPPORTED"):
            f.check([1, 2, 3, 4])
        f.tree.close()
        return
    f.check([1, 2, 3, 4])
    assert f.tree.last_launch_info()["partial_rows"] > 0
    f.check([2])
    f.check([1, 3, 1], [5, 3, 1])
    f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(16, 16, 32), (16, 8, 64), (8, 8, 128)])
def test_many_short_paths(heads):
    """Enough sets of rows for a wavefront each, with a path among them that takes four, and one that goes in pieces."""
    nodes = [(-1, 1 + 7 * i % 50) for i in range(400)] + [(-1, 5500), (-1, 14000)]
    f = Forest(heads, nodes, seed=heads[2])
    f.check(list(range(402)))
    assert f.tree.last_launch_info()["partial_rows"] > 0
    f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(8, 2, 128), (10, 2, 64), (28, 4, 96), (5, 1, 32)])
@pytest.mark.parametrize("tokens", [70, 300])
def test_branches_within_a_row_tile(heads, tokens):
    """Two row tiles, and private blocks that concern one of them, the other, or both: from 16 a wavefront on they are taken apart."""
    nodes = [(-1, 45)] + [(0, tokens + i) for i in range(16)]
    f = Forest(heads, nodes, seed=heads[0], kernel_mode=3, walk_row_tiles=2)
    leaves = list(range(1, 17))
    f.check(leaves)
    f.check(leaves[:5], [1, 3, 1, 2, 1])
    masks = np.concatenate([1 << np.arange(n) for n in [2] * 16]).astype(np.uint32)
    f.check(leaves, [2] * 16, masks)
    f.tree.close()


@pytest.mark.gpu
def test_pieces_that_grow():
    """Appends to branches of a path in pieces: the last piece takes what they start, eagerly and in a graph that is captured again."""
    f = Forest((8, 2, 128), [(-1, 6000)] + [(0, 14 + i) for i in range(4)], seed=3, spare=40)
    leaves = [1, 2, 3, 4]
    ids = [f.ids[u] for u in leaves]
    states = set()
    for step in range(36):
        x = torch.as_tensor(f.rng.standard_normal((2, 4, 2, 128))).to(torch.bfloat16)
        f.tree.append_tokens(ids, x[0].cuda(), x[1].cuda(), quantize=True)
        for i, u in enumerate(leaves):
            f.k[u] = np.concatenate([f.k[u], quantised(x[0, i].double().numpy(), "k")[None]])
            f.v[u] = np.concatenate([f.v[u], quantised(x[1, i].double().numpy(), "v")[None]])
        f.check(leaves)
        states.add(f.tree.last_launch_info()["plan_rebuilt"])
        assert f.tree.last_launch_info()["partial_rows"] > 0
    assert 2 in states  # some plans were patched
    q = torch.as_tensor(f.rng.standard_normal((4, 8, 128))).to(torch.bfloat16).cuda()
    out, lse = f.tree.decode_attention(ids, None, q, 128 ** -0.5)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        f.tree.decode_attention(ids, None, q, 128 ** -0.5, out, lse)
    for i in range(4):
        out.fill_(float("nan"))
        q.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        eager, eager_lse = f.tree.decode_attention(ids, None, q, 128 ** -0.5)
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse)
    f.check(leaves, static=True)
    f.tree.close()


@pytest.mark.gpu
def test_pieces_of_far_scores():
    """Scores far from zero, whose references differ from piece to piece, and rows that one piece of many decides."""
    def value(rng, shape):
        x = rng.standard_normal(shape) * 3
        x[shape[0] // 3] *= 20
        return x

    f = Forest((8, 2, 128), [(-1, 7000), (0, 33)], seed=5, value=value, kernel_mode=3)
    f.check([0, 1], spread=8.0, loose=1e-4)
    assert f.tree.last_launch_info()["partial_rows"] > 0
    f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("mode", [0, 2])
@pytest.mark.parametrize("heads", [(80, 1, 64), (130, 2, 32), (65, 1, 256)])
def test_groups_wider_than_a_wavefront_of_rows(heads, mode):
    f = Forest(heads, [(-1, 200), (0, 33), (0, 1)], seed=heads[0], kernel_mode=mode)
    f.check([1, 2])
    f.check([1, 2, 0], [3, 1, 2])
    f.tree.close()


@pytest.mark.gpu
def test_on_a_stream_of_its_own():
    """Appends, attention in pieces and the reading back ordered by a stream that is not the default one, with work ahead of them."""
    f = Forest((8, 2, 128), [(-1, 4000), (0, 20)], seed=7, spare=8)
    x = [torch.as_tensor(f.rng.standard_normal((16, 2, 128))).to(torch.bfloat16) for _ in range(2)]
    q = torch.as_tensor(f.rng.standard_normal((1, 8, 128))).to(torch.bfloat16)
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    kd, vd, qd = torch.empty_like(x[0], device="cuda"), torch.empty_like(x[1], device="cuda"), torch.empty_like(q, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            busy = busy @ busy * 1e-3
        for dst, src in ((kd, x[0]), (vd, x[1]), (qd, q)):
            dst.copy_(src.cuda())
        f.tree.append_step(f.ids[1], kd, vd, quantize=True)
        out, lse = f.tree.decode_attention([f.ids[1]], None, qd, 128 ** -0.5)
        gk, gv = f.tree.read_back([f.ids[1]])
    side.synchronize()
    for i, w in enumerate("kv"):
        old = (f.k, f.v)[i]
        old[1] = np.concatenate([old[1], quantised(x[i].double().numpy(), w)])
    assert np.array_equal(gk.cpu().double().numpy(), f.k[1]) and np.array_equal(gv.cpu().double().numpy(), f.v[1])
    want, want_lse = f.check([1], q=q)
    assert np.array_equal(out.cpu().double().numpy(), want) and np.array_equal(lse.cpu().double().numpy(), want_lse)
    f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(16, 2, 64), (32, 8, 128), (12, 4, 96)])
def test_a_full_card_gives_the_same_bits_every_time(heads):
    """As many wavefronts as run at a time, all of them working: every pass equals the first, which is right."""
    f = Forest(heads, [(-1, 600 + 20 * i) for i in range(48)] + [(i, 1 + i % 40) for i in range(48)], seed=heads[2])
    leaves = list(range(48, 96))
    q = torch.as_tensor(f.rng.standard_normal((48, heads[0], heads[2])) * 2).to(torch.bfloat16)
    want, want_lse = f.check(leaves, q=q)
    ids, qd = [f.ids[u] for u in leaves], q.cuda()
    first = None
    for _ in range(30):
        out, lse = f.tree.decode_attention(ids, None, qd, heads[2] ** -0.5)
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert np.array_equal(first[0].cpu().double().numpy(), want) and np.array_equal(first[1].cpu().double().numpy(), want_lse)
    f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("mode", [0, 2])
@pytest.mark.parametrize("scale", [1e9, 1e25, 1e-35])
def test_scales_far_from_one(scale, mode):
    """Branches below an empty node, so that rows meet blocks that they do not see before any that they do.  A large scale leaves the
    largest score's value, a small one the mean."""
    f = Forest((4, 2, 64), [(-1, 0)] + [(0, 20 + 9 * i) for i in range(6)], seed=3, kernel_mode=mode)
    q = torch.as_tensor(f.rng.standard_normal((6, 4, 64))).to(torch.bfloat16)
    ids = f.ids[1:]
    out, lse = f.tree.decode_attention(ids, None, q.cuda(), scale)
    out, lse, q = out.cpu().double().numpy(), lse.cpu().double().numpy(), q.double().numpy()
    for i in range(6):
        k, v = f.path(i + 1)
        for h in range(4):
            scores = k[:, h // 2] @ q[i, h]
            want = v[np.argmax(scores), h // 2] if scale > 1 else v[:, h // 2].mean(0)
            # one weight of 2^7 and a division that gives 2^-7, or sums of equal weights: fp32 roundings of numbers up to 6 * 2
            assert np.abs(out[i, h] - want).max() <= 64 * 2.0 ** -24 * 12
            top = scale * scores.max() if scale > 1 else np.log(len(k))
            assert abs(lse[i, h] - top) <= 2.0 ** -20 * abs(top) + 2.0 ** -20
    f.tree.close()
