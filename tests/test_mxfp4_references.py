"""References of softmax states over MXFP4 pools: rows that have met no score yet, and scores of millions in states that are joined."""

import numpy as np
import pytest
import torch

from mxfp4_common import attention, row_error
from test_mxfp4_attention import MODES, Forest


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("top", [0.0, 8.0])
@pytest.mark.parametrize("scale", [1e8, 1e9, 1e25])
def test_rows_that_meet_no_score_at_first(scale, top, mode):
    """Branches below an empty root: a row's first blocks are other branches'.  Scores near zero at a scale that takes the reference of a
    row without scores out of range; one dim a score, so that nothing is summed."""
    f = Forest((4, 2, 64), [(-1, 0)] + [(0, 20 + 9 * i) for i in range(6)], seed=29, kernel_mode=mode)
    q = np.zeros((6, 4, 64))
    if top:
        q[..., 0] = 2.0 ** np.floor(np.log2(top / scale))
    f.check(list(range(1, 7)), scale=scale, q=torch.as_tensor(q).to(torch.bfloat16))
    f.tree.close()


class FarScores:
    """Scores 2^23 + 0 .. 6 times the scale: whole numbers in fp32 whatever the order of the sums."""

    def __init__(self, nodes, heads=(8, 2, 128), **kw):
        def value(rng, shape):
            if self.of_values:
                x = rng.standard_normal(shape)
            else:
                x = np.zeros(shape)
                x[..., 0] = 2.0 ** 12
                most = np.array([1, 3, 2, 6, 4, 1, 6, 0])[np.arange(shape[0]) * 8 // shape[0]]  # of a stretch of the tokens
                x[..., 32] = np.minimum(rng.integers(0, 4, shape[:2]), most[:, None])
                x[::97, :, 32] = most[::97, None]
            self.of_values = not self.of_values
            return x

        self.of_values = False
        self.f = Forest(heads, nodes, value=value, **kw)

    def check(self, leaves, scale, q_lens=None, masks=None):
        f, lens = self.f, q_lens or [1] * len(leaves)
        q = np.zeros((sum(lens), f.hq, f.dim))
        q[..., 0] = 2.0 ** 11
        q[..., 32] = 1
        out, lse = f.tree.decode_attention([f.ids[u] for u in leaves], q_lens, torch.as_tensor(q).to(torch.bfloat16).cuda(), scale, draft_masks=masks)
        out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
        at = 0
        for u, n in zip(leaves, lens):
            k, v = f.path(u)
            see = np.arange(len(k))[None] <= len(k) - n + np.arange(n)[:, None]
            if masks is not None:
                for j in range(n):
                    see[j, len(k) - n:] = [(int(masks[at + j]) >> i) & 1 for i in range(n)]
            for h in range(f.hq):
                g = h // (f.hq // f.hkv)
                o, z, mean, _ = attention(q[at:at + n, h], k[:, g], v[:, g], see, scale)
                # differences of scores, up to 6 and exact, are what is scaled
                assert (np.abs(out[at:at + n, h] - o) <= row_error(f.dim, len(k), np.full(n, 6 * scale), mean)).all(), (u, h)
                # a constant rounded twice, the scaled reference, a sum with a logarithm, another constant and its product
                assert (np.abs(lse[at:at + n, h] - z) <= 6 * 2.0 ** -24 * np.abs(z) + 2.0 ** -15).all(), (u, h)
            at += n


# 2^23 times these and log2 e: below 2^22, where references are subtracted scaled, and above
SCALES = [0.25, 0.34, 0.35, 1.0]


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("scale", SCALES)
def test_far_scores_on_long_paths(scale, mode):
    """A path that several workgroups share, whose states have different references."""
    x = FarScores([(-1, 7000), (0, 33), (0, 5)], seed=31, kernel_mode=mode)
    x.check([0, 1, 2], scale)
    if mode == 3:
        assert x.f.tree.last_launch_info()["partial_rows"] > 0
    x.check([1, 2], scale, [7, 3])
    x.f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("tiles", [1, 2])
@pytest.mark.parametrize("scale", SCALES)
def test_far_scores_of_one_workgroup(scale, tiles):
    """A wavefront for a set of rows, whose reference moves, and four whose states are joined."""
    x = FarScores([(-1, 900)] + [(0, 300 + 7 * i) for i in range(9)], seed=33, kernel_mode=3, walk_row_tiles=tiles)
    x.check(list(range(1, 10)), scale)
    x.f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", SCALES)
def test_far_scores_of_many_short_paths(scale):
    """Enough sets of rows for a wavefront each."""
    x = FarScores([(-1, 10 + 7 * i % 190) for i in range(1400)], seed=35)
    x.check(list(range(1400)), scale)
    x.f.tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("mode", [2, 3])
@pytest.mark.parametrize("tiles", [1, 2])
@pytest.mark.parametrize("heads", [(16, 2, 64), (12, 4, 96), (3, 1, 160), (8, 2, 256)])
@pytest.mark.parametrize("scale", [0.25, 1.0])
def test_far_scores_of_other_heads(scale, heads, tiles, mode):
    """Every shape of the kernels, chains and draft masks, paths in pieces beside short ones."""
    x = FarScores([(-1, 4300), (0, 90), (0, 40), (-1, 300), (3, 33)], heads, seed=37, kernel_mode=mode, walk_row_tiles=tiles)
    x.check([1, 2, 4], scale)
    x.check([1, 4, 2], scale, [6, 2, 5], np.concatenate([1 << np.arange(n) | 1 for n in (6, 2, 5)]).astype(np.uint32))
    x.f.tree.close()
