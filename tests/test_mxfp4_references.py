"""References of softmax states over MXFP4 pools."""

import numpy as np
import pytest
import torch

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
