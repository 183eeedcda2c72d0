"""Weights of the forms of paged attention that carry them in two parts of bf16: their rows are off by their own rounding, not by that of the weights too."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import paged_cases as pc
from tests import window_cases as wc
from tests.test_gpu_paged_attention import Problem, _automatic      # noqa: F401

pytestmark = pytest.mark.gpu


def _check(p):
    """window_cases.attention_bounds without bf16 weights: a weight in two parts is off by 2^-8 of what the first part, off by 2^-8, leaves; the row is rounded once, half a step of 2^-8."""
    p.call()
    torch.cuda.synchronize()
    got = p.out.double().cpu().numpy()
    for b in range(p.B):
        want, _, mass, size = pc.attend(p.q64[b], p.k64[b], p.v64[b], p.see[b])
        row, _ = wc.attention_bounds(want[None], mass[None], size[None], p.prefix[b] + p.T, p.D, False)
        bound = row[0] + mass * 2.0 ** -16 * (1 + 2.0 ** -6) + np.abs(want) * 2.0 ** -8
        err = np.abs(got[b] - want)
        assert (err <= bound).all(), float((err / bound).max())


# D, form of the waves, query tiles (0: the call's own choice)
FORMS = [(64, 4, 1), (64, 4, 2), (128, 4, 1), (128, 4, 2), (256, 4, 1), (256, 8, 1), (256, 8, 2), (256, 0, 0)]


@pytest.mark.parametrize("D,waves,tiles", FORMS)
@pytest.mark.parametrize("splits,more", [(1, {}), (3, dict(groups=[(0, 2, 49)])), (1, dict(sparse=0.4))], ids=["own", "shared", "selected"])
def test_weights_are_not_rounded_to_bf16(D, waves, tiles, splits, more):
    if waves:
        dream.dream_set_tile_waves(waves)
        dream.dream_set_q_tiles(tiles)
        dream.dream_set_kv_splits(splits)
    for T, prefix, page in ((1, [333, 60], 16), (7, [100, 71], 32)):
        _check(Problem(4, 2, D, T, prefix, page, seed=T, **more))
