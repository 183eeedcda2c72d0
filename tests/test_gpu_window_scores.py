"""Scores of -inf that a node does see (dream_window_verify_attn, dream_mx_verify_attn): such a key has weight 0, wherever its tile begins."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import window_cases as wc
from tests.test_gpu_window import _Problem

pytestmark = pytest.mark.gpu

LOW = 128      # keys whose scores are -inf: the first whole tile of every wave, for four of them
# query tiles, waves, splits; the last the kernel that the call takes by itself
SHAPES = [(1, 4, 1), (2, 4, 1), (4, 4, 1), (1, 8, 1), (0, 8, 1), (1, 4, 4), (0, 8, 4), (0, 0, 0)]


@pytest.fixture(autouse=True)
def _as_it_was():
    yield
    dream.dream_set_q_tiles(0)
    dream.dream_set_tile_waves(0)
    dream.dream_set_kv_splits(0)


@pytest.mark.parametrize("kind,dtype,low", [("bf16", "bf16", "inf"), ("bf16", "bf16", "overflow"), ("mx", "bf16", "overflow"), ("f32", "f32", "inf"), ("mx", "f32", "overflow")])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "q%dw%ds%d" % s)
def test_seen_keys_with_scores_of_minus_infinity(shape, D, kind, dtype, low):
    """Channel 0 of every query is 8; that of the first keys is -inf, or as far below zero as their type goes, where 8 times it overflows to -inf.  The rows are those over the keys behind."""
    tiles, waves, splits = shape
    dream.dream_set_q_tiles(tiles)
    dream.dream_set_tile_waves(waves)
    dream.dream_set_kv_splits(splits)
    p = _Problem((2, 8, 2, D, "rand", 12, [LOW + 200, LOW + 33], 0, 0, False), kind, dtype=dtype)
    p.q[..., 0] = 8.0
    p.q64[..., 0] = 8.0
    if kind == "mx":
        p.k[0][:, :, :LOW, :D // 2] = 0
        p.k[0][:, :, :LOW, 0] = 15            # -6
        p.k[1][:, :, :LOW] = 252              # times 2^125
    else:
        p.k[0][:, :, :LOW, 0] = float("-inf") if low == "inf" else -3e38
    p.call()
    torch.cuda.synchronize()
    out, lse, mass, size = wc.attention(p.q64, p.k64[:, :, LOW:], p.v64[:, :, LOW:], [P - LOW for P in p.prefix], p.parent)
    row, ls = wc.attention_bounds(out, mass, size, p.max_kv, D, dtype == "bf16")
    got, got_lse = p.out.double().cpu().numpy(), p.lse.double().cpu().numpy()
    assert np.isfinite(got).all() and np.isfinite(got_lse).all()
    assert (np.abs(got - out) <= row).all()
    assert (np.abs(got_lse - lse) <= ls + np.abs(lse) * 2.0 ** -23).all()


@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "q%dw%ds%d" % s)
def test_nothing_but_scores_of_minus_infinity(shape, kind, dtype):
    """Then there is nothing to weigh: a zero row and lse = -inf, as for a node that sees nothing."""
    tiles, waves, splits = shape
    dream.dream_set_q_tiles(tiles)
    dream.dream_set_tile_waves(waves)
    dream.dream_set_kv_splits(splits)
    p = _Problem((2, 8, 2, 64, "rand", 12, [200, 33], 0, 0, False), kind, dtype=dtype)
    p.q[..., 0] = 8.0
    p.k[0][..., 0] = float("-inf")
    p.call()
    torch.cuda.synchronize()
    assert not p.out.any() and bool(torch.isneginf(p.lse).all())
