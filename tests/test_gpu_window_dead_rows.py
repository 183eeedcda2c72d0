"""Rows behind the live ones, without a window: the kernels may ask for the first tiles of a cache before they know the prefix length (dream_window_verify_attn, dream_mx_verify_attn)."""
import pytest

import paper_2505_19201_amd as dream
from tests.test_gpu_window import _poison, _Problem

pytestmark = pytest.mark.gpu

# query tiles, waves, splits: every kernel that takes the keys in one part, the call's own choice, and two in several parts, which wait for the prefix length
SHAPES = [(1, 4, 1), (2, 4, 1), (4, 4, 1), (1, 8, 1), (0, 8, 1), (0, 0, 0), (1, 4, 2), (0, 8, 2)]
# Hq, Hkv, nodes, prefixes: tiles of all waves but the first wholly behind the live rows, prefixes on, before and off a tile's edge, an empty one; trees that end inside a tile, a large one
CASES = [
    (4, 4, 1, [0, 31], False),
    (4, 2, 9, [0, 5], False),
    (8, 2, 12, [23, 32], False),
    (4, 2, 20, [45, 140], False),
    (2, 1, 70, [11, 64], False),
    (4, 2, 21, [0, 40], True),
]


@pytest.fixture(autouse=True)
def _as_it_was():
    yield
    dream.dream_set_q_tiles(0)
    dream.dream_set_tile_waves(0)
    dream.dream_set_kv_splits(0)


@pytest.mark.parametrize("kind,what", [("bf16", "nan"), ("bf16", "inf"), ("bf16", "-inf"), ("mx", "nan")])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:4]))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "q%dw%ds%d" % s)
def test_what_lies_behind_the_live_rows_changes_nothing(shape, case, D, kind, what):
    """Over 300 rows behind the tree, in K and V of every head: NaN, infinities, groups of scale 255."""
    tiles, waves, splits = shape
    dream.dream_set_q_tiles(tiles)
    dream.dream_set_tile_waves(waves)
    dream.dream_set_kv_splits(splits)
    hq, hkv, n, prefix, masks = case
    p = _Problem((2, hq, hkv, D, "rand", n, prefix, 0, 0, masks), kind, slack=301)
    for b, P in enumerate(prefix):
        _poison(p, b, slice(P + n, None), float(what))
    p.call()
    p.check()
