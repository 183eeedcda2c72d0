"""Every kernel that dream_window_verify_attn and dream_mx_verify_attn can take, forced, on the cases the choice would give to another one."""
import pytest

import paper_2505_19201_amd as dream
from tests.test_gpu_window import _poison, _Problem

pytestmark = pytest.mark.gpu

# query tiles, waves, splits
SHAPES = [(1, 4, 1), (1, 4, 3), (2, 4, 1), (2, 4, 4), (4, 4, 1), (4, 4, 2), (1, 8, 1), (1, 8, 2), (0, 8, 1), (0, 8, 3), (0, 8, 64), (1, 4, 64)]
CASES = [
    (1, 2, 2, "rand", 1, [0], 0, 0, False),
    (3, 4, 2, "rand", 9, [31, 0, 97], 40, 3, False),
    (2, 8, 1, "rand", 60, [300, 45], 100, 4, False),
    (1, 6, 2, "chain", 70, [260], 0, 0, False),
    (1, 2, 1, "rand", 250, [700], 0, 0, False),
    (1, 4, 2, "rand", 130, [70], 50, 2, True),
]


@pytest.fixture(autouse=True)
def _as_it_was():
    yield
    dream.dream_set_q_tiles(0)
    dream.dream_set_tile_waves(0)
    dream.dream_set_kv_splits(0)


def _force(shape):
    tiles, waves, splits = shape
    dream.dream_set_q_tiles(tiles)
    dream.dream_set_tile_waves(waves)
    dream.dream_set_kv_splits(splits)


@pytest.mark.parametrize("kind", ["bf16", "mx"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:5]) + f"-w{c[6]}")
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "q%dw%ds%d" % s)
def test_rows(shape, case, D, kind):
    _force(shape)
    p = _Problem(case[:3] + (D,) + case[3:], kind)
    p.call()
    p.check()


@pytest.mark.parametrize("kind", ["bf16", "mx"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "q%dw%ds%d" % s)
def test_what_no_row_sees_changes_nothing(shape, D, kind):
    _force(shape)
    p = _Problem((2, 4, 2, D, "rand", 9, [150, 70], 41, 3, False), kind)
    for b, P in enumerate(p.prefix):
        _poison(p, b, slice(P + p.T, None), float("nan"))
        _poison(p, b, slice(3, P - 41 + 1), float("inf"))
    p.call()
    p.check()
