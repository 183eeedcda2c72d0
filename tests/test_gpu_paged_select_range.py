"""dream_page_select over pages whose channels lie further apart than float32's exponents reach: bounds are rounded outwards all the same, as the definition in 64 bits has it."""
import numpy as np
import pytest

import paper_2505_19201_amd as dream
from tests import paged_cases as pc
from tests import window_cases as wc
from tests.test_gpu_paged_cache import _desc, _select

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("T", [1, 5])
def test_bounds_are_rounded_outwards_whatever_a_pages_range(dtype, D, T):
    """Every page has a channel near 2^120, which no query asks for, and others around 2^-40 and down to the smallest numbers there are: their steps, up or down, are all that scores differ by."""
    rng = np.random.default_rng([D, T])
    n, page, Hq, Hkv = 70, 16, 4, 2
    small = rng.choice([2.0 ** -40, 2.0 ** -30, 2.0 ** -126, 2.0 ** -133, 0.0, 1.0, 2.0 ** 100], (n + 1, Hkv, 2, D)) * rng.choice([-1.0, 1.0], (n + 1, Hkv, 2, D))
    b64 = np.stack([small.max(2), small.min(2)], 2)
    b64[:, :, 0, 7] = 2.0 ** 120 * rng.choice([1.0, 1.5], (n + 1, Hkv))
    q64 = pc.rounded(rng.standard_normal((1, T, Hq, D)) * (rng.random((1, T, 1, D)) < 0.1), dtype)
    q64[..., 7] = 0.0
    q64[..., 3] = 1.0
    assert np.array_equal(pc.rounded(b64, dtype), b64)
    table = [rng.permutation(n + 1)]
    pd, desc = dream.page_desc(page, n + 1, n + 1), _desc(1, Hq, Hkv, D, dtype)
    got = _select(pc.device(q64, dtype), pc.device(b64, dtype), wc.ints(table), pd, desc, [n * page], T, 1, 1, 9, n * page + T)
    assert np.array_equal(got[0], pc.words(pc.choose(q64[0], b64[table[0][:n]], 1, 1, 9), n + 1))
