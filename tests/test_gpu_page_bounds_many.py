"""dream_page_bounds over many pages of 16 KB, which a wave each takes instead of a workgroup, and over a few less: equal to the definition, NaN and infinities and pages that end early among them."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import paged_cases as pc
from tests import window_cases as wc
from tests.test_gpu_paged_cache import _desc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,page,dtype", [(256, 16, "f32"), (128, 32, "f32"), (64, 64, "f32"), (256, 32, "bf16"), (128, 64, "bf16"), (64, 128, "bf16")])
@pytest.mark.parametrize("n", [17, 15])      # pages of the longest sequence: 2176 or 1920 pages and heads
def test_many_pages_of_16_kb(D, page, dtype, n):
    assert page * D * (4 if dtype == "f32" else 2) == 16384
    Hkv = 32
    rng = np.random.default_rng([D, page])
    rows = [n * page, n * page - page // 2, (n - 1) * page + 1, 3 * page - 1]
    start = [0, page - 1, page, 2 * page + 3]
    pages = pc.Pages(rng, page, rows)
    x = rng.standard_normal((pages.n_pages, Hkv, page, D), dtype=np.float32)
    dx = torch.from_numpy(x).cuda().to(pc.DTYPES[dtype])
    for b, r in ((0, 5), (1, page + 1), (2, rows[2] - 1), (3, 2 * page)):
        at = pages.where(b, r)
        for h, c, value in ((0, 3, np.nan), (Hkv - 1, D - 1, np.inf), (7, 0, -np.inf)):
            dx[int(at[0]), h, at[1], c] = value
    x = dx.float().cpu().numpy()
    for first in (None, start):
        got = torch.full((pages.n_pages, Hkv, 2, D), 9.0, dtype=pc.DTYPES[dtype], device="cuda")
        want = np.full(got.shape, 9.0)
        for b, e in enumerate(rows):
            for i in range((first[b] if first else 0) // page, -(-e // page)):
                want[pages.table[b, i]] = pc.page_bounds(x[pages.table[b, i], :, :min(page, e - i * page)])
        dream.dream_page_bounds(_desc(len(rows), Hkv, Hkv, D, dtype), dream.page_desc(page, pages.n_pages, n), wc.ints(pages.table[:, :n]), dx, wc.ints(first) if first else None, wc.ints(rows),
                                max(rows), got)
        torch.cuda.synchronize()
        assert np.array_equal(got.double().cpu().numpy(), want)
