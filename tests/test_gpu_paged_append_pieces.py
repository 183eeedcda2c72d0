"""dream_paged_append where rows are so many that a workgroup has as much of a row as its threads hold, at sizes on both sides of what that is: all of a row is written."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import paged_cases as pc
from tests import window_cases as wc
from tests.test_gpu_paged_cache import _desc, _turned
from tests.test_gpu_rotary import _freq

pytestmark = pytest.mark.gpu


# query heads at which the pieces of a row (queries, one KV head's key and value of 64 channels) are 1024, or just below, and the next; rot, paired, dtype
@pytest.mark.parametrize("Hq,rot,paired,dtype", [(253, 64, False, "bf16"), (15, 6, False, "bf16"), (126, 64, True, "bf16"), (125, 64, False, "f32"), (62, 64, True, "f32"), (16, 10, False, "f32")])
@pytest.mark.parametrize("more", [0, 1])
def test_all_of_a_row(Hq, rot, paired, dtype, more):
    Hq += more
    R, D, page = 1030, 64, 64
    rng = np.random.default_rng([Hq, rot])
    pages = pc.Pages(rng, page, [R + 7])
    q, k, v = (pc.rounded(rng.standard_normal((1, R, h, D)), dtype) for h in (Hq, 1, 1))
    dq, dk, dv = (pc.device(x, dtype) for x in (q, k, v))
    q_out = torch.full_like(dq, 9.0)
    kp, vp = (torch.full((pages.n_pages, 1, page, D), 9.0, dtype=pc.DTYPES[dtype], device="cuda") for _ in range(2))
    freq = _freq(rot)
    dream.dream_paged_append(_desc(1, Hq, 1, D, dtype), dream.page_desc(page, pages.n_pages, pages.max_pages), pages.device_table(), dq, dk, dv, R, wc.ints([7]), None, None, None, None, None,
                             torch.from_numpy(freq).cuda(), rot, paired, 1.0, q_out, kp, vp)
    torch.cuda.synchronize()
    pos = 7 + np.arange(R)[None]
    _turned(q, pos, freq, rot, paired, 1.0, q_out.double().cpu().numpy(), dtype)
    _turned(k, pos, freq, rot, paired, 1.0, pages.get(kp.double().cpu().numpy(), 0, 7, R).transpose(1, 0, 2)[None], dtype)
    assert np.array_equal(pages.get(vp.double().cpu().numpy(), 0, 7, R).transpose(1, 0, 2), v[0])
