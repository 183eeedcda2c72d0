"""Jobs of one dream_rotary_rows call whose memory overlaps: refused before a launch where both sides are dense (no GPU needed), and the calls beside them that are allowed."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import window_cases as wc
from tests.test_operator_refusals import _caller, _desc, _Job, lib  # noqa: F401

SIZE = 2 * 10 * 128 * 2        # bytes of a head of all rows


def _call(lib, *jobs):  # noqa: F811
    call = _caller(lib, "dream_rotary_rows", desc=_desc(), n_rows=10, rot_dim=128, interleaved=0, amplitude=1.0)
    return call(jobs=(_Job * len(jobs))(*[_Job(*j) for j in jobs]), n_jobs=len(jobs))


X, Y = 0x100000, 0x900000


@pytest.mark.parametrize("jobs", [
    [(X, 8, None, None, X + 16)],                                               # its own rows, shifted
    [(X, 8, None, None, X - 8 * SIZE + 16)],
    [(X, 8, None, None, X + 8 * SIZE - 16)],
    [(X, 8, None, None, X), (X, 8, None, None, Y)],                             # turned in place, and read by another job
    [(X, 8, None, None, Y), (X, 8, None, None, X)],
    [(X, 8, None, None, X), (X, 8, None, None, X)],
    [(X, 8, None, None, X), (X + 7 * SIZE, 2, None, None, Y)],                  # its last head is the other's first
    [(X, 8, None, None, Y), (X + 8 * SIZE, 2, None, None, Y + 8 * SIZE - 16)],  # both write the same bytes
    [(X, 8, None, None, X), (X, 8, 0x40, None, Y)],                             # turned in place, and into a cache from the same rows
], ids=str)
def test_refused(lib, jobs):  # noqa: F811
    assert _call(lib, *jobs) == -1
    assert "overlaps" in dream.dream_last_error()


@pytest.mark.gpu
def test_neighbours_in_one_buffer():
    """Queries and keys side by side in one buffer, turned in place by one call; the same rows read by two jobs that write elsewhere."""
    B, R, H, K, D = 2, 6, 4, 2, 64
    rng = np.random.default_rng(2)
    n, m = B * R * H * D, B * R * K * D
    buf = torch.from_numpy(wc.bf16(rng.standard_normal(n + m + 64))).bfloat16().cuda()
    q, k = buf[:n].view(B, R, H, D), buf[n:n + m].view(B, R, K, D)
    was = buf.double().cpu().numpy()
    f = rng.random(32).astype(np.float32)
    pos = np.arange(B * R).reshape(B, R) * 31
    desc = dream.attn_desc(B, H, K, D, dream.BF16, 1)
    a, b = torch.empty_like(q), torch.empty_like(q)
    dream.dream_rotary_rows(desc, [(q, H, None, None, a), (q, H, None, None, b)], R, wc.ints(pos), None, None, torch.from_numpy(f).cuda(), D)
    dream.dream_rotary_rows(desc, [(q, H, None, None, q), (k, K, None, None, k)], R, wc.ints(pos), None, None, torch.from_numpy(f).cuda(), D)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, q)
    for t, x in ((q, was[:n].reshape(B, R, H, D)), (k, was[n:n + m].reshape(B, R, K, D))):
        want = wc.rotary(x, pos, f, D, False)
        # the row's rounding, and turns and products in float32
        size = np.abs(x) + np.abs(np.roll(x, 32, -1))
        assert (np.abs(t.double().cpu().numpy() - want) <= np.abs(want) * 2.0 ** -8 + size * 2.0 ** -20).all()
    assert np.array_equal(buf[n + m:].double().cpu().numpy(), was[n + m:])
