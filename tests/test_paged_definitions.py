"""No-GPU pins of the definitions in 64 bits that the GPU tests of paged attention compare with (tests/paged_cases.py)."""
import numpy as np
import torch

from tests import paged_cases as pc


def _problem(seed, T=5, Hq=6, Hkv=2, D=16, S=23):
    rng = np.random.default_rng(seed)
    see = rng.random((Hkv, T, S)) < 0.5
    return rng.standard_normal((T, Hq, D)), rng.standard_normal((Hkv, S, D)), rng.standard_normal((Hkv, S, D)), see


def test_attend_is_masked_softmax_attention():
    """Every query head over its KV head's keys, what each KV head's nodes see of their own: torch's attention in 64 bits; log-sum-exps by torch's."""
    for seed, scale in ((0, None), (1, 0.4), (2, -0.3)):
        q, k, v, see = _problem(seed)
        see[:, :, 0] = True
        out, lse, mass, size = pc.attend(q, k, v, see, scale)
        G = q.shape[1] // k.shape[0]
        qt, kt, vt = (torch.from_numpy(x) for x in (q.transpose(1, 0, 2).copy(), np.repeat(k, G, 0), np.repeat(v, G, 0)))
        mask = torch.from_numpy(np.repeat(see, G, 0))
        want = torch.nn.functional.scaled_dot_product_attention(qt, kt, vt, attn_mask=mask, scale=scale)
        assert np.abs(out.transpose(1, 0, 2) - want.numpy()).max() < 1e-12
        x = (qt @ kt.transpose(1, 2) * (q.shape[2] ** -0.5 if scale is None else scale)).masked_fill(~mask, -np.inf)
        assert np.abs(lse - torch.logsumexp(x, -1).numpy()).max() < 1e-12
        p = torch.softmax(x, -1)
        assert np.abs(mass.transpose(1, 0, 2) - (p @ vt.abs()).numpy()).max() < 1e-12
        terms = (kt.abs()[:, None] * qt.abs()[:, :, None]).sum(-1) * abs(q.shape[2] ** -0.5 if scale is None else scale)
        assert np.abs(size - terms.masked_fill(~mask, -np.inf).amax(-1).numpy()).max() < 1e-12


def test_attend_of_nothing_is_zero():
    q, k, v, see = _problem(3)
    see[1, 2] = False
    out, lse, mass, size = pc.attend(q, k, v, see)
    assert not out[2, 3:].any() and np.isneginf(lse[3:, 2]).all() and not mass[2, 3:].any() and not size[3:, 2].any()
    assert out[2, :3].any() and np.isfinite(lse[:3]).all()


def test_attend_looks_at_nothing_unseen_and_skips_scores_of_minus_infinity():
    q, k, v, see = _problem(4)
    q = np.abs(q)
    see[:, :, :2] = True
    see[:, :, 7] = False
    want = pc.attend(q, k, v, see)
    other_k, other_v = k.copy(), v.copy()
    other_k[:, 7] = other_v[:, 7] = np.nan
    for x, y in zip(pc.attend(q, other_k, other_v, see), want):
        assert np.array_equal(x, y)
    seen = see.copy()
    seen[:, :, 7] = True
    other_k[:, 7] = -np.inf
    for x, y in zip(pc.attend(q, other_k, other_v, seen), want):      # (one more row in a product: sums of up to 23 terms below 30 in another order, 2^-53 of each)
        assert np.abs(x - y).max() < 1e-12


def test_pages_hold_rows_in_their_order():
    rng = np.random.default_rng(5)
    pages = pc.Pages(rng, 16, [40, 33, 50], [(0, 0), (0, 2), (2, 0)])
    assert (pages.table[1, :2] == pages.table[0, :2]).all()
    used = [int(p) for b, n in enumerate((3, 3, 4)) for p in pages.table[b, :n]]
    assert len(set(used)) == len(used) - 2 and (pages.table[:, 4:] == -1).all()
    pool, rows = pages.pool(2, 8), rng.standard_normal((2, 50, 8))
    pages.put(pool, 2, 0, rows)
    assert np.array_equal(pages.get(pool, 2, 0, 50), rows)
    for j in (0, 15, 16, 49):
        assert np.array_equal(pool[pages.table[2, j // 16], :, j % 16], rows[:, j])
