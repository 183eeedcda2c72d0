"""Caches in pages for the tests: pools filled from dense caches, and the definitions in 64 bits (numpy, on the host)."""
import numpy as np
import torch

from tests import window_cases as wc

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(x, dtype):
    return wc.bf16(x) if dtype == "bf16" else np.asarray(x, dtype=np.float32).astype(np.float64)


def device(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DTYPES[dtype]).cuda()


class Pages:
    """A page table over a pool that gives its pages out in no order.  shared[b] = (first sequence, whole pages that are the same)."""

    def __init__(self, rng, page, rows, shared=None, spare=2, behind=-1, extra=1):
        self.page, self.B = page, len(rows)
        need = [-(-r // page) for r in rows]
        self.max_pages = max(need) + extra
        self.n_pages = sum(need) + spare
        ids = [int(i) for i in rng.permutation(self.n_pages)]
        self.table = np.full((self.B, self.max_pages), behind, dtype=np.int64)
        for b, n in enumerate(need):
            first, same = shared[b] if shared else (b, 0)
            same = same if first != b else 0
            self.table[b, :same] = self.table[first, :same]
            self.table[b, same:n] = [ids.pop() for _ in range(n - same)]

    def where(self, b, j):
        return self.table[b, j // self.page], j % self.page

    def pool(self, heads, D, fill=np.nan):
        return np.full((self.n_pages, heads, self.page, D), fill)

    def put(self, pool, b, j0, rows):
        """rows [heads, n, D] from position j0 on."""
        for i in range(rows.shape[1]):
            page, at = self.where(b, j0 + i)
            pool[page, :, at] = rows[:, i]

    def get(self, pool, b, j0, n):
        return np.stack([pool[self.where(b, j)[0], :, self.where(b, j)[1]] for j in range(j0, j0 + n)], 1) if n else pool[0, :, :0]

    def device_table(self):
        return wc.ints(self.table)


def attend(q, k, v, see, scale=None):
    """q [T, Hq, D], k, v [Hkv, S, D], see [Hkv, T, S] of one sequence.  Rows, log-sum-exps [Hq, T], sums of p |v|, and the largest sum of |q k| scale [Hq, T].  What a node does not see is
    not looked at."""
    T, Hq, D = q.shape
    G = Hq // k.shape[0]
    scale = D ** -0.5 if scale is None else scale
    out, lse, mass, size = np.zeros(q.shape), np.full((Hq, T), -np.inf), np.zeros(q.shape), np.zeros((Hq, T))
    for h in range(Hq):
        for i in range(T):
            w = np.flatnonzero(see[h // G, i])
            if not len(w):
                continue
            kk, vv = k[h // G][w], v[h // G][w]
            with np.errstate(invalid="ignore", over="ignore"):
                x = kk @ q[i, h] * scale
                keep = x != -np.inf                      # (such a key has weight 0)
                if not keep.any():
                    continue
                x, vv, kk = x[keep], vv[keep], kk[keep]
                top = x.max()
                p = np.exp(x - top)
                lse[h, i] = top + np.log(p.sum())
                p /= p.sum()
                out[i, h] = p @ vv
                mass[i, h] = p @ np.abs(vv)
                size[h, i] = (np.abs(kk) @ np.abs(q[i, h])).max() * abs(scale)
    return out, lse, mass, size


def check_rows(got, got_lse, want, want_lse, mass, size, n_keys, D, dtype):
    """All elements of one sequence's rows within what rounding may move (window_cases.attention_bounds)."""
    row, lse = wc.attention_bounds(want[None], mass[None], size[None], n_keys, D, dtype == "bf16")
    err = np.abs(got - want)
    assert (err <= row[0]).all(), float((err / row[0]).max())
    if got_lse is not None:
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), empty)
        e = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, want_lse))
        # (the result's own rounding: half a step of 2^-23 of it, twice)
        assert (e <= np.broadcast_to(lse[0], e.shape) + 2.0 ** -23 * np.abs(np.where(empty, 0, want_lse)) + 1e-6).all()


# ---- selection -------------------------------------------------------------------------------------------------------
def least_exponent(top):
    """Least e in [-100, 122] with top <= 127 * 2^e."""
    m, e = np.frexp(np.asarray(top, dtype=np.float64) / 127.0)
    return np.where(top > 0, np.clip(e - (m == 0.5), -100, 122), -100).astype(int)


def choose(q, bounds, first, last, best):
    """q [T, Hq, D] and bounds [pages, Hkv, 2, D] of one sequence, float64: [Hkv, T, pages] truth values."""
    T, Hq, D = q.shape
    n, Hkv = bounds.shape[:2]
    picked = np.zeros((Hkv, T, n), dtype=bool)
    picked[:, :, :first] = True
    picked[:, :, max(0, n - last):] = True
    lo, hi = min(first, n), max(n - last, min(first, n))
    for h in range(Hkv):
        strange = ~np.isfinite(bounds[:, h]).all((1, 2))
        x = np.where(strange[:, None, None], 0.0, bounds[:, h])
        e = least_exponent(np.abs(x).max((1, 2)) if n else np.zeros(0))
        x = np.ldexp(x, -e[:, None, None])
        up, down = np.ceil(x[:, 0]), np.floor(x[:, 1])
        for i in range(T):
            rows = q[i, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)]
            c = np.rint(np.ldexp(rows, -least_exponent(np.abs(rows).max())))
            s = up @ np.maximum(c, 0).sum(0) + down @ np.minimum(c, 0).sum(0)
            s = np.ldexp(s.astype(np.float32).astype(np.float64), e)
            with np.errstate(over="ignore"):
                s = s.astype(np.float32)
            s[strange] = np.inf
            order = lo + np.argsort(-s[lo:hi], kind="stable")[:best]
            picked[h, i, order] = True
    return picked


def words(picked, max_pages):
    """[Hkv, max_pages, W] int64 of [Hkv, T, pages]."""
    Hkv, T, n = picked.shape
    w = np.zeros((Hkv, max_pages, (T + 63) // 64), dtype=np.uint64)
    for i in range(T):
        w[:, :n, i // 64] |= picked[:, i].astype(np.uint64) << np.uint64(i % 64)
    return w.view(np.int64)


def page_bounds(rows):
    """rows [heads, n, D] of a page: [heads, 2, D]."""
    strange = ~np.isfinite(rows).all(1)
    x = np.where(np.isfinite(rows), rows, 0.0)
    return np.stack([np.where(strange, np.inf, x.max(1)), np.where(strange, -np.inf, x.min(1))], 1)
