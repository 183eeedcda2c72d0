"""GPU parity of dream_paged_append, dream_paged_commit, dream_page_bounds and dream_page_select against the definitions in 64 bits, all elements; and a round of them together."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import paged_cases as pc
from tests import window_cases as wc
from tests.test_gpu_rotary import _bound, _freq

pytestmark = pytest.mark.gpu


def _desc(B, Hq, Hkv, D, dtype):
    return dream.attn_desc(B, Hq, Hkv, D, dream.BF16 if dtype == "bf16" else dream.F32, 0)


def _turned(x, pos, freq, rot, paired, amplitude, got, dtype):
    want = wc.rotary(x, pos, freq, rot, paired, amplitude)
    assert (np.abs(got - want) <= _bound(x, want, rot, paired, amplitude, dtype)).all()
    assert np.array_equal(got[..., rot:], x[..., rot:])


# Hq, Hkv, D, rows, page, rot, paired, positions, dtype
APPEND = [
    (4, 2, 64, 1, 16, 64, False, "base", "bf16"),
    (8, 2, 128, 60, 64, 128, False, "tree", "bf16"),
    (4, 4, 256, 33, 32, 256, True, "tree", "bf16"),
    (4, 1, 128, 17, 128, 32, True, "pos", "bf16"),
    (2, 2, 64, 100, 16, 6, False, "pos_base", "bf16"),
    (4, 2, 64, 256, 256, 64, False, "chain", "bf16"),
    (4, 2, 64, 21, 16, 64, True, "tree", "f32"),
    (2, 1, 256, 5, 64, 100, False, "pos", "f32"),
    (0, 2, 128, 40, 64, 128, False, "tree", "bf16"),       # keys and values alone
    (4, 2, 128, 40, 64, 0, False, "none", "bf16"),         # nothing turns
    (32, 8, 128, 300, 64, 64, True, "base", "bf16"),
]


@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append(case):
    Hq, Hkv, D, R, page, rot, paired, kind, dtype = case
    rng = np.random.default_rng([Hq, D, R])
    base = [0, 77, 33]
    B = len(base)
    pages = pc.Pages(rng, page, [p + R for p in base])
    q, k, v = (pc.rounded(rng.standard_normal((B, R, h, D)), dtype) for h in (max(Hq, 1), Hkv, Hkv))
    parent = [wc.tree("chain" if kind == "chain" else "rand", R, rng) for _ in base]
    pos = {"base": np.array(base)[:, None] + np.arange(R), "pos_base": np.array([5, 100000, 2 ** 31 - 1 - R])[:, None] + np.arange(R), "pos": rng.integers(-50, 5000, (B, R))}.get(kind)
    if kind in ("tree", "chain"):
        pos = np.array([[p + len(a) - 1 for a in wc.ancestors(t)] for p, t in zip(base, parent)])
    amplitude = 1.25 if paired else 1.0
    freq = _freq(rot) if rot else None
    dq, dk, dv = (pc.device(x, dtype) for x in (q, k, v))
    q_out = torch.full_like(dq, 9.0) if Hq else None
    kp, vp = (torch.full((pages.n_pages, Hkv, page, D), 9.0, dtype=pc.DTYPES[dtype], device="cuda") for _ in range(2))
    dream.dream_paged_append(_desc(B, max(Hq, Hkv), Hkv, D, dtype), dream.page_desc(page, pages.n_pages, pages.max_pages), pages.device_table(), dq if Hq else None, dk, dv, R,
                             wc.ints(base), None, None, wc.ints(pos) if kind == "pos" else None, wc.ints([5, 100000, 2 ** 31 - 1 - R]) if kind == "pos_base" else None,
                             wc.ints(parent) if kind in ("tree", "chain") else None, torch.from_numpy(freq).cuda() if rot else None, rot, paired, amplitude, q_out, kp, vp)
    torch.cuda.synchronize()
    gk, gv = kp.double().cpu().numpy(), vp.double().cpu().numpy()
    for b, p in enumerate(base):
        rows = pages.get(gk, b, p, R).transpose(1, 0, 2)
        if rot:
            _turned(k[b:b + 1], pos[b:b + 1], freq, rot, paired, amplitude, rows[None], dtype)
        else:
            assert np.array_equal(rows, k[b])
        assert np.array_equal(pages.get(gv, b, p, R).transpose(1, 0, 2), v[b])
        for g in (gk, gv):
            pages.put(g, b, p, np.full((Hkv, R, D), 9.0))
    assert (gk == 9.0).all() and (gv == 9.0).all()
    if Hq and rot:
        _turned(q, pos, freq, rot, paired, amplitude, q_out.double().cpu().numpy(), dtype)
    elif Hq:
        assert torch.equal(q_out, dq)


def test_append_in_place_padded_scattered_and_dropped():
    """Queries turned where they stand; padding is neither read nor written; a row outside the table, or whose page is none, is dropped."""
    rng = np.random.default_rng(2)
    B, R, H, D, page = 3, 6, 2, 64, 16
    pages = pc.Pages(rng, page, [40, 40, 40], extra=0)
    t = pages.table.copy()
    t[1, 0], t[2, 0] = -1, pages.n_pages
    k = rng.standard_normal((B, R, H, D))
    k[0, 4:] = np.nan
    dk = pc.device(k, "bf16")
    q = dk.clone()
    q[0, 4:] = 5.0
    held = q.clone()
    index = [[3, 0, 7, 1, 2, 4], [0, 20, 15, 16, 47, 48], [-1, 16, 31, 2 ** 31 - 1, 30, 0]]
    kp, vp = (torch.full((pages.n_pages, H, page, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    freq = torch.from_numpy(_freq(D)).cuda()
    dream.dream_paged_append(_desc(B, H, H, D, "bf16"), dream.page_desc(page, pages.n_pages, pages.max_pages), wc.ints(t), q, dk, dk, R, wc.ints([2, 0, 0]), wc.ints(index),
                             wc.ints([4, 6, 100]), None, None, None, freq, D, False, 1.0, q, kp, vp)
    torch.cuda.synchronize()
    assert torch.equal(q[0, 4:], held[0, 4:]) and not torch.equal(q[0, 1:4], held[0, 1:4])
    gv = vp.double().cpu().numpy()
    written = {(0, 5): 0, (0, 2): 1, (0, 9): 2, (0, 3): 3, (1, 20): 1, (1, 16): 3, (1, 47): 4, (2, 16): 1, (2, 31): 2, (2, 30): 4}
    for (b, j), r in written.items():
        at = pages.where(b, j)
        assert np.array_equal(gv[at[0], :, at[1]], dk[b, r].double().cpu().numpy())
        gv[at[0], :, at[1]] = 9.0
    assert (gv == 9.0).all()
    live = dream.dream_paged_append
    before = kp.clone()
    live(_desc(B, H, H, D, "bf16"), dream.page_desc(page, pages.n_pages, pages.max_pages), wc.ints(t), None, dk, dk, R, wc.ints([2, 0, 0]), None, wc.ints([0, -3, 0]), None, None, None,
         None, 0, False, 1.0, None, kp, vp)
    torch.cuda.synchronize()
    assert torch.equal(kp, before)


@pytest.mark.parametrize("Hkv,D,T,stride,page,n_pools,dtype", [(2, 64, 12, 7, 16, 3, "bf16"), (8, 128, 60, 7, 64, 4, "bf16"), (3, 256, 33, 40, 16, 2, "bf16"), (2, 64, 1, 1, 32, 1, "bf16"),
                                                               (2, 128, 9, 7, 16, 200, "bf16"), (4, 64, 20, 7, 16, 2, "f32"), (1, 128, 256, 200, 128, 2, "bf16")])
def test_commit(Hkv, D, T, stride, page, n_pools, dtype):
    rng = np.random.default_rng([Hkv, D, T])
    prefix = [0, 61, 30, 15]
    B = len(prefix)
    pages = pc.Pages(rng, page, [p + T for p in prefix])
    most = min(stride, T)
    length = [0, most - 1, most // 2, min(2, most - 1)]
    path = np.full((B, stride), -1)
    for b, n in enumerate(length):
        path[b, :n + 1] = [0] + sorted(rng.choice(np.arange(1, T), n, replace=False)) if n else [0]
    pools = [torch.randn(pages.n_pages, Hkv, page, D, device="cuda").to(pc.DTYPES[dtype]) for _ in range(n_pools)]
    want = []
    for x in pools:
        x = x.double().cpu().numpy()
        for b, (p, n) in enumerate(zip(prefix, length)):
            old = pages.get(x, b, p, T)
            pages.put(x, b, p, old[:, path[b, :n + 1]])
        want.append(x)
    new = wc.ints([-1] * B)
    dream.dream_paged_commit(_desc(B, Hkv, Hkv, D, dtype), dream.page_desc(page, pages.n_pages, pages.max_pages), pages.device_table(), pools, wc.ints(prefix), T, wc.ints(path),
                             wc.ints(length), new)
    torch.cuda.synchronize()
    assert new.tolist() == [p + n + 1 for p, n in zip(prefix, length)]
    for x, w in zip(pools, want):
        assert np.array_equal(x.double().cpu().numpy(), w)


def test_commit_drops_rows_of_pages_that_are_none():
    rng = np.random.default_rng(4)
    pages = pc.Pages(rng, 16, [40], extra=0)
    t = pages.table.copy()
    t[0, 2] = 10 ** 6                                  # rows 32 ..
    pool = torch.randn(pages.n_pages, 2, 16, 64, device="cuda").to(torch.bfloat16)
    want = pool.clone()
    a, b = pages.where(0, 30), pages.where(0, 31)
    want[int(a[0]), :, a[1]], want[int(b[0]), :, b[1]] = pool[int(a[0]), :, a[1]], pool[int(b[0]), :, b[1]]
    # destinations 30, 31, 32, 33; sources 30, 35 (no page), 36 (none), 31: nothing that is written may come from, or go to, a page that is none
    dream.dream_paged_commit(_desc(1, 2, 2, 64, "bf16"), dream.page_desc(16, pages.n_pages, 3), wc.ints(t), [pool], wc.ints([30]), 10, wc.ints([[0, 5, 6, 1]]), wc.ints([3]))
    torch.cuda.synchronize()
    assert torch.equal(pool, want)


@pytest.mark.parametrize("Hkv,D,page,dtype", [(2, 64, 16, "bf16"), (3, 128, 64, "bf16"), (1, 256, 256, "bf16"), (2, 128, 32, "f32"), (2, 64, 128, "f32"), (2, 256, 16, "f32"), (5, 64, 32, "bf16"), (3, 128, 16, "f32"), (6, 256, 16, "bf16")])
@pytest.mark.parametrize("max_new", [1, 40, 10 ** 6])
def test_bounds(Hkv, D, page, dtype, max_new):
    rng = np.random.default_rng([Hkv, D, page])
    rows = [500, 33, 64, 20, 10]
    start, end = [0, 17, 64, 19, 3], [500, 33, 64, 20, 3]
    pages = pc.Pages(rng, page, rows)
    x = pages.pool(Hkv, D)
    for b, n in enumerate(rows):
        pages.put(x, b, 0, pc.rounded(rng.standard_normal((Hkv, n, D)) - 3.0 * (b == 1), dtype))
    at = pages.where(0, 7)
    x[at[0], 0, at[1], 3] = np.nan
    x[at[0], Hkv - 1, at[1], 5] = np.inf
    x[at[0], Hkv - 1, at[1], 6] = -np.inf
    got = torch.full((pages.n_pages, Hkv, 2, D), 9.0, dtype=pc.DTYPES[dtype], device="cuda")
    want = np.full(got.shape, 9.0)
    for b, (s, e) in enumerate(zip(start, end)):
        if e > s:
            for i in range(s // page, -(-e // page)):
                want[pages.table[b, i]] = pc.page_bounds(x[pages.table[b, i], :, :min(page, e - i * page)])
    pd = dream.page_desc(page, pages.n_pages, pages.max_pages)
    dream.dream_page_bounds(_desc(len(rows), Hkv, Hkv, D, dtype), pd, pages.device_table(), pc.device(x, dtype), wc.ints(start), wc.ints(end), max_new, got)
    torch.cuda.synchronize()
    assert np.array_equal(got.double().cpu().numpy(), want)
    dream.dream_page_bounds(_desc(len(rows), Hkv, Hkv, D, dtype), pd, pages.device_table(), pc.device(x, dtype), None, wc.ints(end), max_new, got)
    torch.cuda.synchronize()
    for b, e in enumerate(end):
        for i in range(-(-e // page)):
            want[pages.table[b, i]] = pc.page_bounds(x[pages.table[b, i], :, :min(page, e - i * page)])
    assert np.array_equal(got.double().cpu().numpy(), want)


# Hq, Hkv, D, T, pages of the prefixes, first, last, best, dtype
SELECT = [
    (4, 2, 64, 1, [0, 1, 40], 1, 1, 5, "bf16"),
    (4, 4, 128, 7, [300, 17], 0, 1, 16, "bf16"),
    (8, 1, 128, 60, [257, 64], 2, 3, 9, "bf16"),
    (2, 1, 256, 33, [100], 0, 0, 7, "bf16"),
    (4, 2, 64, 64, [65, 63], 1, 0, 1, "bf16"),
    (2, 2, 64, 100, [130], 3, 2, 30, "bf16"),
    (2, 1, 64, 256, [70], 0, 0, 64, "bf16"),
    (4, 2, 64, 3, [2500, 40], 4, 2, 50, "bf16"),
    (16, 1, 64, 2, [100], 0, 0, 0, "bf16"),
    (4, 2, 64, 2, [20], 50, 0, 3, "bf16"),
    (4, 2, 64, 2, [20], 0, 2 ** 31 - 1, 3, "bf16"),
    (4, 2, 64, 2, [20], 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, "bf16"),
    (64, 1, 64, 3, [90], 1, 1, 10, "bf16"),
    (4, 2, 128, 9, [200, 3], 1, 1, 10, "f32"),
    (2, 2, 256, 5, [90], 1, 1, 10, "f32"),
    (4, 2, 64, 1, [300, 2048], 1, 1, 16, "bf16"),
    (2, 2, 64, 1, [3000, 8], 2, 3, 100, "bf16"),
    (1, 1, 64, 1, [8300], 0, 1, 7, "bf16"),
    (4, 2, 64, 20, [600, 1024], 1, 1, 40, "bf16"),
    (2, 1, 64, 70, [1500, 33], 1, 2, 64, "bf16"),
    (14, 2, 128, 67, [400], 1, 1, 12, "bf16"),
    (10, 2, 64, 17, [90, 5], 1, 0, 12, "f32"),
]


def _select(q, bounds, table, pd, desc, prefix, T, first, last, best, max_kv):
    nodes = torch.full((len(prefix), desc.n_kv_heads, pd.max_pages, (T + 63) // 64), 0x55, dtype=torch.int64, device="cuda")
    ws = dream.alloc_workspace(dream.dream_page_select_workspace(desc, pd, T, max_kv)).fill_(0xFF)
    dream.dream_page_select(desc, pd, table, q, bounds, wc.ints(prefix), T, first, last, best, max_kv, nodes, ws)
    torch.cuda.synchronize()
    return nodes.cpu().numpy()


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("case", SELECT, ids=str)
def test_select(case, ties):
    """Equal to the definition, page for page; `ties`: bounds of few values, so that many scores are equal."""
    Hq, Hkv, D, T, n, first, last, best, dtype = case
    rng = np.random.default_rng([Hq, D, T, n[0], ties])
    page = 16
    prefix = [max(0, x * page - int(rng.integers(0, page))) for x in n]
    pages = pc.Pages(rng, page, [p + T for p in prefix])
    if ties:
        b64 = rng.integers(0, 2, (pages.n_pages, Hkv, 2, 1)) * np.ones(D)
        q64 = rng.integers(-1, 2, (len(n), T, Hq, 1)) * np.ones(D)
    else:
        size = np.exp2(rng.integers(-9, 9, (pages.n_pages, Hkv, 1, 1)) * (rng.random((pages.n_pages, 1, 1, 1)) < 0.2))
        x = pc.rounded(rng.standard_normal((pages.n_pages, Hkv, 2, D)) * size, dtype)
        b64 = np.stack([x.max(2), x.min(2)], 2)
        q64 = pc.rounded(rng.standard_normal((len(n), T, Hq, D)) * np.exp2(rng.integers(-20, 20, (len(n), T, 1, 1))), dtype)
    pd, desc = dream.page_desc(page, pages.n_pages, pages.max_pages), _desc(len(n), Hq, Hkv, D, dtype)
    got = _select(pc.device(q64, dtype), pc.device(b64, dtype), pages.device_table(), pd, desc, prefix, T, first, last, best, max(prefix) + T)
    for b, p in enumerate(prefix):
        of = b64[pages.table[b, :-(-p // page)]]
        assert np.array_equal(got[b], pc.words(pc.choose(q64[b], of, first, last, best), pages.max_pages))


def test_select_extreme_values():
    """The largest and smallest numbers, zeros, and bounds that are not finite."""
    rng = np.random.default_rng(9)
    T, Hq, Hkv, D, page, n = 5, 4, 2, 64, 16, 60
    for scale in (2.0 ** 120, 2.0 ** -120, 0.0):
        x = pc.rounded(rng.standard_normal((n + 4, Hkv, 2, D)) * scale, "bf16")
        if scale > 1:
            x[7], x[8] = 3.3895313892515355e38, -3.3895313892515355e38
        b64 = np.stack([x.max(2), x.min(2)], 2)
        b64[11, 0, 0, 3], b64[12, 1, 1, 60], b64[13, 0, 1, 0] = np.inf, -np.inf, np.nan
        q64 = pc.rounded(rng.standard_normal((1, T, Hq, D)) * scale, "bf16")
        pd, desc = dream.page_desc(page, n + 4, n + 1), _desc(1, Hq, Hkv, D, "bf16")
        table = [rng.permutation(n + 4)[:n + 1]]
        got = _select(pc.device(q64, "bf16"), pc.device(b64, "bf16"), wc.ints(table), pd, desc, [n * page], T, 1, 1, 6, n * page + T)
        assert np.array_equal(got[0], pc.words(pc.choose(q64[0], b64[table[0][:n]], 1, 1, 6), n + 1))


def test_select_takes_rows_behind_max_kv_len_as_not_there():
    rng = np.random.default_rng(3)
    T, n, page = 4, 30, 16
    b64, q64 = pc.rounded(rng.standard_normal((n + 1, 2, 2, 64)), "bf16"), pc.rounded(rng.standard_normal((2, T, 4, 64)), "bf16")
    table = [rng.permutation(n + 1), rng.permutation(n + 1)]
    got = _select(pc.device(q64, "bf16"), pc.device(b64, "bf16"), wc.ints(table), dream.page_desc(page, n + 1, n + 1), _desc(2, 4, 2, 64, "bf16"), [n * page, -4], T, 1, 1, 5, 200 + T)
    assert np.array_equal(got[0], pc.words(pc.choose(q64[0], b64[table[0][:13]], 1, 1, 5), n + 1))
    assert not got[1].any()


@pytest.mark.parametrize("captured", [False, True])
def test_a_round_together(captured):
    """A prompt enters the cache with its bounds; then rounds of append, selection, attention, commit and bounds, each checked against the definitions on what the pools hold; captured: the
    round is one graph, replayed."""
    rng = np.random.default_rng(6)
    B, T, Hq, Hkv, D, page, prompt, dtype = 2, 13, 4, 2, 128, 16, [90, 133], "bf16"
    first, last, best = 1, 2, 3
    pages = pc.Pages(rng, page, [p + 60 for p in prompt])
    pd, desc = dream.page_desc(page, pages.n_pages, pages.max_pages), _desc(B, Hq, Hkv, D, dtype)
    table, freq = pages.device_table(), torch.from_numpy(_freq(D)).cuda()
    kp, vp = (torch.zeros(pages.n_pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bounds = torch.zeros(pages.n_pages, Hkv, 2, D, dtype=torch.bfloat16, device="cuda")
    R = max(prompt)
    rows = torch.randn(2, B, R, Hkv, D, device="cuda").to(torch.bfloat16)
    length = wc.ints(prompt)
    dream.dream_paged_append(desc, pd, table, None, rows[0], rows[1], R, wc.ints([0] * B), None, length, None, None, None, freq, D, False, 1.0, None, kp, vp)
    dream.dream_page_bounds(desc, pd, table, kp, None, length, R, bounds)
    parent = [wc.tree("rand", T, rng) for _ in range(B)]
    paths = []
    for t in parent:
        p = wc.ancestors(t)[T - 1][::-1][:7]
        paths.append(p + [-1] * (7 - len(p)))
    accepted = [sum(x >= 0 for x in p) - 1 for p in paths]
    par, path, alen, new = wc.ints(parent), wc.ints(paths), wc.ints(accepted), wc.ints([0] * B)
    q, k, v = (torch.empty(B, T, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(B, Hq, T, device="cuda")
    nodes = torch.empty(B, Hkv, pd.max_pages, 1, dtype=torch.int64, device="cuda")
    cap = max(prompt) + 60
    ws = dream.alloc_workspace(max(dream.dream_page_select_workspace(desc, pd, T, cap), dream.dream_sparse_verify_attn_workspace(desc, pd, T, cap, first + last + best)))

    def step():
        dream.dream_paged_append(desc, pd, table, q, k, v, T, length, None, None, None, None, par, freq, D, False, 1.0, q_out, kp, vp)
        dream.dream_page_select(desc, pd, table, q_out, bounds, length, T, first, last, best, cap, nodes, ws)
        dream.dream_sparse_verify_attn(desc, pd, q_out, kp, vp, table, nodes, length, T, par, None, cap, first + last + best, out, lse, ws)
        dream.dream_paged_commit(desc, pd, table, [kp, vp], length, T, path, alen, new)
        dream.dream_page_bounds(desc, pd, table, kp, length, new, 7, bounds)

    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for _ in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda"))
        old_bounds, old = bounds.double().cpu().numpy(), length.tolist()
        before = [x.double().cpu().numpy() for x in (kp, vp)]
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        pos = np.array([[p + len(a) - 1 for a in wc.ancestors(t)] for p, t in zip(old, parent)])
        q64 = q_out.double().cpu().numpy()
        _turned(q.double().cpu().numpy(), pos, freq.cpu().numpy(), D, False, 1.0, q64, dtype)
        got = [x.double().cpu().numpy() for x in (kp, vp)]
        for b, p in enumerate(old):
            turned = wc.rotary(k[b:b + 1].double().cpu().numpy(), pos[b:b + 1], freq.cpu().numpy(), D, False)
            pages.put(before[0], b, p, wc.bf16(turned)[0].transpose(1, 0, 2))
            pages.put(before[1], b, p, v[b].double().cpu().numpy().transpose(1, 0, 2))
            n = -(-p // page)
            picked = pc.choose(q64[b], old_bounds[pages.table[b, :n]], first, last, best)
            assert np.array_equal(nodes[b].cpu().numpy(), pc.words(picked, pd.max_pages))
            see = np.repeat(wc.visible(parent[b], p, 0, 0)[None], Hkv, 0)
            see[:, :, :p] &= np.repeat(picked, page, -1)[:, :, :p]
            keys, values = (pages.get(x, b, 0, p + T) for x in before)
            want = pc.attend(q64[b], keys, values, see)
            # (a turned key may be the other neighbour of where it was rounded: a step of 2^-8 of it, which moves a score by as much of its terms)
            want[3][:] = want[3] * (1 + 2.0 ** 17 / D)
            pc.check_rows(out[b].double().cpu().numpy(), None, *want, p + T, D, dtype)
            for g, w in zip(got, before):
                moved = pages.get(w, b, p, T)[:, paths[b][:accepted[b] + 1]]
                assert (np.abs(pages.get(g, b, p, accepted[b] + 1) - moved) <= np.abs(moved) * 2.0 ** -7 + 1e-5).all()
            for i in range(p // page, -(-(p + accepted[b] + 1) // page)):
                at = pages.table[b, i]
                assert np.array_equal(bounds[int(at)].double().cpu().numpy(), pc.page_bounds(got[0][at, :, :min(page, p + accepted[b] + 1 - i * page)]))
        assert new.tolist() == [p + n + 1 for p, n in zip(old, accepted)]
        length.copy_(new)
