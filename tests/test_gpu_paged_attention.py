"""GPU parity of dream_paged_verify_attn and dream_sparse_verify_attn against the definition in 64 bits, all elements.  What nobody sees holds NaN: pages of nobody, rows behind the last, pages
that no node selected, and the shared positions of all sequences of a group but the first."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import paged_cases as pc
from tests import window_cases as wc

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _automatic():
    yield
    dream.dream_set_kv_splits(0)
    dream.dream_set_tile_waves(0)
    dream.dream_set_q_tiles(0)


class Problem:
    def __init__(self, Hq, Hkv, D, T, prefix, page, dtype="bf16", groups=(), tree="rand", given=False, sparse=None, seed=1, scale=0.0, lse=True):
        """groups: (first sequence, sequences, shared positions).  sparse: share of the pages that a node sees."""
        B = len(prefix)
        rng = np.random.default_rng([seed, B, Hq, D, T, page, prefix[0]])
        self.B, self.T, self.prefix, self.dtype, self.scale, self.D = B, T, prefix, dtype, scale, D
        origin, shared = list(range(B)), [0] * B
        for first, n, length in groups:
            for b in range(first, first + n):
                origin[b], shared[b] = first, length
        self.pages = pc.Pages(rng, page, [p + T for p in prefix], [(o, min(s, prefix[b]) // page) for b, (o, s) in enumerate(zip(origin, shared))])
        self.q64 = pc.rounded(rng.standard_normal((B, T, Hq, D)), dtype)
        gain = np.exp(0.5 * rng.standard_normal(D))
        self.k64 = [pc.rounded(rng.standard_normal((Hkv, p + T, D)) * gain, dtype) for p in prefix]
        self.v64 = [pc.rounded(rng.standard_normal((Hkv, p + T, D)) * gain, dtype) for p in prefix]
        k, v = self.pages.pool(Hkv, D), self.pages.pool(Hkv, D)
        for b in range(B):
            s = min(shared[b], prefix[b]) if origin[b] != b else 0
            for pool, rows in ((k, self.k64), (v, self.v64)):
                rows[b][:, :s] = rows[origin[b]][:, :s]
                self.pages.put(pool, b, s, rows[b][:, s:])
        self.parent = [wc.tree(tree, T, rng) for _ in range(B)]
        self.masks = wc.masks_of(self.parent, rng) if given else None
        self.see = []
        picked = []
        for b, p in enumerate(prefix):
            see = np.repeat(wc.visible(self.parent[b], p, 0, 0, None if self.masks is None else self.masks[b])[None], Hkv, 0)
            if sparse is not None:
                n = -(-p // page)
                x = rng.random((Hkv, T, n)) < sparse
                picked.append(pc.words(x, self.pages.max_pages))
                see[:, :, :p] &= np.repeat(x, page, -1)[:, :, :p]
                for h in range(Hkv):      # pages that nobody sees
                    for i in np.flatnonzero(~x[h].any(0)):
                        at = self.pages.table[b, i]
                        keep = max(0, min(page, p + T - i * page)) if (i + 1) * page > p else 0      # (the tree's rows in the last one)
                        lo = p - i * page if keep else page
                        k[at, h, :lo] = v[at, h, :lo] = np.nan
            self.see.append(see)
        self.k, self.v = pc.device(k, dtype), pc.device(v, dtype)
        self.q = pc.device(self.q64, dtype)
        self.nodes = torch.from_numpy(np.stack(picked)).cuda() if picked else None
        self.mask = torch.from_numpy(self.masks.view(np.int64)).cuda() if given else None
        self.desc = dream.attn_desc(B, Hq, Hkv, D, dream.BF16 if dtype == "bf16" else dream.F32, 0, scale)
        self.pd = dream.page_desc(page, self.pages.n_pages, self.pages.max_pages)
        self.table, self.len, self.par = self.pages.device_table(), wc.ints(prefix), wc.ints(self.parent)
        self.groups = (len(groups), wc.ints([g[0] for g in groups] + [groups[-1][0] + groups[-1][1]]) if groups else None, wc.ints([g[2] for g in groups]) if groups else None,
                       max([g[2] for g in groups], default=0))
        self.max_kv = max(prefix) + T
        self.out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device="cuda")
        self.lse = torch.full((B, Hq, T), 7.0, device="cuda") if lse else None

    def workspace(self):
        if self.nodes is not None:
            n = dream.dream_sparse_verify_attn_workspace(self.desc, self.pd, self.T, self.max_kv, 0)
        else:
            n = dream.dream_paged_verify_attn_workspace(self.desc, self.pd, self.T, self.max_kv, self.groups[0], self.groups[3])
        return dream.alloc_workspace(n).fill_(0xFF)

    def call(self, ws=None, stream=None):
        ws = self.workspace() if ws is None else ws
        if self.nodes is not None:
            dream.dream_sparse_verify_attn(self.desc, self.pd, self.q, self.k, self.v, self.table, self.nodes, self.len, self.T, self.par, self.mask, self.max_kv, 0, self.out,
                                           self.lse, ws, stream=stream)
        else:
            dream.dream_paged_verify_attn(self.desc, self.pd, self.q, self.k, self.v, self.table, self.len, self.T, self.par, self.mask, *self.groups, self.max_kv, self.out,
                                          self.lse, ws, stream=stream)
        return ws

    def check(self):
        torch.cuda.synchronize()
        got, lse = self.out.double().cpu().numpy(), None if self.lse is None else self.lse.double().cpu().numpy()
        for b in range(self.B):
            want = pc.attend(self.q64[b], self.k64[b], self.v64[b], self.see[b], self.scale or None)
            pc.check_rows(got[b], None if lse is None else lse[b], *want, self.prefix[b] + self.T, self.D, self.dtype)


# Hq, Hkv, D, T, prefixes, page, more
DENSE = [
    (4, 4, 64, 1, [0], 16, {}),
    (2, 1, 128, 1, [1], 32, {}),
    (4, 2, 256, 1, [15, 16, 17], 16, {}),
    (4, 2, 64, 7, [31, 32, 33], 32, {}),
    (4, 2, 128, 9, [31, 0, 97], 64, {}),
    (2, 2, 256, 17, [64, 129], 128, {}),
    (7, 1, 64, 13, [200, 17], 256, {}),
    (8, 1, 128, 60, [300, 45], 16, {}),
    (4, 2, 256, 33, [700], 64, {}),
    (4, 4, 128, 33, [100, 3], 32, dict(tree="chain")),
    (2, 2, 64, 64, [100, 5], 64, dict(tree="star")),
    (2, 2, 64, 65, [90], 16, {}),
    (2, 1, 128, 256, [37], 64, dict(tree="chain")),
    (4, 1, 256, 100, [65], 32, dict(given=True)),
    (4, 2, 64, 21, [0, 40], 16, dict(given=True)),          # a mask may leave a node nothing at all
    (16, 1, 128, 1, [260, 1], 64, {}),
    (3, 1, 128, 1, [5003], 16, {}),                         # keys shared by many workgroups
    (2, 2, 64, 5, [4000, 0], 128, {}),
    (2, 1, 256, 3, [2100, 7], 64, {}),
    (8, 8, 64, 4, [60, 1, 33, 64, 31, 95, 0, 12, 128], 16, {}),
    (4, 2, 128, 5, [9000], 16, {}),                         # more pages than a workgroup lists at a time
    (4, 2, 64, 9, [50, 200], 64, dict(scale=-0.3)),
    (4, 2, 64, 11, [70, 3], 16, dict(dtype="f32")),
    (4, 1, 128, 1, [300, 0], 64, dict(dtype="f32")),
    (2, 2, 256, 70, [40], 32, dict(dtype="f32", given=True)),
    (4, 4, 64, 60, [61, 700], 64, dict(lse=False)),
]
SHARED = [
    (4, 2, 64, 1, [40, 33, 35], 16, dict(groups=[(0, 3, 32)])),
    (8, 2, 128, 7, [100, 130, 65, 77], 32, dict(groups=[(0, 4, 64)])),
    (4, 2, 128, 5, [70, 64, 90, 200, 190], 64, dict(groups=[(0, 3, 63), (3, 2, 129)])),      # inside pages
    (2, 1, 256, 12, [300, 280, 10], 128, dict(groups=[(0, 2, 257), (2, 1, 5)])),
    (4, 4, 64, 33, [90, 95, 91, 92, 93], 16, dict(groups=[(0, 1, 80), (1, 4, 90)])),
    (8, 1, 128, 60, [600, 610, 605], 64, dict(groups=[(0, 3, 600)])),
    (4, 1, 64, 1, [2000] * 9, 16, dict(groups=[(0, 9, 2000)])),                              # nothing of their own but the node
    (4, 2, 128, 3, [50, 20, 0], 16, dict(groups=[(0, 3, 48)])),                              # prefixes that end inside the shared part
    (4, 2, 64, 6, [50, 60], 16, dict(groups=[(0, 2, 0)])),                                   # nothing shared
    (2, 2, 256, 3, [700] * 12, 64, dict(groups=[(0, 12, 640)])),
    (4, 2, 64, 4, [100 + i for i in range(70)], 16, dict(groups=[(i, 1, 40 + i) for i in range(70)])),      # more groups than lanes
    (4, 2, 64, 21, [140, 133], 32, dict(groups=[(0, 2, 128)], given=True)),
    (4, 2, 128, 90, [140, 333], 32, dict(groups=[(0, 2, 128)])),
    (4, 2, 64, 9, [70, 71, 64], 16, dict(dtype="f32", groups=[(0, 3, 50)])),
    (4, 2, 64, 5, [50, 70, 64, 90], 16, dict(groups=[(2, 2, 48)])),                          # sequences in front of the first group
    (4, 2, 128, 40, [50, 70, 64], 16, dict(groups=[(1, 2, 48)])),
    (4, 2, 64, 5, [50, 70, 64, 90], 16, dict(groups=[(1, 2, 48)])),                          # and behind the last
    (4, 2, 64, 5, [50, 70, 64], 16, dict(groups=[(2, 1, 48)], dtype="f32")),
    (4, 2, 128, 9, [70, 71, 64], 64, dict(groups=[(0, 3, 50)], scale=-0.2)),
]
SPARSE = [
    (4, 4, 64, 1, [0], 16, dict(sparse=0.5)),
    (4, 2, 128, 1, [700, 33], 16, dict(sparse=0.2)),
    (2, 1, 256, 1, [900], 64, dict(sparse=0.3)),
    (4, 2, 64, 13, [200, 64, 65], 16, dict(sparse=0.1)),
    (8, 1, 128, 60, [500, 0], 32, dict(sparse=0.15)),
    (2, 2, 256, 33, [700], 128, dict(sparse=0.4)),
    (2, 2, 64, 64, [1000, 5], 64, dict(sparse=0.3)),
    (4, 1, 128, 100, [300], 16, dict(sparse=0.02)),
    (2, 1, 64, 256, [500], 64, dict(sparse=0.01)),
    (4, 2, 128, 5, [17000], 16, dict(sparse=0.05)),           # more pages than are looked at at a time
    (4, 2, 64, 21, [300, 40], 256, dict(sparse=0.5, given=True)),
    (4, 2, 64, 9, [300], 64, dict(sparse=0.0)),               # the tree alone
    (4, 2, 64, 9, [300], 64, dict(sparse=1.0)),
    (4, 2, 64, 9, [300, 31], 32, dict(sparse=0.4, dtype="f32")),
    (4, 2, 256, 70, [300, 31], 32, dict(sparse=0.2, dtype="f32")),
    (4, 2, 128, 9, [300, 31], 32, dict(sparse=0.4, scale=-0.3)),
    (4, 1, 128, 20, [333], 32, dict(sparse=0.3, lse=False)),
]


@pytest.mark.parametrize("case", DENSE, ids=str)
def test_pages(case):
    p = Problem(*case[:6], **case[6])
    p.call()
    p.check()


@pytest.mark.parametrize("case", SHARED, ids=lambda c: str(c)[:60])
def test_shared_prefix(case):
    p = Problem(*case[:6], **case[6])
    p.call()
    p.check()


@pytest.mark.parametrize("case", SPARSE, ids=str)
def test_selected_pages(case):
    p = Problem(*case[:6], **case[6])
    p.call()
    p.check()


@pytest.mark.parametrize("splits", [1, 2, 5, 64])
@pytest.mark.parametrize("case", [DENSE[7], DENSE[8], DENSE[11], DENSE[19], SHARED[1], SHARED[5], SPARSE[1], SPARSE[4], SPARSE[7], DENSE[22], SPARSE[13]], ids=lambda c: str(c)[:50])
def test_every_number_of_splits(case, splits):
    dream.dream_set_kv_splits(splits)
    p = Problem(*case[:6], **case[6])
    p.call()
    p.check()


@pytest.mark.parametrize("rows", [1, 3, 16, 17, 32, 33, 64, 65, 128, 129, 250, 256])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_every_number_of_rows(D, rows):
    """All shapes of workgroups, with and without shared positions and selected pages."""
    for more in ({}, dict(groups=[(0, 2, 48)]), dict(sparse=0.4)):
        p = Problem(1, 1, D, rows, [100, 71], 16, seed=rows, **more)
        p.call()
        p.check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("waves,tiles", [(4, 1), (4, 2), (8, 1), (8, 2)])
def test_every_shape(D, waves, tiles):
    """Whatever the call's sizes would have chosen; one split and several, steps that start and end anywhere."""
    dream.dream_set_tile_waves(waves)
    dream.dream_set_q_tiles(tiles)
    for splits, more in ((1, {}), (3, dict(groups=[(0, 2, 49)])), (2, dict(sparse=0.4)), (1, dict(sparse=0.1))):
        dream.dream_set_kv_splits(splits)
        for T, prefix, page in ((1, [333, 0], 16), (20, [100, 71], 32), (35, [1030, 65], 64), (130, [300, 49], 16)):
            p = Problem(4, 2, D, T, prefix, page, seed=T, **more)
            p.call()
            p.check()


@pytest.mark.parametrize("case", [DENSE[7], DENSE[16], SHARED[1], SHARED[5], SPARSE[4], SPARSE[9]], ids=lambda c: str(c)[:50])
@pytest.mark.parametrize("wrong", [1, 10 ** 12])
def test_lengths_that_are_hints_only_choose_the_launch(case, wrong):
    p = Problem(*case[:6], **case[6])
    p.max_kv = max(wrong, p.T)
    p.groups = p.groups[:3] + (wrong,)
    p.call()
    p.check()


@pytest.mark.parametrize("case", [DENSE[16], DENSE[17], DENSE[23], SHARED[1], SHARED[5], SPARSE[1], SPARSE[4]], ids=lambda c: str(c)[:50])
def test_workspaces_of_other_calls_hold_fewer_parts(case):
    """Any size from that of the fewest parts on; nothing behind it is written."""
    p = Problem(*case[:6], **case[6])
    slot = p.B * case[0] * p.T * (p.D + 2) * 4
    parts = 1 + (p.groups[0] > 0)
    for size in (256 if parts == 1 else parts * slot, parts * slot + 4, (parts + 1) * slot + 36, 5 * slot + 4):
        ws = dream.alloc_workspace(size + 4096).fill_(0x55)
        p.out.fill_(7.0)
        p.call(ws[:size])
        p.check()
        assert bool((ws[size:] == 0x55).all())


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("case", [(4, 2, 64, 9, [70, 40], 16, {}), (8, 1, 128, 60, [200], 64, {}), (2, 2, 256, 33, [100], 32, {}), (4, 2, 128, 7, [100, 90], 32, dict(groups=[(0, 2, 64)])),
                                  (8, 1, 128, 20, [300], 32, dict(sparse=0.3)), (4, 2, 64, 9, [70, 40], 16, dict(dtype="f32"))], ids=lambda c: str(c)[:50])
def test_values_that_are_not_finite_where_only_some_nodes_see(case, value):
    """Rows of nodes that do not see it are as ever; rows that see it in V have that channel NaN or infinite and the others as ever; rows that see it in K are NaN (or, with a score of
    -inf, without that key)."""
    for which in "kv":
        p = Problem(*case[:6], tree="star", **case[6])
        b, h = 0, p.k64[0].shape[0] - 1
        node = p.T - 1                           # seen by itself alone
        j = p.prefix[b] + node
        if p.nodes is not None:                  # and a prefix row that some nodes' selection has
            some = [j for j in range(p.prefix[b]) if 0 < p.see[b][h, :, j].sum() < p.T]
            j = some[len(some) // 2]
        rows64, pool = (p.k64, p.k) if which == "k" else (p.v64, p.v)
        rows64[b][h, j, 5] = value
        page, at = p.pages.where(b, j)
        pool[int(page), h, at, 5] = value
        p.call()
        torch.cuda.synchronize()
        got = p.out.double().cpu().numpy()
        G = got.shape[2] // p.k64[0].shape[0]
        clean_k, clean_v = p.k64[b].copy(), p.v64[b].copy()
        (clean_k if which == "k" else clean_v)[h, j, 5] = 0.0
        seen = np.repeat(p.see[b][:, :, j], G, 0).T.copy()      # [T, Hq]
        seen[:, np.arange(got.shape[2]) // G != h] = False
        want, lse, mass, size = pc.attend(p.q64[b], clean_k, clean_v, p.see[b])
        row, _ = wc.attention_bounds(want[None], mass[None], size[None], j + p.T, p.D, p.dtype == "bf16")
        err = np.abs(got[b] - want)
        assert (err[~seen] <= row[0][~seen]).all()
        if which == "v":
            assert not np.isfinite(got[b][seen][:, 5]).any()
            if not np.isnan(value):
                assert (np.isnan(got[b][seen][:, 5]) | (got[b][seen][:, 5] == value)).all()
            other = np.arange(p.D) != 5
            assert (err[seen][:, other] <= row[0][seen][:, other]).all()
        else:
            for i, head in zip(*np.nonzero(seen)):
                if not np.isnan(value) and p.q64[b, i, head, 5] * value < 0:
                    see = p.see[b].copy()
                    see[h, i, j] = False
                    w2, _, m2, s2 = pc.attend(p.q64[b][i:i + 1], clean_k, clean_v, see[:, i:i + 1])
                    r2, _ = wc.attention_bounds(w2[None], m2[None], s2[None], j + p.T, p.D, p.dtype == "bf16")
                    assert (np.abs(got[b, i, head] - w2[0, head]) <= r2[0, 0, head]).all()
                else:
                    assert np.isnan(got[b, i, head]).all()


@pytest.mark.parametrize("more", [{}, dict(sparse=0.5)])
def test_tables_that_point_nowhere_are_not_followed(more):
    """Entries behind the live pages, negative and huge: the results do not depend on them."""
    for behind in (-1, -2 ** 31, 2 ** 31 - 1):
        p = Problem(4, 2, 128, 5, [100, 64], 64, **more)
        t = p.pages.table.copy()
        live = [-(-(x + p.T) // 64) for x in p.prefix]
        for b, n in enumerate(live):
            t[b, n:] = behind
        p.table = wc.ints(t)
        p.call()
        p.check()


def test_prefix_lengths_outside_the_table_are_clamped():
    """Results for such lengths are unspecified; the call must end, and the other sequences' rows be right."""
    p = Problem(4, 2, 64, 5, [100, 64, 30], 16, groups=[(0, 1, 0), (1, 2, 20)])
    p.len = wc.ints([2 ** 31 - 1, 64, -5])
    p.call()
    torch.cuda.synchronize()
    got = p.out.double().cpu().numpy()
    want = pc.attend(p.q64[1], p.k64[1], p.v64[1], p.see[1])
    pc.check_rows(got[1], None, *want, 70, 64, "bf16")


@pytest.mark.parametrize("case", [DENSE[7], SHARED[2], SPARSE[4]], ids=lambda c: str(c)[:50])
def test_captured_and_replayed(case):
    p = Problem(*case[:6], **case[6])
    ws = p.call()
    p.check()
    first = p.out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.call(ws)
    for _ in range(4):
        p.out.fill_(7.0)
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.out, first)


def test_two_streams_with_a_workspace_each():
    """The same bits on any stream, beside other calls."""
    case = SHARED[5]
    p = Problem(*case[:6], **case[6])
    p.call()
    torch.cuda.synchronize()
    want = p.out.clone()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs, spaces = [torch.empty_like(p.out) for _ in streams], [p.workspace() for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, ws in zip(streams, outs, spaces):
            p.out = o
            p.call(ws, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


def test_a_pool_behind_4_gib():
    """Pages whose addresses need more than 32 bits."""
    D, Hkv, page, n = 128, 8, 64, 36000
    pool = torch.zeros(n, Hkv, page, D, dtype=torch.bfloat16, device="cuda")      # 4.7 GB
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    ids = [n - 1, 5, n - 2, 34000, 33333]
    P, T = 4 * page + 20, 3
    for i in ids:
        pool[i].normal_(generator=gen)
    table = wc.ints([ids + [-1]])
    q = torch.randn(1, T, 32, D, generator=gen, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    desc, pd = dream.attn_desc(1, 32, Hkv, D, dream.BF16, 0), dream.page_desc(page, n, 6)
    par = [-1, 0, 1]
    ws = dream.alloc_workspace(dream.dream_paged_verify_attn_workspace(desc, pd, T, P + T))
    dream.dream_paged_verify_attn(desc, pd, q, pool, pool, table, wc.ints([P]), T, wc.ints([par]), None, 0, None, None, 0, P + T, out, None, ws)
    torch.cuda.synchronize()
    rows = pool[ids].double().cpu().numpy().transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :P + T]
    see = np.repeat(wc.visible(par, P, 0, 0)[None], Hkv, 0)
    pc.check_rows(out[0].double().cpu().numpy(), None, *pc.attend(q[0].double().cpu().numpy(), rows, rows, see), P + T, D, "bf16")
