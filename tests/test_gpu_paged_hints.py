"""dream_sparse_verify_attn where more pages are seen than max_pages_seen and max_kv_len say: they choose the launch, not the result, and a workgroup then goes through several lists of pages."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import paged_cases as pc
from tests import window_cases as wc
from tests.test_gpu_paged_attention import Problem, _automatic      # noqa: F401

pytestmark = pytest.mark.gpu


class Hinted(Problem):
    """The call with a hint of so many pages."""
    seen = 0

    def workspace(self, behind=0):
        n = dream.dream_sparse_verify_attn_workspace(self.desc, self.pd, self.T, self.max_kv, self.seen)
        return dream.alloc_workspace(n + behind).fill_(0xFF)

    def call(self, ws=None, stream=None):
        behind = 4096 if ws is None else 0
        ws = self.workspace(behind) if ws is None else ws
        part = ws[:ws.numel() - behind]
        dream.dream_sparse_verify_attn(self.desc, self.pd, self.q, self.k, self.v, self.table, self.nodes, self.len, self.T, self.par, self.mask, self.max_kv, self.seen, self.out, self.lse,
                                       part, stream=stream)
        if behind:
            torch.cuda.synchronize()
            assert bool((ws[ws.numel() - behind:] == 0xFF).all())
        return ws


def most_pages(p):
    """The most that a node sees."""
    return max(int((w >> np.uint64(i) & np.uint64(1)).sum()) for b in range(p.B) for h in p.nodes[b].cpu().numpy().view(np.uint64) for w in h.T for i in range(64))


# Hq, Hkv, D, T, prefixes, page, more: some of them more than 64 pages for a workgroup and part, some more than 128
CASES = [
    (4, 2, 64, 1, [3000, 33], 16, dict(sparse=0.6)),
    (4, 2, 128, 1, [4000], 16, dict(sparse=0.9)),
    (2, 1, 256, 1, [2500, 1600], 16, dict(sparse=0.7)),
    (4, 2, 64, 13, [2100, 1100], 16, dict(sparse=0.2)),
    (8, 1, 128, 20, [2900, 0], 32, dict(sparse=0.3)),
    (2, 2, 256, 33, [1700], 16, dict(sparse=0.2)),
    (4, 1, 128, 100, [2300], 16, dict(sparse=0.1)),
    (2, 1, 64, 129, [2300, 70], 16, dict(sparse=0.05)),
    (4, 2, 64, 9, [2500], 32, dict(sparse=0.9, lse=False)),
    (4, 2, 128, 9, [2300], 16, dict(sparse=0.5, scale=-0.3)),
    (4, 2, 64, 3, [2300, 90], 16, dict(sparse=0.5, dtype="f32")),
    (4, 2, 64, 21, [2300], 16, dict(sparse=0.3, given=True)),
]


@pytest.mark.parametrize("hint", ["one", "one too few", "right"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:50])
def test_more_pages_than_were_said(case, hint):
    p = Hinted(*case[:6], **case[6])
    p.seen = {"one": 1, "one too few": most_pages(p) - 1, "right": most_pages(p)}[hint]
    p.call()
    p.check()


@pytest.mark.parametrize("case", CASES[:1] + CASES[4:6] + CASES[7:8], ids=lambda c: str(c)[:50])
def test_longer_than_was_said(case):
    p = Hinted(*case[:6], **case[6])
    p.max_kv = p.T
    p.call()
    p.check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("waves,tiles", [(4, 1), (4, 2), (8, 1), (8, 2)])
@pytest.mark.parametrize("splits", [1, 2])
def test_every_shape(D, waves, tiles, splits):
    dream.dream_set_tile_waves(waves)
    dream.dream_set_q_tiles(tiles)
    dream.dream_set_kv_splits(splits)
    for T, prefix, page in ((1, [2300, 0], 16), (20, [3100, 71], 16), (70, [2100], 16)):
        p = Hinted(4, 2, D, T, prefix, page, seed=T, sparse=0.8)
        p.seen = 1
        p.call()
        p.check()


@pytest.mark.parametrize("which", "kv")
@pytest.mark.parametrize("at", [5, 1500, 2200])
@pytest.mark.parametrize("case", [(4, 2, 64, 9, [2300], 16, dict(sparse=0.6)), (8, 1, 128, 20, [2300], 16, dict(sparse=0.4)), (2, 2, 256, 33, [2300], 16, dict(sparse=0.4))], ids=lambda c: str(c)[:30])
def test_a_value_that_is_not_finite_in_any_list(case, at, which):
    """Nodes that do not see it are as ever, whichever list it is in; nodes that do have it in their row."""
    p = Hinted(*case[:6], **case[6])
    p.seen = 1
    h = p.k64[0].shape[0] - 1
    j = next(j for j in range(at, p.prefix[0]) if 0 < p.see[0][h, :, j].sum() < p.T)
    page, row = p.pages.where(0, j)
    (p.k if which == "k" else p.v)[int(page), h, row, 5] = np.inf if which == "v" else np.nan
    p.call()
    torch.cuda.synchronize()
    got = p.out[0].double().cpu().numpy()
    G = got.shape[1] // p.k64[0].shape[0]
    seen = np.repeat(p.see[0][:, :, j], G, 0).T.copy()
    seen[:, np.arange(got.shape[1]) // G != h] = False
    want, _, mass, size = pc.attend(p.q64[0], p.k64[0], p.v64[0], p.see[0])
    row, _ = wc.attention_bounds(want[None], mass[None], size[None], p.prefix[0] + p.T, p.D, True)
    err = np.abs(got - want)
    assert (err[~seen] <= row[0][~seen]).all()
    assert not np.isfinite(got[seen][:, 5]).any()


def test_captured_and_replayed():
    p = Hinted(*CASES[4][:6], **CASES[4][6])
    p.seen = 1
    ws = p.call(p.workspace())
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


@pytest.mark.parametrize("T,splits", [(1, 1), (40, 1), (40, 2)])
def test_a_page_more_than_was_said_does_not_change_the_pace(T, splits):
    """A hint of one page instead of 180, by the same shape of workgroups: lists of 64 entries instead of one, not the rows one by one (which take ten times as long and more)."""
    dream.dream_set_kv_splits(splits)
    dream.dream_set_tile_waves(4 if T == 1 else 8)
    B, Hq, Hkv, D, page, n = 4, 32, 8, 128, 16, 400
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    k, v = (torch.empty(B * (n + 4), Hkv, page, D, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    q = torch.empty(B, T, Hq, D, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    table = wc.ints(np.random.default_rng(1).permutation(B * (n + 4)).reshape(B, -1))
    nodes = torch.zeros(B, Hkv, n + 4, 1, dtype=torch.int64, device="cuda")
    nodes[:, :, 20:200] = (1 << T) - 1
    desc, pd = dream.attn_desc(B, Hq, Hkv, D, dream.BF16, 0), dream.page_desc(page, B * (n + 4), n + 4)
    length, par, out = wc.ints([n * page] * B), wc.ints([[-1] + [0] * (T - 1)] * B), torch.empty_like(q)

    def time_of(seen):
        ws = dream.alloc_workspace(dream.dream_sparse_verify_attn_workspace(desc, pd, T, n * page + T, seen))
        best = float("inf")
        for _ in range(20):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(5):
                dream.dream_sparse_verify_attn(desc, pd, q, k, v, table, nodes, length, T, par, None, n * page + T, seen, out, None, ws)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        return best
    said, less = time_of(180), time_of(1)
    assert less < 3.0 * said, (said, less)


@pytest.mark.parametrize("T,splits", [(1, 2), (1, 0), (9, 2), (70, 2)])
def test_more_pages_than_any_list_holds(T, splits):
    """Without a hint, in the smallest workspace: two parts, several full lists each."""
    dream.dream_set_kv_splits(splits)
    p = Hinted(2, 1, 64, T, [50000 if T == 1 else 30000 if T == 9 else 23000], 16, sparse=0.95, seed=T)
    p.call(p.workspace() if not splits else dream.alloc_workspace(2 * 2 * T * 66 * 4).fill_(0xFF))
    p.check()
