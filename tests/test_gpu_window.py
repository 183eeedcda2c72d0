"""GPU parity of dream_window_verify_attn and dream_mx_verify_attn against the definition in 64 bits, all elements."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import window_cases as wc

pytestmark = pytest.mark.gpu

# B, Hq, Hkv, D, tree kind, T, prefixes, window, sink, masks given
CASES = [
    (1, 4, 4, 64, "rand", 1, [0], 0, 0, False),
    (1, 4, 4, 64, "rand", 1, [0], 5, 2, False),
    (1, 2, 1, 128, "rand", 1, [1], 1, 0, False),
    (3, 4, 2, 64, "rand", 7, [31, 32, 33], 0, 0, False),
    (3, 4, 2, 128, "rand", 9, [31, 0, 97], 40, 3, False),
    (2, 2, 2, 256, "rand", 17, [64, 129], 33, 0, False),
    (2, 7, 1, 64, "rand", 13, [200, 17], 64, 70, False),
    (2, 8, 1, 128, "rand", 60, [300, 45], 100, 4, False),
    (1, 4, 2, 256, "rand", 33, [700], 129, 37, False),
    (2, 4, 4, 64, "chain", 12, [50, 3], 5, 0, False),          # the window ends inside the tree
    (2, 4, 4, 128, "chain", 12, [0, 2], 3, 4, False),          # first tokens inside the tree
    (2, 2, 2, 128, "chain", 20, [40, 60], 1, 0, False),        # a node sees itself only
    (2, 2, 2, 64, "star", 64, [100, 5], 32, 1, False),
    (1, 2, 2, 64, "rand", 65, [90], 50, 0, False),
    (1, 2, 1, 128, "chain", 256, [37], 0, 0, False),
    (1, 2, 1, 64, "chain", 256, [300], 130, 33, False),
    (1, 2, 2, 256, "rand", 100, [65], 0, 0, True),
    (2, 4, 2, 64, "rand", 21, [0, 40], 0, 0, True),            # a mask may leave a node nothing at all
    (2, 4, 2, 128, "rand", 21, [0, 40], 6, 0, True),
    (2, 4, 2, 64, "rand", 130, [0, 70], 50, 2, True),
    (1, 2, 1, 64, "rand", 3, [5003], 0, 0, False),             # keys shared by many workgroups
    (1, 4, 1, 128, "rand", 20, [3000], 0, 0, False),
    (2, 2, 1, 256, "rand", 5, [2100, 7], 0, 0, False),
    (1, 2, 1, 64, "rand", 5, [4000], 1500, 300, False),
    (9, 32, 32, 64, "rand", 4, [60, 1, 33, 64, 31, 95, 0, 12, 128], 30, 2, False),      # more workgroups than CUs
]


def _pair(rng, shape, kind):
    """Cache rows as the call takes them, and what they stand for.  Some dimensions are larger than others."""
    x = rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[-1]))
    if kind == "mx":
        code, byte, _ = wc.quantise(wc.bf16(x))
        return (torch.from_numpy(wc.pack(code)).cuda(), torch.from_numpy(byte).cuda()), wc.decode(wc.pack(code), byte)
    if kind == "bf16":
        x = wc.bf16(x)
        return (torch.from_numpy(x).to(torch.bfloat16).cuda(),), x
    x = x.astype(np.float32)
    return (torch.from_numpy(x).cuda(),), x.astype(np.float64)


class _Problem:
    def __init__(self, case, kind, dtype="bf16", seed=7, scale=0.0, slack=37):
        B, Hq, Hkv, D, tree, T, self.prefix, self.window, self.sink, given = case
        rng = np.random.default_rng([seed, B, Hq, D, T, self.prefix[0]])
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.shape, self.D = (B, T, Hq, D), D
        self.rows = max(self.prefix) + T + slack
        q = rng.standard_normal(self.shape)
        self.q64 = wc.bf16(q) if dtype == "bf16" else q.astype(np.float32).astype(np.float64)
        self.q = torch.from_numpy(self.q64).to(self.dt).cuda()
        self.k, self.k64 = _pair(rng, (B, Hkv, self.rows, D), kind)
        self.v, self.v64 = _pair(rng, (B, Hkv, self.rows, D), kind)
        self.parent = [wc.tree(tree, T, rng) for _ in range(B)]
        self.masks = wc.masks_of(self.parent, rng) if given else None
        self.mask = torch.from_numpy(self.masks.view(np.int64)).cuda() if given else None
        self.kind, self.scale, self.T = kind, scale, T
        self.desc = dream.attn_desc(B, Hq, Hkv, D, dream.BF16 if dtype == "bf16" else dream.F32, self.rows, scale)
        self.max_kv = max(self.prefix) + T
        self.out = torch.full(self.shape, float("nan"), dtype=self.dt, device="cuda")
        self.lse = torch.full((B, Hq, T), float("nan"), device="cuda")
        self.len, self.par = wc.ints(self.prefix), wc.ints(self.parent)
        size = dream.dream_mx_verify_attn_workspace if kind == "mx" else dream.dream_window_verify_attn_workspace
        self.ws = dream.alloc_workspace(size(self.desc, T, self.max_kv, self.window, self.sink)).fill_(0xFF)

    def call(self, stream=None):
        f = dream.dream_mx_verify_attn if self.kind == "mx" else dream.dream_window_verify_attn
        f(self.desc, self.q, *self.k, *self.v, self.len, self.T, self.par, self.mask, self.window, self.sink, self.max_kv, self.out, self.lse, self.ws,
          stream=stream)

    def want(self):
        return wc.attention(self.q64, self.k64, self.v64, self.prefix, self.parent, self.window, self.sink, self.masks, self.scale or None)

    def check(self):
        torch.cuda.synchronize()
        out, lse, mass, size = self.want()
        row, ls = wc.attention_bounds(out, mass, size, self.max_kv, self.D, self.dt == torch.bfloat16)
        got, got_lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - out) <= row).all(), float((np.abs(got - out) / row).max())
        some = np.isfinite(lse)
        assert (np.isneginf(got_lse) == ~some).all()
        assert (np.abs(got_lse[some] - lse[some]) <= ls[some] + np.abs(lse[some]) * 2.0 ** -23).all()


@pytest.mark.parametrize("kind", ["bf16", "mx"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-w{c[7]}-s{c[8]}")
def test_rows_and_log_sum_exps(case, kind):
    p = _Problem(case, kind)
    p.call()
    p.check()


@pytest.mark.parametrize("kind", ["f32", "mx"])
@pytest.mark.parametrize("case", [CASES[i] for i in (0, 1, 3, 4, 5, 9, 10, 15, 17, 18, 19)], ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-w{c[7]}")
def test_float32(case, kind):
    p = _Problem(case, kind, dtype="f32")
    p.call()
    p.check()


@pytest.mark.parametrize("kind", ["bf16", "mx"])
@pytest.mark.parametrize("scale", [0.03, -0.11, 1.0])
def test_given_scale(kind, scale):
    p = _Problem((2, 4, 2, 64, "rand", 18, [100, 40], 60, 2, False), kind, scale=scale)
    p.call()
    p.check()


@pytest.mark.parametrize("kind", ["bf16", "mx"])
def test_a_cache_full_to_its_last_row(kind):
    p = _Problem((2, 2, 2, 128, "rand", 5, [58, 20], 0, 0, False), kind, slack=0)
    p.call()
    p.check()


def _poison(p, b, rows, what):
    """NaN or infinities in rows of a sequence, K and V."""
    for cache in (p.k, p.v):
        if p.kind == "mx":
            cache[1][b, :, rows] = 255
        else:
            cache[0][b, :, rows] = what


@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("mx", "bf16"), ("f32", "f32"), ("mx", "f32")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_what_no_row_sees_changes_nothing(kind, dtype, D, what):
    """Rows behind the live ones, and rows between the first tokens and the root's window, hold NaN."""
    p = _Problem((2, 4, 2, D, "rand", 9, [150, 70], 41, 3, False), kind, dtype=dtype)
    for b, P in enumerate(p.prefix):
        _poison(p, b, slice(P + p.T, None), what)
        _poison(p, b, slice(3, P - 41 + 1), what)
    p.call()
    p.check()


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("mx", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("D", [64, 256])
def test_what_one_row_does_not_see_does_not_reach_it(kind, dtype, D, what):
    """A star's leaves do not see each other, and only the root sees the first row of its window: a node whose own row or window holds NaN has NaN, the others are
    as they were."""
    p = _Problem((1, 2, 1, D, "star", 12, [80], 30, 0, False), kind, dtype=dtype)
    out, lse, mass, size = p.want()
    row, _ = wc.attention_bounds(out, mass, size, p.max_kv, D, dtype == "bf16")
    _poison(p, 0, slice(80 + 5, 80 + 6), what)            # node 5's row
    _poison(p, 0, slice(80 - 29, 80 - 28), what)          # the first row of the root's window
    p.call()
    torch.cuda.synchronize()
    got = p.out.double().cpu().numpy()
    for i in range(12):
        if i in (0, 5):
            assert not np.isfinite(got[0, i]).any()
        else:
            assert (np.abs(got[0, i] - out[0, i]) <= row[0, i]).all(), i


def test_one_value_that_is_not_finite_stays_in_its_channel():
    """V only: the channel of the nodes that see it, in a tile that others see as well and in one that all see."""
    p = _Problem((1, 2, 1, 128, "star", 6, [70], 0, 0, False), "bf16")
    out, lse, mass, size = p.want()
    row, _ = wc.attention_bounds(out, mass, size, p.max_kv, 128, True)
    p.v[0][0, 0, 70 + 3, 17] = float("nan")
    p.v[0][0, 0, 9, 40] = float("nan")
    p.call()
    torch.cuda.synchronize()
    got = p.out.double().cpu().numpy()
    bad = np.zeros(got.shape, dtype=bool)
    bad[0, 3, :, 17] = True
    bad[..., 40] = True
    assert np.isnan(got[bad]).all()
    assert (np.abs(got - out)[~bad] <= row[~bad]).all()


@pytest.mark.parametrize("kind", ["bf16", "mx"])
def test_the_same_bits_every_time_and_under_capture(kind):
    """Two captured calls that share a workspace, replayed with eager work between the replays."""
    cases = [(1, 4, 1, 128, "rand", 20, [3000], 0, 0, False), (2, 4, 2, 64, "rand", 9, [1500, 700], 900, 4, False)]
    ps = [_Problem(c, kind) for c in cases]
    shared = max((p.ws for p in ps), key=lambda t: t.numel())
    first = []
    for p in ps:
        p.ws = shared
        p.call()
        torch.cuda.synchronize()
        p.check()
        first.append((p.out.clone(), p.lse.clone()))
    stream = torch.cuda.Stream()
    graphs = []
    for p in ps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            p.call()
        graphs.append(g)
    for _ in range(3):
        for p, g, (out, lse) in zip(ps, graphs, first):
            p.out.fill_(3.0)
            p.lse.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(p.out, out) and torch.equal(p.lse, lse)
            p.call()
            torch.cuda.synchronize()
            assert torch.equal(p.out, out)


def test_another_stream():
    p = _Problem(CASES[8], "mx")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    p.call(stream=s)
    s.synchronize()
    p.check()


def test_no_window_is_the_framework_s_other_call():
    """Without a window the 16-bit call answers as dream_tree_verify_attn does, within both calls' rounding."""
    p = _Problem((2, 8, 2, 128, "rand", 33, [300, 211], 0, 0, False), "bf16")
    p.call()
    out, lse = torch.empty_like(p.out), torch.empty_like(p.lse)
    ws = dream.alloc_workspace(dream.dream_tree_verify_attn_workspace(p.desc, p.T, p.max_kv))
    dream.dream_tree_verify_attn(p.desc, p.q, p.k[0], p.v[0], p.len, p.T, p.par, None, p.max_kv, out, lse, ws)
    p.check()
    o, l, mass, size = p.want()
    row, ls = wc.attention_bounds(o, mass, size, p.max_kv, 128, True)
    assert (np.abs((out.double() - p.out.double()).cpu().numpy()) <= 2 * row).all()


def test_a_cache_beyond_32_bits():
    """The last head of the last sequence lies more than 4 GB into the codes and more than 2^32 values into the cache."""
    B, H, D, rows = 2, 8, 256, (1 << 21) + 64
    desc = dream.attn_desc(B, H, H, D, dream.BF16, rows)
    codes = torch.zeros(B, H, rows, D // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((B, H, rows, D // 32), 127, dtype=torch.uint8, device="cuda")
    P, T = rows - 3, 3
    rng = np.random.default_rng(3)
    k, v = (wc.bf16(rng.standard_normal((B, 40, H, D))) for _ in range(2))
    vc, vs = codes.clone(), scales.clone()
    base = wc.ints([rows - 40] * B)
    dream.dream_mx_append(desc, torch.from_numpy(k).bfloat16().cuda(), torch.from_numpy(v).bfloat16().cuda(), 40, base, None, codes, scales, vc, vs)
    q = wc.bf16(rng.standard_normal((B, T, H, D)))
    out = torch.empty(B, T, H, D, dtype=torch.bfloat16, device="cuda")
    parent = [[-1, 0, 1]] * B
    ws = dream.alloc_workspace(dream.dream_mx_verify_attn_workspace(desc, T, rows, 20, 0))
    dream.dream_mx_verify_attn(desc, torch.from_numpy(q).bfloat16().cuda(), codes, scales, vc, vs, wc.ints([P] * B), T, wc.ints(parent), None, 20, 0, rows, out,
                               None, ws)
    torch.cuda.synchronize()
    small = []
    for x in (k, v):
        code, byte, _ = wc.quantise(x.transpose(0, 2, 1, 3))
        small.append(wc.decode(wc.pack(code), byte))
    want, _, mass, size = wc.attention(q, small[0], small[1], [37] * B, parent, 20, 0)
    row, _ = wc.attention_bounds(want, mass, size, 40, D, True)
    assert (np.abs(out.double().cpu().numpy() - want) <= row).all()


def test_tensors_of_other_types_and_sizes_are_refused():
    """Before anything is launched: every tensor of the calls too short by one value, and of another type."""
    for kind in ("bf16", "mx"):
        p = _Problem(CASES[17], kind)
        names = ["q", "len", "par", "mask", "out", "lse"]
        for name in names + [(c, i) for c in ("k", "v") for i in range(len(p.k))]:
            if isinstance(name, tuple):
                held = getattr(p, name[0])
                t = held[name[1]]
                put = lambda x: setattr(p, name[0], tuple(x if i == name[1] else y for i, y in enumerate(held)))  # noqa: E731
            else:
                t = getattr(p, name)
                put = lambda x: setattr(p, name, x)  # noqa: E731
            for bad in (t.flatten()[:-1].clone(), torch.zeros(t.shape, dtype=torch.float16, device="cuda")):
                put(bad)
                with pytest.raises(ValueError, match="expected"):
                    p.call()
            put(t)
        p.call()
        p.check()
    desc = dream.attn_desc(1, 2, 2, 64, dream.BF16, 10)
    x, f, c, s = torch.zeros(3, 2, 64, device="cuda").bfloat16(), torch.zeros(32, device="cuda"), torch.zeros(2, 10, 32, device="cuda").byte(), torch.zeros(2, 10, 2, device="cuda").byte()
    at, out = wc.ints([0]), torch.zeros(2, 2, 3, 64, device="cuda").bfloat16()
    for args in (([(x[:2], 2, None, None, x)], 3, None, at, None, f, 64), ([(x, 2, None, None, x[:2])], 3, None, at, None, f, 64),
                 ([(x, 2, at, None, x)], 3, None, at, None, f, 64), ([(x, 2, None, None, x)], 3, None, at, None, f[:31], 64),
                 ([(x, 2, None, None, x)], 3, None, at.float(), None, f, 64), ([(x, 2, None, None, x)], 3, at, None, None, f, 64),
                 ([(x.float(), 2, None, None, x)], 3, None, at, None, f, 64)):
        with pytest.raises(ValueError, match="expected"):
            dream.dream_rotary_rows(desc, *args)
    for args in ((x[:2], x, 3, at, None, c, s, c, s), (x, x, 3, at, at, c, s, c, s), (x, x, 3, at, None, c[:1], s, c, s), (x, x, 3, at, None, c, s, c, s.int())):
        with pytest.raises(ValueError, match="expected"):
            dream.dream_mx_append(desc, *args)
    for args in (([c], [s[:1]], at, 3, out), ([c, c], [s, s], at, 4, out), ([c], [s], at.long(), 3, out)):
        with pytest.raises(ValueError, match="expected"):
            dream.dream_mx_read(desc, *args)
    path = wc.ints([[0, -1]])
    for args in (([c[:1]], [s], at, 3, path, at), ([c], [s], at, 3, path.float(), at), ([c], [s], at.float(), 3, path, at), ([c], [s], at, 3, path, at, at.long())):
        with pytest.raises(ValueError, match="expected"):
            dream.dream_mx_commit(desc, *args)
