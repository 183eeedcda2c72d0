"""GPU parity of dream_rotary_rows against the definition in 64 bits, all elements."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import window_cases as wc

pytestmark = pytest.mark.gpu


def _rows(rng, shape, dtype):
    x = rng.standard_normal(shape)
    x = wc.bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64)
    return x, torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def _freq(rot, base=10000.0):
    return (base ** (-2.0 * np.arange(rot // 2) / rot)).astype(np.float32)


def _bound(x, want, rot, paired, amplitude, dtype):
    """The turn in float32: the reduced angle to 2^-24 of half a turn (pi), sine and cosine to two steps of 2^-24, the two products and their sum to three more; then the rounding."""
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if paired else (slice(0, rot // 2), slice(rot // 2, rot))
    b = np.zeros(x.shape)
    both = (np.abs(x[..., first]) + np.abs(x[..., second])) * amplitude * 10 * 2.0 ** -24
    b[..., first], b[..., second] = both, both
    return b + np.abs(want) * ((2.0 ** -8 if dtype == "bf16" else 0.0) + 2.0 ** -23)


def _check(got, x, pos, freq, rot, paired, amplitude, dtype):
    want = wc.rotary(x, pos, freq, rot, paired, amplitude)
    err = np.abs(got - want)
    bound = _bound(x, want, rot, paired, amplitude, dtype)
    assert (err <= bound).all(), float((err / np.maximum(bound, 1e-30)).max())
    assert np.array_equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 128), (128, 32), (256, 256), (256, 64), (96, 40), (80, 6), (2, 2), (512, 512), (10, 4)])
def test_layouts(D, rot, paired, dtype):
    rng = np.random.default_rng([D, rot])
    B, R, H = 2, 5, 3
    x, dx = _rows(rng, (B, R, H, D), dtype)
    pos = rng.integers(-50, 5000, (B, R))
    freq = _freq(rot)
    out = torch.full(dx.shape, float("nan"), dtype=dx.dtype, device="cuda")
    desc = dream.attn_desc(B, H, H, D, dream.BF16 if dtype == "bf16" else dream.F32, 1)
    dream.dream_rotary_rows(desc, [(dx, H, None, None, out)], R, wc.ints(pos), None, None, torch.from_numpy(freq).cuda(), rot, paired, 1.25)
    torch.cuda.synchronize()
    _check(out.double().cpu().numpy(), x, pos, freq, rot, paired, 1.25, dtype)


@pytest.mark.parametrize("start", [0, 100000, 2 ** 24 + 1, 2 ** 31 - 1 - 8, -2 ** 31])
def test_far_positions(start):
    rng = np.random.default_rng(1)
    x, dx = _rows(rng, (1, 8, 2, 128), "f32")
    freq = _freq(128)
    out = torch.empty_like(dx)
    desc = dream.attn_desc(1, 2, 2, 128, dream.F32, 1)
    dream.dream_rotary_rows(desc, [(dx, 2, None, None, out)], 8, None, wc.ints([start]), None, torch.from_numpy(freq).cuda(), 128)
    torch.cuda.synchronize()
    _check(out.double().cpu().numpy(), x, start + np.arange(8)[None], freq, 128, False, 1.0, "f32")


@pytest.mark.parametrize("kind,T", [("rand", 1), ("rand", 60), ("chain", 256), ("star", 33)])
def test_queries_and_keys_of_a_tree_in_one_launch(kind, T):
    """Positions are prefix plus depth; queries stay dense, keys go to the cache, the rest of which keeps its content."""
    rng = np.random.default_rng(T)
    B, Hq, Hkv, D, rows = 3, 8, 2, 128, 400
    q, dq = _rows(rng, (B, T, Hq, D), "bf16")
    k, dk = _rows(rng, (B, T, Hkv, D), "bf16")
    parent = [wc.tree(kind, T, rng) for _ in range(B)]
    base = [0, 77, rows - T]
    pos = np.array([[p + len(a) - 1 for a in wc.ancestors(t)] for p, t in zip(base, parent)])
    cache = torch.full((B, Hkv, rows, D), 9.0, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(dq)
    freq = _freq(D)
    desc = dream.attn_desc(B, Hq, Hkv, D, dream.BF16, rows)
    dream.dream_rotary_rows(desc, [(dq, Hq, None, None, out), (dk, Hkv, wc.ints(base), None, cache)], T, None, wc.ints(base), wc.ints(parent),
                            torch.from_numpy(freq).cuda(), D)
    torch.cuda.synchronize()
    _check(out.double().cpu().numpy(), q, pos, freq, D, False, 1.0, "bf16")
    got = cache.double().cpu().numpy()
    _check(np.stack([got[b, :, p:p + T].transpose(1, 0, 2) for b, p in enumerate(base)]), k, pos, freq, D, False, 1.0, "bf16")
    for b, p in enumerate(base):
        got[b, :, p:p + T] = 9.0
    assert (got == 9.0).all()


def test_scattered_and_dropped_rows():
    rng = np.random.default_rng(5)
    B, R, H, D, rows = 2, 6, 4, 64, 20
    k, dk = _rows(rng, (B, R, H, D), "bf16")
    index = np.array([[3, 0, 7, -9, 12, 1], [5, 4, 3, 2, 100, 0]])
    base = [2, 8]
    cache = torch.full((B, H, rows, D), 9.0, dtype=torch.bfloat16, device="cuda")
    freq = _freq(D)
    desc = dream.attn_desc(B, H, H, D, dream.BF16, rows)
    dream.dream_rotary_rows(desc, [(dk, H, wc.ints(base), wc.ints(index), cache)], R, None, wc.ints(base), None, torch.from_numpy(freq).cuda(), D)
    torch.cuda.synchronize()
    want = wc.rotary(k, np.array([[b + r for r in range(R)] for b in base]), freq, D, False)
    bound = _bound(k, want, D, False, 1.0, "bf16")
    got = cache.double().cpu().numpy()
    for b in range(B):
        for r in range(R):
            at = base[b] + index[b, r]
            if 0 <= at < rows:
                assert (np.abs(got[b, :, at] - want[b, r]) <= bound[b, r]).all()
                got[b, :, at] = 9.0
    assert (got == 9.0).all()


@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_in_place_and_back(paired, offset):
    """Turned in place and by the negated positions back: the rows again, within both roundings.  offset: tensors that start inside 16 bytes."""
    rng = np.random.default_rng(9)
    B, R, H, D = 2, 7, 3, 64
    x = torch.from_numpy(rng.standard_normal(B * R * H * D + 8).astype(np.float32)).cuda()[offset:offset + B * R * H * D].view(B, R, H, D)
    start = x.double().cpu().numpy()
    pos = rng.integers(0, 10 ** 6, (B, R))
    freq = torch.from_numpy(_freq(D)).cuda()
    desc = dream.attn_desc(B, H, H, D, dream.F32, 1)
    dream.dream_rotary_rows(desc, [(x, H, None, None, x)], R, wc.ints(pos), None, None, freq, D, paired)
    torch.cuda.synchronize()
    _check(x.double().cpu().numpy(), start, pos, _freq(D), D, paired, 1.0, "f32")
    dream.dream_rotary_rows(desc, [(x, H, None, None, x)], R, wc.ints(-pos), None, None, freq, D, paired)
    torch.cuda.synchronize()
    both = _bound(start, start, D, paired, 1.0, "f32")
    assert (np.abs(x.double().cpu().numpy() - start) <= 4 * both + 1e-7).all()


def test_a_prompt_and_replays():
    """More rows than a launch has CUs, many heads, several jobs, under capture."""
    rng = np.random.default_rng(2)
    B, R, D = 3, 301, 128
    jobs, data = [], []
    for H in (32, 8, 5):
        x, dx = _rows(rng, (B, R, H, D), "bf16")
        out = torch.empty_like(dx)
        jobs.append((dx, H, None, None, out))
        data.append((x, out))
    freq = _freq(64)
    f = torch.from_numpy(freq).cuda()
    base = wc.ints([0, 5, 70000])
    desc = dream.attn_desc(B, 32, 8, D, dream.BF16, 1)
    pos = np.array([[b + r for r in range(R)] for b in (0, 5, 70000)])
    dream.dream_rotary_rows(desc, jobs, R, None, base, None, f, 64, True)
    torch.cuda.synchronize()
    for x, out in data:
        _check(out.double().cpu().numpy(), x, pos, freq, 64, True, 1.0, "bf16")
    first = [out.clone() for _, out in data]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dream.dream_rotary_rows(desc, jobs, R, None, base, None, f, 64, True)
    for _ in range(3):
        for _, out in data:
            out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, out) for a, (_, out) in zip(first, data))
