"""Every kernel that dream_window_verify_attn and dream_mx_verify_attn can take, forced, on the cases the choice would give to another one."""
import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from tests import window_cases as wc
from tests.test_gpu_window import _poison, _Problem

pytestmark = pytest.mark.gpu

# query tiles, waves, splits
SHAPES = [(1, 4, 1), (1, 4, 3), (2, 4, 1), (2, 4, 4), (4, 4, 1), (4, 4, 2), (1, 8, 1), (1, 8, 2), (0, 8, 1), (0, 8, 3), (0, 8, 64), (1, 4, 64)]
CASES = [
    (1, 2, 2, "rand", 1, [0], 0, 0, False),
    (3, 4, 2, "rand", 9, [31, 0, 97], 40, 3, False),
    (2, 8, 1, "rand", 60, [300, 45], 100, 4, False),
    (1, 6, 2, "chain", 70, [260], 0, 0, False),
    (1, 2, 1, "rand", 250, [700], 0, 0, False),
    (1, 4, 2, "rand", 130, [70], 50, 2, True),
]


@pytest.fixture(autouse=True)
def _as_it_was():
    yield
    dream.dream_set_q_tiles(0)
    dream.dream_set_tile_waves(0)
    dream.dream_set_kv_splits(0)


def _force(shape):
    tiles, waves, splits = shape
    dream.dream_set_q_tiles(tiles)
    dream.dream_set_tile_waves(waves)
    dream.dream_set_kv_splits(splits)


@pytest.mark.parametrize("kind", ["bf16", "mx"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:5]) + f"-w{c[6]}")
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "q%dw%ds%d" % s)
def test_rows(shape, case, D, kind):
    _force(shape)
    p = _Problem(case[:3] + (D,) + case[3:], kind)
    p.call()
    p.check()


@pytest.mark.parametrize("kind", ["bf16", "mx"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "q%dw%ds%d" % s)
def test_what_no_row_sees_changes_nothing(shape, D, kind):
    _force(shape)
    p = _Problem((2, 4, 2, D, "rand", 9, [150, 70], 41, 3, False), kind)
    for b, P in enumerate(p.prefix):
        _poison(p, b, slice(P + p.T, None), float("nan"))
        _poison(p, b, slice(3, P - 41 + 1), float("inf"))
    p.call()
    p.check()


@pytest.mark.parametrize("waves", [4, 8])
def test_the_longest_cache(waves):
    """Offsets in a head up to 64 KB below 2^32."""
    rows, D, T, n = (1 << 23) - 128, 256, 3, 40
    dream.dream_set_tile_waves(waves)
    desc = dream.attn_desc(1, 2, 1, D, dream.BF16, rows)
    rng = np.random.default_rng(11)
    k, v = (torch.zeros(1, 1, rows, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tails = [wc.bf16(rng.standard_normal((1, 1, n, D))) for _ in range(2)]
    for cache, tail in zip((k, v), tails):
        cache[:, :, rows - n:] = torch.from_numpy(tail).bfloat16().cuda()
    q = wc.bf16(rng.standard_normal((1, T, 2, D)))
    out = torch.empty(1, T, 2, D, dtype=torch.bfloat16, device="cuda")
    ws = dream.alloc_workspace(dream.dream_window_verify_attn_workspace(desc, T, rows, 20, 0))
    dream.dream_window_verify_attn(desc, torch.from_numpy(q).bfloat16().cuda(), k, v, wc.ints([rows - T]), T, wc.ints([[-1, 0, 1]]), None, 20, 0, rows, out, None, ws)
    torch.cuda.synchronize()
    want, _, mass, size = wc.attention(q, *tails, [n - T], [[-1, 0, 1]], 20, 0)
    bound, _ = wc.attention_bounds(want, mass, size, n, D, True)
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("kind", ["bf16", "mx"])
def test_as_many_streams_as_there_may_be(kind):
    """2^20 - 16 KV heads of all sequences together, two keys each."""
    B, H, D = 65535, 16, 64
    torch.manual_seed(5)
    desc = dream.attn_desc(B, H, H, D, dream.BF16, 2)
    q = torch.randn(B, 1, H, D, device="cuda").bfloat16()
    kv, held = [], []
    for _ in range(2):
        if kind == "mx":
            codes = torch.randint(0, 256, (B, H, 2, D // 2), dtype=torch.uint8, device="cuda")
            scales = torch.randint(125, 129, (B, H, 2, D // 32), dtype=torch.uint8, device="cuda")
            held += [codes, scales]
            at = torch.stack([codes & 15, codes >> 4], -1).reshape(B, H, 2, D)
            table = torch.tensor(np.concatenate([wc.VALUES, -wc.VALUES]), dtype=torch.float32, device="cuda")
            kv.append(table[at.long()] * torch.exp2(scales.float() - 127).repeat_interleave(32, -1))
        else:
            held.append(torch.randn(B, H, 2, D, device="cuda").bfloat16())
            kv.append(held[-1].float())
    out = torch.full_like(q, float("nan"))
    lse = torch.empty(B, H, 1, device="cuda")
    size, call = (dream.dream_mx_verify_attn_workspace, dream.dream_mx_verify_attn) if kind == "mx" else (dream.dream_window_verify_attn_workspace, dream.dream_window_verify_attn)
    ws = dream.alloc_workspace(size(desc, 1, 2, 0, 0))
    call(desc, q, *held, torch.ones(B, dtype=torch.int32, device="cuda"), 1, torch.full((B, 1), -1, dtype=torch.int32, device="cuda"), None, 0, 0, 2, out, lse, ws)
    torch.cuda.synchronize()
    # in float32: D products each off by 2^-24 of the sum of their sizes, which the two probabilities take over, besides bf16 probabilities and rows (2^-8 each)
    x = q.float()[:, 0].unsqueeze(2) * kv[0] * D ** -0.5
    s, size = x.sum(-1), x.abs().sum(-1).amax(-1, keepdim=True)
    p = torch.softmax(s, -1).unsqueeze(-1)
    want, mass = (p * kv[1]).sum(2), (p * kv[1].abs()).sum(2)
    bound = mass * (2.0 ** -8 + 4 * (D + 2) * size * 2.0 ** -24 + 2.0 ** -16) * (1 + 2.0 ** -6) + want.abs() * 2.0 ** -8 + 1e-30
    assert bool(((out.float()[:, 0] - want).abs() <= bound).all())
    assert bool(((lse[..., 0] - torch.logsumexp(s, -1)).abs() <= 2 * (D + 2) * size[..., 0] * 2.0 ** -24 + 2.0 ** -17).all())
