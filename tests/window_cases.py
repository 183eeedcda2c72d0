"""Definitions in 64 bits of rotary positions, 4-bit caches and window attention, for the tests (numpy, on the host)."""
import numpy as np
import torch

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def ancestors(parent):
    """Per node: itself and its ancestors, and its depth."""
    paths = []
    for i, p in enumerate(parent):
        paths.append([i] + (paths[p] if 0 <= p < i else []))
    return paths


def visible(parent, P, window, sink, mask=None):
    """[T, P + T] truth values for one sequence."""
    paths = ancestors(parent)
    T = len(parent)
    see = np.zeros((T, P + T), dtype=bool)
    for i in range(T):
        depth = len(paths[i]) - 1
        nodes = paths[i] if mask is None else [a for a in range(T) if int(mask[i][a // 64]) >> (a % 64) & 1]
        at = {j: j for j in range(P)}
        at.update({P + a: P + len(paths[a]) - 1 for a in nodes})
        for j, pos in at.items():
            see[i, j] = not window or P + depth - pos < window or pos < sink
    return see


def attention(q, k, v, prefix, parent, window=0, sink=0, masks=None, scale=None):
    """q [B, T, Hq, D], caches [B, Hkv, s_max, D], all float64.  Rows, log-sum-exps, sums of p |v| and, per row, the largest sum over channels of |q k| scale."""
    B, T, Hq, D = q.shape
    G = Hq // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    out, lse = np.zeros(q.shape), np.full((B, Hq, T), -np.inf)
    mass, size = np.zeros(q.shape), np.zeros((B, Hq, T))
    for b in range(B):
        P = prefix[b]
        see = visible(parent[b], P, window, sink, None if masks is None else masks[b])
        for h in range(Hq):
            kk, vv = k[b, h // G, :P + T], v[b, h // G, :P + T]
            for i in range(T):
                w = np.flatnonzero(see[i])
                if not len(w):
                    continue
                with np.errstate(invalid="ignore"):
                    x = kk[w] @ q[b, i, h] * scale
                    top = x.max()
                    p = np.exp(x - top)
                    lse[b, h, i] = top + np.log(p.sum())
                    p /= p.sum()
                    out[b, i, h] = p @ vv[w]
                    mass[b, i, h] = p @ np.abs(vv[w])
                    size[b, h, i] = (np.abs(kk[w]) @ np.abs(q[b, i, h])).max() * abs(scale)
    return out, lse, mass, size


def attention_bounds(out, mass, size, n_keys, D, bf16):
    """What rounding may move: bf16 probabilities and the row by half a step of 2^-8 each; scores by D products added in float32 (2^-24 of their absolute sum each), which moves
    every probability by as much; sums of n_keys terms in float32; exponentials and the reference's scaling by a few steps of 2^-23."""
    score = (D + 2) * size * 2.0 ** -24
    each = 2 * score.transpose(0, 2, 1)[..., None] + (2 * n_keys + 64) * 2.0 ** -24
    row = mass * ((2.0 ** -8 if bf16 else 0.0) + each) * (1 + 2.0 ** -6) + np.abs(out) * (2.0 ** -8 if bf16 else 2.0 ** -23) + 1e-30
    lse = score + (n_keys + 64) * 2.0 ** -24
    return row, lse


def quantise(x):
    """Codes (sign and magnitude, unpacked) and scale bytes of rows [..., D]."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, 32)
    finite = np.isfinite(g).all(-1)
    g0 = np.where(finite[..., None], g, 0.0)
    top = np.abs(g0).max(-1)
    with np.errstate(divide="ignore"):
        e = np.where(top > 0, np.floor(np.log2(np.where(top > 0, top, 1.0))), -1000).astype(int)
    e = e - 3
    for _ in range(4):
        e = np.where(7.0 * np.exp2(e.astype(float)) < top, e + 1, e)
    e = np.clip(e, -125, 125)
    a = np.abs(g0) / np.exp2(e.astype(float))[..., None]
    dist = np.abs(a[..., None] - VALUES)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])       # even codes first: they keep a tie
    code = order[dist[..., order].argmin(-1)]
    code = code + 8 * np.signbit(g0)
    byte = np.where(finite, e + 127, 255)
    return code.reshape(x.shape), byte.astype(np.uint8), finite


def pack(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def decode(packed, scales):
    code = np.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], -1)
    v = np.where(code > 7, -VALUES[code & 7], VALUES[code & 7])
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(float) - 127))
    return v * np.repeat(s, 32, -1)


def rotary(x, pos, freq, rot, paired, amplitude=1.0):
    """x [B, R, H, D] float64, pos [B, R]."""
    a = pos[:, :, None, None].astype(np.float64) * freq.astype(np.float64)
    c, s = np.cos(a) * amplitude, np.sin(a) * amplitude
    y = x.copy()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if paired else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def tree(kind, n, rng):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    return [-1] + [int(rng.integers(max(0, i - 12), i)) for i in range(1, n)]


def masks_of(parent, rng, drop=0.2, empty=0.2):
    """[B, T, W] uint64: ancestors with some left out, some nodes without any, and nodes that are no ancestors."""
    out = []
    for row in parent:
        T = len(row)
        m = np.zeros((T, (T + 63) // 64), dtype=np.uint64)
        for i, path in enumerate(ancestors(row)):
            if rng.random() < empty:
                continue
            for a in path + [int(rng.integers(T))]:
                if rng.random() > drop:
                    m[i, a // 64] |= np.uint64(1 << (a % 64))
        out.append(m)
    return np.stack(out)


def bf16(x):
    """Rounded to bf16, as float64 (ties to even)."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")
