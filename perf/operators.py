"""Operators of a verification step over long contexts: rotary positions, a key/value cache held in 4 bits, and attention that
sees a sliding window and the first tokens.  Cases to time, each one pass of a decode round's (or a request's) part.

  rotary   queries and keys of the rows a step adds, turned by their positions: the queries stay dense, the keys go to the cache
  append   key and value rows rounded to 4 bits with a scale per 32 values into the caches, and read back
  mx       tree-masked attention over a cache held in 4 bits, with or without a window
  window   tree-masked attention over a 16-bit (or float32) cache that sees a window of positions and the first tokens
  round    what a decode round does with 4-bit caches: append of the drafted rows and attention in every layer, then the commit of
           the accepted path in all caches, whose tree rows are read back

The layout of a 4-bit cache: codes [B, Hkv, s_max, D / 2] (the value of even index in the low half of a byte; a code is a sign and
three bits for 0, 0.5, 1, 1.5, 2, 3, 4, 6) and scales [B, Hkv, s_max, D / 32] (a power of two as its exponent plus 127; 255: not a
number).  The scale of 32 values is the smallest power of two of which their largest magnitude is at most seven times.

A node of the tree sits at position prefix + its depth.  With a window w it sees keys less than w positions back, and the first
n_sink keys.  Calls are made one after the other on torch's current stream with preallocated outputs and workspaces.
"""
import math
import random

import numpy as np
import torch

own = False

# (query heads, KV heads, head_dim, layers, prompt length)
SHAPES = {
    "tiny": (4, 4, 64, 1, 96),
    "llava": (32, 32, 128, 32, 704),
    "pixtral": (32, 8, 128, 40, 1280),
    "gemma3": (16, 8, 256, 48, 1280),
    "smolvlm": (32, 32, 64, 24, 1600),
}
DEPTH = 6            # depth of a drafted tree
MAX_BYTES = 2.0e9    # of a drawn case
MAX_FLOPS = 4.0e11
GROUP = 32           # values that share a scale


def listed():
    return [
        # the rows of one drafted tree, in every layer: launches count
        dict(name="rotary_llava_b1_t60", op="rotary", shape="llava", batch=1, rows=60, prefix=704, layers=32, tree=True, part=1, interleaved=False,
             scaling=1.0, dtype="bf16"),
        # prompts of odd length of a small batch, pairs side by side, half of the head, positions of a long context
        dict(name="rotary_pixtral_b8_prompt", op="rotary", shape="pixtral", batch=8, rows=1279, prefix=120000, layers=1, tree=False, part=2,
             interleaved=True, scaling=4.0, dtype="bf16"),
        # the paper's tree of 32 drafted tokens and its root, one sequence, all layers
        dict(name="append_gemma3_b1_t33", op="append", shape="gemma3", batch=1, rows=33, prefix=1280, layers=48, dtype="bf16"),
        # the prompts of a serving batch, one layer
        dict(name="append_smolvlm_b16_prompt", op="append", shape="smolvlm", batch=16, rows=1600, prefix=0, layers=1, dtype="bf16"),
        # the ordinary decode round of a multi-head model: one sequence, 60 nodes
        dict(name="mx_llava_b1_t60", op="mx", shape="llava", batch=1, prefix=704, tree=60, layers=32, ragged=False, window=0, sink=0, lse=False,
             given=False, dtype="bf16"),
        # grouped queries by four, a small serving batch of odd lengths
        dict(name="mx_pixtral_b8_t60", op="mx", shape="pixtral", batch=8, prefix=1283, tree=60, layers=40, ragged=True, window=0, sink=0, lse=True,
             given=False, dtype="bf16"),
        # the largest: a serving batch of 32 sequences
        dict(name="mx_smolvlm_b32_t60", op="mx", shape="smolvlm", batch=32, prefix=1600, tree=60, layers=24, ragged=False, window=0, sink=0, lse=False,
             given=False, dtype="bf16"),
        # single tokens over long contexts, where the cache's bytes are all that counts
        dict(name="mx_pixtral_b4_t1_long", op="mx", shape="pixtral", batch=4, prefix=32700, tree=1, layers=8, ragged=True, window=0, sink=0, lse=False,
             given=False, dtype="bf16"),
        # layers that see a window, four sequences of odd lengths
        dict(name="window_gemma3_b4_t33", op="window", shape="gemma3", batch=4, prefix=1283, tree=33, layers=40, ragged=True, window=1024, sink=0,
             lse=False, given=False, dtype="bf16"),
        # one token of a stream that has run for long and keeps its first tokens
        dict(name="window_llava_b1_t1_sinks", op="window", shape="llava", batch=1, prefix=8011, tree=1, layers=32, ragged=False, window=1020, sink=4,
             lse=False, given=False, dtype="bf16"),
        # whole rounds over 4-bit caches: a batch of 8, and one sequence whose layers see a window
        dict(name="round_smolvlm_b8_t60", op="round", shape="smolvlm", batch=8, prefix=1601, tree=60, layers=24, ragged=True, window=0, sink=0),
        dict(name="round_gemma3_b1_t33_window", op="round", shape="gemma3", batch=1, prefix=1280, tree=33, layers=48, ragged=False, window=1024, sink=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotary", "append", "mx", "mx", "mx", "window", "window", "round"))
    shape = rng.choice(("llava", "pixtral", "gemma3", "smolvlm"))
    layers = SHAPES[shape][3]
    batch = _log(rng, 1, 32)
    if op in ("rotary", "append"):
        tree = rng.random() < 0.5
        case = dict(op=op, shape=shape, batch=batch, rows=rng.randint(1, 64) if tree else _log(rng, 100, 2400), prefix=_log(rng, 1, 2000),
                    layers=layers if tree else 1, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
        if op == "rotary":
            case.update(tree=tree, part=rng.choice((1, 1, 2, 4)), interleaved=rng.random() < 0.4, scaling=rng.choice((1.0, 1.0, 4.0, 8.0)))
            if not tree:
                case["prefix"] = _log(rng, 1, 1000000)
    elif op == "round":
        window = rng.choice((0, _log(rng, 64, 2000)))
        case = dict(op=op, shape=shape, batch=min(batch, 12), prefix=_log(rng, 200, 4000), tree=rng.randint(8, 64), layers=layers,
                    ragged=rng.random() < 0.5, window=window, sink=rng.randint(0, 8) if window else 0)
    else:
        if op == "window" and rng.random() < 0.15:
            return dict(op=op, shape="tiny", batch=rng.randint(1, 4), prefix=rng.randint(40, 1200), tree=rng.randint(1, 16), layers=1, ragged=False,
                        window=_log(rng, 20, 600), sink=rng.randint(0, 5), lse=True, given=False, dtype="f32")
        tree = rng.choice((1, rng.randint(2, 64), rng.randint(8, 64), rng.randint(8, 64)))
        window = _log(rng, 32, 2000) if op == "window" or rng.random() < 0.3 else 0
        case = dict(op=op, shape=shape, batch=batch, prefix=_log(rng, 200, 2400) if tree > 1 else _log(rng, 200, 40000), tree=tree, layers=layers,
                    ragged=rng.random() < 0.5, window=window, sink=rng.choice((0, rng.randint(1, 70))) if window else 0, lse=rng.random() < 0.3,
                    given=rng.random() < 0.2, dtype="bf16")
    while _cost(case) > 1.0:
        if case["layers"] > 4:
            case["layers"] = case["layers"] * 3 // 4
        elif case["batch"] > 1:
            case["batch"] = case["batch"] * 3 // 4
        else:
            case["layers"] = 1
            break
    return case


def _cost(case):
    w = work(case)
    held = 0.0        # the whole caches are made, whatever a step touches of them
    hq, hkv, d = SHAPES[case["shape"]][:3]
    rows = case["layers"] * case["batch"] * hkv * d
    if case["op"] in ("mx", "window", "round"):
        held = rows * (case["prefix"] + case["tree"]) * 2 * (0.53 if case["op"] != "window" else 2.0) / 6.0e9
    elif case["op"] == "rotary" and case["tree"]:
        held = rows * (case["prefix"] + case["rows"]) * 2 / 2.0e9
    return max(w["bytes"] / MAX_BYTES, w["flops"] / MAX_FLOPS, held)


# ---- sizes -----------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Prefix length of every sequence: the asked one, or spread over its upper half."""
    r = random.Random("lengths %d %d" % (case["batch"], case["prefix"]))
    return [case["prefix"] if not case.get("ragged") or b == 0 else r.randint(case["prefix"] // 2, case["prefix"]) for b in range(case["batch"])]


def _seen(case):
    """Keys that some node of a sequence sees, over the batch."""
    total = 0
    for p in _lengths(case):
        w, s = case["window"], case["sink"]
        first = max(0, p - w + 1) if w else 0
        total += p + case["tree"] - first + min(s if w else 0, first)
    return total


def _cache_rows(n):
    """Row capacity of a cache that holds n live rows (whole pages of 64 rows)."""
    return (n + 63) // 64 * 64


def work(case):
    hq, hkv, d = SHAPES[case["shape"]][:3]
    b, n, op = case["batch"], case["layers"], case["op"]
    e = 4 if case.get("dtype") == "f32" else 2
    packed = d / 2 + d / GROUP                    # bytes of a row of 4-bit values with their scales
    if op == "rotary":
        values = n * b * case["rows"] * (hq + hkv) * d
        return dict(bytes=2 * values * e, flops=3 * values // case["part"])
    if op == "append":
        rows = n * b * case["rows"] * 2 * hkv
        return dict(bytes=rows * (d * e + packed + packed + d * e), flops=4 * rows * d)
    t, seen = case["tree"], _seen(case)
    row = packed if op in ("mx", "round") else d * e
    size = n * (2 * seen * hkv * row + 2 * b * t * hq * d * e + (b * hq * t * 4 if case.get("lse") else 0))
    flops = n * 4 * seen * t * hq * d
    if op == "round":      # half of the drafted depth is accepted on average
        rows = n * b * 2 * hkv
        size += rows * (t * (d * e + packed) + 2 * (1 + DEPTH // 2) * packed + t * (packed + d * e))
    return dict(bytes=int(size), flops=int(flops))


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _tree(r, n, depth=DEPTH):
    """Parents of a level-ordered draft tree of n nodes: levels of about equal size, better ranked parents get more children."""
    depth = min(depth, n - 1)
    if depth < 1:
        return [-1]
    sizes = [1] + [(n - 1) // depth + (l < (n - 1) % depth) for l in range(depth)]
    parent, start = [-1], 0
    for l in range(1, len(sizes)):
        weights = [1.0 / (i + 1) for i in range(sizes[l - 1])]
        picks = sorted(r.choices(range(sizes[l - 1]), weights, k=sizes[l]))
        picks[0] = 0
        parent += [start + p for p in picks]
        start += sizes[l - 1]
    return parent


def _path(r, parent):
    """A root-to-node path."""
    at, path = r.randrange(len(parent)), []
    while at >= 0:
        path.append(at)
        at = parent[at]
    return path[::-1][:DEPTH + 1]


class _Rand:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, *shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="cuda").normal_(generator=self.gen)


def _ints(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device="cuda")


def _type(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _frequencies(case, rot):
    """Turns per position of the pairs, in float32; scaled for long contexts: the slow ones by the factor, the fast ones not."""
    i = np.arange(rot // 2, dtype=np.float64)
    f = 10000.0 ** (-2.0 * i / rot)
    s = case["scaling"]
    if s > 1.0:
        turns = 4096.0 * f / (2.0 * math.pi)
        keep = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
        f = f * keep + f / s * (1.0 - keep)
    return torch.tensor(f.astype(np.float32), device="cuda"), (0.1 * math.log(s) + 1.0 if s > 1.0 else 1.0)


def _rows(rnd, dtype, *shape):
    """Key and value rows: some dimensions of a head are larger than others, as those of keys are."""
    x = rnd.normal(*shape, dtype=torch.float32)
    gain = torch.exp(0.7 * rnd.normal(shape[-2], shape[-1], dtype=torch.float32))
    return (x * gain).to(dtype)


def _cache(rnd, layers, b, hkv, rows, d):
    """A 4-bit cache full of rows."""
    codes = torch.empty(layers, b, hkv, rows, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(layers, b, hkv, rows, d // GROUP, dtype=torch.uint8, device="cuda")
    for l in range(layers):
        codes[l], scales[l] = _quantise(_rows(rnd, torch.bfloat16, b, hkv, rows, d))
    return codes, scales


def _desc(case, rows):
    import paper_2505_19201_amd as dream
    hq, hkv, d = SHAPES[case["shape"]][:3]
    return dream.attn_desc(case["batch"], hq, hkv, d, dream.F32 if case.get("dtype") == "f32" else dream.BF16, rows)


def _prepare_rotary(case, rnd, r):
    hq, hkv, d = SHAPES[case["shape"]][:3]
    b, n, layers, dt = case["batch"], case["rows"], case["layers"], _type(case)
    start = case["prefix"] if case["tree"] else 0     # (a prompt's keys start the cache, wherever its positions start)
    rows = _cache_rows(start + n)
    rot = d // case["part"]
    freq, amplitude = _frequencies(case, rot)
    s = dict(hq=hq, hkv=hkv, n=n, at=start, rot=rot, interleaved=case["interleaved"], freq=freq, amplitude=amplitude, layers=layers,
             q=rnd.normal(layers, b, n, hq, d, dtype=dt), k=rnd.normal(layers, b, n, hkv, d, dtype=dt),
             out=torch.empty(layers, b, n, hq, d, dtype=dt, device="cuda"), cache=torch.zeros(layers, b, hkv, rows, d, dtype=dt, device="cuda"),
             base=_ints([start] * b), pos_base=_ints([case["prefix"] + i for i in range(b)]),
             parent=_ints([_tree(r, n) for _ in range(b)]) if case["tree"] else None)
    if own:
        s["desc"] = _desc(case, rows)
        s["calls"] = [((s["q"][l], hq, None, None, s["out"][l]), (s["k"][l], hkv, s["base"], None, s["cache"][l])) for l in range(layers)]
    return s


def _prepare_append(case, rnd, r):
    hq, hkv, d = SHAPES[case["shape"]][:3]
    b, n, layers, dt = case["batch"], case["rows"], case["layers"], _type(case)
    rows = _cache_rows(case["prefix"] + n)
    s = dict(n=n, at=case["prefix"], layers=layers, base=_ints([case["prefix"]] * b), k=_rows(rnd, dt, layers, b, n, hkv, d), v=rnd.normal(layers, b, n, hkv, d, dtype=dt),
             codes=torch.zeros(layers, 2, b, hkv, rows, d // 2, dtype=torch.uint8, device="cuda"),
             scales=torch.zeros(layers, 2, b, hkv, rows, d // GROUP, dtype=torch.uint8, device="cuda"),
             out=torch.empty(2 * layers, b, hkv, n, d, dtype=dt, device="cuda"))
    if own:
        s["desc"] = _desc(case, rows)
        s["calls"] = [(s["k"][l], s["v"][l], s["codes"][l][0], s["scales"][l][0], s["codes"][l][1], s["scales"][l][1]) for l in range(layers)]
        s["each"] = [c for x in s["codes"] for c in x], [c for x in s["scales"] for c in x]
    return s


def _given_mask(r, parent):
    """A mask as a caller may give it: ancestors and the node itself, some of them left out, some nodes without any."""
    bits = []
    for row in parent:
        for i in range(len(row)):
            m, at = 0, i
            while at >= 0:
                m |= (r.random() < 0.9) << at
                at = row[at]
            m = 0 if r.random() < 0.1 else m
            bits.append(m - (1 << 64) if m >> 63 else m)
    return torch.tensor(np.array(bits, dtype=np.int64).reshape(len(parent), len(parent[0]), 1), device="cuda")


def _prepare_attention(case, rnd, r):
    hq, hkv, d = SHAPES[case["shape"]][:3]
    b, t, layers, dt, op = case["batch"], case["tree"], case["layers"], _type(case), case["op"]
    lengths = _lengths(case)
    rows = _cache_rows(max(lengths) + t)
    parent = [_tree(r, t) for _ in range(b)]
    s = dict(layers=layers, tree=t, max_kv=max(lengths) + t, window=case["window"], sink=case["sink"], prefix_len=_ints(lengths), parent=_ints(parent),
             mask=_given_mask(r, parent) if case.get("given") else None, q=rnd.normal(layers, b, t, hq, d, dtype=dt),
             out=torch.empty(layers, b, t, hq, d, dtype=dt, device="cuda"),
             lse=torch.empty(layers, b, hq, t, device="cuda") if case.get("lse") else None)
    if op == "window":
        s["k"], s["v"] = rnd.normal(layers, b, hkv, rows, d, dtype=dt), rnd.normal(layers, b, hkv, rows, d, dtype=dt)
    else:
        s["k"], s["v"] = _cache(rnd, layers, b, hkv, rows, d), _cache(rnd, layers, b, hkv, rows, d)
    if op == "round":
        paths = [_path(r, p) for p in parent]
        s.update(k_rows=_rows(rnd, dt, layers, b, t, hkv, d), v_rows=rnd.normal(layers, b, t, hkv, d, dtype=dt),
                 path=_ints([p + [-1] * (DEPTH + 1 - len(p)) for p in paths]), length=_ints([len(p) - 1 for p in paths]),
                 new_len=torch.empty(b, dtype=torch.int32, device="cuda"), read=torch.empty(2 * layers, b, hkv, t, d, dtype=dt, device="cuda"))
    if own:
        import paper_2505_19201_amd as dream
        s["desc"] = _desc(case, rows)
        size = dream.dream_window_verify_attn_workspace if op == "window" else dream.dream_mx_verify_attn_workspace
        s["ws"] = dream.alloc_workspace(size(s["desc"], t, s["max_kv"], s["window"], s["sink"]))
        each = [s["k"], s["v"]] if op == "window" else [*s["k"], *s["v"]]
        s["calls"] = [(s["q"][l], [x[l] for x in each], s["out"][l], None if s["lse"] is None else s["lse"][l]) for l in range(layers)]
        if op == "round":
            s["rows"] = [(s["k_rows"][l], s["v_rows"][l]) for l in range(layers)]
            s["each"] = [*s["k"][0], *s["v"][0]], [*s["k"][1], *s["v"][1]]
    return s


_PREPARE = dict(rotary=_prepare_rotary, append=_prepare_append, mx=_prepare_attention, window=_prepare_attention, round=_prepare_attention)


def prepare(case, seed):
    if own:
        import paper_2505_19201_amd as dream
        dream.load()
        dream.dream_init()
    return case["op"], _PREPARE[case["op"]](case, _Rand(seed), random.Random(seed))


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _own_rotary(s):
    import paper_2505_19201_amd as dream
    for jobs in s["calls"]:
        dream.dream_rotary_rows(s["desc"], jobs, s["n"], None, s["pos_base"], s["parent"], s["freq"], s["rot"], s["interleaved"], s["amplitude"])
    return [s["out"], s["cache"]]


def _own_append(s):
    import paper_2505_19201_amd as dream
    for k, v, *caches in s["calls"]:
        dream.dream_mx_append(s["desc"], k, v, s["n"], s["base"], None, *caches)
    dream.dream_mx_read(s["desc"], *s["each"], s["base"], s["n"], s["out"])
    return [s["out"]]


def _own_attention(s, attend):
    for q, caches, out, lse in s["calls"]:
        attend(s["desc"], q, *caches, s["prefix_len"], s["tree"], s["parent"], s["mask"], s["window"], s["sink"], s["max_kv"], out, lse, s["ws"])
    return [s["out"], s["lse"]]


def _own_mx(s):
    import paper_2505_19201_amd as dream
    return _own_attention(s, dream.dream_mx_verify_attn)


def _own_window(s):
    import paper_2505_19201_amd as dream
    return _own_attention(s, dream.dream_window_verify_attn)


def _own_round(s):
    import paper_2505_19201_amd as dream
    for (k, v), (q, caches, out, _) in zip(s["rows"], s["calls"]):
        dream.dream_mx_append(s["desc"], k, v, s["tree"], s["prefix_len"], None, *caches)
        dream.dream_mx_verify_attn(s["desc"], q, *caches, s["prefix_len"], s["tree"], s["parent"], None, s["window"], s["sink"], s["max_kv"], out, None,
                                   s["ws"])
    dream.dream_mx_commit(s["desc"], *s["each"], s["prefix_len"], s["tree"], s["path"], s["length"], s["new_len"])
    dream.dream_mx_read(s["desc"], *s["each"], s["prefix_len"], s["tree"], s["read"])
    return [s["out"], s["new_len"], s["read"]]


# ---- plain forms -----------------------------------------------------------------------------------------------------
def _quantise(x):
    """Codes and scales of rows [..., D]."""
    g = x.float().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    byte = (((top.view(torch.int32) + 0x1FFFFF) >> 23) - 2).clamp(2, 252)         # (mantissas above 1.75 take the next exponent)
    a = g * ((254 - byte) << 23).view(torch.float32).unsqueeze(-1)                # times the scale's inverse, a power of two
    m = a.abs()
    code = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)) + 8 * (a < 0)
    code = code.flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte.to(torch.uint8)


def _values(codes, scales):
    """What codes and scales stand for, in float32."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    table = torch.cat([table, -table])
    x = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    return (table[x.int()].unflatten(-1, (-1, GROUP)) * (scales.int() << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)


def _ancestors(parent):
    """[B, T, T]: node a is node i or an ancestor of it; and the depths."""
    b, t = parent.shape
    reach = torch.eye(t, device=parent.device).expand(b, t, t).clone()
    child = (parent >= 0).nonzero()
    reach[child[:, 0], child[:, 1], parent[child[:, 0], child[:, 1]].long()] = 1.0
    for _ in range(max(1, t - 1).bit_length()):
        reach = (torch.matmul(reach, reach) > 0).float()
    return reach > 0, reach.sum(-1).long() - 1


def _plain_rotary(s):
    q = s["q"]
    b, n = q.shape[1:3]
    step = torch.arange(n, device="cuda").expand(b, n) if s["parent"] is None else _ancestors(s["parent"])[1]
    angle = (s["pos_base"].long().unsqueeze(1) + step).double().unsqueeze(-1) * s["freq"].double()     # far positions: angles in 64 bits
    cos, sin = (angle.cos() * s["amplitude"]).float().unsqueeze(2), (angle.sin() * s["amplitude"]).float().unsqueeze(2)
    rot, half = s["rot"], s["rot"] // 2

    def turn(x):
        y = x.float()
        a, c = (y[..., 0:rot:2], y[..., 1:rot:2]) if s["interleaved"] else (y[..., :half], y[..., half:rot])
        u, w = a * cos - c * sin, a * sin + c * cos
        z = torch.stack([u, w], -1).flatten(-2) if s["interleaved"] else torch.cat([u, w], -1)
        return torch.cat([z, y[..., rot:]], -1).to(x.dtype)

    at = s["at"]
    for l in range(s["layers"]):
        s["out"][l] = turn(q[l])
        s["cache"][l, :, :, at:at + n] = turn(s["k"][l]).transpose(1, 2)
    return [s["out"], s["cache"]]


def _plain_append(s):
    n = s["n"]
    at = s["at"]
    for l in range(s["layers"]):
        for i, x in enumerate((s["k"][l], s["v"][l])):
            c, e = _quantise(x.transpose(1, 2))
            s["codes"][l, i, :, :, at:at + n], s["scales"][l, i, :, :, at:at + n] = c, e
            s["out"][2 * l + i] = _values(s["codes"][l, i, :, :, at:at + n], s["scales"][l, i, :, :, at:at + n]).to(x.dtype)
    return [s["out"]]


def _visible(s, rows):
    """[B, T, rows]: which keys a node sees."""
    p, t, w = s["prefix_len"].long().view(-1, 1, 1), s["tree"], s["window"]
    b = p.shape[0]
    reach, depth = _ancestors(s["parent"])
    if s["mask"] is not None:
        reach = (s["mask"] >> torch.arange(t, device="cuda")) & 1 > 0
    key = torch.arange(rows, device="cuda").view(1, 1, -1)
    rel = (key - p).clamp(0, t - 1)
    vis = (key < p) | ((key < p + t) & reach.gather(2, rel.expand(b, t, rows)))
    if w:
        at = torch.where(key < p, key.expand(b, 1, rows), p + depth.unsqueeze(1).gather(2, rel.expand(b, 1, rows)))
        vis = vis & ((p + depth.unsqueeze(2) - at < w) | (at < s["sink"]))
    return vis


def _attend(q, k, v, vis):
    """softmax(q k^T / sqrt(D)) v over visible keys, in float32: rows [B, T, Hq, D] and log-sum-exps [B, Hq, T]."""
    b, t, hq, d = q.shape
    hkv, g = k.shape[1], q.shape[2] // k.shape[1]
    x = q.float().view(b, t, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, g * t, d)
    x = torch.matmul(x, k.float().transpose(2, 3)).mul_(d ** -0.5).view(b, hkv, g, t, -1)
    x.masked_fill_(~vis[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(b, hkv, g * t, -1), v.float()).view(b, hkv, g, t, d) / total.clamp(min=1e-38)
    return o.permute(0, 3, 1, 2, 4).reshape(b, t, hq, d), (top + total.log()).reshape(b, hq, t)


def _plain_mx(s):
    vis = _visible(s, s["k"][0].shape[3])
    for l in range(s["layers"]):
        o, lse = _attend(s["q"][l], _values(s["k"][0][l], s["k"][1][l]), _values(s["v"][0][l], s["v"][1][l]), vis)
        s["out"][l] = o.to(s["q"].dtype)
        if s["lse"] is not None:
            s["lse"][l] = lse
    return [s["out"], s["lse"]]


def _plain_window(s):
    vis = _visible(s, s["k"].shape[3])
    for l in range(s["layers"]):
        o, lse = _attend(s["q"][l], s["k"][l], s["v"][l], vis)
        s["out"][l] = o.to(s["q"].dtype)
        if s["lse"] is not None:
            s["lse"][l] = lse
    return [s["out"], s["lse"]]


def _plain_round(s):
    t, p = s["tree"], s["prefix_len"].long()
    b = p.shape[0]
    who = torch.arange(b, device="cuda").unsqueeze(1)
    at = p.unsqueeze(1) + torch.arange(t, device="cuda")
    vis = _visible(s, s["k"][0].shape[3])
    for l in range(s["layers"]):
        for (codes, scales), x in ((s["k"], s["k_rows"]), (s["v"], s["v_rows"])):
            codes[l][who, :, at], scales[l][who, :, at] = _quantise(x[l])
        s["out"][l] = _attend(s["q"][l], _values(s["k"][0][l], s["k"][1][l]), _values(s["v"][0][l], s["v"][1][l]), vis)[0].to(s["q"].dtype)
    # rows of the path move up; entries behind its end stay where they are
    step = torch.arange(s["path"].shape[1], device="cuda")[None, :t]
    source = torch.where(step <= s["length"].unsqueeze(1), s["path"][:, :t], step).long()
    for i, (codes, scales) in enumerate((s["k"], s["v"])):
        for l in range(s["layers"]):
            for c in (codes[l], scales[l]):
                c[who, :, p.unsqueeze(1) + step] = c[who, :, p.unsqueeze(1) + source]
            s["read"][i * s["layers"] + l] = _values(codes[l][who, :, at], scales[l][who, :, at]).transpose(1, 2).to(s["read"].dtype)
    s["new_len"].copy_(s["prefix_len"] + s["length"] + 1)
    return [s["out"], s["new_len"], s["read"]]


_PLAIN = dict(rotary=_plain_rotary, append=_plain_append, mx=_plain_mx, window=_plain_window, round=_plain_round)
_OWN = dict(rotary=_own_rotary, append=_own_append, mx=_own_mx, window=_own_window, round=_own_round)


def run(state):
    op, s = state
    return (_OWN if own else _PLAIN)[op](s)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def _walk(parent):
    """Per sequence and node: the node and its ancestors, root last."""
    rows = parent.tolist()
    out = []
    for row in rows:
        paths = []
        for i, p in enumerate(row):
            paths.append([i] + (paths[p] if p >= 0 else []))
        out.append(paths)
    return out


def _power(e):
    """2^e in 64 bits, for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x):
    """The 4-bit values of rows [..., D] in 64 bits: per 32 values the smallest power of two of which none is more than seven times, then the nearest value,
    the even code where two are."""
    g = x.double().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(torch.where(top > 0, top / 7.0, torch.ones_like(top))))
    power = torch.where(7.0 * _power(power - 1) >= top, power - 1, power)      # (log2 is rounded)
    power = torch.where(7.0 * _power(power) < top, power + 1, power)
    power = torch.where(top > 0, power, torch.zeros_like(power)).clamp(-125, 125)
    unit = _power(power)
    best, dist = torch.zeros_like(g), g.abs()
    for code, v in ((2, 1.0), (4, 2.0), (6, 4.0), (1, 0.5), (3, 1.5), (5, 3.0), (7, 6.0)):      # even codes first: they keep a tie
        d = (g.abs() - v * unit).abs()
        best, dist = torch.where(d < dist, v * unit, best), torch.minimum(d, dist)
    return (best * torch.sign(g)).flatten(-2)


def _exact_values(codes, scales):
    x = torch.stack([codes % 16, codes // 16], -1).flatten(-2).long()
    e, m = (x % 8) // 2, (x % 2).double()
    v = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * _power(e - 1)) * torch.where(x > 7, -1.0, 1.0)
    return v * torch.repeat_interleave(_power(scales.long() - 127), GROUP, -1)


def _exact_rotary(s):
    walk = None if s["parent"] is None else _walk(s["parent"])
    b, n = s["q"].shape[1:3]
    pos = [[int(p) + (i if walk is None else len(walk[j][i]) - 1) for i in range(n)] for j, p in enumerate(s["pos_base"].tolist())]
    phase = torch.tensor(pos, dtype=torch.float64, device="cuda")[:, :, None, None] * s["freq"].double()
    unit = torch.polar(torch.full_like(phase, s["amplitude"]), phase)
    rot = s["rot"]

    def turn(x):
        y = x.double()
        pair = y[..., :rot].unflatten(-1, (rot // 2, 2)) if s["interleaved"] else y[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * unit)
        y[..., :rot] = (z if s["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        return y

    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    cache = s["cache"].double()
    at = s["at"]
    for l in range(s["layers"]):
        out[l] = turn(s["q"][l])
        cache[l, :, :, at:at + n] = turn(s["k"][l]).transpose(1, 2)
    return [out, cache]


def _exact_append(s):
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    for l in range(s["layers"]):
        out[2 * l], out[2 * l + 1] = _nearest(s["k"][l].transpose(1, 2)), _nearest(s["v"][l].transpose(1, 2))
    return [out]


def _exact_sequences(s, out, lse, layer, keys, values, walk):
    """One layer: each node over the list of keys that it sees."""
    w, sink, d = s["window"], s["sink"], s["q"].shape[-1]
    given = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint64)
    for b, p in enumerate(s["prefix_len"].tolist()):
        t, live = s["tree"], p + s["tree"]
        seen = np.zeros((t, live), dtype=bool)
        for i, path in enumerate(walk[b]):
            depth = len(path) - 1
            first = max(0, p + depth - w + 1) if w else 0
            seen[i, min(first, p):p] = True
            seen[i, :min(sink if w else 0, p)] = True
            nodes = path if given is None else [a for a in range(t) if int(given[b, i, 0]) >> a & 1]
            for a in nodes:
                back = depth - (len(walk[b][a]) - 1)
                if not w or back < w or p + len(walk[b][a]) - 1 < sink:
                    seen[i, p + a] = True
        seen = torch.tensor(seen, device="cuda")
        k, v = keys(b, live), values(b, live)
        q = s["q"][layer, b].double().transpose(0, 1)                      # [Hq, T, D]
        group = q.shape[0] // k.shape[0]
        x = torch.matmul(q, k.repeat_interleave(group, 0).transpose(1, 2).contiguous()) / math.sqrt(d)
        x = torch.where(seen, x, torch.full_like(x, float("-inf")))
        total = torch.logsumexp(x, -1)                                     # [Hq, T]
        x = torch.where(seen, torch.exp(x - total.unsqueeze(-1)), torch.zeros_like(x))
        out[layer, b] = torch.matmul(x, v.repeat_interleave(group, 0)).transpose(0, 1)
        if lse is not None:
            lse[layer, b] = total


def _exact_attention(s, op):
    walk = _walk(s["parent"])
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = None if s["lse"] is None else torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    for l in range(s["layers"]):
        if op == "window":
            of = [lambda b, n, x=x: x[l, b, :, :n].double() for x in (s["k"], s["v"])]
        else:
            of = [lambda b, n, x=x: _exact_values(x[0][l, b, :, :n], x[1][l, b, :, :n]) for x in (s["k"], s["v"])]
        _exact_sequences(s, out, lse, l, of[0], of[1], walk)
    return [out, lse]


def _exact_round(s):
    walk = _walk(s["parent"])
    t, layers = s["tree"], s["layers"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    read = torch.empty(s["read"].shape, dtype=torch.float64, device="cuda")
    lengths, paths, prefix = s["length"].tolist(), s["path"].tolist(), s["prefix_len"].tolist()
    for l in range(layers):
        new = [_nearest(x[l].transpose(1, 2)) for x in (s["k_rows"], s["v_rows"])]      # [B, Hkv, T, D]
        of = []
        for x, y in zip((s["k"], s["v"]), new):
            of.append(lambda b, n, x=x, y=y: torch.cat([_exact_values(x[0][l, b, :, :n - t], x[1][l, b, :, :n - t]), y[b]], 1))
        _exact_sequences(s, out, None, l, of[0], of[1], walk)
        for i in range(2):
            for b in range(len(prefix)):
                order = paths[b][:lengths[b] + 1] + list(range(lengths[b] + 1, t))
                read[i * layers + l, b] = new[i][b][:, order]
    return [out, torch.tensor([p + n + 1 for p, n in zip(prefix, lengths)], device="cuda"), read]


def exact(case, seed):
    global own
    held, own = own, False
    try:
        op, s = prepare(case, seed)
    finally:
        own = held
    if op == "rotary":
        return _exact_rotary(s)
    if op == "append":
        return _exact_append(s)
    return _exact_round(s) if op == "round" else _exact_attention(s, op)
