"""Operators of serving out of a paged cache: rows enter it with their positions turned on the way, a batch that shares a long prefix attends to it
once for all, and over long contexts a node attends only to the pages that a cheap score selects for it.  Cases to time, each one pass.

  append   queries and keys of new rows turned by their positions, keys and values written to the pages of their sequences; a prompt's pages get
           their bounds as well
  attend   tree-masked attention over pages; the prefix that the sequences of a group share is read once for all of them
  sparse   pages selected for every node and KV head by their bounds, then tree-masked attention over those pages and the tree
  round    what a decode round does with such caches: append of the drafted rows, selection and attention in every layer, then the commit of the
           accepted path in all of them and the bounds of the pages that it reached

A cache's pages are [n_pages, Hkv, page_size, D]; row j of sequence b stands in page page_table[b, j / page_size].  The bounds of a page are the
largest and the smallest of its keys in every channel, [n_pages, Hkv, 2, D].  A score bounds the product of a node's queries with any key of the page:
queries are held as whole numbers up to 127 times a power of two (one for the query heads of a KV head, to nearest), bounds likewise (one for a page
and head, rounded outwards), and with q+ and q- the positive and negative parts of the queries, summed over the heads, the score is
(q+ . upper + q- . lower) times the page's power of two, in whole numbers that are rounded once to float32.  Of the pages of a sequence's prefix a node
sees the first, the last, and those of the highest scores in between, the earlier ones where scores are equal.

A node of the tree stands at position prefix + its depth.  Calls are made one after the other on torch's current stream with preallocated outputs and
workspaces.
"""
import math
import random

import numpy as np
import torch

own = False

# (query heads, KV heads, head_dim)
SHAPES = {
    "tiny": (4, 2, 64),
    "llava": (32, 32, 128),
    "pixtral": (32, 8, 128),
    "gemma3": (16, 8, 256),
    "smolvlm": (32, 32, 64),
}
DEPTH = 6            # depth of a drafted tree
MAX_BYTES = 8.5e8    # of a drawn case
MAX_FLOPS = 2.7e11
MAX_HELD = 1.3e9      # bytes of its caches


def listed():
    return [
        # the rows of one drafted tree, in every layer: launches count
        dict(name="append_llava_b1_t60", op="append", shape="llava", batch=1, rows=60, prefix=704, page=64, layers=32, tree=True, part=1,
             interleaved=False, scaling=1.0, bounds=False, dtype="bf16"),
        # prompts of different lengths in a padded batch, pairs side by side, half of the head; the bounds of their pages
        dict(name="append_pixtral_b8_prompt", op="append", shape="pixtral", batch=8, rows=2391, prefix=0, page=64, layers=1, tree=False, part=2,
             interleaved=True, scaling=4.0, bounds=True, dtype="bf16"),
        # the ordinary verification of one sequence, nothing shared
        dict(name="attend_llava_b1_t60", op="attend", shape="llava", batch=1, prefix=704, shared=0, groups=0, tree=60, page=64, layers=32,
             ragged=False, lse=False, given=False, dtype="bf16"),
        # single tokens over long contexts of different lengths: the cache's bytes count
        dict(name="attend_pixtral_b8_t1_long", op="attend", shape="pixtral", batch=8, prefix=16100, shared=0, groups=0, tree=1, page=64, layers=2,
             ragged=True, lse=False, given=False, dtype="bf16"),
        # eight questions about one long document: their trees over its pages and over some text of their own
        dict(name="attend_pixtral_b8_t60_shared", op="attend", shape="pixtral", batch=8, prefix=4347, shared=4096, groups=1, tree=60, page=64, layers=8,
             ragged=True, lse=True, given=False, dtype="bf16"),
        # the largest: 32 streams in four groups, each with images of its own, small pages
        dict(name="attend_smolvlm_b32_t33_groups", op="attend", shape="smolvlm", batch=32, prefix=1701, shared=1600, groups=4, tree=33, page=16, layers=6,
             ragged=True, lse=False, given=False, dtype="bf16"),
        # single tokens of a batch behind one long instruction, an odd number of rows of which are shared
        dict(name="attend_gemma3_b16_t1_shared", op="attend", shape="gemma3", batch=16, prefix=8250, shared=8011, groups=1, tree=1, page=128, layers=4,
             ragged=True, lse=False, given=False, dtype="bf16"),
        # one token over a very long context
        dict(name="sparse_pixtral_b1_t1_long", op="sparse", shape="pixtral", batch=1, prefix=131000, tree=1, page=64, first=1, last=2, best=32, layers=2,
             ragged=False, lse=False, given=False, dtype="bf16"),
        # trees of a serving batch over long contexts
        dict(name="sparse_pixtral_b8_t60", op="sparse", shape="pixtral", batch=8, prefix=16003, tree=60, page=64, first=1, last=2, best=16, layers=2,
             ragged=True, lse=False, given=False, dtype="bf16"),
        # wide heads, small pages, odd lengths
        dict(name="sparse_gemma3_b4_t33", op="sparse", shape="gemma3", batch=4, prefix=12011, tree=33, page=32, first=4, last=3, best=40, layers=2,
             ragged=True, lse=True, given=False, dtype="bf16"),
        # whole rounds: one sequence in many layers, and a batch of odd lengths
        dict(name="round_pixtral_b1_t60", op="round", shape="pixtral", batch=1, prefix=4100, tree=60, page=64, first=1, last=2, best=16, layers=20,
             ragged=False),
        dict(name="round_smolvlm_b4_t33", op="round", shape="smolvlm", batch=4, prefix=5001, tree=33, page=16, first=2, last=4, best=48, layers=6,
             ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "append", "attend", "attend", "attend", "attend", "sparse", "sparse", "sparse", "round"))
    shape = rng.choice(("llava", "pixtral", "gemma3", "smolvlm"))
    batch = _log(rng, 1, 32)
    page = rng.choice((16, 32, 64, 64, 128))
    if op == "append":
        tree = rng.random() < 0.5
        case = dict(op=op, shape=shape, batch=batch, rows=rng.randint(1, 64) if tree else _log(rng, 100, 4000), prefix=_log(rng, 1, 2000) if tree else 0,
                    page=page, layers=rng.randint(8, 32) if tree else 1, tree=tree, part=rng.choice((1, 1, 2, 4)), interleaved=rng.random() < 0.4,
                    scaling=rng.choice((1.0, 1.0, 4.0, 8.0)), bounds=not tree and rng.random() < 0.6, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
    elif op == "attend":
        if rng.random() < 0.12:
            shared = rng.choice((0, rng.randint(20, 300)))
            return dict(op=op, shape="tiny", batch=rng.randint(1, 6), prefix=shared + rng.randint(10, 600), shared=shared, groups=1 if shared else 0,
                        tree=rng.randint(1, 20), page=page, layers=1, ragged=True, lse=True, given=False, dtype="f32")
        tree = rng.choice((1, rng.randint(2, 64), rng.randint(8, 64), rng.randint(65, 100)))
        shared = _log(rng, 200, 16000 if tree == 1 else 6000) if rng.random() < 0.65 else 0
        case = dict(op=op, shape=shape, batch=batch, prefix=shared + _log(rng, 1, 700) if shared else _log(rng, 100, 20000 if tree == 1 else 4000),
                    shared=shared, groups=rng.randint(1, max(1, batch // 2)) if shared else 0, tree=tree, page=page, layers=rng.randint(2, 8),
                    ragged=rng.random() < 0.6, lse=rng.random() < 0.3, given=tree <= 64 and rng.random() < 0.2, dtype="bf16")
    else:
        tree = rng.choice((1, rng.randint(2, 64), rng.randint(8, 64))) if op == "sparse" else rng.randint(8, 64)
        first, last = rng.randint(0, 4), rng.randint(1, 4)
        case = dict(op=op, shape=shape, batch=batch if op == "sparse" else min(batch, 8), prefix=_log(rng, 500, 100000 if tree == 1 else 20000), tree=tree,
                    page=page, first=first, last=last, best=_log(rng, 4, 64), layers=rng.randint(2, 4) if op == "sparse" else rng.randint(4, 16),
                    ragged=rng.random() < 0.6)
        if op == "sparse":
            case.update(lse=rng.random() < 0.3, given=rng.random() < 0.2, dtype="bf16")
    while _cost(case) > 1.0:
        if case["layers"] > 1:
            case["layers"] -= 1
        elif case["batch"] > 1:
            case["batch"] = case["batch"] * 3 // 4
            case["groups"] = min(case["groups"], case["batch"]) if "groups" in case else 0
        elif "rows" in case:
            case["rows"] = case["rows"] * 3 // 4
        else:
            case["prefix"], case["shared"] = case["prefix"] * 3 // 4, case.get("shared", 0) * 3 // 4
    return case


def _cost(case):
    w = work(case)
    hq, hkv, d = SHAPES[case["shape"]]
    lengths, _, shared = _lengths(case)
    rows = sum(p + case.get("tree", 0) for p in lengths) - sum((n - 1) * s for n, s in shared) if case["op"] != "append" else \
        case["batch"] * (case["prefix"] + case["rows"])
    held = case["layers"] * rows * hkv * d * 4.0
    scores = 4.0 * case["batch"] * hq * case.get("tree", 0) * case["prefix"]      # of the plain forms
    return max(w["bytes"] / MAX_BYTES, w["flops"] / MAX_FLOPS, held / MAX_HELD, scores / 3.0e9)


# ---- sizes -----------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Prefix length of every sequence (the asked one, or what is its own spread over the upper half), first sequences of the groups, and (sequences,
    shared rows) of each."""
    r = random.Random("lengths %d %d" % (case["batch"], case["prefix"]))
    b, n = case["batch"], case.get("groups", 0)
    base = case.get("shared", 0)
    if case["op"] == "append" and not case["tree"]:
        return [case["prefix"]] * b, [], []
    own_rows = [case["prefix"] - base] * b
    if case.get("ragged"):
        own_rows = [own_rows[0] if i == 0 else r.randint(own_rows[0] // 2, own_rows[0]) for i in range(b)]
    starts = sorted([0] + r.sample(range(1, b), n - 1)) if n else []
    ends = starts[1:] + [b]
    shared = [(e - s, base if g == 0 else r.randint(base // 2, base)) for g, (s, e) in enumerate(zip(starts, ends))]
    of = [0] * b if not n else [shared[g][1] for g in range(n) for _ in range(shared[g][0])]
    return [x + s for x, s in zip(own_rows, of)], starts, shared


def _live(case):
    """Rows of an append that are no padding, of every sequence."""
    r = random.Random("live %d %d" % (case["batch"], case["rows"]))
    return [case["rows"] if case["tree"] or b == 0 else r.randint((case["rows"] + 1) // 2, case["rows"]) for b in range(case["batch"])]


def work(case):
    hq, hkv, d = SHAPES[case["shape"]]
    b, n, op, ps = case["batch"], case["layers"], case["op"], case["page"]
    e = 4 if case.get("dtype") == "f32" else 2
    if op == "append":
        rows = n * sum(_live(case))
        size = 2 * rows * (hq + 2 * hkv) * d * e
        if case["bounds"]:
            size += n * sum(-(-x // ps) for x in _live(case)) * hkv * 2 * d * e
        return dict(bytes=size, flops=3 * rows * (hq + hkv) * d // case["part"])
    t = case["tree"]
    lengths, _, shared = _lengths(case)
    if op == "attend":
        keys = sum(p + t for p in lengths)
        read = keys - sum((k - 1) * s for k, s in shared)
        size = n * (2 * read * hkv * d * e + 2 * b * t * hq * d * e + (b * hq * t * 4 if case["lse"] else 0))
        return dict(bytes=size, flops=n * 4 * keys * t * hq * d)
    pages = [-(-p // ps) for p in lengths]
    picked = [min(x, case["first"] + case["last"] + case["best"]) for x in pages]
    seen = [min(p, x * ps) + t for p, x in zip(lengths, picked)]      # keys a node sees, and the fewest that all nodes of a sequence together may
    size = n * (2 * sum(seen) * hkv * d * e + sum(pages) * hkv * (2 * d * e + 8 * ((t + 63) // 64)) + 2 * b * t * hq * d * e)
    if case.get("lse"):
        size += n * b * hq * t * 4
    flops = n * (4 * sum(seen) * t * hq * d + 4 * sum(pages) * t * hkv * d)
    if op == "round":      # half of the drafted depth is accepted on average; two pages get new bounds
        size += n * b * hkv * (4 * t * d * e + 4 * (1 + DEPTH // 2) * d * e + (ps + 2) * d * e)
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
    s = case.get("scaling", 1.0)
    if s > 1.0:
        turns = 4096.0 * f / (2.0 * math.pi)
        keep = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
        f = f * keep + f / s * (1.0 - keep)
    return torch.tensor(f.astype(np.float32), device="cuda"), (0.1 * math.log(s) + 1.0 if s > 1.0 else 1.0)


def _table(r, rows, page, starts=(), shared=()):
    """Pages of sequences that hold so many rows, as a pool that has served others gives them out: in no order, -1 behind the last.  Whole pages of a
    shared prefix are the same ones."""
    need = [-(-n // page) for n in rows]
    common = [0] * len(rows)
    first = list(range(len(rows)))
    for s, (n, length) in zip(starts, shared):
        for b in range(s, s + n):
            common[b], first[b] = length // page, s
    total = sum(n - (c if f != b else 0) for b, (n, c, f) in enumerate(zip(need, common, first)))
    ids = list(range(total + 3))
    r.shuffle(ids)
    table = np.full((len(rows), max(need) + 1), -1, dtype=np.int32)
    for b, n in enumerate(need):
        have = common[b] if first[b] != b else 0
        table[b, :have] = table[first[b], :have]
        table[b, have:n] = [ids.pop() for _ in range(n - have)]
    return _ints(table), total + 3


def _pools(rnd, dtype, layers, n, hkv, page, d):
    """Keys and values in pages.  Some channels of a key are larger than others, and the keys of a page have something in common."""
    k = torch.empty(layers, n, hkv, page, d, dtype=dtype, device="cuda")
    for l in range(layers):
        gain = torch.exp(0.5 * rnd.normal(hkv, 1, d, dtype=torch.float32))
        for h in range(hkv):
            k[l, :, h] = (rnd.normal(n, page, d, dtype=torch.float32) + 0.7 * rnd.normal(n, 1, d, dtype=torch.float32)) * gain[h]
    return k, rnd.normal(layers, n, hkv, page, d, dtype=dtype)


def _queries(rnd, dtype, layers, b, t, hq, d):
    """The nodes of a tree ask much the same."""
    q = torch.empty(layers, b, t, hq, d, dtype=dtype, device="cuda")
    for l in range(layers):
        q[l] = 0.5 * rnd.normal(b, t, hq, d, dtype=torch.float32) + 0.8 * rnd.normal(b, 1, hq, d, dtype=torch.float32)
    return q


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


def _prepare_append(case, rnd, r):
    hq, hkv, d = SHAPES[case["shape"]]
    b, n, layers, dt, ps = case["batch"], case["rows"], case["layers"], _type(case), case["page"]
    live = _live(case)
    table, n_pages = _table(r, [case["prefix"] + x for x in live], ps)
    rot = d // case["part"]
    freq, amplitude = _frequencies(case, rot)
    s = dict(hkv=hkv, n=n, page=ps, rot=rot, interleaved=case["interleaved"], freq=freq, amplitude=amplitude, layers=layers, table=table,
             live=None if case["tree"] else _ints(live), base=_ints([case["prefix"]] * b), parent=_ints([_tree(r, n) for _ in range(b)]) if case["tree"] else None,
             q=rnd.normal(layers, b, n, hq, d, dtype=dt), k=rnd.normal(layers, b, n, hkv, d, dtype=dt), v=rnd.normal(layers, b, n, hkv, d, dtype=dt),
             q_out=torch.zeros(layers, b, n, hq, d, dtype=dt, device="cuda"), k_pages=torch.zeros(layers, n_pages, hkv, ps, d, dtype=dt, device="cuda"),
             v_pages=torch.zeros(layers, n_pages, hkv, ps, d, dtype=dt, device="cuda"),
             bounds=torch.zeros(layers, n_pages, hkv, 2, d, dtype=dt, device="cuda") if case["bounds"] else None, to=_ints([case["prefix"] + x for x in live]))
    if own:
        import paper_2505_19201_amd as dream
        s["desc"] = dream.attn_desc(b, hq, hkv, d, dream.F32 if dt == torch.float32 else dream.BF16, 0)
        s["pages"] = dream.page_desc(ps, n_pages, table.shape[1])
        s["calls"] = [[s[x][l] for x in ("q", "k", "v", "q_out", "k_pages", "v_pages")] for l in range(layers)]
    return s


def _prepare_attention(case, rnd, r):
    hq, hkv, d = SHAPES[case["shape"]]
    b, t, layers, dt, ps = case["batch"], case["tree"], case["layers"], _type(case), case["page"]
    lengths, starts, shared = _lengths(case)
    table, n_pages = _table(r, [p + t for p in lengths], ps, starts, shared)
    parent = [_tree(r, t) for _ in range(b)]
    s = dict(op=case["op"], layers=layers, tree=t, page=ps, max_kv=max(lengths) + t, table=table, prefix_len=_ints(lengths), parent=_ints(parent),
             starts=_ints(starts + [b]) if starts else None, shared=_ints([x for _, x in shared]) if starts else None, groups=len(starts),
             max_shared=max([x for _, x in shared], default=0), mask=_given_mask(r, parent) if case.get("given") else None,
             q=_queries(rnd, dt, layers, b, t, hq, d), out=torch.empty(layers, b, t, hq, d, dtype=dt, device="cuda"),
             lse=torch.empty(layers, b, hq, t, device="cuda") if case.get("lse") else None)
    s["k_pages"], s["v_pages"] = _pools(rnd, dt, layers, n_pages, hkv, ps, d)
    if case["op"] != "attend":
        s.update(first=case["first"], last=case["last"], best=case["best"],
                 nodes=torch.empty(layers, b, hkv, table.shape[1], (t + 63) // 64, dtype=torch.int64, device="cuda"))
        s["bounds"] = torch.stack([s["k_pages"].amax(3), s["k_pages"].amin(3)], 3)      # (whole pages: rows to come are inputs like any other here)
    if case["op"] == "round":
        freq, amplitude = _frequencies(case, d)
        paths = [_path(r, p) for p in parent]
        s.update(k_rows=rnd.normal(layers, b, t, hkv, d, dtype=dt), v_rows=rnd.normal(layers, b, t, hkv, d, dtype=dt), freq=freq, rot=d,
                 path=_ints([p + [-1] * (DEPTH + 1 - len(p)) for p in paths]), length=_ints([len(p) - 1 for p in paths]),
                 new_len=torch.empty(b, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2505_19201_amd as dream
        s["desc"] = dream.attn_desc(b, hq, hkv, d, dream.F32 if dt == torch.float32 else dream.BF16, 0)
        s["pages"] = dream.page_desc(ps, n_pages, table.shape[1])
        if case["op"] == "attend":
            size = dream.dream_paged_verify_attn_workspace(s["desc"], s["pages"], t, s["max_kv"], s["groups"], s["max_shared"])
        else:
            size = max(dream.dream_page_select_workspace(s["desc"], s["pages"], t, s["max_kv"]),
                       dream.dream_sparse_verify_attn_workspace(s["desc"], s["pages"], t, s["max_kv"], s["first"] + s["last"] + s["best"]))
        s["ws"] = dream.alloc_workspace(size)
        s["calls"] = [[s["q"][l], s["k_pages"][l], s["v_pages"][l], s["out"][l], None if s["lse"] is None else s["lse"][l]] +
                      ([s["bounds"][l], s["nodes"][l]] if "bounds" in s else []) for l in range(layers)]
        if case["op"] == "round":
            s["rows"] = [(s["k_rows"][l], s["v_rows"][l]) for l in range(layers)]
            s["each"] = [*s["k_pages"], *s["v_pages"]]
    return s


def prepare(case, seed):
    if own:
        import paper_2505_19201_amd as dream
        dream.load()
        dream.dream_init()
    make = _prepare_append if case["op"] == "append" else _prepare_attention
    return case["op"], make(case, _Rand(seed), random.Random(seed))


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _own_append(s):
    import paper_2505_19201_amd as dream
    for l, (q, k, v, q_out, k_pages, v_pages) in enumerate(s["calls"]):
        dream.dream_paged_append(s["desc"], s["pages"], s["table"], q, k, v, s["n"], s["base"], None, s["live"], None, None, s["parent"], s["freq"], s["rot"],
                                 s["interleaved"], s["amplitude"], q_out, k_pages, v_pages)
        if s["bounds"] is not None:
            dream.dream_page_bounds(s["desc"], s["pages"], s["table"], k_pages, s["base"], s["to"], s["n"], s["bounds"][l])
    return [s["q_out"], s["k_pages"], s["v_pages"], s["bounds"]]


def _own_attend(s):
    import paper_2505_19201_amd as dream
    for q, k, v, out, lse in s["calls"]:
        dream.dream_paged_verify_attn(s["desc"], s["pages"], q, k, v, s["table"], s["prefix_len"], s["tree"], s["parent"], s["mask"], s["groups"], s["starts"],
                                      s["shared"], s["max_shared"], s["max_kv"], out, lse, s["ws"])
    return [s["out"], s["lse"]]


def _select_and_attend(dream, s, q, k, v, out, lse, bounds, nodes):
    dream.dream_page_select(s["desc"], s["pages"], s["table"], q, bounds, s["prefix_len"], s["tree"], s["first"], s["last"], s["best"], s["max_kv"], nodes,
                            s["ws"])
    dream.dream_sparse_verify_attn(s["desc"], s["pages"], q, k, v, s["table"], nodes, s["prefix_len"], s["tree"], s["parent"], s["mask"], s["max_kv"],
                                   s["first"] + s["last"] + s["best"], out, lse, s["ws"])


def _own_sparse(s):
    import paper_2505_19201_amd as dream
    for call in s["calls"]:
        _select_and_attend(dream, s, *call)
    return [s["nodes"], s["out"], s["lse"]]


def _own_round(s):
    import paper_2505_19201_amd as dream
    for (k, v), call in zip(s["rows"], s["calls"]):
        dream.dream_paged_append(s["desc"], s["pages"], s["table"], None, k, v, s["tree"], s["prefix_len"], None, None, None, None, s["parent"], s["freq"],
                                 s["rot"], False, 1.0, None, call[1], call[2])
        _select_and_attend(dream, s, *call)
    dream.dream_paged_commit(s["desc"], s["pages"], s["table"], s["each"], s["prefix_len"], s["tree"], s["path"], s["length"], s["new_len"])
    for _, k, _, _, _, bounds, _ in s["calls"]:
        dream.dream_page_bounds(s["desc"], s["pages"], s["table"], k, s["prefix_len"], s["new_len"], DEPTH + 1, bounds)
    return [s["nodes"], s["out"], s["new_len"], s["k_pages"], s["v_pages"], s["bounds"]]


# ---- plain forms -----------------------------------------------------------------------------------------------------
def _ancestors(parent):
    """[B, T, T]: node a is node i or an ancestor of it; and the depths."""
    b, t = parent.shape
    reach = torch.eye(t, device=parent.device).expand(b, t, t).clone()
    child = (parent >= 0).nonzero()
    reach[child[:, 0], child[:, 1], parent[child[:, 0], child[:, 1]].long()] = 1.0
    for _ in range(max(1, t - 1).bit_length()):
        reach = (torch.matmul(reach, reach) > 0).float()
    return reach > 0, reach.sum(-1).long() - 1


def _rotation(base, parent, n, freq, amplitude):
    step = torch.arange(n, device="cuda").expand(base.shape[0], n) if parent is None else _ancestors(parent)[1]
    angle = (base.long().unsqueeze(1) + step).double().unsqueeze(-1) * freq.double()     # far positions: angles in 64 bits
    return (angle.cos() * amplitude).float().unsqueeze(2), (angle.sin() * amplitude).float().unsqueeze(2)


def _turn(x, cos, sin, rot, interleaved):
    y, half = x.float(), rot // 2
    a, c = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :half], y[..., half:rot])
    u, w = a * cos - c * sin, a * sin + c * cos
    z = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([z, y[..., rot:]], -1).to(x.dtype)


def _places(table, page, rows):
    """Page and row in it of rows [B, N] of the sequences."""
    return table.gather(1, rows // page).long(), rows % page


def _page_bounds(k_pages, table, page, start, end, bounds):
    """Of the pages that rows start .. end - 1 lie in, over the rows in front of `end`."""
    index = torch.arange(table.shape[1], device="cuda").unsqueeze(0)
    b, i = ((index >= (start // page).unsqueeze(1)) & (index * page < end.unsqueeze(1)) & (end > start).unsqueeze(1)).nonzero(as_tuple=True)
    rows = k_pages[table[b, i].long()]
    live = (i * page).unsqueeze(1) + torch.arange(page, device="cuda") < end[b].unsqueeze(1)
    live = live[:, None, :, None]
    inf = torch.full((), float("inf"), device="cuda", dtype=rows.dtype)
    bounds[table[b, i].long()] = torch.stack([torch.where(live, rows, -inf).amax(2), torch.where(live, rows, inf).amin(2)], 2)


def _plain_append(s):
    n = s["n"]
    cos, sin = _rotation(s["base"], s["parent"], n, s["freq"], s["amplitude"])
    step = torch.arange(n, device="cuda")
    live = torch.ones(s["base"].shape[0], n, dtype=torch.bool, device="cuda") if s["live"] is None else step < s["live"].unsqueeze(1)
    who, which = live.nonzero(as_tuple=True)
    at = s["base"].long()[who] + which
    page, row = s["table"][who, at // s["page"]].long(), at % s["page"]
    for l in range(s["layers"]):
        s["q_out"][l, who, which] = _turn(s["q"][l], cos, sin, s["rot"], s["interleaved"])[who, which]
        s["k_pages"][l, page, :, row] = _turn(s["k"][l], cos, sin, s["rot"], s["interleaved"])[who, which]
        s["v_pages"][l, page, :, row] = s["v"][l, who, which]
        if s["bounds"] is not None:
            _page_bounds(s["k_pages"][l], s["table"], s["page"], s["base"], s["to"], s["bounds"][l])
    return [s["q_out"], s["k_pages"], s["v_pages"], s["bounds"]]


def _sources(s):
    """[B, S]: the page of every position of a sequence; a shared one is the group's first sequence's."""
    n = -(-s["max_kv"] // s["page"]) * s["page"]
    b = s["table"].shape[0]
    at = torch.arange(n, device="cuda")
    who = torch.arange(b, device="cuda").unsqueeze(1).expand(b, n).clone()
    for g in range(s["groups"]):
        lo, hi = s["starts"][g], s["starts"][g + 1]
        row = torch.arange(b, device="cuda").unsqueeze(1)
        who = torch.where((row >= lo) & (row < hi) & (at < s["shared"][g]), lo.long(), who)
    return s["table"][who, (at // s["page"]).expand(b, n)].clamp(min=0).long(), at % s["page"]


def _visible(s):
    """[B, T, S]: which keys a node sees."""
    t = s["tree"]
    p = s["prefix_len"].long().view(-1, 1, 1)
    b = p.shape[0]
    n = -(-s["max_kv"] // s["page"]) * s["page"]
    reach = _ancestors(s["parent"])[0]
    if s["mask"] is not None:
        reach = (s["mask"] >> torch.arange(t, device="cuda")) & 1 > 0
    key = torch.arange(n, device="cuda").view(1, 1, -1)
    rel = (key - p).clamp(0, t - 1).expand(b, t, n)
    return key < p, (key >= p) & (key < p + t) & reach.gather(2, rel)


def _attend(q, k, v, vis):
    """softmax(q k^T / sqrt(D)) v over visible keys ([B, Hkv or 1, T, S]), in float32: rows [B, T, Hq, D] and log-sum-exps [B, Hq, T]."""
    b, t, hq, d = q.shape
    hkv, g = k.shape[1], q.shape[2] // k.shape[1]
    x = q.float().view(b, t, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, g * t, d)
    x = torch.matmul(x, k.float().transpose(2, 3)).mul_(d ** -0.5).view(b, hkv, g, t, -1)
    x.masked_fill_(~vis.unsqueeze(2), float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(b, hkv, g * t, -1), v.float()).view(b, hkv, g, t, d) / total.clamp(min=1e-38)
    return o.permute(0, 3, 1, 2, 4).reshape(b, t, hq, d), (top + total.log()).reshape(b, hq, t)


def _layer(s, l, page, row, vis):
    k, v = (s[x][l][page, :, row].transpose(1, 2) for x in ("k_pages", "v_pages"))      # [B, Hkv, S, D]
    o, lse = _attend(s["q"][l], k, v, vis)
    s["out"][l] = o.to(s["q"].dtype)
    if s["lse"] is not None:
        s["lse"][l] = lse


def _plain_attend(s):
    page, row = _sources(s)
    row = row.expand_as(page)
    prefix, tree = _visible(s)
    for l in range(s["layers"]):
        _layer(s, l, page, row, (prefix | tree).unsqueeze(1))
    return [s["out"], s["lse"]]


def _exponent(top):
    """The least whole e in [-100, 121] with top <= 127 * 2^e."""
    return (((top.float().view(torch.int32) + 0x1FFFF) >> 23) - 133).clamp(-100, 121)


def _scale(e):
    """2^e in float32, |e| <= 121."""
    return ((e + 127) << 23).view(torch.float32)


def _choose(s, l):
    """[B, Hkv, T, max_pages]: the pages a node sees."""
    q, t = s["q"][l].float(), s["tree"]
    b, _, hq, d = q.shape
    hkv = s["bounds"].shape[2]
    q = q.view(b, t, hkv, hq // hkv, d).transpose(1, 2)
    q = torch.round(q * _scale(-_exponent(q.abs().amax((-1, -2))))[..., None, None])
    x = s["bounds"][l][s["table"].clamp(min=0).long()].float().permute(0, 2, 1, 3, 4)      # [B, Hkv, pages, 2, D]
    e = _exponent(x.abs().amax((-1, -2)))
    x = x * _scale(-e)[..., None, None]
    upper, lower = torch.ceil(x[..., 0, :]), torch.floor(x[..., 1, :])
    # sums of whole numbers: exact in 64 bits
    score = torch.matmul(q.clamp(min=0).sum(3).double(), upper.double().transpose(2, 3).contiguous()) + \
        torch.matmul(q.clamp(max=0).sum(3).double(), lower.double().transpose(2, 3).contiguous())
    score = score.float() * _scale(e).unsqueeze(2)
    index = torch.arange(score.shape[-1], device="cuda")
    n = ((s["prefix_len"] + s["page"] - 1) // s["page"]).view(b, 1, 1, 1)
    always = ((index < s["first"]) | (index >= n - s["last"])) & (index < n)
    between = (index < n) & ~always
    order = torch.where(between, score, torch.full_like(score, float("-inf"))).sort(dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(-1, order, index.expand_as(order))
    return (between & (rank < s["best"])) | always.expand_as(between)


def _words(picked):
    """[B, Hkv, pages, words]: bit i % 64 of word i / 64 is node i's."""
    bits = torch.nn.functional.pad(picked.transpose(2, 3).long(), (0, -picked.shape[2] % 64)).unflatten(-1, (-1, 64))
    return (bits << torch.arange(64, device="cuda")).sum(-1)


def _sparse_layer(s, l, page, row, prefix, tree):
    picked = _choose(s, l)
    s["nodes"][l] = _words(picked)
    n = page.shape[1] // s["page"]
    _layer(s, l, page, row, (picked[..., :n].repeat_interleave(s["page"], -1) & prefix.unsqueeze(1)) | tree.unsqueeze(1))


def _plain_sparse(s):
    page, row = _sources(s)
    row = row.expand_as(page)
    prefix, tree = _visible(s)
    for l in range(s["layers"]):
        _sparse_layer(s, l, page, row, prefix, tree)
    return [s["nodes"], s["out"], s["lse"]]


def _plain_round(s):
    t, p = s["tree"], s["prefix_len"].long()
    step = torch.arange(t, device="cuda")
    new_page, new_row = _places(s["table"], s["page"], p.unsqueeze(1) + step)
    cos, sin = _rotation(s["prefix_len"], s["parent"], t, s["freq"], 1.0)
    page, row = _sources(s)
    row = row.expand_as(page)
    prefix, tree = _visible(s)
    for l in range(s["layers"]):
        s["k_pages"][l][new_page, :, new_row] = _turn(s["k_rows"][l], cos, sin, s["rot"], False)
        s["v_pages"][l][new_page, :, new_row] = s["v_rows"][l]
        _sparse_layer(s, l, page, row, prefix, tree)
    # rows of the path move up; entries behind its end stay where they are
    step = torch.arange(s["path"].shape[1], device="cuda")[None, :t]
    source = torch.where(step <= s["length"].unsqueeze(1), s["path"][:, :t], step).long()
    from_page, from_row = _places(s["table"], s["page"], p.unsqueeze(1) + source)
    to_page, to_row = _places(s["table"], s["page"], p.unsqueeze(1) + step)
    s["new_len"].copy_(s["prefix_len"] + s["length"] + 1)
    for l in range(s["layers"]):
        for c in (s["k_pages"][l], s["v_pages"][l]):
            c[to_page, :, to_row] = c[from_page, :, from_row]
        _page_bounds(s["k_pages"][l], s["table"], s["page"], s["prefix_len"], s["new_len"], s["bounds"][l])
    return [s["nodes"], s["out"], s["new_len"], s["k_pages"], s["v_pages"], s["bounds"]]


_PLAIN = dict(append=_plain_append, attend=_plain_attend, sparse=_plain_sparse, round=_plain_round)
_OWN = dict(append=_own_append, attend=_own_attend, sparse=_own_sparse, round=_own_round)


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


def _exact_turn(x, pos, freq, rot, interleaved, amplitude):
    phase = torch.tensor(pos, dtype=torch.float64, device="cuda")[:, :, None, None] * freq.double()
    unit = torch.polar(torch.full_like(phase, amplitude), phase)
    y = x.double()
    pair = y[..., :rot].unflatten(-1, (rot // 2, 2)) if interleaved else y[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * unit)
    y[..., :rot] = (z if interleaved else z.transpose(-1, -2)).flatten(-2)
    return y


def _exact_bounds(pages, table, size, start, end, bounds):
    for b, row in enumerate(table):
        for i in range(start[b] // size, -(-end[b] // size)):
            rows = pages[row[i], :, :min(size, end[b] - i * size)]
            bounds[row[i], :, 0], bounds[row[i], :, 1] = rows.max(1)[0], rows.min(1)[0]


def _exact_append(s):
    walk = None if s["parent"] is None else _walk(s["parent"])
    n, size = s["n"], s["page"]
    base, table = s["base"].tolist(), s["table"].tolist()
    live = [n] * len(base) if s["live"] is None else s["live"].tolist()
    pos = [[p + (i if walk is None else len(walk[j][i]) - 1) for i in range(n)] for j, p in enumerate(base)]
    out = [s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double(), None if s["bounds"] is None else s["bounds"].double()]
    for l in range(s["layers"]):
        q, k = (_exact_turn(s[x][l], pos, s["freq"], s["rot"], s["interleaved"], s["amplitude"]) for x in ("q", "k"))
        for b, p in enumerate(base):
            out[0][l, b, :live[b]] = q[b, :live[b]]
            for i in range(p // size, -(-(p + live[b]) // size)):
                lo, hi = max(p, i * size), min(p + live[b], (i + 1) * size)
                out[1][l, table[b][i], :, lo - i * size:hi - i * size] = k[b, lo - p:hi - p].transpose(0, 1)
                out[2][l, table[b][i], :, lo - i * size:hi - i * size] = s["v"][l, b, lo - p:hi - p].double().transpose(0, 1)
        if out[3] is not None:
            _exact_bounds(out[1][l], table, size, base, [p + x for p, x in zip(base, live)], out[3][l])
    return out


def _least_power(top):
    """Least whole e in [-100, 121] with top <= 127 * 2^e, of numpy arrays in 64 bits."""
    m, e = np.frexp(top / 127.0)
    return np.where(top > 0, np.clip(e - (m == 0.5), -100, 121), -100)


def _exact_choice(s, l, b, walk_len, table):
    """[Hkv, T, pages] of one sequence."""
    pages = -(-walk_len // s["page"])
    x = s["bounds"][l][table[:pages]].double().cpu().numpy()                       # [pages, Hkv, 2, D]
    q = s["q"][l, b].double().cpu().numpy()
    t, hq, d = q.shape
    hkv = x.shape[1]
    q = q.reshape(t, hkv, hq // hkv, d)
    q = np.rint(np.ldexp(q, -_least_power(np.abs(q).max((2, 3)))[:, :, None, None]))
    e = _least_power(np.abs(x).max((2, 3)) if pages else np.zeros((0, hkv)))      # [pages, Hkv]
    x = np.ldexp(x, -e[:, :, None, None])
    score = np.einsum("tkd,pkd->ktp", np.maximum(q, 0).sum(2), np.ceil(x[:, :, 0])) + np.einsum("tkd,pkd->ktp", np.minimum(q, 0).sum(2), np.floor(x[:, :, 1]))
    score = np.ldexp(score.astype(np.float32).astype(np.float64), e.T[:, None, :])
    picked = np.zeros((hkv, t, pages), dtype=bool)
    picked[:, :, :s["first"]] = True
    picked[:, :, max(0, pages - s["last"]):] = True
    lo, hi = min(s["first"], pages), max(0, pages - s["last"])
    if hi > lo:
        order = np.argsort(-score[:, :, lo:hi], axis=-1, kind="stable")[:, :, :s["best"]] + lo
        np.put_along_axis(picked, order, True, -1)
    return picked


def _exact_attention(s, k_pages, v_pages):
    """k_pages(l), v_pages(l): the pages of a layer in 64 bits."""
    walk, table, size, t, d = _walk(s["parent"]), s["table"].tolist(), s["page"], s["tree"], s["q"].shape[-1]
    lengths = s["prefix_len"].tolist()
    given = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint64)
    origin, until = list(range(len(lengths))), [0] * len(lengths)
    for g in range(s["groups"]):
        for b in range(int(s["starts"][g]), int(s["starts"][g + 1])):
            origin[b], until[b] = int(s["starts"][g]), int(s["shared"][g])
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = None if s["lse"] is None else torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    nodes = torch.zeros_like(s["nodes"]) if "nodes" in s else None
    for l in range(s["layers"]):
        pools = [k_pages(l), v_pages(l)]
        for b, p in enumerate(lengths):
            live = p + t
            pages = -(-live // size)
            seen = np.zeros((1 if nodes is None else pools[0].shape[1], t, pages * size), dtype=bool)
            if nodes is None:
                seen[:, :, :p] = True
            else:
                picked = _exact_choice(s, l, b, p, table[b])
                seen[:, :, :picked.shape[2] * size] = np.repeat(picked, size, -1)
                seen[:, :, p:] = False
                word = np.zeros(picked.shape[::2] + (nodes.shape[-1],), dtype=np.uint64)      # [Hkv, pages, words]
                for i in range(t):
                    word[:, :, i // 64] |= picked[:, i].astype(np.uint64) << np.uint64(i % 64)
                nodes[l, b, :, :picked.shape[2]] = torch.tensor(word.view(np.int64), device="cuda")
            for i, path in enumerate(walk[b]):
                of = path if given is None else [a for a in range(t) if int(given[b, i, 0]) >> a & 1]
                seen[:, i, [p + a for a in of]] = True
            seen = torch.tensor(seen[:, :, :live], device="cuda")
            split = min(until[b], p)
            k, v = [], []
            for x, pool in ((k, pools[0]), (v, pools[1])):
                mine = pool[table[b][:pages]].transpose(0, 1).flatten(1, 2)[:, :live].double()
                if split and origin[b] != b:
                    theirs = pool[table[origin[b]][:-(-split // size)]].transpose(0, 1).flatten(1, 2).double()
                    mine = torch.cat([theirs[:, :split], mine[:, split:]], 1)
                x.append(mine)
            q = s["q"][l, b].double().transpose(0, 1)                      # [Hq, T, D]
            group = q.shape[0] // k[0].shape[0]
            for h in range(k[0].shape[0]):
                rows = q[h * group:(h + 1) * group].reshape(group * t, d)
                can = seen[h % seen.shape[0]].repeat(group, 1)
                x = torch.mm(rows, k[0][h].t()) / math.sqrt(d)
                x = torch.where(can, x, torch.full_like(x, float("-inf")))
                total = torch.logsumexp(x, -1)
                x = torch.where(can, torch.exp(x - total.unsqueeze(-1)), torch.zeros_like(x))
                out[l, b, :, h * group:(h + 1) * group] = torch.mm(x, v[0][h]).view(group, t, d).transpose(0, 1)
                if lse is not None:
                    lse[l, b, h * group:(h + 1) * group] = total.view(group, t)
    return nodes, out, lse


def _exact_round(s):
    walk, t, size = _walk(s["parent"]), s["tree"], s["page"]
    lengths, table, paths, accepted = s["prefix_len"].tolist(), s["table"].tolist(), s["path"].tolist(), s["length"].tolist()
    pos = [[p + len(w) - 1 for w in walk[b]] for b, p in enumerate(lengths)]
    k, v, bounds = s["k_pages"].double(), s["v_pages"].double(), s["bounds"].double()
    new = [p + n + 1 for p, n in zip(lengths, accepted)]
    for l in range(s["layers"]):
        turned = _exact_turn(s["k_rows"][l], pos, s["freq"], s["rot"], False, 1.0).to(s["q"].dtype).double()      # a cache's rows are of its type
        for b, p in enumerate(lengths):
            for i in range(t):
                k[l, table[b][(p + i) // size], :, (p + i) % size] = turned[b, i]
                v[l, table[b][(p + i) // size], :, (p + i) % size] = s["v_rows"][l, b, i].double()
    nodes, out, _ = _exact_attention(s, lambda l: k[l], lambda l: v[l])
    for b, p in enumerate(lengths):
        at = [(table[b][(p + i) // size], (p + i) % size) for i in range(t)]
        for pool in (k, v):
            old = [pool[:, page, :, row].clone() for page, row in at]
            for j in range(accepted[b] + 1):
                pool[:, at[j][0], :, at[j][1]] = old[paths[b][j]]
    for l in range(s["layers"]):
        _exact_bounds(k[l], table, size, lengths, new, bounds[l])
    return [nodes, out, torch.tensor(new, device="cuda"), k, v, bounds]


def exact(case, seed):
    global own
    held, own = own, False
    try:
        op, s = prepare(case, seed)
    finally:
        own = held
    if op == "append":
        return _exact_append(s)
    if op == "round":
        return _exact_round(s)
    nodes, out, lse = _exact_attention(s, lambda l: s["k_pages"][l], lambda l: s["v_pages"][l])
    return [out, lse] if op == "attend" else [nodes, out, lse]
