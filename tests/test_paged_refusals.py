"""No-GPU checks of what the calls for caches in pages refuse before anything is launched, at the limits that include/dream.h states, and of the definitions that the GPU tests compare with."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from paper_2505_19201_amd import build as dream_build
from tests import paged_cases as pc
from tests import window_cases as wc
from tests.test_abi import _signature
from tests.test_operator_limits import _constant, _text
from tests.test_operator_refusals import FAKE, ODD, _desc

CALLS = ["dream_paged_append", "dream_paged_commit", "dream_paged_verify_attn", "dream_page_bounds", "dream_page_select", "dream_sparse_verify_attn"]
# arguments that may be left out
OPTIONAL = {"dream_paged_append": {"row_index", "n_live", "pos", "pos_base", "parent", "inv_freq"}, "dream_paged_commit": {"prefix_len_out"},
            "dream_paged_verify_attn": {"tree_mask", "lse", "parent"}, "dream_page_bounds": {"from_len"}, "dream_page_select": set(),
            "dream_sparse_verify_attn": {"tree_mask", "lse", "parent"}}
# arguments that have to be 16-byte aligned
ALIGNED = {"dream_paged_append": ["q", "k", "v", "q_out", "k_pages", "v_pages"], "dream_paged_commit": [], "dream_page_bounds": ["k_pages", "bounds"],
           "dream_page_select": ["q", "bounds", "workspace"], "dream_paged_verify_attn": ["q", "k_pages", "v_pages", "out", "workspace"],
           "dream_sparse_verify_attn": ["q", "k_pages", "v_pages", "out", "workspace"]}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dream.library_path()):
        dream_build.build(verbose=False)
    return dream.load()


def _far(i):      # pointers whose tensors do not meet
    return C.c_void_p((i + 1) << 44)


@pytest.fixture
def call(lib, request):
    """Calls an entry point by its parameters' names; pointers are far apart from each other, and never followed: the calls below fail before a launch."""
    name = request.param
    defaults = dict(desc=_desc(), pages=dream.page_desc(64, 40, 20), n_rows=10, rot_dim=64, interleaved=0, amplitude=1.0, n_tree=20, path_stride=7, n_groups=0, max_shared_len=0,
                    max_kv_len=500, max_new=10, n_first=1, n_last=1, n_best=4, max_pages_seen=0, workspace_bytes=1 << 40, n_pools=3,
                    pools_host=(C.c_void_p * 3)(0x1000, 0x2000, 0x3000))

    def do(**kw):
        args = []
        for i, (kind, param) in enumerate(_signature(name)):
            v = kw[param] if param in kw else defaults.get(param, _far(i) if "*" in kind else 1)
            if isinstance(v, (dream.AttnDesc, dream.PageDesc)):
                v = C.byref(v)
            elif isinstance(v, (int, float)) and v is not None:
                v = C.c_float(v) if "float" in kind else C.c_size_t(v) if "size_t" in kind else C.c_int64(v) if "int64" in kind else C.c_int32(v)
            args.append(v)
        return getattr(lib, name)(*args)
    do.name = name
    return do


every = pytest.mark.parametrize("call", CALLS, indirect=True)


@every
def test_arguments(call):
    wrong = [dict(desc=None), dict(pages=None), dict(desc=_desc(dtype=3)), dict(desc=_desc(batch=0)), dict(desc=_desc(n_q_heads=7)), dict(desc=_desc(n_kv_heads=0)),
             dict(desc=_desc(n_q_heads=0)), dict(pages=dream.page_desc(64, 0, 20)), dict(pages=dream.page_desc(64, 40, 0))]
    for kind, param in _signature(call.name):
        if "*" in kind and param not in OPTIONAL[call.name] | {"stream", "group_start", "shared_len"}:
            wrong.append({param: None})
    wrong += [{param: ODD} for param in ALIGNED[call.name]]
    wrong += {"dream_paged_append": [dict(n_rows=0), dict(n_rows=(1 << 19) + 1), dict(q_out=None), dict(rot_dim=0), dict(rot_dim=5), dict(rot_dim=130), dict(rot_dim=-2)],
              "dream_paged_commit": [dict(n_pools=0), dict(n_tree=0), dict(path_stride=0), dict(pools_host=(C.c_void_p * 3)(0x1000, None, 0x2000)),
                                     dict(pools_host=(C.c_void_p * 3)(0x1000, 0x2008, 0x3000)), dict(prefix_len=FAKE, prefix_len_out=FAKE), dict(accept_len=FAKE, prefix_len_out=FAKE)],
              "dream_page_bounds": [dict(max_new=0), dict(max_new=-3)],
              "dream_page_select": [dict(n_tree=0), dict(n_tree=257), dict(n_first=-1), dict(n_last=-1), dict(n_best=-1), dict(max_kv_len=19)],
              "dream_paged_verify_attn": [dict(n_tree=0), dict(n_tree=257), dict(parent=None, tree_mask=None), dict(n_groups=-1), dict(n_groups=3), dict(n_groups=1, group_start=None),
                                          dict(n_groups=1, shared_len=None)],
              "dream_sparse_verify_attn": [dict(n_tree=0), dict(n_tree=257), dict(parent=None, tree_mask=None)]}[call.name]
    for kw in wrong:
        assert call(**kw) == -1, kw
        assert dream.dream_last_error().startswith(call.name), kw


# a call that is wrong in its last check too, so that what is allowed does not launch either
LAST = {"dream_paged_append": dict(q_out=ODD), "dream_paged_commit": dict(path_stride=0), "dream_paged_verify_attn": dict(out=ODD), "dream_page_bounds": dict(bounds=ODD),
        "dream_page_select": dict(q=ODD), "dream_sparse_verify_attn": dict(out=ODD)}


@every
def test_limits(call):
    text, last = _text(), LAST[call.name]
    assert "page_size is 16, 32, 64, 128 or 256; max_pages * page_size is at most DREAM_MAX_WINDOW_ROWS, batch at most 65535" in text and "n_q_heads and n_kv_heads at most 4096, D in {64, 128, 256}" in text
    rows = _constant("DREAM_MAX_WINDOW_ROWS")
    for ps in (16, 32, 64, 128, 256):
        assert call(pages=dream.page_desc(ps, 40, rows // ps), **last) == -1
        assert call(pages=dream.page_desc(ps, 40, rows // ps + 1), **last) == -2
    for ps in (0, -16, 8, 48, 100, 512):
        assert call(pages=dream.page_desc(ps, 40, 20), **last) == -2
    for D in (64, 128, 256):
        assert call(desc=_desc(head_dim=D), rot_dim=D, **last) == -1
    for D in (0, 32, 96, 512):
        assert call(desc=_desc(head_dim=D), **last) == -2
    few = dict(desc=_desc(batch=65535, n_q_heads=2), n_rows=1, n_tree=1)
    assert call(**few, **last) == -1
    said = dream.dream_last_error()
    assert call(**dict(few, desc=_desc(batch=65536, n_q_heads=2)), **last) == -1
    assert "batch 65536" in dream.dream_last_error() and "batch" not in said
    assert call(desc=_desc(n_q_heads=4096, n_kv_heads=128), **last) == -1
    said = dream.dream_last_error()
    assert call(desc=_desc(n_q_heads=4097, n_kv_heads=1), **last) == -1
    assert "4097 query heads" in dream.dream_last_error() and "query heads" not in said


@pytest.mark.parametrize("call", ["dream_paged_verify_attn", "dream_sparse_verify_attn", "dream_page_select"], indirect=True)
def test_limits_of_attention(call):
    last = LAST[call.name]
    if call.name == "dream_page_select":
        assert "Hq / Hkv at most 64" in _text()
        assert call(desc=_desc(n_q_heads=128), **last) == -1
        assert call(desc=_desc(n_q_heads=130), **last) == -2
    else:
        assert "batch * n_q_heads at most 2^20" in _text()
        assert call(desc=_desc(batch=1 << 15, n_q_heads=32), **last) == -1
        assert call(desc=_desc(batch=1 << 15, n_q_heads=34), **last) == -2
    short = dream.page_desc(16, 40, 1)
    assert call(pages=short, n_tree=16, **last) == -1 and "n_tree" not in dream.dream_last_error()
    assert call(pages=short, n_tree=17, **last) == -1 and "n_tree 17" in dream.dream_last_error()


@pytest.mark.parametrize("call", ["dream_paged_append"], indirect=True)
def test_what_an_append_may_not_overlap(call):
    size = 2 * 10 * 128 * 2      # bytes of a head of all rows
    at = 1 << 40
    p = C.c_void_p
    for kw in (dict(q_out=p(at), q=p(at + 16)), dict(q_out=p(at), q=p(at + 8 * size - 16)), dict(q_out=p(at), k=p(at)), dict(q_out=p(at), v=p(at)), dict(q_out=p(at), k_pages=p(at)),
               dict(k_pages=p(at), v_pages=p(at)), dict(k_pages=p(at), k=p(at)), dict(v_pages=p(at), v=p(at + 16)), dict(k_pages=p(at), v_pages=p(at + 40 * 2 * 64 * 128 * 2 - 16))):
        assert call(**kw) == -1 and "overlaps" in dream.dream_last_error(), kw
    assert call(n_rows=257, pos=None) == -2 and "257 rows of a tree" in dream.dream_last_error()


@pytest.mark.parametrize("call", ["dream_paged_commit"], indirect=True)
def test_rows_that_a_commit_moves_at_once(call):
    assert "DREAM_ERR_UNSUPPORTED if min(path_stride, n_tree) rows exceed 64 KB" in _text()
    bad = (C.c_void_p * 3)(0x1000, 0x2008, 0x3000)
    d = _desc(head_dim=256, dtype=dream.F32)
    for stride, tree in ((64, 1000), (1000, 64)):
        assert call(desc=d, path_stride=stride, n_tree=tree, pools_host=bad) == -1
        assert call(desc=d, path_stride=stride + (stride == 64), n_tree=tree + (tree == 64), pools_host=bad) == -2


@pytest.mark.parametrize("call", ["dream_paged_verify_attn", "dream_sparse_verify_attn", "dream_page_select"], indirect=True)
def test_workspaces(lib, call):
    """That of a call does for every shorter one of the same sequences and nodes: the error, if any, is not the workspace's."""
    size = getattr(dream, call.name + "_workspace")
    for D, hq, hkv, B, n in ((64, 8, 8, 1, 1), (128, 32, 8, 1, 60), (128, 32, 8, 12, 33), (256, 16, 8, 3, 200), (128, 8, 1, 40, 1)):
        d, pages = _desc(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=D), dream.page_desc(64, 5000, 1100)
        need = size(d, pages, n, 70000)
        assert need >= 256
        for keys in (n, 300, 5000, 69999):
            if keys >= n and call.name == "dream_page_select":
                assert size(d, pages, n, keys) <= need
    d, pages = _desc(n_q_heads=32, n_kv_heads=8), dream.page_desc(64, 5000, 1100)
    if call.name == "dream_page_select":
        need = size(d, pages, 60, 70000)
        assert call(desc=d, pages=pages, n_tree=60, max_kv_len=70000, workspace_bytes=need - 257) == -3
    elif call.name == "dream_paged_verify_attn":      # the rows of two parts have to find room
        assert call(desc=d, pages=pages, n_tree=60, max_kv_len=70000, n_groups=1, max_shared_len=60000, workspace_bytes=2 * 2 * 60 * 32 * 130 * 4 - 1) == -3
    else:                                             # a list holds 1024 pages
        assert call(desc=d, pages=pages, n_tree=60, max_kv_len=70000, workspace_bytes=2 * 2 * 60 * 32 * 130 * 4 - 1) == -3
        assert str(size(d, pages, 60, 70000)) in dream.dream_last_error()


def test_launches_stay_within_their_limits(lib, tmp_path):
    """tests/c/paged_launch_check.c stands in for HIP's launch functions: 22 kernels have a raised limit (4, 4 and 3 shapes at the three head_dims, each with and without selected pages), all are launched."""
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    root, libdir, exe = os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(dream.library_path()), str(tmp_path / "paged_launch_check")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-rdynamic", "-I", os.path.join(root, "include"), os.path.join(root, "tests", "c", "paged_launch_check.c"), "-o", exe,
                    "-L", libdir, "-ldream", "-Wl,-rpath," + libdir], check=True, capture_output=True, text=True)
    p = subprocess.run([exe], capture_output=True, text=True)
    assert p.returncode == 0 and p.stdout.count("22 with a raised limit") == 2, p.stdout[-3000:] + p.stderr[-1000:]


@every
def test_device_pointers_take_device_tensors_only(call):
    from paper_2505_19201_amd.binding import _native
    native = getattr(_native(), call.name)
    fixed = dict(desc=_desc(), pages=dream.page_desc(64, 40, 20), pools_host=(), stream=0)

    def plain():
        return [fixed.get(param, None if "*" in kind else 1) for kind, param in _signature(call.name)]
    assert native(*plain()) < 0
    for i, (kind, param) in enumerate(_signature(call.name)):
        if "*" not in kind or param in ("desc", "pages", "stream"):
            continue
        for bad, error in ((np.zeros(64), TypeError), (0x1000, TypeError), (torch.zeros(64), ValueError)):
            args = plain()
            args[i] = (bad,) if param == "pools_host" else bad
            with pytest.raises(error):
                native(*args)


# ---- pins of the definitions the GPU tests compare with ----------------------------------------------------------------
def test_definition_of_the_exponents():
    """The least power of two that holds a number in 127 steps, by trying."""
    rng = np.random.default_rng(0)
    tops = np.concatenate([np.exp2(rng.uniform(-110, 127, 200)), 127.0 * np.exp2(np.arange(-100, 120)), np.nextafter(127.0 * np.exp2(np.arange(-100, 120)), np.inf), [0.0]])
    for t in tops:
        want = next((e for e in range(-100, 122) if t <= 127.0 * 2.0 ** e), 122)
        assert pc.least_exponent(t) == want, t


def test_definition_of_the_scores_bounds_every_key():
    """What a page's score stands for: no key of the page has a larger sum of products with the queries as they are rounded."""
    rng = np.random.default_rng(1)
    rows, q = rng.standard_normal((3, 1, 16, 64)), rng.standard_normal((1, 4, 64))
    bounds = np.stack([pc.page_bounds(r) for r in rows])
    c = np.rint(np.ldexp(q[0], -pc.least_exponent(np.abs(q).max())))
    top = np.einsum("hd,pgrd->pr", c, rows).max(1)
    x = bounds[:, 0]
    e = pc.least_exponent(np.abs(x).max((1, 2)))
    up, down = np.ceil(np.ldexp(x[:, 0], -e[:, None])), np.floor(np.ldexp(x[:, 1], -e[:, None]))
    score = np.ldexp(up @ np.maximum(c, 0).sum(0) + down @ np.minimum(c, 0).sum(0), e)
    assert (score >= top).all()
    assert np.array_equal(pc.choose(q, bounds, 0, 0, 1)[0, 0], np.arange(3) == score.argmax())


def test_definition_of_attention_is_plain_attention_over_the_rows_in_order():
    """One sequence in pages out of order, a chain of two nodes: dense softmax by torch in 64 bits."""
    rng = np.random.default_rng(2)
    P, D, page = 37, 64, 16
    pages = pc.Pages(rng, page, [P + 2])
    k, v, q = rng.standard_normal((2, P + 2, D)), rng.standard_normal((2, P + 2, D)), rng.standard_normal((2, 2, D))
    pool = pages.pool(2, D)
    pages.put(pool, 0, 0, k)
    at = np.array([pages.where(0, r) for r in range(P + 2)])
    assert np.array_equal(pool[at[:, 0], :, at[:, 1]].transpose(1, 0, 2), k)
    out = wc.attention(q[None], k[None], v[None], [P], [[-1, 0]], 0, 0)[0]
    for i in range(2):
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[i][:, None]), torch.from_numpy(k[:, :P + 1 + i]), torch.from_numpy(v[:, :P + 1 + i]))
        assert np.abs(out[0, i] - want[:, 0].numpy()).max() < 1e-12
