"""No-GPU checks of what dream_rotary_rows, the 4-bit cache calls and the window attention calls refuse before anything is launched, and of their definitions' own pins."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import paper_2505_19201_amd as dream
from paper_2505_19201_amd import build as dream_build
from tests import window_cases as wc
from tests.test_abi import _signature

FAKE = C.c_void_p(0x1000)      # never dereferenced: every call below fails before a launch
ODD = C.c_void_p(0x1004)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dream.library_path()):
        dream_build.build(verbose=False)
    return dream.load()


def _desc(**kw):
    d = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=dream.BF16, s_max=500)
    d.update(kw)
    return dream.attn_desc(**d)


def _caller(lib, name, **defaults):
    """Calls an entry point by its parameters' names; what is not named is a pointer or 1."""
    params = _signature(name)

    def call(**kw):
        args = []
        for kind, param in params:
            v = kw[param] if param in kw else defaults.get(param, FAKE if "*" in kind else 1)
            if isinstance(v, dream.AttnDesc):
                v = C.byref(v)
            elif isinstance(v, (int, float)) and v is not None:
                v = C.c_float(v) if "float" in kind else C.c_size_t(v) if "size_t" in kind else C.c_int64(v) if "int64" in kind else C.c_int32(v)
            args.append(v)
        return getattr(lib, name)(*args)
    return call


class _Job(C.Structure):
    _fields_ = [("x", C.c_void_p), ("n_heads", C.c_int32), ("row_base", C.c_void_p), ("row_index", C.c_void_p), ("out", C.c_void_p)]


def test_rotary(lib):
    jobs = (_Job * 5)(*[_Job(0x1000, 8, None, None, 0x2000)] * 5)
    call = _caller(lib, "dream_rotary_rows", desc=_desc(), jobs=jobs, n_jobs=1, n_rows=10, rot_dim=128, interleaved=0, amplitude=1.0)
    for kw in (dict(desc=None), dict(jobs=None), dict(inv_freq=None), dict(n_jobs=0), dict(n_jobs=5), dict(n_rows=0), dict(n_rows=1 << 20),
               dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=130), dict(rot_dim=-2), dict(pos=None, pos_base=None), dict(desc=_desc(dtype=7)),
               dict(desc=_desc(batch=0)), dict(jobs=(_Job * 1)(_Job(None, 8, None, None, 0x2000))), dict(jobs=(_Job * 1)(_Job(0x1000, 0, None, None, 0x2000))),
               dict(jobs=(_Job * 1)(_Job(0x1000, 8, None, 0x3000, 0x2000))), dict(jobs=(_Job * 1)(_Job(0x1001, 8, None, None, 0x2000))),
               dict(jobs=(_Job * 1)(_Job(0x1000, 8, 0x3000, None, 0x1000)))):
        assert call(**kw) == -1, kw
        assert dream.dream_last_error().startswith("dream_rotary_rows")
    for kw in (dict(desc=_desc(head_dim=127)), dict(desc=_desc(head_dim=514)), dict(pos=None, n_rows=257)):
        assert call(**kw) == -2, kw


@pytest.mark.parametrize("name", ["dream_mx_append", "dream_mx_read", "dream_mx_commit"])
def test_caches(lib, name):
    one = (C.c_void_p * 3)(0x1000, 0x2000, 0x3000)
    call = _caller(lib, name, desc=_desc(), codes_host=one, scales_host=one, n_caches=3, n_rows=10, n_tree=20, path_stride=7, prefix_len_out=None)
    wrong = [dict(desc=None), dict(desc=_desc(batch=0)), dict(desc=_desc(n_kv_heads=0)), dict(desc=_desc(s_max=0)), dict(desc=_desc(dtype=2))]
    for kind, param in _signature(name):
        if "*" in kind and param not in ("stream", "row_index", "prefix_len_out") and not (name == "dream_mx_read" and param == "row_base"):
            wrong.append({param: None})
    if name == "dream_mx_append":
        wrong += [dict(n_rows=0), dict(n_rows=1 << 20), dict(k_rows=ODD), dict(v_rows=ODD), dict(k_codes=ODD), dict(k_scales=ODD), dict(v_codes=ODD), dict(v_scales=ODD)]
    else:
        bad = (C.c_void_p * 3)(0x1000, 0x2004, 0x3000)
        none = (C.c_void_p * 3)(0x1000, 0x2000, None)
        wrong += [dict(n_caches=0), dict(codes_host=bad), dict(scales_host=bad), dict(codes_host=none), dict(scales_host=none)]
    if name == "dream_mx_read":
        wrong += [dict(n_rows=0), dict(n_rows=501), dict(out=ODD)]
    if name == "dream_mx_commit":
        wrong += [dict(n_tree=0), dict(n_tree=501), dict(path_stride=0), dict(prefix_len_out=FAKE)]
    for kw in wrong:
        assert call(**kw) == -1, kw
        assert dream.dream_last_error().startswith(name)
    assert call(desc=_desc(head_dim=96)) == -2
    assert call(desc=_desc(batch=40000)) == -2
    if name == "dream_mx_commit":
        assert call(n_tree=500, path_stride=500) == -2


@pytest.mark.parametrize("name", ["dream_window_verify_attn", "dream_mx_verify_attn"])
def test_attention(lib, name):
    call = _caller(lib, name, desc=_desc(), n_tree=20, window=100, n_sink=4, max_kv_len=300, workspace_bytes=1 << 40)
    wrong = [dict(desc=None), dict(desc=_desc(n_q_heads=7)), dict(desc=_desc(batch=0)), dict(desc=_desc(dtype=5)), dict(window=-1), dict(n_sink=-1),
             dict(max_kv_len=19), dict(max_kv_len=501), dict(window=(1 << 30) + 1), dict(parent=None), dict(parent=None, tree_mask=None, window=0)]
    for kind, param in _signature(name):
        if "*" in kind and param not in ("stream", "lse", "tree_mask", "workspace"):
            wrong.append({param: None})
        if param in ("q", "k_cache", "v_cache", "k_codes", "v_codes", "k_scales", "v_scales", "out"):
            wrong.append({param: ODD})
    for kw in wrong:
        assert call(**kw) == -1, kw
        assert dream.dream_last_error().startswith(name)
    for kw in (dict(n_tree=0), dict(n_tree=257), dict(desc=_desc(head_dim=96)), dict(desc=_desc(batch=40000, n_q_heads=64)), dict(desc=_desc(s_max=1 << 31))):
        assert call(**kw) == -2, kw
    long = _desc(batch=1, s_max=9000)
    size = getattr(dream, name + "_workspace")
    need = size(long, 20, 8000, 0, 0)
    assert need > 256
    assert call(desc=long, max_kv_len=8000, window=0, workspace_bytes=need - 1) == -3
    assert call(desc=long, max_kv_len=8000, window=0, workspace=None) == -3
    assert call(desc=long, max_kv_len=8000, window=0, workspace=ODD) == -3


@pytest.mark.parametrize("name", ["dream_window_verify_attn", "dream_mx_verify_attn"])
def test_a_workspace_for_the_longest_range_fits_every_shorter_call(lib, name):
    size = getattr(dream, name + "_workspace")
    for D in (64, 128, 256):
        for hq, hkv in ((8, 8), (32, 8), (8, 1)):
            for B in (1, 3, 12):
                for n in (1, 33, 200):
                    for window in (0, 1000):
                        need = [size(_desc(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=D, s_max=70000), n, keys, window, 4) for keys in range(n, 70000, 997)]
                        assert need == sorted(need), (D, hq, hkv, B, n, window)


def test_the_binding_takes_pairs_of_caches():
    t = torch.zeros(8, dtype=torch.uint8)
    for call in (lambda: dream.dream_mx_read(_desc(), [t, t], [t], None, 1, t), lambda: dream.dream_mx_commit(_desc(), [t], [], t, 1, t, t)):
        with pytest.raises(ValueError, match="caches of codes"):
            call()


def test_a_rotary_job_is_any_sequence_of_five(lib):
    """Lists, tuples and iterators reach the library, which refuses the missing frequencies; four fields do not."""
    class NoStream:
        cuda_stream = 0
    for form in (tuple, list, iter):
        with pytest.raises(dream.DreamError, match="NULL argument"):
            dream.dream_rotary_rows(_desc(), [form((None, 4, None, None, None))], 1, None, None, None, None, 128, stream=NoStream())
    with pytest.raises(ValueError, match="a job is"):
        dream.dream_rotary_rows(_desc(), [(None, 4, None, None)], 1, None, None, None, None, 128, stream=NoStream())


@pytest.mark.parametrize("name", ["dream_rotary_rows", "dream_mx_append", "dream_mx_read", "dream_mx_commit", "dream_window_verify_attn", "dream_mx_verify_attn"])
def test_device_pointers_take_device_tensors_only(lib, name):
    from paper_2505_19201_amd.binding import _native
    call = getattr(_native(), name)

    def plain():
        args = []
        for kind, param in _signature(name):
            args.append(_desc() if param == "desc" else () if param in ("jobs", "codes_host", "scales_host") else 0 if param == "stream" else None if "*" in kind else 1)
        return args
    assert call(*plain()) < 0
    for i, (kind, param) in enumerate(_signature(name)):
        if param in ("desc", "stream") or "*" not in kind:
            continue
        for bad, error in ((np.zeros(64), TypeError), (0x1000, TypeError), (torch.zeros(64), ValueError)):
            args = plain()
            args[i] = bad
            if param == "jobs":
                args[i] = ((bad, 1, None, None, None),)
            elif param.endswith("_host"):
                args[i] = (bad,)
            with pytest.raises(error):
                call(*args)


# ---- pins of the definitions the GPU tests compare with ----------------------------------------------------------------
def test_definition_of_the_window_is_plain_attention_over_what_is_left():
    """One node, a window of w and s first tokens: dense softmax over those keys alone, by torch in 64 bits."""
    rng = np.random.default_rng(0)
    P, w, s, D = 50, 12, 3, 16
    q, k, v = rng.standard_normal((1, 1, 2, D)), rng.standard_normal((1, 2, P + 1, D)), rng.standard_normal((1, 2, P + 1, D))
    out, lse, _, _ = wc.attention(q, k, v, [P], [[-1]], w, s)
    keep = list(range(s)) + list(range(P - w + 1, P + 1))
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(1, 2), torch.from_numpy(k[:, :, keep]), torch.from_numpy(v[:, :, keep]))
    assert np.abs(out - want.transpose(1, 2).numpy()).max() < 1e-12


def test_definition_of_a_chain_is_the_banded_causal_mask():
    see = wc.visible([-1, 0, 1, 2, 3], 4, 3, 1)
    want = np.array([[1, 0, 1, 1, 1, 0, 0, 0, 0], [1, 0, 0, 1, 1, 1, 0, 0, 0], [1, 0, 0, 0, 1, 1, 1, 0, 0], [1, 0, 0, 0, 0, 1, 1, 1, 0],
                     [1, 0, 0, 0, 0, 0, 1, 1, 1]], dtype=bool)
    assert np.array_equal(see, want)


def test_definition_of_the_codes():
    x = np.zeros((1, 32))
    x[0, :9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -7.0, 6.9]
    code, byte, _ = wc.quantise(x)
    assert byte[0, 0] == 127 and code[0, :9].tolist() == [0, 2, 2, 4, 4, 6, 6, 15, 7]
    x[0, 7] = -7.01
    assert wc.quantise(x)[1][0, 0] == 128
    back = wc.decode(wc.pack(wc.quantise(x)[0]), wc.quantise(x)[1])
    assert np.abs(back - x).max() <= 2.0
    assert wc.quantise(np.zeros((1, 32)))[1][0, 0] == 2


def test_definition_of_rotary_is_a_complex_product():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((1, 3, 1, 8))
    f = np.array([1.0, 0.1, 0.01], dtype=np.float32)
    y = wc.rotary(x, np.array([[0, 5, -7]]), f, 6, True, 2.0)
    z = (x[..., 0:6:2] + 1j * x[..., 1:6:2]) * 2.0 * np.exp(1j * np.array([0, 5, -7])[None, :, None, None] * f.astype(np.float64))
    assert np.allclose(y[..., 0:6:2], z.real, atol=1e-14) and np.allclose(y[..., 1:6:2], z.imag, atol=1e-14) and np.array_equal(y[..., 6:], x[..., 6:])
