"""The limits that include/dream.h states for rotary positions, 4-bit caches and window attention are those that the calls enforce (no GPU: every call below ends before a launch)."""
import ctypes as C
import os
import re

import pytest

import paper_2505_19201_amd as dream
from paper_2505_19201_amd import build as dream_build
from tests.test_operator_refusals import ODD, _caller, _desc, _Job

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dream.h")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dream.library_path()):
        dream_build.build(verbose=False)
    return dream.load()


def _text():
    return re.sub(r"\s*\n \*\s*", " ", open(HEADER).read())


def _constant(name):
    value = re.search(rf"#define {name} (.+?)\s*/\*", open(HEADER).read()).group(1)
    assert re.fullmatch(r"[\d()<\s-]+", value)
    return eval(value)


def _refusal(call, **kw):
    """Status and message of a call whose last checked argument is wrong too, so that it never launches."""
    status = call(**kw)
    assert status < 0
    return status, dream.dream_last_error()


@pytest.mark.parametrize("name,last", [("dream_mx_append", dict(k_rows=ODD)), ("dream_mx_read", dict(out=ODD)), ("dream_mx_commit", dict(path_stride=0))])
def test_sequences_and_heads_of_a_4_bit_cache(lib, name, last):
    one = (C.c_void_p * 3)(0x1000, 0x2000, 0x3000)
    call = _caller(lib, name, codes_host=one, scales_host=one, n_caches=3, n_rows=10, n_tree=20, path_stride=7, prefix_len_out=None)
    most = _constant("DREAM_MAX_MX_BATCH")
    assert most == 32767 and "n_kv_heads up to 65535" in _text()
    assert _refusal(call, desc=_desc(batch=most), **last)[0] == -1
    assert _refusal(call, desc=_desc(batch=most + 1), **last) == (-2, f"{name}: batch is limited to {most}, n_kv_heads to 65535")
    assert _refusal(call, desc=_desc(n_kv_heads=65535), **last)[0] == -1
    assert _refusal(call, desc=_desc(n_kv_heads=65536), **last)[0] == -2


def test_rows_read_at_once(lib):
    one = (C.c_void_p * 1)(0x1000)
    call = _caller(lib, "dream_mx_read", codes_host=one, scales_host=one, n_caches=1)
    assert "n_rows at most s_max and 2^24" in _text()
    for s_max, most in ((500, 500), ((1 << 24) + 5, 1 << 24)):
        assert "out must be" in _refusal(call, desc=_desc(s_max=s_max), n_rows=most, out=ODD)[1]
        assert "n_rows" in _refusal(call, desc=_desc(s_max=s_max), n_rows=most + 1, out=ODD)[1]


def test_heads_of_a_rotary_job(lib):
    call = _caller(lib, "dream_rotary_rows", desc=_desc(), n_jobs=1, n_rows=10, rot_dim=128, interleaved=0, amplitude=1.0)
    assert "n_heads at most 65535" in _text()
    for heads, what in ((65535, "not aligned"), (65536, "n_heads")):
        assert what in _refusal(call, jobs=(_Job * 1)(_Job(0x1001, heads, None, None, 0x2000)))[1]


@pytest.mark.parametrize("name", ["dream_window_verify_attn", "dream_mx_verify_attn"])
def test_sequences_heads_rows_and_windows(lib, name):
    call = _caller(lib, name, desc=_desc(), n_tree=20, window=100, n_sink=4, max_kv_len=300, workspace=None)
    text = _text()
    assert "batch at most 65535, n_q_heads at most 4096, their product at most 2^20" in text and "Both at most 2^30" in text
    rows = _constant("DREAM_MAX_WINDOW_ROWS")
    for fits, not_ in ((dict(batch=65535, n_q_heads=16), dict(batch=65536, n_q_heads=16)), (dict(n_q_heads=4096), dict(n_q_heads=4098)),
                       (dict(batch=256, n_q_heads=4096), dict(batch=257, n_q_heads=4096)), (dict(s_max=rows), dict(s_max=rows + 1))):
        assert _refusal(call, desc=_desc(**fits))[0] == -3
        assert _refusal(call, desc=_desc(**not_))[0] == -2
    for param in ("window", "n_sink"):
        assert _refusal(call, **{param: 1 << 30})[0] == -3
        assert _refusal(call, **{param: (1 << 30) + 1})[0] == -1
