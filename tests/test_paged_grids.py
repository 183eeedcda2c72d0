"""No-GPU check of how many threads the attention calls over pages ask for at the largest sizes."""
import os
import shutil
import subprocess

import pytest

import paper_2505_19201_amd as dream
from tests.test_operator_limits import _text
from tests.test_paged_refusals import lib      # noqa: F401


def test_launches_of_too_many_threads_are_refused(lib, tmp_path):
    """tests/c/paged_grid_check.c in HIP's place."""
    assert "Calls whose launch would have 2^32 threads are DREAM_ERR_UNSUPPORTED; with batch * n_q_heads * n_tree at most 2^23 none has" in _text()
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    root, libdir, exe = os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(dream.library_path()), str(tmp_path / "paged_grid_check")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-Wno-unused-function", "-rdynamic", "-I", os.path.join(root, "include"), os.path.join(root, "tests", "c", "paged_grid_check.c"),
                    "-o", exe, "-L", libdir, "-ldream", "-Wl,-rpath," + libdir], check=True, capture_output=True, text=True)
    p = subprocess.run([exe], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout[-3000:] + p.stderr[-1000:]
