"""No-GPU check of the workspaces that the attention calls over pages take: what dream.h says does for other calls is taken, less is refused, and what is asked for stays in proportion."""
import os
import shutil
import subprocess

import pytest

import paper_2505_19201_amd as dream
from tests.test_operator_limits import _text
from tests.test_paged_refusals import lib      # noqa: F401


def test_which_workspaces_do(lib, tmp_path):
    """tests/c/paged_workspace_check.c, over one to five parts of the rows."""
    assert "if it holds one part of the rows (two, with groups, or where more than 1024 selected pages, 512 above 64 nodes, may be seen)" in _text()
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    root, libdir, exe = os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(dream.library_path()), str(tmp_path / "paged_workspace_check")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-Wno-unused-function", "-rdynamic", "-I", os.path.join(root, "include"), os.path.join(root, "tests", "c", "paged_workspace_check.c"),
                    "-o", exe, "-L", libdir, "-ldream", "-Wl,-rpath," + libdir], check=True, capture_output=True, text=True)
    p = subprocess.run([exe], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout[-3000:] + p.stderr[-1000:]
