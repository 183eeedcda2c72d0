"""Which kernel the window and 4-bit attention calls launch, forced and by themselves, and that its workgroups are every row group of every unit once (no GPU: tests/c/window_launch_check.c in HIP's place)."""
import itertools
import os
import re
import shutil
import subprocess

import pytest

import paper_2505_19201_amd as dream
from paper_2505_19201_amd import build as dream_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = dream.F32, dream.BF16


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if not os.path.exists(dream.library_path()):
        dream_build.build(verbose=False)
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    libdir, exe = os.path.dirname(dream.library_path()), str(tmp_path_factory.mktemp("launch") / "window_launch_check")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-rdynamic", "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "c", "window_launch_check.c"), "-o", exe,
                    "-L", libdir, "-ldream", "-Wl,-rpath," + libdir], check=True, capture_output=True, text=True)

    def run(calls):
        """Per call its status and launches: (kernel, template arguments, grid, threads, words)."""
        text = "".join(" ".join(str(int(x)) for x in c) + "\n" for c in calls)
        p = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
        out = []
        for line in p.stdout.splitlines():
            words, got = line.split(), []
            while len(words) > 1:
                name, grid, threads = words[0], tuple(map(int, words[1:4])), int(words[4])
                extra = 3 if threads in (256, 512) else 0
                got.append((*_read(name), grid, threads, tuple(map(int, words[5:5 + extra]))))
                words = words[5 + extra:]
            out.append((int(words[0]), got))
        assert len(out) == len(calls)
        return out
    return run


def _read(mangled):
    """window_attn_kernelILi64ELi1ELi8ELb1EE.. -> the name and (64, 1, 8, 1)."""
    m = re.search(r"(window_\w+?_kernel)I((?:L[ib]\d+E)+)E", mangled)
    assert m, mangled
    return m.group(1), tuple(int(x) for x in re.findall(r"L[ib](\d+)E", m.group(2)))


def _place(words, block):
    """Unit and row group of a workgroup (place_of in csrc/attn_window.hip)."""
    x, y, z = block
    lg = words[0] >> 24
    part = (z * 32768 + y) * 8 + (x & 7)
    return part >> lg, (x >> 3) << lg | (part & ((1 << lg) - 1))


# The forced shapes of the GPU tests and the kernels that they have to reach, where a head_dim and a cache have them: (query tiles, waves) -> per (4 bits, head_dim)
FORCED = {
    (1, 4): {(mx, D): ("window_attn_kernel", (D, 1, 4, mx)) for mx in (0, 1) for D in (64, 128, 256)},
    (2, 4): {(0, 64): ("window_attn_kernel", (64, 2, 4, 0)), (1, 64): ("window_attn_kernel", (64, 2, 4, 1)), (1, 128): ("window_attn_kernel", (128, 2, 4, 1))},
    (4, 4): {(1, 64): ("window_attn_kernel", (64, 4, 4, 1))},
    (1, 8): {(1, D): ("window_attn_kernel", (D, 1, 8, 1)) for D in (64, 128, 256)},
    (0, 8): {(0, 64): ("window_shared_kernel", (64, 2, 0)), (0, 128): ("window_shared_kernel", (128, 1, 0)), (0, 256): ("window_shared_kernel", (256, 1, 0)),
             (1, 128): ("window_shared_kernel", (128, 1, 1)), (1, 256): ("window_shared_kernel", (256, 1, 1))},
}


@pytest.mark.parametrize("mx", [0, 1])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("tiles,waves", sorted(FORCED))
def test_forced_shapes_reach_their_kernels(launches, tiles, waves, D, mx):
    """Trees that the GPU tests force them on; a shape that a head_dim does not have takes one that it has."""
    shapes = [(hq, hkv, n, keys, w, s) for hq, hkv, n, keys, w, s in ((2, 2, 1, 1, 0, 0), (4, 2, 9, 106, 40, 3), (8, 1, 60, 360, 100, 4), (2, 1, 250, 950, 0, 0), (4, 2, 12, 340, 0, 0))]
    for splits in (1, 4):
        got = launches([(mx, BF16, 2, hq, hkv, D, n, keys, w, s, tiles, waves, splits) for hq, hkv, n, keys, w, s in shapes])
        for status, kernels in got:
            assert status == 0
            want = FORCED[tiles, waves].get((mx, D))
            if want:
                assert kernels[0][:2] == want
            else:
                assert kernels[0][1][0] == D and kernels[0][1][-1] == mx
            assert [k[0] for k in kernels[1:]] == (["window_merge_kernel"] if splits > 1 else [])
            assert kernels[0][4][0] >> 16 & 0xff == {1: 0, 4: 2}[splits]


def test_what_the_documents_name_is_what_is_launched(launches):
    """The kernels of the timed cases, and one workgroup for as many CUs as the documents say."""
    calls = {
        (1, BF16, 1, 32, 32, 128, 60, 704, 0, 0): ("window_attn_kernel", (128, 1, 4, 1), 128, 1),
        (1, BF16, 8, 32, 8, 128, 60, 1283, 0, 0): ("window_attn_kernel", (128, 2, 4, 1), 512, 1),
        (1, BF16, 32, 32, 32, 64, 60, 1600, 0, 0): ("window_attn_kernel", (64, 4, 4, 1), 1024, 1),
        (1, BF16, 4, 32, 8, 128, 1, 32700, 0, 0): ("window_attn_kernel", (128, 1, 8, 1), 256, 8),
        (0, BF16, 4, 16, 8, 256, 33, 1283, 1024, 0): ("window_shared_kernel", (256, 1, 0), 256, 8),
        (0, BF16, 1, 32, 32, 128, 1, 4000, 1020, 4): ("window_attn_kernel", (128, 1, 4, 0), 256, 8),
    }
    for (status, kernels), (name, args, groups, splits) in zip(launches([c + (0, 0, 0) for c in calls]), calls.values()):
        grid = kernels[0][2]
        assert status == 0 and kernels[0][:2] == (name, args)
        assert (grid[0] * grid[1] * grid[2], 1 << (kernels[0][4][0] >> 16 & 0xff)) == (groups, splits)
        assert len(kernels) == (2 if splits > 1 else 1)


def test_float32_has_a_kernel_of_its_own(launches):
    calls = [(mx, F32, 2, 4, 2, D, 9, 100, w, 3, 0, 0, 0) for mx in (0, 1) for D in (64, 128, 256) for w in (0, 41)]
    for c, (status, kernels) in zip(calls, launches(calls)):
        assert status == 0 and [(k[0], k[1], k[2]) for k in kernels] == [("window_f32_kernel", (c[5], c[0]), (9, 4, 2))]


def test_workgroups_are_every_row_group_of_every_unit_once(launches):
    """Over head layouts, batches, trees, lengths and forced splits: grids within HIP's limits, each pair of a unit and a row group once, whatever else a grid has lies outside and ends at once;
    a unit's sequence and KV head from one multiplication."""
    calls = [(mx, BF16, b, hq, hkv, D, n, keys, w, 4, 0, 0, s)
             for mx in (0, 1) for D in (64, 128, 256) for b, (hq, hkv) in itertools.product((1, 3, 16, 40), ((8, 8), (32, 8), (14, 2), (2, 1), (71, 1)))
             for n, keys, w, s in ((1, 40, 0, 0), (17, 900, 0, 0), (60, 1300, 512, 0), (250, 5000, 0, 0), (33, 40000, 0, 0), (9, 700, 64, 8))]
    calls += [(mx, BF16, 65535, 16, 16, 64, 1, 2, 0, 0, 0, 0, s) for mx in (0, 1) for s in (0, 64)]
    for c, (status, kernels) in zip(calls, launches(calls)):
        mx, _, b, hq, hkv, D, n = c[:7]
        assert status == 0
        (name, args, grid, threads, words), merge = kernels[0], kernels[1:]
        splits, units = 1 << (words[0] >> 16 & 0xff), words[2] >> 10
        assert words[0] & 0xffff == hkv and words[2] & 0x1ff == n and (words[2] >> 9 & 1) == (c[8] != 0)
        assert units == b * hkv * splits and len(merge) == (splits > 1)
        shared = name == "window_shared_kernel"
        rows_a_group = 16 * args[1] * (8 if shared else 1)
        groups = -(-n * (hq // hkv) // rows_a_group)
        assert threads == (512 if shared else 64 * args[2])
        for k in kernels:
            assert 0 < k[2][0] < 2 ** 31 and 0 < k[2][1] <= 65535 and 0 < k[2][2] <= 65535
        for stream in {0, 1, b * hkv // 2, b * hkv - 1}:
            assert (stream * words[1] >> 32 if words[1] else stream) == stream // hkv
        if b > 1000:
            continue
        seen = {}
        for block in itertools.product(*map(range, grid)):
            unit, rg = _place(words, block)
            if unit < units and rg < groups:
                seen[unit, rg] = seen.get((unit, rg), 0) + 1
        assert len(seen) == units * groups and set(seen.values()) == {1}, c
        if merge:
            g = merge[0][2]
            assert merge[0][1] == (D,) and g[1] * g[2] >= b * hkv and g[0] * (1024 // D) >= n * (hq // hkv)
