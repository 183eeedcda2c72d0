"""Host model of what the window and 4-bit attention kernels read through range-checked descriptors (csrc/attn_window.hip).  The address maps are the kernels' own (csrc/window_maps.h, built for the
host); this file says what they have to do: which row and channels every lane's load has, that a load is wholly within a live row or wholly behind the descriptor's size, that no offset passes
32 bits, and which tiles are asked for."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from tests import window_cases as wc

HERE = os.path.dirname(os.path.abspath(__file__))
FIELDS = ["tensor", "lane", "half", "piece", "at", "width", "row", "channel"]
# head_dim, 4 bits, the kernel whose waves take a tile each or the one whose waves share a tile
FORMS = [(D, mx, False) for D in (64, 128, 256) for mx in (0, 1)] + [(64, 0, True), (128, 0, True), (128, 1, True), (256, 0, True), (256, 1, True)]
IDS = ["%d-%s-%s" % (D, "4bit" if mx else "16bit", "shared" if shared else "wave") for D, mx, shared in FORMS]


@pytest.fixture(scope="module", autouse=True)
def maps(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("maps") / "window_maps_check.so")
    root = os.path.dirname(HERE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I" + os.path.join(root, "paper_2505_19201_amd", "csrc"), "-I" + os.path.join(root, "include"),
                    os.path.join(HERE, "c", "window_maps_check.cpp"), "-o", out], check=True)
    global LIB
    LIB = ctypes.CDLL(out)
    LIB.behind.restype = LIB.early.restype = LIB.asked_for.restype = ctypes.c_uint32
    LIB.most_rows.restype = ctypes.c_int64


def loads(form, tile):
    D, mx, shared = form
    raw = np.zeros((8192, 8), dtype=np.int64)
    n = (LIB.group_loads if shared else LIB.wave_loads)(D, mx, ctypes.c_uint32(tile), raw.ctypes.data_as(ctypes.c_void_p))
    assert 0 < n <= len(raw)
    return {f: raw[:n, i] for i, f in enumerate(FIELDS)}


def sizes(form):
    """Bytes of a row of each tensor."""
    D, mx, _ = form
    return np.array([LIB.bytes_of_row(D, mx)] * 2 + [LIB.bytes_of_scales(D)] * 2)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_the_loads_of_a_tile_are_the_tile(form):
    """Rows and values each byte once, in the row that the load is used for; the scale of a load's values beside it."""
    D, mx, shared = form
    x, size = loads(form, 0), sizes(form)
    assert size[0] == (D // 2 if mx else 2 * D) and size[2] == D // 32
    row_of = x["at"] // size[x["tensor"]]
    assert (row_of == x["row"]).all() and (x["row"] < 32).all()
    in_row = x["at"] - row_of * size[x["tensor"]]
    assert (in_row + x["width"] <= size[x["tensor"]]).all()
    per_value = (0.5 if mx else 2)
    for tensor in (0, 1):
        mine = x["tensor"] == tensor
        got = np.sort(np.concatenate([np.arange(a, a + w) for a, w in zip(x["at"][mine], x["width"][mine])]))
        assert np.array_equal(got, np.arange(32 * size[0]))
    known = x["channel"] >= 0
    values = known & (x["tensor"] < 2)
    assert (in_row[values] == x["channel"][values] * per_value).all()
    scales = known & (x["tensor"] >= 2)
    assert (in_row[scales] == x["channel"][scales] // 32).all()
    if mx:                     # a load's values have one scale
        assert (x["width"][values] / per_value <= 32).all() and (x["channel"][values] % 32 + x["width"][values] / per_value <= 32).all()
    if shared:
        assert known.all()
        return
    # K of the kernel whose waves take a tile each: what a lane has of a k-step is what the other operand, the queries, takes from channel_of on
    for i in np.flatnonzero(x["tensor"] == 0):
        lane, half, piece = (int(x[f][i]) for f in ("lane", "half", "piece"))
        c, g = lane & 15, lane >> 4
        assert row_of[i] == half * 16 + c
        words = 1 if not mx else int(x["width"][i]) // 4      # of 8 values
        for e in range(words):
            ks = piece if not mx else piece * 4 + e
            assert LIB.wave_channel(D, mx, ks, g) == in_row[i] / per_value + 8 * e
    for i in np.flatnonzero(x["tensor"] == 2):
        lane, piece = int(x["lane"][i]), int(x["piece"][i])
        for ks in range(piece * 4, min(piece * 4 + 4, D // 32)):
            assert in_row[i] == LIB.wave_channel(D, mx, ks, lane >> 4) // 32
    # every lane asks for as many pieces as its k-steps need
    assert sorted({LIB.wave_channel(D, mx, ks, g) for ks in range(D // 32) for g in range(4)}) == list(range(0, D, 8))


def check_range(form, rows, tile, exact):
    """What a tile's loads return under a descriptor of `rows` rows: the row that was meant where it is one of them, nothing of it otherwise."""
    x, size = loads(form, tile), sizes(form)
    base = exact[0] + tile * 32 * size[exact[1]]
    assert np.array_equal(x["at"], base)                    # 32 bits have held the sum
    assert (x["at"] + x["width"] <= 1 << 32).all()
    records = rows * size[exact[1]]
    assert (records < 1 << 32).all()
    live = tile * 32 + exact[2] < rows
    assert (x["at"][live] + x["width"][live] <= records[live]).all()
    assert (x["at"][~live] >= records[~live]).all()


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_every_load_is_within_a_live_row_or_behind_the_descriptor(form):
    x = loads(form, 0)
    exact = (x["at"], x["tensor"], x["row"])
    most = LIB.most_rows()
    assert most == (1 << 23) - 128
    for rows in [1, 2, 16, 31, 32, 33, 63, 64, 65, 97, 700, 1283, 32700, most - 33, most - 32, most - 31, most - 1, most]:
        none = LIB.behind(rows)
        assert (none - 1) * 32 < rows <= none * 32
        for tile in sorted({0, 1, none // 2, max(none - 2, 0), none - 1, none}):
            check_range(form, rows, tile, exact)
        # the tile behind the live rows reads nothing
        assert (loads(form, none)["at"] >= rows * sizes(form)[exact[1]]).all()
    # under a descriptor of the whole cache, before the prefix is known
    for s_max in [1, 5, 32, 33, 100, 257, 5000, most]:
        for wave in range(8):
            tile = LIB.early(wave, s_max)
            assert tile == min(wave, -(-s_max // 32)) and tile * 32 < 256
            check_range(form, s_max, tile, exact)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_a_head_s_base_and_its_descriptor_stay_inside_the_cache(form):
    """Base: the head's rows in front; size: its live rows.  The last byte of the last head is the cache's last at most (bases are 64 bits)."""
    size = sizes(form)
    for streams, s_max in ((1, 1), (7, 100), (16, 1 << 20), (1 << 20, LIB.most_rows())):
        for stream in {0, streams // 2, streams - 1}:
            for given in (-5, 0, 1, s_max - 1, s_max, s_max + 9, 2 ** 31 - 1):
                for T in (1, min(s_max, 60)):
                    P = LIB.live_prefix(given, s_max, T)
                    assert 0 <= P and P + T <= s_max and (P == given or not 0 <= given <= s_max - T)
                    for bytes_ in size:
                        base = stream * s_max * int(bytes_)
                        assert base < 1 << 63 and base + (P + T) * int(bytes_) <= streams * s_max * int(bytes_)


@pytest.mark.parametrize("waves,ahead", [(4, 1), (8, 1), (1, 3)], ids=["4 waves", "8 waves", "shared"])
@pytest.mark.parametrize("lg_splits", [0, 1, 3, 6])
def test_which_tiles_are_asked_for(lg_splits, waves, ahead):
    """Every tile that holds a key some node sees, once over all splits and waves; in every other place, up to `ahead` steps behind the end, the tile behind the live rows."""
    room = (ctypes.c_int32 * 4096)()
    ends = (ctypes.c_int32 * 2)()
    rng = np.random.default_rng(lg_splits)
    for window, sink in ((0, 0), (1, 0), (5, 2), (33, 0), (64, 70), (100, 4), (1020, 4), (1024, 0), (1 << 30, 1 << 30), (3, 1 << 30)):
        for P in (0, 1, 3, 31, 32, 33, 63, 64, 65, 97, 300, 1281):
            for T in (1, 2, 31, 60, 64, 70, 256):
                n = LIB.tile_list(window, sink, T, P, room, 4096)
                tiles = list(room[:n])
                assert n > 0 and tiles == sorted(set(tiles)) and tiles[-1] == (P + T - 1) // 32
                assert all(t < LIB.behind(P + T) for t in tiles)
                parent = wc.tree("rand", T, rng) if T < 100 else wc.tree("chain", T, rng)
                depth = [len(p) - 1 for p in wc.ancestors(parent)]
                # keys of the prefix that the root sees (it sees the most of them), and the tree's rows
                seen = {j for j in range(P) if not window or P - j < window or j < sink} | {P + a for a in range(T)}
                assert {j // 32 for j in seen} == set(tiles), (window, sink, P, T, max(depth))
                asked, none = [], LIB.behind(P + T)
                for split in range(1 << lg_splits):
                    LIB.share(n, split, lg_splits, ends)
                    for wave in range(waves):
                        t = ends[0] + wave
                        while t < ends[1]:
                            asked.append(LIB.asked_for(window, sink, T, P, split, lg_splits, t))
                            t += waves
                        for more in range(ahead):
                            assert LIB.asked_for(window, sink, T, P, split, lg_splits, t + more * waves) == none
                assert sorted(asked) == tiles
