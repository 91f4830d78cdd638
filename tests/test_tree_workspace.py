"""How many partial rows the tree attention's pieces reach (csrc/shared_prefix_layout.h's
bound, compiled for the host), against a plain walk over the pieces of the cut that
csrc/shared_prefix_kernel.cuh describes: each CTA has a range of the axis on which the
segments' key tiles lie, and a piece for each segment that its range meets."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2505_12728_gb300 import build_lib

SOURCE = """
#include "shared_prefix_layout.h"
extern "C" long long rows(int B, int n_q, int group, int H_kv, int G) { return sf::sp_tree_rows(B, n_q, group, H_kv, G); }
"""
TILE, SEG_ONE, SEG_TWO, FEW, ONE, TWO = 128, 5, 10, 4, 3, 4


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree_workspace")
    src, so = os.path.join(d, "t.cpp"), os.path.join(d, "t.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", build_lib.CSRC, src, "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.rows.restype = ctypes.c_longlong
    return lib


def pieces(keys, n_q, group, H_kv, sms):
    """(fold, first partial row, rows) of every piece and row tile."""
    B, per_tile = len(keys), TILE // group
    row_tiles = -(-n_q // per_tile)
    folds = (row_tiles + 1) // 2
    G = sms // folds
    paired = row_tiles == 1 and B * H_kv >= sms
    units, segments, at, slot = (H_kv + 1) // 2 if paired else H_kv, [], 0, 0
    slot_rows = 2 * n_q * group if paired else 2 * TILE if row_tiles > 1 else n_q * group
    for k in keys:
        tiles = -(-k // TILE)
        for u in range(units if k else 0):
            heads = 2 if paired and 2 * u + 1 < H_kv else 1
            start, each = (SEG_TWO, TWO) if row_tiles > 1 else (SEG_ONE, ONE)
            length = start + FEW + each * tiles * heads
            segments.append((at, at + start + FEW, each, tiles * heads, heads, slot))
            at += length
            slot += slot_rows
    if not at:
        return folds, []
    out, chunk = [], -(-at // G)
    for c in range(G):
        low, high = min(c * chunk, at), min((c + 1) * chunk, at)
        for base, first, each, tiles, heads, slot in segments:
            if base >= high or first + each * tiles <= low:
                continue
            t0, t1 = (0 if x <= first else min(-(-(x - first) // each), tiles) for x in (low, high))
            if t1 <= t0:
                continue
            for fold in range(folds):
                mine = min(2 * fold + 2, row_tiles) - 2 * fold
                for s in range(heads if row_tiles == 1 else mine):
                    tile_rows = min(n_q - (2 * fold + s) * per_tile, per_tile) * group if row_tiles > 1 else n_q * group
                    here = slot + 2 * TILE * c + (s * TILE if row_tiles > 1 else s * n_q * group)
                    out.append((fold, here, tile_rows))
    return folds, out


def test_pieces_stay_within_their_fold_and_apart(lib):
    g = random.Random(1)
    seen = set()
    for case in range(600):
        group = g.randint(1, 8)
        n_q, H_kv = g.randint(1, 64), g.choice([1, 2, 3, 4, 5, 8, 16, 31])
        B = g.choice([1, 1, 2, 3, 7, 20, 60, 150])
        most = g.choice([70, 400, 5000, 40000])
        keys = [0 if g.random() < 0.1 else g.randint(n_q, n_q + most) for _ in range(B)]
        sms = g.choice([152, 148, 132])
        folds, got = pieces(keys, n_q, group, H_kv, sms)
        rows = lib.rows(B, n_q, group, H_kv, sms)
        assert rows % folds == 0
        seen.add((folds, n_q * group > TILE, B * H_kv >= sms))
        for fold in range(folds):
            spans = sorted((at, n) for f, at, n in got if f == fold)
            assert all(a + n <= b for (a, n), (b, _) in zip(spans, spans[1:]))
            assert not spans or spans[-1][0] + spans[-1][1] <= rows // folds
    assert len(seen) >= 5


def test_the_bound_grows_with_the_queries_not_with_whole_tiles(lib):
    assert lib.rows(1024, 8, 1, 32, 152) == 1024 * 33 * 8 + 256 * 152
    assert lib.rows(16, 61, 7, 4, 152) == 2 * (16 * 4 * 256 + 256 * 152)
