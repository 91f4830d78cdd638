"""The shared memory of the attention over shared prefixes (csrc/shared_prefix_layout.h),
compiled for the host: which ring it leaves room for, and that nothing overlaps."""
import ctypes
import os
import subprocess

import pytest

from paper_2505_12728_gb300 import build_lib

SOURCE = """
#include "shared_prefix_layout.h"
using namespace sf;
extern "C" int stages(int D, int B, int G) { return sp_stages(D, B, G); }
extern "C" int bytes(int D, int S, int B, int G) {
  if (D == 128) return S == 5 ? sp_smem_bytes<128, 5>(B, G) : sp_smem_bytes<128, 4>(B, G);
  return S == 10 ? sp_smem_bytes<64, 10>(B, G) : sp_smem_bytes<64, 8>(B, G);
}
template <int D, int S> void put(int *o) {
  using L = SpSmem<D, S>;
  const int v[] = {L::kQOffset, L::kBarOffset, L::kMiscOffset, L::kItemOffset, L::kMlOffset, L::kInfoOffset, L::kPlanOffset,
                   L::kTileBytes, L::kNumBars, kSpItems * static_cast<int>(sizeof(SpItem))};
  for (int i = 0; i < 10; ++i) o[i] = v[i];
}
extern "C" void offsets(int D, int S, int *o) {
  if (D == 128) { if (S == 5) put<128, 5>(o); else put<128, 4>(o); }
  else { if (S == 10) put<64, 10>(o); else put<64, 8>(o); }
}
"""
SMEM = 227 * 1024


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("shared_prefix_layout")
    src, so = os.path.join(d, "t.cpp"), os.path.join(d, "t.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", build_lib.CSRC, src, "-o", so], check=True)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("B, groups", [(1, 1), (2, 1), (8, 1), (16, 1), (16, 16), (32, 4), (48, 8), (64, 1), (64, 4)])
def test_batches_of_ordinary_size_have_the_deep_ring(lib, B, groups):
    assert lib.stages(128, B, groups) == 5
    assert lib.stages(64, B, groups) == 10


def test_every_batch_has_a_ring_that_fits(lib):
    for D, rings in ((128, (5, 4)), (64, (10, 8))):
        for B in list(range(1, 130)) + [500, 1023, 1024]:
            for groups in sorted({1, B // 7 + 1, B // 2 + 1, B}):
                s = lib.stages(D, B, groups)
                assert s in rings and lib.bytes(D, s, B, groups) <= SMEM
                if s == rings[1]:
                    assert lib.bytes(D, rings[0], B, groups) > SMEM


@pytest.mark.parametrize("D, stages", [(128, 5), (128, 4), (64, 10), (64, 8)])
def test_the_parts_do_not_overlap(lib, D, stages):
    o = (ctypes.c_int * 10)()
    lib.offsets(D, stages, o)
    q, bar, misc, item, ml, info, plan, tile, bars, items = o
    assert tile == 128 * D * 2 and q == stages * tile and q % 1024 == 0
    assert bar == q + 2 * tile and bar % 8 == 0
    assert misc == bar + 8 * bars and misc % 4 == 0
    assert item >= misc + 8 and item % 16 == 0
    assert ml >= item + items and ml % 8 == 0
    assert info == ml + 2 * 128 * 8
    assert plan >= info + 8 * 5 * 4 + 4 * 4 and plan % 4 == 0
