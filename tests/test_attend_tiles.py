"""Tiles of slots that the attention kernels go over (rkc_tiles.h), compiled for the host: every slot that a row sees is in
one of them, and no table entry is looked up that the sequence does not have."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_24259_amd", "csrc")
SOURCE = r"""
#include "rkc_tiles.h"
// n; slots of the tiles; slots that were looked up, and loaded, before the loop (ahead = 2 or the kernel's 1, 3)
template <int STEP, int AHEAD> int walk(int c0, int end, int pre, int any_from, int* slot, int* looked, int* loaded) {
  const rkc_tiles<STEP> t(c0, end, pre, any_from);
  for (int i = 0; i < t.n; i++) slot[i] = t.slot(i);
  int a = 0, b = 0;
  rkc_first_tiles<AHEAD>(t.n, [&](int i) { looked[a++] = t.slot(i); }, [&](int i, int place) { loaded[b++] = t.slot(i), loaded[b++] = place; });
  looked[a] = loaded[b] = -1;
  return t.n;
}
extern "C" int tiles(int step, int ahead, int c0, int end, int pre, int any_from, int* slot, int* looked, int* loaded) {
  if (step == 32) return ahead == 2 ? walk<32, 2>(c0, end, pre, any_from, slot, looked, loaded) : walk<32, 3>(c0, end, pre, any_from, slot, looked, loaded);
  return ahead == 1 ? walk<64, 1>(c0, end, pre, any_from, slot, looked, loaded) : ahead == 2 ? walk<64, 2>(c0, end, pre, any_from, slot, looked, loaded)
                                                                                             : walk<64, 3>(c0, end, pre, any_from, slot, looked, loaded);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    src, so = d / "tiles.cpp", d / "libtiles.so"
    src.write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unknown-pragmas", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)])
    return ctypes.CDLL(str(so))


@pytest.mark.parametrize("step,ahead", [(32, 2), (32, 3), (64, 1), (64, 2), (64, 3)])
def test_tiles(lib, step, ahead):
    """Sequences of whole and of broken tiles, whole ones and parts, prefixes, and rows that begin anywhere, also behind the
    last slot."""
    ints = ctypes.c_int * 64
    slot, looked, loaded = ints(), ints(), ints()
    empty = 0
    for c0 in (0, 256):
        for end in [c0 + x for x in (1, 15, 16, 33, 63, 64, 65, 128, 200, 256)]:
            for pre in (0, 1, 31, 64, 100, end):
                if pre > end:
                    continue
                for any_from in (0, 1, 31, 32, 64, 97, c0 + 64, end - 1, end, end + 1, 1 << 30, (1 << 31) - 1):
                    n = lib.tiles(step, ahead, c0, end, pre, any_from, slot, looked, loaded)
                    at = slot[:n]
                    seen = [j for j in range(c0, end) if j < pre or j >= any_from]
                    assert at == sorted(set(at)) and all(t % step == 0 and c0 <= t < end for t in at)
                    assert all(j // step * step in at for j in seen)
                    first = looked[: list(looked).index(-1)]
                    assert first == at[: ahead + 1]  # nothing of a sequence without tiles: its table may end at `end`
                    assert loaded[: list(loaded).index(-1)] == [x for i, t in enumerate(at[:ahead]) for x in (t, i)]
                    empty += n == 0
    assert empty


def test_kernels_go_by_them():
    """No other place looks a page up before the loop."""
    text = open(os.path.join(CSRC, "rkc_attend_tile.hip")).read()
    assert text.count("rkc_first_tiles<") == 2 and "look_up(0)" not in text and text.count("rkc_tiles<BK>") == 1
