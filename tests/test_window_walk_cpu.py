"""The key tiles that two query tiles walk under a window (csrc/flash_rows.h, compiled here for the host): every slot that a
row sees lies in exactly one of them, and in none that its query tile sits out."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_15865_gb300", "csrc")
SRC = '''#include "flash_rows.h"
extern "C" void walk(int a, int b, int w, int s, int t, int* out) {
    const attn::WindowWalk x = attn::window_walk(a, b, w, s, t);
    out[0] = x.ns, out[1] = x.skip, out[2] = x.off0, out[3] = x.off1;
}
'''
TILE = 8


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("walk") / "walk.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-x", "c++", "-", "-o", so], input=SRC, text=True,
                   check=True)
    out = (ctypes.c_int * 4)()

    def call(*args):
        ctypes.CDLL(so).walk(*args, out)
        return tuple(out)
    return call


@pytest.mark.parametrize("window", [1, 2, 7, 8, 9, 16, 23, 40, 100])
@pytest.mark.parametrize("sinks", [0, 1, 7, 8, 9, 20, 41, 100])
@pytest.mark.parametrize("tok", [1, 3, 8])
def test_every_slot_that_a_row_sees_is_walked_once(walk, window, sinks, tok):
    for a in range(0, 64, 1 if tok == 3 else 5):
        b = a + tok
        ns, skip, off0, off1 = walk(a, b, window, sinks, TILE)
        assert 0 <= ns and 0 <= skip and ns <= off0 <= off1
        for t, first in ((0, a), (1, b)):
            n = (first + tok + TILE - 1) // TILE - skip
            tiles = [(j if j < ns else j + skip) for j in range(n) if not (t and off0 <= j < off1)]
            assert len(set(tiles)) == len(tiles) and tiles
            for p in range(first, first + tok):
                seen = {s // TILE for s in range(p + 1) if p - s < window or s < sinks}
                assert seen <= set(tiles), (t, p)
            if not t:  # what is read holds something that a row of the pair sees
                live = {s // TILE for p in range(a, b + tok) for s in range(p + 1) if p - s < window or s < sinks}
                n_b = (b + tok + TILE - 1) // TILE - skip
                assert {j if j < ns else j + skip for j in range(n_b)} <= live


def test_the_longest_windows_stay_in_range(walk):
    big = 2 ** 31 - 1
    assert walk(big - 1000, big - 900, big - 1, 0, 128) == (0, 0, 0, 0)
    assert walk(big - 1000, big - 900, 1, big - 500, 128)[1] == 0
