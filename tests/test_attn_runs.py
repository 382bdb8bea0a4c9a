"""The runs of slots that attention's copying lanes take of 4-bit rows (csrc/attn_plan.h, compiled for the host): no
product passes 32 bits at any block size that a view may have, and no slot stands before its tile."""
import ctypes as C
import shutil
import subprocess

import pytest

from .plans import CSRC

_SOURCE = r"""
#include "attn_plan.h"
extern "C" {
int run_slots(int side, int flat, int block_size) { return epikv::run_slots(side, flat, block_size); }
int slots_behind(int n, int s0, int run0, int run) { return epikv::slots_behind(n, s0, run0, run); }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    out = str(tmp_path_factory.mktemp("runs") / "runs.so")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I" + CSRC, "-x", "c++",
                        "-", "-shared", "-fPIC", "-o", out], input=_SOURCE, capture_output=True, text=True)
    if r.returncode:     # a compiler without the sanitizer's runtime: the values alone
        r = subprocess.run([cxx, "-std=c++17", "-O1", "-I" + CSRC, "-x", "c++", "-", "-shared", "-fPIC", "-o", out],
                           input=_SOURCE, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return C.CDLL(out)


@pytest.mark.parametrize("block", [1, 2, 7, 16, 48, 1000, 2 ** 20, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, 2 ** 26, 2 ** 27,
                                   2 ** 30, 2 ** 31 - 1])
@pytest.mark.parametrize("side,flat", [(1, 0), (1, 1), (0, 0), (0, 1)])
def test_every_slot_of_a_tile_once(plan, block, side, flat):
    rl = plan.run_slots(side, flat, block)
    assert 1 <= rl <= 2 ** 24 and (side or rl == 1)
    if side and not flat:
        assert rl == min(block, 2 ** 24)     # within a block, and as long as a sequence can be
    for tile in (16, 64, 512):
        for s0 in (0, tile, 33 * tile, 2 ** 20, 2 ** 24 - tile):
            for n in (0, 1, tile - 1, tile):
                run0 = s0 // rl
                lanes = sum(max(0, min((run0 + k + 1) * rl, s0 + n) - max((run0 + k) * rl, s0)) for k in range(32))
                behind = plan.slots_behind(n, s0, run0, rl)
                assert 0 <= behind <= n and lanes + behind == n, (tile, s0, n)
