"""How attention counts a batch's tiles (csrc/attn_plan.h, compiled for the host): prompts of ordinary lengths are taken
whatever stands beside them, sums that pass 32 bits stop in the same place however they are formed, and the CTAs' shares
hold up to the largest sum."""
import ctypes as C
import random
import shutil
import subprocess

import pytest

from .plans import CSRC

_SOURCE = r"""
#include "attn_plan.h"
using namespace epikv;
extern "C" {
int64_t tiles_of(int H, int rep, int d, int q4, int units, int slots, int n_seq, int max_new, int causal, int n, int len) {
  return entry_tiles(attn_geometry(H, rep, d, q4, units, slots, n_seq, max_new, causal).sh, n, len);
}
unsigned counted(int64_t t) { return count_of(t); }
unsigned added(unsigned a, unsigned b) { return add_counts(a, b); }
// 0, or the line of the first check that fails
int shares_hold(int total) {
  for (int c = 0; c <= kAttnCtas; ++c)
    if (first_tile(c, total) != (int64_t)total * c / kAttnCtas) return __LINE__;
  for (int c = 0; c < kAttnCtas; ++c) {
    const int lo = first_tile(c, total), hi = first_tile(c + 1, total);
    if (lo == hi) continue;
    if (cta_of_tile(lo, total) != c || cta_of_tile(hi - 1, total) != c || cta_of_tile(lo + (hi - lo) / 2, total) != c) return __LINE__;
  }
  return 0;
}
}
"""
TOO_MANY = 2 ** 31 - 1


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    out = str(tmp_path_factory.mktemp("counts") / "counts.so")
    r = subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-I" + CSRC, "-x", "c++", "-", "-shared", "-fPIC", "-o", out],
                       input=_SOURCE, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lib = C.CDLL(out)
    lib.tiles_of.restype = C.c_int64
    lib.counted.argtypes, lib.counted.restype = [C.c_int64], C.c_uint
    lib.added.argtypes, lib.added.restype = [C.c_uint, C.c_uint], C.c_uint
    return lib


@pytest.mark.parametrize("H,rep,d,new,held", [(8, 4, 128, 32768, 0), (8, 4, 128, 4096, 131072), (8, 8, 256, 20000, 0),
                                              (8, 4, 128, 131072, 0), (16, 4, 128, 65536, 65536), (32, 1, 64, 200000, 0)])
def test_prompts_are_taken(plan, H, rep, d, new, held):
    tiles = plan.tiles_of(H, rep, d, 0, H * d, new + held, 1, new, 1, new, held)
    assert 2 ** 23 < tiles < TOO_MANY
    assert plan.counted(tiles) == tiles < TOO_MANY


def test_sums_do_not_depend_on_their_order(plan):
    rng = random.Random(1)
    for _ in range(300):
        n = rng.choice([3, 40, 700])
        t = [rng.choice([0, 1, 1000, rng.randint(0, 2 ** 23), rng.randint(0, 2 ** 30), 2 ** 31, 2 ** 44]) if rng.random() < 0.1
             else rng.randint(0, 100) for _ in range(n)]
        c = [plan.counted(x) for x in t]
        want = min(sum(t), TOO_MANY)
        ahead = 0
        for x in c:
            ahead = plan.added(ahead, x)
        pairs = list(c)                        # as a tree
        while len(pairs) > 1:
            pairs = [plan.added(*pairs[i:i + 2]) if i + 1 < len(pairs) else pairs[i] for i in range(0, len(pairs), 2)]
        assert ahead == pairs[0] == want


def test_shares_of_large_sums(plan):
    rng = random.Random(2)
    for total in [1, 151, 152, 153, 2 ** 23, 2 ** 24 + 1, TOO_MANY - 1, TOO_MANY - 2] + [rng.randint(2 ** 24, TOO_MANY - 1) for _ in range(200)]:
        assert plan.shares_hold(total) == 0, total
