"""How the chunk's attention and the weights cut their work (csrc/chunk_plan.h), compiled for the host and walked share by
share as the kernels walk it: every tile and step once, in order, parts counted as the joining kernels count them."""
import ctypes as C
import itertools
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_26472_gb300", "csrc")

_SOURCE = r"""
#include "chunk_plan.h"
using namespace epikv;
extern "C" {
static ChunkPlan cp(const int* p) { return {p[0], p[1], p[2], p[3], p[4], p[5], p[6]}; }
int64_t chunk_places(const int* p, int n, int len) { return head_places(cp(p), n, len); }
int chunk_block_count(const int* p, int n) { return chunk_blocks(cp(p), n); }
int chunk_block_places(const int* p, int n, int len, int b) { return block_places(cp(p), n, len, b); }
int chunk_sees(const int* p, int n, int len, int b) { return block_sees(cp(p), n, len, b); }
int chunk_row_sees(const int* p, int len, int r) { return row_sees(cp(p), len, r); }
int chunk_tile_of(int places) { return tile_of_place(places); }
int chunk_cta_count(unsigned total, int64_t items) { return chunk_ctas(total, items); }
unsigned chunk_start(int c, unsigned total, int ctas) { return share_start(c, total, ctas); }
unsigned chunk_moved(unsigned x, unsigned at, unsigned places) { return moved_start(x, at, places); }
int chunk_last(unsigned at, unsigned places, unsigned total, int ctas) { return last_share(at, places, total, ctas); }
static WeightPlan wp(const int* p) { return {p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8]}; }
int64_t weight_line(const int* p, int n, int len) { return weight_entry(wp(p), n, len); }
int weight_unit_count(const int* p, int n, int len) { return weight_units(wp(p), n, len); }
int weight_unit_places(const int* p, int n, int len, int u) { return weight_places(wp(p), n, len, u); }
int weight_unit_steps(const int* p, int n, int len, int u) { return weight_steps(wp(p), n, len, u); }
int weight_unit_token(const int* p, int n, int len, int u) { return weight_token(wp(p), n, len, u); }
int weight_step_of(const int* p, int places) { return step_of_place(wp(p), places); }
unsigned weight_moved(const int* p, unsigned x, unsigned at) { return moved_unit_start(wp(p), x, at); }
int weight_share_of(unsigned x, unsigned total, int ctas) { return share_of(x, total, ctas); }
int apart(int S, int H, int T, int64_t a, int64_t b) { return weights_apart(S, H, T, a, b); }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    out = str(tmp_path_factory.mktemp("plan") / "plan.so")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Wno-unknown-pragmas", "-I" + CSRC, "-shared", "-fPIC", "-x", "c++",
                        "-", "-o", out], input=_SOURCE, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lib = C.CDLL(out)
    for f in ("chunk_places", "weight_line"):
        getattr(lib, f).restype = C.c_int64
    for f in ("chunk_start", "chunk_moved", "weight_moved"):
        getattr(lib, f).restype = C.c_uint
    lib.chunk_cta_count.argtypes = [C.c_uint, C.c_int64]
    lib.apart.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int64]
    return lib


def batches(rng, count):
    yield [(1, 0)]
    yield [(4096, 0)]
    yield [(16, 4096)] * 8
    yield [(2048, 14336)]
    yield [(1, 65535)]
    yield [(0, 5), (1, 0), (0, 0), (3, 7)]
    for _ in range(count):
        n = int(rng.integers(1, 12))
        yield [(int(rng.choice([0, 1, 2, rng.integers(1, 300), rng.integers(1, 3000)])),
                int(rng.choice([0, 1, rng.integers(0, 300), rng.integers(0, 20000)]))) for _ in range(n)]


@pytest.mark.parametrize("rows,slots,rep,heads,causal", [(256, 128, 4, 8, 1), (128, 64, 1, 1, 1), (128, 128, 7, 3, 1),
                                                         (256, 128, 71, 2, 1), (256, 128, 4, 2, 0), (128, 64, 8, 4, 0)])
def test_chunks(plan, rows, slots, rep, heads, causal):
    p = (C.c_int * 7)(rows, slots, rows.bit_length() - 1, slots.bit_length() - 1, rep, causal, heads)
    for batch in batches(np.random.default_rng(rows + rep), 25):
        items, at = [], 0
        for b, (n, ln) in enumerate(batch):
            blocks = plan.chunk_block_count(p, n)
            assert blocks == -(-n * rep // rows)
            assert plan.chunk_places(p, n, ln) == sum(plan.chunk_block_places(p, n, ln, i) for i in range(blocks))
            for h, i in itertools.product(range(heads), range(blocks)):
                sees = plan.chunk_sees(p, n, ln, i)
                assert sees == (ln + (min((i + 1) * rows, n * rep) - 1) // rep + 1 if causal else ln)
                assert plan.chunk_row_sees(p, ln, i * rows) <= sees
                places = plan.chunk_block_places(p, n, ln, i)
                items.append((at, places, -(-sees // slots)))
                at += places
        total = at
        if not total:
            continue
        ctas = plan.chunk_cta_count(total, len(items))
        assert 1 <= ctas <= min(152, total)

        def moved(x):
            if x == total:
                return total
            k = np.searchsorted([i[0] for i in items], x, side="right") - 1
            return plan.chunk_moved(x, items[k][0], items[k][1])

        starts = [moved(plan.chunk_start(c, total, ctas)) for c in range(ctas)] + [total]
        assert starts[0] == 0 and all(a <= b for a, b in zip(starts, starts[1:]))
        for at, places, tiles in items:
            mine = [c for c in range(ctas) if max(starts[c], at) < min(starts[c + 1], at + places)]
            assert mine == list(range(mine[0], mine[-1] + 1))
            seen = []
            for c in mine:
                a, e = max(starts[c], at) - at, min(starts[c + 1], at + places) - at
                t0, t1 = plan.chunk_tile_of(a), plan.chunk_tile_of(e)
                seen += range(t0, t1)
                if len(mine) > 1:
                    assert t1 - t0 >= 1                       # a part holds something
            assert seen == list(range(tiles))
            if len(mine) > 1:
                assert plan.chunk_last(at, places, total, ctas) - mine[0] + 1 == len(mine)


@pytest.mark.parametrize("slots,rows,rep,heads,causal,last,extra", [
    (256, 128, 4, 8, 1, 0, 4), (256, 128, 6, 4, 1, 64, 4), (128, 128, 7, 3, 1, 5, 4), (256, 16, 4, 8, 1, 0, 0),
    (128, 16, 16, 1, 1, 1, 0), (256, 128, 4, 2, 0, 0, 4), (256, 128, 71, 1, 1, 0, 4), (256, 16, 1, 3, 0, 0, 0)])
def test_weights(plan, slots, rows, rep, heads, causal, last, extra):
    p = (C.c_int * 9)(slots, slots.bit_length() - 1, rows, rows.bit_length() - 1, rep, causal, heads, last, extra)
    for batch in batches(np.random.default_rng(slots + rep + last), 25):
        if not extra:                                           # one step a unit at most, as that form's calls have
            batch = [(min(n, max(1, rows // rep)), ln) for n, ln in batch]
        units, at = [], 0
        for n, ln in batch:
            top = ln + (n if causal else 0)
            count = plan.weight_unit_count(p, n, ln)
            assert count == -(-top // slots)
            first = max(0, n - last) if last else 0
            for u, _ in itertools.product(range(count), range(heads)):
                token = plan.weight_unit_token(p, n, ln, u)
                # the first token that counts and sees the unit's first slot
                sees = [i for i in range(first, n) if u * slots < (ln + i + 1 if causal else ln)]
                assert not sees or token == sees[0]
                steps = plan.weight_unit_steps(p, n, ln, u)
                assert steps == -(-len(sees) * rep // rows)
                places = plan.weight_unit_places(p, n, ln, u)
                assert places == max(1, steps + extra)
                units.append((at, places, steps))
                at += places
            assert plan.weight_line(p, n, ln) == sum(x[1] for x in units[len(units) - count * heads:])
        total = at
        if not total:
            continue
        ctas = min(total, 152)

        def moved(x):
            if x == total:
                return total
            k = np.searchsorted([i[0] for i in units], x, side="right") - 1
            return plan.weight_moved(p, x, units[k][0])

        starts = [moved(plan.chunk_start(c, total, ctas)) for c in range(ctas)] + [total]
        assert starts[0] == 0 and all(a <= b for a, b in zip(starts, starts[1:]))
        for at, places, steps in units:
            mine = [c for c in range(ctas) if max(starts[c], at) < min(starts[c + 1], at + places)]
            assert mine == list(range(mine[0], mine[-1] + 1))
            seen = []
            for c in mine:
                a, e = max(starts[c], at) - at, min(starts[c + 1], at + places) - at
                s0, s1 = plan.weight_step_of(p, a), min(plan.weight_step_of(p, e), steps)
                seen += range(s0, s1)
                if len(mine) > 1:
                    assert s1 > s0
            assert seen == list(range(steps))
            if len(mine) > 1:
                assert extra and plan.weight_share_of(at + places - 1, total, ctas) - mine[0] + 1 == len(mine)


def test_rows_of_weights_apart(plan):
    """Against the intervals themselves."""
    rng = np.random.default_rng(0)
    for _ in range(4000):
        S, H, T = (int(x) for x in rng.integers(1, 6, 3))
        ss, sh = (int(x) for x in rng.integers(-2, 40, 2))
        rows = [(s * ss + h * sh, s * ss + h * sh + T) for s in range(S) for h in range(H)]
        rows.sort()
        free = ss >= 0 and sh >= 0 and all(a[1] <= b[0] for a, b in zip(rows, rows[1:]))
        said = plan.apart(S, H, T, ss, sh)
        assert not said or free                                  # never taken where they meet
        if free and (S == 1 or H == 1 or max(ss, sh) >= (min(ss, sh) * ((S if ss < sh else H) - 1) + T)):
            assert said
    big = 1 << 60
    assert plan.apart(2, 2, 5, big, big // 2) == 1 and plan.apart(4096, 32, 1 << 24, 1 << 24, 1 << 24) == 0


def simulate(stages, warps, steps, rng, consumers_lag):
    """Warps that take turns at a ring's stages, each waiting with one bit of a phase count: a stage is never written while
    its last step is in use, and nobody waits for ever."""
    done = [0] * stages                       # phases completed: steps consumed of each stage
    filled = set()
    consumed = 0
    nxt = list(range(warps))
    while consumed < steps:
        moved = False
        for w in rng.permutation(warps):
            s = nxt[w]
            if s >= steps:
                continue
            q = s % stages
            if s >= stages and done[q] % 2 == (s // stages - 1) % 2:
                continue                      # the wait for phase s / stages - 1 blocks while that parity is current
            assert done[q] == s // stages, "written too early"
            filled.add(s)
            nxt[w] = s + warps
            moved = True
            if rng.random() < 0.5:
                break
        if consumed in filled and rng.random() < consumers_lag:
            done[consumed % stages] += 1
            consumed += 1
            moved = True
        elif consumed in filled:
            moved = True
        assert moved, "everybody waits"


@pytest.mark.parametrize("stages,warps", [(5, 4), (4, 4), (3, 3), (2, 2)])
def test_turns_at_a_ring(stages, warps):
    """The pairs that the weights of few rows use: as many warps as stages, at most."""
    rng = np.random.default_rng(stages)
    for lag in (0.05, 0.5, 1.0):
        for _ in range(30):
            simulate(stages, warps, 60, rng, lag)


def test_more_warps_than_stages_would_not_do():
    with pytest.raises(AssertionError):
        for seed in range(200):
            simulate(3, 4, 60, np.random.default_rng(seed), 0.1)
