"""Attention's plan (csrc/attn_plan.h, compiled for the host): every configuration's shared memory holds what its warps
address, and the CTAs' shares cover each item's tiles once, with at most one partial result of either kind per CTA."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from .plans import CSRC

_SOURCE = r"""
#include "attn_plan.h"
using namespace epikv;
#define NEED(x) do { if (!(x)) return __LINE__; } while (0)
extern "C" {
// 0, or the line of the first check that fails
int geometry_holds(int H, int rep, int d, int q4, int units, int slots, int n_seq, int max_new) {
  const AttnGeometry g = attn_geometry(H, rep, d, q4, units, slots, n_seq, max_new, true);
  const int nt = attn_row_blocks(d, rep, max_new), sub = g.sub, group = attn_group(d);
  NEED(g.stages >= 2 && g.stages <= kMaxStages && g.smem_bytes <= kAttnSmem);
  NEED(g.copiers >= 1 && g.copiers <= kAttnCopyWarps && g.copiers <= g.stages);
  NEED(g.sh.rows == 1 << g.sh.rows_log && g.sh.tile == 1 << g.sh.tile_log);
  NEED(g.sh.rows == 8 * nt && nt * d <= 256);
  NEED(g.sh.tile % 16 == 0 && g.sh.tile >= 16 && g.sh.tile <= (q4 ? 512 : 128));
  unsigned rows = 0;
  for (int r = 0; r < 8; ++r) rows |= 1u << (g.order >> (4 * r) & 7);
  NEED(rows == 255 && !(g.order & 0x88888888u));
  NEED(g.row_s % 16 == 0 && g.half_bytes % 1024 == 0 && g.half_bytes >= g.sh.tile * g.row_s);
  NEED(g.join_off >= g.stages * 2 * g.half_bytes && g.join_off % 16 == 0 && g.bar_off % 8 == 0 && g.pre_off % 8 == 0);
  NEED(g.pre_off >= g.bar_off + (2 * kMaxStages + 1) * 8 && g.smem_bytes >= g.pre_off + (n_seq + 1) * 4);
  NEED(g.sh.groups * group >= H && (g.sh.groups - 1) * group < H);
  for (int i = 0; i < g.sh.groups; ++i) {
    const int heads = H - i * group < group ? H - i * group : group;
    const int teams = attn_teams(heads, group);
    NEED(teams == 1 || teams == 2 || teams == 4 || teams == 8);
    NEED(teams * heads <= group);
    for (int s = 0; s < g.sh.tile / 16; ++s) {   // each block of 16 slots is one team's, within its reach
      int n = 0;
      for (int team = 0; team < teams; ++team)
        for (int u = 0; u < sub; ++u) n += u * teams + team == s;
      NEED(n == 1);
    }
    const int row = q4 ? heads * (d / 2) + ((heads * (d / 16) + 15) & ~15) : heads * d * 2;
    NEED(row <= g.row_s);
    for (int step = teams / 2; step > 0; step >>= 1)
      for (int team = 0; team < step; ++team)
        for (int head = 0; head < heads; ++head)
          NEED(g.join_off + (int64_t)(team * heads + head + 1) * attn_box_floats(d, nt) * 4 <= g.bar_off);
  }
  const AttnGeometry most = attn_geometry(H, rep, d, q4, units, slots, 1, max_new, true);   // what the workspace is sized by
  for (int n = 1; n <= max_new; n *= 2) NEED(attn_geometry(H, rep, d, q4, units, slots, n_seq, n, false).slot_floats <= most.slot_floats);
  return 0;
}

int shares_hold(int H, int rep, int d, int q4, int units, int slots, int max_new, int causal, int n_seq, const int* n, const int* len) {
  const AttnGeometry g = attn_geometry(H, rep, d, q4, units, slots, n_seq, max_new, causal);
  int64_t sum = 0;
  for (int b = 0; b < n_seq; ++b) sum += entry_tiles(g.sh, n[b], len[b]);
  if (!sum) return 0;
  NEED(sum < int64_t(1) << 31);
  const int total = (int)sum;
  for (int c = 0; c <= kAttnCtas; ++c) NEED(first_tile(c, total) == sum * c / kAttnCtas);
  NEED(first_tile(0, total) == 0 && first_tile(kAttnCtas, total) == total);
  for (int c = 0; c < kAttnCtas; ++c) NEED(first_tile(c, total) <= first_tile(c + 1, total));
  int parts[kAttnCtas][2] = {};
  int at = 0;
  for (int b = 0; b < n_seq; ++b)
    for (int group = 0; group < g.sh.groups; ++group)
      for (int run = 0; run < row_runs(g.sh, n[b]); ++run) {
        const int t = item_tiles(g.sh, n[b], len[b], run);
        NEED(t >= 1 && slots_seen(g.sh, n[b], len[b], run) <= len[b] + (causal ? n[b] : 0));
        NEED((int64_t)t * g.sh.tile >= slots_seen(g.sh, n[b], len[b], run));
        const int c0 = cta_of_tile(at, total), c1 = cta_of_tile(at + t - 1, total);
        NEED(c0 >= 0 && c1 >= c0 && c1 < kAttnCtas);
        for (int x = at; x < at + t; ++x) {
          const int c = cta_of_tile(x, total);
          NEED(first_tile(c, total) <= x && x < first_tile(c + 1, total));
        }
        if (c0 != c1)
          for (int c = c0; c <= c1; ++c) {
            if (first_tile(c, total) == first_tile(c + 1, total)) continue;
            const int kind = at < first_tile(c, total) ? 0 : 1;   // as the computing kernel stores it
            NEED(kind == (c == c0 ? 1 : 0));                      // as the joining kernel looks for it
            NEED(++parts[c][kind] == 1);
          }
        at += t;
      }
  NEED(at == total);
  return 0;
}
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    out = str(tmp_path_factory.mktemp("plan") / "plan.so")
    r = subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-I" + CSRC, "-x", "c++", "-", "-shared", "-fPIC", "-o", out],
                       input=_SOURCE, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert os.path.exists(out)
    return C.CDLL(out)


def units_of(H, d, q4):
    from paper_2606_26472_gb300 import build, epikv as E
    build.build()
    h, x = E.epikv_cache_row(H, d, E.EPIKV_CACHE_E2M1 if q4 else E.EPIKV_CACHE_BF16)
    return h * x


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("q4", [0, 1])
def test_shared_memory(plan, d, q4):
    for H in range(1, 33):
        if (H * d > 2048 and not q4) or (q4 and H * (d // 2 + d // 16) > 4096):
            continue
        units = units_of(H, d, q4)
        for rep in (1, 2, 3, 4, 7, 8, 9, 71):
            for n_seq in (1, 64, 4096):
                for max_new, slots in ((1, 100), (1, 1 << 20), (2, 100), (5, 1 << 24), (64, 3000), (4096, 70000)):
                    assert plan.geometry_holds(H, rep, d, q4, units, slots, n_seq, max_new) == 0, (H, rep, n_seq, max_new)


def test_shares(plan):
    import random
    rng = random.Random(0)
    for _ in range(400):
        H, rep, d, q4 = rng.randint(1, 12), rng.choice([1, 3, 4, 8, 71]), rng.choice([64, 128]), rng.randint(0, 1)
        n_seq = rng.choice([1, 1, 3, 20, 200])
        most = rng.choice([1, 1, 4, 40])
        n = [rng.randint(0 if rng.random() < 0.3 else 1, most) for _ in range(n_seq)]
        ln = [rng.choice([0, 1, 15, 16, 17, rng.randint(0, 3000)]) for _ in range(n_seq)]
        causal = rng.randint(0, 1)
        arr = C.c_int * n_seq
        assert plan.shares_hold(H, rep, d, q4, units_of(H, d, q4), rng.choice([5000, 1 << 22]), max(max(n), 1), causal, n_seq, arr(*n), arr(*ln)) == 0, (H, rep, d, q4, n, ln)
