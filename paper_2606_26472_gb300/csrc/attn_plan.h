// How attention's work is cut, for the kernels and, compiled for the host, for
// its tests.
//
// An item is (batch entry, group of KV heads, run of query rows): what one
// softmax state per row covers.  Its slots are cut into tiles.  All items'
// tiles stand in one line, entry by entry, which the grid's CTAs take in equal
// contiguous shares; so an item may be spread over several CTAs, each of which
// then leaves a partial result: at most one that starts inside an item (the
// CTA's first) and one that starts an item it does not end (its last).
#pragma once

#include <stdint.h>

#include "plans.h"

namespace epikv {

constexpr int kAttnCtas = 152;   // one per SM of a GB300
constexpr int kAttnWarps = 8;    // warps that compute
constexpr int kAttnGroup = 8;    // KV heads of an item, at most

struct AttnShape {
  int groups;    // of KV heads, kAttnGroup in each but the last
  int rows;      // query rows of an item
  int tile;      // slots of a tile
  int rep;       // query heads of a KV head
  int causal;
};

// Slots that the last of an item's rows sees: query row r of a KV head is
// token r / rep's, and token i of an entry sees len + i + 1 slots.
EPIKV_PLAN int rows_of(const AttnShape& s, int n) { return n * s.rep; }
EPIKV_PLAN int row_runs(const AttnShape& s, int n) { return (n * s.rep + s.rows - 1) / s.rows; }
EPIKV_PLAN int slots_seen(const AttnShape& s, int n, int len, int run) {
  if (!s.causal) return len;
  const int last = (run + 1) * s.rows < n * s.rep ? (run + 1) * s.rows : n * s.rep;
  return len + (last - 1) / s.rep + 1;
}
// An item that sees nothing still has a tile: its rows' zeros are written.
EPIKV_PLAN int item_tiles(const AttnShape& s, int n, int len, int run) {
  const int t = (slots_seen(s, n, len, run) + s.tile - 1) / s.tile;
  return t > 1 ? t : 1;
}
EPIKV_PLAN int64_t entry_tiles(const AttnShape& s, int n, int len) {
  int64_t t = 0;
  for (int r = 0; r < row_runs(s, n); ++r) t += item_tiles(s, n, len, r);
  return t * s.groups;
}

EPIKV_PLAN int64_t first_tile(int cta, int64_t total) { return total * cta / kAttnCtas; }
// The CTA whose share tile x is in.
EPIKV_PLAN int cta_of_tile(int64_t x, int64_t total) { return (int)(((x + 1) * kAttnCtas - 1) / total); }

// ---- shared memory of a CTA: the ring of tiles, boxes to join a head's warps, barriers, the entries' first tiles
constexpr int kAttnSmem = 226 * 1024;   // dynamic shared memory, at most
constexpr int kMaxUnits = 16;           // tiles of the ring
constexpr int kRowsPerLane = 4;         // rows of a tile that a lane of the copying warp looks after

struct AttnGeometry {
  AttnShape sh;
  int row_s;         // bytes between a tile's rows in shared memory
  int unit_bytes;    // one tile of K or V
  int units;         // tiles in the ring
  int join_off, bar_off, pre_off, smem_bytes;   // behind the ring
  int slot_floats;   // of a CTA's partial result
};

// 8-row blocks of queries of an item: as many as the registers hold (256 / d) and the call's rows fill.
EPIKV_PLAN int attn_row_blocks(int d, int rep, int max_new) {
  const int64_t want = ((int64_t)max_new * rep + 7) / 8;
  int nt = 1;
  while (nt < 256 / d && nt < want) nt *= 2;
  return nt;
}
// 16-slot blocks of a tile that a warp takes.
constexpr int attn_sub_blocks(bool q4, int nt) { return q4 && nt == 1 ? 2 : 1; }
// Warps of a head in a group of so many heads: 8, 4, 2 or 1.
EPIKV_PLAN int attn_teams(int heads) { return kAttnWarps / heads; }
// What a warp leaves for another to join: its outputs, maxima and sums.
constexpr int attn_box_floats(int d, int nt) { return (d / 16 * nt * 4 + 4 * nt) * 32; }

EPIKV_PLAN AttnGeometry attn_geometry(int H, int rep, int d, bool q4, int n_seq, int max_new, bool causal) {
  AttnGeometry ge;
  const int nt = attn_row_blocks(d, rep, max_new);
  const int heads = H < kAttnGroup ? H : kAttnGroup;              // of the first group
  const int rest = H > kAttnGroup && H % kAttnGroup ? H % kAttnGroup : heads;   // of the last one
  int tile = 16 * attn_teams(heads) * attn_sub_blocks(q4, nt);
  if (tile > 32 * kRowsPerLane) tile = 32 * kRowsPerLane;
  ge.sh = {(H + kAttnGroup - 1) / kAttnGroup, nt * 8, tile, rep, causal ? 1 : 0};
  if (!q4) {
    ge.row_s = heads * d * 2 + 16;           // 16 past a multiple of 128: eight rows' 16-byte pieces fill the banks
  } else {
    const int used = heads * (d / 2) + ((heads * (d / 16) + 15) & ~15);
    ge.row_s = used + ((32 - used) & 127);   // 32 past a multiple of 128
  }
  ge.unit_bytes = (ge.sh.tile * ge.row_s + 127) & ~127;
  // any group whose heads have several warps needs the boxes: half of the warps write one at a time
  const bool join = attn_teams(heads) > 1 || attn_teams(rest) > 1;
  const int boxes = join ? kAttnWarps / 2 * attn_box_floats(d, nt) * 4 : 0;
  const int bars = (2 * kMaxUnits + 1) * 8, pre = (n_seq + 1) * 8;
  ge.units = (kAttnSmem - boxes - bars - pre) / ge.unit_bytes;
  if (ge.units > kMaxUnits) ge.units = kMaxUnits;
  ge.join_off = ge.units * ge.unit_bytes;
  ge.bar_off = ge.join_off + boxes;
  ge.pre_off = ge.bar_off + bars;
  ge.smem_bytes = ge.pre_off + pre;
  ge.slot_floats = kAttnGroup * ge.sh.rows * (d + 2);
  return ge;
}

}  // namespace epikv
