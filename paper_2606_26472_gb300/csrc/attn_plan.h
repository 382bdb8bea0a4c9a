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
constexpr int kAttnCopyWarps = 4;   // warps that copy, at most
// KV heads of an item, at most, and warps that compute: a head's 16 slots of K and V are 8 KB at d = 128 in bf16, and a
// ring needs several tiles.
constexpr int attn_group(int d) { return d == 256 ? 4 : 8; }

struct AttnShape {
  int groups;    // of KV heads, attn_group(d) in each but the last
  int rows;      // query rows of an item, 1 << rows_log
  int tile;      // slots of a tile, 1 << tile_log
  int rows_log, tile_log;
  int rep;       // query heads of a KV head
  int causal;
};

// Slots that the last of an item's rows sees: query row r of a KV head is
// token r / rep's, and token i of an entry sees len + i + 1 slots.
EPIKV_PLAN int rows_of(const AttnShape& s, int n) { return n * s.rep; }
EPIKV_PLAN int row_runs(const AttnShape& s, int n) { return (n * s.rep + s.rows - 1) >> s.rows_log; }
EPIKV_PLAN int slots_seen(const AttnShape& s, int n, int len, int run) {
  if (!s.causal) return len;
  const int end = (run + 1) << s.rows_log;
  return end >= n * s.rep ? len + n : len + (end - 1) / s.rep + 1;
}
// An item that sees nothing still has a tile: its rows' zeros are written.
EPIKV_PLAN int item_tiles(const AttnShape& s, int n, int len, int run) {
  const int t = (slots_seen(s, n, len, run) + s.tile - 1) >> s.tile_log;
  return t > 1 ? t : 1;
}
EPIKV_PLAN int64_t entry_tiles(const AttnShape& s, int n, int len) {
  int64_t t = 0;
  for (int r = 0; r < row_runs(s, n); ++r) t += item_tiles(s, n, len, r);
  return t * s.groups;
}

// A batch's tiles are counted in 32 bits.  Sums that would reach kTooManyTiles stay there, in whatever order they are
// formed: the entry that takes the sum there and those behind it are refused.
constexpr unsigned kTooManyTiles = 0x7fffffffu;
EPIKV_PLAN unsigned count_of(int64_t tiles) { return tiles < (int64_t)kTooManyTiles ? (unsigned)tiles : kTooManyTiles; }
EPIKV_PLAN unsigned add_counts(unsigned a, unsigned b) {   // neither above kTooManyTiles: no carry
  const unsigned s = a + b;
  return s < kTooManyTiles ? s : kTooManyTiles;
}

// floor(total * cta / kAttnCtas) without 64-bit products
EPIKV_PLAN int first_tile(int cta, int total) {
  const unsigned q = (unsigned)total / kAttnCtas, r = (unsigned)total % kAttnCtas;
  return (int)(q * cta + r * cta / kAttnCtas);
}
// The CTA whose share tile x is in.
EPIKV_PLAN int cta_of_tile(int x, int total) {
  int c = (int)((float)x * (float)kAttnCtas / (float)total);   // near it; put right by the shares themselves
  if (c > kAttnCtas - 1) c = kAttnCtas - 1;
  while (first_tile(c, total) > x) --c;
  while (first_tile(c + 1, total) <= x) ++c;
  return c;
}

// ---- runs of slots whose rows are one piece of memory, each of which a lane copies
constexpr int kMostSlots = 1 << 24;   // of a sequence: a block that holds more is as good as one that holds so many
// `side`: a token's rows stand side by side; `flat`: without blocks.
EPIKV_PLAN int run_slots(bool side, bool flat, int block_size) {
  return !side ? 1 : flat || block_size > kMostSlots ? kMostSlots : block_size;
}
// Of a tile's n slots from s0 on, which lie in run run0 and those behind it: slots behind the 32 lanes' runs.
EPIKV_PLAN int slots_behind(int n, int s0, int run0, int run) {
  const int rest = n - (32 * run - (s0 - run0 * run));
  return rest > 0 ? rest : 0;
}

// ---- shared memory of a CTA: the ring of tiles, boxes to join a head's warps, barriers, the entries' first tiles
constexpr int kAttnSmem = 225 * 1024;   // dynamic shared memory, at most (its start is moved up to a multiple of 1,024)
constexpr int kMaxStages = 8;           // tiles of the ring

struct AttnGeometry {
  AttnShape sh;
  int row_s;         // bytes between a tile's rows in shared memory
  int half_bytes;    // a tile's K (its V follows)
  int stages;        // tiles in the ring
  int copiers;       // copying warps: each takes every copiers-th tile
  int join_off, bar_off, pre_off, smem_bytes;   // behind the ring
  int sub;           // 16-slot blocks of a tile that a warp takes
  int slot_floats;   // of a CTA's partial result
  uint32_t order;    // 4-bit rows: nibble r, the slot of eight that row r of the tensor instruction's rows takes
};

// Shared memory serves a quarter warp's 16-byte loads (the codes of keys: two rows, four lanes each) or a half warp's
// 8-byte ones (of values: every second row, four lanes each) at once if they fall on different banks.  Rows r bytes
// apart, mod 128:
//   32, 96   rows 0 2 1 3 6 4 7 5: neighbours differ by 2 mod 4, every second one by 0, 1, 2, 3
//   64       rows 0 1 3 2 4 5 7 6: neighbours differ by an odd number; the values' loads go in two
//   else     as they stand (one, two or more heads in a row that is not padded: at worst four ways)
EPIKV_PLAN uint32_t attn_row_order(int row_s) {
  const int r = row_s & 127;
  return r == 32 || r == 96 ? 0x57463120u : r == 64 ? 0x67542310u : 0x76543210u;
}

// 8-row blocks of queries of an item: as many as the registers hold (256 / d) and the call's rows fill.
EPIKV_PLAN int attn_row_blocks(int d, int rep, int max_new) {
  const int64_t want = ((int64_t)max_new * rep + 7) / 8;
  int nt = 1;
  while (nt < 256 / d && nt < want) nt *= 2;
  return nt;
}
// 16-slot blocks of a tile that a warp takes of 4-bit rows (bf16: one, whose tiles are 64 KB at 8 x 128): what a tile
// costs besides its products (waits, the check against the maximum) is shared by so many.  Four where the caches, if
// full, give each CTA 16 such tiles (`slots`: of all entries; 32 x 8,256 slots two 77, four 75 us; d = 64, 32 x 16,384 92
// and 82), else two (4 x 136 slots two 14.4, four 18.1 us; one sequence of 65,536 34.1 and 34.9).  The host knows what
// the caches can hold, not what they do: 32 sequences of 131,072 slots that hold 500 to 1,000 take 23.0 with four, 22.0
// with two, 2,000 to 4,000 42.8 and 41.3, 500 to 8,000 53.3 and 51.0.  A caller whose caches stay that far from full
// does better with the capacity that they reach as max_cache_tokens.
EPIKV_PLAN int attn_sub_blocks(bool q4, int d, int nt, int64_t slots) {
  return !q4 ? 1 : nt == 1 && d <= 128 && slots >= (int64_t)kAttnCtas * 16 * 64 ? 4 : 2;
}
// Warps of a head in a group of so many heads: 8, 4, 2 or 1.
EPIKV_PLAN int attn_teams(int heads, int warps) {
  const int t = warps / heads;
  return t >= 8 ? 8 : t >= 4 ? 4 : t >= 2 ? 2 : 1;
}
// What a warp leaves for another to join: its outputs, maxima and sums.
constexpr int attn_box_floats(int d, int nt) { return (d / 16 * nt * 4 + 4 * nt) * 32; }

// units: 2-byte units of a cache row; slots: of a sequence's cache.
EPIKV_PLAN AttnGeometry attn_geometry_of(int H, int rep, int d, bool q4, int units, int sub, int n_seq, int max_new,
                                         bool causal) {
  AttnGeometry ge;
  const int nt = attn_row_blocks(d, rep, max_new), group = attn_group(d);
  const int heads = H < group ? H : group;                          // of the first group
  const int rest = H > group && H % group ? H % group : heads;      // of the last one
  const int tile = 16 * attn_teams(heads, group) * sub;
  ge.sub = sub;
  int rows_log = 3, tile_log = 4;
  while (1 << rows_log < nt * 8) ++rows_log;
  while (1 << tile_log < tile) ++tile_log;
  ge.sh = {(H + group - 1) / group, nt * 8, tile, rows_log, tile_log, rep, causal ? 1 : 0};
  if (!q4) {
    // 16 slots' pieces of 64 channels stand together (2 KB), a row's eight 16-byte parts exchanged by its number mod 8:
    // as a tensor copy with 128-byte swizzling leaves them, and eight rows' parts fall on different banks
    ge.row_s = heads * d * 2;
  } else {
    // as in the cache, so that several rows come in one copy; parts of rows are laid out for the banks
    const int used = heads * (d / 2) + ((heads * (d / 16) + 15) & ~15);
    ge.row_s = H > group ? used + ((32 - used) & 127) : units * 2;
  }
  ge.order = attn_row_order(ge.row_s);
  ge.half_bytes = (ge.sh.tile * ge.row_s + 1023) & ~1023;
  // any group whose heads have several warps needs the boxes: half of the warps write one at a time
  const bool join = attn_teams(heads, group) > 1 || attn_teams(rest, group) > 1;
  const int boxes = join ? group / 2 * attn_box_floats(d, nt) * 4 : 0;
  const int bars = (2 * kMaxStages + 1) * 8, pre = (n_seq + 1) * 4;
  ge.stages = (kAttnSmem - boxes - bars - pre) / (2 * ge.half_bytes);
  if (ge.stages > kMaxStages) ge.stages = kMaxStages;
  // A copying warp tells a place's turns apart by one bit.  It waits for tile j after it has filled tile j - copiers, for
  // which tile j - copiers - stages was left: at least tile j - 2 stages if copiers <= stages, and then the bit is enough.
  ge.copiers = ge.stages < kAttnCopyWarps ? ge.stages : kAttnCopyWarps;
  ge.join_off = ge.stages * 2 * ge.half_bytes;
  ge.bar_off = ge.join_off + boxes;
  ge.pre_off = ge.bar_off + bars;
  ge.smem_bytes = ge.pre_off + pre;
  ge.slot_floats = group * ge.sh.rows * (d + 2);
  return ge;
}

EPIKV_PLAN AttnGeometry attn_geometry(int H, int rep, int d, bool q4, int units, int slots, int n_seq, int max_new,
                                      bool causal) {
  const int sub = attn_sub_blocks(q4, d, attn_row_blocks(d, rep, max_new), (int64_t)slots * n_seq);
  const AttnGeometry ge = attn_geometry_of(H, rep, d, q4, units, sub, n_seq, max_new, causal);
  // four blocks a warp only where the ring then holds three tiles (4 KV heads of 128, 64 x 8,192 slots, two tiles of four
  // blocks 105 us, five of two 75)
  return ge.stages < 3 && sub == 4 ? attn_geometry_of(H, rep, d, q4, units, 2, n_seq, max_new, causal) : ge;
}

}  // namespace epikv
