// How the work of the operators of many query rows is cut, for the kernels and,
// compiled for the host, for its tests.
//
// An item of the chunk's attention is (batch entry, KV head, block of query
// rows).  Its slots are cut into tiles; all items' tiles stand in one line, which
// the CTAs take in about equal contiguous shares.  A share's piece of an item is a
// segment; an item of several segments is joined by a second kernel.
#pragma once

#include <stdint.h>

#include "attn_plan.h"

namespace epikv {

struct ChunkPlan {
  int rows;      // query rows of an item, 1 << rows_log
  int slots;     // of a tile, 1 << slots_log
  int rows_log, slots_log;
  int rep;       // query heads of a KV head
  int causal;
  int heads;     // KV heads
};

// (a call's tokens are at most 2^20, a KV head's query heads 1,024)
EPIKV_PLAN int chunk_blocks(const ChunkPlan& p, int n) { return (n * p.rep + p.rows - 1) >> p.rows_log; }
// Slots that query row r sees, and the last row of a block.
EPIKV_PLAN int row_sees(const ChunkPlan& p, int len, int r) { return p.causal ? len + r / p.rep + 1 : len; }
EPIKV_PLAN int block_sees(const ChunkPlan& p, int n, int len, int block) {
  const int end = (block + 1) << p.rows_log, rows = n * p.rep;
  return row_sees(p, len, (end < rows ? end : rows) - 1);
}
// An item's places in the line: its tiles and kItemPlaces for its queries and results, which cost about as much as so many
// tiles (4 to 8 us; counted by tiles alone, the shares of a prompt's first, short blocks took twice the others' time).  An
// item that sees nothing has these all the same: its rows' zeros are written.
constexpr int kItemPlaces = 4;
EPIKV_PLAN int block_places(const ChunkPlan& p, int n, int len, int block) {
  return ((block_sees(p, n, len, block) + p.slots - 1) >> p.slots_log) + kItemPlaces;
}
EPIKV_PLAN int64_t head_places(const ChunkPlan& p, int n, int len) {
  int64_t t = 0;
  for (int i = 0; i < chunk_blocks(p, n); ++i) t += block_places(p, n, len, i);
  return t;
}
// First tile behind so many of an item's places.
EPIKV_PLAN int tile_of_place(int places) { return places > kItemPlaces ? places - kItemPlaces : 0; }

// CTAs that share the line: one an item up to the GPU's, more where a share would be of over kLeastPlaces.
constexpr int kLeastPlaces = 8;
EPIKV_PLAN int chunk_ctas(unsigned total, int64_t items) {
  int64_t n = ((int64_t)total + kLeastPlaces - 1) / kLeastPlaces;
  if (n < items) n = items;
  if (n > kAttnCtas) n = kAttnCtas;
  return n < (int64_t)total ? (int)n : (int)total;
}
// First place of CTA c's share, floor(total * c / ctas) in 32 bits.
EPIKV_PLAN unsigned share_start(int c, unsigned total, int ctas) {
  const unsigned q = total / (unsigned)ctas, r = total % (unsigned)ctas;
  return q * c + r * c / (unsigned)ctas;
}
// The CTA whose share place x is in.
EPIKV_PLAN int share_of(unsigned x, unsigned total, int ctas) {
  int c = (int)((float)x * (float)ctas / (float)total);   // near it; put right by the shares themselves
  if (c > ctas - 1) c = ctas - 1;
  while (share_start(c, total, ctas) > x) --c;
  while (share_start(c + 1, total, ctas) <= x) ++c;
  return c;
}

// A share that would start among the first or behind the last few tiles of an item starts with it or behind it: a segment of
// so few tiles is not worth a part.
constexpr int kFewTiles = 2;
EPIKV_PLAN unsigned moved_start(unsigned x, unsigned at, unsigned places) {
  if (x - at <= (unsigned)(kItemPlaces + kFewTiles)) return at;
  return at + places - x <= (unsigned)kFewTiles ? at + places : x;
}
// The CTA that an item's last segment stands in.
EPIKV_PLAN int last_share(unsigned at, unsigned places, unsigned total, int ctas) {
  const int c = share_of(at + places - 1, total, ctas);
  const unsigned x = share_start(c, total, ctas);
  return x > at && moved_start(x, at, places) == at + places ? c - 1 : c;
}

// ---- what slots receive
// A unit is (entry, run of slots, KV head); its steps are tiles of query rows.  A slot is seen by the rows from some row on
// (causal), so a unit has the rows from the first that sees its first slot to the last.  All units' steps stand in one line,
// slots before heads; shares and segments as above.
struct WeightPlan {
  int slots, slots_log;   // of a unit
  int rows, rows_log;     // of a step
  int rep, causal, heads;
  int last;               // tokens that count, 0: all
  int extra;              // places of a unit besides its steps: 0 or kUnitPlaces
};
// What a unit's keys and results cost, in steps of 128 rows (of 16 rows a unit has one step at most, and all cost the same).
constexpr int kUnitPlaces = 4;

EPIKV_PLAN int weight_slots(const WeightPlan& p, int n, int len) { return len + (p.causal ? n : 0); }
EPIKV_PLAN int weight_units(const WeightPlan& p, int n, int len) {
  return (weight_slots(p, n, len) + p.slots - 1) >> p.slots_log;
}
// First new token of a unit.
EPIKV_PLAN int weight_token(const WeightPlan& p, int n, int len, int unit) {
  const int first = p.last && p.last < n ? n - p.last : 0, s0 = unit << p.slots_log;
  const int sees = p.causal && s0 > len ? s0 - len : 0;
  return sees > first ? sees : first;
}
// Steps of a unit: 0 where no row counts ...
EPIKV_PLAN int weight_steps(const WeightPlan& p, int n, int len, int unit) {
  return ((n - weight_token(p, n, len, unit)) * p.rep + p.rows - 1) >> p.rows_log;
}
// ... which still has a place in the line: its zeros are stored.
EPIKV_PLAN int weight_places(const WeightPlan& p, int n, int len, int unit) {
  const int t = weight_steps(p, n, len, unit) + p.extra;
  return t > 1 ? t : 1;
}
// First step behind so many of a unit's places; where a share starts that would start at place x of the line, in a unit
// whose places start at `at` (with the unit rather than before its first step).
EPIKV_PLAN int step_of_place(const WeightPlan& p, int places) { return places > p.extra ? places - p.extra : 0; }
EPIKV_PLAN unsigned moved_unit_start(const WeightPlan& p, unsigned x, unsigned at) { return x - at <= (unsigned)p.extra ? at : x; }
// Units from an entry's start on that have as many places as its first.
EPIKV_PLAN int weight_alike(const WeightPlan& p, int n, int len) {
  const int all = weight_units(p, n, len);
  if (!p.causal) return all;
  const int t = (len >> p.slots_log) + 1;   // start at or before the first new slot
  return t < all ? t : all;
}
EPIKV_PLAN int64_t weight_entry(const WeightPlan& p, int n, int len) {
  const int all = weight_units(p, n, len), alike = weight_alike(p, n, len);
  int64_t t = all ? (int64_t)alike * weight_places(p, n, len, 0) : 0;
  for (int i = alike; i < all; ++i) t += weight_places(p, n, len, i);
  return t * p.heads;
}

// What the second kernel joins: an item that starts in one CTA's share and does not end there.
struct ChunkSplit {
  int there;       // 0: the CTA starts no such item
  int b, kh, row0, rows;
  int parts;       // CTAs that hold a segment of it: this one and the next ones
  int pad[2];
};

// Rows of T slots for every sequence and head, none of which meets another.
EPIKV_PLAN bool weights_apart(int S, int H, int T, int64_t stride_seq, int64_t stride_head) {
  if (stride_seq < 0 || stride_head < 0) return false;
  if (S == 1 && H == 1) return true;
  if (S == 1) return stride_head >= T;
  if (H == 1) return stride_seq >= T;
  const bool seqs_inside = stride_seq < stride_head;   // the rows of one head stand together
  const int64_t lo = seqs_inside ? stride_seq : stride_head, hi = seqs_inside ? stride_head : stride_seq;
  const int64_t n = seqs_inside ? S : H;
  // lo * (n - 1) + T <= hi, without leaving 64 bits
  return lo >= T && (hi - T) / lo >= n - 1;
}

}  // namespace epikv
