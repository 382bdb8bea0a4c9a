// Attention of a chunk of new tokens over the slots of the cache, many query
// rows at a time on the tensor instructions.
//
//   out = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q.k_j - m),   c = scale log2(e)
//
// A query row is a token and one of the rep query heads that share a KV head.
// An item is up to 256 such rows of one entry and KV head, as one or two tiles
// of 128; it goes over the slots that its rows see in tiles of 128 (64 at 256
// channels).  S = Q K^T and O += P V run on tcgen05 with S and O in tensor
// memory; a thread owns a row, so maxima and sums need no exchange; P replaces
// S in tensor memory, in 16 bits.  One CTA an SM takes an equal share of all
// items' tiles (chunk_plan.h); items that several CTAs hold a segment of are
// joined by a second kernel in the order of the slots.
//
// Two tiles of rows, because one's exponentials are formed while the other's
// products run, and because K and V are read once for both.  P is rounded to
// the operand's 16 bits: bf16 beside bf16 values (2^-9 of each probability,
// 0.0023 of the output's size instead of 0.0017, which the output's own
// rounding gives), halves beside 4-bit ones.
//
// 32 query and 8 KV heads of 128.  Long chunks wait from warp to warp (the
// tensor pipe is busy 67 % of the cycles, the exponential unit 34): 2,048 tokens
// behind 14,336 369 us in a long run of them, 341 in a short one, at higher
// clocks (1.4 and 1.5 PFLOP/s, 72 and 78 % of the measured rate), a prompt of
// 4,096 128 us (1.08, 56 %: items of 1 to 32 tiles, each with its queries,
// results and half-empty last tiles).  Few tokens are bound by the cache's bytes
// and the chain of launch, lookups, first tiles and join: 8 x 16 tokens behind
// 4,096 43 us (3.2 TB/s).  4-bit rows by the copying warps' instructions: 8 x 256
// behind 2,048 to 4,096 133 us, over bf16 109.
#include "chunk_plan.h"
#include "tensor.cuh"

namespace epikv {
namespace {

constexpr float kSlack = 8.f;           // a maximum is moved when a score passes it by 2^8
// 8 warps own rows, one issues products; the others copy: three, seven where they turn 4-bit rows into halves.  They exchange
// registers: launched with the same number each, the owners of rows take more from the others.
constexpr int chunk_threads(int fmt) { return fmt == EPIKV_CACHE_BF16 ? 384 : 512; }
constexpr int launch_regs(int fmt) { return 65536 / chunk_threads(fmt) & ~7; }
constexpr int kOtherRegs = 88;
constexpr int owner_regs(int fmt, int tiles) { return tiles == 1 ? 232 : fmt == EPIKV_CACHE_BF16 ? 208 : 168; }
constexpr bool enough_regs(int fmt, int tiles) {
  const int groups = chunk_threads(fmt) / 128;
  return tiles * owner_regs(fmt, tiles) + (groups - tiles) * kOtherRegs <= groups * launch_regs(fmt);
}
static_assert(enough_regs(EPIKV_CACHE_BF16, 1) && enough_regs(EPIKV_CACHE_BF16, 2) && enough_regs(EPIKV_CACHE_E2M1, 1) &&
              enough_regs(EPIKV_CACHE_E2M1, 2), "the owners would wait for registers that nobody gives");

template <int D>
struct ChunkShape {
  static constexpr int kSlots = D == 256 ? 64 : 128;   // of a tile
  static constexpr int kStage = kSlots * D * 2;
  static constexpr int kQuery = 128 * D * 2;           // bytes of a tile of query rows
  static constexpr int kStages = D == 64 ? 8 : 4;
};

// A CTA's piece of an item.
struct Segment {
  Entry e;
  int b, kh;
  int row0, rows;    // the item's first query row of that KV head, rows
  int t0, t1;        // tiles of slots
  int least, most;   // slots that the item's first row sees, and its last
  bool first, last;  // the item starts, ends here
  unsigned at, places;   // of the item in the line
};

// Where a CTA's share starts: entry, KV head, block, and the line's place that the block starts at.
struct ShareStart {
  int b, kh, block;
  unsigned at;
  Entry e;
};

// A warp's walk along its CTA's share, in shared memory: its first lane moves it on, and what the loops over tiles do not
// need stays out of their registers.  Segment i stands in now[i & 1] while the next one is looked at.
struct WarpWalk {
  ShareStart here;
  unsigned x;          // the share's next place
  Segment now[2];
};

__device__ __forceinline__ Entry entry_of(const Batch& ba, int b) {
  Entry e;
  e.tok0 = ba.cu_new[b];
  e.n = ba.cu_new[b + 1] - e.tok0;
  e.seq = ba.seq_ids[b];
  e.len = ba.len[(int64_t)b * ba.len_stride];
  return e;
}

struct SegmentWalk {
  WarpWalk* w;
  const unsigned* pre;   // [n_seq + 1] places before each entry
  const Batch& ba;
  const ChunkPlan& plan;
  unsigned end;          // of the share
  int lane;
  __device__ __forceinline__ void begin(const ShareStart& start, unsigned x) const {
    if (lane == 0) {
      w->here = start;
      w->x = x;
    }
    __syncwarp();
  }
  __device__ __forceinline__ void step(Segment* s) const {
    ShareStart h = w->here;
    const Entry e = h.e;
    const unsigned x = w->x;
    const unsigned places = (unsigned)block_places(plan, e.n, e.len, h.block), take = min(h.at + places, end) - x;
    s->e = e;
    s->b = h.b;
    s->kh = h.kh;
    s->row0 = h.block * plan.rows;
    s->rows = min(e.n * plan.rep - s->row0, plan.rows);
    s->least = row_sees(plan, e.len, s->row0);
    s->most = block_sees(plan, e.n, e.len, h.block);
    s->t0 = tile_of_place((int)(x - h.at));
    s->t1 = tile_of_place((int)(x - h.at + take));
    s->first = x == h.at;
    s->last = x + take == h.at + places;
    s->at = h.at;
    s->places = places;
    w->x = x + take;
    if (s->last) {
      h.at += places;
      if (++h.block == chunk_blocks(plan, e.n)) {
        h.block = 0;
        if (++h.kh == plan.heads) {
          h.kh = 0;
          if (w->x < end) {
            do ++h.b;
            while (pre[h.b + 1] == pre[h.b]);
            h.e = entry_of(ba, h.b);
          }
        }
      }
      w->here = h;
    }
  }
  // The whole warp; false at the share's end.
  __device__ __forceinline__ bool next(int i) const {
    const bool more = w->x < end;
    __syncwarp();
    if (more && lane == 0) step(&w->now[i & 1]);
    __syncwarp();
    return more;
  }
  __device__ __forceinline__ const Segment& segment(int i) const { return w->now[i & 1]; }
};

template <int D>
struct alignas(16) ChunkShared {
  static constexpr int kStages = ChunkShape<D>::kStages;
  uint64_t query, full[kStages], empty[kStages], scores[2], weights[2][2], sums, done, landed, drained;
  uint32_t tmem;
  int gave_up;
  // 1 + the last segment with an infinite or NaN value in a slot that not all its rows see.  The copying warps may be a ring of
  // tiles ahead of the segment that the owners of rows have yet to look up.
  volatile int unclean[8];
  static_assert(kStages / 2 < 8, "a place for each segment that the ring can hold, and one more");
  int64_t offset[2][ChunkShape<D>::kSlots]; // of a tile's slots, elements; -1: none
  ShareStart start;
  unsigned from, to;                        // the CTA's share
  WarpWalk walk[16];
  ChunkSplit split;
  Entry entries[32];                        // the batch's first
};

// Places before each entry of the batch, by a warp; returns the items.  An entry that cannot be taken has none, nor has one
// that takes the sum to kTooManyTiles and those behind it.
__device__ __forceinline__ int64_t line_up(unsigned* pre, Entry* entries, const Batch& ba, const AttnDims& dm, const ChunkPlan& plan,
                                           int32_t* err, int lane) {
  unsigned before = 0;
  int64_t items = 0;
  for (int b0 = 0; b0 < ba.n_seq; b0 += 32) {
    const int b = b0 + lane;
    Entry e;
    unsigned n = 0;
    int64_t it = 0;
    const bool taken = b < ba.n_seq && batch_entry(ba, dm, b, plan.causal, err, &e);
    if (b0 == 0 && taken) entries[lane] = e;
    const int blocks = taken ? chunk_blocks(plan, e.n) : 0;
    int64_t tiles = 0;
    if (__all_sync(0xffffffffu, blocks <= 8)) {
      if (taken) tiles = head_places(plan, e.n, e.len);
    } else {   // long entries one by one
      for (unsigned left = __ballot_sync(0xffffffffu, blocks > 0); left; left &= left - 1) {
        const int who = __ffs(left) - 1;
        const int en = __shfl_sync(0xffffffffu, e.n, who), len = __shfl_sync(0xffffffffu, e.len, who);
        const int eb = __shfl_sync(0xffffffffu, blocks, who);
        int64_t sum = 0;
        for (int i = lane; i < eb; i += 32) sum += block_places(plan, en, len, i);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == who) tiles = sum;
      }
    }
    if (taken) {
      n = count_of(tiles * plan.heads);
      it = (int64_t)blocks * plan.heads;
    }
    unsigned upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto = add_counts(upto, v);
      it += __shfl_xor_sync(0xffffffffu, it, o);
    }
    upto = add_counts(upto, before);
    if (upto == kTooManyTiles && n) set_error(err, EPIKV_DEV_CAPACITY);
    // the last sum below the limit stands for all entries behind it
    const unsigned over = __ballot_sync(0xffffffffu, upto == kTooManyTiles);
    const unsigned kept = __shfl_sync(0xffffffffu, upto, over ? max(__ffs(over) - 2, 0) : 31);
    const unsigned good = over == 0 ? upto : over & 1 ? before : kept;
    if (upto == kTooManyTiles) upto = good;
    if (b < ba.n_seq) pre[b + 1] = upto;
    before = __shfl_sync(0xffffffffu, upto, 31);
    items += it;
    if (over) {   // everything behind is refused too
      for (int i = b0 + 32 + lane; i < ba.n_seq; i += 32) pre[i + 1] = before;
      break;
    }
  }
  if (lane == 0) pre[0] = 0;
  return items;
}

// Where in the line place x is, by a warp; returns where a share that starts there does.
__device__ __forceinline__ unsigned find_place(ShareStart* start, unsigned x, const unsigned* pre, const Entry* entries,
                                               const Batch& ba, const ChunkPlan& plan, int lane) {
  int lo = 0, hi = ba.n_seq - 1;   // the entry with pre[b] <= x < pre[b + 1]
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (x < pre[mid + 1]) hi = mid;
    else lo = mid + 1;
  }
  const Entry e = lo < 32 ? entries[lo] : entry_of(ba, lo);
  const int n = e.n, len = e.len;
  const unsigned of_head = (pre[lo + 1] - pre[lo]) / (unsigned)plan.heads, kh = (x - pre[lo]) / of_head;
  unsigned at = pre[lo] + kh * of_head;
  const int blocks = chunk_blocks(plan, n);
  int block = 0;
  unsigned places = 0;
  for (int b0 = 0; b0 < blocks; b0 += 32) {
    const unsigned t = b0 + lane < blocks ? (unsigned)block_places(plan, n, len, b0 + lane) : 0u;
    unsigned upto = t;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    const unsigned behind = __ballot_sync(0xffffffffu, at + upto > x);
    if (behind) {
      const int k = __ffs(behind) - 1;
      block = b0 + k;
      at += __shfl_sync(0xffffffffu, upto - t, k);
      places = __shfl_sync(0xffffffffu, t, k);
      break;
    }
    at += __shfl_sync(0xffffffffu, upto, 31);
  }
  if (lane == 0) *start = {lo, (int)kh, block, at, e};
  return moved_start(x, at, places);
}

// Element offset of each of the tile's slots, or -1.
__device__ __forceinline__ void tile_offsets(int64_t* offset, int n, int s0, int most, const KvDev& kv, int layer, int seq,
                                             int T, int32_t* err, int tid, int threads) {
  for (int r = tid; r < n; r += threads) {
    int64_t o = -1;
    if (s0 + r < most) {
      o = kv_row_offset(kv, layer, seq, s0 + r, T);
      if (o < 0) set_error(err, EPIKV_DEV_SLOT);
    }
    offset[r] = o;
  }
}

// Whether any of eight 16-bit values has an exponent of all ones (kBit: its lowest bit): infinite or NaN.
template <uint32_t kBit>
__device__ __forceinline__ bool unbounded(const uint4& v) {
  constexpr uint32_t kExp = (0x8000u - kBit) * 0x10001u, kOne = kBit * 0x10001u;
  return (((v.x & kExp) + kOne) | ((v.y & kExp) + kOne) | ((v.z & kExp) + kOne) | ((v.w & kExp) + kOne)) & 0x80008000u;
}
// acc + 0 a: NaN in a half from the first value on that is infinite or NaN.
template <bool kBf16>
__device__ __forceinline__ void note_unbounded(uint32_t& acc, uint32_t a) {
  if constexpr (kBf16) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(a), "r"(0u));
  else asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(a), "r"(0u));
}
// The values with 0 in the place of those.
template <uint32_t kBit>
__device__ __forceinline__ uint32_t bounded(uint32_t w) {
  constexpr uint32_t kExp = 0x8000u - kBit;
  if ((w & kExp) == kExp) w &= 0xffff0000u;
  if ((w >> 16 & kExp) == kExp) w &= 0xffffu;
  return w;
}

// The copying warps.  A stage of the ring holds a tile's keys or its values, in turn; each warp arrives once when its part
// of a stage is there.  Tiles come as tensor copies where the layer is a tensor, else by lanes.
template <int D, int FMT>
struct Copier {
  using Shape = ChunkShape<D>;
  static constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  static constexpr uint32_t kBit = kBf16 ? 0x80u : 0x400u;   // lowest of the exponent
  static constexpr int kWarps = chunk_threads(FMT) / 32 - 9, kCopyThreads = kWarps * 32;
  char* ring;
  ChunkShared<D>& sh;
  const TensorWaiter& wait;
  const AttnDims& dm;
  const KvDev& kv;
  const LayerMaps& maps;
  int layer;
  int32_t* err;
  int tid, lane, warp;

  __device__ __forceinline__ uint32_t stage(int i) const { return smem_u32(ring + i % Shape::kStages * Shape::kStage); }
  __device__ __forceinline__ void left(int i) const {
    if (i >= Shape::kStages) wait(&sh.empty[i % Shape::kStages], (uint32_t)(i / Shape::kStages - 1) & 1);
  }
  // A probability of 0 must not meet an infinity or a NaN in a slot that other rows see or none: of a stage of values, rows
  // that not all query rows see are looked through (0 times a value, added up: NaN from the first that is not bounded), and
  // those that none sees cleared.
  __device__ __forceinline__ void clean(int i, int s0, const Segment& g, int seg) const {
    constexpr int kRow = D / 8, kAtOnce = 4;
    const uint32_t dst = stage(i);
    const int from = max(g.least - s0, 0) * kRow, to = min(g.most - s0, Shape::kSlots) * kRow;
    auto place = [&](int x) { return dst + tile_at<D>(x / kRow, x % kRow); };
    uint32_t acc[4] = {0, 0, 0, 0};
    for (int x0 = from + tid; x0 < to; x0 += kAtOnce * kCopyThreads) {
      uint4 v[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) v[u] = lds16_pure(place(min(x0 + u * kCopyThreads, to - 1)));
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        note_unbounded<kBf16>(acc[0], v[u].x);
        note_unbounded<kBf16>(acc[1], v[u].y);
        note_unbounded<kBf16>(acc[2], v[u].z);
        note_unbounded<kBf16>(acc[3], v[u].w);
      }
    }
    if (unbounded<kBit>(make_uint4(acc[0], acc[1], acc[2], acc[3])))   // (the last piece of all may be another thread's)
      for (int x = from + tid; x < to; x += kCopyThreads) {
        const uint4 v = lds16(place(x));
        if (unbounded<kBit>(v)) {
          sts16(place(x), make_uint4(bounded<kBit>(v.x), bounded<kBit>(v.y), bounded<kBit>(v.z), bounded<kBit>(v.w)));
          sh.unclean[seg & 7] = seg + 1;
        }
      }
    for (int x = max(to, 0) + tid; x < Shape::kSlots * kRow; x += kCopyThreads) sts16(place(x), make_uint4(0, 0, 0, 0));
  }
  // The warp's part of a stage that was written by lanes is there.
  __device__ __forceinline__ void deliver(int i) const {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive_one(&sh.full[i % Shape::kStages]);
  }

  // Lane l looks after box l of the tile.  Keys that no row sees may stay as they are (their scores are replaced); boxes that
  // hold nothing but those are left out.
  __device__ __forceinline__ void tensor_tile(int i, int j, int y, int z, const Segment& g, int seg, int* turns) const {
    const int s0 = j * Shape::kSlots;
    const int slots = min(Shape::kSlots, (g.most - s0 + maps.slots - 1) & -maps.slots);   // that come
    const bool whole = s0 + Shape::kSlots <= g.least;
#pragma unroll 1
    for (int w = 0; w < 2; ++w, ++i) {
      left(i);
      uint64_t* full = &sh.full[i % Shape::kStages];
      uint64_t* bar = w && !whole ? &sh.landed : full;
      if (warp == 0) {
        if (lane == 0) mbar_arrive_expect_tx(bar, slots * D * 2);
        __syncwarp();
        if (lane * maps.slots < slots)
          tma_load_rows(stage(i) + lane * maps.slots * (D * 2), &maps.kv[w], g.kh * (D / 64), y >> 3, z, bar);
        __syncwarp();
      } else if (bar == full && lane == 0) {
        mbar_arrive_one(full);
      }
      if (bar == full) continue;
      wait(bar, (uint32_t)(*turns)++ & 1);
      // One bit tells the phase, and the first warp arms the next one: not before all are behind this one's wait.
      named_sync(1, kCopyThreads);
      clean(i, s0, g, seg);
      deliver(i);
    }
  }

  __device__ __forceinline__ void bf16_segment(const Segment& g, int i, int seg, int* turns) const {
    const bool flat = kv.layout == EPIKV_LAYOUT_CONTIGUOUS;
    int tables = 0;
    for (int j = g.t0; j < g.t1; ++j, i += 2) {
      const int s0 = j * Shape::kSlots;
      bool whole = maps.slots && min(s0 + Shape::kSlots, g.most) <= maps.end;
      if (whole) {
        int y = s0 + lane * maps.slots, z = g.e.seq;
        bool there = true;
        if (!flat && y < g.most && lane * maps.slots < Shape::kSlots) {
          const int bi = y / kv.block_size;
          y -= bi * kv.block_size;
          z = bi < kv.max_blocks
                  ? __ldg(kv.block_table + (int64_t)layer * kv.table_stride_layer + (int64_t)g.e.seq * kv.max_blocks + bi)
                  : -1;
          there = z >= 0 && z < kv.num_blocks;
        }
        whole = __all_sync(0xffffffffu, there);   // else by lanes, which report it
        if (whole) tensor_tile(i, j, y, z, g, seg, turns);
      }
      if (!whole) lane_tile(i, j, g, seg, &tables);
    }
    named_sync(1, kCopyThreads);   // the offsets are free for the next segment
  }

  // By lanes: the values' copies are under way while the keys' are waited for.
  __device__ __forceinline__ void lane_tile(int i, int j, const Segment& g, int seg, int* tables) const {
    const int s0 = j * Shape::kSlots;
    // two take turns among the tiles that come here: all threads met at the last such tile, behind reading the one before it
    int64_t* offset = sh.offset[(*tables)++ & 1];
    tile_offsets(offset, Shape::kSlots, s0, g.most, kv, layer, g.e.seq, dm.T, err, tid, kCopyThreads);
    named_sync(1, kCopyThreads);
#pragma unroll 1
    for (int w = 0; w < 2; ++w) {
      left(i + w);
      const uint32_t dst = stage(i + w);
      const char* base = kv.base[w];
      constexpr int kAtOnce = 8, kPer = D / 8;   // 16-byte pieces of a row
      for (int x0 = tid; x0 < Shape::kSlots * kPer; x0 += kAtOnce * kCopyThreads) {
        int64_t o[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) o[u] = offset[min((x0 + u * kCopyThreads) / kPer, Shape::kSlots - 1)];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int x = x0 + u * kCopyThreads, r = x / kPer, c = x % kPer;
          if (x < Shape::kSlots * kPer)
            copy_async16(dst + tile_at<D>(r, c),
                         base + (o[u] < 0 ? 0 : (o[u] + g.kh * D + c * 8) * 2), o[u] < 0 ? 0 : 16);
        }
      }
      copy_commit();
    }
    copy_wait<1>();
    deliver(i);
    copy_wait<0>();
    if (s0 + Shape::kSlots > g.least) {
      named_sync(1, kCopyThreads);   // what others copied is looked through too
      clean(i + 1, s0, g, seg);
    }
    deliver(i + 1);
  }

  // 4-bit rows: the next tile's codes are under way while this one's become halves, and the table's entries of the one behind
  // it.
  __device__ __forceinline__ void q4_segment(const Segment& g, int i, int seg) const {
    constexpr int kStep = kCopyThreads / (D / 32), kRounds = (Shape::kSlots + kStep - 1) / kStep;
    static_assert(kCopyThreads >= Shape::kSlots, "a thread a slot");
    using Codes = CodeRows<D, kCopyThreads, kRounds>;
    const int codes = g.kh * (D / 2), scales = scale_offset(dm, g.kh);
    auto look = [&](int j) {   // the thread's slot of tile j
      const int s = j * Shape::kSlots + tid;
      if (tid >= Shape::kSlots || s >= g.most) return (int64_t)-1;
      const int64_t o = kv_row_offset(kv, layer, g.e.seq, s, dm.T);
      if (o < 0) set_error(err, EPIKV_DEV_SLOT);
      return o;
    };
    auto tell = [&](int j, int64_t o) {
      if (tid < Shape::kSlots) sh.offset[j & 1][tid] = o;
      named_sync(1, kCopyThreads);
    };
    auto load = [&](Codes& c, int w, int j) {
      c.load(kv.base[w], sh.offset[j & 1], codes, scales, 0, Shape::kSlots, tid);
    };
    Codes k, v;
    tell(g.t0, look(g.t0));
    load(k, 0, g.t0);
    load(v, 1, g.t0);
    int64_t ahead = g.t0 + 1 < g.t1 ? look(g.t0 + 1) : -1;
    for (int j = g.t0; j < g.t1; ++j, i += 2) {
      const int s0 = j * Shape::kSlots;
      const bool more = j + 1 < g.t1;
      if (more) {
        tell(j + 1, ahead);
        ahead = j + 2 < g.t1 ? look(j + 2) : -1;
      }
      left(i);
      k.store(stage(i), 0, Shape::kSlots, tid);
      deliver(i);
      if (more) load(k, 0, j + 1);
      left(i + 1);
      v.store(stage(i + 1), 0, Shape::kSlots, tid);
      if (s0 + Shape::kSlots > g.least) {
        named_sync(1, kCopyThreads);   // what others wrote is looked through too
        clean(i + 1, s0, g, seg);
      }
      deliver(i + 1);
      if (more) load(v, 1, j + 1);
    }
    named_sync(1, kCopyThreads);   // the offsets are free for the next segment
  }

  __device__ __forceinline__ void run(const SegmentWalk& walk) const {
    int i = 0, turns = 0;
    for (int seg = 0, at = 0; walk.next(at); ++at) {
      const Segment& g = walk.segment(at);
      const int tiles = g.t1 - g.t0;
      if (tiles <= 0) continue;
      if constexpr (kBf16) bf16_segment(g, i, seg, &turns);
      else q4_segment(g, i, seg);
      i += 2 * tiles;
      ++seg;
    }
    if (*wait.gave_up && warp == 0)   // the CTA may not end before its copies have landed
      for (int k = max(0, i - Shape::kStages); k < i; ++k)
        mbar_wait_bounded(&sh.full[k % Shape::kStages], (uint32_t)(k / Shape::kStages) & 1, kTensorWaitNs);
    if (*wait.gave_up && warp == 0 && turns) mbar_wait_bounded(&sh.landed, (uint32_t)(turns - 1) & 1, kTensorWaitNs);
  }
};

// The issuing warp.  All its lanes go through the loops, so that the operands' descriptions are formed once for the warp (by
// one lane alone, the registers' way to the instruction took 110 cycles a product, of 64 that the product takes).
template <int D, int FMT, int kTiles>
__device__ __forceinline__ void issue_products(uint32_t query, uint32_t ring, ChunkShared<D>& sh, const TensorWaiter& wait,
                                               const SegmentWalk& walk, uint32_t tmem) {
  using Shape = ChunkShape<D>;
  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  constexpr uint32_t kScores = product_of(128, Shape::kSlots, kBf16, false), kSums = product_of(128, D, kBf16, true);
  const uint64_t q0 = rows_operand<D>(query), k0 = rows_operand<D>(ring), v0 = columns_operand<D>(ring);
  auto scores = [&](int t, int buf, int st) {
    const uint64_t q = q0 + (uint32_t)(t * (Shape::kQuery >> 4)), k = k0 + (uint32_t)(st * (Shape::kStage >> 4));
    const uint32_t d = tmem + buf * 128;
    if (elected()) {
#pragma unroll
      for (int x = 0; x < D / 16; ++x)
        multiply(d, q + rows_step(x), k + rows_step(x), kScores, x > 0);
      products_done(&sh.scores[buf]);
    }
    __syncwarp();
  };
  // the products with the first half of a tile's slots go ahead while the others' probabilities are formed
  auto sums = [&](int t, int buf, int st, bool add, uint32_t parity) {
    const uint64_t v = v0 + (uint32_t)(st * (Shape::kStage >> 4));
    const uint32_t d = tmem + 256 + t * 128, p = tmem + buf * 128;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      wait(&sh.weights[buf][h], parity);
      tensor_fence_after();
      if (elected()) {
#pragma unroll
        for (int x = h * Shape::kSlots / 32; x < (h + 1) * Shape::kSlots / 32; ++x)
          multiply_tmem(d, p + x * 8, v + columns_step<D>(x), kSums, add || x > 0);
      }
      __syncwarp();
    }
  };
  auto filled = [&](int i) {
    wait(&sh.full[i % Shape::kStages], (uint32_t)(i / Shape::kStages) & 1);
    tensor_fence_after();
  };
  auto done = [&](uint64_t* bar) {
    if (elected()) products_done(bar);
    __syncwarp();
  };
  // i: the tile's keys in the ring; a: tiles so far
  for (int i = 0, a = 0, seg = 0, at = 0; walk.next(at); ++at) {
    const int tiles = __shfl_sync(0xffffffffu, walk.segment(at).t1 - walk.segment(at).t0, 0);
    if (tiles <= 0) continue;
    wait(&sh.query, (uint32_t)seg & 1);
    tensor_fence_after();
    filled(i);
    if constexpr (kTiles == 1) {
      scores(0, a & 1, i % Shape::kStages);
    } else {
      for (int t = 0; t < 2; ++t) scores(t, t, i % Shape::kStages);
    }
    done(&sh.empty[i % Shape::kStages]);
    for (int j = 0; j < tiles; ++j, i += 2, ++a) {
      const int v = (i + 1) % Shape::kStages, k = (i + 2) % Shape::kStages;
      const bool more = j + 1 < tiles;
      if constexpr (kTiles == 1) {   // two places for scores: the next tile's are formed beside this one's probabilities
        if (more) {
          filled(i + 2);
          scores(0, (a + 1) & 1, k);
          done(&sh.empty[k]);
        }
        filled(i + 1);
        sums(0, a & 1, v, j > 0, (uint32_t)(a >> 1) & 1);
        done(&sh.empty[v]);
        done(&sh.sums);
      } else {
        filled(i + 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          sums(t, t, v, j > 0, (uint32_t)a & 1);
          if (t == 1) done(&sh.empty[v]);
          if (!more) continue;
          if (t == 0) filled(i + 2);
          scores(t, t, k);   // in order behind the products that read the probabilities in its place
        }
        if (more) done(&sh.empty[k]);
      }
    }
    done(&sh.done);
    ++seg;
  }
}

// The owners of rows: a segment's tiles, the first of them the CTA's tile `a`.
template <int D, int FMT, int kTiles>
__device__ __forceinline__ void soften(ChunkShared<D>& sh, const TensorWaiter& wait, int t0, int t1, int a, int seen, float c,
                                       uint32_t tmem, int t, float* m_out, float* l_out) {
  using Shape = ChunkShape<D>;
  constexpr int N = Shape::kSlots;
  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  float m = -INFINITY, l = 0.f;
  const uint32_t o = tmem + 256 + t * 128;
  for (int j = t0; j < t1; ++j, ++a) {
    const int buf = kTiles == 1 ? a & 1 : t;
    const uint32_t s = tmem + buf * 128;
    wait(&sh.scores[buf], kTiles == 1 ? (uint32_t)(a >> 1) & 1 : (uint32_t)a & 1);
    tensor_fence_after();
    // bf16: a tile's scores are held, its columns one run of instructions.  Where warps beside these turn 4-bit rows into
    // halves, that run and theirs do not fit the instruction cache together (8 x 256 tokens: 160 us, the cache behind it at
    // 72 % of its rate): the scores are read twice there, in a loop over 32 columns.
    constexpr bool kHeld = kBf16;
    constexpr int kParts = N / 32;
    uint32_t x[kHeld ? kParts : 1][32];
    const int s0 = j * N;
    const bool edge = __any_sync(0xffffffffu, seen < s0 + N);   // (warp-uniform)
    auto load = [&](int i) { tmem_load32(s + 32 * i, x[kHeld ? i : 0]); };
    auto part = [&](int i) -> uint32_t(&)[32] { return x[kHeld ? i : 0]; };
    auto mask = [&](int i) {   // what the row does not see is minus infinity
      if (edge) {
#pragma unroll
        for (int u = 0; u < 32; ++u)
          if (s0 + 32 * i + u >= seen) part(i)[u] = 0xff800000u;
      }
    };
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    auto highest = [&](int i) {
      mask(i);
#pragma unroll
      for (int u = 0; u < 32; u += 8)
#pragma unroll
        for (int w = 0; w < 4; ++w)
          top[w] = max3(top[w], __uint_as_float(part(i)[u + w]), __uint_as_float(part(i)[u + w + 4]));
    };
    if constexpr (kHeld) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) load(i);
      tmem_wait_load<32 * kParts>(x[0]);
#pragma unroll
      for (int i = 0; i < kParts; ++i) highest(i);
    } else {
#pragma unroll 1
      for (int i = 0; i < kParts; ++i) {
        load(i);
        tmem_wait_load<32>(x[0]);
        highest(i);
      }
    }
    const float high = fmaxf(max3(top[0], top[1], top[2]), top[3]) * c;
    const bool up = high > m + kSlack;
    if (__any_sync(0xffffffffu, up)) {
      const float mul = !up ? 1.f : m == -INFINITY ? 0.f : exp2_fast(m - high);
      if (up) m = high;
      l *= mul;
      if (j > t0) {
        if constexpr (kTiles == 1) {   // the last tile's products may still be under way
          wait(&sh.sums, (uint32_t)(a - 1) & 1);
          tensor_fence_after();
        }
#pragma unroll 1
        for (int i = 0; i < D; i += 16) {
          uint32_t y[16];
          tmem_load16(o + i, y);
          tmem_wait_load<16>(y);
#pragma unroll
          for (int u = 0; u < 16; ++u) y[u] = __float_as_uint(__uint_as_float(y[u]) * mul);
          tmem_store16(o + i, y);
        }
      }
    }
    // a half's range is used up to 2^15: below 2^-24 it has no bits left
    const float base = (m == -INFINITY ? 0.f : m) - (kBf16 ? 0.f : 7.f);
    const f32x2 cc = f2_pack(c, c), bb = f2_pack(-base, -base);
    f32x2 sum[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
    auto soft = [&](int i) {
      uint32_t y[16];
      const uint32_t(&x)[32] = part(i);
#pragma unroll
      for (int u = 0; u < 32; u += 2) {
        const f32x2 z = f2_fma(f2_pack(__uint_as_float(x[u]), __uint_as_float(x[u + 1])), cc, bb);
        const float p = exp2_fast(f2_lo(z)), q = exp2_fast(f2_hi(z));
        sum[u >> 1 & 1] = f2_add(sum[u >> 1 & 1], f2_pack(p, q));
        y[u / 2] = kBf16 ? bf16_pair(p, q) : half_pair(p, q);
      }
      tmem_store16(s + 16 * i, y);
      if (i + 1 == kParts / 2 || i + 1 == kParts) {
        tmem_wait_store();
        tensor_fence_before();
        mbar_arrive_one(&sh.weights[buf][i + 1 == kParts]);
      }
    };
    if constexpr (kHeld) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) soft(i);
    } else {
#pragma unroll 1
      for (int i = 0; i < kParts; ++i) {
        load(i);
        tmem_wait_load<32>(x[0]);
        mask(i);
        soft(i);
      }
    }
    const f32x2 both = f2_add(sum[0], sum[1]);
    l += f2_lo(both) + f2_hi(both);
  }
  *m_out = m;
  *l_out = l;
}

// Lanes o apart: the one without the bit keeps a and gets the other's a for its b, the one with it keeps b and gets the
// other's b for its a.
__device__ __forceinline__ void exchange(uint4& a, uint4& b, int o, int lane) {
  const bool up = lane & o;
  const uint4 give = up ? a : b;
  const uint4 get = make_uint4(__shfl_xor_sync(0xffffffffu, give.x, o), __shfl_xor_sync(0xffffffffu, give.y, o),
                               __shfl_xor_sync(0xffffffffu, give.z, o), __shfl_xor_sync(0xffffffffu, give.w, o));
  if (up) a = get;
  else b = get;
}

// A segment's results: of a whole item its rows' outputs, else a part for the second kernel (outputs by fours of channels,
// row by row; maxima and sums behind them).
template <int D, int FMT>
__device__ __forceinline__ void put_rows(const AttnState& st, const AttnDims& dm, const Segment& g, const Rows& out, float* lse,
                                         const KvDev& kv, int layer, float* part, int part_rows, uint32_t o, int row, float m,
                                         float l, int seen, bool unclean) {
  constexpr int N = ChunkShape<D>::kSlots;
  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  const bool live = row < g.rows;
  const int r = g.row0 + row, token = r / dm.rep, hq = g.kh * dm.rep + r % dm.rep;
  float mul = l == 0.f ? 0.f : 1.f / l;
  if constexpr (!kBf16) mul *= head_scale(st, dm, 1, layer, g.kh);
  if (part) mul = 1.f;
  const bool none = l == 0.f;
  const float shift = kBf16 ? 0.f : 7.f;   // of the exponentials
  char* to = live ? out.p + ((int64_t)(g.e.tok0 + token) * out.st + hq * out.sh) * 2 : nullptr;
  const int from = max(g.least, g.t0 * N), upto = live && unclean ? min(seen, g.t1 * N) : 0;
  const int lane = threadIdx.x & 31;
  char* row_of[4];   // of the four lanes that exchange pieces
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    row_of[u] = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, (uint64_t)to, (lane & 28) + u));
    if (row_of[u]) row_of[u] += (lane & 3) * 16;
  }
#pragma unroll 2
  for (int i = 0; i < D; i += 32) {
    uint32_t y[32];
    if (g.t0 < g.t1) {
      tmem_load32(o + i, y);
      tmem_wait_load<32>(y);
    }
#pragma unroll
    for (int u = 0; u < 32; ++u) y[u] = none ? 0u : __float_as_uint(__uint_as_float(y[u]) * mul);
    // what the copying warps took out of slots that not all rows see: an infinity is the output of the rows that see it
#pragma unroll 1
    for (int s = from; s < upto; ++s) {
      const int64_t at = kv_row_offset(kv, layer, g.e.seq, s, dm.T);
      if (at < 0) continue;
      const char* v = kv.base[1] + at * 2;
      if constexpr (kBf16) {
#pragma unroll
        for (int u = 0; u < 32; ++u) {
          const uint32_t b = *reinterpret_cast<const uint16_t*>(v + (g.kh * D + i + u) * 2);
          if ((b & 0x7f80u) == 0x7f80u) y[u] = __float_as_uint(__uint_as_float(y[u]) + __uint_as_float(b << 16));
        }
      } else {   // a scale of NaN
#pragma unroll
        for (int u = 0; u < 32; ++u)
          if (((uint8_t)v[scale_offset(dm, g.kh) + (i + u) / kQuantGroup] & 0x7f) == 0x7f) y[u] = 0x7fc00000u;
      }
    }
    if (part) {
      if (live) {
#pragma unroll
        for (int u = 0; u < 32; u += 4)
          reinterpret_cast<uint4*>(part)[(int64_t)((i + u) / 4) * part_rows + row] = make_uint4(y[u], y[u + 1], y[u + 2], y[u + 3]);
      }
    } else {
      uint4 v[4];   // the row's 64 bytes
#pragma unroll
      for (int u = 0; u < 4; ++u)
        v[u] = make_uint4(bf16_pair(__uint_as_float(y[8 * u]), __uint_as_float(y[8 * u + 1])),
                          bf16_pair(__uint_as_float(y[8 * u + 2]), __uint_as_float(y[8 * u + 3])),
                          bf16_pair(__uint_as_float(y[8 * u + 4]), __uint_as_float(y[8 * u + 5])),
                          bf16_pair(__uint_as_float(y[8 * u + 6]), __uint_as_float(y[8 * u + 7])));
      // four lanes exchange: v[u] becomes the lane's piece of the u-th of their rows, so that they write its 64 bytes at once
      exchange(v[0], v[1], 1, lane);
      exchange(v[2], v[3], 1, lane);
      exchange(v[0], v[2], 2, lane);
      exchange(v[1], v[3], 2, lane);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (row_of[u]) *reinterpret_cast<uint4*>(row_of[u] + i * 2) = v[u];
    }
  }
  if (!live) return;
  if (part) {
    reinterpret_cast<float2*>(part + (int64_t)part_rows * D)[row] = make_float2(m - shift, l);
  } else if (lse) {
    lse[(int64_t)(g.e.tok0 + token) * dm.Hq + hq] = none ? -INFINITY : (m - shift + log2f(l)) * 0.69314718055994531f;
  }
}

template <int D, int FMT, int kTiles>
__global__ void __launch_bounds__(chunk_threads(FMT), 1)
    chunk_kernel(AttnState st, AttnDims dm, ChunkPlan plan, int layer, Batch ba, Rows q, Rows out, float* lse, KvDev kv,
                 const __grid_constant__ LayerMaps maps, float c, int part_rows) {
  using Shape = ChunkShape<D>;
  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  extern __shared__ char dynamic[];
  char* smem = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  __shared__ ChunkShared<D> sh;
  char* ring = smem + kTiles * Shape::kQuery;
  unsigned* pre = reinterpret_cast<unsigned*>(ring + Shape::kStages * Shape::kStage);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == 8) tmem_alloc(&sh.tmem, 512);
  if (tid == 0) {
    mbar_init(&sh.query, 128 * kTiles);
    for (int i = 0; i < Shape::kStages; ++i) {
      mbar_init(&sh.full[i], Copier<D, FMT>::kWarps);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.scores[i], 1);
      for (int h = 0; h < 2; ++h) mbar_init(&sh.weights[i][h], 128);
    }
    mbar_init(&sh.sums, 1);
    mbar_init(&sh.done, 1);
    mbar_init(&sh.landed, 1);
    mbar_init(&sh.drained, 1);
    sh.gave_up = 0;
    sh.split = {};
    for (int i = 0; i < 8; ++i) sh.unclean[i] = 0;
    fence_barrier_init();
  }
  pdl_wait();
  pdl_trigger();
  __shared__ int64_t items;
  if (warp == 0) {
    const int64_t n = line_up(pre, sh.entries, ba, dm, plan, st.err, lane);
    if (lane == 0) items = n;
    __syncwarp();
    const unsigned total = pre[ba.n_seq];
    const int ctas = chunk_ctas(total, n), cta = blockIdx.x;
    if (cta < ctas) {
      unsigned to = total;
      if (cta + 1 < ctas) to = find_place(&sh.start, share_start(cta + 1, total, ctas), pre, sh.entries, ba, plan, lane);
      unsigned from = find_place(&sh.start, share_start(cta, total, ctas), pre, sh.entries, ba, plan, lane);
      if (from < to) from = find_place(&sh.start, from, pre, sh.entries, ba, plan, lane);   // (the item behind, or the same)
      if (lane == 0) {
        sh.from = from;
        sh.to = to;
      }
    }
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  const uint32_t tmem = sh.tmem;
  const unsigned total = pre[ba.n_seq];
  const int cta = blockIdx.x, ctas = chunk_ctas(total, items);
  if (cta < ctas) {
    const TensorWaiter wait{&sh.gave_up, st.err};
    const SegmentWalk walk{&sh.walk[warp], pre, ba, plan, sh.to, lane};
    walk.begin(sh.start, sh.from);
    if (warp < 4 * kTiles) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(owner_regs(FMT, kTiles)));
      const int t = warp >> 2;
      const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
      int seen = 0;
      float factor = c;
      auto take_query = [&](const Segment& g) {
        const int r = g.row0 + tid, token = r / dm.rep, hq = g.kh * dm.rep + r % dm.rep;
        const bool live = tid < g.rows;
        // rows that are not there see all slots of the tiles
        seen = live ? row_sees(plan, g.e.len, r) : INT_MAX;
        if (g.t0 >= g.t1) return;
        // (a row that is not there has the item's first one's queries: nobody looks at its results)
        const char* src = q.p + (live ? (int64_t)(g.e.tok0 + token) * q.st + hq * q.sh
                                      : (int64_t)(g.e.tok0 + g.row0 / dm.rep) * q.st + (g.kh * dm.rep + g.row0 % dm.rep) * q.sh) * 2;
        factor = c * store_queries<D, !kBf16>(smem_u32(smem + t * Shape::kQuery), tid & 96, src, lane);
        if constexpr (!kBf16) factor *= head_scale(st, dm, 0, layer, g.kh);
        factor = score_factor(factor);
        fence_proxy_async_smem();
        mbar_arrive_one(&sh.query);
      };
      bool more = walk.next(0);
      if (more) take_query(walk.segment(0));
      for (int a = 0, seg = 0, at = 0; more; ++at) {
        float m = -INFINITY, l = 0.f;
        const int t0 = walk.segment(at).t0, t1 = walk.segment(at).t1, saw = seen;
        bool unclean = false;
        if (t0 < t1) {
          soften<D, FMT, kTiles>(sh, wait, t0, t1, a, seen, factor, lanes, t, &m, &l);
          wait(&sh.done, (uint32_t)seg & 1);
          tensor_fence_after();
          unclean = sh.unclean[seg & 7] == seg + 1;
          a += t1 - t0;
          ++seg;
        }
        more = walk.next(at + 1);
        if (more) take_query(walk.segment(at + 1));   // the next segment's first scores are formed beside this one's results
        const Segment& now = walk.segment(at);
        float* part = now.first && now.last ? nullptr
                                            : st.part + (int64_t)(2 * cta + (now.first ? 1 : 0)) * part_rows * (D + 2);
        put_rows<D, FMT>(st, dm, now, out, lse, kv, layer, part, part_rows, lanes + 256 + t * 128, tid, m, l, saw, unclean);
        if (tid == 0 && now.first && !now.last)
          sh.split = {1, now.b, now.kh, now.row0, now.rows, last_share(now.at, now.places, total, ctas) - cta + 1, {0, 0}};
      }
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kOtherRegs));
      if (warp == 8) {
        issue_products<D, FMT, kTiles>(smem_u32(smem), smem_u32(ring), sh, wait, walk, tmem);
        if (elected()) products_done(&sh.drained);   // tensor memory is not freed under products, whatever waits gave up
        __syncwarp();
        mbar_wait_bounded(&sh.drained, 0, kTensorWaitNs);
      } else if (warp > 8) {
        const Copier<D, FMT> copier{ring, sh, wait, dm, kv, maps, layer, st.err, tid - 288, lane, warp - 9};
        copier.run(walk);
      }
    }
  }
  if (tid == 0) reinterpret_cast<ChunkSplit*>(st.splits)[cta] = sh.split;
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  if (warp == 8) tmem_free(tmem, 512);
}

// Joins the segments of an item: a CTA for the rows of a block of the item that starts in CTA blockIdx.x's share.  A thread
// adds up four channels of a row, segment by segment.
template <int D>
__global__ void __launch_bounds__(256) chunk_join_kernel(AttnState st, AttnDims dm, int layer, Batch ba, Rows out, float* lse,
                                                         int part_rows) {
  constexpr int kRows = 1024 / D;   // of a CTA
  pdl_wait();
  pdl_trigger();
  const ChunkSplit s = reinterpret_cast<const ChunkSplit*>(st.splits)[blockIdx.x];
  const int row = blockIdx.y * kRows + threadIdx.x % kRows, ch = threadIdx.x / kRows;
  if (!s.there || row >= s.rows) return;
  const int64_t size = (int64_t)part_rows * (D + 2);
  auto part = [&](int i) { return st.part + (2 * ((int64_t)blockIdx.x + i) + (i == 0 ? 1 : 0)) * size; };
  auto max_sum = [&](int i) { return reinterpret_cast<const float2*>(part(i) + (int64_t)part_rows * D)[row]; };
  float top = -INFINITY;
  for (int i = 0; i < s.parts; ++i) top = fmaxf(top, max_sum(i).x);
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = 0; i < s.parts; ++i) {
    const float2 ml = max_sum(i);
    const float4 v = reinterpret_cast<const float4*>(part(i))[(int64_t)ch * part_rows + row];
    // never 0: 2^-149 of a bounded sum is nothing, of an infinite one infinite
    const float w = fmaxf(exp2_fast(ml.x - base), __uint_as_float(1u));
    sum += ml.y * w;
    acc.x += v.x * w;
    acc.y += v.y * w;
    acc.z += v.z * w;
    acc.w += v.w * w;
  }
  const int r = s.row0 + row;
  const int64_t token = ba.cu_new[s.b] + r / dm.rep;
  const int hq = s.kh * dm.rep + r % dm.rep;
  float mul = sum == 0.f ? 0.f : 1.f / sum;
  if (dm.fmt != EPIKV_CACHE_BF16) mul *= head_scale(st, dm, 1, layer, s.kh);
  *reinterpret_cast<uint2*>(out.p + (token * out.st + hq * out.sh + ch * 4) * 2) =
      make_uint2(bf16_pair(acc.x * mul, acc.y * mul), bf16_pair(acc.z * mul, acc.w * mul));
  if (lse && ch == 0) lse[token * dm.Hq + hq] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.69314718055994531f;
}

template <int D, int kTiles>
constexpr int chunk_smem(int n_seq) {
  return kTiles * ChunkShape<D>::kQuery + ChunkShape<D>::kStages * ChunkShape<D>::kStage + 1024 + (n_seq + 1) * 4;
}
// Rows that a part has room for: a multiple of 4, so that each part starts on 16 bytes.
int part_rows_of(const AttnDims& dm, int max_new) {
  const int64_t rows = (int64_t)max_new * dm.rep, most = dm.d == 256 ? 128 : 256;
  return (int)((rows < most ? rows : most) + 3) & ~3;
}

template <int D, int FMT, int kTiles>
cudaError_t run_chunk(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal, const Rows& q,
                      const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  using Shape = ChunkShape<D>;
  static_assert(chunk_smem<D, kTiles>(kMaxSeqs) + sizeof(ChunkShared<D>) + 64 <= 227 * 1024, "shared memory");
  const ChunkPlan plan = {128 * kTiles, Shape::kSlots, kTiles == 2 ? 8 : 7, Shape::kSlots == 128 ? 7 : 6, dm.rep, causal ? 1 : 0, dm.H};
  const int rows = part_rows_of(dm, ba.max_new);
  cudaError_t e = pdl_launch(chunk_kernel<D, FMT, kTiles>, dim3(kAttnCtas), chunk_threads(FMT), chunk_smem<D, kTiles>(ba.n_seq),
                             stream, st, dm, plan, layer, ba, q, out, lse, kv, layer_maps(dm, layer, kv, Shape::kSlots),
                             dm.scale * 1.4426950408889634f, rows);
  if (e != cudaSuccess) return e;
  return pdl_launch(chunk_join_kernel<D>, dim3(kAttnCtas, (rows * D + 1023) / 1024), 256, 0, stream, st, dm, layer, ba, out,
                    lse, rows);
}

// *runs becomes false where the compiler gave the kernel other registers than its warps' exchange of them counts on:
// launched, it would wait for registers that nobody gives.
template <int D, int FMT, int kTiles>
cudaError_t allow_chunk(bool* runs) {
  cudaFuncAttributes at;
  const cudaError_t e = cudaFuncGetAttributes(&at, chunk_kernel<D, FMT, kTiles>);
  if (e != cudaSuccess) return e;
  if (at.numRegs != launch_regs(FMT)) *runs = false;
  return cudaFuncSetAttribute(chunk_kernel<D, FMT, kTiles>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              chunk_smem<D, kTiles>(kMaxSeqs));
}

template <int FMT>
cudaError_t prepare_format(int d, bool* runs) {
  if (d == 256) return allow_chunk<256, FMT, 1>(runs);
  if (d == 128) {
    const cudaError_t e = allow_chunk<128, FMT, 1>(runs);
    return e == cudaSuccess ? allow_chunk<128, FMT, 2>(runs) : e;
  }
  const cudaError_t e = allow_chunk<64, FMT, 1>(runs);
  return e == cudaSuccess ? allow_chunk<64, FMT, 2>(runs) : e;
}

template <int FMT>
cudaError_t run_format(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal, const Rows& q,
                       const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  const bool two = (int64_t)ba.max_new * dm.rep > 128;
  auto go = dm.d == 256   ? run_chunk<256, FMT, 1>
            : dm.d == 128 ? (two ? run_chunk<128, FMT, 2> : run_chunk<128, FMT, 1>)
                          : (two ? run_chunk<64, FMT, 2> : run_chunk<64, FMT, 1>);
  return go(st, dm, layer, ba, causal, q, out, lse, kv, stream);
}

}  // namespace

size_t chunk_part_floats(const AttnDims& dm) {
  return (size_t)2 * kAttnCtas * part_rows_of(dm, dm.max_new) * (dm.d + 2);
}

cudaError_t chunk_prepare(const AttnDims& dm, bool* runs) {
  *runs = true;
  return dm.fmt == EPIKV_CACHE_BF16 ? prepare_format<EPIKV_CACHE_BF16>(dm.d, runs) : prepare_format<EPIKV_CACHE_E2M1>(dm.d, runs);
}

cudaError_t launch_attention_chunk(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal,
                                   const Rows& q, const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  auto go = dm.fmt == EPIKV_CACHE_BF16 ? run_format<EPIKV_CACHE_BF16> : run_format<EPIKV_CACHE_E2M1>;
  return go(st, dm, layer, ba, causal, q, out, lse, kv, stream);
}

}  // namespace epikv
