// What slots receive of attention, and its way into the eviction context.
//
//   w[h][slot] (+)= sum over rows r of KV head h of 2^(c q_r.k_slot - lse_r log2(e)),   c = scale log2(e)
//
// The products run on tcgen05 with the slots as the instruction's 128 rows and
// the query rows as its columns, so that a thread owns a slot and adds up its
// columns: no exchange between threads, and each slot's sum is formed in a fixed
// order (eight partial sums, each of every eighth column).  A unit is a run of
// 256 slots (128 at 256 channels) of one entry and KV head: its keys stay in
// shared memory while tiles of query rows (steps) pass by.  Two forms: steps of
// 16 rows where a call has no more (a decode step: reading the keys bounds it),
// and of 128 (a chunk: exponentials and products).  One CTA an SM takes an equal
// share of all units' steps (chunk_plan.h); the few units that two shares meet in
// are joined by a second kernel, part by part.
//
// 32 query and 8 KV heads of 128: a decode step of 64 bf16 caches of 2,048 to
// 8,192 slots 112 us (6.1 TB/s, 90 % of the measured rate); of 32 4-bit caches of
// 8,192 72 us (2.2 TB/s; 6,000 warp instructions a unit at 2.3 a cycle, some
// 1,700 of them the expansion to halves, the others walks, addresses and copies);
// a prompt of 4,096 81 us (57 steps an
// SM of 2,200 cycles, of which products and exponentials take 1,030 each: the two
// warps of a scheduler that own slots load, raise and add up at the same time).
#include <algorithm>
#include <new>

#include "chunk_plan.h"
#include "kernels.h"
#include "tensor.cuh"

namespace epikv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Steps of 128 rows: the 8 warps that own slots hold 128 scores each, and take registers from the 8 others.
constexpr int kLaunchRegs = 128, kOwnerRegs = 184, kOtherRegs = 72;
static_assert(kOwnerRegs + kOtherRegs <= 2 * kLaunchRegs, "the owners would wait for registers that nobody gives");

// N query rows a step; T tiles of 128 slots a unit, each with four warps that own its slots.
template <int D, int FMT, int N>
struct WeightShape {
  static constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  // What 4-bit keys become: halves beside steps of 16 rows, which become halves too (that many are soon done); bf16, which takes
  // two instructions more a pair, where each step's 128 rows would have to (a prompt of 4,096: 89 us, 208 by halves).
  static constexpr bool kHalf = !kBf16 && N == 16;
  static constexpr int T = D == 256 ? 1 : 2;
  static constexpr int kThreads = N == 16 ? 768 : 512;
  static constexpr int kQueryWarps = 4;
  static constexpr int kSlots = 128 * T;
  static constexpr int kKeys = kSlots * D * 2;         // bytes of a unit's keys
  static constexpr int kQuery = N * D * 2;             // of a step's rows
  static constexpr int kKeyStages = N != 16 ? (D == 64 ? 2 : 1) : kBf16 ? (D == 64 ? 5 : D == 128 ? 3 : 2) : D == 64 ? 4 : 2;
  static constexpr int kQueryStages = N == 16 ? (D == 256 ? 4 : kBf16 ? kKeyStages : 3) : D == 256 ? 2 : 4;
  // A step's rows come by one of those warps, the steps in turn; else by all.  No more of them take turns than the ring has
  // stages: a warp then knows, by its last step's wait for a stage, that all uses of the next step's stage are over but the
  // last, and one bit tells that one's end.
  static constexpr bool kTurns = N == 16;
  static constexpr int kTurnWarps = kQueryWarps < kQueryStages ? kQueryWarps : kQueryStages;
  static constexpr int kMmaWarp = 4 * T, kQueryWarp = kMmaWarp + 1, kKeyWarp = kQueryWarp + kQueryWarps;
  static constexpr int kKeyWarps = kThreads / 32 - kKeyWarp;
  static constexpr int kKeyThreads = kKeyWarps * 32;
  // Units of 4-bit rows on their way.  (Beside steps of 128 rows there is no room.)
  static constexpr int kCodeStages = kBf16 || N != 16 ? 0 : D == 64 ? 5 : D == 128 ? 3 : 2;
  using Codes = CodeRing<D, kKeyThreads, kSlots, kCodeStages>;
  static constexpr int kCodes = kKeyStages * kKeys + kQueryStages * kQuery, kRing = kCodes + Codes::kBytes;
  static constexpr uint32_t kColumns = 2 * N * T < 32 ? 32 : 2 * N * T;   // two tiles of scores for each tile of slots
};

// Units on their way, at most: codes (up to 5), the ring of keys (up to 5), two that are read and two at the waits.
constexpr int kViews = 16;

// Where a CTA's share starts, and a walk along it.
struct WeightStart {
  int b, unit, kh, place;   // places of the unit that are behind
  Entry e;
};

template <int D, int FMT, int N>
struct alignas(16) WeightShared {
  using Shape = WeightShape<D, FMT, N>;
  uint64_t keys[Shape::kKeyStages], keys_left[Shape::kKeyStages], query[Shape::kQueryStages], query_left[Shape::kQueryStages];
  uint64_t scores[2][2], taken[2][2], drained;
  uint32_t tmem;
  int gave_up;
  uint32_t there[kViews][Shape::kSlots / 32];              // the slot is in the view; units in turn
  alignas(16) float factor[Shape::kQueryStages][N];        // of a row's scores (halves; else the same for all)
  alignas(16) float lse2[Shape::kQueryStages][N];          // minus log2 of a row's sum
  alignas(16) int seen[Shape::kQueryStages][N];            // slots that the row sees
  int partly[Shape::kQueryStages][Shape::kQueryWarps];     // steps of 128 rows: not every row sees all slots of the unit
  int64_t offset[2][Shape::kSlots];
  uint32_t in_view[2][Shape::kSlots / 32];                 // beside the offsets: which of them are some
  WeightStart start[2];                                    // of the CTA's share, of the next one's
  unsigned from[2];
};

struct WeightCall {
  int layer, add;
  float* w;
  int64_t stride_seq, stride_head;
  const float* lse;
  float c;
};

// A CTA's piece of a unit.
struct WeightSegment {
  Entry e;
  int b, kh, unit;
  int slots;        // of the entry
  int token;        // the unit's first new token
  int step, steps;  // the segment's first step of the unit, steps (0: the unit has no rows, its zeros are stored)
  bool first, last; // the unit starts, ends here
  unsigned end;     // the line's place behind the unit
};

// (What is the same for all heads of a unit is formed once: units of a decode step come every 1,400 cycles.)
struct WeightWalk {
  const unsigned* pre;
  const Batch& ba;
  const WeightPlan& plan;
  unsigned x, end;
  int place, units, all, places;
  WeightSegment now;
  __device__ __forceinline__ WeightWalk(const unsigned* pre_, const Batch& ba_, const WeightPlan& plan_, const WeightStart& s,
                                        unsigned x_, unsigned end_)
      : pre(pre_), ba(ba_), plan(plan_), x(x_), end(end_), place(s.place) {
    now = {};
    now.e = s.e;
    now.b = s.b;
    now.unit = s.unit;
    now.kh = s.kh - 1;   // before the first
    entry();
    unit();
    now.last = true;
  }
  __device__ __forceinline__ void entry() {
    units = weight_units(plan, now.e.n, now.e.len);
    now.slots = weight_slots(plan, now.e.n, now.e.len);
  }
  __device__ __forceinline__ void unit() {
    now.token = weight_token(plan, now.e.n, now.e.len, now.unit);
    all = weight_steps(plan, now.e.n, now.e.len, now.unit);
    places = max(all + plan.extra, 1);
  }
  __device__ __forceinline__ void to_next_unit() {
    if (++now.kh < plan.heads) return;
    now.kh = 0;
    if (++now.unit == units) {
      now.unit = 0;
      do ++now.b;
      while (pre[now.b + 1] == pre[now.b]);
      now.e.tok0 = ba.cu_new[now.b];
      now.e.n = ba.cu_new[now.b + 1] - now.e.tok0;
      now.e.seq = ba.seq_ids[now.b];
      now.e.len = ba.len[(int64_t)now.b * ba.len_stride];
      entry();
    }
    unit();
  }
  // Where units have one step or none: on to the n-th of those with one that follow; false at the share's end.
  __device__ __forceinline__ bool skip(int n) {
    do {
      if (x >= end) return false;
      to_next_unit();
      ++x;
    } while (all == 0 || --n > 0);
    now.step = 0;
    now.steps = 1;
    return true;
  }
  // Moves `now` on to the next segment; false at the share's end.  kOne: units have one step or none.
  template <bool kOne>
  __device__ __forceinline__ bool next() {
    if (x >= end) return false;
    to_next_unit();   // (a segment that does not end its unit is the share's last)
    if constexpr (kOne) {
      ++x;
      now.step = 0;
      now.steps = all;
      now.first = now.last = true;
      return true;
    }
    const int take = (int)min((unsigned)(places - place), end - x);
    now.step = step_of_place(plan, place);
    now.steps = min(step_of_place(plan, place + take), all) - now.step;
    now.first = place == 0;
    now.last = place + take == places;
    now.end = x + (places - place);
    x += take;
    place = 0;
    return true;
  }
};

// kShared: the walk stands in shared memory, for a warp whose registers are full (steps of 128 rows), and its first lane moves
// it on.
template <bool kShared>
__device__ __forceinline__ bool move_on(WeightWalk& walk, int lane) {
  if constexpr (!kShared) return walk.next<true>();
  __syncwarp();
  int more = 0;
  if (lane == 0) more = walk.next<false>();
  __syncwarp();   // (a shuffle does not order what the others read of the walk)
  return __shfl_sync(0xffffffffu, more, 0);
}

// Places before each entry of the batch, by a warp; an entry that cannot be taken has none, nor has one that takes the sum to
// kTooManyTiles and those behind it.
__device__ __forceinline__ void line_up_weights(unsigned* pre, const Batch& ba, const AttnDims& dm, const WeightPlan& plan,
                                                int32_t* err, int lane) {
  unsigned before = 0;
  for (int b0 = 0; b0 < ba.n_seq; b0 += 32) {
    const int b = b0 + lane;
    Entry e;
    unsigned n = 0;
    if (b < ba.n_seq && batch_entry(ba, dm, b, plan.causal, err, &e)) n = count_of(weight_entry(plan, e.n, e.len));
    unsigned upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto = add_counts(upto, v);
    }
    upto = add_counts(upto, before);
    if (upto == kTooManyTiles && n) set_error(err, EPIKV_DEV_CAPACITY);
    const unsigned over = __ballot_sync(0xffffffffu, upto == kTooManyTiles);
    const unsigned kept = __shfl_sync(0xffffffffu, upto, over ? max(__ffs(over) - 2, 0) : 31);
    const unsigned good = over == 0 ? upto : over & 1 ? before : kept;   // the last sum below the limit
    if (upto == kTooManyTiles) upto = good;
    if (b < ba.n_seq) pre[b + 1] = upto;
    before = __shfl_sync(0xffffffffu, upto, 31);
    if (over) {   // everything behind is refused too
      for (int i = b0 + 32 + lane; i < ba.n_seq; i += 32) pre[i + 1] = before;
      break;
    }
  }
  if (lane == 0) pre[0] = 0;
}

// Where in the line place x is, by one thread; returns where a share that starts there does.
__device__ __forceinline__ unsigned find_place(WeightStart* s, unsigned x, const unsigned* pre, const Batch& ba,
                                           const WeightPlan& plan) {
  int lo = 0, hi = ba.n_seq - 1;   // the entry with pre[b] <= x < pre[b + 1]
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (x < pre[mid + 1]) hi = mid;
    else lo = mid + 1;
  }
  Entry e;
  e.tok0 = ba.cu_new[lo];
  e.n = ba.cu_new[lo + 1] - e.tok0;
  e.seq = ba.seq_ids[lo];
  e.len = ba.len[(int64_t)lo * ba.len_stride];
  unsigned at = x - pre[lo];
  const int alike = weight_alike(plan, e.n, e.len), last = weight_units(plan, e.n, e.len) - 1;
  unsigned wide = (unsigned)weight_places(plan, e.n, e.len, 0) * plan.heads;
  int unit = min((int)(at / wide), alike);
  at -= unit * wide;
  for (; unit < last; ++unit) {
    wide = (unsigned)weight_places(plan, e.n, e.len, unit) * plan.heads;
    if (at < wide) break;
    at -= wide;
  }
  const unsigned places = (unsigned)weight_places(plan, e.n, e.len, unit);
  s->b = lo;
  s->unit = unit;
  s->kh = (int)(at / places);
  const unsigned behind = at % places, from = moved_unit_start(plan, x, x - behind);
  s->place = (int)(from - (x - behind));
  s->e = e;
  return from;
}

// ------------------------------------------------------------------ keys
template <int D, int FMT, int N>
struct KeyCopier {
  using Shape = WeightShape<D, FMT, N>;
  static constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  static constexpr int kThreads = Shape::kKeyThreads, kPer = kBf16 ? D / 8 : D / 32;   // 16-byte pieces of a head's row in the cache
  enum {
    kPieces = Shape::kSlots * kPer,
    kLag = Shape::kKeyStages - 1 < 3 ? Shape::kKeyStages - 1 : 3,   // units in flight behind the newest
  };
  char* ring;
  WeightShared<D, FMT, N>& sh;
  const TensorWaiter& wait;
  const AttnDims& dm;
  const KvDev& kv;
  const LayerMaps& maps;
  int layer;
  int32_t* err;
  int tid, lane, warp;

  __device__ __forceinline__ uint32_t stage(int i) const { return smem_u32(ring + i % Shape::kKeyStages * Shape::kKeys); }
  __device__ __forceinline__ void left(int i) const {
    if (i >= Shape::kKeyStages) wait(&sh.keys_left[i % Shape::kKeyStages], (uint32_t)(i / Shape::kKeyStages - 1) & 1);
  }
  __device__ __forceinline__ void deliver(int i) const {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive_one(&sh.keys[i % Shape::kKeyStages]);
  }
  // Element offsets of a unit's slots (-1: none) and which of them are there, for all key threads.
  __device__ __forceinline__ void offsets(int64_t* offset, uint32_t* there, const WeightSegment& g) const {
    const int s0 = g.unit * Shape::kSlots;
    for (int r = tid; r < Shape::kSlots; r += kThreads) {
      int64_t o = -1;
      if (s0 + r < g.slots) {
        o = kv_row_offset(kv, layer, g.e.seq, s0 + r, dm.T);
        if (o < 0) set_error(err, EPIKV_DEV_SLOT);
      }
      offset[r] = o;
      const uint32_t in = __ballot_sync(0xffffffffu, o >= 0);
      if (lane == 0) there[r / 32] = in;
    }
    named_sync(1, kThreads);
  }
  __device__ __forceinline__ void mark(int i, const uint32_t* there) const {   // null: all of them
    for (int w = tid; w < Shape::kSlots / 32; w += kThreads) sh.there[i % kViews][w] = there ? there[w] : 0xffffffffu;
  }

  __device__ __forceinline__ void run_bf16(WeightWalk walk) const {
    const bool flat = kv.layout == EPIKV_LAYOUT_CONTIGUOUS;
    int i = 0, pending = 0, tables = 0, table = 0, unit = -1, b = -1;
    int64_t* offset = sh.offset[0];
    int y = 0, z = 0;
    bool whole = false, known = false;
    const WeightSegment& g = walk.now;
    while (walk.next<N == 16>()) {
      if (g.steps == 0) continue;
      const int s0 = g.unit * Shape::kSlots;
      if (g.unit != unit || g.b != b) {   // the heads of the same slots follow one another
        unit = g.unit;
        b = g.b;
        known = false;
        whole = maps.slots && min(s0 + Shape::kSlots, g.slots) <= maps.end;
        if (whole) {
          y = s0 + lane * maps.slots;
          z = g.e.seq;
          bool there = true;
          if (!flat && y < g.slots && lane * maps.slots < Shape::kSlots) {
            const int bi = y / kv.block_size;
            y -= bi * kv.block_size;
            z = bi < kv.max_blocks
                    ? __ldg(kv.block_table + (int64_t)layer * kv.table_stride_layer + (int64_t)g.e.seq * kv.max_blocks + bi)
                    : -1;
            there = z >= 0 && z < kv.num_blocks;
          }
          whole = __all_sync(0xffffffffu, there);   // else by lanes, which report it
        }
      }
      if (whole) {
        if (pending) {
          copy_wait<0>();
          for (; pending > 0; --pending) deliver(i - pending);
        }
        left(i);
        mark(i, nullptr);
        uint64_t* bar = &sh.keys[i % Shape::kKeyStages];
        if (warp == 0) {
          const int slots = min(Shape::kSlots, (g.slots - s0 + maps.slots - 1) & -maps.slots);   // that come
          if (lane == 0) mbar_arrive_expect_tx(bar, slots * D * 2);
          __syncwarp();
          if (lane * maps.slots < slots)
            tma_load_rows(stage(i) + lane * maps.slots * (D * 2), &maps.kv[0], g.kh * (D / 64), y >> 3, z, bar);
        } else if (lane == 0) {
          mbar_arrive_one(bar);
        }
        __syncwarp();
        ++i;
        continue;
      }
      if (!known) {   // the table before may still be read: two take turns, and all threads were here for the last one
        table = tables++ & 1;
        offset = sh.offset[table];
        offsets(offset, sh.in_view[table], g);
        known = true;
      }
      left(i);
      mark(i, sh.in_view[table]);
      const uint32_t dst = stage(i);
      constexpr int kRound = 8;
      for (int x0 = tid; x0 < kPieces; x0 += kRound * kThreads) {
        int64_t o[kRound];
#pragma unroll
        for (int u = 0; u < kRound; ++u) o[u] = offset[min((x0 + u * kThreads) / kPer, Shape::kSlots - 1)];
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
          const int x = x0 + u * kThreads, r = x / kPer, c = x % kPer;
          if (x < kPieces)
            copy_async16(dst + tile_at<D>(r, c), kv.base[0] + (o[u] < 0 ? 0 : (o[u] + g.kh * D + c * 8) * 2), o[u] < 0 ? 0 : 16);
        }
      }
      copy_commit();
      ++i;
      if (++pending > kLag) {
        copy_wait<kLag>();
        deliver(i - pending);
        --pending;
      }
    }
    copy_wait<0>();
    for (; pending > 0; --pending) deliver(i - pending);
    if (*wait.gave_up && warp == 0)   // the CTA may not end before its copies have landed
      for (int k = max(0, i - Shape::kKeyStages); k < i; ++k)
        mbar_wait_bounded(&sh.keys[k % Shape::kKeyStages], (uint32_t)(k / Shape::kKeyStages) & 1, kTensorWaitNs);
  }

  // 4-bit rows: the codes of the next units are under way while one's become halves.
  __device__ __forceinline__ void run_q4(WeightWalk walk) const {
    int tables = 0, unit = -1, b = -1, found = 0, table = 0;
    const WeightSegment& g = walk.now;
    bool moved = false;  // to other slots
    auto ahead = [&] {   // the next segment with rows, its slots' offsets, and which of them are there
      while (walk.next<N == 16>()) {
        if (g.steps == 0) continue;
        moved = g.unit != unit || g.b != b;   // the heads of the same slots follow one another
        if (moved) {
          unit = g.unit;
          b = g.b;
          table = tables++ & 1;
          offsets(sh.offset[table], sh.in_view[table], g);
        }
        mark(found++, sh.in_view[table]);
        return true;
      }
      return false;
    };
    if constexpr (Shape::kCodeStages > 0) {
      constexpr int kStages = Shape::kCodeStages;
      static_assert(kStages <= 8, "places");
      const typename Shape::Codes raw{smem_u32(ring + Shape::kCodes)};
      typename Shape::Codes::Sources from;
      uint32_t places = 0;   // 4 bits for each unit on its way: where the head's scales stand in their 16 bytes
      auto send = [&] {      // a group for each unit, empty behind the share's end
        if (ahead()) {
          const int scales = scale_offset(dm, g.kh), at = (found - 1) % 8 * 4;
          if (moved) raw.look(&from, kv.base[0], sh.offset[table], tid);
          raw.issue(found - 1, from, g.kh * (D / 2), scales, tid);
          places = (places & ~(15u << at)) | (scales & 15u) << at;
        }
        copy_commit();
      };
#pragma unroll 1
      for (int k = 0; k < kStages; ++k) send();
#pragma unroll 1
      for (int i = 0; i < found; ++i) {
        copy_wait<kStages - 1>();
        __syncwarp();
        left(i);
        raw.store(i, stage(i), places >> i % 8 * 4 & 15, tid);
        deliver(i);
        send();
      }
    } else {
      constexpr int kStep = kThreads / (D / 32), kRounds = (Shape::kSlots + kStep - 1) / kStep, kAtOnce = kRounds < 6 ? kRounds : 6;
      for (int i = 0; ahead(); ++i) {
        left(i);
        for (int first = 0; first < Shape::kSlots; first += kAtOnce * kStep) {
          CodeRows<D, kThreads, kAtOnce, true> c;
          c.load(kv.base[0], sh.offset[table], g.kh * (D / 2), scale_offset(dm, g.kh), first, Shape::kSlots, tid);
          c.store(stage(i), first, Shape::kSlots, tid);
        }
        deliver(i);
      }
    }
  }
};

// ------------------------------------------------------------------ query rows
// bf16 rows are copied as they are, those that become halves are under way while the warp's step before is stored.  (A unit of
// a decode step takes a warp 2,900 cycles from end to end, so several take turns; of 128 rows each takes a quarter.)
template <int D, int FMT, int N>
__device__ __forceinline__ void copy_queries(char* ring, WeightShared<D, FMT, N>& sh, const TensorWaiter& wait, const AttnState& st,
                                             const AttnDims& dm, const WeightCall& call, const Rows& q, WeightWalk& walk,
                                             int warp, int lane) {
  using Shape = WeightShape<D, FMT, N>;
  constexpr bool kHalf = Shape::kHalf;
  constexpr int R = Shape::kTurns ? N : N / Shape::kQueryWarps;   // rows of the warp
  constexpr int kPer = D / 8, kRows = 32 / kPer;         // pieces of a row; rows at once
  constexpr int kLoads = (R + kRows - 1) / kRows;
  const int piece = lane % kPer, sub = lane / kPer;
  const WeightSegment& g = walk.now;
  // the lane's row of a step is head `head` of the unit's token `token`; both go on from step to step
  const int rep = dm.rep, row0 = Shape::kTurns ? 0 : warp * R, own = row0 + lane, own_token = own / rep, own_head = own - own_token * rep;
  const int more_tokens = N / rep, more_heads = N - more_tokens * rep;
  int k = -1, token = 0, head = 0;
  struct Row {
    uint64_t src;    // the lane's row (one that is not there: the step's first, nobody looks at it)
    float lse;
    int seen;
  };
  auto row_of = [&] {
    Row r;
    const int at = g.token + token, hq = g.kh * rep + head;
    const bool in = lane < R && at < g.e.n;
    r.src = (uint64_t)(q.p + ((int64_t)(g.e.tok0 + (in ? at : g.token)) * q.st + (in ? hq : g.kh * rep) * q.sh) * 2);
    r.lse = in ? load_now(call.lse + (int64_t)(g.e.tok0 + at) * dm.Hq + hq) : -INFINITY;
    r.seen = walk.plan.causal ? g.e.len + at + 1 : g.e.len;
    return r;
  };
  auto advance = [&] {   // to the next step; false at the share's end
    if (++k < g.steps) {
      token += more_tokens;
      head += more_heads;
      if (head >= rep) {
        head -= rep;
        ++token;
      }
      return true;
    }
    do {
      if (!move_on<N != 16>(walk, lane)) return false;
    } while (g.steps == 0);
    k = 0;
    token = own_token;
    head = own_head;
    if (g.step) {
      token = (g.step * N + own) / rep;
      head = g.step * N + own - token * rep;
    }
    return true;
  };
  auto source = [&](const Row& r, int row) {   // the lane's piece of a row
    return reinterpret_cast<const uint4*>(__shfl_sync(0xffffffffu, r.src, row & 31)) + piece;
  };
  auto tell = [&](const Row& r, int qs, float back) {   // what is needed beside the rows
    if (lane < R) {
      sh.lse2[qs][own] = -r.lse * kLog2e;
      if constexpr (kHalf) sh.factor[qs][own] = score_factor(call.c * back * head_scale(st, dm, 0, call.layer, g.kh));
      sh.seen[qs][own] = r.lse == -INFINITY ? 0 : r.seen;   // (the row saw nothing)
    }
    if constexpr (N != 16) {
      const int upto = min(g.unit * Shape::kSlots + Shape::kSlots, g.slots);
      const bool partly = __any_sync(0xffffffffu, lane < R && (r.lse == -INFINITY || r.seen < upto));
      if (lane == 0) sh.partly[qs][warp] = partly;
    }
  };
  auto deliver = [&](int step) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive_one(&sh.query[step % Shape::kQueryStages]);
  };
  auto stage = [&](int step) {   // waits for it to be free
    const int qs = step % Shape::kQueryStages;
    if (step >= Shape::kQueryStages) wait(&sh.query_left[qs], (uint32_t)(step / Shape::kQueryStages - 1) & 1);
    return smem_u32(ring + Shape::kKeyStages * Shape::kKeys + qs * Shape::kQuery);
  };
  // Of a step of 16 rows only those that are some: what stands in the others' columns is not looked at.
  auto loads_of = [&] { return N == 16 ? (min(N, (g.e.n - g.token) * rep) + kRows - 1) / kRows : kLoads; };
  int step = -1;
  auto go_on = [&] {   // to the warp's next step
    if constexpr (Shape::kTurns) {
      const int by = step < 0 ? warp + 1 : Shape::kTurnWarps;
      token = own_token;
      head = own_head;
      step += by;
      return warp < Shape::kTurnWarps && walk.skip(by);
    } else {
      ++step;
      return advance();
    }
  };
  bool more = go_on();
  Row next = {};
  if (more) next = row_of();
  if constexpr (!kHalf) {
    // Steps in flight behind the newest: none where warps take turns (the stage of a warp's next step may be that of one
    // behind this one's).
    constexpr int kLag = Shape::kTurns ? 0 : 1;
    int pending = 0, last = -1;
    auto drain = [&] {
      copy_wait<0>();
      for (; pending > 0; --pending) deliver(last + 1 - pending);
    };
    while (more) {
      // before it waits for a stage the warp hands on what is on its way
      if (step >= Shape::kQueryStages && pending &&
          !__all_sync(0xffffffffu, mbar_try_wait(&sh.query_left[step % Shape::kQueryStages],
                                                 (uint32_t)(step / Shape::kQueryStages - 1) & 1)))
        drain();
      const uint32_t dst = stage(step);
      const int loads = loads_of();
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        if (l >= loads) break;
        const int row = l * kRows + sub;
        const uint4* from = source(next, row);
        if (row < R) copy_async16(dst + tile_at<D>(row0 + row, piece), from, 16);
      }
      copy_commit();
      tell(next, step % Shape::kQueryStages, 1.f);
      last = step;
      more = go_on();
      if (more) next = row_of();
      if (++pending > kLag) {
        copy_wait<kLag>();
        deliver(last + 1 - pending);
        --pending;
      }
    }
    drain();
  } else {
    constexpr int kMost = N == 16 ? 4 : 8, kBatch = kLoads < kMost ? kLoads : kMost;   // loads in flight
    uint4 v[kBatch];
    auto load = [&](const Row& r, int l0) {
#pragma unroll
      for (int l = 0; l < kBatch; ++l) v[l] = load_now(source(r, (l0 + l) * kRows + sub));
    };
    if (more) load(next, 0);
    while (more) {
      const Row now = next;
      const int loads = loads_of();
      const uint32_t dst = stage(step);
      float back = 1.f;
#pragma unroll 1
      for (int l0 = 0; l0 < loads; l0 += kBatch) {
        if (l0) load(now, l0);
        float undo[kBatch];   // of the row that the lane's piece is of
        halves_of<kPer, kBatch>(v, undo);
#pragma unroll
        for (int l = 0; l < kBatch; ++l) {
          const int row = (l0 + l) * kRows + sub;
          const float mine = __shfl_sync(0xffffffffu, undo[l], lane % kRows * kPer);
          if (lane / kRows == l0 + l) back = mine;
          if (row < R) sts16(dst + tile_at<D>(row0 + row, piece), v[l]);
        }
      }
      tell(now, step % Shape::kQueryStages, back);
      deliver(step);
      more = go_on();
      if (more) {
        next = row_of();
        load(next, 0);
      }
    }
  }
}

// ------------------------------------------------------------------ products
template <int D, int FMT, int N>
__device__ __forceinline__ void issue_units(uint32_t ring, WeightShared<D, FMT, N>& sh, const TensorWaiter& wait, WeightWalk walk,
                                            uint32_t tmem) {
  using Shape = WeightShape<D, FMT, N>;
  constexpr uint32_t kScores = product_of(128, N, !Shape::kHalf, false);
  const uint64_t k0 = rows_operand<D>(ring), q0 = rows_operand<D>(ring + Shape::kKeyStages * Shape::kKeys);
  const WeightSegment& g = walk.now;
  int step = 0;
  for (int i = 0; walk.next<N == 16>();) {
    const int steps = __shfl_sync(0xffffffffu, g.steps, 0);
    if (steps == 0) continue;
    const int ks = i % Shape::kKeyStages;
    wait(&sh.keys[ks], (uint32_t)(i / Shape::kKeyStages) & 1);
    for (int k = 0; k < steps; ++k, ++step) {
      const int qs = step % Shape::kQueryStages, buf = step & 1;
      wait(&sh.query[qs], (uint32_t)(step / Shape::kQueryStages) & 1);
      const uint64_t b = q0 + (uint32_t)(qs * (Shape::kQuery >> 4));
#pragma unroll
      for (int t = 0; t < Shape::T; ++t) {
        const uint64_t a = k0 + (uint32_t)(ks * (Shape::kKeys >> 4) + t * (128 * D * 2 >> 4));
        if (step >= 2) wait(&sh.taken[t][buf], (uint32_t)(step / 2 - 1) & 1);
        tensor_fence_after();
        if (elected()) {
#pragma unroll
          for (int x = 0; x < D / 16; ++x)
            multiply(tmem + (2 * t + buf) * N, a + rows_step(x), b + rows_step(x), kScores, x > 0);
          products_done(&sh.scores[t][buf]);
          if (t + 1 == Shape::T) {
            products_done(&sh.query_left[qs]);
            if (k + 1 == steps) products_done(&sh.keys_left[ks]);
          }
        }
        __syncwarp();
      }
    }
    ++i;
  }
}

// ------------------------------------------------------------------ sums
template <int D, int FMT, int N>
__device__ __forceinline__ void add_up(WeightShared<D, FMT, N>& sh, const TensorWaiter& wait, const AttnState& st,
                                       const AttnDims& dm, const WeightCall& call, float* part0,
                                       float* part1, ChunkSplit* split, unsigned total, int ctas, WeightWalk& walk,
                                       uint32_t tmem, int t, int tid) {
  using Shape = WeightShape<D, FMT, N>;
  const WeightSegment& g = walk.now;
  int step = 0;
  const int lane = tid & 31, own = t * 128 + tid;
  for (int i = 0; move_on<N != 16>(walk, lane);) {
    const int s = g.unit * Shape::kSlots + own;
    float* to = call.w + g.e.seq * call.stride_seq + g.kh * call.stride_head + s;
    const bool alone = g.first && g.last, mine = s < g.slots;
    float old = 0.f;   // on its way while the scores are formed
    if (call.add && alone && mine) old = *to;
    if (g.steps == 0) {
      if (mine && !call.add) *to = 0.f;
      continue;
    }
    const int ks = i % Shape::kKeyStages, rows = (g.e.n - g.token) * walk.plan.rep;   // (16 rows are one step)
    const float c = score_factor(FMT == EPIKV_CACHE_BF16 ? call.c : call.c * head_scale(st, dm, 0, call.layer, g.kh));
    f32x2 sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = f2_pack(0.f, 0.f);
    for (int k = 0; k < g.steps; ++k, ++step) {
      const int qs = step % Shape::kQueryStages, buf = step & 1;
      wait(&sh.scores[t][buf], (uint32_t)(step / 2) & 1);
      tensor_fence_after();
      const float4* lse2 = reinterpret_cast<const float4*>(sh.lse2[qs]);
      const float4* factor = reinterpret_cast<const float4*>(sh.factor[qs]);
      bool partly = false;
      if constexpr (N != 16) {
#pragma unroll
        for (int w = 0; w < Shape::kQueryWarps; ++w) partly |= sh.partly[qs][w] != 0;
      }
      uint32_t x[N];   // all columns at once: their exponentials follow one another without a pause
      const uint32_t from = tmem + (2 * t + buf) * N;
      if constexpr (N == 16) {
        tmem_load16(from, x);
      } else {
#pragma unroll
        for (int j = 0; j < N; j += 32) tmem_load32(from + j, x + j);
      }
      tmem_wait_load<N>(x);
      tensor_fence_before();
      mbar_arrive_one(&sh.taken[t][buf]);
      auto columns = [&](auto masked) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
          if (N == 16 && j >= rows) break;
          const float4 l = lse2[j / 4];
          const float4 f = Shape::kHalf ? factor[j / 4] : make_float4(c, c, c, c);
          const f32x2 a = f2_fma(f2_pack(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), f2_pack(f.x, f.y), f2_pack(l.x, l.y));
          const f32x2 b = f2_fma(f2_pack(__uint_as_float(x[j + 2]), __uint_as_float(x[j + 3])), f2_pack(f.z, f.w), f2_pack(l.z, l.w));
          float p[4] = {exp2_fast(f2_lo(a)), exp2_fast(f2_hi(a)), exp2_fast(f2_lo(b)), exp2_fast(f2_hi(b))};
          if constexpr (decltype(masked)::value) {
            const int4 e = reinterpret_cast<const int4*>(sh.seen[qs])[j / 4];
            p[0] = s < e.x ? p[0] : 0.f;
            p[1] = s < e.y ? p[1] : 0.f;
            p[2] = s < e.z ? p[2] : 0.f;
            p[3] = s < e.w ? p[3] : 0.f;
          }
          sum[j / 2 & 2] = f2_add(sum[j / 2 & 2], f2_pack(p[0], p[1]));
          sum[(j / 2 & 2) + 1] = f2_add(sum[(j / 2 & 2) + 1], f2_pack(p[2], p[3]));
        }
      };
      if (N == 16 || partly) columns(std::true_type{});
      else columns(std::false_type{});
      __syncwarp();
      if (lane == 0) mbar_arrive_one(&sh.query_left[qs]);
    }
    const f32x2 both = f2_add(f2_add(sum[0], sum[1]), f2_add(sum[2], sum[3]));
    float w = f2_lo(both) + f2_hi(both);
    const bool there = sh.there[i % kViews][own / 32] >> lane & 1;
    __syncwarp();
    if (lane == 0) mbar_arrive_one(&sh.keys_left[ks]);
    if (!there) w = 0.f;
    if (alone) {
      if (mine) *to = old + w;
    } else {   // a part for the second kernel
      (g.first ? part1 : part0)[own] = w;
      if (own == 0 && g.first)
        *split = {1, g.b, g.kh, g.unit * Shape::kSlots, min(Shape::kSlots, g.slots - g.unit * Shape::kSlots),
                  share_of(g.end - 1, total, ctas) - (int)blockIdx.x + 1, {0, 0}};
    }
    ++i;
  }
}

template <int D, int FMT, int N>
__global__ void __launch_bounds__(WeightShape<D, FMT, N>::kThreads, 1)
    weights_kernel(AttnState st, AttnDims dm, const __grid_constant__ WeightPlan plan, const __grid_constant__ Batch ba,
                   WeightCall call, Rows q, KvDev kv, const __grid_constant__ LayerMaps maps) {
  using Shape = WeightShape<D, FMT, N>;
  extern __shared__ char dynamic[];
  char* ring = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  unsigned* pre = reinterpret_cast<unsigned*>(ring + Shape::kRing);
  __shared__ WeightShared<D, FMT, N> sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == Shape::kMmaWarp) tmem_alloc(&sh.tmem, Shape::kColumns);
  if (tid == 0) {
    for (int i = 0; i < Shape::kQueryStages; ++i) {
      mbar_init(&sh.query[i], Shape::kTurns ? 1 : Shape::kQueryWarps);
      mbar_init(&sh.query_left[i], 1 + Shape::kMmaWarp);
    }
    for (int i = 0; i < Shape::kKeyStages; ++i) {
      mbar_init(&sh.keys[i], Shape::kKeyWarps);
      mbar_init(&sh.keys_left[i], 1 + Shape::kMmaWarp);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sh.scores[i >> 1][i & 1], 1);
      mbar_init(&sh.taken[i >> 1][i & 1], 128);
    }
    mbar_init(&sh.drained, 1);
    sh.gave_up = 0;
    fence_barrier_init();
  }
  pdl_wait();
  pdl_trigger();
  ChunkSplit* split = reinterpret_cast<ChunkSplit*>(st.splits) + blockIdx.x;
  if (warp == 0) {
    line_up_weights(pre, ba, dm, plan, st.err, lane);
    __syncwarp();
    const unsigned total = pre[ba.n_seq];
    const int ctas = (int)min(total, (unsigned)kAttnCtas);
    if (lane == 0) *split = {};
    if (lane < 2 && (int)blockIdx.x < ctas)
      sh.from[lane] = (int)blockIdx.x + lane < ctas
                          ? find_place(&sh.start[lane], share_start(blockIdx.x + lane, total, ctas), pre, ba, plan)
                          : total;
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  const uint32_t tmem = sh.tmem;
  const unsigned total = pre[ba.n_seq];
  const int cta = blockIdx.x, ctas = (int)min(total, (unsigned)kAttnCtas);
  if (cta < ctas) {
    const TensorWaiter wait{&sh.gave_up, st.err};
    const WeightWalk start(pre, ba, plan, sh.start[0], sh.from[0], sh.from[1]);
    __shared__ alignas(16) char walks[N == 16 ? 1 : Shape::kKeyWarp][sizeof(WeightWalk)];
    WeightWalk own = start;
    WeightWalk* shared = reinterpret_cast<WeightWalk*>(walks[N == 16 ? 0 : min(warp, Shape::kKeyWarp - 1)]);
    if (N != 16 && lane == 0 && warp < Shape::kKeyWarp) new (shared) WeightWalk(start);
    __syncwarp();
    WeightWalk& walk = N == 16 ? own : *shared;
    if (warp < Shape::kMmaWarp) {
      if constexpr (N != 16) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kOwnerRegs));
      float* part = st.part + (int64_t)cta * 2 * Shape::kSlots;
      add_up<D, FMT, N>(sh, wait, st, dm, call, part, part + Shape::kSlots, split, total, ctas, walk,
                        tmem + ((uint32_t)(warp & 3) << 21), warp >> 2, tid & 127);
    } else {
      if constexpr (N != 16) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kOtherRegs));
      if (warp == Shape::kMmaWarp) {
        issue_units<D, FMT, N>(smem_u32(ring), sh, wait, own, tmem);
        if (elected()) products_done(&sh.drained);   // tensor memory is not freed under products, whatever waits gave up
        __syncwarp();
        mbar_wait_bounded(&sh.drained, 0, kTensorWaitNs);
      } else if (warp < Shape::kKeyWarp) {
        copy_queries<D, FMT, N>(ring, sh, wait, st, dm, call, q, walk, warp - Shape::kQueryWarp, lane);
      } else {
        const KeyCopier<D, FMT, N> copier{ring, sh, wait, dm, kv, maps, call.layer, st.err, tid - Shape::kKeyWarp * 32, lane,
                                          warp - Shape::kKeyWarp};
        if constexpr (FMT == EPIKV_CACHE_BF16) copier.run_bf16(own);
        else copier.run_q4(own);
      }
    }
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  if (warp == Shape::kMmaWarp) tmem_free(tmem, Shape::kColumns);
}

// Joins the parts of a unit that several shares hold, in their order.  A CTA for each share that starts such a unit; a
// thread a slot.
__global__ void __launch_bounds__(256) weights_join_kernel(AttnState st, Batch ba, WeightCall call, int slots) {
  pdl_wait();
  pdl_trigger();
  const ChunkSplit s = reinterpret_cast<const ChunkSplit*>(st.splits)[blockIdx.x];
  const int own = threadIdx.x;
  if (!s.there || own >= s.rows) return;
  float w = st.part[(int64_t)(2 * blockIdx.x + 1) * slots + own];
  for (int i = 1; i < s.parts; ++i) w += st.part[(int64_t)2 * (blockIdx.x + i) * slots + own];
  float* to = call.w + ba.seq_ids[s.b] * call.stride_seq + s.kh * call.stride_head + s.row0 + own;
  *to = call.add ? *to + w : w;
}

template <int D, int FMT, int N>
constexpr int weights_smem(int n_seq) { return WeightShape<D, FMT, N>::kRing + 1024 + (n_seq + 1) * 4; }

template <int D, int FMT, int N>
cudaError_t run_weights(const AttnState& st, const AttnDims& dm, const Batch& ba, bool causal, int last,
                        const WeightCall& call, const Rows& q, const KvDev& kv, cudaStream_t stream) {
  using Shape = WeightShape<D, FMT, N>;
  static_assert(weights_smem<D, FMT, N>(kMaxSeqs) + sizeof(WeightShared<D, FMT, N>) <= 227 * 1024, "shared memory");
  const WeightPlan plan = {Shape::kSlots, Shape::T == 1 ? 7 : 8, N, N == 16 ? 4 : 7, dm.rep, causal ? 1 : 0, dm.H, last, N == 16 ? 0 : kUnitPlaces};
  const cudaError_t e = pdl_launch(weights_kernel<D, FMT, N>, dim3(kAttnCtas), Shape::kThreads, weights_smem<D, FMT, N>(ba.n_seq),
                                   stream, st, dm, plan, ba, call, q, kv, layer_maps(dm, call.layer, kv, 128));
  if (e != cudaSuccess || N == 16) return e;   // 16 rows are one step: no unit is split
  return pdl_launch(weights_join_kernel, dim3(kAttnCtas), Shape::kSlots, 0, stream, st, ba, call, (int)Shape::kSlots);
}

// *runs becomes false where the compiler gave the kernel other registers than its warps' exchange of them counts on.
template <int D, int FMT, int N>
cudaError_t allow_weights(bool* runs) {
  cudaFuncAttributes at;
  const cudaError_t e = cudaFuncGetAttributes(&at, weights_kernel<D, FMT, N>);
  if (e != cudaSuccess) return e;
  if (N != 16 && at.numRegs != kLaunchRegs) *runs = false;
  return cudaFuncSetAttribute(weights_kernel<D, FMT, N>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              weights_smem<D, FMT, N>(kMaxSeqs));
}

template <int D, int FMT>
cudaError_t prepare_dim(bool* runs) {
  const cudaError_t e = allow_weights<D, FMT, 16>(runs);
  return e == cudaSuccess ? allow_weights<D, FMT, 128>(runs) : e;
}

// ------------------------------------------------------------ into the eviction context
__global__ void __launch_bounds__(256) weigh_kernel(DevState st, Dims dm, const int32_t* __restrict__ seq_ids,
                                                    const float* __restrict__ w, int64_t stride_seq, int64_t stride_head,
                                                    int heads, float decay) {
  pdl_wait();
  pdl_trigger();
  const int seq = seq_ids[blockIdx.y];
  if ((unsigned)seq >= (unsigned)dm.S) {
    if (threadIdx.x == 0) set_error(st.err, EPIKV_DEV_BATCH);
    return;
  }
  const int n = st.n_cache[seq];
  if (st.first_changed[seq] < n) {   // selected, not compacted: the scores stand by other slots than the weights
    if (threadIdx.x == 0) set_error(st.err, EPIKV_DEV_KEPT);
    return;
  }
  float* score = st.score[kind_index(EPIKV_SCORE_WEIGHT)] + (size_t)seq * dm.T;
  for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < n; s += gridDim.x * blockDim.x) {
    const float* p = w + seq * stride_seq + s;
    const float old = score[s];
    float sum = p[0];
#pragma unroll 8
    for (int h = 1; h < heads; ++h) sum = __fadd_rn(sum, p[h * stride_head]);
    score[s] = __fadd_rn(__fmul_rn(decay, old), sum);
  }
}

}  // namespace

cudaError_t weights_prepare(const AttnDims& dm, bool* runs) {
  *runs = true;
  const bool bf16 = dm.fmt == EPIKV_CACHE_BF16;
  if (dm.d == 64) return bf16 ? prepare_dim<64, EPIKV_CACHE_BF16>(runs) : prepare_dim<64, EPIKV_CACHE_E2M1>(runs);
  if (dm.d == 128) return bf16 ? prepare_dim<128, EPIKV_CACHE_BF16>(runs) : prepare_dim<128, EPIKV_CACHE_E2M1>(runs);
  return bf16 ? prepare_dim<256, EPIKV_CACHE_BF16>(runs) : prepare_dim<256, EPIKV_CACHE_E2M1>(runs);
}

size_t weights_part_floats() { return (size_t)2 * kAttnCtas * 256; }

cudaError_t launch_attention_weights(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal,
                                     int last, const Rows& q, const float* lse, bool add, float* w, int64_t stride_seq,
                                     int64_t stride_head, const KvDev& kv, cudaStream_t stream) {
  const WeightCall call = {layer, add, w, stride_seq, stride_head, lse, dm.scale * kLog2e};
  const int64_t tokens = last && last < ba.max_new ? last : ba.max_new;
  const bool few = tokens * dm.rep <= 16, bf16 = dm.fmt == EPIKV_CACHE_BF16;
  auto pick = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return bf16 ? (few ? run_weights<D, EPIKV_CACHE_BF16, 16> : run_weights<D, EPIKV_CACHE_BF16, 128>)
                : (few ? run_weights<D, EPIKV_CACHE_E2M1, 16> : run_weights<D, EPIKV_CACHE_E2M1, 128>);
  };
  auto go = dm.d == 64    ? pick(std::integral_constant<int, 64>{})
            : dm.d == 128 ? pick(std::integral_constant<int, 128>{})
                          : pick(std::integral_constant<int, 256>{});
  return go(st, dm, ba, causal, last, call, q, kv, stream);
}

cudaError_t launch_weigh(const DevState& st, const Dims& dm, int n_seq, const int32_t* seq_ids, const float* w,
                         int64_t stride_seq, int64_t stride_head, int heads, float decay, cudaStream_t stream) {
  const int blocks = (dm.T + 255) / 256, most = kAttnCtas * 8 / n_seq;   // 8 fit an SM
  return pdl_launch(weigh_kernel, dim3(std::max(1, std::min(blocks, most)), n_seq), 256, 0, stream, st, dm, seq_ids, w, stride_seq,
                    stride_head, heads, decay);
}

}  // namespace epikv
