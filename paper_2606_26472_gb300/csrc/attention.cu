// Attention of new tokens' queries over the slots of the cache.
//
//   out = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q.k_j - m),   c = scale log2(e)
//
// One pass over the slots with a running maximum m and sum per row.  What
// bounds a decode step is reading K and V once, so everything follows from
// how the bytes come in:
//
//  - A CTA takes all heads of a group (up to 8) of a run of slots, because a
//    token's row holds all heads together: whole rows go to shared memory by
//    asynchronous copies from four warps of their own, through a ring of tiles
//    deep enough to cover HBM's latency; eight warps compute, one head each
//    (fewer heads: several warps a head, each with its own part of the tile's
//    slots, joined through shared memory at the end).
//  - The slots of all entries are one line of tiles that the 152 CTAs share
//    equally (attn_plan.h), so ragged batches and single long sequences load
//    every SM alike.  What a CTA finds for an item that others work on too
//    goes to the workspace, and a second kernel joins the parts in a fixed
//    order.
//  - Products run on the warp-level tensor instructions with the slots as rows
//    (S^T = K Q^T, O^T = V^T P^T): a KV head has 1 to 8 queries in a decode
//    step, and the instruction's narrow side is 8 wide, where tcgen05's
//    narrowest shape would spend 128 x 8 outputs and a trip through tensor
//    memory on them.  P goes from one product's result layout to the other's
//    operand layout by one transposing move per 8 x 8.
//
// A 4-bit cache stays in 4 bits until the registers: the layout is such that a
// lane's channels are neighbours (any order of channels serves a dot product
// if the queries follow it), a conversion turns two codes into a half pair,
// and the product with the E4M3 scale is exact in half precision (2 + 4
// significant bits).  Queries enter as halves scaled by a power of two per
// row (exact but for channels below 2^-31 of the row's largest).
//
// Roundings to fewer than 32 bits, all of single factors (maxima, sums and
// products are held in 32):
//  - a probability over a 4-bit cache: a half times 2^7, 11 bits down to 2^-21
//    of the maximum that it is taken against, within 2^-32 below.
//    Its 2^-12 stands beside the output's own 2^-9 (the error against 64 bits
//    grows from 0.00166 to 0.00167 of the output) and beside values of 3 bits; a
//    second term would be half as many tensor instructions again, where
//    instructions bound the kernel.
//  - a probability over a bf16 cache: two bf16 terms, 16 bits, for which the
//    tensor instructions have time (HBM bounds it); one alone, of 8 bits, would
//    add an error of the output's own rounding.
//  - exponentials by the hardware's base-2 approximation: 2^-22 of each, and 0
//    below 2^-126 of the largest.
// The sums of probabilities take them unrounded, so lse has 32-bit accuracy.
//
// What it measured (one token an entry, 32 query and 8 KV heads of 128): bf16,
// 64 x 5,120 slots 201 to 204 us, 6.6 TB/s; 32 x 8,192 163 us: HBM.  4 bits, 32
// x 8,256 slots 72 to 75 us, 4.1 TB/s: 269 instructions for 16 slots of a head
// (64 of them conversions, 64 products with scales, 16 tensor instructions) at
// 0.46 a cycle and scheduler, with two computing warps each; four warps a
// scheduler (96 or 128 registers) were slower, 104 to 121 us.  2,048 slots of
// one sequence 13 us, 4 x 136 14 us: two launches and their chains of reads.
// Far from its floor where an item's 8 to 32 rows read the cache anew: 8 x 64
// tokens over 4,096 slots 270 us in bf16, 209 in 4 bits (floor 21 and 18), a
// prompt of 4,096 tokens 1.36 ms (floor 0.07).
#include "attn.cuh"
#include "attn_plan.h"
#include "maps.cuh"

namespace epikv {
namespace {

constexpr int threads_of(int d) { return 32 * (attn_group(d) + kAttnCopyWarps); }
constexpr uint64_t kWaitNs = 2000000000ull;
using Geometry = AttnGeometry;

// Row r of the tensor instruction's rows takes this slot of eight (attn_plan.h's AttnGeometry.order).
__device__ __forceinline__ int slot_of_row(uint32_t order, int r) { return (order >> (4 * r)) & 7; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int FMT>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (FMT == EPIKV_CACHE_BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The same, the sums starting at 0.
template <int FMT>
__device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (FMT == EPIKV_CACHE_BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

template <bool kTrans>
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  if constexpr (kTrans)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// Words, a 2-byte value or a byte at a shared-memory address.
template <int kWords>
__device__ __forceinline__ void lds_words(uint32_t (&w)[kWords], uint32_t p) {
  if constexpr (kWords == 1) {
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(p));
  } else if constexpr (kWords == 2) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(p));
  } else {
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3]) : "r"(p + 16 * i));
  }
}
__device__ __forceinline__ uint32_t lds_u16(uint32_t p) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(p));
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t p) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(p));
  return v;
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Both halves of a times the low or the high half of b.
template <bool kHigh>
__device__ __forceinline__ uint32_t hmul2_by(uint32_t a, uint32_t b) {
  const __half2 s = *reinterpret_cast<const __half2*>(&b);
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), kHigh ? __high2half2(s) : __low2half2(s));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 r = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t bf162_of(float lo, float hi) {
  const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}
// acc + 0 a: NaN in a half from the first value on that is infinite or NaN.
__device__ __forceinline__ void note_unbounded(uint32_t& acc, uint32_t a) {
  asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(a), "r"(0u));
}

// What brings sums that were taken against one maximum to a larger one; never 0 (2^-149 of a bounded sum is nothing,
// of an infinite one infinite).
__device__ __forceinline__ float weight_of(float x) { return fmaxf(ex2(x), __uint_as_float(1u)); }

// A warp's walk along its CTA's items, in shared memory: its first lane moves it on, and what the loops over tiles do
// not need stays out of their registers.  Tiles are counted from the CTA's first.
struct Walk {
  int b, group, run, at, tiles;   // the item, its first tile (below 0: an earlier CTA's), its tiles
  Entry e;
};
// Tiles of the runs before `end` of a group of an entry, by a whole warp: a lane has up to 2^42, so the low 26 bits and
// the others go by themselves.
__device__ __forceinline__ int64_t tiles_before(const AttnShape& sh, int n, int len, int end, int lane) {
  int64_t sum = 0;
  for (int r = lane; r < end; r += 32) sum += item_tiles(sh, n, len, r);
  const unsigned low = __reduce_add_sync(0xffffffffu, (unsigned)sum & 0x3ffffffu);
  const unsigned high = __reduce_add_sync(0xffffffffu, (unsigned)(sum >> 26));
  return ((int64_t)high << 26) + low;
}

struct Walker {
  const int* pre;
  const Batch& ba;
  const AttnDims& dm;
  const AttnShape& sh;
  int32_t* err;

  __device__ __forceinline__ void entry(Walk* w) const {
    w->group = w->run = 0;
    Entry e;
    batch_entry(ba, dm, w->b, sh.causal, err, &e);
    w->e = e;
    w->tiles = item_tiles(sh, e.n, e.len, 0);
  }
  __device__ __forceinline__ void step(Walk* w) const {
    w->at += w->tiles;
    if (++w->run == row_runs(sh, w->e.n)) {
      w->run = 0;
      if (++w->group == sh.groups) {
        do ++w->b;
        while (w->b < ba.n_seq && pre[w->b + 1] == pre[w->b]);
        if (w->b < ba.n_seq) entry(w);
        return;
      }
    }
    w->tiles = item_tiles(sh, w->e.n, w->e.len, w->run);
  }
  // From the entry's first item, `from`, to the one of the CTA's first tile, by a whole warp.
  __device__ __forceinline__ void seek(Walk* w, const Walk& from, int lane) const {
    Walk at = from;
    const int runs = row_runs(sh, at.e.n);
    if (sh.groups > 1 || runs > 1) {
      const int of_group = (pre[at.b + 1] - pre[at.b]) / sh.groups;
      at.group = -at.at / of_group;
      at.at += at.group * of_group;
      for (int r0 = 0;; r0 += 32) {
        const int t = r0 + lane < runs ? item_tiles(sh, at.e.n, at.e.len, r0 + lane) : 0;
        int upto = t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += v;
        }
        const unsigned behind = __ballot_sync(0xffffffffu, at.at + upto > 0);
        if (behind || r0 + 32 >= runs) {
          const int k = behind ? __ffs(behind) - 1 : 0;
          at.run = r0 + k;
          at.tiles = __shfl_sync(0xffffffffu, t, k);
          at.at += __shfl_sync(0xffffffffu, upto - t, k);
          break;
        }
        at.at += __shfl_sync(0xffffffffu, upto, 31);
      }
    }
    if (lane == 0) *w = at;
    __syncwarp();
  }
  // Moves the warp's walk on to the item of tile i.
  __device__ __forceinline__ void to(Walk* w, int i, int lane) const {
    if (i < w->at + w->tiles) return;
    __syncwarp();
    if (lane == 0)
      while (i >= w->at + w->tiles) step(w);
    __syncwarp();
  }
};

struct Waiter {
  volatile int* gave_up;
  int32_t* err;
  // Ends when the phase completes, or (with the error word set) when any wait of the CTA has taken too long: what
  // follows then runs on without waiting, on data that the error word disowns.
  __device__ __forceinline__ void operator()(uint64_t* bar, uint32_t parity) const {
    if (mbar_try_wait(bar, parity)) return;
    const uint64_t t0 = global_ns();
    while (!mbar_try_wait(bar, parity)) {
      if (*gave_up) return;
      if (global_ns() - t0 > kWaitNs) {
        *gave_up = 1;
        set_error(err, EPIKV_DEV_TIMEOUT);
        return;
      }
    }
  }
};

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" :: "r"(smem_u32(bar)) : "memory");
}

// ------------------------------------------------------------------ the copying warps
__device__ __forceinline__ void zero_rows(char* dst, int bytes) {
  for (int i = 0; i < bytes; i += 16) *reinterpret_cast<uint4*>(dst + i) = make_uint4(0, 0, 0, 0);
}

// A copying warp's instruction chains are what its tiles cost (one warp alone took 2,000 cycles for 18 KB, a third of
// HBM's rate), so the tiles go round four warps; what a tile needs is formed once for K and V, its table entries are read
// a turn ahead, and quotients go by a float reciprocal (exact: slots are below 2^24, and a quotient
// that is off by one is put right).
struct Divider {
  int d;
  float inv;
  __device__ __forceinline__ explicit Divider(int d_) : d(d_), inv(1.f / (float)d_) {}
  __device__ __forceinline__ int operator()(int n, int* rest) const {
    int q = (int)((float)n * inv);
    int r = n - q * d;
    if (r < 0) {
      --q;
      r += d;
    } else if (r >= d) {
      ++q;
      r -= d;
    }
    *rest = r;
    return q;
  }
};

struct Place {   // of one slot
  int entry;     // of the block table (contiguous: 0)
  int rest;      // slot within the block
};
__device__ __forceinline__ Place place_of(const KvDev& kv, const Divider& block, int layer, int seq, int slot) {
  Place p{0, slot};
  if (kv.layout == EPIKV_LAYOUT_CONTIGUOUS) return p;
  const int bi = block(slot, &p.rest);
  p.entry = bi < kv.max_blocks
                ? __ldg(kv.block_table + (int64_t)layer * kv.table_stride_layer + (int64_t)seq * kv.max_blocks + bi)
                : -1;
  return p;
}
// Element offset, or -1.
__device__ __forceinline__ int64_t offset_of(const KvDev& kv, int layer, int seq, const Place& p) {
  const int64_t base = (int64_t)layer * kv.stride_layer + (int64_t)p.rest * kv.stride_token;
  if (kv.layout == EPIKV_LAYOUT_CONTIGUOUS) return base + (int64_t)seq * kv.stride_seq;
  if (p.entry < 0 || p.entry >= kv.num_blocks) return -1;
  return base + (int64_t)p.entry * kv.stride_block;
}

// Tile i of the CTA stands in the ring's place i mod stages, and waits for the computing warps to have left it.
struct Ring {
  int stages, place, turn;   // place of the warp's next tile, times round the ring
  __device__ __forceinline__ Ring(int stages_, int first) : stages(stages_), place(first), turn(0) { wrap(); }
  __device__ __forceinline__ void wrap() {
    while (place >= stages) {
      place -= stages;
      ++turn;
    }
  }
  __device__ __forceinline__ void on(int n) {
    place += n;
    wrap();
  }
};

// 4-bit rows: a bulk copy for each run of slots that is one piece of memory (a block's, where its rows stand side by
// side), each 4 to 18 KB (a copy of a row alone keeps the copy engine for about 110 cycles: a third of HBM's rate, which
// is what rows apart or in parts cost: 32 x 4,096 slots of 11 heads 127 us, a quarter of the rate).  A lane looks after
// one run; where a tile has over 32 (rows that stand apart), the others are looked up as they are copied.
template <int D>
__device__ void copy_q4(char* smem, uint64_t* full, uint64_t* empty, const Waiter& wait, const AttnState& st,
                        const AttnDims& dm, const Geometry& ge, const KvDev& kv, int layer, const Walker& walker,
                        Walk* w, int tiles, int warp, int lane) {
  const AttnShape& sh = ge.sh;
  const bool side = kv.stride_token * 2 == ge.row_s && sh.groups == 1;
  const bool flat = kv.layout == EPIKV_LAYOUT_CONTIGUOUS;
  const int rl = run_slots(side, flat, kv.block_size);
  const Divider block(flat ? 1 : kv.block_size), runs_of(rl);
  Ring ring(ge.stages, warp);
  int seq = 0, s0 = 0, n = 0, h0 = 0, run0 = 0, at = 0, upto = 0;
  Place next{0, 0};
  // run k of the tile: slots at .. upto - 1
  auto run_of = [&](int k, int* a, int* u) {
    const int64_t begin = (int64_t)(run0 + k) * rl;
    *a = (int)max((int64_t)s0, min(begin, (int64_t)s0 + n));
    *u = (int)min(begin + rl, (int64_t)s0 + n);
  };
  auto look = [&](int x) {
    walker.to(w, x, lane);
    seq = w->e.seq;
    s0 = (x - w->at) * sh.tile;
    n = max(min(sh.tile, slots_seen(sh, w->e.n, w->e.len, w->run) - s0), 0);
    h0 = w->group * attn_group(D);
    int rest;
    run0 = runs_of(s0, &rest);
    run_of(lane, &at, &upto);
    if (at < upto) next = place_of(kv, block, layer, seq, at);
  };
  int x = warp;
  if (x < tiles) look(x);
  for (; x < tiles; x += ge.copiers) {
    const int rows = max(upto - at, 0), row0 = at - s0, n_now = n, seq_now = seq, s_now = s0, run_now = run0;
    const int64_t off = rows ? offset_of(kv, layer, seq, next) : -1;
    if (rows && off < 0) set_error(st.err, EPIKV_DEV_SLOT);
    int there = off >= 0 ? rows : 0;
    const int more = slots_behind(n_now, s_now, run_now, rl);
    for (int r = n_now - more + lane; r < n_now; r += 32) {
      const bool in = offset_of(kv, layer, seq, place_of(kv, block, layer, seq, s0 + r)) >= 0;
      there += in;
      if (!in) set_error(st.err, EPIKV_DEV_SLOT);
    }
    there = __reduce_add_sync(0xffffffffu, there);
    int a_off = 0, a_bytes = ge.row_s, b_off = 0, b_bytes = 0;   // of a row: one piece, or codes and scales
    if (!side) {
      const int heads = min(attn_group(D), dm.H - h0);
      a_off = h0 * (D / 2);
      a_bytes = heads * (D / 2);
      b_off = scale_offset(dm, h0);
      b_bytes = (heads * (D / kQuantGroup) + 15) & ~15;
    }
    if (x + ge.copiers < tiles) look(x + ge.copiers);
    uint64_t* bar = &full[ring.place];
    char* dst = smem + ring.place * (2 * ge.half_bytes);
    if (ring.turn) wait(&empty[ring.place], (ring.turn & 1) ^ 1);
    if (there < sh.tile) {  // rows that nothing fills: a probability of 0 must not meet what stood there before
      char* values = dst + ge.half_bytes;
      for (int r = n_now + lane; r < sh.tile; r += 32) zero_rows(values + r * ge.row_s, ge.row_s);
      if (off < 0)
        for (int r = 0; r < rows; ++r) {
          zero_rows(dst + (row0 + r) * ge.row_s, ge.row_s);
          zero_rows(values + (row0 + r) * ge.row_s, ge.row_s);
        }
      for (int r = n_now - more + lane; r < n_now; r += 32)
        if (offset_of(kv, layer, seq_now, place_of(kv, block, layer, seq_now, s_now + r)) < 0) {
          zero_rows(dst + r * ge.row_s, ge.row_s);
          zero_rows(values + r * ge.row_s, ge.row_s);
        }
      fence_proxy_async_smem();
      __syncwarp();
    }
    if (lane == 0) mbar_arrive_expect_tx(bar, 2 * there * (a_bytes + b_bytes));
    __syncwarp();
    auto copy = [&](int row, int64_t o, int n_rows) {
      char* d = dst + row * ge.row_s;
      const char* k = kv.base[0] + o * 2;
      const char* v = kv.base[1] + o * 2;
      tma_load_1d(d, k + a_off, n_rows * a_bytes, bar);
      tma_load_1d(d + ge.half_bytes, v + a_off, n_rows * a_bytes, bar);
      if (b_bytes) {   // single rows
        tma_load_1d(d + a_bytes, k + b_off, b_bytes, bar);
        tma_load_1d(d + ge.half_bytes + a_bytes, v + b_off, b_bytes, bar);
      }
    };
    if (off >= 0) copy(row0, off, rows);
    for (int r = n_now - more + lane; r < n_now; r += 32) {
      const int64_t o = offset_of(kv, layer, seq_now, place_of(kv, block, layer, seq_now, s_now + r));
      if (o >= 0) copy(r, o, 1);
    }
    ring.on(ge.copiers);
  }
  if (*wait.gave_up) {   // the CTA may not end before its copies have landed: this warp's last ones
    for (int j = tiles - 1; j >= 0 && j >= tiles - ge.stages; --j)
      if (j % ge.copiers == warp) mbar_wait_bounded(&full[j % ge.stages], (uint32_t)(j / ge.stages) & 1, kWaitNs);
  }
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Where 16-byte part `part` of a row's piece of 64 channels stands: rows of a block are 128 bytes apart.
__device__ __forceinline__ uint32_t swizzled(int row, int part) { return row * 128 + ((part ^ (row & 7)) << 4); }

// The cache as a tensor [pieces of 64 channels][blocks or sequences][slots of one][64 channels]; a copy takes 16 slots of
// a group's heads.
struct CacheMaps {
  CUtensorMap kv[2];
  int on;   // 0: the cache cannot be described so (blocks that 16 does not divide); rows are copied by lanes
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int c1, int c2, int c3, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      :: "r"(smem_u32(dst)), "l"(map), "r"(0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar)) : "memory");
}

// bf16 rows, 16 slots of a group's heads in one tensor copy (32 KB at 8 x 128): lane i looks after block i of the tile.
// Slots behind the last seen one come as they are; the computing warps mask them.
template <int D>
__device__ void copy_tensor(char* smem, uint64_t* full, uint64_t* empty, const Waiter& wait, const AttnState& st,
                            const AttnDims& dm, const Geometry& ge, const KvDev& kv, const CacheMaps& maps, int layer,
                            const Walker& walker, Walk* w, int tiles, int warp, int lane) {
  const AttnShape& sh = ge.sh;
  const bool flat = kv.layout == EPIKV_LAYOUT_CONTIGUOUS;
  const Divider block(flat ? 1 : kv.block_size);
  const int bytes = 16 * ge.row_s;
  Ring ring(ge.stages, warp);
  int seq = 0, group = 0;
  bool mine = false;
  Place next{0, 0};
  auto look = [&](int x) {
    walker.to(w, x, lane);
    const int at = (x - w->at) * sh.tile + 16 * lane;
    seq = w->e.seq;
    group = w->group;
    mine = 16 * lane < sh.tile && at < slots_seen(sh, w->e.n, w->e.len, w->run);
    if (mine) next = place_of(kv, block, layer, seq, at);
  };
  int x = warp;
  if (x < tiles) look(x);
  for (; x < tiles; x += ge.copiers) {
    const bool there = mine && (flat || (next.entry >= 0 && next.entry < kv.num_blocks));
    if (mine && !there) set_error(st.err, EPIKV_DEV_SLOT);
    const int c1 = next.rest, c2 = flat ? seq : next.entry, c3 = group * (attn_group(D) * D / 64);
    if (x + ge.copiers < tiles) look(x + ge.copiers);
    uint64_t* bar = &full[ring.place];
    char* dst = smem + ring.place * (2 * ge.half_bytes) + lane * bytes;
    if (ring.turn) wait(&empty[ring.place], (ring.turn & 1) ^ 1);
    const uint32_t blocks = __ballot_sync(0xffffffffu, there);
    if (__popc(blocks) * 16 < sh.tile) {   // blocks that nothing fills: a probability of 0 must not meet what stood there
      for (int b = 0; b < sh.tile / 16; ++b)
        if (!(blocks >> b & 1))
          for (int i = lane * 16; i < bytes; i += 512) {
            char* at = smem + ring.place * (2 * ge.half_bytes) + b * bytes + i;
            *reinterpret_cast<uint4*>(at) = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(at + ge.half_bytes) = make_uint4(0, 0, 0, 0);
          }
      fence_proxy_async_smem();
      __syncwarp();
    }
    if (lane == 0) mbar_arrive_expect_tx(bar, 2 * __popc(blocks) * bytes);
    __syncwarp();
    if (there) {
      tma_load_4d(dst, &maps.kv[0], c1, c2, c3, bar);
      tma_load_4d(dst + ge.half_bytes, &maps.kv[1], c1, c2, c3, bar);
    }
    ring.on(ge.copiers);
  }
  if (*wait.gave_up) {   // the CTA may not end before its copies have landed: this warp's last ones
    for (int j = tiles - 1; j >= 0 && j >= tiles - ge.stages; --j)
      if (j % ge.copiers == warp) mbar_wait_bounded(&full[j % ge.stages], (uint32_t)(j / ge.stages) & 1, kWaitNs);
  }
}

// bf16 rows of any layout, 16 bytes a lane, to where a tensor copy would put them.  Lane i reads the table entries of
// rows i, i + 32, ...  (64 x 4,096 slots, blocks of 7: 234 us; of 16, by tensor copies: 165 to 169.)
template <int D>
__device__ void copy_bf16(char* smem, uint64_t* full, uint64_t* empty, const Waiter& wait, const AttnState& st,
                          const AttnDims& dm, const Geometry& ge, const KvDev& kv, int layer, const Walker& walker,
                          Walk* w, int tiles, int warp, int lane) {
  const AttnShape& sh = ge.sh;
  constexpr int kMost = 4;   // 16 slots of up to eight warps
  const Divider block(kv.layout == EPIKV_LAYOUT_CONTIGUOUS ? 1 : kv.block_size);
  Ring ring(ge.stages, warp);
  int group = -1, pieces = 0, at_once = 1, sub = 0, col = 0;   // 16-byte pieces of a row; rows taken at once
  int seq = 0, n = 0, next_group = 0;
  Place next[kMost];
  auto look = [&](int x) {
    walker.to(w, x, lane);
    const int s0 = (x - w->at) * sh.tile;
    seq = w->e.seq;
    n = min(sh.tile, slots_seen(sh, w->e.n, w->e.len, w->run) - s0);
    next_group = w->group;
#pragma unroll
    for (int k = 0; k < kMost; ++k)
      if (lane + 32 * k < n) next[k] = place_of(kv, block, layer, seq, s0 + lane + 32 * k);
  };
  int x = warp;
  if (x < tiles) look(x);
  for (; x < tiles; x += ge.copiers) {
    if (next_group != group) {
      group = next_group;
      pieces = min(attn_group(D), dm.H - group * attn_group(D)) * (D / 8);
      at_once = pieces < 32 ? 32 / pieces : 1;
      sub = pieces < 32 ? lane / pieces : 0;
      col = pieces < 32 ? lane % pieces : lane;
    }
    int64_t from[kMost];   // byte offsets, -1: a row that is not there, which is filled with zeros
#pragma unroll
    for (int k = 0; k < kMost; ++k) {
      from[k] = -1;
      if (lane + 32 * k < n) {
        const int64_t off = offset_of(kv, layer, seq, next[k]);
        if (off < 0) set_error(st.err, EPIKV_DEV_SLOT);
        else from[k] = off * 2;
      }
    }
    if (x + ge.copiers < tiles) look(x + ge.copiers);
    if (ring.turn) wait(&empty[ring.place], (ring.turn & 1) ^ 1);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
      const uint32_t dst = smem_u32(smem) + (2 * ring.place + which) * ge.half_bytes;
      const char* base = kv.base[which] + group * (attn_group(D) * D * 2) + col * 16;
#pragma unroll
      for (int k = 0; k < kMost; ++k) {
        const int end = min(sh.tile - 32 * k, 32);
#pragma unroll 4
        for (int i = 0; i < end; i += at_once) {
          const int row = i + sub;
          const int64_t o = __shfl_sync(0xffffffffu, from[k], row & 31);
          const char* s = base + (o < 0 ? 0 : o);
          const int take = o < 0 ? 0 : 16;
          const int slot = 32 * k + row;
          const uint32_t d = dst + (slot >> 4) * (16 * ge.row_s) + (col >> 3) * 2048 + swizzled(slot & 15, col & 7);
          if (sub < at_once && row < end) {
            if (col < pieces) cp_async16(d, s, take);
#pragma unroll
            for (int c = 1; c < attn_group(D) * D / 8 / 32; ++c)   // 32 parts on: four pieces
              if (col + 32 * c < pieces) cp_async16(d + 8192 * c, s + 512 * c, take);
          }
        }
      }
    }
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" :: "r"(smem_u32(&full[ring.place])) : "memory");
    ring.on(ge.copiers);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");   // the CTA may not end before its copies have landed
}

// ------------------------------------------------------------------ the computing warps
// SUB: 16-slot blocks of a tile that a warp takes; NT: 8-row blocks of queries.
template <int D, int FMT, int NT, int SUB>
__global__ void __launch_bounds__(threads_of(D), 1)
    attention_kernel(AttnState st, AttnDims dm, Geometry ge, int layer, Batch ba, Rows q, Rows out, float* lse,
                     KvDev kv, const __grid_constant__ CacheMaps maps, float scale_log2) {
  constexpr int kWarps = attn_group(D), kThreads = threads_of(D);
  extern __shared__ __align__(1024) char smem_raw[];
  char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + ge.bar_off);
  uint64_t* empty = full + kMaxStages;
  int* gave_up = reinterpret_cast<int*>(empty + kMaxStages);
  int* pre = reinterpret_cast<int*>(smem + ge.pre_off);
  __shared__ unsigned s_warp[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const AttnShape& sh = ge.sh;

  __shared__ Walk s_walk[kWarps + kAttnCopyWarps], s_first;
  if (tid == 0) {   // the fences order this thread's own initialisations before the copy engine's use of them: all are its own
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(&full[s], FMT == EPIKV_CACHE_BF16 && !maps.on ? 32 : 1);
      mbar_init(&empty[s], kWarps);
    }
    *gave_up = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  pdl_wait();
  pdl_trigger();
  // tiles before each entry, and the entry that the CTA's first tile is in
  const int per = (ba.n_seq + 255) >> 8;
  unsigned mine = 0;
  Entry e0{};
  if (tid < 256)
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      const bool there = b < ba.n_seq && batch_entry(ba, dm, b, sh.causal, st.err, &e0);
      const int runs = there ? row_runs(sh, e0.n) : 0;
      int64_t t = runs == 1 ? item_tiles(sh, e0.n, e0.len, 0) : 0;
      for (unsigned many = __ballot_sync(0xffffffffu, runs > 1); many; many &= many - 1) {   // such entries' runs by the warp
        const int k = __ffs(many) - 1;
        const int64_t sum = tiles_before(sh, __shfl_sync(0xffffffffu, e0.n, k), __shfl_sync(0xffffffffu, e0.len, k),
                                         __shfl_sync(0xffffffffu, runs, k), lane);
        if (lane == k) t = sum;
      }
      const unsigned count = count_of(t * sh.groups);
      mine = add_counts(mine, count);
      if (b < ba.n_seq) pre[b + 1] = (int)count;
    }
  unsigned run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned v = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run = add_counts(run, v);
  }
  if (lane == 31 && warp < 8) s_warp[warp] = run;
  unsigned before = __shfl_up_sync(0xffffffffu, run, 1), sum = 0;
  if (lane == 0) before = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k < warp) before = add_counts(before, s_warp[k]);
    sum = add_counts(sum, s_warp[k]);
  }
  if (sum == kTooManyTiles) {   // rare: what stands behind the last entry that can be taken is skipped
    __shared__ unsigned s_sum;
    if (tid == 0) s_sum = 0;
    __syncthreads();
    if (tid < 256) {
      unsigned end = before;
      for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b >= ba.n_seq) break;
        end = add_counts(end, (unsigned)pre[b + 1]);
        if (end < kTooManyTiles) {
          atomicMax(&s_sum, end);
        } else if (pre[b + 1]) {
          pre[b + 1] = 0;
          set_error(st.err, EPIKV_DEV_CAPACITY);
        }
      }
    }
    __syncthreads();
    sum = s_sum;
    before = min(before, sum);
  }
  const int total = (int)sum;
  int at0 = (int)before;
  const int lo = first_tile(blockIdx.x, total), hi = first_tile(blockIdx.x + 1, total);
  if (tid < 256) {
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b >= ba.n_seq) break;
      const int end = at0 + pre[b + 1];
      if (at0 <= lo && lo < end) {
        if (per > 1) batch_entry(ba, dm, b, sh.causal, st.err, &e0);
        s_first = Walk{b, 0, 0, at0 - lo, item_tiles(sh, e0.n, e0.len, 0), e0};
      }
      pre[b + 1] = at0 = end;
    }
    if (tid == 0) pre[0] = 0;
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int b = tid; b <= ba.n_seq; b += kThreads) st.plan[b] = pre[b];
  if (lo == hi) return;
  Walk* w = &s_walk[warp];
  const Walker walker{pre, ba, dm, sh, st.err};
  walker.seek(w, s_first, lane);
  const int tiles = hi - lo;
  const Waiter wait{gave_up, st.err};
  // With 8 + 4 warps of 168 registers the copying ones give most of theirs to the computing ones:
  // 256 x 216 + 128 x 72 = 256 x 200 + 128 x 104 = 384 x 168.
  constexpr bool kSplit = kThreads == 384;
  constexpr int kCopyRegs = FMT == EPIKV_CACHE_BF16 ? 104 : 72, kMoreRegs = FMT == EPIKV_CACHE_BF16 ? 200 : 216;
  static_assert(FMT != EPIKV_CACHE_BF16 || SUB == 1, "the path of infinite values takes one block of slots");
  static_assert(kWarps * kMoreRegs + kAttnCopyWarps * kCopyRegs <= (kWarps + kAttnCopyWarps) * 168 || !kSplit,
                "the computing warps would wait for registers that nobody gives");
  if (warp >= kWarps) {
    if constexpr (kSplit) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kCopyRegs));
    if (warp - kWarps >= ge.copiers) return;
    if (FMT == EPIKV_CACHE_BF16 && maps.on)
      copy_tensor<D>(smem, full, empty, wait, st, dm, ge, kv, maps, layer, walker, w, tiles, warp - kWarps, lane);
    else if constexpr (FMT == EPIKV_CACHE_BF16)
      copy_bf16<D>(smem, full, empty, wait, st, dm, ge, kv, layer, walker, w, tiles, warp - kWarps, lane);
    else
      copy_q4<D>(smem, full, empty, wait, st, dm, ge, kv, layer, walker, w, tiles, warp - kWarps, lane);
    return;
  }

  if constexpr (kSplit) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kMoreRegs));
  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  constexpr int KS = D / 16;                 // blocks of 16 channels
  // probabilities are held times 2^kUp: as halves they reach from 2^-14 (2^-24 with fewer bits) to 2^16, and may pass the
  // maximum that they are taken against by 2^kSlack
  constexpr float kUp = kBf16 ? 0.f : 7.f, kSlack = 8.f;
  const int g = lane >> 2, t = lane & 3;
  int stage = 0;
  uint32_t phase = 0;
  for (int x = 0; x < tiles;) {
    walker.to(w, x, lane);
    const Entry e = w->e;
    const int h0 = w->group * attn_group(D), heads = min(attn_group(D), dm.H - h0);
    const int teams = attn_teams(heads, kWarps);
    const bool idle = warp >= teams * heads;
    const int head = warp % heads, team = idle ? 0 : warp / heads;   // idle warps follow team 0 and keep nothing
    const int kh = h0 + head;
    const int row0 = w->run * sh.rows, nrows = min(sh.rows, rows_of(sh, e.n) - row0);

    // where the lane reads in a tile: keys are rows (slots), values columns of the first operand
    const uint32_t ring0 = smem_u32(smem);
    // where the warp's blocks of slots start, and from there to its block u (what lies behind the tile: the first block
    // again, masked); 8 slots on
    const int block0 = team * 16 < sh.tile ? team * 16 : 0, blocks = sh.tile / (16 * teams);
    const uint32_t hop = teams * 16 * ge.row_s, eight = 8 * ge.row_s;
    auto block_at = [&](int u) { return u == 0 || u < blocks ? u * hop : 0u; };
    const int k0 = kBf16 ? 2 * t : slot_of_row(ge.order, 2 * t), k1 = kBf16 ? 2 * t + 1 : slot_of_row(ge.order, 2 * t + 1);
    uint32_t key_code, key_scale, value_code, value_scale;
    uint32_t key_code8 = 0, key_scale8 = 0, value_odd = 0, value_code8 = 0, value_odd8 = 0, scale_odd = 0, value_scale8 = 0, scale_odd8 = 0;
    if constexpr (kBf16) {
      const uint32_t mine = block0 * ge.row_s + head * (D / 64) * 2048;
      key_code = mine + (lane & 15) * 128;
      key_scale = (lane >> 4) ^ (lane & 7);          // of a row's parts: 2 j + this lane's half, exchanged by the row
      value_code = ge.half_bytes + mine + ((lane & 7) + (lane >> 4) * 8) * 128;
      value_scale = ((lane >> 3) & 1) ^ (lane & 7);
    } else {
      const uint32_t key_row = (block0 + slot_of_row(ge.order, g)) * ge.row_s;
      const uint32_t value_row = (block0 + k0) * ge.row_s, scales = heads * (D / 2) + head * (D / 16);
      key_code = key_row + head * (D / 2) + t * (D / 8);
      key_scale = key_row + scales + t * (D / 64);
      value_code = ge.half_bytes + value_row + head * (D / 2) + g * (D / 16);
      value_scale = ge.half_bytes + value_row + scales + g * (D / 8) / 16;
      const uint32_t odd = (k1 - k0) * ge.row_s;
      key_code8 = key_code + eight;
      key_scale8 = key_scale + eight;
      value_odd = value_code + odd;
      value_code8 = value_code + eight;
      value_odd8 = value_odd + eight;
      scale_odd = value_scale + odd;
      value_scale8 = value_scale + eight;
      scale_odd8 = scale_odd + eight;
    }

    // the queries as the second operand: column n of block nt is row nt * 8 + n
    uint32_t qf[NT][KS][2];
    float cf[NT][2];       // what turns a raw score into log2 units, per column 2t and 2t + 1
    const float gk = kBf16 ? scale_log2 : scale_log2 * head_scale(st, dm, 0, layer, kh);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = row0 + nt * 8 + g;
      const bool there = nt * 8 + g < nrows && !idle;
      const __nv_bfloat16* qp = reinterpret_cast<const __nv_bfloat16*>(q.p) +
                                (there ? (int64_t)(e.tok0 + r / sh.rep) * q.st + (kh * sh.rep + r % sh.rep) * q.sh : 0);
      float mul = 1.f;
      if constexpr (kBf16) {
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          qf[nt][j][0] = there ? *reinterpret_cast<const uint32_t*>(qp + 16 * j + 2 * t) : 0u;
          qf[nt][j][1] = there ? *reinterpret_cast<const uint32_t*>(qp + 16 * j + 8 + 2 * t) : 0u;
        }
      } else {
        // a lane's channels are t * D/4 .. : as halves, scaled by a power of two that brings the row's largest to
        // 2^14 .. 2^15: bf16's 8 bits then stand whole in channels down to 2^-31 of it (of rows below 2^-112, which get
        // 2^126, down to 2^-17 or more).  256 products with keys of up to 2,688 stay below 2^35.
        uint2 raw[KS];
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          raw[j] = there ? *reinterpret_cast<const uint2*>(qp + t * (D / 4) + 4 * j) : make_uint2(0, 0);
          top = fmaxf(top, fmaxf(fmaxf(fabsf(bf16_lo(raw[j].x)), fabsf(bf16_hi(raw[j].x))),
                                 fmaxf(fabsf(bf16_lo(raw[j].y)), fabsf(bf16_hi(raw[j].y)))));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^(141 - ex) of the biased exponent ex and its inverse, both normal numbers (ex = 255: the finite ones' largest)
        const int ex = min(max((int)(__float_as_uint(top) >> 23), 15), 254);
        const float down = __uint_as_float((uint32_t)(268 - ex) << 23);
        mul = __uint_as_float((uint32_t)(ex - 14) << 23);
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          qf[nt][j][0] = half2_of(bf16_lo(raw[j].x) * down, bf16_hi(raw[j].x) * down);
          qf[nt][j][1] = half2_of(bf16_lo(raw[j].y) * down, bf16_hi(raw[j].y) * down);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float f = gk * __shfl_sync(0xffffffffu, mul, (2 * t + c) * 4);
        cf[nt][c] = f < 0x1p-126f ? 0x1p-126f : f > 0x1.fffffep127f ? 0x1.fffffep127f : f;   // 0 x -inf and inf x 0 are NaN
      }
    }
    const int least = e.len + (sh.causal ? row0 / sh.rep + 1 : 0);   // slots that every row of the item sees

    float o[KS][NT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][nt][i] = 0.f;
    }

    // The scores of the tile at `base`.
    auto keys = [&](uint32_t base, float (&s)[SUB][NT][4]) {
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        if constexpr (kBf16) {
          const uint32_t addr = base + block_at(u) + key_code;
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            uint32_t a[4];
            ldmatrix4<false>(a, addr + j / 4 * 2048 + (((2 * j & 6) ^ key_scale) << 4));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if (j == 0) mma_first<FMT>(s[u][nt], a, qf[nt][j][0], qf[nt][j][1]);
              else mma<FMT>(s[u][nt], a, qf[nt][j][0], qf[nt][j][1]);
            }
          }
        } else {
          const uint32_t at = base + block_at(u);
          uint32_t w0[D / 32], w1[D / 32];
          lds_words(w0, at + key_code);
          lds_words(w1, at + key_code8);
          uint32_t s0x[D / 128 + 1], s1x[D / 128 + 1];   // the scales, two a register
          if constexpr (D == 64) {
            s0x[0] = e4m3x2_to_half2((uint16_t)lds_u8(at + key_scale));
            s1x[0] = e4m3x2_to_half2((uint16_t)lds_u8(at + key_scale8));
          } else {
#pragma unroll
            for (int p = 0; p < D / 128; ++p) {
              s0x[p] = e4m3x2_to_half2((uint16_t)lds_u16(at + key_scale + 2 * p));
              s1x[p] = e4m3x2_to_half2((uint16_t)lds_u16(at + key_scale8 + 2 * p));
            }
          }
          float two[NT][4];   // a second chain of sums, half the first one's latencies
#pragma unroll
          for (int v = 0; v < D / 32; ++v) {   // eight channels of a lane: two blocks
            uint32_t x0[4], x1[4];
            e2m1x8_to_half2(w0[v], x0);
            e2m1x8_to_half2(w1[v], x1);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              uint32_t a[4];
              if ((v / 2) % 2 == 0) {
                a[0] = hmul2_by<false>(x0[2 * y], s0x[v / 4]);
                a[1] = hmul2_by<false>(x1[2 * y], s1x[v / 4]);
                a[2] = hmul2_by<false>(x0[2 * y + 1], s0x[v / 4]);
                a[3] = hmul2_by<false>(x1[2 * y + 1], s1x[v / 4]);
              } else {
                a[0] = hmul2_by<true>(x0[2 * y], s0x[v / 4]);
                a[1] = hmul2_by<true>(x1[2 * y], s1x[v / 4]);
                a[2] = hmul2_by<true>(x0[2 * y + 1], s0x[v / 4]);
                a[3] = hmul2_by<true>(x1[2 * y + 1], s1x[v / 4]);
              }
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float (&sum)[4] = y ? two[nt] : s[u][nt];
                if (v == 0) mma_first<FMT>(sum, a, qf[nt][2 * v + y][0], qf[nt][2 * v + y][1]);
                else mma<FMT>(sum, a, qf[nt][2 * v + y][0], qf[nt][2 * v + y][1]);
              }
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[u][nt][i] += two[nt][i];
        }
      }
    };
    // Gives block mt of the operand (channels x slots; the lane's slots are k0, k1 and 8 on) to f, for every mt.
    auto each = [&](uint32_t base, int u, auto&& f) {
      if constexpr (kBf16) {
        const uint32_t addr = base + block_at(u) + value_code;
#pragma unroll
        for (int mt = 0; mt < KS; ++mt) {
          uint32_t a[4];
          ldmatrix4<true>(a, addr + mt / 4 * 2048 + (((2 * mt & 6) ^ value_scale) << 4));
          f(mt, a);
        }
      } else {
        const uint32_t at = base + block_at(u);
        uint32_t wa[D / 64], wb[D / 64], wc[D / 64], wd[D / 64];
        lds_words(wa, at + value_code);
        lds_words(wb, at + value_odd);
        lds_words(wc, at + value_code8);
        lds_words(wd, at + value_odd8);
        uint32_t sl = 0, sh8 = 0;
#pragma unroll
        for (int v = 0; v < D / 64; ++v) {   // eight channels: four blocks
          if (v % 2 == 0) {
            sl = e4m3x2_to_half2((uint16_t)(lds_u8(at + value_scale + v / 2) + (lds_u8(at + scale_odd + v / 2) << 8)));
            sh8 = e4m3x2_to_half2((uint16_t)(lds_u8(at + value_scale8 + v / 2) + (lds_u8(at + scale_odd8 + v / 2) << 8)));
          }
          // pairs of slots instead of pairs of channels: even channels, odd channels
          constexpr uint32_t kLow = 0x0f0f0f0fu;
          uint32_t e0[4], e1[4], e2[4], e3[4];
          e2m1x8_to_half2((wa[v] & kLow) | ((wb[v] << 4) & ~kLow), e0);
          e2m1x8_to_half2(((wa[v] >> 4) & kLow) | (wb[v] & ~kLow), e1);
          e2m1x8_to_half2((wc[v] & kLow) | ((wd[v] << 4) & ~kLow), e2);
          e2m1x8_to_half2(((wc[v] >> 4) & kLow) | (wd[v] & ~kLow), e3);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            uint32_t a[4] = {hmul2(e0[y], sl), hmul2(e1[y], sl), hmul2(e2[y], sh8), hmul2(e3[y], sh8)};
            f(4 * v + y, a);
          }
        }
      }
    };
    // Adds the tile's values, weighted, to the outputs.
    auto values = [&](uint32_t base, const uint32_t (&pb)[SUB][NT][kBf16 ? 4 : 2]) {
#pragma unroll
      for (int u = 0; u < SUB; ++u)
        each(base, u, [&](int mt, uint32_t (&a)[4]) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma<FMT>(o[mt][nt], a, pb[u][nt][0], pb[u][nt][1]);
            if constexpr (kBf16) mma<FMT>(o[mt][nt], a, pb[u][nt][2], pb[u][nt][3]);
          }
        });
    };

    const int end = min(w->at + w->tiles, tiles);
    int s0 = (x - w->at) * sh.tile;
    float s[SUB][NT][4];
    bool scored = false;
    for (; x < end; ++x, s0 += sh.tile) {
      const uint32_t base = __shfl_sync(0xffffffffu, ring0 + stage * (2 * ge.half_bytes), 0);   // known to be the same in all lanes
      if (!scored) {
        wait(&full[stage], phase);
        keys(base, s);
      }
      // ---- probabilities.  They are taken against a maximum that is moved only when a score passes it by 2^kSlack: the
      // sums and outputs then need no rescaling, and the warp no exchange, in nearly every tile.
      if (s0 + sh.tile > least || idle || SUB * teams * 16 > sh.tile) {
        const int first_row = w->run * sh.rows, last_row = min(first_row + sh.rows, rows_of(sh, w->e.n));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          int lim[2];   // slots that the columns' rows see
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int r = first_row + nt * 8 + 2 * t + c;
            lim[c] = r < last_row ? w->e.len + (sh.causal ? r / sh.rep + 1 : 0) : 0;
          }
#pragma unroll
          for (int u = 0; u < SUB; ++u) {
            const int sub = u * teams + team;
            const int at = s0 + sub * 16 + (kBf16 ? g : slot_of_row(ge.order, g));
            const bool in = !idle && sub * 16 < sh.tile;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!in || at + (i >> 1) * 8 >= lim[i & 1]) s[u][nt][i] = -INFINITY;
          }
        }
      }
      float top[NT][2];
      bool past = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[nt][c] = -INFINITY;
#pragma unroll
          for (int u = 0; u < SUB; ++u) top[nt][c] = fmaxf(top[nt][c], fmaxf(s[u][nt][c], s[u][nt][2 + c]));
          past |= top[nt][c] * cf[nt][c] > m[nt][c] + kSlack;
        }
      if (__any_sync(0xffffffffu, past)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float alpha[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float v = top[nt][c];
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
            const float mn = fmaxf(m[nt][c], v * cf[nt][c]);
            alpha[c] = mn == -INFINITY ? 1.f : weight_of(m[nt][c] - mn);
            m[nt][c] = mn;
            l[nt][c] *= alpha[c];
          }
#pragma unroll
          for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j][nt][i] *= alpha[i & 1];
        }
      }
      uint32_t odd[4] = {0u, 0u, 0u, 0u};   // bf16: whether a value is infinite or NaN
      if constexpr (kBf16) {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
          each(base, u, [&](int, uint32_t (&a)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) note_unbounded(odd[i], a[i]);
          });
      }
      uint32_t pb[SUB][NT][kBf16 ? 4 : 2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float add[2];   // a row without a score so far: against 0
#pragma unroll
        for (int c = 0; c < 2; ++c) add[c] = kUp - (m[nt][c] == -INFINITY ? 0.f : m[nt][c]);
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[u][nt][i] = ex2(fmaf(s[u][nt][i], cf[nt][i & 1], add[i & 1]));
            l[nt][i & 1] += s[u][nt][i];
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            if constexpr (kBf16) {
              const uint32_t hi2 = bf162_of(s[u][nt][2 * y], s[u][nt][2 * y + 1]);
              pb[u][nt][y] = transpose8x8(hi2);
              pb[u][nt][2 + y] = transpose8x8(bf162_of(s[u][nt][2 * y] - bf16_lo(hi2), s[u][nt][2 * y + 1] - bf16_hi(hi2)));
            } else {
              pb[u][nt][y] = transpose8x8(half2_of(s[u][nt][2 * y], s[u][nt][2 * y + 1]));
            }
          }
        }
      }

      // ---- their sum of values, and the next tile's scores: two chains that do not wait for each other
      // An infinity or a NaN among the values goes by a path of its own.  In a slot that some rows do not see, a
      // probability of 0 does not silence it.  In one that they see it has to be weighted by one number above 0, and
      // bf16's two terms of a probability may be of unlike signs or 0.  (4-bit values are finite or NaN, and NaN in a seen
      // slot stays NaN: only tiles with unseen slots are looked through.)
      bool apart = false;
      if constexpr (kBf16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) apart |= (odd[i] & 0x7fff7fffu) != 0;   // else 0 or -0
        apart = __any_sync(0xffffffffu, apart);
      } else if (s0 + sh.tile > least) {
#pragma unroll 1
        for (int u = 0; u < SUB; ++u)
          each(base, u, [&](int, uint32_t (&a)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) apart |= (a[i] & 0x7c00u) == 0x7c00u || (a[i] >> 16 & 0x7c00u) == 0x7c00u;
          });
        apart = __any_sync(0xffffffffu, apart);
      }
      int next = stage + 1;
      uint32_t next_phase = phase;
      if (next == ge.stages) {
        next = 0;
        next_phase ^= 1;
      }
      scored = !apart && x + 1 < end;
      if (scored) {
        wait(&full[next], next_phase);
        keys(__shfl_sync(0xffffffffu, ring0 + next * (2 * ge.half_bytes), 0), s);
        values(base, pb);
      } else if (!apart) {
        values(base, pb);
      } else {
        const int first_row = w->run * sh.rows, last_row = min(first_row + sh.rows, rows_of(sh, w->e.n)) - 1;
        // the weights of infinities: 1, or 0 where the score is minus infinity
        uint32_t whole[kBf16 ? SUB : 1][NT][2];
        if constexpr (kBf16) {
          float raw[SUB][NT][4];
          keys(base, raw);
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = first_row + nt * 8 + 2 * t + (i & 1);
                const bool sees = s0 + (u * teams + team) * 16 + g + (i >> 1) * 8 < w->e.len + (sh.causal ? r / sh.rep + 1 : 0);
                raw[u][nt][i] = !sees || raw[u][nt][i] == -INFINITY ? 0.f : raw[u][nt][i] != raw[u][nt][i] ? raw[u][nt][i] : 1.f;
              }
#pragma unroll
              for (int y = 0; y < 2; ++y) whole[u][nt][y] = transpose8x8(bf162_of(raw[u][nt][2 * y], raw[u][nt][2 * y + 1]));
            }
        }
#pragma unroll 1   // rare: its instructions should not stand between the others
        for (int u = 0; u < SUB; ++u) {
          uint32_t pu[NT][kBf16 ? 4 : 2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int y = 0; y < (kBf16 ? 4 : 2); ++y) {
              pu[nt][y] = pb[0][nt][y];
#pragma unroll
              for (int v = 1; v < SUB; ++v)
                if (u == v) pu[nt][y] = pb[v][nt][y];
            }
          // the rows of each token by themselves, the values that they do not see taken as 0; a block behind the tile: all
          for (int i = first_row / sh.rep; i <= last_row / sh.rep; ++i) {
            // of these slots, those that token i sees
            const int at = (u * teams + team) * 16;
            const int n = !kBf16 || at < sh.tile ? w->e.len + (sh.causal ? i + 1 : 0) - (s0 + at) : 0;
            uint32_t mine = 0;   // bit 2 nt + c: column c of block nt is token i's
#pragma unroll 1
            for (int k = 0; k < 2 * NT; ++k) mine |= ((first_row + k / 2 * 8 + 2 * t + (k & 1)) / sh.rep == i ? 1u : 0u) << k;
            const uint32_t m0 = (k0 < n ? 0xffffu : 0u) | (k1 < n ? 0xffff0000u : 0u);
            const uint32_t m8 = (k0 + 8 < n ? 0xffffu : 0u) | (k1 + 8 < n ? 0xffff0000u : 0u);
            each(base, u, [&](int mt, uint32_t (&a)[4]) {
              uint32_t z[4] = {a[0] & m0, a[1] & m0, a[2] & m8, a[3] & m8}, inf[4];
              if constexpr (kBf16) {
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                  const uint32_t odd = ((z[y] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((z[y] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                  inf[y] = z[y] & odd;
                  z[y] &= ~odd;
                }
              }
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                // only the columns of token i; the others keep their sums
                float keep[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) keep[y] = o[mt][nt][y];
                mma<FMT>(o[mt][nt], z, pu[nt][0], pu[nt][1]);
                if constexpr (kBf16) {
                  mma<FMT>(o[mt][nt], z, pu[nt][2], pu[nt][3]);
                  mma<FMT>(o[mt][nt], inf, whole[0][nt][0], whole[0][nt][1]);
                }
#pragma unroll
                for (int y = 0; y < 4; ++y)
                  if (!(mine >> (2 * nt + (y & 1)) & 1)) o[mt][nt][y] = keep[y];
              }
            });
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[stage]);
      stage = next;
      phase = next_phase;
    }

    // ---- the end of the CTA's part of the item
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 4);
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 8);
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 16);
      }
    // the warps of a head, in halves
    for (int step = teams / 2; step > 0; step >>= 1) {
      float* box = reinterpret_cast<float*>(smem + ge.join_off);
      constexpr int kBox = attn_box_floats(D, NT);
      asm volatile("bar.sync 1, %0;" :: "n"(32 * kWarps) : "memory");
      if (!idle && team >= step && team < 2 * step) {
        float* mineb = box + ((team - step) * heads + head) * kBox + lane;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) mineb[((j * NT + nt) * 4 + i) * 32] = o[j][nt][i];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            mineb[(KS * NT * 4 + nt * 4 + c) * 32] = m[nt][c];
            mineb[(KS * NT * 4 + nt * 4 + 2 + c) * 32] = l[nt][c];
          }
        }
      }
      asm volatile("bar.sync 1, %0;" :: "n"(32 * kWarps) : "memory");
      if (!idle && team < step) {
        const float* from = box + (team * heads + head) * kBox + lane;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float a[2], b[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float m2 = from[(KS * NT * 4 + nt * 4 + c) * 32], l2 = from[(KS * NT * 4 + nt * 4 + 2 + c) * 32];
            const float mn = fmaxf(m[nt][c], m2), base = mn == -INFINITY ? 0.f : mn;
            a[c] = weight_of(m[nt][c] - base);
            b[c] = weight_of(m2 - base);
            l[nt][c] = l[nt][c] * a[c] + l2 * b[c];
            m[nt][c] = mn;
          }
#pragma unroll
          for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              o[j][nt][i] = o[j][nt][i] * a[i & 1] + from[((j * NT + nt) * 4 + i) * 32] * b[i & 1];
        }
      }
    }
    if (!idle && team == 0) {
      const bool inside = w->at < 0;   // the item began in an earlier CTA
      const bool whole = !inside && x == w->at + w->tiles;
      const Entry e = w->e;
      const int row0 = w->run * sh.rows, nrows = min(sh.rows, rows_of(sh, e.n) - row0);
      const int kh = w->group * attn_group(D) + head;
      const float gv = kBf16 ? 1.f : head_scale(st, dm, 1, layer, kh);
      float* part = st.part + (int64_t)(blockIdx.x * 2 + (inside ? 0 : 1)) * ge.slot_floats;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int row = nt * 8 + 2 * t + c;
          if (row >= nrows) continue;
          const float mul = !whole ? gv : l[nt][c] == 0.f ? 0.f : gv / l[nt][c];
          const int r = row0 + row;
          const int64_t token = e.tok0 + r / sh.rep;
          const int hq = kh * sh.rep + r % sh.rep;
          float* po = part + (int64_t)(head * sh.rows + row) * D;
          __nv_bfloat16* yo = reinterpret_cast<__nv_bfloat16*>(out.p) + token * out.st + hq * out.sh;
          if constexpr (kBf16) {
#pragma unroll
            for (int j = 0; j < KS; ++j)
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int ch = 16 * j + 8 * y + g;
                const float v = l[nt][c] == 0.f && whole ? 0.f : o[j][nt][2 * y + c] * mul;
                if (whole) yo[ch] = __float2bfloat16_rn(v);
                else po[ch] = v;
              }
          } else {
#pragma unroll
            for (int j = 0; j < KS; j += 2) {   // four neighbouring channels
              const float v0 = o[j][nt][c] * mul, v1 = o[j][nt][2 + c] * mul;
              const float v2 = o[j + 1][nt][c] * mul, v3 = o[j + 1][nt][2 + c] * mul;
              const int ch = g * (D / 8) + 2 * j;
              if (whole) *reinterpret_cast<uint2*>(yo + ch) = make_uint2(bf162_of(v0, v1), bf162_of(v2, v3));
              else *reinterpret_cast<float4*>(po + ch) = make_float4(v0, v1, v2, v3);
            }
          }
          if (g == 0) {
            if (!whole) {
              *reinterpret_cast<float2*>(part + attn_group(D) * sh.rows * D + (head * sh.rows + row) * 2) =
                  make_float2(m[nt][c] - kUp, l[nt][c]);
            } else if (lse) {
              lse[token * dm.Hq + hq] = l[nt][c] == 0.f ? -INFINITY : (m[nt][c] - kUp + log2f(l[nt][c])) * 0.69314718055994531f;
            }
          }
        }
    }
  }
}

// ------------------------------------------------------------------ joining the parts of an item
// One block kRows rows of an item's KV head.  The parts' weights 2^(m_i - max) come first, all parts at
// once; then each thread adds up four channels of a row over a share of the parts, and the shares are added in order.
// What bounds it is a chain of dependent reads (the plan, the maxima, the outputs), so each step reads all that it can.
template <int kRows, int kThreads>
__global__ void __launch_bounds__(kThreads) attention_join_kernel(AttnState st, AttnDims dm, Geometry ge, Batch ba,
                                                                  Rows out, float* lse, int lanes_log) {
  constexpr int rb = kRows;
  __shared__ float2 s_ml[kAttnCtas][rb];          // maximum and sum, then the weight in place of the maximum
  __shared__ int s_slot[kAttnCtas];
  __shared__ float2 s_row[rb];                    // maximum and sum of all parts
  __shared__ float4 s_acc[kThreads];
  const AttnShape& sh = ge.sh;
  const int b = blockIdx.y, kh = blockIdx.x % dm.H, r0 = blockIdx.x / dm.H * rb, run = r0 >> sh.rows_log;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  const int p0 = st.plan[b], p1 = st.plan[b + 1], total = st.plan[ba.n_seq];
  Entry e;
  e.tok0 = ba.cu_new[b];
  e.n = ba.cu_new[b + 1] - e.tok0;
  e.len = ba.len[(int64_t)b * ba.len_stride];
  const int there = min(rb, rows_of(sh, e.n) - r0);
  if (p0 == p1 || there <= 0) return;   // no tiles: an entry without new tokens, or one that was refused
  const int group = kh / attn_group(dm.d), head = kh % attn_group(dm.d);
  int at = p0;
  if (sh.groups > 1) at += group * ((p1 - p0) / sh.groups);
  if (run) at += (int)tiles_before(sh, e.n, e.len, run, lane);
  const int tiles = item_tiles(sh, e.n, e.len, run);
  const int c0 = cta_of_tile(at, total), c1 = cta_of_tile(at + tiles - 1, total);
  if (c0 == c1) return;
  // below one tile a CTA some CTAs have none: then every tile is a part
  const int parts = total < kAttnCtas ? tiles : c1 - c0 + 1;
  const int64_t ml0 = attn_group(dm.d) * sh.rows * dm.d + (head * sh.rows + (r0 & (sh.rows - 1))) * 2;
  for (int i = tid; i < parts * rb; i += kThreads) {
    const int part = i / rb, row = i - part * rb;
    const int c = total < kAttnCtas ? cta_of_tile(at + part, total) : c0 + part;
    const int slot = c * 2 + (c == c0 ? 1 : 0);
    if (row == 0) s_slot[part] = slot;
    if (row < there) s_ml[part][row] = *reinterpret_cast<const float2*>(st.part + (int64_t)slot * ge.slot_floats + ml0 + 2 * row);
  }
  __syncthreads();
  if (warp < there) {
    float top = -INFINITY, sum = 0.f;
    for (int i = lane; i < parts; i += 32) top = fmaxf(top, s_ml[i][warp].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float base = top == -INFINITY ? 0.f : top;
    for (int i = lane; i < parts; i += 32) {
      const float2 ml = s_ml[i][warp];
      const float weight = weight_of(ml.x - base);
      s_ml[i][warp].x = weight;
      sum += ml.y * weight;
    }
    sum = warp_sum(sum);
    if (lane == 0) s_row[warp] = make_float2(base, sum);
  }
  __syncthreads();
  const int wide = rb << lanes_log, shares = kThreads / wide;   // float4 columns of the block's rows; threads for each
  const int share = tid / wide, col = tid & (wide - 1), row = col >> lanes_log, ch = (col & ((1 << lanes_log) - 1)) * 4;
  const bool on = share < shares && row < there;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (on) {
    const float* from = st.part + (int64_t)(head * sh.rows + (r0 & (sh.rows - 1)) + row) * dm.d + ch;
#pragma unroll 1
    for (int i0 = share; i0 < parts; i0 += 8 * shares) {
      float4 v[8];
      float z[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * shares;
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        z[k] = 0.f;
        if (i < parts) {
          v[k] = *reinterpret_cast<const float4*>(from + (int64_t)s_slot[i] * ge.slot_floats);
          z[k] = s_ml[i][row].x;
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        acc.x += v[k].x * z[k];
        acc.y += v[k].y * z[k];
        acc.z += v[k].z * z[k];
        acc.w += v[k].w * z[k];
      }
    }
  }
  s_acc[tid] = acc;
  __syncthreads();
  if (!on || share) return;
  for (int k = 1; k < shares; ++k) {
    const float4 v = s_acc[tid + k * wide];
    acc.x += v.x;
    acc.y += v.y;
    acc.z += v.z;
    acc.w += v.w;
  }
  const int r = r0 + row;
  const int64_t token = e.tok0 + r / sh.rep;
  const int hq = kh * sh.rep + r % sh.rep;
  const float2 all = s_row[row];
  const float mul = all.y == 0.f ? 0.f : 1.f / all.y;
  *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(out.p) + token * out.st + hq * out.sh + ch) =
      make_uint2(bf162_of(acc.x * mul, acc.y * mul), bf162_of(acc.z * mul, acc.w * mul));
  if (lse && ch == 0) lse[token * dm.Hq + hq] = all.y == 0.f ? -INFINITY : (all.x + log2f(all.y)) * 0.69314718055994531f;
}

// ------------------------------------------------------------------ host
Geometry geometry(const AttnDims& dm, int n_seq, int max_new, bool causal) {
  return attn_geometry(dm.H, dm.rep, dm.d, dm.fmt == EPIKV_CACHE_E2M1, dm.units, dm.T, n_seq, max_new, causal);
}

// The layer's K and V as tensors, where their layout allows it.
CacheMaps cache_maps(const AttnDims& dm, const Geometry& ge, int layer, const KvDev& kv) {
  CacheMaps maps = {};
  if (dm.fmt != EPIKV_CACHE_BF16) return maps;
  const bool flat = kv.layout == EPIKV_LAYOUT_CONTIGUOUS;
  if (!flat && kv.block_size % 16) return maps;
  const int64_t outer = flat ? kv.stride_seq : kv.stride_block;   // elements
  // Fewer slots before the next sequence than the configuration allows: a tensor that ends there would lack the slots of
  // a single sequence (whose stride says nothing) or of sequences that overlap, one that does not may end behind the
  // memory.  Copied by lanes, every slot is its row and nothing else is read.
  if (flat && kv.stride_seq >= kv.stride_token && kv.stride_seq / kv.stride_token < dm.T) return maps;
  const cuuint64_t dims[4] = {64, (cuuint64_t)(flat ? dm.T : kv.block_size), (cuuint64_t)(flat ? dm.S : kv.num_blocks), (cuuint64_t)(dm.H * dm.d / 64)};
  const cuuint64_t strides[3] = {(cuuint64_t)kv.stride_token * 2, (cuuint64_t)outer * 2, 128};
  for (int i = 0; i < 2; ++i)
    if (strides[i] == 0 || strides[i] >= (cuuint64_t(1) << 40)) return maps;
  const cuuint32_t box[4] = {64, 16, 1, (cuuint32_t)(ge.row_s / 128)}, ones[4] = {1, 1, 1, 1};
  const EncodeTiled encode = encode_tiled();
  if (!encode) return maps;
  for (int w = 0; w < 2; ++w)
    if (encode(&maps.kv[w], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, kv.base[w] + (int64_t)layer * kv.stride_layer * 2, dims,
               strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return maps;
  maps.on = 1;
  return maps;
}

template <int D, int FMT, int NT, int SUB>
cudaError_t run(const AttnState& st, const AttnDims& dm, const Geometry& ge, int layer, const Batch& ba, const Rows& q,
                const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  return pdl_launch(attention_kernel<D, FMT, NT, SUB>, kAttnCtas, threads_of(D), ge.smem_bytes + 1024,
                    stream, st, dm, ge, layer, ba, q, out, lse, kv, cache_maps(dm, ge, layer, kv),
                    dm.scale * 1.4426950408889634f);
}

template <int D, int FMT>
cudaError_t run_rows(const AttnState& st, const AttnDims& dm, const Geometry& ge, int layer, const Batch& ba,
                     const Rows& q, const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  constexpr int kSub = FMT == EPIKV_CACHE_BF16 ? 1 : 2;
  if constexpr (D <= 64)
    if (ge.sh.rows == 32) return run<D, FMT, 4, kSub>(st, dm, ge, layer, ba, q, out, lse, kv, stream);
  if constexpr (D <= 128) {
    if (ge.sh.rows == 16) return run<D, FMT, 2, kSub>(st, dm, ge, layer, ba, q, out, lse, kv, stream);
    if constexpr (kSub == 2)
      if (ge.sub == 4) return run<D, FMT, 1, 4>(st, dm, ge, layer, ba, q, out, lse, kv, stream);
  }
  return run<D, FMT, 1, kSub>(st, dm, ge, layer, ba, q, out, lse, kv, stream);
}

// *runs becomes false where the compiler gave the kernel other registers than its warps' exchange of them counts on:
// launched, it would wait for registers that nobody gives.
template <int D, int FMT, int NT, int SUB>
cudaError_t prepare_one(bool* runs) {
  auto kernel = attention_kernel<D, FMT, NT, SUB>;
  cudaFuncAttributes at;
  cudaError_t e = cudaFuncGetAttributes(&at, kernel);
  if (e != cudaSuccess) return e;
  if (threads_of(D) == 384 && at.numRegs != 168) *runs = false;
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmem + 1024);
}

template <int D, int FMT>
cudaError_t prepare_rows(bool* runs) {
  constexpr int kSub = FMT == EPIKV_CACHE_BF16 ? 1 : 2;
  cudaError_t e = prepare_one<D, FMT, 1, kSub>(runs);
  if constexpr (D <= 128) {
    if (e == cudaSuccess) e = prepare_one<D, FMT, 2, kSub>(runs);
    if constexpr (kSub == 2)
      if (e == cudaSuccess) e = prepare_one<D, FMT, 1, 4>(runs);
  }
  if constexpr (D <= 64)
    if (e == cudaSuccess) e = prepare_one<D, FMT, 4, kSub>(runs);
  return e;
}

}  // namespace

size_t attention_part_floats(const AttnDims& dm) {
  const Geometry ge = geometry(dm, 1, dm.max_new, true);
  return (size_t)2 * kAttnCtas * ge.slot_floats;
}

cudaError_t attention_prepare(const AttnDims& dm, bool* runs) {
  const bool q4 = dm.fmt == EPIKV_CACHE_E2M1;
  *runs = true;
  if (dm.d == 64) return q4 ? prepare_rows<64, EPIKV_CACHE_E2M1>(runs) : prepare_rows<64, EPIKV_CACHE_BF16>(runs);
  if (dm.d == 128) return q4 ? prepare_rows<128, EPIKV_CACHE_E2M1>(runs) : prepare_rows<128, EPIKV_CACHE_BF16>(runs);
  return q4 ? prepare_rows<256, EPIKV_CACHE_E2M1>(runs) : prepare_rows<256, EPIKV_CACHE_BF16>(runs);
}

cudaError_t launch_attention(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal,
                             const Rows& q, const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  const Geometry ge = geometry(dm, ba.n_seq, ba.max_new, causal);
  const bool q4 = dm.fmt == EPIKV_CACHE_E2M1;
  auto go = dm.d == 64    ? (q4 ? run_rows<64, EPIKV_CACHE_E2M1> : run_rows<64, EPIKV_CACHE_BF16>)
            : dm.d == 128 ? (q4 ? run_rows<128, EPIKV_CACHE_E2M1> : run_rows<128, EPIKV_CACHE_BF16>)
                          : (q4 ? run_rows<256, EPIKV_CACHE_E2M1> : run_rows<256, EPIKV_CACHE_BF16>);
  const cudaError_t err = go(st, dm, ge, layer, ba, q, out, lse, kv, stream);
  if (err != cudaSuccess) return err;
  // A joining block of 512 threads takes one row where that gives at most two blocks an SM, and parts may be many (one
  // sequence of 65,536 slots: 256 threads 36.2, 512 34.0 us in all); four rows, or the eight of several tokens, and 256
  // threads where blocks are plenty (64 sequences: one row 213, four 204 us; chunks of 13 to 47 tokens: 61 / 50).
  const int64_t rows = (int64_t)ba.max_new * dm.rep;
  const int lanes_log = dm.d == 64 ? 4 : dm.d == 128 ? 5 : 6;
  auto join = [&](auto kernel, int n, int threads) {
    return pdl_launch(kernel, dim3((unsigned)((rows + n - 1) / n * dm.H), ba.n_seq), threads, 0, stream, st, dm, ge, ba, out,
                      lse, lanes_log);
  };
  if (rows * dm.H * ba.n_seq <= 2 * kAttnCtas) return join(attention_join_kernel<1, 512>, 1, 512);
  return rows >= 8 ? join(attention_join_kernel<8, 512>, 8, 512) : join(attention_join_kernel<4, 256>, 4, 256);
}

}  // namespace epikv
