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
//    bulk copies from one warp, through a ring of tiles (K and V in turn)
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
//    memory on them.  The rotation of P from one product's result layout to the other's
//    operand layout is one transposing move per 8 x 8.
//
// A 4-bit cache stays in 4 bits until the registers: the layout is such that a
// lane's channels are neighbours (any order of channels serves a dot product
// if the queries follow it), a conversion turns two codes into a half pair,
// and the product with the E4M3 scale is exact in half precision (2 + 4
// significant bits).  Queries enter as halves scaled by a power of two per
// row, probabilities as halves times 2^15 (11 bits from 1 down to 2^-29).  For
// a bf16 cache the probabilities go in as two bf16 terms (16 bits).
#include "attn.cuh"
#include "attn_plan.h"

namespace epikv {
namespace {

constexpr int kThreads = 32 * (kAttnWarps + 1);
constexpr uint64_t kWaitNs = 2000000000ull;
using Geometry = AttnGeometry;

// The rows of a 16-slot block in the order that the tensor instruction's rows
// take them: with rows 32 bytes past a multiple of 128 apart, each load of a
// quarter or half warp then touches every bank once.
__device__ __forceinline__ int slot_of_row(int r) { return (0x57463120 >> (4 * r)) & 7; }   // 0 2 1 3 6 4 7 5

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

template <int kWords>
__device__ __forceinline__ void lds_words(uint32_t (&w)[kWords], const char* p) {
  if constexpr (kWords == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (kWords == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
    }
  }
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
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

// The walk along a CTA's items, the same in every thread.
struct Walk {
  const int64_t* pre;
  const Batch* ba;
  const AttnDims* dm;
  const AttnShape* sh;
  int32_t* err;
  int b, group, run, tiles;
  int64_t at;   // the item's first tile
  Entry e;

  __device__ __forceinline__ void entry() {
    group = run = 0;
    batch_entry(*ba, *dm, b, sh->causal, err, &e);
    tiles = item_tiles(*sh, e.n, e.len, 0);
  }
  __device__ __forceinline__ void step() {
    at += tiles;
    if (++run == row_runs(*sh, e.n)) {
      run = 0;
      if (++group == sh->groups) {
        do ++b;
        while (b < ba->n_seq && pre[b + 1] == pre[b]);
        if (b < ba->n_seq) entry();
        return;
      }
    }
    tiles = item_tiles(*sh, e.n, e.len, run);
  }
  // The item that tile x is in (x below the batch's tiles).
  __device__ __forceinline__ void seek(int64_t x) {
    int lo = 0, hi = ba->n_seq - 1;   // the last entry that starts at or before x and has tiles
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (pre[mid + 1] > x) hi = mid;
      else lo = mid + 1;
    }
    b = lo;
    at = pre[b];
    entry();
    while (at + tiles <= x) step();
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

// ------------------------------------------------------------------ the copying warp
template <int D, int FMT>
__device__ void copy_tiles(char* smem, uint64_t* full, uint64_t* empty, const Waiter& wait, const AttnState& st,
                           const AttnDims& dm, const Geometry& ge, const KvDev& kv, int layer, Walk w, int64_t lo,
                           int64_t hi, int lane) {
  const AttnShape& sh = ge.sh;
  int unit = 0;
  uint32_t phase = 0;
  int issued = 0;
  for (int64_t x = lo; x < hi;) {
    const int64_t end = w.at + w.tiles < hi ? w.at + w.tiles : hi;
    const int seen = slots_seen(sh, w.e.n, w.e.len, w.run);
    const int h0 = w.group * kAttnGroup, heads = min(kAttnGroup, dm.H - h0);
    // a row's part: one or two runs of bytes
    int a_off, a_bytes, b_off = 0, b_bytes = 0;
    if (FMT == EPIKV_CACHE_BF16) {
      a_off = h0 * D * 2;
      a_bytes = heads * D * 2;
    } else if (sh.groups == 1) {
      a_off = 0;
      a_bytes = (dm.H * (D / 2 + D / kQuantGroup) + 15) & ~15;
    } else {
      a_off = h0 * (D / 2);
      a_bytes = heads * (D / 2);
      b_off = scale_offset(dm, h0);
      b_bytes = (heads * (D / kQuantGroup) + 15) & ~15;
    }
    for (; x < end; ++x) {
      const int s0 = (int)(x - w.at) * sh.tile;
      int64_t off[kRowsPerLane];
      int rows = 0;
      bool hole = false;
#pragma unroll
      for (int k = 0; k < kRowsPerLane; ++k) {
        const int r = lane + 32 * k;
        off[k] = -1;
        if (r < sh.tile && s0 + r < seen) {
          off[k] = kv_row_offset(kv, layer, w.e.seq, s0 + r, dm.T);
          if (off[k] < 0) set_error(st.err, EPIKV_DEV_SLOT);
        }
        hole |= r < sh.tile && off[k] < 0;
        rows += __popc(__ballot_sync(0xffffffffu, off[k] >= 0));
      }
      hole = __any_sync(0xffffffffu, hole);
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        if (issued >= ge.units) wait(&empty[unit], phase ^ 1);
        char* dst = smem + unit * ge.unit_bytes;
        if (hole) {  // rows that nothing fills: a probability of 0 must not meet what stood there before
#pragma unroll
          for (int k = 0; k < kRowsPerLane; ++k) {
            const int r = lane + 32 * k;
            if (r < sh.tile && off[k] < 0)
              for (int i = 0; i < ge.row_s; i += 16) *reinterpret_cast<uint4*>(dst + r * ge.row_s + i) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(&full[unit], rows * (a_bytes + b_bytes));
        __syncwarp();
        const char* base = kv.base[which];
#pragma unroll
        for (int k = 0; k < kRowsPerLane; ++k) {
          if (off[k] >= 0) {
            char* d = dst + (lane + 32 * k) * ge.row_s;
            const char* s = base + off[k] * 2;
            tma_load_1d(d, s + a_off, a_bytes, &full[unit]);
            if (b_bytes) tma_load_1d(d + a_bytes, s + b_off, b_bytes, &full[unit]);
          }
        }
        ++issued;
        if (++unit == ge.units) {
          unit = 0;
          phase ^= 1;
        }
      }
    }
    w.step();
  }
  if (*wait.gave_up) {  // the CTA may not end before its copies have landed
    for (int u = 0; u < ge.units && u < issued; ++u) {
      const uint32_t parity = u < unit ? phase : phase ^ 1;
      mbar_wait_bounded(&full[u], parity, kWaitNs);
    }
  }
}

// ------------------------------------------------------------------ the computing warps
// SUB: 16-slot blocks of a tile that a warp takes; NT: 8-row blocks of queries.
template <int D, int FMT, int NT, int SUB>
__global__ void __launch_bounds__(kThreads, 1)
    attention_kernel(AttnState st, AttnDims dm, Geometry ge, int layer, Batch ba, Rows q, Rows out, float* lse,
                     KvDev kv, float scale_log2) {
  extern __shared__ __align__(128) char smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + ge.bar_off);
  uint64_t* empty = full + kMaxUnits;
  int* gave_up = reinterpret_cast<int*>(empty + kMaxUnits);
  int64_t* pre = reinterpret_cast<int64_t*>(smem + ge.pre_off);
  __shared__ int64_t s_warp[kAttnWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const AttnShape& sh = ge.sh;

  // tiles before each entry
  if (tid < 2 * kMaxUnits) mbar_init(&full[tid], tid < kMaxUnits ? 1 : kAttnWarps);
  if (tid == 0) *gave_up = 0;
  const int per = (ba.n_seq + 255) / 256;
  int64_t mine = 0;
  if (tid < 256)
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      Entry e;
      if (b < ba.n_seq && batch_entry(ba, dm, b, sh.causal, st.err, &e)) {
        const int64_t t = entry_tiles(sh, e.n, e.len);
        mine += t;
        pre[b + 1] = t;
      } else if (b < ba.n_seq) {
        pre[b + 1] = 0;
      }
    }
  int64_t run = mine;
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += v;
  }
  if (lane == 31 && warp < kAttnWarps) s_warp[warp] = run;
  if (tid == 0) fence_barrier_init();
  __syncthreads();
  if (tid < 256) {
    int64_t at = run - mine;
    for (int k = 0; k < warp; ++k) at += s_warp[k];
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b < ba.n_seq) at = pre[b + 1] += at;
    }
    if (tid == 0) pre[0] = 0;
  }
  __syncthreads();
  pdl_trigger();
  if (blockIdx.x == 0)
    for (int b = tid; b <= ba.n_seq; b += kThreads) st.plan[b] = pre[b];
  const int64_t total = pre[ba.n_seq];
  const int64_t lo = first_tile(blockIdx.x, total), hi = first_tile(blockIdx.x + 1, total);
  if (lo == hi) return;
  Walk w{pre, &ba, &dm, &sh, st.err};
  w.seek(lo);
  const Waiter wait{gave_up, st.err};
  if (warp == kAttnWarps) {
    copy_tiles<D, FMT>(smem, full, empty, wait, st, dm, ge, kv, layer, w, lo, hi, lane);
    return;
  }

  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  constexpr int KS = D / 16;                 // blocks of 16 channels
  constexpr float kUp = kBf16 ? 0.f : 15.f;  // probabilities are held times 2^kUp
  const int g = lane >> 2, t = lane & 3;
  int unit = 0;
  uint32_t phase = 0;
  for (int64_t x = lo; x < hi;) {
    const int64_t end = w.at + w.tiles < hi ? w.at + w.tiles : hi;
    const Entry e = w.e;
    const int h0 = w.group * kAttnGroup, heads = min(kAttnGroup, dm.H - h0);
    const int teams = kAttnWarps / heads;    // warps of a head: 8, 4, 2 or 1
    const bool idle = warp >= teams * heads;
    const int head = warp % heads, team = warp / heads;
    const int kh = h0 + head;
    const int row0 = w.run * sh.rows, nrows = min(sh.rows, rows_of(sh, e.n) - row0);

    // the queries as the second operand: column n of block nt is row nt * 8 + n
    uint32_t qf[NT][KS][2];
    float cf[NT][2];       // what turns a raw score into log2 units, per column 2t and 2t + 1
    int lim[NT][2];        // slots that the columns' rows see
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
        // a lane's channels are t * D/4 .. : as halves, scaled by a power of two that brings the row's largest
        // below 2 (a row with an infinity or a NaN is left as it is)
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
        const int ex = (int)(__float_as_uint(top) >> 23);      // biased exponent
        // 2^(127 - ex) and its inverse, both normal numbers
        const int sh2 = ex == 255 ? 127 : min(max(ex, 1), 253);
        const float down = __uint_as_float((uint32_t)(254 - sh2) << 23);
        mul = __uint_as_float((uint32_t)sh2 << 23);
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          qf[nt][j][0] = half2_of(bf16_lo(raw[j].x) * down, bf16_hi(raw[j].x) * down);
          qf[nt][j][1] = half2_of(bf16_lo(raw[j].y) * down, bf16_hi(raw[j].y) * down);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int col = nt * 8 + 2 * t + c;
        cf[nt][c] = gk * __shfl_sync(0xffffffffu, mul, (2 * t + c) * 4);
        lim[nt][c] = col < nrows ? e.len + (sh.causal ? (row0 + col) / sh.rep + 1 : 0) : 0;
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

    for (; x < end; ++x) {
      const int s0 = (int)(x - w.at) * sh.tile;
      // ---- scores
      float s[SUB][NT][4];
      wait(&full[unit], phase);
      {
        const char* tile = smem + unit * ge.unit_bytes;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          const int sub = u * teams + team;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[u][nt][i] = 0.f;
          if (idle || sub * 16 >= sh.tile) continue;
          if constexpr (kBf16) {
            const uint32_t addr = smem_u32(tile) + (sub * 16 + (lane & 15)) * ge.row_s + head * (D * 2) + (lane >> 4) * 16;
#pragma unroll
            for (int j = 0; j < KS; ++j) {
              uint32_t a[4];
              ldmatrix4<false>(a, addr + j * 32);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma<FMT>(s[u][nt], a, qf[nt][j][0], qf[nt][j][1]);
            }
          } else {
            const char* r0 = tile + (sub * 16 + slot_of_row(g)) * ge.row_s;
            const char* r1 = r0 + 8 * ge.row_s;
            uint32_t w0[D / 32], w1[D / 32];
            lds_words(w0, r0 + head * (D / 2) + t * (D / 8));
            lds_words(w1, r1 + head * (D / 2) + t * (D / 8));
            const int so = heads * (D / 2) + head * (D / 16) + t * (D / 64);
#pragma unroll
            for (int p = 0; p < D / 64; ++p) {   // 16 channels that share a scale
              const uint32_t b0 = (uint8_t)r0[so + p], b1 = (uint8_t)r1[so + p];
              const uint32_t sc = e4m3x2_to_half2((uint16_t)(b0 | b1 << 8));
              const uint32_t sc0 = __byte_perm(sc, sc, 0x1010), sc1 = __byte_perm(sc, sc, 0x3232);
#pragma unroll
              for (int v = 0; v < 2; ++v) {
                uint32_t x0[4], x1[4];
                e2m1x8_to_half2(w0[2 * p + v], x0);
                e2m1x8_to_half2(w1[2 * p + v], x1);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                  const uint32_t a[4] = {hmul2(x0[2 * y], sc0), hmul2(x1[2 * y], sc1), hmul2(x0[2 * y + 1], sc0),
                                         hmul2(x1[2 * y + 1], sc1)};
                  const int j = 4 * p + 2 * v + y;
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt) mma<FMT>(s[u][nt], a, qf[nt][j][0], qf[nt][j][1]);
                }
              }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[unit]);
      if (++unit == ge.units) {
        unit = 0;
        phase ^= 1;
      }

      // ---- probabilities
      const bool edge = s0 + sh.tile > least;
      uint32_t pb[SUB][NT][kBf16 ? 4 : 2];
      float alpha[NT][2];
      bool moved = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          const int sub = u * teams + team;
          const int at = s0 + sub * 16 + (kBf16 ? g : slot_of_row(g));
          const bool in = !idle && sub * 16 < sh.tile;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = s[u][nt][i] * cf[nt][i & 1];
            if (!in || (edge && at + (i >> 1) * 8 >= lim[nt][i & 1])) v = -INFINITY;
            s[u][nt][i] = v;
            top[i & 1] = fmaxf(top[i & 1], v);
          }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 4));
          top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 8));
          top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 16));
          const float mn = fmaxf(m[nt][c], top[c]), base = mn == -INFINITY ? 0.f : mn;
          alpha[nt][c] = ex2(m[nt][c] - base);
          moved |= mn != m[nt][c];
          m[nt][c] = mn;
          l[nt][c] *= alpha[nt][c];
          top[c] = base - kUp;
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[u][nt][i] = ex2(s[u][nt][i] - top[i & 1]);
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
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j][nt][i] *= alpha[nt][i & 1];
      }

      // ---- their sum of values
      wait(&full[unit], phase);
      {
        const char* tile = smem + unit * ge.unit_bytes;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          const int sub = u * teams + team;
          if (idle || sub * 16 >= sh.tile) continue;
          const int at = s0 + sub * 16;
          // the slots of this lane's operand elements: k = 2t, 2t + 1 (and those + 8)
          const int k0 = kBf16 ? 2 * t : slot_of_row(2 * t), k1 = kBf16 ? 2 * t + 1 : slot_of_row(2 * t + 1);
          // Gives block mt of the operand (channels x slots) to f, for every mt.
          auto each = [&](auto&& f) {
            if constexpr (kBf16) {
              const uint32_t addr = smem_u32(tile) + (sub * 16 + (lane & 7) + (lane >> 4) * 8) * ge.row_s +
                                    head * (D * 2) + ((lane >> 3) & 1) * 16;
#pragma unroll
              for (int mt = 0; mt < KS; ++mt) {
                uint32_t a[4];
                ldmatrix4<true>(a, addr + mt * 32);
                f(mt, a);
              }
            } else {
              const char* base = tile + sub * 16 * ge.row_s;
              const char* p0 = base + k0 * ge.row_s;
              const char* p1 = base + k1 * ge.row_s;
              const int co = head * (D / 2) + g * (D / 16), so = heads * (D / 2) + head * (D / 16) + g * (D / 8) / 16;
              uint32_t wa[D / 64], wb[D / 64], wc[D / 64], wd[D / 64];
              lds_words(wa, p0 + co);
              lds_words(wb, p1 + co);
              lds_words(wc, p0 + 8 * ge.row_s + co);
              lds_words(wd, p1 + 8 * ge.row_s + co);
              uint32_t sl = 0, sh8 = 0;
#pragma unroll
              for (int v = 0; v < D / 64; ++v) {   // eight channels: four blocks
                if (v % 2 == 0) {
                  const int o2 = so + v / 2;
                  sl = e4m3x2_to_half2((uint16_t)((uint8_t)p0[o2] | (uint32_t)(uint8_t)p1[o2] << 8));
                  sh8 = e4m3x2_to_half2((uint16_t)((uint8_t)p0[8 * ge.row_s + o2] | (uint32_t)(uint8_t)p1[8 * ge.row_s + o2] << 8));
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
          // Slots that some rows see and others do not may hold an infinity or a NaN, which a probability of 0 does not
          // silence: then the rows of each token go by themselves, the values that they do not see taken as 0.
          bool apart = false;
          if (at + 16 > least) {
            constexpr uint32_t kExp = kBf16 ? 0x7f80u : 0x7c00u;
            each([&](int, uint32_t (&a)[4]) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                apart |= (a[i] & kExp) == kExp || (a[i] >> 16 & kExp) == kExp;
            });
            apart = __any_sync(0xffffffffu, apart);
          }
          if (!apart) {
            each([&](int mt, uint32_t (&a)[4]) {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma<FMT>(o[mt][nt], a, pb[u][nt][0], pb[u][nt][1]);
                if constexpr (kBf16) mma<FMT>(o[mt][nt], a, pb[u][nt][2], pb[u][nt][3]);
              }
            });
          } else {
            const int last = (row0 + nrows - 1) / sh.rep;
            for (int i = row0 / sh.rep; i <= last; ++i) {
              const int n = e.len + (sh.causal ? i + 1 : 0) - at;   // of these slots, those that token i sees
              const uint32_t m0 = (k0 < n ? 0xffffu : 0u) | (k1 < n ? 0xffff0000u : 0u);
              const uint32_t m8 = (k0 + 8 < n ? 0xffffu : 0u) | (k1 + 8 < n ? 0xffff0000u : 0u);
              each([&](int mt, uint32_t (&a)[4]) {
                const uint32_t z[4] = {a[0] & m0, a[1] & m0, a[2] & m8, a[3] & m8};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  // only the columns of token i; the others keep their sums
                  float keep[4];
#pragma unroll
                  for (int y = 0; y < 4; ++y) keep[y] = o[mt][nt][y];
                  mma<FMT>(o[mt][nt], z, pb[u][nt][0], pb[u][nt][1]);
                  if constexpr (kBf16) mma<FMT>(o[mt][nt], z, pb[u][nt][2], pb[u][nt][3]);
#pragma unroll
                  for (int y = 0; y < 4; ++y)
                    if ((row0 + nt * 8 + 2 * t + (y & 1)) / sh.rep != i) o[mt][nt][y] = keep[y];
                }
              });
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[unit]);
      if (++unit == ge.units) {
        unit = 0;
        phase ^= 1;
      }
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
      asm volatile("bar.sync 1, 256;" ::: "memory");
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
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (!idle && team < step) {
        const float* from = box + (team * heads + head) * kBox + lane;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float a[2], b[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float m2 = from[(KS * NT * 4 + nt * 4 + c) * 32], l2 = from[(KS * NT * 4 + nt * 4 + 2 + c) * 32];
            const float mn = fmaxf(m[nt][c], m2), base = mn == -INFINITY ? 0.f : mn;
            a[c] = ex2(m[nt][c] - base);
            b[c] = ex2(m2 - base);
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
      const bool whole = x == w.at + w.tiles && x - w.tiles >= lo;
      const bool inside = w.at < lo;   // the item began in an earlier CTA
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
              *reinterpret_cast<float2*>(part + kAttnGroup * sh.rows * D + (head * sh.rows + row) * 2) =
                  make_float2(m[nt][c] - kUp, l[nt][c]);
            } else if (lse) {
              lse[token * dm.Hq + hq] = l[nt][c] == 0.f ? -INFINITY : (m[nt][c] - kUp + log2f(l[nt][c])) * 0.69314718055994531f;
            }
          }
        }
    }
    w.step();
  }
}

// ------------------------------------------------------------------ joining the parts of an item
constexpr int kJoinThreads = 256;

// One block an item's KV head: the CTAs that worked on the item left their maxima, sums and unscaled outputs; threads
// take four channels of a row each and, where rows are few, a share of the parts.
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(AttnState st, AttnDims dm, Geometry ge, Batch ba,
                                                                      Rows out, float* lse) {
  __shared__ float s_acc[kJoinThreads][6];
  const AttnShape& sh = ge.sh;
  const int b = blockIdx.y, kh = blockIdx.x % dm.H, run = blockIdx.x / dm.H;
  pdl_wait();
  const int64_t p0 = st.plan[b], p1 = st.plan[b + 1];
  if (p0 == p1) return;
  const int64_t total = st.plan[ba.n_seq];
  Entry e;
  if (!batch_entry(ba, dm, b, sh.causal, st.err, &e) || run >= row_runs(sh, e.n)) return;
  const int group = kh / kAttnGroup, head = kh % kAttnGroup;
  int64_t at = p0 + group * ((p1 - p0) / sh.groups);
  for (int r = 0; r < run; ++r) at += item_tiles(sh, e.n, e.len, r);
  const int c0 = cta_of_tile(at, total), c1 = cta_of_tile(at + item_tiles(sh, e.n, e.len, run) - 1, total);
  if (c0 == c1) return;
  const int row0 = run * sh.rows, nrows = min(sh.rows, rows_of(sh, e.n) - row0);
  const int lanes = dm.d / 4, work = nrows * lanes;          // float4 columns of the item's head
  int shares = kJoinThreads / work;
  shares = shares < 1 ? 1 : shares;
  const int share = threadIdx.x / work;
  for (int i0 = 0; i0 < work; i0 += kJoinThreads) {
    const int i = shares > 1 ? threadIdx.x % work : i0 + threadIdx.x;
    const bool on = i < work && share < shares;
    const int row = i / lanes, ch = i % lanes * 4;
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (on) {
#pragma unroll 4
      for (int c = c0 + (shares > 1 ? share : 0); c <= c1; c += shares) {
        if (first_tile(c, total) == first_tile(c + 1, total)) continue;   // fewer tiles than CTAs: no share, no part
        const float* part = st.part + (int64_t)(c * 2 + (c == c0 ? 1 : 0)) * ge.slot_floats;
        const float2 ml = *reinterpret_cast<const float2*>(part + kAttnGroup * sh.rows * dm.d + (head * sh.rows + row) * 2);
        const float4 v = *reinterpret_cast<const float4*>(part + (int64_t)(head * sh.rows + row) * dm.d + ch);
        const float mn = fmaxf(m, ml.x), base = mn == -INFINITY ? 0.f : mn;
        const float a = ex2(m - base), z = ex2(ml.x - base);
        l = l * a + ml.y * z;
        acc.x = acc.x * a + v.x * z;
        acc.y = acc.y * a + v.y * z;
        acc.z = acc.z * a + v.z * z;
        acc.w = acc.w * a + v.w * z;
        m = mn;
      }
    }
    if (shares > 1) {
      float* mine = s_acc[threadIdx.x];
      mine[0] = m; mine[1] = l; mine[2] = acc.x; mine[3] = acc.y; mine[4] = acc.z; mine[5] = acc.w;
      __syncthreads();
      if (share == 0) {
        for (int k = 1; k < shares; ++k) {
          const float* o = s_acc[threadIdx.x + k * work];
          const float mn = fmaxf(m, o[0]), base = mn == -INFINITY ? 0.f : mn;
          const float a = ex2(m - base), z = ex2(o[0] - base);
          l = l * a + o[1] * z;
          acc.x = acc.x * a + o[2] * z;
          acc.y = acc.y * a + o[3] * z;
          acc.z = acc.z * a + o[4] * z;
          acc.w = acc.w * a + o[5] * z;
          m = mn;
        }
      }
    }
    if (on && (shares == 1 || share == 0)) {
      const int r = row0 + row;
      const int64_t token = e.tok0 + r / sh.rep;
      const int hq = kh * sh.rep + r % sh.rep;
      const float mul = l == 0.f ? 0.f : 1.f / l;
      *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(out.p) + token * out.st + hq * out.sh + ch) =
          make_uint2(bf162_of(acc.x * mul, acc.y * mul), bf162_of(acc.z * mul, acc.w * mul));
      if (lse && ch == 0) lse[token * dm.Hq + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
    }
  }
}

// ------------------------------------------------------------------ host
Geometry geometry(const AttnDims& dm, int n_seq, int max_new, bool causal) {
  return attn_geometry(dm.H, dm.rep, dm.d, dm.fmt == EPIKV_CACHE_E2M1, n_seq, max_new, causal);
}

constexpr int sub_blocks(int fmt, int nt) { return attn_sub_blocks(fmt == EPIKV_CACHE_E2M1, nt); }

template <int D, int FMT, int NT>
cudaError_t run(const AttnState& st, const AttnDims& dm, const Geometry& ge, int layer, const Batch& ba, const Rows& q,
                const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  return plain_launch(attention_kernel<D, FMT, NT, sub_blocks(FMT, NT)>, kAttnCtas, kThreads, ge.smem_bytes, stream, st, dm, ge,
                      layer, ba, q, out, lse, kv, dm.scale * 1.4426950408889634f);
}

template <int D, int FMT>
cudaError_t run_rows(const AttnState& st, const AttnDims& dm, const Geometry& ge, int layer, const Batch& ba,
                     const Rows& q, const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  if constexpr (D <= 64)
    if (ge.sh.rows == 32) return run<D, FMT, 4>(st, dm, ge, layer, ba, q, out, lse, kv, stream);
  if constexpr (D <= 128)
    if (ge.sh.rows == 16) return run<D, FMT, 2>(st, dm, ge, layer, ba, q, out, lse, kv, stream);
  return run<D, FMT, 1>(st, dm, ge, layer, ba, q, out, lse, kv, stream);
}

template <int D, int FMT, int NT>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attention_kernel<D, FMT, NT, sub_blocks(FMT, NT)>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmem);
}

template <int D, int FMT>
cudaError_t prepare_rows() {
  cudaError_t e = prepare_one<D, FMT, 1>();
  if constexpr (D <= 128)
    if (e == cudaSuccess) e = prepare_one<D, FMT, 2>();
  if constexpr (D <= 64)
    if (e == cudaSuccess) e = prepare_one<D, FMT, 4>();
  return e;
}

}  // namespace

size_t attention_part_floats(const AttnDims& dm) {
  const Geometry ge = geometry(dm, 1, dm.max_new, true);
  return (size_t)2 * kAttnCtas * ge.slot_floats;
}

cudaError_t attention_prepare(const AttnDims& dm) {
  const bool q4 = dm.fmt == EPIKV_CACHE_E2M1;
  if (dm.d == 64) return q4 ? prepare_rows<64, EPIKV_CACHE_E2M1>() : prepare_rows<64, EPIKV_CACHE_BF16>();
  if (dm.d == 128) return q4 ? prepare_rows<128, EPIKV_CACHE_E2M1>() : prepare_rows<128, EPIKV_CACHE_BF16>();
  return q4 ? prepare_rows<256, EPIKV_CACHE_E2M1>() : prepare_rows<256, EPIKV_CACHE_BF16>();
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
  const dim3 grid((unsigned)(dm.H * (int64_t)row_runs(ge.sh, ba.max_new)), ba.n_seq);
  return pdl_launch(attention_join_kernel, grid, kJoinThreads, 0, stream, st, dm, ge, ba, out, lse);
}

}  // namespace epikv
