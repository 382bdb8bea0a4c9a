// The fifth-generation tensor instructions as the operators of many query rows
// use them: operands in shared memory in rows of 128 bytes (swizzled), results
// and probabilities in tensor memory, and bounded waits between the warps.
#pragma once

#include "attn.cuh"
#include "attn_plan.h"
#include "maps.cuh"

namespace epikv {

// ------------------------------------------------------------ tensor memory
// Whole warp; columns a power of two from 32 to 512.  The address is written to shared memory.
__device__ __forceinline__ void tmem_alloc(uint32_t* dst, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
               :: "r"(smem_u32(dst)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(addr), "r"(columns));
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes; r[i] is column i of the thread's lane.  Valid after tmem_wait_load.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      :: "r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
         "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// All loads so far are there, r's K columns among them (what uses them stays behind it).
template <int K>
__device__ __forceinline__ void tmem_wait_load(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < K; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ------------------------------------------------------------ products
// A tile stands in shared memory by eight rows: for each 64 channels the eight rows' 128 bytes side by side, a row's eight
// 16-byte parts exchanged by its number mod 8 (1,024 bytes, aligned to it: a swizzled block), then the next 64 channels.
// A tensor copy of any number of such rows, all channels, leaves them so.
template <int D>
__device__ __forceinline__ uint32_t tile_at(int row, int part) {   // part: of the row's 16 bytes
  return (row >> 3) * (D * 16) + (part >> 3) * 1024 + (row & 7) * 128 + (((part ^ row) & 7) << 4);
}

// Such rows as an operand whose products run along the channels (16 channels are a step of 32 bytes, 64 of 1,024) ...
template <int D>
__device__ __forceinline__ uint64_t rows_operand(uint32_t smem) {
  return (uint64_t)((smem & 0x3ffff) >> 4) | (uint64_t)1 << 16 | (uint64_t)(D * 16 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
constexpr uint32_t rows_step(int x) { return ((x >> 2) * 1024 + (x & 3) * 32) >> 4; }
// ... and as one whose products run along the rows (16 rows are a step).
template <int D>
__device__ __forceinline__ uint64_t columns_operand(uint32_t smem) {
  return (uint64_t)((smem & 0x3ffff) >> 4) | (uint64_t)(1024 >> 4) << 16 | (uint64_t)(D * 16 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
template <int D>
constexpr uint32_t columns_step(int x) { return x * D * 32 >> 4; }
// Sums in 32 bits; both operands half or bf16.  `along_rows`: the second operand is a columns_operand.
constexpr uint32_t product_of(int m, int n, bool bf16, bool along_rows) {
  return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (along_rows ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 |
         (uint32_t)(m >> 4) << 24;
}
// The warp's lane that issues: the same one each time.
__device__ __forceinline__ bool elected() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is;
}
// One thread; d (+)= a b over 16 values.
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
// The same, a in tensor memory (two values a column).
__device__ __forceinline__ void multiply_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               :: "r"(d), "r"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
// The barrier completes when all that this thread issued before has.
__device__ __forceinline__ void products_done(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];"
               :: "r"(smem_u32(bar)) : "memory");
}

// ------------------------------------------------------------ waits
__device__ __forceinline__ void mbar_arrive_one(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" :: "r"(smem_u32(bar)) : "memory");
}

constexpr uint64_t kTensorWaitNs = 2000000000ull;
struct TensorWaiter {
  volatile int* gave_up;
  int32_t* err;
  // Ends when the phase completes, or (with the error word set) when any wait of the CTA has taken too long: what
  // follows then runs on without waiting, on data that the error word disowns.
  __device__ __forceinline__ void operator()(uint64_t* bar, uint32_t parity) const {
    if (mbar_try_wait(bar, parity)) return;
    const uint64_t t0 = global_ns();
    while (!mbar_try_wait(bar, parity)) {
      if (*gave_up) return;
      if (global_ns() - t0 > kTensorWaitNs) {
        *gave_up = 1;
        set_error(err, EPIKV_DEV_TIMEOUT);
        return;
      }
    }
  }
};

__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, int bytes) {   // the rest of the 16 is zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ void named_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory");
}

__device__ __forceinline__ uint32_t lds2(uint32_t p) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds16(uint32_t p) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(p) : "memory");
  return v;
}
// The same, which the compiler may move up to the last barrier or wait.
__device__ __forceinline__ uint4 lds16_pure(uint32_t p) {
  return *reinterpret_cast<const uint4*>(__cvta_shared_to_generic(p));
}
__device__ __forceinline__ void sts16(uint32_t p, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" :: "r"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Loads that stay where they are written, ahead of the waits that they are to pass.
__device__ __forceinline__ float load_now(const float* p) {
  float v;
  asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t load_now(const uint16_t* p) {
  uint16_t v;
  asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint4 load_now(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

__device__ __forceinline__ float exp2_fast(float x) {   // 2^-22 of the value; 0 below 2^-126
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
  const __half2 r = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Both halves of a times the half in the low or high bits of b.
__device__ __forceinline__ uint32_t half_pair_times(uint32_t a, uint32_t b, bool high) {
  const __half2 s = *reinterpret_cast<const __half2*>(&b);
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), high ? __high2half2(s) : __low2half2(s));
  return *reinterpret_cast<const uint32_t*>(&r);
}

__device__ __forceinline__ uint32_t bf16_pair_times(uint32_t a, uint32_t b, bool high) {
  const __nv_bfloat162 s = *reinterpret_cast<const __nv_bfloat162*>(&b);
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), high ? __high2bfloat162(s) : __low2bfloat162(s));
  return *reinterpret_cast<const uint32_t*>(&r);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// ------------------------------------------------------------ a layer's rows as a tensor
// [blocks or sequences][eights of slots][64s of channels of all heads][8 slots][64 channels]; a copy takes all channels of a
// head of `slots` slots, which stand in one block.
struct LayerMaps {
  CUtensorMap kv[2];
  int slots;   // 0: the layer cannot be described so; rows are copied by lanes
  int end;     // slots of a sequence that the tensor has (a contiguous cache: eights only)
};

__device__ __forceinline__ void tma_load_rows(uint32_t dst, const CUtensorMap* map, int channels, int eight, int block,
                                              uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
      :: "r"(dst), "l"(map), "r"(0), "r"(0), "r"(channels), "r"(eight), "r"(block), "r"(smem_u32(bar)) : "memory");
}

// `most`: slots of a copy, at most (a power of two).
inline LayerMaps layer_maps(const AttnDims& dm, int layer, const KvDev& kv, int most) {
  LayerMaps maps = {};
  if (dm.fmt != EPIKV_CACHE_BF16) return maps;
  const bool flat = kv.layout == EPIKV_LAYOUT_CONTIGUOUS;
  int slots = most;
  while (!flat && slots > 4 && kv.block_size % slots) slots /= 2;
  if (slots < 8 || (flat && dm.T < 8)) return maps;
  const int64_t outer = flat ? kv.stride_seq : kv.stride_block;   // elements
  // sequences closer together than they are long: no tensor says that (see cache_maps in attention.cu)
  if (flat && kv.stride_seq / kv.stride_token < dm.T) return maps;
  const cuuint64_t dims[5] = {64, 8, (cuuint64_t)dm.H * dm.d / 64, (cuuint64_t)(flat ? dm.T : kv.block_size) / 8,
                              (cuuint64_t)(flat ? dm.S : kv.num_blocks)};
  const cuuint64_t strides[4] = {(cuuint64_t)kv.stride_token * 2, 128, (cuuint64_t)kv.stride_token * 16, (cuuint64_t)outer * 2};
  for (int i = 0; i < 4; ++i)
    if (strides[i] == 0 || strides[i] >= (cuuint64_t(1) << 40)) return maps;
  const cuuint32_t box[5] = {64, 8, (cuuint32_t)dm.d / 64, (cuuint32_t)slots / 8, 1}, ones[5] = {1, 1, 1, 1, 1};
  const EncodeTiled encode = encode_tiled();
  if (!encode) return maps;
  for (int w = 0; w < 2; ++w)
    if (encode(&maps.kv[w], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, kv.base[w] + (int64_t)layer * kv.stride_layer * 2, dims,
               strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return maps;
  maps.slots = slots;
  maps.end = flat ? dm.T & ~7 : INT32_MAX;
  return maps;
}

// ------------------------------------------------------------ rows of a tile
// 32 channels of a 4-bit row (16 bytes of codes, two scales) as 64 bytes of halves, exact: 2 + 4 significant bits between
// 2^-10 and 2688.  kWide: as bf16, exact too.  A code's half, moved by the three bits that bf16 has fewer of, is the bf16 of
// 2^-112 times the value; the scale makes good for it.
template <bool kWide>
__device__ __forceinline__ void expand32(const uint4& codes, uint32_t scales, uint4 (&out)[4]) {
  uint32_t s = e4m3x2_to_half2((uint16_t)scales);
  if constexpr (kWide) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&s));
    const float up = __uint_as_float(0x77800000u);   // 2^112
    s = bf16_pair(f.x * up, f.y * up);
  }
  const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t h[4];
    e2m1x8_to_half2(w[i], h);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if constexpr (kWide) h[u] = bf16_pair_times((h[u] >> 3 & 0x0fff0fffu) | (h[u] & 0x80008000u), s, i >= 2);
      else h[u] = half_pair_times(h[u], s, i >= 2);
    }
    out[i] = make_uint4(h[0], h[1], h[2], h[3]);
  }
}

// What turns a score as it is summed into log2 units, kept a normal number: 0 x -inf (a slot that a row does not see) and
// inf x 0 are NaN.
__host__ __device__ __forceinline__ float score_factor(float f) {
  return f < 0x1p-126f ? 0x1p-126f : f > 0x1.fffffep127f ? 0x1.fffffep127f : f;
}

// Pieces of eight bf16 queries, M rows', as halves.  The kPer lanes that hold a row scale it by a power of two to below 2^15:
// bf16's 8 bits then stand whole in channels down to 2^-31 of the row's largest (of rows below 2^-112, which get 2^126, down to
// 2^-17 or more).  undo: what undoes the scaling.
template <int kPer, int M>
__device__ __forceinline__ void halves_of(uint4 (&x)[M], float (&undo)[M]) {
  uint32_t top[M];   // largest magnitudes, as bf16 bits: they are ordered like the values
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    top[i] = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) top[i] = max(top[i], max(w[u] & 0x7fffu, w[u] >> 16 & 0x7fffu));
  }
#pragma unroll
  for (int o = kPer / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < M; ++i) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
#pragma unroll
  for (int i = 0; i < M; ++i) {
    // 2^(141 - ex) of the biased exponent ex and its inverse, both normal numbers (ex = 255: the finite ones' largest)
    const int ex = min(max((int)(top[i] >> 7), 15), 254);
    const float mul = __uint_as_float((uint32_t)(268 - ex) << 23);
    undo[i] = __uint_as_float((uint32_t)(ex - 14) << 23);
    x[i] = make_uint4(half_pair(bf16_lo(x[i].x) * mul, bf16_hi(x[i].x) * mul), half_pair(bf16_lo(x[i].y) * mul, bf16_hi(x[i].y) * mul),
                      half_pair(bf16_lo(x[i].z) * mul, bf16_hi(x[i].z) * mul), half_pair(bf16_lo(x[i].w) * mul, bf16_hi(x[i].w) * mul));
  }
}

// A warp's 32 rows of D bf16 queries into rows `row0` to row0 + 31 of a tile; src: each lane's row.  Lanes beside each other
// load neighbouring pieces.  Over a 4-bit cache the queries become halves; what undoes the scaling of the lane's row is
// returned.
template <int D, bool kHalf>
__device__ __forceinline__ float store_queries(uint32_t tile, int row0, const void* src, int lane) {
  constexpr int kPer = D / 8;            // 16-byte pieces of a row: 8, 16 or 32
  constexpr int kRows = 32 / kPer;       // rows at once
  constexpr int kAtOnce = 32 / kRows < 16 ? 32 / kRows : 16;   // loads in flight
  const int piece = lane % kPer, sub = lane / kPer;
  const uint64_t mine = (uint64_t)src;
  float back = 1.f;
#pragma unroll
  for (int r0 = 0; r0 < 32 / kRows; r0 += kAtOnce) {
    uint4 v[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
      v[i] = load_now(reinterpret_cast<const uint4*>(__shfl_sync(0xffffffffu, mine, (r0 + i) * kRows + sub)) + piece);
    float undo[kAtOnce];   // of the row that the lane's piece is of
    if constexpr (kHalf) halves_of<kPer, kAtOnce>(v, undo);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if constexpr (kHalf) {
        const float mine = __shfl_sync(0xffffffffu, undo[i], lane % kRows * kPer);   // to the lane that owns the row
        if (lane / kRows == r0 + i) back = mine;
      }
      sts16(tile + tile_at<D>(row0 + (r0 + i) * kRows + sub, piece), v[i]);
    }
  }
  return back;
}

// Pieces of 4-bit rows that each of kThreads threads turns into halves (kWide: bf16): 32 channels of every kStep-th row from row `first` on,
// R rows at a time.  Eight neighbouring lanes have two pieces of four rows, whose parts fall on all eight places of a
// swizzled block's 128 bytes.
template <int D, int kThreads, int R, bool kWide = false>
struct CodeRows {
  static constexpr int kPer = D / 32, kStep = kThreads / kPer;
  static_assert(kThreads % 32 == 0 && kPer <= 8, "a warp has whole rows");
  uint4 code[R];
  uint32_t scale[R];
  uint32_t in;       // bit u: row u of the thread's is one
  static __device__ __forceinline__ int piece_of(int tid) { return (tid >> 3) % (kPer / 2) * 2 + (tid & 1); }
  static __device__ __forceinline__ int row_of(int tid) {
    return tid / 32 * (32 / kPer) + (tid & 31) / (4 * kPer) * 4 + (tid >> 1 & 3);
  }
  // `codes`, `scales`: the head's, in bytes of a row; offset: of the rows, elements (-1: zeros)
  __device__ __forceinline__ void load(const char* base, const int64_t* offset, int codes, int scales, int first, int rows,
                                       int tid) {
    const int p = piece_of(tid), r0 = first + row_of(tid);
    int64_t o[R];
#pragma unroll
    for (int u = 0; u < R; ++u) o[u] = offset[min(r0 + u * kStep, rows - 1)];
    codes += p * 16;
    scales += p * 2;
    in = 0;
#pragma unroll
    for (int u = 0; u < R; ++u) {   // (a row that is not there: the first one's memory, times 0)
      if (o[u] >= 0) in |= 1u << u;
      const char* row = base + max(o[u], (int64_t)0) * 2;
      code[u] = load_now(reinterpret_cast<const uint4*>(row + codes));
      scale[u] = load_now(reinterpret_cast<const uint16_t*>(row + scales));
    }
  }
  __device__ __forceinline__ void store(uint32_t tile, int first, int rows, int tid) const {
    const int p = piece_of(tid), r0 = first + row_of(tid);
    uint32_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = tile + tile_at<D>(r0, p * 4 + k);
#pragma unroll
    for (int u = 0; u < R; ++u) {
      if (r0 + u * kStep >= rows) break;
      uint4 v[4];
      expand32<kWide>(code[u], in >> u & 1 ? scale[u] : 0u, v);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        sts16(kStep % 8 == 0 ? at[k] + u * (kStep / 8) * (D * 16) : tile + tile_at<D>(r0 + u * kStep, p * 4 + k), v[k]);
    }
  }
};

// The same rows by way of a ring of raw codes in shared memory, kStages tiles of kRows rows: asynchronous copies keep more of
// them under way than registers would hold.  A thread turns into halves what it has copied itself; the scales (the 16 bytes
// that hold a row's) are copied by one lane of the row's.
template <int D, int kThreads, int kRows, int kStages>
struct CodeRing {
  using Rows = CodeRows<D, kThreads, 1>;
  static constexpr int kPer = Rows::kPer, kStep = Rows::kStep, kRounds = (kRows + kStep - 1) / kStep;
  static_assert(kRows % (32 / kPer) == 0, "the last round's warps have whole rows");
  static constexpr int kCodes = kRows * kPer * 16, kStage = kCodes + kRows * 16, kBytes = kStages * kStage;
  uint32_t ring;
  __device__ __forceinline__ uint32_t codes_at(int i, int u, int tid) const {
    return ring + i % kStages * kStage + (u * kThreads + tid) * 16;
  }
  __device__ __forceinline__ uint32_t scales_at(int i, int u, int row) const {
    return ring + i % kStages * kStage + kCodes + (u * kStep + row) * 16;
  }
  // Where the thread's pieces come from, of a head's that begin a row: the same for all heads of the same slots.
  struct Sources {
    const char *code[kRounds], *scale[kRounds];
    uint32_t codes, scales;   // bit u: there is such a row, which is there
  };
  __device__ __forceinline__ void look(Sources* from, const char* base, const int64_t* offset, int tid) const {
    constexpr int kWarpRows = 32 / kPer;
    const int own = Rows::row_of(tid), lane = tid & 31, scaled = tid / 32 * kWarpRows + lane;
    from->codes = from->scales = 0;
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      const int64_t o = u * kStep + own < kRows ? offset[u * kStep + own] : -1;
      from->code[u] = base + (o < 0 ? 0 : o * 2 + Rows::piece_of(tid) * 16);
      if (o >= 0) from->codes |= 1u << u;
      const int64_t p = lane < kWarpRows && u * kStep + scaled < kRows ? offset[u * kStep + scaled] : -1;
      from->scale[u] = base + (p < 0 ? 0 : p * 2);
      if (p >= 0) from->scales |= 1u << u;
    }
  }
  // Copies of tile i (rows that are not there become zeros); codes, scales: where the head's start in a row, bytes.
  __device__ __forceinline__ void issue(int i, const Sources& from, int codes, int scales, int tid) const {
    constexpr int kWarpRows = 32 / kPer;
    const int own = Rows::row_of(tid), lane = tid & 31, scaled = tid / 32 * kWarpRows + lane;
    scales &= ~15;
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      const bool code = from.codes >> u & 1, scale = from.scales >> u & 1;
      if (u * kStep + own < kRows) copy_async16(codes_at(i, u, tid), from.code[u] + (code ? codes : 0), code ? 16 : 0);
      if (lane < kWarpRows && u * kStep + scaled < kRows)
        copy_async16(scales_at(i, u, scaled), from.scale[u] + (scale ? scales : 0), scale ? 16 : 0);
    }
  }
  // Tile i, which is there for the whole warp, as halves; scales: the head's first in the 16 bytes.
  __device__ __forceinline__ void store(int i, uint32_t tile, int scales, int tid) const {
    const int p = Rows::piece_of(tid), own = Rows::row_of(tid);
    uint32_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = tile + tile_at<D>(own, p * 4 + k);
    scales += p * 2;
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      if (u * kStep + own >= kRows) break;
      uint4 v[4];
      expand32<false>(lds16(codes_at(i, u, tid)), lds2(scales_at(i, u, own) + scales), v);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        sts16(kStep % 8 == 0 ? at[k] + u * (kStep / 8) * (D * 16) : tile + tile_at<D>(own + u * kStep, p * 4 + k), v[k]);
    }
  }
};

}  // namespace epikv
