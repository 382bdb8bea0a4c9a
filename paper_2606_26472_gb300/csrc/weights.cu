// What slots receive of attention, and its way into the eviction context.
//
//   w[h][slot] (+)= sum over rows r of KV head h of 2^(c q_r.k_slot - lse_r log2(e)),   c = scale log2(e)
//
// A unit is 128 slots of one entry and KV head.  Its products run on tcgen05
// with the slots as the instruction's 128 rows and the query rows as its
// columns, so that a thread owns a slot and adds up its columns: no exchange
// between threads, and no sum that two CTAs share.  Keys stay in shared memory
// while tiles of query rows pass by; each slot's sum is formed in the order of
// the rows.
#include "attn_plan.h"
#include "kernels.h"
#include "tensor.cuh"

namespace epikv {
namespace {

constexpr int kUnitSlots = 128;
constexpr int kWeightThreads = 384;    // 8 warps add up, one issues products, three copy
constexpr int kCopyThreads = 96;
constexpr float kLog2e = 1.4426950408889634f;

template <int D, int N>
struct WeightShape {
  static constexpr int kKeys = kUnitSlots * D * 2;     // bytes of a unit's keys
  static constexpr int kQuery = N * D * 2;
  static constexpr int kKeyStages = N == 16 ? (D == 64 ? 8 : D == 128 ? 5 : 2) : 2;
  static constexpr int kQueryStages = N == 16 ? kKeyStages : D == 256 ? 1 : 3;
  static constexpr int kLag = (kKeyStages < kQueryStages ? kKeyStages : kQueryStages) - 1;   // steps in flight behind the newest
  static constexpr int kRing = kKeyStages * kKeys + kQueryStages * kQuery;
};

template <int D, int N>
struct alignas(16) WeightShared {
  using Shape = WeightShape<D, N>;
  uint64_t full[Shape::kQueryStages], query_left[Shape::kQueryStages], keys_left[Shape::kKeyStages], scores[2], taken[2];
  uint32_t tmem;
  int gave_up;
  int64_t offset[2][kUnitSlots];
  uint8_t there[Shape::kKeyStages][kUnitSlots];        // the slot is in the view
  float2 row[Shape::kQueryStages][N];                  // factor of the row's scores, log2 of its sum
  int seen[Shape::kQueryStages][N];                    // slots that the row sees
  int partly[Shape::kQueryStages];                     // not every row sees all slots of the unit that any sees
  float half[2][kUnitSlots];                           // a unit's sums of every second tile of rows
};

template <int D, bool kHalf>
__device__ __forceinline__ float store_query(uint32_t tile, int row, const uint4* src) {
  uint32_t top = 0;
  if (src)
    for (int c = 0; c < D / 8; ++c) {
      const uint4 v = __ldg(src + c);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
    }
  const int up = min(14 - ((int)(top >> 7) - 127), 100);
  const float mul = __uint_as_float((uint32_t)(up + 127) << 23);
  for (int c = 0; c < D / 8; ++c) {
    const uint4 v = src ? __ldg(src + c) : make_uint4(0, 0, 0, 0);
    sts16(tile + tile_at<D>(row, c),
          make_uint4(half_pair(bf16_lo(v.x) * mul, bf16_hi(v.x) * mul), half_pair(bf16_lo(v.y) * mul, bf16_hi(v.y) * mul),
                     half_pair(bf16_lo(v.z) * mul, bf16_hi(v.z) * mul), half_pair(bf16_lo(v.w) * mul, bf16_hi(v.w) * mul)));
  }
  return __uint_as_float((uint32_t)(127 - up) << 23);
}

struct WeightCall {
  int layer, causal, last, add;
  float* w;
  int64_t stride_seq, stride_head;
  const float* lse;
  float c;
};

struct Unit {
  int b, kh, s0;       // entry, KV head, first slot
  Entry e;
  int slots;           // of the entry
  int row0, steps;     // first query row that sees the unit, tiles of rows from there
};

// Goes through the units of a CTA: every gridDim.x-th of the line of (entry, 128 slots, KV head).
template <int N>
struct UnitWalk {
  const uint32_t* pre;    // [n_seq + 1] tiles before each entry
  const Batch& ba;
  const AttnDims& dm;
  const WeightCall& call;
  int64_t at;
  int b = -1;
  Entry e = {};
  int first = 0;          // first row that counts
  __device__ __forceinline__ UnitWalk(const uint32_t* pre_, const Batch& ba_, const AttnDims& dm_, const WeightCall& call_)
      : pre(pre_), ba(ba_), dm(dm_), call(call_), at((int64_t)blockIdx.x - gridDim.x) {}
  __device__ __forceinline__ bool next(Unit* u) {
    at += gridDim.x;
    const int64_t total = (int64_t)pre[ba.n_seq] * dm.H;
    if (at >= total) return false;
    const uint32_t tile = (uint32_t)(at / dm.H);
    int nb = b < 0 ? 0 : b;
    while (tile >= pre[nb + 1]) ++nb;
    if (nb != b) {
      b = nb;
      e.tok0 = ba.cu_new[b];
      e.n = ba.cu_new[b + 1] - e.tok0;
      e.seq = ba.seq_ids[b];
      e.len = ba.len[(int64_t)b * ba.len_stride];
      first = call.last && call.last < e.n ? (e.n - call.last) * dm.rep : 0;
    }
    u->b = b;
    u->e = e;
    u->kh = (int)(at - (int64_t)tile * dm.H);
    u->s0 = (int)(tile - pre[b]) * kUnitSlots;
    u->slots = e.len + (call.causal ? e.n : 0);
    u->row0 = first;
    if (call.causal && u->s0 > e.len) u->row0 = max(first, (u->s0 - e.len) * dm.rep);
    u->steps = (max(e.n * dm.rep - u->row0, 0) + N - 1) / N;
    return true;
  }
};

template <int D, int FMT, int N>
__device__ __forceinline__ void copy_unit_keys(uint32_t dst, const int64_t* offset, const AttnDims& dm, const KvDev& kv, int kh,
                                               int tid) {
  using Shape = WeightShape<D, N>;
  const char* base = kv.base[0];
  if constexpr (FMT == EPIKV_CACHE_BF16) {
    constexpr int kPer = D / 8;
#pragma unroll 4
    for (int x = tid; x < kUnitSlots * kPer; x += kCopyThreads) {
      const int r = x / kPer, c = x % kPer;
      const int64_t o = offset[r];
      copy_async16(dst + tile_at<D>(r, c), base + (o < 0 ? 0 : (o + kh * D + c * 8) * 2),
                   o < 0 ? 0 : 16);
    }
  } else {
    constexpr int kPer = D / 32;
    constexpr int kAtOnce = 6;
#pragma unroll 1
    for (int x0 = tid; x0 < kUnitSlots * kPer; x0 += kAtOnce * kCopyThreads) {
      uint4 codes[kAtOnce];
      uint32_t scales[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int x = x0 + u * kCopyThreads, r = x / kPer, c = x % kPer;
        codes[u] = make_uint4(0, 0, 0, 0);
        scales[u] = 0;
        const int64_t o = x < kUnitSlots * kPer ? offset[r] : -1;
        if (o >= 0) {
          const char* row = base + o * 2;
          codes[u] = *reinterpret_cast<const uint4*>(row + kh * (D / 2) + c * 16);
          scales[u] = *reinterpret_cast<const uint16_t*>(row + scale_offset(dm, kh) + c * 2);
        }
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int x = x0 + u * kCopyThreads, r = x / kPer, c = x % kPer;
        if (x < kUnitSlots * kPer) {
          uint4 v[4];
          expand32(codes[u], scales[u], v);
#pragma unroll
          for (int k = 0; k < 4; ++k) sts16(dst + tile_at<D>(r, c * 4 + k), v[k]);
        }
      }
    }
  }
}

template <int D, int FMT, int N>
__device__ __forceinline__ void copy_units(char* ring, WeightShared<D, N>& sh, const TensorWaiter& wait, const AttnState& st,
                                           const AttnDims& dm, const WeightCall& call, const Rows& q, const KvDev& kv,
                                           UnitWalk<N> walk, int tid) {
  using Shape = WeightShape<D, N>;
  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  Unit u;
  int step = 0, unit = 0;   // counted over the CTA's units that have steps
  auto deliver = [&](int i) {
    fence_proxy_async_smem();
    mbar_arrive_one(&sh.full[i % Shape::kQueryStages]);
  };
  while (walk.next(&u)) {
    if (u.steps == 0) continue;
    const int ks = unit % Shape::kKeyStages;
    int64_t* offset = sh.offset[unit & 1];
    if (unit >= Shape::kKeyStages) wait(&sh.keys_left[ks], (uint32_t)(unit / Shape::kKeyStages - 1) & 1);
    for (int r = tid; r < kUnitSlots; r += kCopyThreads) {
      const int s = u.s0 + r;
      int64_t o = -1;
      if (s < u.slots) {
        o = kv_row_offset(kv, call.layer, u.e.seq, s, dm.T);
        if (o < 0) set_error(st.err, EPIKV_DEV_SLOT);
      }
      offset[r] = o;
      sh.there[ks][r] = o >= 0;
    }
    named_sync(1, kCopyThreads);
    const float mul_k = kBf16 ? 1.f : head_scale(st, dm, 0, call.layer, u.kh);
    for (int k = 0; k < u.steps; ++k, ++step) {
      const int qs = step % Shape::kQueryStages, row0 = u.row0 + k * N;
      if (step >= Shape::kQueryStages) wait(&sh.query_left[qs], (uint32_t)(step / Shape::kQueryStages - 1) & 1);
      if (k == 0) copy_unit_keys<D, FMT, N>(smem_u32(ring + ks * Shape::kKeys), offset, dm, kv, u.kh, tid);
      const uint32_t dst = smem_u32(ring + Shape::kKeyStages * Shape::kKeys + qs * Shape::kQuery);
      const int rows = min(u.e.n * dm.rep - row0, N);
      if constexpr (kBf16) {
        constexpr int kPer = D / 8;
#pragma unroll 4
        for (int x = tid; x < N * kPer; x += kCopyThreads) {
          const int r = x / kPer, c = x % kPer, at = row0 + r;
          const bool in = r < rows;
          const int token = at / dm.rep, hq = u.kh * dm.rep + at % dm.rep;
          copy_async16(dst + tile_at<D>(r, c),
                       q.p + (in ? ((int64_t)(u.e.tok0 + token) * q.st + hq * q.sh + c * 8) * 2 : 0), in ? 16 : 0);
        }
      }
      bool partly = false;
      for (int r = tid; r < N; r += kCopyThreads) {
        const bool in = r < rows;
        const int at = row0 + r, token = at / dm.rep, hq = u.kh * dm.rep + at % dm.rep;
        const float lse = in ? __ldg(call.lse + (int64_t)(u.e.tok0 + token) * dm.Hq + hq) : -INFINITY;
        float c = call.c * mul_k;
        if constexpr (!kBf16)
          c *= store_query<D, true>(dst, r,
                                    in ? reinterpret_cast<const uint4*>(q.p + ((int64_t)(u.e.tok0 + token) * q.st + hq * q.sh) * 2)
                                       : nullptr);
        const int seen = lse == -INFINITY ? 0 : call.causal ? u.e.len + token + 1 : u.e.len;
        sh.row[qs][r] = make_float2(c, lse * kLog2e);
        sh.seen[qs][r] = seen;
        partly |= seen < min(u.s0 + kUnitSlots, u.slots);
      }
      if (tid == 0) sh.partly[qs] = 0;
      named_sync(1, kCopyThreads);
      if (partly) sh.partly[qs] = 1;
      copy_commit();
      if (step >= Shape::kLag) {
        copy_wait<Shape::kLag>();
        deliver(step - Shape::kLag);
      }
    }
    ++unit;
  }
  copy_wait<0>();
  for (int i = max(step - Shape::kLag, 0); i < step; ++i) deliver(i);
}

template <int D, int FMT, int N>
__device__ __forceinline__ void issue_units(uint32_t ring, WeightShared<D, N>& sh, const TensorWaiter& wait, UnitWalk<N> walk,
                                            uint32_t tmem) {
  using Shape = WeightShape<D, N>;
  constexpr uint32_t kScores = product_of(128, N, FMT == EPIKV_CACHE_BF16, false);
  Unit u;
  int step = 0, unit = 0;
  while (walk.next(&u)) {
    if (u.steps == 0) continue;
    const int ks = unit % Shape::kKeyStages;
    for (int k = 0; k < u.steps; ++k, ++step) {
      const int qs = step % Shape::kQueryStages, buf = step & 1;
      wait(&sh.full[qs], (uint32_t)(step / Shape::kQueryStages) & 1);
      if (step >= 2) wait(&sh.taken[buf], (uint32_t)(step / 2 - 1) & 1);
      tensor_fence_after();
      const uint32_t a = ring + ks * Shape::kKeys, b = ring + Shape::kKeyStages * Shape::kKeys + qs * Shape::kQuery;
#pragma unroll
      for (int x = 0; x < D / 16; ++x)
        multiply(tmem + buf * N, rows_operand<D>(a) + rows_step(x), rows_operand<D>(b) + rows_step(x), kScores, x > 0);
      products_done(&sh.scores[buf]);
      products_done(&sh.query_left[qs]);
      if (k + 1 == u.steps) products_done(&sh.keys_left[ks]);
    }
    ++unit;
  }
}

template <int D, int N>
__device__ __forceinline__ void add_up(WeightShared<D, N>& sh, const TensorWaiter& wait, const AttnDims& dm,
                                       const WeightCall& call, UnitWalk<N> walk, uint32_t tmem, int group, int tid) {
  using Shape = WeightShape<D, N>;
  Unit u;
  int step = 0, unit = 0, joint = 0;
  const int lane = tid & 31;
  while (walk.next(&u)) {
    float* to = call.w + u.e.seq * call.stride_seq + u.kh * call.stride_head + u.s0 + tid;
    const int s = u.s0 + tid;
    if (u.steps == 0) {
      if (group == 0 && s < u.slots && !call.add) *to = 0.f;
      continue;
    }
    const int ks = unit % Shape::kKeyStages;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < u.steps; ++k, ++step) {
      const int qs = step % Shape::kQueryStages, buf = step & 1;
      if (buf != group) continue;   // the two groups take tiles of rows in turn
      wait(&sh.scores[buf], (uint32_t)(step / 2) & 1);
      tensor_fence_after();
      uint32_t x[N];
      if constexpr (N == 16) {
        tmem_load16(tmem + buf * N, x);
      } else {
#pragma unroll
        for (int i = 0; i < N; i += 32) tmem_load32(tmem + buf * N + i, x + i);
      }
      tmem_wait_load();
      tensor_fence_before();
      mbar_arrive_one(&sh.taken[buf]);
      const float2* row = sh.row[qs];
      if (!sh.partly[qs]) {
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i & 3] += exp2_fast(__uint_as_float(x[i]) * row[i].x - row[i].y);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float p = exp2_fast(__uint_as_float(x[i]) * row[i].x - row[i].y);
          sum[i & 3] += s < sh.seen[qs][i] ? p : 0.f;
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive_one(&sh.query_left[qs]);
    }
    float w = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    bool mine = ((step - 1) & 1) == group;   // the group of the last tile writes
    if (u.steps > 1) {
      if (!mine) sh.half[joint & 1][tid] = w;
      named_sync(2, 256);
      if (mine) w += sh.half[joint & 1][tid];
      ++joint;
    }
    if (mine) {
      const bool there = sh.there[ks][tid];
      __syncwarp();
      if (lane == 0) mbar_arrive_one(&sh.keys_left[ks]);
      if (s < u.slots) {
        if (!there) w = 0.f;
        *to = call.add ? *to + w : w;
      }
    }
    ++unit;
  }
}

template <int D, int FMT, int N>
__global__ void __launch_bounds__(kWeightThreads, 1)
    weights_kernel(AttnState st, AttnDims dm, Batch ba, WeightCall call, Rows q, KvDev kv) {
  using Shape = WeightShape<D, N>;
  extern __shared__ char dynamic[];
  char* ring = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  uint32_t* pre = reinterpret_cast<uint32_t*>(ring + Shape::kRing);
  __shared__ WeightShared<D, N> sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr uint32_t kColumns = 2 * N < 32 ? 32 : 2 * N;
  if (warp == 8) tmem_alloc(&sh.tmem, kColumns);
  if (tid == 0) {
    for (int i = 0; i < Shape::kQueryStages; ++i) {
      mbar_init(&sh.full[i], kCopyThreads);
      mbar_init(&sh.query_left[i], 1 + 4);
    }
    for (int i = 0; i < Shape::kKeyStages; ++i) mbar_init(&sh.keys_left[i], 1 + 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.scores[i], 1);
      mbar_init(&sh.taken[i], 128);
    }
    sh.gave_up = 0;
    fence_barrier_init();
  }
  pdl_wait();
  pdl_trigger();
  if (warp == 0) {   // tiles before each entry; an entry that cannot be taken has none
    uint32_t before = 0;
    for (int b0 = 0; b0 < ba.n_seq; b0 += 32) {
      uint32_t n = 0;
      Entry e;
      if (b0 + lane < ba.n_seq && batch_entry(ba, dm, b0 + lane, call.causal, st.err, &e))
        n = (e.len + (call.causal ? e.n : 0) + kUnitSlots - 1) / kUnitSlots;
      uint32_t upto = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      if (b0 + lane < ba.n_seq) pre[b0 + lane + 1] = before + upto;
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) pre[0] = 0;
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  const uint32_t tmem = sh.tmem;
  const TensorWaiter wait{&sh.gave_up, st.err};
  const UnitWalk<N> walk(pre, ba, dm, call);
  if (warp < 8) {
    add_up<D, N>(sh, wait, dm, call, walk, tmem + ((uint32_t)(warp & 3) << 21), warp >> 2, tid & 127);
  } else if (warp == 8) {
    if (lane == 0) issue_units<D, FMT, N>(smem_u32(ring), sh, wait, walk, tmem);
    __syncwarp();
  } else {
    copy_units<D, FMT, N>(ring, sh, wait, st, dm, call, q, kv, walk, tid - 288);
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  if (warp == 8) tmem_free(tmem, kColumns);
}

template <int D, int N>
constexpr int weights_smem(int n_seq) { return WeightShape<D, N>::kRing + 1024 + (n_seq + 1) * 4; }

template <int D, int FMT, int N>
cudaError_t run_weights(const AttnState& st, const AttnDims& dm, const Batch& ba, const WeightCall& call, const Rows& q,
                        const KvDev& kv, cudaStream_t stream) {
  static_assert(weights_smem<D, N>(kMaxSeqs) + sizeof(WeightShared<D, N>) <= 227 * 1024, "shared memory");
  return pdl_launch(weights_kernel<D, FMT, N>, dim3(kAttnCtas), kWeightThreads, weights_smem<D, N>(ba.n_seq), stream, st, dm, ba,
                    call, q, kv);
}

template <int D, int FMT, int N>
cudaError_t allow_weights() {
  return cudaFuncSetAttribute(weights_kernel<D, FMT, N>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              weights_smem<D, N>(kMaxSeqs));
}

template <int D, int FMT>
cudaError_t prepare_dim() {
  const cudaError_t e = allow_weights<D, FMT, 16>();
  return e == cudaSuccess ? allow_weights<D, FMT, 128>() : e;
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

cudaError_t weights_prepare(const AttnDims& dm) {
  const bool bf16 = dm.fmt == EPIKV_CACHE_BF16;
  if (dm.d == 64) return bf16 ? prepare_dim<64, EPIKV_CACHE_BF16>() : prepare_dim<64, EPIKV_CACHE_E2M1>();
  if (dm.d == 128) return bf16 ? prepare_dim<128, EPIKV_CACHE_BF16>() : prepare_dim<128, EPIKV_CACHE_E2M1>();
  return bf16 ? prepare_dim<256, EPIKV_CACHE_BF16>() : prepare_dim<256, EPIKV_CACHE_E2M1>();
}

cudaError_t launch_attention_weights(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal,
                                     int last, const Rows& q, const float* lse, bool add, float* w, int64_t stride_seq,
                                     int64_t stride_head, const KvDev& kv, cudaStream_t stream) {
  const WeightCall call = {layer, causal, last, add, w, stride_seq, stride_head, lse, dm.scale * kLog2e};
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
  return go(st, dm, ba, call, q, kv, stream);
}

cudaError_t launch_weigh(const DevState& st, const Dims& dm, int n_seq, const int32_t* seq_ids, const float* w,
                         int64_t stride_seq, int64_t stride_head, int heads, float decay, cudaStream_t stream) {
  const int blocks = (dm.T + 255) / 256;
  return pdl_launch(weigh_kernel, dim3(blocks < 64 ? blocks : 64, n_seq), 256, 0, stream, st, dm, seq_ids, w, stride_seq,
                    stride_head, heads, decay);
}

}  // namespace epikv
