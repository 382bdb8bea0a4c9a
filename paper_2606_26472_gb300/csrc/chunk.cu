// Attention of a chunk of new tokens over the slots of the cache, many query
// rows at a time on the tensor instructions.
//
//   out = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q.k_j - m),   c = scale log2(e)
//
// A query row is a token and one of the rep query heads that share a KV head;
// a CTA takes up to 256 such rows of one entry and KV head, as one or two
// tiles of 128, and goes over the slots that they see in tiles of 128 (64 at
// 256 channels).  S = Q K^T and O += P V run on tcgen05 with S and O in tensor
// memory; a thread owns a row, so maxima and sums need no exchange; P replaces
// S in tensor memory, in 16 bits.
#include "tensor.cuh"

namespace epikv {
namespace {

constexpr int kChunkThreads = 384;      // 8 warps own rows, one issues products, three copy
constexpr int kCopyThreads = 96;
constexpr float kSlack = 8.f;           // a maximum is moved when a score passes it by 2^8

template <int D>
struct ChunkShape {
  static constexpr int kSlots = D == 256 ? 64 : 128;   // of a tile
  static constexpr int kPanel = kSlots * 128;          // bytes of 64 channels of a tile's slots
  static constexpr int kStage = kSlots * D * 2;
  static constexpr int kQuery = 128 * D * 2;           // bytes of a tile of query rows
  static constexpr int kStages = D == 64 ? 8 : 4;
};

template <int D, int kTiles>
struct alignas(16) ChunkShared {
  static constexpr int kStages = ChunkShape<D>::kStages;
  uint64_t query, full[kStages], empty[kStages], scores[2], weights[2], sums, done;
  uint32_t tmem;
  int gave_up;
  int unclean;                              // an infinite or NaN value stands in a slot that not all rows see
  int64_t offset[2][ChunkShape<D>::kSlots]; // of a tile's slots, elements; -1: none
};

struct ChunkItem {
  Entry e;
  int kh;          // KV head
  int row0, rows;  // the item's first query row of that head, rows
  int tiles;       // of slots
  int least;       // slots that the item's first row sees
  int most;        // and its last
};

// The slots that query row r sees.
__device__ __forceinline__ int seen_of(const Entry& e, int rep, bool causal, int r) {
  return causal ? e.len + r / rep + 1 : e.len;
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

__device__ __forceinline__ bool unbounded16(uint32_t w, uint32_t mask) {   // an exponent of all ones in either half
  return (w & mask) == mask || (w >> 16 & mask) == mask;
}
// The value with 0 in the place of what is infinite or NaN.
__device__ __forceinline__ uint32_t bounded16(uint32_t w, uint32_t mask) {
  if ((w & mask) == mask) w &= 0xffff0000u;
  if ((w >> 16 & mask) == mask) w &= 0xffffu;
  return w;
}

template <int D, int FMT, int kTiles>
__device__ __forceinline__ void copy_tiles(char* ring, ChunkShared<D, kTiles>& sh, const TensorWaiter& wait,
                                           const AttnDims& dm, const ChunkItem& it, const KvDev& kv, int layer,
                                           int32_t* err, int tid) {
  using Shape = ChunkShape<D>;
  constexpr uint32_t kExp = FMT == EPIKV_CACHE_BF16 ? 0x7f80u : 0x7c00u;
  constexpr int kLag = 2;   // stages whose copies are in flight
  const int stages = 2 * it.tiles;
  auto put_clean = [&](uint32_t at, uint4 v) {
    if (unbounded16(v.x, kExp) || unbounded16(v.y, kExp) || unbounded16(v.z, kExp) || unbounded16(v.w, kExp)) {
      sts16(at, make_uint4(bounded16(v.x, kExp), bounded16(v.y, kExp), bounded16(v.z, kExp), bounded16(v.w, kExp)));
      sh.unclean = 1;
    }
  };
  // stage i holds the keys (even) or values (odd) of tile i / 2
  auto deliver = [&](int i) {
    const int s0 = (i >> 1) * Shape::kSlots;
    if ((i & 1) && s0 + Shape::kSlots > it.least) {
      // A probability of 0 must not meet an infinity or a NaN in a slot that only other rows see: each thread looks
      // through what it copied.
      const uint32_t dst = smem_u32(ring + i % Shape::kStages * Shape::kStage);
      constexpr int kPer = FMT == EPIKV_CACHE_BF16 ? D / 8 : D / 32;
      for (int x = tid; x < Shape::kSlots * kPer; x += kCopyThreads) {
        const int r = x / kPer, c = x % kPer;
        if (s0 + r < it.least) continue;
        if constexpr (FMT == EPIKV_CACHE_BF16) {
          const uint32_t at = dst + (c >> 3) * Shape::kPanel + panel_at(r, c & 7);
          put_clean(at, lds16(at));
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint32_t at = dst + (c >> 1) * Shape::kPanel + panel_at(r, (c & 1) * 4 + u);
            put_clean(at, lds16(at));
          }
        }
      }
    }
    fence_proxy_async_smem();
    mbar_arrive_one(&sh.full[i % Shape::kStages]);
  };
  for (int i = 0; i < stages; ++i) {
    const int j = i >> 1, st = i % Shape::kStages, turn = i / Shape::kStages;
    int64_t* offset = sh.offset[j & 1];
    if (!(i & 1)) {
      // the other tile's offsets may still be read; this one's are free since all threads were here for the last tile
      tile_offsets(offset, Shape::kSlots, j * Shape::kSlots, it.most, kv, layer, it.e.seq, dm.T, err, tid, kCopyThreads);
      named_sync(1, kCopyThreads);
    }
    if (turn) wait(&sh.empty[st], (turn & 1) ^ 1);
    const uint32_t dst = smem_u32(ring + st * Shape::kStage);
    const char* base = kv.base[i & 1];
    if constexpr (FMT == EPIKV_CACHE_BF16) {
      constexpr int kPer = D / 8;
#pragma unroll 4
      for (int x = tid; x < Shape::kSlots * kPer; x += kCopyThreads) {
        const int r = x / kPer, c = x % kPer;
        const int64_t o = offset[r];
        copy_async16(dst + (c >> 3) * Shape::kPanel + panel_at(r, c & 7),
                     base + (o < 0 ? 0 : (o + it.kh * D + c * 8) * 2), o < 0 ? 0 : 16);
      }
      copy_commit();
      if (i >= kLag) {
        copy_wait<kLag>();
        deliver(i - kLag);
      }
    } else {
      constexpr int kPer = D / 32;
      constexpr int kMost = (Shape::kSlots * kPer + kCopyThreads - 1) / kCopyThreads;
      uint4 codes[kMost];
      uint32_t scales[kMost];
#pragma unroll
      for (int u = 0; u < kMost; ++u) {
        const int x = tid + u * kCopyThreads, r = x / kPer, c = x % kPer;
        codes[u] = make_uint4(0, 0, 0, 0);
        scales[u] = 0;
        const int64_t o = x < Shape::kSlots * kPer ? offset[r] : -1;
        if (o >= 0) {
          const char* row = base + o * 2;
          codes[u] = *reinterpret_cast<const uint4*>(row + it.kh * (D / 2) + c * 16);
          scales[u] = *reinterpret_cast<const uint16_t*>(row + scale_offset(dm, it.kh) + c * 2);
        }
      }
#pragma unroll
      for (int u = 0; u < kMost; ++u) {
        const int x = tid + u * kCopyThreads, r = x / kPer, c = x % kPer;
        if (x < Shape::kSlots * kPer) {
          uint4 v[4];
          expand32(codes[u], scales[u], v);
#pragma unroll
          for (int k = 0; k < 4; ++k) sts16(dst + (c >> 1) * Shape::kPanel + panel_at(r, (c & 1) * 4 + k), v[k]);
        }
      }
      deliver(i);
    }
  }
  if constexpr (FMT == EPIKV_CACHE_BF16) {
    if (stages >= 2) {
      copy_wait<1>();
      deliver(stages - 2);
    }
    copy_wait<0>();
    if (stages >= 1) deliver(stages - 1);
  }
}

template <int D, int FMT, int kTiles>
__device__ __forceinline__ void issue_products(uint32_t query, uint32_t ring, ChunkShared<D, kTiles>& sh,
                                               const TensorWaiter& wait, int tiles, uint32_t tmem) {
  using Shape = ChunkShape<D>;
  constexpr bool kBf16 = FMT == EPIKV_CACHE_BF16;
  constexpr uint32_t kScores = product_of(128, Shape::kSlots, kBf16, false), kSums = product_of(128, D, kBf16, true);
  auto scores = [&](int t, int buf, int st) {
    const uint32_t q = query + t * Shape::kQuery, k = ring + st * Shape::kStage;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      multiply(tmem + buf * 128, rows_operand(q + (x >> 2) * (128 * 128) + (x & 3) * 32),
               rows_operand(k + (x >> 2) * Shape::kPanel + (x & 3) * 32), kScores, x > 0);
    products_done(&sh.scores[buf]);
  };
  auto sums = [&](int t, int buf, int st, bool add) {
    const uint32_t v = ring + st * Shape::kStage;
#pragma unroll
    for (int x = 0; x < Shape::kSlots / 16; ++x)
      multiply_tmem(tmem + 256 + t * 128, tmem + buf * 128 + x * 8, columns_operand(v + x * 2048, Shape::kPanel), kSums,
                    add || x > 0);
  };
  auto filled = [&](int i) {
    wait(&sh.full[i % Shape::kStages], (uint32_t)(i / Shape::kStages) & 1);
    tensor_fence_after();
  };
  wait(&sh.query, 0);
  tensor_fence_after();
  filled(0);
  for (int t = 0; t < kTiles; ++t) scores(t, t, 0);
  products_done(&sh.empty[0]);
  for (int j = 0; j < tiles; ++j) {
    const int v = (2 * j + 1) % Shape::kStages, k = (2 * j + 2) % Shape::kStages;
    const bool more = j + 1 < tiles;
    if constexpr (kTiles == 1) {   // two places for scores: the next tile's are formed beside this one's probabilities
      if (more) {
        filled(2 * j + 2);
        scores(0, (j + 1) & 1, k);
        products_done(&sh.empty[k]);
      }
      filled(2 * j + 1);
      wait(&sh.weights[j & 1], (uint32_t)(j >> 1) & 1);
      tensor_fence_after();
      sums(0, j & 1, v, j > 0);
      products_done(&sh.empty[v]);
      products_done(&sh.sums);
    } else {
      filled(2 * j + 1);
      if (more) filled(2 * j + 2);
      for (int t = 0; t < 2; ++t) {
        wait(&sh.weights[t], (uint32_t)j & 1);
        tensor_fence_after();
        sums(t, t, v, j > 0);
        if (more) scores(t, t, k);   // in order behind the products that read the probabilities in its place
      }
      products_done(&sh.empty[v]);
      if (more) products_done(&sh.empty[k]);
    }
  }
  products_done(&sh.done);
}

template <int D, int FMT, int kTiles>
__device__ __forceinline__ void soften(ChunkShared<D, kTiles>& sh, const TensorWaiter& wait, int tiles, int seen, float c,
                                       uint32_t tmem, int t, float* m_out, float* l_out) {
  using Shape = ChunkShape<D>;
  constexpr int N = Shape::kSlots;
  float m = -INFINITY, l = 0.f;
  const uint32_t o = tmem + 256 + t * 128;
  for (int j = 0; j < tiles; ++j) {
    const int buf = kTiles == 1 ? j & 1 : t;
    const uint32_t s = tmem + buf * 128;
    wait(&sh.scores[buf], kTiles == 1 ? (uint32_t)(j >> 1) & 1 : (uint32_t)j & 1);
    tensor_fence_after();
    uint32_t x[N];
#pragma unroll
    for (int i = 0; i < N; i += 32) tmem_load32(s + i, x + i);
    tmem_wait_load();
    const int s0 = j * N;
    if (__any_sync(0xffffffffu, seen < s0 + N)) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (s0 + i >= seen) x[i] = 0xff800000u;
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, __uint_as_float(x[i]));
    top *= c;
    const bool up = top > m + kSlack;
    if (__any_sync(0xffffffffu, up)) {
      const float mul = !up ? 1.f : m == -INFINITY ? 0.f : exp2_fast(m - top);
      if (up) m = top;
      l *= mul;
      if (j > 0) {
        if constexpr (kTiles == 1) {   // the last tile's products may still be under way
          wait(&sh.sums, (uint32_t)(j - 1) & 1);
          tensor_fence_after();
        }
#pragma unroll 1
        for (int i = 0; i < D; i += 32) {
          uint32_t y[32];
          tmem_load32(o + i, y);
          tmem_wait_load();
#pragma unroll
          for (int u = 0; u < 32; ++u) y[u] = __float_as_uint(__uint_as_float(y[u]) * mul);
          tmem_store32(o + i, y);
        }
      }
    }
    // a half's range is used up to 2^15: below 2^-24 it has no bits left
    const float base = (m == -INFINITY ? 0.f : m) - (FMT == EPIKV_CACHE_BF16 ? 0.f : 7.f);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; i += 32) {
      uint32_t y[16];
#pragma unroll
      for (int u = 0; u < 32; u += 2) {
        const float a = exp2_fast(__uint_as_float(x[i + u]) * c - base), b = exp2_fast(__uint_as_float(x[i + u + 1]) * c - base);
        sum[u & 3] += a;
        sum[(u & 3) + 1] += b;
        y[u / 2] = FMT == EPIKV_CACHE_BF16 ? bf16_pair(a, b) : half_pair(a, b);
      }
      tmem_store16(s + i / 2, y);
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    tmem_wait_store();
    tensor_fence_before();
    mbar_arrive_one(&sh.weights[buf]);
  }
  *m_out = m;
  *l_out = l;
}

template <int D, int FMT, int kTiles>
__global__ void __launch_bounds__(kChunkThreads, 1)
    chunk_kernel(AttnState st, AttnDims dm, int layer, Batch ba, bool causal, Rows q, Rows out, float* lse, KvDev kv,
                 float c) {
  using Shape = ChunkShape<D>;
  extern __shared__ char dynamic[];
  char* smem = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  __shared__ ChunkShared<D, kTiles> sh;
  char* ring = smem + kTiles * Shape::kQuery;
  const int tid = threadIdx.x, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.y;
  ChunkItem it;
  if (!batch_entry(ba, dm, b, causal, st.err, &it.e)) return;
  it.kh = blockIdx.x % dm.H;
  it.row0 = blockIdx.x / dm.H * (128 * kTiles);
  it.rows = min(it.e.n * dm.rep - it.row0, 128 * kTiles);
  if (it.rows <= 0) return;
  it.least = seen_of(it.e, dm.rep, causal, it.row0);
  it.most = seen_of(it.e, dm.rep, causal, it.row0 + it.rows - 1);
  it.tiles = (it.most + Shape::kSlots - 1) / Shape::kSlots;
  if (tid == 0) {
    mbar_init(&sh.query, 128 * kTiles);
    for (int i = 0; i < Shape::kStages; ++i) {
      mbar_init(&sh.full[i], kCopyThreads);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.scores[i], 1);
      mbar_init(&sh.weights[i], 128);
    }
    mbar_init(&sh.sums, 1);
    mbar_init(&sh.done, 1);
    sh.gave_up = sh.unclean = 0;
    fence_barrier_init();
  }
  if (warp == 0) tmem_alloc(&sh.tmem, 512);
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  const uint32_t tmem = sh.tmem;
  const TensorWaiter wait{&sh.gave_up, st.err};
  const int t = warp >> 2;
  float m = -INFINITY, l = 0.f;
  const int r = it.row0 + tid, token = r / dm.rep, hq = it.kh * dm.rep + r % dm.rep;
  const bool live = tid < it.rows;   // of the threads that own rows
  if (warp < 4 * kTiles) {
    const uint4* src = live ? reinterpret_cast<const uint4*>(q.p + ((int64_t)(it.e.tok0 + token) * q.st + hq * q.sh) * 2) : nullptr;
    float mul = store_query<D, FMT != EPIKV_CACHE_BF16>(smem_u32(smem + t * Shape::kQuery), 128 * 128, tid & 127, src);
    if constexpr (FMT != EPIKV_CACHE_BF16) mul *= head_scale(st, dm, 0, layer, it.kh);
    fence_proxy_async_smem();
    mbar_arrive_one(&sh.query);
    // rows that are not there see all slots of the tiles: their queries are 0
    soften<D, FMT, kTiles>(sh, wait, it.tiles, live ? seen_of(it.e, dm.rep, causal, r) : INT_MAX, c * mul,
                           tmem + ((uint32_t)(warp & 3) << 21), t, &m, &l);
  } else if (warp == 8) {
    if (tid == 256 && it.tiles > 0)
      issue_products<D, FMT, kTiles>(smem_u32(smem), smem_u32(ring), sh, wait, it.tiles, tmem);
    __syncwarp();
  } else if (warp > 8) {
    copy_tiles<D, FMT, kTiles>(ring, sh, wait, dm, it, kv, layer, st.err, tid - 288);
  }
  if (warp < 4 * kTiles && it.tiles > 0) wait(&sh.done, 0);
  tensor_fence_after();
  __syncthreads();
  if (warp < 4 * kTiles) {
    float mul = l == 0.f ? 0.f : 1.f / l;
    if constexpr (FMT != EPIKV_CACHE_BF16) mul *= head_scale(st, dm, 1, layer, it.kh);
    const uint32_t o = tmem + ((uint32_t)(warp & 3) << 21) + 256 + t * 128;
    char* to = live ? out.p + ((int64_t)(it.e.tok0 + token) * out.st + hq * out.sh) * 2 : nullptr;
    const int upto = live && sh.unclean ? seen_of(it.e, dm.rep, causal, r) : 0;
#pragma unroll 1
    for (int i = 0; i < D; i += 32) {
      uint32_t y[32];
      if (it.tiles > 0) {
        tmem_load32(o + i, y);
        tmem_wait_load();
      }
#pragma unroll
      for (int u = 0; u < 32; ++u) y[u] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(y[u]) * mul);
      // what the copying warps took out of slots that not all rows see: an infinity is the output of the rows that see it
#pragma unroll 1
      for (int s = it.least; s < upto; ++s) {
        const int64_t at = kv_row_offset(kv, layer, it.e.seq, s, dm.T);
        if (at < 0) continue;
        const char* row = kv.base[1] + at * 2;
        if constexpr (FMT == EPIKV_CACHE_BF16) {
#pragma unroll
          for (int u = 0; u < 32; ++u) {
            const uint32_t v = *reinterpret_cast<const uint16_t*>(row + (it.kh * D + i + u) * 2);
            if ((v & 0x7f80u) == 0x7f80u) y[u] = __float_as_uint(__uint_as_float(y[u]) + __uint_as_float(v << 16));
          }
        } else {   // a scale of NaN
#pragma unroll
          for (int u = 0; u < 32; ++u)
            if (((uint8_t)row[scale_offset(dm, it.kh) + (i + u) / kQuantGroup] & 0x7f) == 0x7f) y[u] = 0x7fc00000u;
        }
      }
      if (live) {
#pragma unroll
        for (int u = 0; u < 32; u += 8)
          *reinterpret_cast<uint4*>(to + (i + u) * 2) =
              make_uint4(bf16_pair(__uint_as_float(y[u]), __uint_as_float(y[u + 1])),
                         bf16_pair(__uint_as_float(y[u + 2]), __uint_as_float(y[u + 3])),
                         bf16_pair(__uint_as_float(y[u + 4]), __uint_as_float(y[u + 5])),
                         bf16_pair(__uint_as_float(y[u + 6]), __uint_as_float(y[u + 7])));
      }
    }
    if (live && lse) {
      const float shift = FMT == EPIKV_CACHE_BF16 ? 0.f : 7.f;
      lse[(int64_t)(it.e.tok0 + token) * dm.Hq + hq] = l == 0.f ? -INFINITY : (m - shift + log2f(l)) * 0.69314718055994531f;
    }
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  if (warp == 0) tmem_free(tmem, 512);
}

template <int D, int kTiles>
constexpr int chunk_smem() {
  return kTiles * ChunkShape<D>::kQuery + ChunkShape<D>::kStages * ChunkShape<D>::kStage + 1024;
}

template <int D, int FMT, int kTiles>
cudaError_t run_chunk(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal, const Rows& q,
                      const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  static_assert(chunk_smem<D, kTiles>() + sizeof(ChunkShared<D, kTiles>) <= 227 * 1024, "shared memory");
  const int64_t blocks = ((int64_t)ba.max_new * dm.rep + 128 * kTiles - 1) / (128 * kTiles);
  return pdl_launch(chunk_kernel<D, FMT, kTiles>, dim3((unsigned)(blocks * dm.H), ba.n_seq), kChunkThreads,
                    chunk_smem<D, kTiles>(), stream, st, dm, layer, ba, causal, q, out, lse, kv,
                    dm.scale * 1.4426950408889634f);
}

template <int D, int FMT, int kTiles>
cudaError_t allow_chunk() {
  return cudaFuncSetAttribute(chunk_kernel<D, FMT, kTiles>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              chunk_smem<D, kTiles>());
}

template <int FMT>
cudaError_t prepare_format(int d) {
  if (d == 256) return allow_chunk<256, FMT, 1>();
  if (d == 128) {
    const cudaError_t e = allow_chunk<128, FMT, 1>();
    return e == cudaSuccess ? allow_chunk<128, FMT, 2>() : e;
  }
  const cudaError_t e = allow_chunk<64, FMT, 1>();
  return e == cudaSuccess ? allow_chunk<64, FMT, 2>() : e;
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

cudaError_t chunk_prepare(const AttnDims& dm) {
  return dm.fmt == EPIKV_CACHE_BF16 ? prepare_format<EPIKV_CACHE_BF16>(dm.d) : prepare_format<EPIKV_CACHE_E2M1>(dm.d);
}

cudaError_t launch_attention_chunk(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal,
                                   const Rows& q, const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  auto go = dm.fmt == EPIKV_CACHE_BF16 ? run_format<EPIKV_CACHE_BF16> : run_format<EPIKV_CACHE_E2M1>;
  return go(st, dm, layer, ba, causal, q, out, lse, kv, stream);
}

}  // namespace epikv
