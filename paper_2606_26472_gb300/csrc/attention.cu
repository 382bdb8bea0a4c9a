// Attention of new tokens' queries over the slots of the cache.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - max_j)
//
// in one pass over the slots with a running maximum and sum.
#include "attn.cuh"

namespace epikv {
namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ float row_value(const char* row, const AttnDims& dm, int h, int c, float gs) {
  if (dm.fmt == EPIKV_CACHE_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[h * dm.d + c]);
  const uint32_t byte = (uint8_t)row[h * (dm.d / 2) + c / 2];
  uint32_t hw[4];
  e2m1x8_to_half2(byte, hw);
  const uint32_t sc = e4m3x2_to_half2((uint8_t)row[scale_offset(dm, h) + c / kQuantGroup]);
  const uint32_t v = c & 1 ? hw[0] >> 16 : hw[0] & 0xffffu;
  return __half2float(__ushort_as_half((unsigned short)v)) * __half2float(__ushort_as_half((unsigned short)(sc & 0xffffu))) * gs;
}

// One block a (query head, token); its warps take every fourth slot.
template <int kPer>  // channels of a lane
__global__ void __launch_bounds__(32 * kWarps) attention_kernel(AttnState st, AttnDims dm, int layer, Batch ba,
                                                                int causal, Rows q, Rows out, float* lse, KvDev kv) {
  __shared__ float s_m[kWarps], s_l[kWarps], s_o[kWarps][kPer * 32];
  const int hq = blockIdx.x, b = blockIdx.z, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  Entry e;
  if (!batch_entry(ba, dm, b, causal, st.err, &e)) return;
  const float gk = head_scale(st, dm, 0, layer, hq / dm.rep), gv = head_scale(st, dm, 1, layer, hq / dm.rep);
  for (int i = blockIdx.y; i < e.n; i += gridDim.y) {
    const int64_t token = (int64_t)e.tok0 + i;
    const __nv_bfloat16* qp = reinterpret_cast<const __nv_bfloat16*>(q.p) + token * q.st + hq * q.sh;
    float qf[kPer], o[kPer];
#pragma unroll
    for (int c = 0; c < kPer; ++c) {
      qf[c] = __bfloat162float(qp[lane + 32 * c]) * dm.scale;
      o[c] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    const int n = e.len + (causal ? i + 1 : 0);
    for (int j = w; j < n; j += kWarps) {
      const int64_t row = kv_row_offset(kv, layer, e.seq, j, dm.T);
      if (row < 0) {
        set_error(st.err, EPIKV_DEV_SLOT);
        continue;
      }
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < kPer; ++c) s += qf[c] * row_value(kv.base[0] + row * 2, dm, hq / dm.rep, lane + 32 * c, gk);
      s = warp_sum(s);
      const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn;
      const float a = expf(m - base), p = expf(s - base);
      l = l * a + p;
#pragma unroll
      for (int c = 0; c < kPer; ++c)
        o[c] = o[c] * a + p * row_value(kv.base[1] + row * 2, dm, hq / dm.rep, lane + 32 * c, gv);
      m = mn;
    }
    if (lane == 0) {
      s_m[w] = m;
      s_l[w] = l;
    }
#pragma unroll
    for (int c = 0; c < kPer; ++c) s_o[w][lane + 32 * c] = o[c];
    __syncthreads();
    float top = -INFINITY, total = 0.f;
    for (int k = 0; k < kWarps; ++k) top = fmaxf(top, s_m[k]);
    const float base = top == -INFINITY ? 0.f : top;
    for (int k = 0; k < kWarps; ++k) total += s_l[k] * expf(s_m[k] - base);
    for (int c = threadIdx.x; c < dm.d; c += 32 * kWarps) {
      float v = 0.f;
      for (int k = 0; k < kWarps; ++k) v += s_o[k][c] * expf(s_m[k] - base);
      reinterpret_cast<__nv_bfloat16*>(out.p)[token * out.st + hq * out.sh + c] =
          __float2bfloat16_rn(total == 0.f ? 0.f : v / total);
    }
    if (lse && threadIdx.x == 0) lse[token * dm.Hq + hq] = total == 0.f ? -INFINITY : base + logf(total);
    __syncthreads();
  }
}

}  // namespace

size_t attention_part_floats(const AttnDims&) { return 0; }
cudaError_t attention_prepare(const AttnDims&) { return cudaSuccess; }

cudaError_t launch_attention(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal,
                             const Rows& q, const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream) {
  const dim3 grid(dm.Hq, ba.max_new < 65535 ? ba.max_new : 65535, ba.n_seq);
  auto kern = dm.d == 64 ? attention_kernel<2> : dm.d == 128 ? attention_kernel<4> : attention_kernel<8>;
  return plain_launch(kern, grid, 32 * kWarps, 0, stream, st, dm, layer, ba, (int)causal, q, out, lse, kv);
}

}  // namespace epikv
