// Shared by the cache operators (rotation, append, read-back, attention): the
// context's dimensions, where a batch entry's tokens are, and the 4-bit rows.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "kernels.h"

namespace epikv {

constexpr int kQuantGroup = 16;  // channels that share one E4M3 scale

struct AttnDims {
  int S, T, max_new, L, Hq, H, d, rep;
  int fmt;         // EPIKV_CACHE_*
  int units;       // 2-byte units of one token's row
  float scale;     // of the scores
};

struct AttnState {
  int32_t* err;           // [1] sticky device error word
  const float* kv_scale;  // [2][L][H] or null (the caller's)
  float* part;            // partial results of split rows
  int32_t* plan;          // [max_seqs + 1] tiles before each entry
};

// A batch as the entry points take it.
struct Batch {
  const int32_t* seq_ids;
  const int32_t* cu_new;
  const int32_t* len;
  int64_t len_stride;
  int n_seq, max_new;
};

struct Rows {
  char* p;
  int64_t st, sh;  // elements
};

struct RopeDev {
  const float2* table;  // [n_pos][dim / 2] cos, sin
  int n_pos, dim, layout;
};

struct Entry {
  int seq, tok0, n, len;
};

// Entry b of the batch; false (and the error word set) if it cannot be taken.
// `grow`: its new tokens need slots behind the held ones.
__device__ __forceinline__ bool batch_entry(const Batch& ba, const AttnDims& dm, int b, bool grow, int32_t* err,
                                            Entry* e) {
  e->tok0 = ba.cu_new[b];
  e->n = ba.cu_new[b + 1] - e->tok0;
  e->seq = ba.seq_ids[b];
  e->len = ba.len[(int64_t)b * ba.len_stride];
  if (e->tok0 < 0 || e->n < 0 || e->n > ba.max_new || (unsigned)e->seq >= (unsigned)dm.S) {
    set_error(err, EPIKV_DEV_BATCH);
    return false;
  }
  if (e->len < 0 || (int64_t)e->len + (grow ? e->n : 0) > dm.T) {
    set_error(err, EPIKV_DEV_CAPACITY);
    return false;
  }
  return true;
}

// Scale bytes of head h in a 4-bit row; its codes stand at h * d / 2.
__host__ __device__ __forceinline__ int scale_offset(const AttnDims& dm, int h) {
  return dm.H * dm.d / 2 + h * (dm.d / kQuantGroup);
}

__device__ __forceinline__ float head_scale(const AttnState& st, const AttnDims& dm, int which, int layer, int h) {
  return st.kv_scale ? st.kv_scale[((int64_t)which * dm.L + layer) * dm.H + h] : 1.f;
}

// Eight E2M1 codes (channel i in bits 4i..4i+3) as four half pairs.
__device__ __forceinline__ void e2m1x8_to_half2(uint32_t w, uint32_t (&r)[4]) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
}

// Two E4M3 values (low byte first) as a half pair.
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint16_t v) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(v));
  return r;
}

// Two floats as E2M1 codes (a in the low four bits), to nearest even, saturating.
__device__ __forceinline__ uint32_t float2_to_e2m1x2(float a, float b) {
  uint32_t r;
  asm("{\n\t.reg .b8 v;\n\tcvt.rn.satfinite.e2m1x2.f32 v, %2, %1;\n\tmov.b32 %0, {v, 0, 0, 0};\n\t}"
      : "=r"(r) : "f"(a), "f"(b));
  return r;
}

// A non-negative float as an E4M3 byte, to nearest even, saturating at 448; NaN stays NaN.
__device__ __forceinline__ uint32_t float_to_e4m3(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
  return r & 0xffu;
}

cudaError_t launch_rope_table(const epikv_rope_config& c, int n_pos, float* table, cudaStream_t stream);
cudaError_t launch_rope(const AttnState& st, const AttnDims& dm, int n_tokens, int n_heads, const Rows& x,
                        const Rows& out, int type, const int32_t* pos, const RopeDev& rope, bool inverse,
                        cudaStream_t stream);
cudaError_t launch_append(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, const int32_t* pos,
                          const Rows& q, const Rows& q_out, const Rows& k, const Rows& v, const RopeDev& rope,
                          const KvDev& kv, cudaStream_t stream);
cudaError_t launch_cache_read(const AttnState& st, const AttnDims& dm, int layer, int n_rows, const int32_t* seqs,
                              const int32_t* slots, const Rows& k, const Rows& v, const KvDev& kv,
                              cudaStream_t stream);
cudaError_t launch_attention(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, bool causal,
                             const Rows& q, const Rows& out, float* lse, const KvDev& kv, cudaStream_t stream);
size_t attention_part_floats(const AttnDims& dm);
cudaError_t attention_prepare(const AttnDims& dm, bool* runs);

}  // namespace epikv
