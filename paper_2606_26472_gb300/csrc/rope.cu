// Rotary positions, appending to the cache with the rotation on the way, and
// reading cache rows back.
//
// The rotation turns each pair (a, b) of a head's channels by its position's
// angle for that pair's frequency: a' = a cos - b sin, b' = b cos + a sin.  The
// cosines come from a table (made once, in 64 bits: an angle formed in 32 bits
// is off by 0.03 radians at position 10^6), the products and sums are rounded
// one by one in 32 bits, so a 4-bit code never depends on how a compiler
// contracts them.
//
// A thread takes a unit of 2 V channels that the rotation keeps among
// themselves (V and V channels half a rotated range apart, or 2 V neighbours),
// loads the unit's V cosines and sines once and then turns that unit of several
// heads, so in place works and the table is read once per token and not per
// head.  V = 8 (16-byte accesses) where the rotated range allows it, else 1.
//
// Reading and writing bounds all of it: 8,192 tokens x 40 heads of 128 rotated
// in 31.6 us (5.4 TB/s), four prompts of 517 to 4,099 tokens (32 + 8 + 8 heads)
// appended in 45.0 us (5.1 TB/s).  Into a 4-bit cache the quantisation does: 32
// x 128 tokens 20 us, 890 instructions a warp.  One token an entry is a launch
// and a chain of four reads (lengths, block, position's row, rows): 5.5 us.  With
// V = 1, for a rotated range that 16 does not divide, heads go by single
// elements: 8,192 x 40 heads 48 us, the four prompts 69 us.
#include "attn.cuh"

namespace epikv {
namespace {

constexpr int kBlock = 128;

// V values as they stand in memory: what a thread has in flight takes no more registers than that.
template <typename T, int V>
struct Raw {
  T v;
};
template <typename T>
struct Raw<T, 8> {
  uint4 v[sizeof(T) / 2];
};

template <typename T, int V>
__device__ __forceinline__ void load_raw(const T* p, Raw<T, V>& r) {
  if constexpr (V == 1) {
    r.v = *p;
  } else {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = reinterpret_cast<const uint4*>(p)[i];
  }
}

template <typename T, int V>
__device__ __forceinline__ void to_float(const Raw<T, V>& r, float* f) {
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) f[0] = r.v;
    else if constexpr (__is_same(T, __half)) f[0] = __half2float(r.v);
    else f[0] = __bfloat162float(r.v);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f[4 * i] = __uint_as_float(r.v[i].x);
      f[4 * i + 1] = __uint_as_float(r.v[i].y);
      f[4 * i + 2] = __uint_as_float(r.v[i].z);
      f[4 * i + 3] = __uint_as_float(r.v[i].w);
    }
  } else if constexpr (__is_same(T, __half)) {
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      f[2 * i] = v.x;
      f[2 * i + 1] = v.y;
    }
  } else {
    unpack8(r.v[0], f);
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <typename T, int V>
__device__ __forceinline__ void store_v(T* p, const float* f) {
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) *p = f[0];
    else if constexpr (__is_same(T, __half)) *p = __float2half_rn(f[0]);
    else *p = __float2bfloat16_rn(f[0]);
  } else if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (__is_same(T, __half)) {
        const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
      } else {
        w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
      }
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// First channels of unit u's two runs of V channels.
template <int V>
__device__ __forceinline__ int2 unit_channels(int u, int dim, int layout) {
  if (u < dim / (2 * V) && layout == EPIKV_ROPE_HALF) return make_int2(u * V, dim / 2 + u * V);
  return make_int2(2 * u * V, 2 * u * V + V);
}

template <int V>
__device__ __forceinline__ void load_angles(const RopeDev& r, int pos, int u, float sign, float* c, float* s) {
  const float2* t = r.table + (int64_t)pos * (r.dim / 2) + u * V;
  if constexpr (V == 1) {
    const float2 v = __ldg(t);
    c[0] = v.x;
    s[0] = sign * v.y;
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(t) + i);
      c[2 * i] = v.x; s[2 * i] = sign * v.y;
      c[2 * i + 1] = v.z; s[2 * i + 1] = sign * v.w;
    }
  }
}

// a cos - b sin and b cos + a sin, every operation rounded on its own.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = x;
}

template <int V>
__device__ __forceinline__ void turn_unit(float* a, float* b, const float* c, const float* s, int layout) {
  if (V == 1 || layout == EPIKV_ROPE_HALF) {
#pragma unroll
    for (int i = 0; i < V; ++i) turn(a[i], b[i], c[i], s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      turn(a[2 * i], a[2 * i + 1], c[i], s[i]);
      turn(b[2 * i], b[2 * i + 1], c[V / 2 + i], s[V / 2 + i]);
    }
  }
}

__global__ void rope_table_kernel(epikv_rope_config c, int n_pos, float2* table) {
  const int half = c.dim / 2;
  const int64_t n = (int64_t)n_pos * half;
  for (int64_t k = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; k < n; k += (int64_t)gridDim.x * blockDim.x) {
    const int pos = (int)(k / half), i = (int)(k - (int64_t)pos * half);
    double theta = c.theta;
    if (c.scaling == EPIKV_ROPE_NTK) theta *= pow((double)c.factor, (double)c.dim / (c.dim - 2));
    double freq = pow(theta, -2.0 * i / c.dim);
    if (c.scaling == EPIKV_ROPE_LINEAR) freq /= c.factor;
    if (c.scaling == EPIKV_ROPE_BYPARTS) {
      const double rot = c.original * freq / 6.283185307179586476925287;
      const double g = fmin(fmax((rot - c.low) / ((double)c.high - c.low), 0.0), 1.0);
      freq *= (1.0 - g) / c.factor + g;
    }
    double s, co;
    sincos(pos * freq, &s, &co);
    table[k] = make_float2((float)(co * c.magnitude), (float)(s * c.magnitude));
  }
}

// kBatch heads of a thread are in flight; their loads go out before the position and the table's row are known.  More of
// them, or registers held down for more CTAs, cost occupancy or loads in flight: 8,192 x 40 heads of bf16 two 32.4, three
// 31.7 us (held to 72 registers 34.1); 4,096 x 40 heads of 32-bit data one 27.5, two 30.5 us.
template <typename T, int V>
__global__ void __launch_bounds__(kBlock) rope_kernel(int32_t* err, Rows x, Rows y, const int32_t* __restrict__ pos,
                                                      RopeDev r, int n_tokens, int heads, int d, float sign) {
  constexpr int kBatch = sizeof(T) == 4 ? 1 : 3;
  const int U = d / (2 * V), slots = kBlock / U;  // units of a head; heads that the block takes at once
  const int u = threadIdx.x % U, slot = threadIdx.x / U;
  const int tpb = max(1, slots / heads);          // tokens of this block
  const int step = heads < slots ? heads : slots;
  if (slot >= tpb * step) return;
  const int64_t token = (int64_t)blockIdx.x * tpb + slot / step;
  if (token >= n_tokens) return;
  const bool turned = u < r.dim / (2 * V);
  const int2 ch = unit_channels<V>(u, r.dim, r.layout);
  const T* src = reinterpret_cast<const T*>(x.p) + token * x.st;
  T* dst = reinterpret_cast<T*>(y.p) + token * y.st;
  float c[V], s[V];
  int p = 0;
  bool first = true;
  pdl_wait();
  for (int h0 = slot % step; h0 < heads; h0 += step * kBatch) {
    Raw<T, V> a[kBatch], b[kBatch];
    if (first) p = pos[token];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int h = h0 + k * step;
      if (h < heads) {
        load_raw<T, V>(src + h * x.sh + ch.x, a[k]);
        load_raw<T, V>(src + h * x.sh + ch.y, b[k]);
      }
    }
    if (first) {
      if ((unsigned)p >= (unsigned)r.n_pos) {
        set_error(err, EPIKV_DEV_POSITION);
        return;
      }
      if (turned) load_angles<V>(r, p, u, sign, c, s);
      first = false;
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int h = h0 + k * step;
      if (h < heads) {
        float fa[V], fb[V];
        to_float<T, V>(a[k], fa);
        to_float<T, V>(b[k], fb);
        if (turned) turn_unit<V>(fa, fb, c, s, r.layout);
        store_v<T, V>(dst + h * y.sh + ch.x, fa);
        store_v<T, V>(dst + h * y.sh + ch.y, fb);
      }
    }
  }
}

// ------------------------------------------------------------------ append

// Sixteen values in 4 bits: their codes (8 bytes) and scale.  Without a head scale the values are bf16, and a quotient
// needs no division: x has 8 significant bits, a boundary between two codes times the scale 7, so x / scale is such a
// boundary or at least 2^-8 of it away.  The product with the rounded reciprocal, rounded to 12 bits, is then the boundary
// itself or on the same side.  (32 x 128 tokens of 8 x 128, with the queries and the read-back: 33.7 instead of 35.0 us when
// it was taken in, 30.9 with what came later.)
__device__ __forceinline__ uint2 quantize16(const float* x, float g, uint32_t* scale) {
  float y[16];
  float top = 0.f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    y[i] = g == 1.f ? x[i] : __fdiv_rn(x[i], g);
    nan |= y[i] != y[i];
    top = fmaxf(top, fabsf(y[i]));
  }
  if (nan) {
    *scale = 0x7f;  // E4M3's NaN: the group reads as NaN
    return make_uint2(0, 0);
  }
  *scale = float_to_e4m3(fminf(__fdiv_rn(top, 6.f), 448.f));
  const uint32_t h = e4m3x2_to_half2((uint16_t)*scale);
  const float s = __half2float(__ushort_as_half((unsigned short)(h & 0xffffu)));
  uint32_t w[2] = {0, 0};
  if (s > 0.f) {
    float z[16];
    if (g == 1.f) {
      const float r = __frcp_rn(s);
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = __uint_as_float((__float_as_uint(y[i] * r) + 0x800u) & ~0xfffu);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = __fdiv_rn(y[i], s);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4] |= float2_to_e2m1x2(z[2 * i], z[2 * i + 1]) << (8 * (i % 4));
  }
  return make_uint2(w[0], w[1]);
}

// Sixteen channels of a key or a value and, for a half layout whose halves are whole runs of 16, their partners.
struct Run16 {
  Raw<__nv_bfloat16, 8> x[2], z[2];
};
__device__ __forceinline__ bool whole_partners(const RopeDev& r, int c0) {
  return r.layout == EPIKV_ROPE_HALF && r.dim % 32 == 0 && c0 < r.dim;
}
__device__ __forceinline__ void load16(const __nv_bfloat16* k, int c0, bool partners, const RopeDev& r, Run16& run) {
  load_raw<__nv_bfloat16, 8>(k + c0, run.x[0]);
  load_raw<__nv_bfloat16, 8>(k + c0 + 8, run.x[1]);
  if (partners) {
    const int at = c0 < r.dim / 2 ? c0 + r.dim / 2 : c0 - r.dim / 2;
    load_raw<__nv_bfloat16, 8>(k + at, run.z[0]);
    load_raw<__nv_bfloat16, 8>(k + at + 8, run.z[1]);
  }
}

// Channels c0 .. c0+15 of a key, rotated and rounded to bf16 (kept as floats).
__device__ __forceinline__ void turned16(const Run16& run, const __nv_bfloat16* k, int c0, const RopeDev& r, int pos,
                                         float* x) {
  to_float<__nv_bfloat16, 8>(run.x[0], x);
  to_float<__nv_bfloat16, 8>(run.x[1], x + 8);
  if (c0 >= r.dim) return;
  const float2* t = r.table + (int64_t)pos * (r.dim / 2);
  const int half = r.dim / 2;
  if (r.layout == EPIKV_ROPE_INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + 2 * i < r.dim) {
        const float2 a = __ldg(t + c0 / 2 + i);
        turn(x[2 * i], x[2 * i + 1], a.x, a.y);
        x[2 * i] = __bfloat162float(__float2bfloat16_rn(x[2 * i]));
        x[2 * i + 1] = __bfloat162float(__float2bfloat16_rn(x[2 * i + 1]));
      }
    return;
  }
  float z[16];
  if (whole_partners(r, c0)) {
    to_float<__nv_bfloat16, 8>(run.z[0], z);
    to_float<__nv_bfloat16, 8>(run.z[1], z + 8);
    // all on one side of the pairs: a cos - b sin of the first half's, b cos + a sin of the second's
    const float4* t4 = reinterpret_cast<const float4*>(t + (c0 < half ? c0 : c0 - half));
    const bool low = c0 < half;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 a = __ldg(t4 + i);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float c = y ? a.z : a.x, s = y ? a.w : a.y;
        const float p = __fmul_rn(x[2 * i + y], c), q = __fmul_rn(z[2 * i + y], s);
        x[2 * i + y] = __bfloat162float(__float2bfloat16_rn(low ? __fsub_rn(p, q) : __fadd_rn(p, q)));
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int c = c0 + i;
    if (c < r.dim) {
      const float2 a = __ldg(t + (c < half ? c : c - half));
      const float other = __bfloat162float(k[c < half ? c + half : c - half]);
      float lo = c < half ? x[i] : other, hi = c < half ? other : x[i];
      turn(lo, hi, a.x, a.y);
      x[i] = __bfloat162float(__float2bfloat16_rn(c < half ? lo : hi));
    }
  }
}

// One block a token.  The queries (and, into a bf16 cache, the keys and values)
// go by units; into a 4-bit cache a thread takes 16 channels that share a scale.
template <int V, int kFmt>
__global__ void __launch_bounds__(kBlock) append_kernel(AttnState st, AttnDims dm, int layer, Batch ba,
                                                        const int32_t* __restrict__ pos, Rows q, Rows qo, Rows kr,
                                                        Rows vr, RopeDev r, KvDev kv) {
  constexpr int kBatch = 3;
  using bf = __nv_bfloat16;
  const int b = blockIdx.y, i = blockIdx.x;
  const int nq = q.p ? dm.Hq : 0;
  const int n = nq + (kFmt == EPIKV_CACHE_BF16 ? 2 * dm.H : 0);
  const int U = dm.d / (2 * V), slots = kBlock / U;
  const int u = threadIdx.x % U, slot = threadIdx.x / U;
  const bool turned = u < r.dim / (2 * V);
  const int2 ch = unit_channels<V>(u, r.dim, r.layout);
  Entry e;
  pdl_wait();
  const int p0 = r.dim ? pos[b] : 0;
  if (!batch_entry(ba, dm, b, true, st.err, &e) || i >= e.n) return;
  const int64_t token = (int64_t)e.tok0 + i;
  const bf* q0 = reinterpret_cast<const bf*>(q.p) + token * q.st;
  const bf* k0 = reinterpret_cast<const bf*>(kr.p) + token * kr.st;
  const bf* v0 = reinterpret_cast<const bf*>(vr.p) + token * vr.st;
  // the first heads' loads go out with those of the position's row and the slot's block
  Raw<bf, V> a[kBatch], z[kBatch];
  auto load = [&](int h0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int h = h0 + k * slots;
      if (h < n) {
        const bf* src = h < nq ? q0 + h * q.sh : h < nq + dm.H ? k0 + (h - nq) * kr.sh : v0 + (h - nq - dm.H) * vr.sh;
        load_raw<bf, V>(src + ch.x, a[k]);
        load_raw<bf, V>(src + ch.y, z[k]);
      }
    }
  };
  if (slot < slots) load(slot);
  const int p = (int)((unsigned)p0 + (unsigned)i);
  if (r.dim && (p0 < 0 || p0 >= r.n_pos || i >= r.n_pos - p0)) {
    set_error(st.err, EPIKV_DEV_POSITION);
    return;
  }
  float c[V], s[V];
  if (turned) load_angles<V>(r, p, u, 1.f, c, s);
  const int64_t row = kv_row_offset(kv, layer, e.seq, e.len + i, dm.T);
  if (row < 0) {
    set_error(st.err, EPIKV_DEV_SLOT);
    return;
  }
  if (slot < slots)
    for (int h0 = slot; h0 < n; h0 += slots * kBatch) {
      if (h0 != slot) load(h0);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int h = h0 + k * slots;
        if (h < n) {
          float fa[V], fz[V];
          to_float<bf, V>(a[k], fa);
          to_float<bf, V>(z[k], fz);
          if (turned && h < nq + dm.H) turn_unit<V>(fa, fz, c, s, r.layout);
          bf* dst = h < nq ? reinterpret_cast<bf*>(qo.p) + token * qo.st + h * qo.sh
                    : h < nq + dm.H ? reinterpret_cast<bf*>(kv.base[0]) + row + (int64_t)(h - nq) * dm.d
                                    : reinterpret_cast<bf*>(kv.base[1]) + row + (int64_t)(h - nq - dm.H) * dm.d;
          store_v<bf, V>(dst + ch.x, fa);
          store_v<bf, V>(dst + ch.y, fz);
        }
      }
    }
  // 4 bits: job j is 16 channels of a head of K (the first H * G jobs) or V
  const int G = dm.d / kQuantGroup, jobs = kFmt == EPIKV_CACHE_E2M1 ? 2 * dm.H * G : 0;
  for (int j = threadIdx.x; j < jobs; j += kBlock) {
    const int which = j >= dm.H * G, h = (which ? j - dm.H * G : j) / G, g = j % G;
    float x[16];
    Run16 run;
    if (which == 0) {
      load16(k0 + h * kr.sh, g * 16, whole_partners(r, g * 16), r, run);
      turned16(run, k0 + h * kr.sh, g * 16, r, p, x);
    } else {
      load16(v0 + h * vr.sh, g * 16, false, r, run);
      to_float<bf, 8>(run.x[0], x);
      to_float<bf, 8>(run.x[1], x + 8);
    }
    uint32_t scale;
    const uint2 code = quantize16(x, head_scale(st, dm, which, layer, h), &scale);
    char* dst = (which ? kv.base[1] : kv.base[0]) + row * 2;
    *reinterpret_cast<uint2*>(dst + h * (dm.d / 2) + g * 8) = code;
    dst[scale_offset(dm, h) + g] = (char)scale;
  }
}

// ------------------------------------------------------------------ read-back

// A thread takes 16 channels of one head of a row (4,096 rows of 8 x 128 out of 4 bits: 11 us, where their 21 MB would take
// 3, for the latency of its reads: the sequence and slot, the block, the row).
__global__ void __launch_bounds__(kBlock) cache_read_kernel(AttnState st, AttnDims dm, int layer, int n_rows,
                                                            const int32_t* __restrict__ seqs,
                                                            const int32_t* __restrict__ slots, Rows k, Rows v,
                                                            KvDev kv) {
  const int G = dm.d / 16, per = dm.H * G;
  const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (j >= (int64_t)n_rows * per) return;
  pdl_wait();
  const int64_t i = j / per;
  const int h = (int)(j - i * per) / G, g = (int)(j - i * per) % G;
  const int seq = seqs[i];
  const int64_t row = (unsigned)seq < (unsigned)dm.S ? kv_row_offset(kv, layer, seq, slots[i], dm.T) : -1;
  if (row < 0) {
    set_error(st.err, EPIKV_DEV_SLOT);
    return;
  }
  using bf = __nv_bfloat16;
  for (int w = 0; w < 2; ++w) {
    char* to = w ? v.p : k.p;
    if (!to) continue;
    bf* dst = reinterpret_cast<bf*>(to) + i * (w ? v.st : k.st) + h * (w ? v.sh : k.sh) + g * 16;
    const char* src = (w ? kv.base[1] : kv.base[0]) + row * 2;
    if (dm.fmt == EPIKV_CACHE_BF16) {
      const uint4* s = reinterpret_cast<const uint4*>(src + (h * dm.d + g * 16) * 2);
      reinterpret_cast<uint4*>(dst)[0] = s[0];
      reinterpret_cast<uint4*>(dst)[1] = s[1];
      continue;
    }
    const uint2 code = *reinterpret_cast<const uint2*>(src + h * (dm.d / 2) + g * 8);
    const uint32_t sc = e4m3x2_to_half2((uint8_t)src[scale_offset(dm, h) + g]);
    const float scale = __half2float(__ushort_as_half((unsigned short)(sc & 0xffffu)));
    const float gs = head_scale(st, dm, w, layer, h);
    uint32_t hw[8];
    e2m1x8_to_half2(code.x, reinterpret_cast<uint32_t(&)[4]>(hw[0]));
    e2m1x8_to_half2(code.y, reinterpret_cast<uint32_t(&)[4]>(hw[4]));
    float f[16];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&hw[c]));
      f[2 * c] = x.x * scale * gs;
      f[2 * c + 1] = x.y * scale * gs;
    }
    store_v<bf, 8>(dst, f);
    store_v<bf, 8>(dst + 8, f + 8);
  }
}

template <typename T>
cudaError_t rope_of(const AttnState& st, const AttnDims& dm, int n_tokens, int n_heads, const Rows& x, const Rows& y,
                    const int32_t* pos, const RopeDev& rope, float sign, cudaStream_t stream) {
  const bool vec = rope.dim % 16 == 0;
  const int slots = kBlock / (vec ? dm.d / 16 : dm.d / 2);
  const int tpb = slots / n_heads > 1 ? slots / n_heads : 1;
  const unsigned grid = (unsigned)(((int64_t)n_tokens + tpb - 1) / tpb);
  return vec ? pdl_launch(rope_kernel<T, 8>, grid, kBlock, 0, stream, st.err, x, y, pos, rope, n_tokens, n_heads,
                            dm.d, sign)
             : pdl_launch(rope_kernel<T, 1>, grid, kBlock, 0, stream, st.err, x, y, pos, rope, n_tokens, n_heads,
                            dm.d, sign);
}

}  // namespace

cudaError_t launch_rope_table(const epikv_rope_config& c, int n_pos, float* table, cudaStream_t stream) {
  const int64_t n = (int64_t)n_pos * (c.dim / 2);
  const int64_t want = (n + 255) / 256;
  rope_table_kernel<<<(unsigned)(want < 4096 ? want : 4096), 256, 0, stream>>>(c, n_pos,
                                                                              reinterpret_cast<float2*>(table));
  return cudaGetLastError();
}

cudaError_t launch_rope(const AttnState& st, const AttnDims& dm, int n_tokens, int n_heads, const Rows& x,
                        const Rows& y, int type, const int32_t* pos, const RopeDev& rope, bool inverse,
                        cudaStream_t stream) {
  const float sign = inverse ? -1.f : 1.f;
  if (type == EPIKV_TYPE_F32) return rope_of<float>(st, dm, n_tokens, n_heads, x, y, pos, rope, sign, stream);
  if (type == EPIKV_TYPE_F16) return rope_of<__half>(st, dm, n_tokens, n_heads, x, y, pos, rope, sign, stream);
  return rope_of<__nv_bfloat16>(st, dm, n_tokens, n_heads, x, y, pos, rope, sign, stream);
}

cudaError_t launch_append(const AttnState& st, const AttnDims& dm, int layer, const Batch& ba, const int32_t* pos,
                          const Rows& q, const Rows& qo, const Rows& k, const Rows& v, const RopeDev& rope,
                          const KvDev& kv, cudaStream_t stream) {
  const dim3 grid(ba.max_new, ba.n_seq);
  const bool vec = rope.dim % 16 == 0;
  const bool q4 = dm.fmt == EPIKV_CACHE_E2M1;
  auto kern = vec ? (q4 ? append_kernel<8, EPIKV_CACHE_E2M1> : append_kernel<8, EPIKV_CACHE_BF16>)
                  : (q4 ? append_kernel<1, EPIKV_CACHE_E2M1> : append_kernel<1, EPIKV_CACHE_BF16>);
  return pdl_launch(kern, grid, kBlock, 0, stream, st, dm, layer, ba, pos, q, qo, k, v, rope, kv);
}

cudaError_t launch_cache_read(const AttnState& st, const AttnDims& dm, int layer, int n_rows, const int32_t* seqs,
                              const int32_t* slots, const Rows& k, const Rows& v, const KvDev& kv,
                              cudaStream_t stream) {
  const int64_t n = (int64_t)n_rows * dm.H * (dm.d / 16);
  return pdl_launch(cache_read_kernel, (unsigned)((n + kBlock - 1) / kBlock), kBlock, 0, stream, st, dm, layer,
                      n_rows, seqs, slots, k, v, kv);
}

}  // namespace epikv
