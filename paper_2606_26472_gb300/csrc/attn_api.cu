// C ABI of the cache operators: argument validation and the context of
// epikv_rope, epikv_append, epikv_attention and epikv_cache_read.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include "attn.cuh"
#include "attn_plan.h"

using namespace epikv;

struct epikv_attn_ctx {
  AttnDims dm;
  AttnState st;
  cudaStream_t last_stream;
  bool attention_runs;   // false: this build's attention kernels cannot be launched; the other operators can
};

namespace {

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// A row as H' * d' units, d' a power of two up to 256 and H' at most 32, the
// shapes that the eviction calls take: 4-bit rows are padded until they are one.
bool cache_row(int H, int d, int fmt, int* heads, int* dim) {
  if (H < 1 || H > 32 || (d != 64 && d != 128 && d != 256)) return false;
  if (fmt == EPIKV_CACHE_BF16) {
    if (H * d > 2048) return false;
    *heads = H;
    *dim = d;
    return true;
  }
  if (fmt != EPIKV_CACHE_E2M1) return false;
  const int bytes = H * (d / 2 + d / kQuantGroup);
  for (int units = (bytes + 15) / 16 * 8; units <= 2048; units += 8) {
    int p = units & -units;
    if (p > 256) p = 256;
    if (units / p <= 32) {
      *heads = units / p;
      *dim = p;
      return true;
    }
  }
  return false;
}

bool make_attn_dims(const epikv_attn_config* c, AttnDims* d) {
  if (!c) return false;
  if (c->max_seqs < 1 || c->max_seqs > kMaxSeqs) return false;
  if (c->max_cache_tokens < 1 || c->max_cache_tokens > kMostSlots) return false;
  if (c->max_new_tokens < 1 || c->max_new_tokens > (1 << 20)) return false;
  if (c->num_layers < 1 || c->num_heads < 1 || c->num_heads > 1024) return false;
  int heads, dim;
  if (!cache_row(c->num_kv_heads, c->head_dim, c->cache_format, &heads, &dim)) return false;
  if (c->num_heads % c->num_kv_heads) return false;
  if (!(c->softmax_scale >= 0.f) || !(c->softmax_scale < INFINITY)) return false;
  if (c->kv_scale && c->cache_format != EPIKV_CACHE_E2M1) return false;
  memset(d, 0, sizeof(*d));
  d->S = c->max_seqs;
  d->T = c->max_cache_tokens;
  d->max_new = c->max_new_tokens;
  d->L = c->num_layers;
  d->Hq = c->num_heads;
  d->H = c->num_kv_heads;
  d->d = c->head_dim;
  d->rep = c->num_heads / c->num_kv_heads;
  d->fmt = c->cache_format;
  d->units = heads * dim;
  d->scale = c->softmax_scale > 0.f ? c->softmax_scale : (float)(1.0 / sqrt((double)c->head_dim));
  return true;
}

size_t carve(const AttnDims& d, AttnState* st, char* base) {
  size_t off = 0;
  auto take = [&](size_t bytes) -> void* {
    off = align_up(off, 256);
    void* p = base ? base + off : nullptr;
    off += bytes;
    return p;
  };
  memset(st, 0, sizeof(*st));
  st->err = (int32_t*)take(4);
  st->plan = (int32_t*)take(((size_t)d.S + 1) * 4);
  st->part = (float*)take(attention_part_floats(d) * 4);
  return align_up(off, 256);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

int type_bytes(int type) { return type == EPIKV_TYPE_F32 ? 4 : 2; }

bool valid_rows(const epikv_rows* r, Rows* out) {
  if (!r || !r->ptr || !aligned16(r->ptr) || r->type < EPIKV_TYPE_BF16 || r->type > EPIKV_TYPE_F32) return false;
  const int per16 = 16 / type_bytes(r->type);
  if (r->stride_token < 0 || r->stride_head < 0 || r->stride_token % per16 || r->stride_head % per16) return false;
  out->p = (char*)r->ptr;
  out->st = r->stride_token;
  out->sh = r->stride_head;
  return true;
}

bool valid_rope(const AttnDims& dm, const epikv_rope_view* r, RopeDev* out) {
  if (!r->table || !aligned16(r->table) || r->n_pos < 1 || r->dim < 2 || r->dim % 2 || r->dim > dm.d) return false;
  if (r->layout != EPIKV_ROPE_HALF && r->layout != EPIKV_ROPE_INTERLEAVED) return false;
  out->table = (const float2*)r->table;
  out->n_pos = r->n_pos;
  out->dim = r->dim;
  out->layout = r->layout;
  return true;
}

bool valid_cache(const AttnDims& dm, int layer, const epikv_kv_view* kv, KvDev* out) {
  if (layer < 0 || layer >= dm.L) return false;
  if (!kv || !kv->k || !kv->v || !aligned16(kv->k) || !aligned16(kv->v)) return false;
  if (kv->stride_token < dm.units || kv->stride_token % 8 || kv->stride_layer < 0 || kv->stride_layer % 8) return false;
  memset(out, 0, sizeof(*out));
  out->base[0] = (char*)kv->k;
  out->base[1] = (char*)kv->v;
  out->layout = kv->layout;
  out->stride_layer = kv->stride_layer;
  out->stride_token = kv->stride_token;
  if (kv->layout == EPIKV_LAYOUT_CONTIGUOUS) {
    if (kv->stride_seq < 0 || kv->stride_seq % 8) return false;
    out->stride_seq = kv->stride_seq;
    return true;
  }
  if (kv->layout != EPIKV_LAYOUT_PAGED) return false;
  if (!kv->block_table || kv->block_size < 1 || kv->max_blocks_per_seq < 1 || kv->num_blocks < 1) return false;
  if (kv->stride_block < 0 || kv->stride_block % 8 || kv->stride_table_layer < 0) return false;
  out->stride_block = kv->stride_block;
  out->table_stride_layer = kv->stride_table_layer;
  out->block_table = kv->block_table;
  out->max_blocks = kv->max_blocks_per_seq;
  out->block_size = kv->block_size;
  out->num_blocks = kv->num_blocks;
  return true;
}

epikv_status cuda_status(cudaError_t e) { return e == cudaSuccess ? EPIKV_OK : EPIKV_ECUDA; }

bool valid_batch(int32_t n_seq, const int32_t* seq_ids, const int32_t* cu_new, int32_t max_new, const int32_t* len,
                 int32_t len_stride, Batch* out) {
  if (!seq_ids || !cu_new || !len || len_stride < 1) return false;
  out->seq_ids = seq_ids;
  out->cu_new = cu_new;
  out->len = len;
  out->len_stride = len_stride;
  out->n_seq = n_seq;
  out->max_new = max_new;
  return true;
}

}  // namespace

extern "C" {

epikv_status epikv_cache_row(int32_t num_kv_heads, int32_t head_dim, int32_t cache_format, int32_t* heads,
                             int32_t* dim) {
  int h, d;
  if (!heads || !dim || !cache_row(num_kv_heads, head_dim, cache_format, &h, &d)) return EPIKV_EINVAL;
  *heads = h;
  *dim = d;
  return EPIKV_OK;
}

size_t epikv_attn_workspace_bytes(const epikv_attn_config* cfg) {
  AttnDims dm;
  if (!make_attn_dims(cfg, &dm)) return 0;
  AttnState st;
  return carve(dm, &st, nullptr);
}

epikv_status epikv_attn_init(epikv_attn_ctx** out, const epikv_attn_config* cfg, void* d_workspace,
                             size_t workspace_bytes, cudaStream_t stream) {
  AttnDims dm;
  if (!out || !make_attn_dims(cfg, &dm) || !d_workspace || ((uintptr_t)d_workspace & 255u)) return EPIKV_EINVAL;
  *out = nullptr;
  if (workspace_bytes < epikv_attn_workspace_bytes(cfg)) return EPIKV_EINVAL;
  epikv_attn_ctx* ctx = (epikv_attn_ctx*)calloc(1, sizeof(epikv_attn_ctx));
  if (!ctx) return EPIKV_EINVAL;
  ctx->dm = dm;
  carve(dm, &ctx->st, (char*)d_workspace);
  ctx->st.kv_scale = cfg->kv_scale;
  ctx->last_stream = stream;
  cudaError_t e = attention_prepare(dm, &ctx->attention_runs);
  if (e == cudaSuccess) e = cudaMemsetAsync(ctx->st.err, 0, 4, stream);
  if (e != cudaSuccess) {
    free(ctx);
    return EPIKV_ECUDA;
  }
  *out = ctx;
  return EPIKV_OK;
}

epikv_status epikv_rope_table(const epikv_rope_config* cfg, int32_t n_pos, float* d_table, cudaStream_t stream) {
  if (!cfg || n_pos < 1 || !d_table || !aligned16(d_table)) return EPIKV_EINVAL;
  if (cfg->dim < 2 || cfg->dim % 2 || cfg->dim > 256 || !(cfg->theta > 1.f) || !(cfg->theta < INFINITY))
    return EPIKV_EINVAL;
  if (cfg->scaling < EPIKV_ROPE_PLAIN || cfg->scaling > EPIKV_ROPE_BYPARTS) return EPIKV_EINVAL;
  if (cfg->scaling != EPIKV_ROPE_PLAIN && (!(cfg->factor >= 1.f) || !(cfg->factor < INFINITY))) return EPIKV_EINVAL;
  if (cfg->scaling == EPIKV_ROPE_NTK && cfg->dim < 4) return EPIKV_EINVAL;
  if (cfg->scaling == EPIKV_ROPE_BYPARTS &&
      (!(cfg->low >= 0.f) || !(cfg->high > cfg->low) || !(cfg->high < INFINITY) || cfg->original < 1))
    return EPIKV_EINVAL;
  if (!(fabsf(cfg->magnitude) < INFINITY)) return EPIKV_EINVAL;
  return cuda_status(launch_rope_table(*cfg, n_pos, d_table, stream));
}

epikv_status epikv_rope(epikv_attn_ctx* ctx, int32_t n_tokens, int32_t n_heads, const epikv_rows* x,
                        const epikv_rows* out, const int32_t* d_pos, const epikv_rope_view* rope, int32_t inverse,
                        cudaStream_t stream) {
  if (!ctx || n_tokens < 0 || n_heads < 0 || (inverse != 0 && inverse != 1)) return EPIKV_EINVAL;
  if (n_tokens == 0 || n_heads == 0) return EPIKV_OK;  // nothing to rotate
  Rows xr, yr;
  RopeDev rd;
  if (!valid_rows(x, &xr) || !valid_rows(out, &yr) || x->type != out->type || !d_pos || !rope ||
      !valid_rope(ctx->dm, rope, &rd))
    return EPIKV_EINVAL;
  ctx->last_stream = stream;
  return cuda_status(launch_rope(ctx->st, ctx->dm, n_tokens, n_heads, xr, yr, x->type, d_pos, rd, inverse, stream));
}

epikv_status epikv_append(epikv_attn_ctx* ctx, int32_t layer, int32_t n_seq, const int32_t* d_seq_ids,
                          const int32_t* d_cu_new, int32_t max_new, const int32_t* d_len, int32_t len_stride,
                          const int32_t* d_pos, const epikv_rows* q, const epikv_rows* q_out, const epikv_rows* k,
                          const epikv_rows* v, const epikv_rope_view* rope, const epikv_kv_view* kv,
                          cudaStream_t stream) {
  if (!ctx || n_seq < 0 || n_seq > ctx->dm.S || max_new < 0 || max_new > ctx->dm.max_new) return EPIKV_EINVAL;
  if (n_seq == 0 || max_new == 0) return EPIKV_OK;  // nothing to append
  Batch ba;
  if (!valid_batch(n_seq, d_seq_ids, d_cu_new, max_new, d_len, len_stride, &ba)) return EPIKV_EINVAL;
  Rows qr = {}, qo = {}, kr, vr;
  RopeDev rd = {};
  KvDev kd;
  if ((q == nullptr) != (q_out == nullptr)) return EPIKV_EINVAL;
  if (q && (!valid_rows(q, &qr) || !valid_rows(q_out, &qo) || q->type != EPIKV_TYPE_BF16 ||
            q_out->type != EPIKV_TYPE_BF16))
    return EPIKV_EINVAL;
  if (!valid_rows(k, &kr) || !valid_rows(v, &vr) || k->type != EPIKV_TYPE_BF16 || v->type != EPIKV_TYPE_BF16)
    return EPIKV_EINVAL;
  if (rope && (!d_pos || !valid_rope(ctx->dm, rope, &rd))) return EPIKV_EINVAL;
  if (!valid_cache(ctx->dm, layer, kv, &kd)) return EPIKV_EINVAL;
  ctx->last_stream = stream;
  return cuda_status(launch_append(ctx->st, ctx->dm, layer, ba, d_pos, qr, qo, kr, vr, rd, kd, stream));
}

epikv_status epikv_attention(epikv_attn_ctx* ctx, int32_t layer, int32_t n_seq, const int32_t* d_seq_ids,
                             const int32_t* d_cu_new, int32_t max_new, const int32_t* d_len, int32_t len_stride,
                             int32_t causal, const epikv_rows* q, const epikv_rows* out, float* d_lse,
                             const epikv_kv_view* kv, cudaStream_t stream) {
  if (!ctx || n_seq < 0 || n_seq > ctx->dm.S || max_new < 0 || max_new > ctx->dm.max_new ||
      (causal != 0 && causal != 1))
    return EPIKV_EINVAL;
  if (n_seq == 0 || max_new == 0) return EPIKV_OK;  // no queries
  Batch ba;
  Rows qr, yr;
  KvDev kd;
  if (!valid_batch(n_seq, d_seq_ids, d_cu_new, max_new, d_len, len_stride, &ba)) return EPIKV_EINVAL;
  if (!valid_rows(q, &qr) || !valid_rows(out, &yr) || q->type != EPIKV_TYPE_BF16 || out->type != EPIKV_TYPE_BF16)
    return EPIKV_EINVAL;
  if (((uintptr_t)d_lse & 3u) || !valid_cache(ctx->dm, layer, kv, &kd)) return EPIKV_EINVAL;
  if (!ctx->attention_runs) return EPIKV_ECUDA;
  ctx->last_stream = stream;
  return cuda_status(launch_attention(ctx->st, ctx->dm, layer, ba, causal, qr, yr, d_lse, kd, stream));
}

epikv_status epikv_cache_read(epikv_attn_ctx* ctx, int32_t layer, int32_t n_rows, const int32_t* d_seqs,
                              const int32_t* d_slots, const epikv_rows* k, const epikv_rows* v,
                              const epikv_kv_view* kv, cudaStream_t stream) {
  if (!ctx || n_rows < 0) return EPIKV_EINVAL;
  if (n_rows == 0) return EPIKV_OK;  // nothing to read
  Rows kr = {}, vr = {};
  KvDev kd;
  if (!d_seqs || !d_slots || (!k && !v)) return EPIKV_EINVAL;
  if (k && (!valid_rows(k, &kr) || k->type != EPIKV_TYPE_BF16)) return EPIKV_EINVAL;
  if (v && (!valid_rows(v, &vr) || v->type != EPIKV_TYPE_BF16)) return EPIKV_EINVAL;
  if (!valid_cache(ctx->dm, layer, kv, &kd)) return EPIKV_EINVAL;
  ctx->last_stream = stream;
  return cuda_status(launch_cache_read(ctx->st, ctx->dm, layer, n_rows, d_seqs, d_slots, kr, vr, kd, stream));
}

epikv_status epikv_attn_get_error(epikv_attn_ctx* ctx, int32_t* code) {
  if (!ctx) return EPIKV_EINVAL;
  int32_t v = 0;
  cudaError_t e = cudaStreamSynchronize(ctx->last_stream);
  if (e == cudaSuccess) e = cudaMemcpy(&v, ctx->st.err, 4, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && v != 0) e = cudaMemset(ctx->st.err, 0, 4);
  if (e != cudaSuccess) return EPIKV_ECUDA;
  if (code) *code = v;
  return v ? EPIKV_EDEVICE : EPIKV_OK;
}

void epikv_attn_destroy(epikv_attn_ctx* ctx) { free(ctx); }

}  // extern "C"
