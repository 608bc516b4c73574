// C entry points of the serving operators: argument checks (host only, before
// any device work), workspaces, launches.
#include "serve.h"

#include <algorithm>
#include <cmath>

#include "tensor_args.h"

using namespace pard;

namespace {

bool blocked(int dtype) { return dtype == PARD_E4M3 || dtype == PARD_E2M1; }

pard_status cache_check(const pard_kv_cache* c) {
  if (!c || c->n_pages < 1 || c->n_kv_heads < 1 || c->page_size < 16 || c->page_size > 4096 ||
      (c->page_size & (c->page_size - 1)) || !c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16))
    return PARD_ERR_ARG;
  if (c->dtype != PARD_BF16 && c->dtype != PARD_F16 && !blocked(c->dtype)) return PARD_ERR_UNSUPPORTED;
  if (blocked(c->dtype) && (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)))
    return PARD_ERR_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->n_kv_heads > 65535) return PARD_ERR_UNSUPPORTED;
  return PARD_OK;
}

pard_status batch_check(const pard_kv_batch* b, const pard_kv_cache* c) {
  if (!b || b->rows < 0 || b->n_seqs < 1 || b->max_pages < 1 || b->max_seq_rows < 0 || !b->page_table || !b->row_start ||
      !b->kv_len)
    return PARD_ERR_ARG;
  if (b->rows >= 1 << 30 || b->n_seqs > 1 << 20 || (int64_t)b->max_pages * c->page_size > 1 << 30)
    return PARD_ERR_UNSUPPORTED;
  return PARD_OK;
}

KvCacheView cache_view(const pard_kv_cache* c) {
  const bool scales = blocked(c->dtype);
  KvCacheView v{static_cast<char*>(c->k), static_cast<char*>(c->v), scales ? c->k_scale : nullptr, scales ? c->v_scale : nullptr,
                c->n_pages, c->n_kv_heads, 0};
  while ((1 << v.page_log2) < c->page_size) ++v.page_log2;
  return v;
}

KvBatchView batch_view(const pard_kv_batch* b, const pard_kv_cache* c) {
  return KvBatchView{b->page_table, b->row_start, b->kv_len, b->n_seqs, b->max_pages, (int)b->rows,
                     b->max_pages * c->page_size};
}

pard_status copy(bool write, const pard_kv_cache* cache, const pard_kv_batch* batch, int32_t dtype, const pard_heads* k,
                 const pard_heads* v, void* hip_stream) {
  pard_status st = cache_check(cache);
  if (st == PARD_OK) st = batch_check(batch, cache);
  if (st != PARD_OK) return st;
  const int size = elem_size(dtype), hd = cache->head_dim, nk = cache->n_kv_heads;
  if (!size) return PARD_ERR_UNSUPPORTED;
  if (!heads_ok(k, batch->rows, nk, hd, !write) || !heads_ok(v, batch->rows, nk, hd, !write) ||
      !aligned(k->data, size) || !aligned(v->data, size))
    return PARD_ERR_ARG;
  if (batch->rows == 0) return PARD_OK;
  if (!write && (!apart(k, v) || k->data == cache->k || k->data == cache->v || v->data == cache->k || v->data == cache->v))
    return PARD_ERR_ARG;
  bool vec = true;
  for (const pard_heads* t : {k, v})
    vec = vec && aligned(t->data, 16) && t->row_stride * size % 16 == 0 && t->head_stride * size % 16 == 0;
  const KvCopyArgs a{cache_view(cache), batch_view(batch, cache), view(k), view(v)};
  return status_of(launch_kv_copy(write, hd, dtype, cache->dtype, vec, a, reinterpret_cast<hipStream_t>(hip_stream)));
}

pard_status attn_check(const pard_kv_attn_args* a) {
  if (!a) return PARD_ERR_ARG;
  pard_status st = cache_check(a->cache);
  if (st == PARD_OK) st = batch_check(a->batch, a->cache);
  if (st != PARD_OK) return st;
  const int nk = a->cache->n_kv_heads;
  if (a->n_heads < 1 || a->n_heads % nk || !std::isfinite(a->scale) || a->window < 0 || a->sinks < 0) return PARD_ERR_ARG;
  if ((a->dtype != PARD_BF16 && a->dtype != PARD_F16) || (!blocked(a->cache->dtype) && a->cache->dtype != a->dtype))
    return PARD_ERR_UNSUPPORTED;
  // (pairs of a row and a head of a key head are numbered in 30 bits)
  if (a->n_heads / nk > 1024 || a->batch->rows * (a->n_heads / nk) >= 1 << 30) return PARD_ERR_UNSUPPORTED;
  return PARD_OK;
}

KvAttnArgs attn_args(const pard_kv_attn_args* a) {
  KvAttnArgs r{};
  r.cache = cache_view(a->cache);
  r.batch = batch_view(a->batch, a->cache);
  r.n_heads = a->n_heads;
  r.group = a->n_heads / a->cache->n_kv_heads;
  r.by_group = fast_div(r.group);
  r.window = std::min(a->window, 1 << 30);  // (positions with a page are below 2^30)
  r.sinks = std::min(a->sinks, 1 << 30);
  r.scale = a->scale;
  return r;
}

// The kernels read and write 16 bytes of a head at a time, and take strides in
// bytes of 32 bits.
constexpr int64_t kMaxStride = 0x7fffffff;
bool attn_heads_ok(const pard_heads* t, const pard_kv_attn_args* a, bool out) {
  return heads_ok(t, a->batch->rows, a->n_heads, a->cache->head_dim, out) && aligned(t->data, 16) &&
         t->row_stride % 8 == 0 && t->head_stride % 8 == 0 && t->row_stride <= kMaxStride && t->head_stride <= kMaxStride;
}

pard_status logits_check(const pard_logits_args* a) {
  if (!a || a->rows < 0 || a->vocab < 1 || a->n_seqs < 1) return PARD_ERR_ARG;
  const int size = elem_size(a->dtype);
  if (!size || a->rows >= 1 << 30 || a->vocab > 1 << 28) return PARD_ERR_UNSUPPORTED;
  if (a->rows == 0) return PARD_OK;
  if (!a->logits || !a->out || !aligned(a->logits, size) || !aligned(a->out, size)) return PARD_ERR_ARG;
  if (a->logits_stride < 0 || a->out_stride < 0 || (a->rows > 1 && (a->logits_stride < a->vocab || a->out_stride < a->vocab)))
    return PARD_ERR_ARG;
  if (a->rows > 1 && a->out == a->logits && a->out_stride != a->logits_stride) return PARD_ERR_ARG;
  if (!a->row_seq && a->rows > a->n_seqs) return PARD_ERR_ARG;
  if (a->tokens ? a->tokens_stride < 0 || !a->row_len : a->repetition || a->presence || a->frequency) return PARD_ERR_ARG;
  if (a->bias_start && (a->n_bias < 0 || (a->n_bias > 0 && (!a->bias_ids || !a->bias_values)))) return PARD_ERR_ARG;
  if (a->mask && (a->n_masks < 0 || a->mask_stride < 0 || (a->n_masks > 1 && a->mask_stride < (a->vocab + 31) / 32)))
    return PARD_ERR_ARG;
  return PARD_OK;
}

}  // namespace

extern "C" {

pard_status pard_kv_write(const pard_kv_cache* cache, const pard_kv_batch* batch, int32_t dtype, const pard_heads* k,
                          const pard_heads* v, void* hip_stream) {
  return copy(true, cache, batch, dtype, k, v, hip_stream);
}

pard_status pard_kv_read(const pard_kv_cache* cache, const pard_kv_batch* batch, int32_t dtype, const pard_heads* k,
                         const pard_heads* v, void* hip_stream) {
  return copy(false, cache, batch, dtype, k, v, hip_stream);
}

size_t pard_kv_attn_workspace_bytes(const pard_kv_attn_args* args) {
  return attn_check(args) == PARD_OK ? kv_attn_workspace(attn_args(args), args->cache->head_dim, args->batch->max_seq_rows) : 0;
}

pard_status pard_kv_attn(const pard_kv_attn_args* args, const pard_heads* q, const pard_heads* out, float* lse,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  const pard_status st = attn_check(args);
  if (st != PARD_OK) return st;
  if (!attn_heads_ok(q, args, false) || !attn_heads_ok(out, args, true)) return PARD_ERR_ARG;
  if (args->batch->rows == 0) return PARD_OK;
  if (!apart(q, out) || out->data == args->cache->k || out->data == args->cache->v) return PARD_ERR_ARG;
  KvAttnArgs r = attn_args(args);
  const size_t need = kv_attn_workspace(r, args->cache->head_dim, args->batch->max_seq_rows);
  if (!workspace || !aligned(workspace, 256)) return PARD_ERR_ARG;
  if (workspace_bytes < need) return PARD_ERR_NOMEM;
  r.q = view16(q);
  r.out = view16(out);
  r.lse = lse;
  r.work = workspace;
  return status_of(launch_kv_attn(args->cache->head_dim, args->dtype, args->cache->dtype, r, args->batch->max_seq_rows,
                                  reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t pard_logits_workspace_bytes(const pard_logits_args* args) {
  if (logits_check(args) != PARD_OK || !args->best) return 0;
  return align256((size_t)args->rows * logits_keys(args->vocab) * sizeof(uint64_t));
}

pard_status pard_logits_adjust(const pard_logits_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const pard_status st = logits_check(args);
  if (st != PARD_OK) return st;
  const pard_logits_args& a = *args;
  if (a.rows == 0) return PARD_OK;
  if (a.best && (!workspace || !aligned(workspace, 256))) return PARD_ERR_ARG;
  if (workspace_bytes < pard_logits_workspace_bytes(args)) return PARD_ERR_NOMEM;
  const LogitsArgs r{(int)a.rows, a.vocab, a.n_seqs, static_cast<const char*>(a.logits), a.logits_stride, static_cast<char*>(a.out),
                     a.out_stride, a.tokens, a.row_seq, a.row_len, a.prompt_len, a.tokens_stride, a.repetition, a.presence,
                     a.frequency, a.bias_start, a.bias_ids, a.bias_values, a.n_bias, a.mask, a.mask_stride, a.mask_row,
                     a.n_masks, a.best, static_cast<uint64_t*>(workspace), 0};
  return status_of(launch_logits_adjust(a.dtype, r, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
