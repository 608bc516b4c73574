// C entry points of the mask-token training operators: argument checks (host
// only, before any device work), workspaces, launches.
#include "tensor_args.h"

#include <algorithm>
#include <cmath>

using namespace pard;

namespace {

bool rope_spec_ok(const pard_rope_spec* s, int32_t n_pos) {
  if (!s || s->rot_dim < 2 || s->rot_dim > 1024 || s->rot_dim % 2 || n_pos < 1 || n_pos > (1 << 24)) return false;
  if (!(s->theta > 1.f) || !std::isfinite(s->theta)) return false;
  if (s->scaling == PARD_ROPE_PLAIN) return true;
  if (s->scaling < 0 || s->scaling > PARD_ROPE_YARN || !(s->factor >= 1.f) || !std::isfinite(s->factor)) return false;
  if (s->scaling == PARD_ROPE_LINEAR) return true;
  return s->low > 0.f && s->high > s->low && std::isfinite(s->high) && s->original_max_pos >= 1;
}

pard_status rope_check(const pard_rope_args* a) {
  if (!a) return PARD_ERR_ARG;
  if (a->rows < 0 || a->n_q < 1 || a->n_k < 0 || a->head_dim < 2 || a->head_dim > 1024 || a->rot_dim < 2 ||
      a->rot_dim > a->head_dim || a->rot_dim % 2 || a->n_pos < 1 || a->n_pos > (1 << 24) ||
      (a->layout != PARD_ROPE_HALF && a->layout != PARD_ROPE_INTERLEAVED) || !(a->eps >= 0.f) || !std::isfinite(a->eps))
    return PARD_ERR_ARG;
  if (a->n_k > 0 && !a->q_gain != !a->k_gain) return PARD_ERR_ARG;
  if (a->rows > 0 && (!a->positions || !a->table || !aligned(a->table, 16))) return PARD_ERR_ARG;
  if (!elem_size(a->dtype)) return PARD_ERR_UNSUPPORTED;
  if ((__int128)a->rows * ((int64_t)a->n_q + a->n_k) > 0x7fffffff) return PARD_ERR_UNSUPPORTED;
  return PARD_OK;
}

RopeArgs rope_args(const pard_rope_args* a) {
  RopeArgs r{};
  r.rows = (int)a->rows;
  r.n_q = a->n_q;
  r.n_k = a->n_k;
  r.hd = a->head_dim;
  r.rot = a->rot_dim;
  r.n_pos = a->n_pos;
  r.eps = a->eps;
  r.pos = a->positions;
  r.table = reinterpret_cast<const float2*>(a->table);
  r.q_gain = a->q_gain;
  r.k_gain = a->k_gain;
  return r;
}

pard_status attn_check(const pard_cod_attn_args* a) {
  if (!a || !a->plan || !a->plan->data || a->plan->rows < 0 || a->plan->n_samples < 1 || a->plan->n_tiles < 0 ||
      a->n_heads < 1 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads || !std::isfinite(a->scale))
    return PARD_ERR_ARG;
  if ((a->head_dim != 64 && a->head_dim != 128) || (a->dtype != PARD_BF16 && a->dtype != PARD_F16))
    return PARD_ERR_UNSUPPORTED;
  // (pairs of a sample and key head are numbered in 32 bits; a launch has fewer
  // than 2^32 threads, 256 to a workgroup)
  if (a->n_heads > 65535 || a->n_heads / a->n_kv_heads > 1024 ||
      (int64_t)a->plan->n_tiles * std::max(a->n_heads, 4 * a->n_kv_heads) >= 1 << 24)
    return PARD_ERR_UNSUPPORTED;
  return PARD_OK;
}

// The kernels read and write 16 bytes of a head at a time, and take strides in
// bytes of 32 bits.
constexpr int64_t kMaxStride = 0x7fffffff;
bool attn_heads_ok(const pard_heads* t, const pard_cod_attn_args* a, int heads, bool out) {
  return heads_ok(t, a->plan->rows, heads, a->head_dim, out) && aligned(t->data, 16) && t->row_stride % 8 == 0 &&
         t->head_stride % 8 == 0 && t->row_stride <= kMaxStride && t->head_stride <= kMaxStride;
}

CodAttnArgs attn_args(const pard_cod_attn_args* a) {
  CodAttnArgs r{};
  cod_plan_layout(a->plan->rows, a->plan->n_samples, const_cast<void*>(a->plan->data), &r.plan);
  r.n_tiles = a->plan->n_tiles;
  r.n_samples = a->plan->n_samples;
  r.n_heads = a->n_heads;
  r.n_kv = a->n_kv_heads;
  r.group = a->n_heads / a->n_kv_heads;
  r.by_group = fast_div(r.group);
  r.rows = a->plan->rows;
  r.scale = a->scale;
  return r;
}

bool loss_ok(const pard_cod_loss_args* a) {
  return a && a->rows >= 0 && a->vocab >= 1 && a->n_sections >= 1 && a->n_sections <= kCodMaxSections;
}

// Workspace of the loss: partial counts, the ticket, the workgroups' sums.
size_t loss_layout(const pard_cod_loss_args* a, char* base, CodLossArgs* r) {
  const size_t counts = align256(sizeof(int) * kLossCountBlocks * kCodMaxSections);
  if (r) {
    r->counts = reinterpret_cast<int*>(base);
    r->ticket = reinterpret_cast<int*>(base + counts);
    r->sums = reinterpret_cast<double*>(base + counts + 256);
  }
  return counts + 256 + align256(sizeof(double) * kLossMaxBlocks * a->n_sections);
}

}  // namespace

extern "C" {

size_t pard_rope_table_bytes(const pard_rope_spec* spec, int32_t n_pos) {
  return rope_spec_ok(spec, n_pos) ? (size_t)n_pos * spec->rot_dim * sizeof(float) : 0;
}

pard_status pard_rope_table(const pard_rope_spec* spec, int32_t n_pos, float* table, void* hip_stream) {
  if (!rope_spec_ok(spec, n_pos) || !table || !aligned(table, 16)) return PARD_ERR_ARG;
  return status_of(launch_rope_spec_table(*spec, n_pos, reinterpret_cast<float2*>(table),
                                          reinterpret_cast<hipStream_t>(hip_stream)));
}

pard_status pard_qk_rope(const pard_rope_args* args, const pard_heads* q, const pard_heads* k, const pard_heads* q_out,
                         const pard_heads* k_out, void* hip_stream) {
  const pard_status st = rope_check(args);
  if (st != PARD_OK) return st;
  const pard_rope_args& a = *args;
  if (!heads_ok(q, a.rows, a.n_q, a.head_dim, false) || !heads_ok(q_out, a.rows, a.n_q, a.head_dim, true) ||
      (a.n_k > 0 && (!heads_ok(k, a.rows, a.n_k, a.head_dim, false) || !heads_ok(k_out, a.rows, a.n_k, a.head_dim, true))))
    return PARD_ERR_ARG;
  if (a.rows == 0) return PARD_OK;
  if (!same_or_apart(q, q_out, a.rows, a.n_q) ||
      (a.n_k > 0 && (!same_or_apart(k, k_out, a.rows, a.n_k) || !apart(q, k_out) || !apart(k, q_out) || !apart(q_out, k_out))))
    return PARD_ERR_ARG;
  RopeArgs r = rope_args(args);
  r.q_in = view(q);
  r.q_out = view(q_out);
  if (a.n_k > 0) {
    r.k_in = view(k);
    r.k_out = view(k_out);
  }
  return status_of(launch_qk_rope(a.dtype, a.layout, false, r, nullptr, nullptr, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t pard_qk_rope_workspace_bytes(const pard_rope_args* args) {
  if (rope_check(args) != PARD_OK || !args->q_gain) return 0;
  return align256((size_t)rope_grad_blocks(rope_args(args)) * 2 * args->head_dim * sizeof(float));
}

pard_status pard_qk_rope_grad(const pard_rope_args* args, const pard_heads* q_dy, const pard_heads* k_dy,
                              const pard_heads* q, const pard_heads* k, const pard_heads* q_dx, const pard_heads* k_dx,
                              float* q_dgain, float* k_dgain, void* workspace, size_t workspace_bytes,
                              void* hip_stream) {
  const pard_status st = rope_check(args);
  if (st != PARD_OK) return st;
  const pard_rope_args& a = *args;
  const bool norm = a.q_gain != nullptr, keys = a.n_k > 0;
  auto in = [&](const pard_heads* t, int n) { return heads_ok(t, a.rows, n, a.head_dim, false); };
  auto out = [&](const pard_heads* t, int n) { return heads_ok(t, a.rows, n, a.head_dim, true); };
  if (!in(q_dy, a.n_q) || !out(q_dx, a.n_q) || (keys && (!in(k_dy, a.n_k) || !out(k_dx, a.n_k)))) return PARD_ERR_ARG;
  if (norm && (!in(q, a.n_q) || !q_dgain || (keys && (!in(k, a.n_k) || !k_dgain)))) return PARD_ERR_ARG;
  if (norm && (!workspace || !aligned(workspace, 256))) return PARD_ERR_ARG;
  if (norm && workspace_bytes < pard_qk_rope_workspace_bytes(args)) return PARD_ERR_NOMEM;
  if (a.rows > 0 &&
      (!same_or_apart(q_dy, q_dx, a.rows, a.n_q) || (norm && !apart(q, q_dx)) ||
       (keys && (!same_or_apart(k_dy, k_dx, a.rows, a.n_k) || !apart(q_dy, k_dx) || !apart(k_dy, q_dx) || !apart(q_dx, k_dx) ||
                 (norm && (!apart(k, k_dx) || !apart(q, k_dx) || !apart(k, q_dx)))))))
    return PARD_ERR_ARG;
  if (a.rows == 0 && !norm) return PARD_OK;
  RopeArgs r = rope_args(args);
  r.q_in = view(q_dy);
  r.q_out = view(q_dx);
  if (keys) {
    r.k_in = view(k_dy);
    r.k_out = view(k_dx);
  }
  if (norm) {
    r.q_x = view(q);
    if (keys) r.k_x = view(k);
    r.part = static_cast<float*>(workspace);
  }
  return status_of(launch_qk_rope(a.dtype, a.layout, true, r, q_dgain, k_dgain, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t pard_cod_plan_bytes(int64_t rows, int32_t n_samples) {
  if (rows < 0 || rows > 0x7fffffff || n_samples < 1) return 0;
  return cod_plan_layout(rows, n_samples, nullptr, nullptr);
}

pard_status pard_cod_plan_build(const int32_t* section, const int32_t* column, const int64_t* out_offsets,
                                const int32_t* out_len, int32_t n_samples, void* plan_data, size_t plan_bytes,
                                void* hip_stream, pard_cod_plan* plan) {
  if (!out_offsets || !out_len || !plan || n_samples < 1 || !plan_data || !aligned(plan_data, 256) || out_offsets[0] < 0)
    return PARD_ERR_ARG;
  int64_t tiles = 0, longest = 0;
  for (int s = 0; s < n_samples; ++s) {
    const int64_t cap = out_offsets[s + 1] - out_offsets[s];
    if (cap < 0) return PARD_ERR_ARG;
    tiles += (cap + kCodTile - 1) / kCodTile;
    longest = std::max(longest, cap);
  }
  const int64_t rows = out_offsets[n_samples];
  if (rows > 0 && (!section || !column)) return PARD_ERR_ARG;
  // (n_samples: workgroups of 1024 threads, fewer than 2^32 in a launch)
  if (rows > 0x7fffffff || longest > (int64_t)kCodMaxSections * 8192 || n_samples >= 1 << 22) return PARD_ERR_UNSUPPORTED;
  if (plan_bytes < pard_cod_plan_bytes(rows, n_samples)) return PARD_ERR_NOMEM;
  CodPlanView v;
  cod_plan_layout(rows, n_samples, plan_data, &v);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  int bad = 0;
  if (hipMemcpyAsync(v.offsets, out_offsets, sizeof(int64_t) * ((size_t)n_samples + 1), hipMemcpyHostToDevice, st) !=
          hipSuccess ||
      hipMemcpyAsync(v.bad, &bad, sizeof bad, hipMemcpyHostToDevice, st) != hipSuccess ||
      launch_cod_plan(section, column, out_len, n_samples, (int)longest, v, st) != hipSuccess ||
      hipMemcpyAsync(&bad, v.bad, sizeof bad, hipMemcpyDeviceToHost, st) != hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return PARD_ERR_DEVICE;
  if (bad) return PARD_ERR_ARG;
  *plan = pard_cod_plan{rows, n_samples, (int32_t)tiles, plan_data};
  return PARD_OK;
}

pard_status pard_cod_attn(const pard_cod_attn_args* args, const pard_heads* q, const pard_heads* k, const pard_heads* v,
                          const pard_heads* out, float* lse, void* hip_stream) {
  const pard_status st = attn_check(args);
  if (st != PARD_OK) return st;
  const int nq = args->n_heads, nk = args->n_kv_heads;
  if (!attn_heads_ok(q, args, nq, false) || !attn_heads_ok(k, args, nk, false) || !attn_heads_ok(v, args, nk, false) ||
      !attn_heads_ok(out, args, nq, true))
    return PARD_ERR_ARG;
  if (args->plan->n_tiles == 0) return PARD_OK;
  if (!apart(q, out) || !apart(k, out) || !apart(v, out)) return PARD_ERR_ARG;
  CodAttnArgs r = attn_args(args);
  r.q = view16(q);
  r.k = view16(k);
  r.v = view16(v);
  r.out = view16(out);
  r.lse = lse;
  return status_of(launch_cod_attn(args->head_dim, args->dtype, r, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t pard_cod_attn_workspace_bytes(const pard_cod_attn_args* args) {
  if (attn_check(args) != PARD_OK) return 0;
  return cod_attn_grad_workspace(args->plan->rows, args->plan->n_samples, args->n_kv_heads,
                                 args->n_heads / args->n_kv_heads);
}

pard_status pard_cod_attn_grad(const pard_cod_attn_args* args, const pard_heads* d_out, const pard_heads* q,
                               const pard_heads* k, const pard_heads* v, const pard_heads* out, const float* lse,
                               const pard_heads* dq, const pard_heads* dk, const pard_heads* dv, void* workspace,
                               size_t workspace_bytes, void* hip_stream) {
  const pard_status st = attn_check(args);
  if (st != PARD_OK) return st;
  const int nq = args->n_heads, nk = args->n_kv_heads;
  if (!attn_heads_ok(d_out, args, nq, false) || !attn_heads_ok(q, args, nq, false) ||
      !attn_heads_ok(k, args, nk, false) || !attn_heads_ok(v, args, nk, false) || !attn_heads_ok(out, args, nq, false) ||
      !attn_heads_ok(dq, args, nq, true) || !attn_heads_ok(dk, args, nk, true) || !attn_heads_ok(dv, args, nk, true))
    return PARD_ERR_ARG;
  if (args->plan->n_tiles == 0) return PARD_OK;
  if (!lse || !workspace || !aligned(workspace, 256)) return PARD_ERR_ARG;
  if (workspace_bytes < pard_cod_attn_workspace_bytes(args)) return PARD_ERR_NOMEM;
  for (const pard_heads* y : {dq, dk, dv})
    for (const pard_heads* x : {d_out, q, k, v, out})
      if (!apart(x, y)) return PARD_ERR_ARG;
  if (!apart(dq, dk) || !apart(dq, dv) || !apart(dk, dv)) return PARD_ERR_ARG;
  CodAttnArgs r = attn_args(args);
  r.q = view16(q);
  r.k = view16(k);
  r.v = view16(v);
  r.out = view16(out);
  r.lse = const_cast<float*>(lse);
  r.d_out = view16(d_out);
  r.dq = view16(dq);
  r.dk = view16(dk);
  r.dv = view16(dv);
  r.stats = workspace;
  return status_of(launch_cod_attn_grad(args->head_dim, args->dtype, r, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t pard_cod_loss_workspace_bytes(const pard_cod_loss_args* args) {
  return loss_ok(args) ? loss_layout(args, nullptr, nullptr) : 0;
}

pard_status pard_cod_loss(const pard_cod_loss_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!loss_ok(args) || !args->loss || !std::isfinite(args->grad_scale)) return PARD_ERR_ARG;
  const pard_cod_loss_args& a = *args;
  if (a.rows > 0 && (!a.logits || !a.labels || (!a.section && a.n_sections != 1))) return PARD_ERR_ARG;
  if (a.rows > 1 && (a.logits_stride < a.vocab || (a.d_logits && a.d_stride < a.vocab))) return PARD_ERR_ARG;
  if (a.rows > 1 && a.d_logits == a.logits && a.d_stride != a.logits_stride) return PARD_ERR_ARG;
  for (int k = 0; a.weights && k < a.n_sections; ++k)
    if (!std::isfinite(a.weights[k])) return PARD_ERR_ARG;
  const int size = elem_size(a.dtype);
  if (!size || a.rows > (1 << 30) || a.vocab > (1 << 28)) return PARD_ERR_UNSUPPORTED;
  if (!aligned(a.logits, size) || !aligned(a.d_logits, size) || !workspace || !aligned(workspace, 256)) return PARD_ERR_ARG;
  if (workspace_bytes < pard_cod_loss_workspace_bytes(args)) return PARD_ERR_NOMEM;
  CodLossArgs r{};
  r.rows = (int)a.rows;
  r.vocab = a.vocab;
  r.n_sections = a.n_sections;
  r.logits = static_cast<const char*>(a.logits);
  r.stride = a.logits_stride;
  r.labels = a.labels;
  r.section = a.section;
  r.d_logits = static_cast<char*>(a.d_logits);
  r.d_stride = a.d_stride;
  r.grad_scale = a.grad_scale;
  r.weighted = a.weights != nullptr;
  for (int k = 0; a.weights && k < a.n_sections; ++k) r.weights[k] = a.weights[k];
  r.loss = a.loss;
  r.row_loss = a.row_loss;
  loss_layout(args, static_cast<char*>(workspace), &r);
  return status_of(launch_cod_loss(a.dtype, r, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
