// C-ABI entry points of the cache, its attention and the residual norm: host-side checks only.  No kernel lives here.
#include <math.h>

#include "vq_kv.cuh"
#include "vq_residual_norm.cuh"

namespace vq {
namespace {

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

vq_status check_kv_format(const vq_kv_format* f, KvGeometry* g) {
  if (!f) return VQ_ERR_NULL;
  if (f->kv_type != VQ_KV_FP16 && f->kv_type != VQ_KV_INT8) return VQ_ERR_FORMAT;
  int shift = 3;
  while (shift < 8 && (1 << shift) != f->page_tokens) ++shift;
  if ((1 << shift) != f->page_tokens) return VQ_ERR_FORMAT;
  if (f->head_dim < 16 || f->head_dim > 256 || f->head_dim % 16) return VQ_ERR_FORMAT;
  if (f->n_pages <= 0 || f->n_pages > (1 << 30) || f->n_kv_heads <= 0 || f->n_kv_heads > 65536) return VQ_ERR_SHAPE;
  g->n_pages = f->n_pages;
  g->page_tokens = f->page_tokens;
  g->page_shift = shift;
  g->heads = f->n_kv_heads;
  g->dim = f->head_dim;
  g->int8 = f->kv_type == VQ_KV_INT8;
  g->row_bytes = f->head_dim * (g->int8 ? 1 : 2);
  return VQ_OK;
}

vq_status check_pool(const KvGeometry& g, const vq_kv_pool* p, KvPool* out) {
  if (!p || !p->d_k || !p->d_v) return VQ_ERR_NULL;
  if (g.int8 ? (!p->d_k_scale || !p->d_v_scale) : (p->d_k_scale || p->d_v_scale)) return VQ_ERR_NULL;
  if (!aligned(p->d_k, 16) || !aligned(p->d_v, 16) || !aligned(p->d_k_scale, 16) || !aligned(p->d_v_scale, 16)) return VQ_ERR_ALIGN;
  out->k = static_cast<uint8_t*>(p->d_k);
  out->v = static_cast<uint8_t*>(p->d_v);
  out->ks = static_cast<float*>(p->d_k_scale);
  out->vs = static_cast<float*>(p->d_v_scale);
  return VQ_OK;
}

vq_status check_pools(const KvGeometry& g, const vq_kv_pool* pools, int n_layers, KvPools* out) {
  if (!pools) return VQ_ERR_NULL;
  if (n_layers < 1 || n_layers > VQ_KV_MAX_LAYERS) return VQ_ERR_SHAPE;
  out->n_layers = n_layers;
  for (int i = 0; i < n_layers; ++i) {
    const vq_status st = check_pool(g, pools + i, &out->p[i]);
    if (st != VQ_OK) return st;
  }
  return VQ_OK;
}

vq_status check_seqs(const KvGeometry& g, const vq_kv_seqs* q, KvBooks* out) {
  if (!q || !q->d_table || !q->d_len) return VQ_ERR_NULL;
  if (q->n_seqs < 1 || q->n_seqs > 65536 || q->table_stride < 1) return VQ_ERR_SHAPE;
  if (static_cast<long long>(q->table_stride) * g.page_tokens > (1ll << 30)) return VQ_ERR_SHAPE;
  if (!aligned(q->d_table, 4) || !aligned(q->d_len, 4)) return VQ_ERR_ALIGN;
  out->table = static_cast<int*>(q->d_table);
  out->len = static_cast<int*>(q->d_len);
  out->n_seqs = q->n_seqs;
  out->table_stride = q->table_stride;
  out->max_len = q->table_stride * g.page_tokens;
  return VQ_OK;
}

vq_status check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return VQ_ERR_WORKSPACE;
  return aligned(ws, 16) ? VQ_OK : VQ_ERR_ALIGN;
}

// Rows of `width` elements, `stride` apart, read in pieces of eight binary16 values.
vq_status check_rows(long long stride, long long width) {
  if (stride < width) return VQ_ERR_SHAPE;
  return stride % 8 ? VQ_ERR_ALIGN : VQ_OK;
}

}  // namespace
}  // namespace vq

using namespace vq;

#define VQ_TRY(expr)                      \
  do {                                    \
    const vq_status vq_try_st = (expr);   \
    if (vq_try_st != VQ_OK) return vq_try_st; \
  } while (0)

extern "C" {

vq_status vq_kv_info(const vq_kv_format* fmt, vq_kv_info_t* out) {
  if (!out) return VQ_ERR_NULL;
  KvGeometry g;
  VQ_TRY(check_kv_format(fmt, &g));
  const size_t rows = static_cast<size_t>(g.heads) * g.page_tokens;
  out->pool_bytes = rows * g.n_pages * g.row_bytes;
  out->scale_bytes = g.int8 ? rows * g.n_pages * sizeof(float) : 0;
  out->page_bytes = 2 * rows * (g.row_bytes + (g.int8 ? sizeof(float) : 0));
  return VQ_OK;
}

size_t vq_kv_attention_workspace_bytes(const vq_kv_format* fmt) {
  KvGeometry g;
  return check_kv_format(fmt, &g) == VQ_OK && kv_attention_covers(g) ? kv_attention_workspace_bytes(g.dim) : 0;
}

vq_status vq_kv_attention(const vq_kv_format* fmt, const vq_kv_pool* pool, const vq_kv_seqs* seqs, int n_q_heads, const void* d_q,
                          int64_t q_stride, void* d_out, int64_t out_stride, void* d_lse, float scale, int window, void* d_ws,
                          size_t ws_bytes, void* stream) {
  KvGeometry g;
  KvPool p;
  KvBooks b;
  VQ_TRY(check_kv_format(fmt, &g));
  VQ_TRY(check_pool(g, pool, &p));
  VQ_TRY(check_seqs(g, seqs, &b));
  if (!d_q || !d_out) return VQ_ERR_NULL;
  if (n_q_heads < 1 || n_q_heads % g.heads || n_q_heads > 65536 || window < 0) return VQ_ERR_SHAPE;
  const long long width = static_cast<long long>(n_q_heads) * g.dim;
  VQ_TRY(check_rows(q_stride, width));
  VQ_TRY(check_rows(out_stride, width));
  if (!aligned(d_q, 16) || !aligned(d_out, 16) || !aligned(d_lse, 4)) return VQ_ERR_ALIGN;
  if (!kv_attention_covers(g)) return VQ_ERR_UNSUPPORTED;
  VQ_TRY(check_ws(d_ws, ws_bytes, kv_attention_workspace_bytes(g.dim)));
  return launch_kv_attention(g, p, b, n_q_heads, static_cast<const __half*>(d_q), q_stride, static_cast<__half*>(d_out), out_stride,
                             static_cast<float*>(d_lse), scale, window, d_ws, static_cast<cudaStream_t>(stream));
}

vq_status vq_kv_append(const vq_kv_format* fmt, const vq_kv_pool* pool, const vq_kv_seqs* seqs, const void* d_starts, int n_tokens,
                       const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride, const vq_kv_rotary* rotary, void* stream) {
  KvGeometry g;
  KvPool p;
  KvBooks b;
  VQ_TRY(check_kv_format(fmt, &g));
  VQ_TRY(check_pool(g, pool, &p));
  VQ_TRY(check_seqs(g, seqs, &b));
  if (!d_k || !d_v) return VQ_ERR_NULL;
  if (n_tokens < 1 || (!d_starts && n_tokens != b.n_seqs)) return VQ_ERR_SHAPE;
  const long long width = static_cast<long long>(g.heads) * g.dim;
  VQ_TRY(check_rows(k_stride, width));
  VQ_TRY(check_rows(v_stride, width));
  if (!aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_starts, 4)) return VQ_ERR_ALIGN;
  KvRotary r = {};
  if (rotary) {
    if (!rotary->d_cos_sin || (rotary->n_q_heads ? !rotary->d_q || !rotary->d_q_out : rotary->d_q || rotary->d_q_out)) return VQ_ERR_NULL;
    if (rotary->rot_dim < 16 || rotary->rot_dim > g.dim || rotary->rot_dim % 16 || rotary->n_q_heads < 0 || rotary->n_q_heads > 65536 ||
        rotary->n_positions < b.max_len || (rotary->interleaved != 0 && rotary->interleaved != 1))
      return VQ_ERR_SHAPE;
    if (!aligned(rotary->d_cos_sin, 16)) return VQ_ERR_ALIGN;
    if (rotary->n_q_heads) {
      const long long q_width = static_cast<long long>(rotary->n_q_heads) * g.dim;
      VQ_TRY(check_rows(rotary->q_stride, q_width));
      VQ_TRY(check_rows(rotary->q_out_stride, q_width));
      if (!aligned(rotary->d_q, 16) || !aligned(rotary->d_q_out, 16)) return VQ_ERR_ALIGN;
      if (rotary->d_q == rotary->d_q_out && rotary->q_stride != rotary->q_out_stride) return VQ_ERR_SHAPE;
    }
    r.cs = static_cast<const float2*>(rotary->d_cos_sin);
    r.rot_dim = rotary->rot_dim;
    r.interleaved = rotary->interleaved;
    r.n_q_heads = rotary->n_q_heads;
    r.q = static_cast<const __half*>(rotary->d_q);
    r.q_out = static_cast<__half*>(rotary->d_q_out);
    r.q_stride = rotary->q_stride;
    r.q_out_stride = rotary->q_out_stride;
  }
  return launch_kv_append(g, p, b, static_cast<const int*>(d_starts), n_tokens, static_cast<const __half*>(d_k), k_stride,
                          static_cast<const __half*>(d_v), v_stride, r, static_cast<cudaStream_t>(stream));
}

size_t vq_kv_pages_workspace_bytes(const vq_kv_format* fmt, int n_seqs) {
  KvGeometry g;
  return check_kv_format(fmt, &g) == VQ_OK && n_seqs >= 1 && n_seqs <= 65536 ? kv_pages_workspace_bytes(g, n_seqs) : 0;
}

vq_status vq_kv_reserve(const vq_kv_format* fmt, const vq_kv_seqs* seqs, void* d_refs, const void* d_new, void* d_status, void* d_ws,
                        size_t ws_bytes, void* stream) {
  KvGeometry g;
  KvBooks b;
  VQ_TRY(check_kv_format(fmt, &g));
  VQ_TRY(check_seqs(g, seqs, &b));
  if (!d_refs || !d_status) return VQ_ERR_NULL;
  if (!aligned(d_refs, 4) || !aligned(d_new, 4) || !aligned(d_status, 4)) return VQ_ERR_ALIGN;
  VQ_TRY(check_ws(d_ws, ws_bytes, kv_pages_workspace_bytes(g, b.n_seqs)));
  return launch_kv_reserve(g, b, static_cast<int*>(d_refs), static_cast<const int*>(d_new), static_cast<int*>(d_status), d_ws,
                           static_cast<cudaStream_t>(stream));
}

vq_status vq_kv_fork(const vq_kv_format* fmt, const vq_kv_pool* pools, int n_layers, const vq_kv_seqs* seqs, void* d_refs,
                     const void* d_pairs, int n_pairs, void* d_status, void* d_ws, size_t ws_bytes, void* stream) {
  KvGeometry g;
  KvPools p;
  KvBooks b;
  VQ_TRY(check_kv_format(fmt, &g));
  VQ_TRY(check_pools(g, pools, n_layers, &p));
  VQ_TRY(check_seqs(g, seqs, &b));
  if (!d_refs || !d_pairs || !d_status) return VQ_ERR_NULL;
  if (n_pairs < 1 || n_pairs > 1024) return VQ_ERR_SHAPE;
  if (!aligned(d_refs, 4) || !aligned(d_pairs, 4) || !aligned(d_status, 4)) return VQ_ERR_ALIGN;
  VQ_TRY(check_ws(d_ws, ws_bytes, kv_pages_workspace_bytes(g, b.n_seqs)));
  return launch_kv_fork(g, p, b, static_cast<int*>(d_refs), static_cast<const int*>(d_pairs), n_pairs, static_cast<int*>(d_status), d_ws,
                        static_cast<cudaStream_t>(stream));
}

vq_status vq_kv_free(const vq_kv_format* fmt, const vq_kv_seqs* seqs, void* d_refs, const void* d_slots, int n_slots, void* stream) {
  KvGeometry g;
  KvBooks b;
  VQ_TRY(check_kv_format(fmt, &g));
  VQ_TRY(check_seqs(g, seqs, &b));
  if (!d_refs || !d_slots) return VQ_ERR_NULL;
  if (n_slots < 1 || n_slots > 65536) return VQ_ERR_SHAPE;
  if (!aligned(d_refs, 4) || !aligned(d_slots, 4)) return VQ_ERR_ALIGN;
  return launch_kv_free(g, b, static_cast<int*>(d_refs), static_cast<const int*>(d_slots), n_slots, static_cast<cudaStream_t>(stream));
}

vq_status vq_kv_compact(const vq_kv_format* fmt, const vq_kv_pool* pools, int n_layers, const vq_kv_seqs* seqs, void* d_refs,
                        void* d_status, void* d_ws, size_t ws_bytes, void* stream) {
  KvGeometry g;
  KvPools p;
  KvBooks b;
  VQ_TRY(check_kv_format(fmt, &g));
  VQ_TRY(check_pools(g, pools, n_layers, &p));
  VQ_TRY(check_seqs(g, seqs, &b));
  if (!d_refs || !d_status) return VQ_ERR_NULL;
  if (!aligned(d_refs, 4) || !aligned(d_status, 4)) return VQ_ERR_ALIGN;
  VQ_TRY(check_ws(d_ws, ws_bytes, kv_pages_workspace_bytes(g, b.n_seqs)));
  return launch_kv_compact(g, p, b, static_cast<int*>(d_refs), static_cast<int*>(d_status), d_ws, static_cast<cudaStream_t>(stream));
}

vq_status vq_kv_copy_pages(const vq_kv_format* fmt, const vq_kv_pool* pools, int n_layers, const void* d_pairs, int n_pairs,
                           void* stream) {
  KvGeometry g;
  KvPools p;
  VQ_TRY(check_kv_format(fmt, &g));
  VQ_TRY(check_pools(g, pools, n_layers, &p));
  if (!d_pairs) return VQ_ERR_NULL;
  if (n_pairs < 1 || n_pairs > (1 << 24)) return VQ_ERR_SHAPE;
  if (!aligned(d_pairs, 4)) return VQ_ERR_ALIGN;
  return launch_kv_copy_pages(g, p, static_cast<const int*>(d_pairs), n_pairs, static_cast<cudaStream_t>(stream));
}

vq_status vq_residual_norm(const vq_norm_block* d, const void* d_x, const void* d_y, const void* d_gate, const void* d_post_w,
                           const void* d_post_b, const void* d_pre_w, const void* d_pre_b, void* d_x_out, void* d_h, void* stream) {
  if (!d || !d_x || (!d_x_out && !d_h)) return VQ_ERR_NULL;
  if ((d->kind != VQ_NORM_RMS && d->kind != VQ_NORM_LAYER) || (d->residual_type != VQ_RESIDUAL_FP16 && d->residual_type != VQ_RESIDUAL_FP32) ||
      d->gate < VQ_GATE_NONE || d->gate > VQ_GATE_ELEMENT)
    return VQ_ERR_FORMAT;
  if ((d->gate != VQ_GATE_NONE) != (d_gate != nullptr) || (d_h != nullptr) != (d_pre_w != nullptr)) return VQ_ERR_NULL;
  if ((d_post_b && !d_post_w) || (d_pre_b && !d_pre_w) || (!d_y && (d_gate || d_post_w))) return VQ_ERR_NULL;
  if (d->n_rows < 1 || d->n_cols < 1 || d->n_cols > 32768) return VQ_ERR_SHAPE;
  if (d->x_stride < d->n_cols || (d_y && d->y_stride < d->n_cols) || (d->gate == VQ_GATE_ELEMENT && d->gate_stride < d->n_cols) ||
      (d_x_out && d->x_out_stride < d->n_cols) || (d_h && d->h_stride < d->n_cols))
    return VQ_ERR_SHAPE;
  if ((d_x_out == d_x && d->x_out_stride != d->x_stride) || (d_h && d_h == d_y && d->h_stride != d->y_stride)) return VQ_ERR_SHAPE;
  const void* all[] = {d_x, d_y, d_gate, d_post_w, d_post_b, d_pre_w, d_pre_b, d_x_out, d_h};
  for (const void* p : all)
    if (!aligned(p, 16)) return VQ_ERR_ALIGN;
  ResidualNorm a = {};
  a.x = d_x;
  a.y = static_cast<const __half*>(d_y);
  a.gate = static_cast<const __half*>(d_gate);
  a.post_w = static_cast<const __half*>(d_post_w);
  a.post_b = static_cast<const __half*>(d_post_b);
  a.pre_w = static_cast<const __half*>(d_pre_w);
  a.pre_b = static_cast<const __half*>(d_pre_b);
  a.x_out = d_x_out;
  a.h = static_cast<__half*>(d_h);
  a.rows = d->n_rows;
  a.cols = d->n_cols;
  a.layer = d->kind == VQ_NORM_LAYER;
  a.wide = d->residual_type == VQ_RESIDUAL_FP32;
  a.x_stride = d->x_stride;
  a.y_stride = d_y ? d->y_stride : 0;
  a.gate_stride = d->gate == VQ_GATE_ELEMENT ? d->gate_stride : 0;   // one row for all where the gate is per channel
  a.x_out_stride = d_x_out ? d->x_out_stride : 0;
  a.h_stride = d_h ? d->h_stride : 0;
  a.eps = d->eps;
  a.scale = d->residual_scale;
  return launch_residual_norm(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
