// C-ABI entry points over packed rows (the second part of include/oomb.h): host-side validation and dispatch.  As in api.hip nothing is
// allocated, freed or synchronised, and nothing is enqueued unless every check passes.
#include <cmath>

#include "common.h"
#include "launch.h"
#include "rows.h"

using namespace oomb;

namespace {

enum PoolKind { SAME, GRAD_F32, GRAD_BF16, KVQ };

size_t elem_size(int32_t dt) { return dt == OOMB_BF16 ? 2 : 4; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// the descriptor alone
oomb_status check_rows(const oomb_rows_desc* d, PoolKind pools, RowsParams* p) {
  if (!d) return OOMB_ERR_INVALID_ARG;
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->n_q_heads % d->n_kv_heads || d->head_dim <= 0 || d->page_size <= 0) return OOMB_ERR_INVALID_ARG;
  if ((d->dtype != OOMB_F32 && d->dtype != OOMB_BF16) || d->reserved) return OOMB_ERR_INVALID_ARG;
  if (d->n_seqs <= 0 || d->n_rows <= 0 || d->max_rows <= 0 || d->max_rows > d->n_rows) return OOMB_ERR_INVALID_ARG;
  if (d->max_len <= 0 || d->table_stride <= 0 || d->num_phys_pages <= 0) return OOMB_ERR_INVALID_ARG;
  if ((d->head_dim != 64 && d->head_dim != 128) || (d->page_size & (d->page_size - 1)) || d->page_size < 16 || d->page_size > 128)
    return OOMB_ERR_UNSUPPORTED;
  const int P = d->page_size, D = d->head_dim;
  if (d->max_len > (int64_t)INT32_MAX - 256 || d->table_stride > INT32_MAX || d->num_phys_pages > INT32_MAX) return OOMB_ERR_UNSUPPORTED;
  if ((d->max_len + P - 1) / P > d->table_stride) return OOMB_ERR_INVALID_ARG;
  const int32_t G = d->n_q_heads / d->n_kv_heads;
  if ((int64_t)d->max_rows * G > (1 << 30)) return OOMB_ERR_UNSUPPORTED;
  if (pools == KVQ) {
    const int64_t tile = kvq_tile_bytes(P, D);
    if (d->pool_page_stride < tile || d->pool_head_stride < tile || d->pool_page_stride % 16 || d->pool_head_stride % 16) return OOMB_ERR_INVALID_ARG;
  } else {
    const int64_t es = pools == SAME ? (int64_t)elem_size(d->dtype) : pools == GRAD_BF16 ? 2 : 4;
    for (int64_t s : {d->pool_page_stride, d->pool_head_stride, d->pool_tok_stride})
      if (s < D || (s * es) % 16) return OOMB_ERR_INVALID_ARG;
  }
  p->Hq = d->n_q_heads; p->Hkv = d->n_kv_heads; p->G = G; p->D = D; p->P = P;
  p->n_seqs = d->n_seqs; p->n_rows = d->n_rows; p->max_rows = d->max_rows; p->max_len = (int32_t)d->max_len;
  p->log2_p = __builtin_ctz((unsigned)P);
  p->sm_scale = d->sm_scale;
  p->table_stride = d->table_stride; p->num_phys = d->num_phys_pages;
  p->pool_page_stride = d->pool_page_stride; p->pool_head_stride = d->pool_head_stride; p->pool_tok_stride = d->pool_tok_stride;
  return OOMB_OK;
}

oomb_status check_seqs(const oomb_seqs* s, RowsParams* p) {
  if (!s || !s->page_tables) return OOMB_ERR_INVALID_ARG;
  if (!s->row_starts && (p->n_rows % p->n_seqs || p->n_rows / p->n_seqs > p->max_rows)) return OOMB_ERR_INVALID_ARG;
  p->tables = s->page_tables; p->lens = s->seq_lens; p->starts = s->row_starts;
  return OOMB_OK;
}

oomb_status check_rope(const oomb_rope* r, RowsParams* p) {
  if (!r || r->rot_dim == 0) return OOMB_OK;
  if (!r->cos || !r->sin || !aligned16(r->cos) || !aligned16(r->sin)) return OOMB_ERR_INVALID_ARG;
  if (r->rot_dim < 0 || r->rot_dim % 16 || r->rot_dim > p->D || r->n_pos < p->max_len) return OOMB_ERR_INVALID_ARG;
  p->cos = r->cos; p->sin = r->sin; p->rot_dim = r->rot_dim; p->interleaved = r->interleaved != 0;
  return OOMB_OK;
}

oomb_status check_tensor(const oomb_rows* r, const RowsParams& p, int32_t heads, size_t es, oomb_rows* out) {
  if (!r || !r->data || !aligned16(r->data)) return OOMB_ERR_INVALID_ARG;
  if (p.n_rows > 1 && (r->tok_stride < p.D || (r->tok_stride * (int64_t)es) % 16)) return OOMB_ERR_INVALID_ARG;
  if (heads > 1 && (r->head_stride < p.D || (r->head_stride * (int64_t)es) % 16)) return OOMB_ERR_INVALID_ARG;
  *out = *r;
  return OOMB_OK;
}

// a launch holds less than 2^32 threads
bool grid_fits(int64_t blocks) { return blocks > 0 && blocks < (1 << 24); }
oomb_status launched(hipError_t e) { return e == hipSuccess ? OOMB_OK : OOMB_ERR_LAUNCH; }

#define OOMB_CHECK(expr) \
  if (const oomb_status s_ = (expr); s_ != OOMB_OK) return s_

oomb_status append_rope(const oomb_rows_desc* desc, const oomb_seqs* seqs, const oomb_rope* rope, const oomb_rows* q, const oomb_rows* q_out,
                        const oomb_rows* k, const oomb_rows* v, void* k_pool, void* v_pool, float* kbar_cache, void* hip_stream, bool kvq) {
  RowsParams p{};
  OOMB_CHECK(check_rows(desc, kvq ? KVQ : SAME, &p));
  OOMB_CHECK(check_seqs(seqs, &p));
  OOMB_CHECK(check_rope(rope, &p));
  const size_t es = elem_size(desc->dtype);
  if ((q == nullptr) != (q_out == nullptr)) return OOMB_ERR_INVALID_ARG;
  if (q) {
    OOMB_CHECK(check_tensor(q, p, p.Hq, es, &p.q));
    OOMB_CHECK(check_tensor(q_out, p, p.Hq, es, &p.q_out));
  }
  OOMB_CHECK(check_tensor(k, p, p.Hkv, es, &p.k));
  OOMB_CHECK(check_tensor(v, p, p.Hkv, es, &p.v));
  if (!k_pool || !v_pool || !aligned16(k_pool) || !aligned16(v_pool) || k_pool == v_pool) return OOMB_ERR_INVALID_ARG;
  p.k_pool = k_pool; p.v_pool = v_pool; p.kbar = kbar_cache;
  if (!grid_fits(append_rope_blocks(p, kvq))) return OOMB_ERR_UNSUPPORTED;
  return launched(launch_append_rope(p, desc->dtype == OOMB_BF16, kvq, (hipStream_t)hip_stream));
}

}  // namespace

extern "C" {

oomb_status oomb_kv_append_rope(const oomb_rows_desc* desc, const oomb_seqs* seqs, const oomb_rope* rope, const oomb_rows* q,
                                const oomb_rows* q_out, const oomb_rows* k, const oomb_rows* v, void* k_pool, void* v_pool,
                                float* kbar_cache, void* hip_stream) {
  return append_rope(desc, seqs, rope, q, q_out, k, v, k_pool, v_pool, kbar_cache, hip_stream, false);
}

oomb_status oomb_kvq_append_rope(const oomb_rows_desc* desc, const oomb_seqs* seqs, const oomb_rope* rope, const oomb_rows* q,
                                 const oomb_rows* q_out, const oomb_rows* k, const oomb_rows* v, void* k_pool, void* v_pool,
                                 float* kbar_cache, void* hip_stream) {
  return append_rope(desc, seqs, rope, q, q_out, k, v, k_pool, v_pool, kbar_cache, hip_stream, true);
}

oomb_status oomb_kv_append_rope_bwd(const oomb_rows_desc* desc, const oomb_seqs* seqs, const oomb_rope* rope,
                                    const oomb_rows* d_q, const oomb_rows* d_q_out, const void* dk_pool, const void* dv_pool,
                                    int32_t grad_dtype, const oomb_rows* d_k, const oomb_rows* d_v, void* hip_stream) {
  if (grad_dtype != OOMB_F32 && grad_dtype != OOMB_BF16) return OOMB_ERR_INVALID_ARG;
  RowsParams p{};
  OOMB_CHECK(check_rows(desc, grad_dtype == OOMB_BF16 ? GRAD_BF16 : GRAD_F32, &p));
  OOMB_CHECK(check_seqs(seqs, &p));
  OOMB_CHECK(check_rope(rope, &p));
  const size_t es = elem_size(desc->dtype);
  if ((d_q == nullptr) != (d_q_out == nullptr)) return OOMB_ERR_INVALID_ARG;
  if (d_q) {
    OOMB_CHECK(check_tensor(d_q, p, p.Hq, es, &p.q));
    OOMB_CHECK(check_tensor(d_q_out, p, p.Hq, es, &p.q_out));
  }
  OOMB_CHECK(check_tensor(d_k, p, p.Hkv, es, &p.k));
  OOMB_CHECK(check_tensor(d_v, p, p.Hkv, es, &p.v));
  if (!dk_pool || !dv_pool || !aligned16(dk_pool) || !aligned16(dv_pool)) return OOMB_ERR_INVALID_ARG;
  p.k_pool = const_cast<void*>(dk_pool); p.v_pool = const_cast<void*>(dv_pool);
  if (!grid_fits(append_rope_blocks(p, false))) return OOMB_ERR_UNSUPPORTED;
  return launched(launch_append_rope_bwd(p, desc->dtype == OOMB_BF16, grad_dtype == OOMB_BF16, (hipStream_t)hip_stream));
}

oomb_status oomb_kvq_read(const oomb_rows_desc* desc, const oomb_seqs* seqs, const void* k_pool, const void* v_pool,
                          const oomb_rows* k_out, const oomb_rows* v_out, void* hip_stream) {
  RowsParams p{};
  OOMB_CHECK(check_rows(desc, KVQ, &p));
  OOMB_CHECK(check_seqs(seqs, &p));
  const size_t es = elem_size(desc->dtype);
  OOMB_CHECK(check_tensor(k_out, p, p.Hkv, es, &p.k));
  OOMB_CHECK(check_tensor(v_out, p, p.Hkv, es, &p.v));
  if (!k_pool || !v_pool || !aligned16(k_pool) || !aligned16(v_pool)) return OOMB_ERR_INVALID_ARG;
  p.k_pool = const_cast<void*>(k_pool); p.v_pool = const_cast<void*>(v_pool);
  if (!grid_fits(kvq_read_blocks(p))) return OOMB_ERR_UNSUPPORTED;
  return launched(launch_kvq_read(p, desc->dtype == OOMB_BF16, (hipStream_t)hip_stream));
}

size_t oomb_kvq_workspace_bytes(const oomb_rows_desc* desc, int32_t sel_stride) {
  RowsParams p{};
  if (check_rows(desc, KVQ, &p) != OOMB_OK) return 0;
  return kvq_attn_workspace_bytes(p, desc->dtype == OOMB_BF16, sel_stride);
}

oomb_status oomb_paged_attn_fwd_kvq(const oomb_rows_desc* desc, const oomb_seqs* seqs, const oomb_rows* q, const void* k_pool,
                                    const void* v_pool, const int32_t* sel_pages, const int32_t* sel_count, int32_t sel_stride,
                                    const oomb_rows* o, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  RowsParams p{};
  OOMB_CHECK(check_rows(desc, KVQ, &p));
  if (!(desc->sm_scale > 0.f) || !std::isfinite(desc->sm_scale)) return OOMB_ERR_INVALID_ARG;
  OOMB_CHECK(check_seqs(seqs, &p));
  if (sel_pages && (!sel_count || sel_stride < 0)) return OOMB_ERR_INVALID_ARG;
  const bool bf = desc->dtype == OOMB_BF16;
  const int32_t width = sel_pages ? sel_stride : -1;
  if (!grid_fits(kvq_attn_blocks(p, bf, width))) return OOMB_ERR_UNSUPPORTED;
  const size_t es = elem_size(desc->dtype);
  OOMB_CHECK(check_tensor(q, p, p.Hq, es, &p.q));
  OOMB_CHECK(check_tensor(o, p, p.Hq, es, &p.q_out));
  if (!k_pool || !v_pool || !lse || !aligned16(k_pool) || !aligned16(v_pool)) return OOMB_ERR_INVALID_ARG;
  p.k_pool = const_cast<void*>(k_pool); p.v_pool = const_cast<void*>(v_pool);
  p.sel = sel_pages; p.sel_count = sel_count; p.sel_stride = sel_stride;
  p.lse = lse;
  const size_t need = kvq_attn_workspace_bytes(p, bf, width);
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return OOMB_ERR_WORKSPACE;
  return launched(launch_attn_kvq(p, bf, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
