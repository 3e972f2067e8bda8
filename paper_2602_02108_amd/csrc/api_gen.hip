// C-ABI entry points of generation's steps between two passes of attention (the third part of include/oomb.h): host-side validation and dispatch.  As in
// api.hip nothing is allocated, freed or synchronised, and nothing is enqueued unless every check passes.
#include "gen.h"

using namespace oomb;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool grid_fits(int64_t blocks) { return blocks > 0 && blocks < (1 << 24); }
oomb_status launched(hipError_t e) { return e == hipSuccess ? OOMB_OK : OOMB_ERR_LAUNCH; }
// whether two arrays share memory
bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}
// bytes from the first to past the last entry of a table
int64_t table_bytes(int64_t rows, int64_t cols, int64_t stride) { return ((rows - 1) * stride + cols) * 4; }

#define OOMB_CHECK(expr) \
  if (const oomb_status s_ = (expr); s_ != OOMB_OK) return s_

oomb_status check_pages(const oomb_pages_desc* d) {
  if (!d || d->reserved || d->n_seqs <= 0 || d->n_out <= 0 || d->page_size <= 0 || d->num_phys_pages <= 0) return OOMB_ERR_INVALID_ARG;
  if (d->page_size & (d->page_size - 1)) return OOMB_ERR_UNSUPPORTED;
  if (d->table_cols <= 0 || d->out_cols <= 0 || (d->n_seqs > 1 && d->table_stride < d->table_cols) || (d->n_out > 1 && d->out_stride < d->out_cols))
    return OOMB_ERR_INVALID_ARG;
  if (d->num_phys_pages > (1 << 30)) return OOMB_ERR_UNSUPPORTED;
  const int64_t most = INT32_MAX - 256;   // tokens of a sequence; entries of all rows
  if (d->table_cols > most / d->page_size || d->out_cols > most / d->page_size) return OOMB_ERR_UNSUPPORTED;
  if (d->table_cols > most / d->n_seqs || d->out_cols > most / d->n_out) return OOMB_ERR_UNSUPPORTED;
  return OOMB_OK;
}

oomb_status check_beam(const oomb_beam_desc* d, BeamParams* p) {
  if (!d || d->n_groups <= 0 || d->n_beams <= 0 || d->vocab <= 0 || d->n_out <= 0) return OOMB_ERR_INVALID_ARG;
  if (d->dtype != OOMB_F32 && d->dtype != OOMB_BF16) return OOMB_ERR_INVALID_ARG;
  if ((int64_t)d->n_groups * d->n_beams > 1 && d->row_stride < d->vocab) return OOMB_ERR_INVALID_ARG;
  if (d->n_out > BEAM_MOST_OUT || d->n_beams > BEAM_MOST_BEAMS || d->vocab > INT32_MAX - 65536) return OOMB_ERR_UNSUPPORTED;
  if (d->n_groups > INT32_MAX / d->n_beams) return OOMB_ERR_UNSUPPORTED;
  p->n_groups = d->n_groups; p->n_beams = d->n_beams; p->vocab = d->vocab; p->n_out = d->n_out; p->pad_token = d->pad_token;
  p->row_stride = d->row_stride;
  if (!grid_fits(beam_blocks(*p, d->dtype == OOMB_BF16))) return OOMB_ERR_UNSUPPORTED;
  return OOMB_OK;
}

}  // namespace

extern "C" {

size_t oomb_page_fork_workspace_bytes(int32_t n_seqs, int32_t n_out, int64_t num_phys_pages) {
  if (n_seqs <= 0 || n_out <= 0 || n_seqs > FORK_MOST_SEQS || n_out > FORK_MOST_SEQS || num_phys_pages <= 0 || num_phys_pages > (1 << 30)) return 0;
  return fork_workspace_bytes(n_seqs, n_out, num_phys_pages);
}

oomb_status oomb_page_fork(const oomb_pages_desc* d, const int32_t* page_tables, const int32_t* seq_lens, const int32_t* parents, const int32_t* grow,
                           const int32_t* refs, int32_t* tables_out, int32_t* lens_out, int32_t* refs_out, int32_t* copies, int32_t* status,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  OOMB_CHECK(check_pages(d));
  if (d->n_seqs > FORK_MOST_SEQS || d->n_out > FORK_MOST_SEQS) return OOMB_ERR_UNSUPPORTED;
  if (!page_tables || !seq_lens || !parents || !refs || !tables_out || !lens_out || !refs_out || !copies || !status) return OOMB_ERR_INVALID_ARG;
  if (overlap(page_tables, table_bytes(d->n_seqs, d->table_cols, d->table_stride), tables_out, table_bytes(d->n_out, d->out_cols, d->out_stride)))
    return OOMB_ERR_INVALID_ARG;
  if (refs != refs_out && overlap(refs, d->num_phys_pages * 4, refs_out, d->num_phys_pages * 4)) return OOMB_ERR_INVALID_ARG;
  ForkParams p{};
  p.n_seqs = d->n_seqs; p.n_out = d->n_out; p.log2_p = __builtin_ctz((unsigned)d->page_size);
  p.cols = (int32_t)d->table_cols; p.out_cols = (int32_t)d->out_cols; p.stride = d->table_stride; p.out_stride = d->out_stride;
  p.num_phys = (int32_t)d->num_phys_pages;
  p.tables = page_tables; p.lens = seq_lens; p.parents = parents; p.grow = grow; p.refs = refs;
  p.tables_out = tables_out; p.lens_out = lens_out; p.refs_out = refs_out; p.copies = copies; p.status = status;
  if (!grid_fits(fork_blocks(p))) return OOMB_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < fork_workspace_bytes(p.n_seqs, p.n_out, p.num_phys) || !aligned(workspace, 16)) return OOMB_ERR_WORKSPACE;
  return launched(launch_page_fork(p, workspace, (hipStream_t)hip_stream));
}

size_t oomb_page_compact_workspace_bytes(int64_t num_phys_pages) {
  return num_phys_pages <= 0 || num_phys_pages > (1 << 30) ? 0 : compact_workspace_bytes(num_phys_pages);
}

oomb_status oomb_page_compact(const oomb_pages_desc* d, const int32_t* page_tables, const int32_t* seq_lens, const int32_t* refs, int32_t* tables_out,
                              int32_t* refs_out, int32_t* moves, int64_t max_moves, int32_t* page_map, int32_t* status, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
  OOMB_CHECK(check_pages(d));
  if (d->n_out != d->n_seqs || d->out_cols != d->table_cols) return OOMB_ERR_INVALID_ARG;
  if (!page_tables || !seq_lens || !refs || !tables_out || !refs_out || !moves || !page_map || !status) return OOMB_ERR_INVALID_ARG;
  if (max_moves < d->num_phys_pages / 2) return OOMB_ERR_INVALID_ARG;
  const bool same_rows = page_tables == tables_out && (d->n_seqs == 1 || d->table_stride == d->out_stride);
  if (!same_rows && overlap(page_tables, table_bytes(d->n_seqs, d->table_cols, d->table_stride), tables_out, table_bytes(d->n_out, d->out_cols, d->out_stride)))
    return OOMB_ERR_INVALID_ARG;
  if (refs != refs_out && overlap(refs, d->num_phys_pages * 4, refs_out, d->num_phys_pages * 4)) return OOMB_ERR_INVALID_ARG;
  CompactParams p{};
  p.n_seqs = d->n_seqs; p.page = d->page_size; p.log2_p = __builtin_ctz((unsigned)d->page_size);
  p.cols = (int32_t)d->table_cols; p.stride = d->table_stride; p.out_stride = d->out_stride; p.num_phys = (int32_t)d->num_phys_pages;
  p.tables = page_tables; p.lens = seq_lens; p.refs = refs; p.tables_out = tables_out; p.refs_out = refs_out; p.moves = moves; p.map = page_map; p.status = status;
  if (!grid_fits(compact_blocks(p))) return OOMB_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < compact_workspace_bytes(p.num_phys) || !aligned(workspace, 16)) return OOMB_ERR_WORKSPACE;
  return launched(launch_page_compact(p, workspace, (hipStream_t)hip_stream));
}

oomb_status oomb_page_copy(const oomb_copy_desc* d, void* const* pools, const int32_t* copies, const int32_t* count, void* hip_stream) {
  if (!d || d->n_pools <= 0 || d->n_heads <= 0 || d->page_size <= 0 || d->row_bytes <= 0 || d->max_copies < 0 || d->num_phys_pages <= 0) return OOMB_ERR_INVALID_ARG;
  if (!pools || !copies) return OOMB_ERR_INVALID_ARG;
  if (d->row_bytes % 16 || d->page_stride % 16 || d->head_stride % 16 || d->tok_stride % 16) return OOMB_ERR_INVALID_ARG;
  if (d->tok_stride != 0 && d->tok_stride < d->row_bytes) return OOMB_ERR_INVALID_ARG;
  if ((d->num_phys_pages > 1 && d->page_stride < d->row_bytes) || (d->n_heads > 1 && d->head_stride < d->row_bytes)) return OOMB_ERR_INVALID_ARG;
  if (d->num_phys_pages > (1 << 30) || d->max_copies > INT32_MAX || (int64_t)d->page_size * d->row_bytes > INT32_MAX - 65536) return OOMB_ERR_UNSUPPORTED;
  if (d->n_heads > 65535 / COPY_POOLS) return OOMB_ERR_UNSUPPORTED;
  for (int32_t i = 0; i < d->n_pools; ++i)
    if (!pools[i] || !aligned(pools[i], 16)) return OOMB_ERR_INVALID_ARG;
  if (d->max_copies == 0) return OOMB_OK;
  CopyParams p{};
  p.n_heads = d->n_heads; p.page = d->page_size; p.row_bytes = d->row_bytes; p.n_copies = (int32_t)d->max_copies; p.num_phys = (int32_t)d->num_phys_pages;
  p.page_stride = d->page_stride; p.head_stride = d->head_stride; p.tok_stride = d->tok_stride;
  p.copies = copies; p.count = count;
  return launched(launch_page_copy(p, pools, d->n_pools, (hipStream_t)hip_stream));
}

size_t oomb_beam_workspace_bytes(const oomb_beam_desc* d) {
  BeamParams p{};
  return check_beam(d, &p) != OOMB_OK ? 0 : beam_workspace_bytes(p, d->dtype == OOMB_BF16);
}

oomb_status oomb_beam_topk(const oomb_beam_desc* d, const void* logits, const float* scores, const int32_t* done, int32_t* parents, int32_t* tokens,
                           float* scores_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  BeamParams p{};
  OOMB_CHECK(check_beam(d, &p));
  const bool bf = d->dtype == OOMB_BF16;
  if (!logits || !scores || !parents || !tokens || !scores_out || !aligned(logits, bf ? 2 : 4)) return OOMB_ERR_INVALID_ARG;
  const int64_t in = (int64_t)d->n_groups * d->n_beams * 4, out = (int64_t)d->n_groups * d->n_out * 4;
  if (overlap(scores, in, scores_out, out)) return OOMB_ERR_INVALID_ARG;
  p.logits = logits; p.scores = scores; p.done = done; p.parents = parents; p.tokens = tokens; p.best = scores_out;
  if (!workspace || workspace_bytes < beam_workspace_bytes(p, bf) || !aligned(workspace, 16)) return OOMB_ERR_WORKSPACE;
  return launched(launch_beam_topk(p, bf, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
