// Attention of packed rows over pools of bf16 / fp32 rows: workspace, grid and dispatch.  The kernels are in attn_rows.h.
#include "attn_rows.h"

namespace oomb {

size_t rows_attn_workspace_bytes(const RowsParams& p, bool is_bf16, int32_t sel_stride) { return part_bytes(p, plan_of(p, is_bf16, sel_stride)); }
int64_t rows_attn_blocks(const RowsParams& p, bool is_bf16, int32_t sel_stride) {
  const Plan c = plan_of(p, is_bf16, sel_stride);
  const int64_t combine = c.split ? combine_blocks(p, c) : 0;
  return c.blocks > combine ? c.blocks : combine;
}

hipError_t launch_attn_rows(const RowsParams& p, bool is_bf16, void* ws, hipStream_t st) {
  if (is_bf16) return p.D == 128 ? launch_attn_rows_bf16_128(p, ws, st) : launch_attn_rows_bf16_64(p, ws, st);
  return p.D == 128 ? launch_attn_rows_f32_128(p, ws, st) : launch_attn_rows_f32_64(p, ws, st);
}

}  // namespace oomb
