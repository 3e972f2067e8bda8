// Attention over a cache of 4-bit codes: workspace, grid and dispatch.  The kernels are in attn_kvq.h.
#include "attn_kvq.h"

namespace oomb {

size_t kvq_attn_workspace_bytes(const RowsParams& p, bool is_bf16, int32_t sel_stride) {
  const Plan c = plan_of(p, is_bf16, sel_stride);
  if (!c.split) return 0;
  return (size_t)c.parts * c.row_blocks * 16 * c.rt * (p.D + 2) * sizeof(float) + (size_t)p.n_seqs * p.Hkv * sizeof(int2);
}
int64_t kvq_attn_blocks(const RowsParams& p, bool is_bf16, int32_t sel_stride) {
  const Plan c = plan_of(p, is_bf16, sel_stride);
  const int64_t attn = c.parts * c.row_blocks * (c.waves / 4), combine = c.split ? combine_blocks(p, c) : 0;   // (in workgroups of 256 threads)
  return attn > combine ? attn : combine;
}

hipError_t launch_attn_kvq(const RowsParams& p, bool is_bf16, void* ws, hipStream_t st) {
  if (is_bf16) return p.D == 128 ? launch_attn_kvq_bf16_128(p, ws, st) : launch_attn_kvq_bf16_64(p, ws, st);
  return p.D == 128 ? launch_attn_kvq_f32_128(p, ws, st) : launch_attn_kvq_f32_64(p, ws, st);
}

}  // namespace oomb
