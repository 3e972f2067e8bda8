// The kernels of attn_rows.h for fp32 rows of head dim 64.
#include "attn_rows.h"

namespace oomb {

hipError_t launch_attn_rows_f32_64(const RowsParams& p, void* ws, hipStream_t st) { return attn<float, 64>(p, ws, st); }

}  // namespace oomb
