// The kernels of attn_rows.h for fp32 rows of head dim 128.
#include "attn_rows.h"

namespace oomb {

hipError_t launch_attn_rows_f32_128(const RowsParams& p, void* ws, hipStream_t st) { return attn<float, 128>(p, ws, st); }

}  // namespace oomb
