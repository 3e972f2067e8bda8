// The kernels of attn_rows.h for bf16 rows of head dim 128.
#include "attn_rows.h"

namespace oomb {

hipError_t launch_attn_rows_bf16_128(const RowsParams& p, void* ws, hipStream_t st) { return attn<bf16_t, 128>(p, ws, st); }

}  // namespace oomb
