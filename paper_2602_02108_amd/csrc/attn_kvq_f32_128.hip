// The kernels of attn_kvq.h for fp32 rows of head dim 128.
#include "attn_kvq.h"

namespace oomb {

hipError_t launch_attn_kvq_f32_128(const RowsParams& p, void* ws, hipStream_t st) { return attn<float, 128>(p, ws, st); }

}  // namespace oomb
