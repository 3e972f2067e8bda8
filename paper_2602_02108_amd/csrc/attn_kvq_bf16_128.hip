// The kernels of attn_kvq.h for bf16 rows of head dim 128.
#include "attn_kvq.h"

namespace oomb {

hipError_t launch_attn_kvq_bf16_128(const RowsParams& p, void* ws, hipStream_t st) { return attn<bf16_t, 128>(p, ws, st); }

}  // namespace oomb
