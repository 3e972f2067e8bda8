// The kernels of attn_kvq.h for bf16 rows of head dim 64.
#include "attn_kvq.h"

namespace oomb {

hipError_t launch_attn_kvq_bf16_64(const RowsParams& p, void* ws, hipStream_t st) { return attn<bf16_t, 64>(p, ws, st); }

}  // namespace oomb
