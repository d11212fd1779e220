// mx_kv_attention over a cache of INT8 rows.
#include "mx_kv_attention.cuh"

namespace mx {
namespace attn {
cudaError_t launch_int8(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream) {
  return launch_format<MX_INT8>(a, dim, wide, ctas, stream);
}
}  // namespace attn
}  // namespace mx
