// mx_kv_attention over a cache of E5M2 rows.
#include "mx_kv_attention.cuh"

namespace mx {
namespace attn {
cudaError_t launch_e5m2(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream) {
  return launch_format<MX_E5M2>(a, dim, wide, ctas, stream);
}
}  // namespace attn
}  // namespace mx
