// mx_kv_attention over a cache of E4M3 rows.
#include "mx_kv_attention.cuh"

namespace mx {
namespace attn {
cudaError_t launch_e4m3(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream) {
  return launch_format<MX_E4M3>(a, dim, wide, ctas, stream);
}
}  // namespace attn
}  // namespace mx
