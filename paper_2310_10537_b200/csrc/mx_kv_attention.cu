// Attention of the newest tokens over a paged cache of MX rows (see mx_kv_attention in mx.h).
//
// The first form: one block per query row, a warp per token, an element of every block per lane.
#include <cuda_fp16.h>

#include "mx_device.cuh"
#include "mx_launch.h"
#include "mx_rows.cuh"

namespace mx {
namespace {

constexpr int kWarps = 8;
constexpr float kLog2e = 1.4426950408889634f;

template <int FMT>
__device__ __forceinline__ float decode1(const uint8_t* row, uint32_t e) {
  if (FMT == MX_INT8) return (float)(int8_t)row[e] * 0.015625f;
  uint32_t h2;
  if (FMT == MX_E2M1) {
    const uint16_t p = (uint16_t)(row[e / 2] >> 4 * (e & 1));
    asm("{ .reg .b8 lo, hi; mov.b16 {lo, hi}, %1; cvt.rn.f16x2.e2m1x2 %0, lo; }" : "=r"(h2) : "h"(p));
  } else {
    const uint16_t p = row[e];
    if (FMT == MX_E4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(p));
    else asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h2) : "h"(p));
  }
  return __low2float(*reinterpret_cast<const __half2*>(&h2));
}
__device__ __forceinline__ float e8m0(uint32_t sb) {
  return __uint_as_float(sb == 0 ? 0x00400000u : (sb == 255 ? 0x7FC00000u : sb << 23));
}

template <int FMT, int DTYPE, int BLOCKS>
__global__ void __launch_bounds__(kWarps * 32) kv_attention_simple(KvAttentionArgs a) {
  __shared__ float sm[kWarps], sl[kWarps], so[kWarps][BLOCKS * 32];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t row = blockIdx.x, head = row % (uint32_t)a.q_heads, token = row / (uint32_t)a.q_heads;
  const uint32_t b = token / (uint32_t)a.new_tokens, i = token % (uint32_t)a.new_tokens;
  const uint32_t h = head / (uint32_t)(a.q_heads / a.kv.heads);
  constexpr uint32_t code_bytes = BLOCKS * 32 * FmtTraits<FMT>::bits / 8, scale_bytes = (BLOCKS + 3) / 4 * 4;
  int64_t len = a.lengths[b];
  const int64_t cap = a.max_pages * a.kv.page_size;
  len = len < 0 ? 0 : len > cap ? cap : len;
  const int64_t end = len - (a.new_tokens - 1 - i), begin = a.window > 0 && end > a.window ? end - a.window : 0;
  float q[BLOCKS], o[BLOCKS];
#pragma unroll
  for (int d = 0; d < BLOCKS; ++d) {
    q[d] = load1<DTYPE>(a.q, (size_t)token * a.q_stride + (size_t)head * BLOCKS * 32 + d * 32 + lane);
    o[d] = 0.0f;
  }
  float m = -INFINITY, l = 0.0f;
  for (int64_t j = begin + warp; j < end; j += kWarps) {
    const int64_t page = a.table[b * a.max_pages + j / a.kv.page_size];
    if (page < 0 || page >= a.kv.pages) continue;
    const size_t r = ((size_t)page * a.kv.heads + h) * a.kv.page_size + j % a.kv.page_size;
    float s = 0.0f;
#pragma unroll
    for (int d = 0; d < BLOCKS; ++d)
      s += q[d] * decode1<FMT>(a.kv.k_elems + r * code_bytes, d * 32 + lane) * e8m0(a.kv.k_scales[r * scale_bytes + d]);
#pragma unroll
    for (int n = 16; n; n >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, n);
    s *= a.scale * kLog2e;
    const float top = fmaxf(m, s), keep = top == -INFINITY ? 0.0f : exp2f(m - top), p = exp2f(s - (top == -INFINITY ? 0.0f : top));
    l = l * keep + p;
#pragma unroll
    for (int d = 0; d < BLOCKS; ++d)
      o[d] = o[d] * keep + p * (decode1<FMT>(a.kv.v_elems + r * code_bytes, d * 32 + lane) * e8m0(a.kv.v_scales[r * scale_bytes + d]));
    m = top;
  }
  if (lane == 0) { sm[warp] = m; sl[warp] = l; }
#pragma unroll
  for (int d = 0; d < BLOCKS; ++d) so[warp][d * 32 + lane] = o[d];
  __syncthreads();
  float top = -INFINITY, total = 0.0f;
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm[w]);
  for (int w = 0; w < kWarps; ++w) total += sm[w] == -INFINITY && sl[w] == 0.0f ? 0.0f : sl[w] * exp2f(sm[w] - top);
  for (int e = threadIdx.x; e < BLOCKS * 32; e += kWarps * 32) {
    float v = 0.0f;
    for (int w = 0; w < kWarps; ++w) v += sm[w] == -INFINITY && sl[w] == 0.0f ? 0.0f : so[w][e] * exp2f(sm[w] - top);
    store1<DTYPE>(a.out, (size_t)row * BLOCKS * 32 + e, total == 0.0f ? 0.0f : v / total);
  }
  if (a.lse && threadIdx.x == 0) a.lse[row] = total == 0.0f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
}

template <int FMT, int DTYPE>
cudaError_t by_dim(const KvAttentionArgs& a) {
  const dim3 grid((uint32_t)(a.batch * a.new_tokens * a.q_heads));
  switch (a.kv.dim) {
    case 64: kv_attention_simple<FMT, DTYPE, 2><<<grid, kWarps * 32, 0, a.stream>>>(a); break;
    case 96: kv_attention_simple<FMT, DTYPE, 3><<<grid, kWarps * 32, 0, a.stream>>>(a); break;
    case 128: kv_attention_simple<FMT, DTYPE, 4><<<grid, kWarps * 32, 0, a.stream>>>(a); break;
    case 192: kv_attention_simple<FMT, DTYPE, 6><<<grid, kWarps * 32, 0, a.stream>>>(a); break;
    default: kv_attention_simple<FMT, DTYPE, 8><<<grid, kWarps * 32, 0, a.stream>>>(a); break;
  }
  return cudaGetLastError();
}

}  // namespace

size_t kv_attention_workspace(const KvArgs&, int64_t, int64_t, int64_t) { return 256; }

cudaError_t launch_kv_attention(const KvAttentionArgs& a) {
  const bool h = a.dtype == MX_BF16;
  switch (a.kv.fmt) {
    case MX_E4M3: return h ? by_dim<MX_E4M3, MX_BF16>(a) : by_dim<MX_E4M3, MX_F32>(a);
    case MX_E5M2: return h ? by_dim<MX_E5M2, MX_BF16>(a) : by_dim<MX_E5M2, MX_F32>(a);
    case MX_E2M1: return h ? by_dim<MX_E2M1, MX_BF16>(a) : by_dim<MX_E2M1, MX_F32>(a);
    default: return h ? by_dim<MX_INT8, MX_BF16>(a) : by_dim<MX_INT8, MX_F32>(a);
  }
}

}  // namespace mx
