// mx_kv_attention: its workspace, the choice of an instance, and the kernel that joins the parts of sequences that more than one
// block worked on (the attention itself: mx_kv_attention.cuh).
#include "mx_kv_attention_args.h"
#include "mx_launch.h"
#include "mx_rows.cuh"

namespace mx {
namespace attn {
namespace {

constexpr int kJoinWarps = 8;
constexpr float kLn2 = 0.6931471805599453f;

// Query row blockIdx.y (of its tile of rows) of the sequence and head that begins in block blockIdx.x of the attention kernel and
// goes on behind it, if there is one.  Warps take the parts in turn, a lane four elements: out = sum of the parts'
// means by their weights 2^lse, in the order of the parts within a warp and then of the warps.
template <int DTYPE>
__global__ void __launch_bounds__(kJoinWarps * 32) kv_join_kernel(const Args a, uint32_t dim) {
  __shared__ float sums[kJoinWarps][256];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // (the lengths are there: the attention kernel let this one start when it had waited for them)
  const Share share = a.share(lane);
  const uint32_t first = blockIdx.x * share.per, last = first + share.per;
  Segment s = {};
  if (last < share.total) s = a.find(share, last, lane);
  const uint32_t in_tile = blockIdx.y, r = s.row_tile(a) * a.row_tile + in_tile;
  // every block waits, also one without work: the stream's next kernel goes by this grid's end
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (last >= share.total || s.start < first || s.start >= last || r >= a.rows) return;
  const uint32_t parts = (s.end - 1) / share.per - blockIdx.x + 1;
  // part 0 is the second slot of this block, the others are the first ones of the blocks behind it
  auto slot = [&](uint32_t p) { return (size_t)((blockIdx.x + p) * 2 + (p == 0 ? 1 : 0)) * a.row_tile + in_tile; };
  float top = -INFINITY, total = 0.0f;
#pragma unroll 1
  for (uint32_t p = lane; p < parts; p += 32) top = fmaxf(top, a.part_lse[slot(p)]);
#pragma unroll
  for (int d = 1; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
#pragma unroll 1
  for (uint32_t p = lane; p < parts; p += 32) {
    const float v = a.part_lse[slot(p)];
    total += v == -INFINITY ? 0.0f : exp2f(v - top);
  }
#pragma unroll
  for (int d = 1; d < 32; d *= 2) total += __shfl_xor_sync(0xFFFFFFFFu, total, d);
  for (uint32_t e = lane * 4; e < dim; e += 128) {
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (uint32_t p = warp; p < parts; p += kJoinWarps) {
      const size_t at = slot(p);
      const float v = a.part_lse[at], w = v == -INFINITY ? 0.0f : exp2f(v - top);
      const float4 x = *reinterpret_cast<const float4*>(a.parts + at * dim + e);
      if (v != -INFINITY) {
        sum.x = fmaf(w, x.x, sum.x); sum.y = fmaf(w, x.y, sum.y);
        sum.z = fmaf(w, x.z, sum.z); sum.w = fmaf(w, x.w, sum.w);
      }
    }
    *reinterpret_cast<float4*>(&sums[warp][e]) = sum;
  }
  __syncthreads();
  const uint32_t i = fastdiv(r, a.by_group), head = s.head(a) * a.group + (r - i * a.group);
  const size_t row = ((size_t)s.b * a.new_tokens + i) * a.q_heads + head;
  for (uint32_t e = threadIdx.x; e < dim; e += kJoinWarps * 32) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) v += sums[w][e];
    store1<DTYPE>(a.out, row * dim + e, total == 0.0f ? 0.0f : v / total);
  }
  if (a.lse && threadIdx.x == 0) a.lse[row] = total == 0.0f ? -INFINITY : (top + log2f(total)) * kLn2;
}

// Query rows of a unit: 8, or 16 where there are more (FP32 and rows above 128 elements: 8, for the registers).
uint32_t row_tile(int64_t rows, int64_t dim, bool wide) { return rows > 8 && dim <= 128 && !wide ? 16 : 8; }
size_t part_bytes(uint32_t rows, int64_t dim) { return ((size_t)2 * kCtas * rows * (size_t)(dim + 1) * 4 + 255) / 256 * 256; }

}  // namespace
}  // namespace attn

size_t kv_attention_workspace(const KvArgs& kv) { return attn::part_bytes(16, kv.dim); }

cudaError_t launch_kv_attention(const KvAttentionArgs& a) {
  using namespace attn;
  const bool wide = a.dtype == MX_F32;
  Args k = {};
  k.k_elems = a.kv.k_elems; k.k_scales = a.kv.k_scales; k.v_elems = a.kv.v_elems; k.v_scales = a.kv.v_scales;
  k.q = a.q; k.table = a.table; k.lengths = a.lengths; k.out = a.out; k.lse = a.lse;
  k.q_stride = a.q_stride;
  k.pages = (uint32_t)a.kv.pages; k.page_size = (uint32_t)a.kv.page_size; k.heads = (uint32_t)a.kv.heads;
  k.batch = (uint32_t)a.batch; k.new_tokens = (uint32_t)a.new_tokens; k.q_heads = (uint32_t)a.q_heads;
  k.max_pages = (uint32_t)a.max_pages;
  k.window = (uint32_t)(a.window < 0x7FFFFFFF ? a.window : 0);  // (no sequence is longer)
  k.group = k.q_heads / k.heads;
  k.rows = k.new_tokens * k.group;
  k.row_tile = row_tile(k.rows, a.kv.dim, wide);
  k.row_tiles = (k.rows + k.row_tile - 1) / k.row_tile;
  const int64_t row_bytes = a.kv.dim * (a.kv.fmt == MX_E2M1 ? 4 : 8) / 8;
  k.tile_log2 = (uint32_t)tile_log2((int)row_bytes);
  k.chunk = (k.batch + 31) / 32;
  k.by_page = make_fastdiv(k.page_size); k.by_group = make_fastdiv(k.group); k.by_row_tiles = make_fastdiv(k.row_tiles);
  k.scale_log2 = a.scale * 1.4426950408889634f;
  k.parts = (float*)a.workspace;
  k.part_lse = k.parts + (size_t)2 * kCtas * k.row_tile * (size_t)a.kv.dim;
  const uint32_t ctas = (uint32_t)a.sm_count * 2 < kCtas ? (uint32_t)a.sm_count * 2 : kCtas;
  cudaError_t e;
  switch (a.kv.fmt) {
    case MX_E4M3: e = launch_e4m3(k, (int)a.kv.dim, wide, ctas, a.stream); break;
    case MX_E5M2: e = launch_e5m2(k, (int)a.kv.dim, wide, ctas, a.stream); break;
    case MX_E2M1: e = launch_e2m1(k, (int)a.kv.dim, wide, ctas, a.stream); break;
    default: e = launch_int8(k, (int)a.kv.dim, wide, ctas, a.stream); break;
  }
  if (e != cudaSuccess) return e;
  const dim3 grid(ctas, k.row_tile), block(kJoinWarps * 32);
  return wide ? launch_pdl(kv_join_kernel<MX_F32>, grid, block, 0, a.stream, k, (uint32_t)a.kv.dim)
              : launch_pdl(kv_join_kernel<MX_BF16>, grid, block, 0, a.stream, k, (uint32_t)a.kv.dim);
}

}  // namespace mx
