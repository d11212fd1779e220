// mx_kv_attention: its workspace, the choice of an instance, and the kernel that joins the parts of sequences that more than one
// block worked on (the attention itself: mx_kv_attention.cuh).
#include <math.h>

#include "mx_kv_attention_args.h"
#include "mx_launch.h"
#include "mx_rows.cuh"

namespace mx {
namespace attn {
namespace {

constexpr int kJoinWarps = 8;
constexpr float kLn2 = 0.6931471805599453f;

// A few query rows (ROWS of their tile of rows, the ones blockIdx.y * ROWS ..) of the sequence and head that begins in block blockIdx.x
// of the attention kernel and goes on behind it, if there is one; with by_segment of the blockIdx.x-th of all.  The warps of a row take its parts in turn, a lane four elements:
// out = sum of the parts' means by their weights 2^lse over the sum of the weights, in the order of the parts within a warp and
// then of the warps.
template <int DTYPE, int ROWS>
__global__ void __launch_bounds__(kJoinWarps * 32) kv_join_kernel(const Args a, uint32_t dim) {
  constexpr uint32_t kPer = kJoinWarps / ROWS;  // warps of a row
  __shared__ float4 sums[kJoinWarps][64];
  __shared__ float2 weights[kJoinWarps];        // the largest lse of a warp's parts, the sum of their weights
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // Sequences without a token to see, which have no tile.  (The lengths are there: the attention kernel let this one start when
  // it had waited for them.)
  const uint32_t rows = a.new_tokens * a.q_heads;
  for (uint32_t b = blockIdx.y * gridDim.x + blockIdx.x; b < a.batch; b += gridDim.x * gridDim.y) {
    if (a.tiles(a.length(b)) != 0) continue;
    for (uint32_t i = threadIdx.x; i < rows * (dim / 8); i += kJoinWarps * 32) {
      const float zero[8] = {};
      store8<DTYPE>(a.out, (size_t)b * rows * dim + (size_t)i * 8, zero);
    }
    if (a.lse)
      for (uint32_t i = threadIdx.x; i < rows; i += kJoinWarps * 32) a.lse[(size_t)b * rows + i] = -INFINITY;
  }
  // every block waits, also one without work: the stream's next kernel goes by this grid's end
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (a.by_segment && a.tiles(a.length(blockIdx.x / (a.heads * a.row_tiles))) == 0) return;  // (nobody has written its entry)
  const Unfinished s = a.unfinished[blockIdx.x];
  if (s.parts == 0) return;
  const uint32_t head0 = fastdiv(s.hr, a.by_row_tiles), row_tile = s.hr - head0 * a.row_tiles;
  const uint32_t in_tile = blockIdx.y * ROWS + warp / kPer, r = row_tile * kRows + in_tile;
  float top = -INFINITY, total = 0.0f;
  float4 sum[2] = {};
  if (r < a.rows) {
    constexpr int kBatch = 8;  // parts in flight
#pragma unroll 1
    for (uint32_t p0 = warp % kPer; p0 < s.parts; p0 += kPer * kBatch) {
      float lse[kBatch];
      float4 x[kBatch][2];
      float most = top;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const uint32_t p = p0 + k * kPer;
        lse[k] = -INFINITY;
        x[k][0] = x[k][1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p < s.parts) {
          // part 0 is the second slot of this block, the others are the first ones of the blocks behind it
          const size_t at = (size_t)((s.block + p) * 2 + (p == 0 ? 1 : 0)) * kRows + in_tile;
          lse[k] = a.part_lse[at];
          if (lane * 4 < dim) x[k][0] = *reinterpret_cast<const float4*>(a.parts + at * dim + lane * 4);
          if (lane * 4 + 128 < dim) x[k][1] = *reinterpret_cast<const float4*>(a.parts + at * dim + lane * 4 + 128);
        }
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) most = fmaxf(most, lse[k]);
      const float keep = top == -INFINITY ? 0.0f : exp2f(top - most);
      top = most;
      total *= keep;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sum[h].x *= keep; sum[h].y *= keep; sum[h].z *= keep; sum[h].w *= keep;
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (lse[k] == -INFINITY) continue;  // nothing seen in this part
        const float w = exp2f(lse[k] - top);
        total += w;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          sum[h].x = fmaf(w, x[k][h].x, sum[h].x); sum[h].y = fmaf(w, x[k][h].y, sum[h].y);
          sum[h].z = fmaf(w, x[k][h].z, sum[h].z); sum[h].w = fmaf(w, x[k][h].w, sum[h].w);
        }
      }
    }
  }
  sums[warp][lane] = sum[0];
  sums[warp][32 + lane] = sum[1];
  if (lane == 0) weights[warp] = make_float2(top, total);
  __syncthreads();
  // a row's warps put out a part of it each
  const uint32_t w0 = warp / kPer * kPer;
  float most = -INFINITY, all = 0.0f, by[kPer];
#pragma unroll
  for (uint32_t w = 0; w < kPer; ++w) most = fmaxf(most, weights[w0 + w].x);
#pragma unroll
  for (uint32_t w = 0; w < kPer; ++w) {
    const float2 v = weights[w0 + w];
    by[w] = v.y == 0.0f ? 0.0f : exp2f(v.x - most);
    all += v.y * by[w];
  }
  if (r >= a.rows) return;
  const uint32_t i = fastdiv(r, a.by_group), head = head0 * a.group + (r - i * a.group);
  const size_t row = ((size_t)s.b * a.new_tokens + i) * a.q_heads + head;
  for (uint32_t e = warp % kPer * 32 + lane; e < dim / 4; e += kPer * 32) {
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (uint32_t w = 0; w < kPer; ++w) {
      const float4 u = sums[w0 + w][e];
      if (by[w] == 0.0f) continue;
      v.x = fmaf(by[w], u.x, v.x); v.y = fmaf(by[w], u.y, v.y);
      v.z = fmaf(by[w], u.z, v.z); v.w = fmaf(by[w], u.w, v.w);
    }
    const float whole = all == 0.0f ? 0.0f : 1.0f / all;
    v.x *= whole; v.y *= whole; v.z *= whole; v.w *= whole;
    if (DTYPE == MX_BF16) *reinterpret_cast<uint2*>((uint16_t*)a.out + row * dim + e * 4) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    else *reinterpret_cast<float4*>((float*)a.out + row * dim + e * 4) = v;
  }
  if (a.lse && warp % kPer == 0 && lane == 0) a.lse[row] = all == 0.0f ? -INFINITY : (most + log2f(all)) * kLn2;
}

// Sequences of up to so many tiles are not split, more where there are blocks enough without: eight rounds of a block's warps take less than
// a split and a second kernel (8 heads of 128, 16 sequences to 450 tokens 8.8 against 12.3 us, to 900 13.3 against 14.9, to 1800 21 against 17; 64
// sequences to 900 24 against 32, to 1800 41 against 44, to 4000 78 against 67; 128 sequences to 1800 63 against 72, to 4000 121 against 124).
// At most four times that: one long sequence among many short ones would keep its block long after all others.  What counts is what the table could
// hold, not the lengths, which the host does not know: in a table for 131072 tokens 333 tokens take 10.6 us instead of 7.2, 64 sequences to 450
// 27 instead of 16, to 900 33 instead of 24.  (All measured on 8-bit rows of 128 and BF16 results.)
constexpr int64_t kWhole = 8 * kWarps;

size_t workspace_bytes(int64_t dim) { return kCtas * (sizeof(Unfinished) + (size_t)2 * kRows * (size_t)(dim + 1) * 4); }

}  // namespace
}  // namespace attn

size_t kv_attention_workspace(const KvArgs& kv) { return attn::workspace_bytes(kv.dim); }

cudaError_t launch_kv_attention(const KvAttentionArgs& a) {
  using namespace attn;
  const bool wide = a.dtype == MX_F32;
  Args k = {};
  k.k_elems = a.kv.k_elems; k.k_scales = a.kv.k_scales; k.v_elems = a.kv.v_elems; k.v_scales = a.kv.v_scales;
  k.q = a.q; k.table = a.table; k.lengths = a.lengths; k.out = a.out; k.lse = a.lse;
  k.q_stride = a.q_stride;
  k.pages = (uint32_t)a.kv.pages; k.page_size = (uint32_t)a.kv.page_size; k.heads = (uint32_t)a.kv.heads;
  k.batch = (uint32_t)a.batch; k.new_tokens = (uint32_t)a.new_tokens; k.q_heads = (uint32_t)a.q_heads;
  k.max_pages = a.kv.pages > 0 ? (uint32_t)a.max_pages : 0;  // (no page: nobody sees a token)
  k.window = (uint32_t)(a.window < 0x7FFFFFFF ? a.window : 0);  // (no sequence is longer)
  k.group = k.q_heads / k.heads;
  k.rows = k.new_tokens * k.group;
  k.tile_log2 = (uint32_t)tile_log2((int)a.kv.dim, a.kv.fmt == MX_E2M1 ? 4 : 8);
  // no sequence has more tiles than this
  const int64_t cap = (int64_t)k.max_pages * a.kv.page_size, reach = k.window ? (int64_t)k.window + k.new_tokens : cap;
  const int64_t tiles = ((reach < cap ? reach : cap) >> k.tile_log2) + 2;
  k.row_tiles = (k.rows + kRows - 1) / kRows;
  k.chunk = (k.batch + 31) / 32;
  k.by_page = make_fastdiv(k.page_size); k.by_group = make_fastdiv(k.group); k.by_row_tiles = make_fastdiv(k.row_tiles);
  k.scale_mant = frexpf(a.scale, &k.scale_exp) * 1.4426950408889634f;  // (the product itself may be out of range)
  k.unfinished = (Unfinished*)a.workspace;
  k.parts = (float*)(k.unfinished + kCtas);
  k.part_lse = k.parts + (size_t)2 * kCtas * kRows * (size_t)a.kv.dim;
  const uint32_t segments = k.batch * k.heads * k.row_tiles;  // (below 2^31, as the units are)
  const uint32_t most = (uint32_t)(a.sm_count * blocks_per_sm((int)a.kv.dim, wide));
  // no more blocks than the longest sequences would employ; with few tiles a block for each segment
  const int64_t units = (int64_t)segments * tiles;
  uint32_t ctas = most < kCtas ? most : kCtas;
  k.whole = tiles <= kWhole * (segments / ctas < 3 ? 1 + segments / ctas : 4);
  if (units < (int64_t)ctas * kLeast) ctas = (uint32_t)((units + kLeast - 1) / kLeast);
  if (k.whole) ctas = segments;
  // Few sequences and heads may have many parts each: a block of the join for every row of each.  Many have few: blocks of four rows
  // for each block of this kernel.
  k.by_segment = segments * 8 <= kCtas;
  k.by_grid = make_fastdiv(ctas);
  cudaError_t e;
  switch (a.kv.fmt) {
    case MX_E4M3: e = launch_e4m3(k, (int)a.kv.dim, wide, ctas, a.stream); break;
    case MX_E5M2: e = launch_e5m2(k, (int)a.kv.dim, wide, ctas, a.stream); break;
    case MX_E2M1: e = launch_e2m1(k, (int)a.kv.dim, wide, ctas, a.stream); break;
    default: e = launch_int8(k, (int)a.kv.dim, wide, ctas, a.stream); break;
  }
  if (e != cudaSuccess || k.whole) return e;
  auto join = [&](auto kernel, uint32_t blocks, uint32_t rows) {
    return launch_pdl(kernel, dim3(blocks, kRows / rows), dim3(kJoinWarps * 32), 0, a.stream, k, (uint32_t)a.kv.dim);
  };
  if (wide) return k.by_segment ? join(kv_join_kernel<MX_F32, 1>, segments, 1) : join(kv_join_kernel<MX_F32, 4>, ctas, 4);
  return k.by_segment ? join(kv_join_kernel<MX_BF16, 1>, segments, 1) : join(kv_join_kernel<MX_BF16, 4>, ctas, 4);
}

}  // namespace mx
