// Internal interface between the C ABI (mx_api.cu) and the kernel files.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "mx.h"

namespace mx {

struct QuantizeArgs {
  const void* in;
  uint8_t* elems;
  uint8_t* scales;
  int64_t outer, L, inner;  // input viewed as [outer, L, inner], blocks along L
  int64_t L_store;          // elements per stored row: L rounded up to whole blocks, or to 128 (zero codes)
  int64_t numel;
  int fmt, rounding, dtype, layout;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_quantize(const QuantizeArgs& a);

struct DualArgs {
  const void* in;
  uint8_t *elems_row, *scales_row;  // blocks along the contiguous axis: [R x C]
  uint8_t *elems_col, *scales_col;  // blocks along axis 0: [C x R]
  int64_t R, C;
  int fmt, rounding, dtype, layout;
  int sm_count;
  cudaStream_t stream;
};
// FP32 input, register kernel (mx_quantize_dual.cu).
cudaError_t launch_quantize_dual(const DualArgs& a);
// The same for BF16 input through TMA tiles in shared memory (mx_quantize_tile.cu).
cudaError_t launch_quantize_tile(const DualArgs& a);
// FP32 input, 6-bit codes, R and C multiples of 128, through the same kind of kernel.
cudaError_t launch_quantize_tile_f32(const DualArgs& a);
// The BF16 kernel's column pass alone (elems_row / scales_row unused): axis-0 quantize of a 2-D BF16
// tensor with 6- or 4-bit codes, R, C % 128 == 0.
cudaError_t launch_quantize_tile_cols(const DualArgs& a);
// Synchronises the stream, then reads and clears the tile kernels' status word (nonzero: a
// bounded device-side wait gave up).
cudaError_t quantize_tile_status(cudaStream_t stream, unsigned int* status);

struct DequantizeArgs {
  const uint8_t* elems;
  const uint8_t* scales;
  void* out;
  int64_t rows, L;
  int fmt, dtype, layout;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_dequantize(const DequantizeArgs& a);

// Activation x[N, H, W, C] quantized along C -> K-major operand [N Ho Wo x kh kw C] (see mx_im2col()).
struct Im2colArgs {
  const uint8_t* elems_in;
  const uint8_t* scales_in;
  uint8_t* elems_out;
  uint8_t* scales_out;  // swizzled
  int64_t N, H, W, C, Ho, Wo;
  int kh, kw, stride_h, stride_w, pad_h, pad_w, dil_h, dil_w;
  int bits, layout_in;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_im2col(const Im2colArgs& a);

// Convolution without a materialized operand (see mx_conv2d()): x quantized along C (8-bit codes),
// filter w[Cout][kh kw C] quantized along its last axis (any block-scaled format, swizzled scales).
struct ConvArgs {
  const uint8_t* x_elems;
  const uint8_t* x_scales;
  const void* w_elems;
  const uint8_t* w_scales;
  void* y;  // FP32 or BF16 [N Ho Wo x Cout]
  int y_bf16;
  int64_t N, H, W, C, Ho, Wo, Cout;
  int kh, kw, stride_h, stride_w, pad_h, pad_w, dil_h, dil_w;
  int fmt_x, fmt_w, x_layout;
  int sm_count;
  cudaStream_t stream;
};
// Returns MX_OK or a negative mx_status_t; fills *cuda_err on MX_ERR_CUDA.
int launch_conv(const ConvArgs& a, cudaError_t* cuda_err);

struct GemmArgs {
  const void* A;
  const uint8_t* sA;
  const void* B;
  const uint8_t* sB;
  void* C;      // FP32 [M x N], or BF16 when c_bf16 is nonzero
  int c_bf16;
  // When q_elems is set the epilogue quantizes C along N instead of storing it: packed codes
  // [batch*M x N] and swizzled scales (rows batch*M, N / 32 blocks); C is then unused.
  void* q_elems;
  uint8_t* q_scales;
  int q_fmt, q_round;
  // dense != 0: A and B are BF16 K-major matrices (dequantized MX tensors), sA / sB unused.
  int dense;
  int64_t batch;  // independent products; operands and C are the matrices stacked along rows
  int64_t M, N, K;
  int fmtA, fmtB;
  int force_bn;  // 0: let launch_gemm choose the tile width; 256 / 384: pin it (tuning and tests)
  int skinny_m;  // products with M <= skinny_m (at most 128) take the swapped-operand kernel
  int64_t wait_cycles;  // budget of a device-side wait in SM clock cycles; <= 0: the default (~1 s)
  int drop_fill;        // failure drill: the operand producer leaves out this pipeline fill; < 0: off
  int sm_count;
  cudaStream_t stream;
};
// Returns MX_OK or a negative mx_status_t; fills *cuda_err on MX_ERR_CUDA.
int launch_gemm(const GemmArgs& a, cudaError_t* cuda_err);
// Synchronises the stream, then reads and clears the per-device status word that a
// bounded device-side wait sets when it gives up (0 = every wait completed).
int gemm_status(cudaStream_t stream, unsigned int* status, cudaError_t* cuda_err);

struct RmsnormArgs {
  const void *x, *residual, *weight;
  void *h_out, *y_out;
  uint8_t *elems, *scales;
  int64_t rows, dim;
  float eps;
  int w_bf16, fmt, rounding, dtype, layout;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_rmsnorm_quantize(const RmsnormArgs& a);
// Shared memory that a row takes in the forward kernel for rows of any length: FP32, whole runs of 128
// elements, for BF16 rows a word more after every 8.  In 64 bits: a row may have 2^31 - 1 elements.  Rows
// beyond kNormRowBytes take the kernel that reads them twice.
constexpr uint64_t kNormRowBytes = 200 * 1024;
constexpr uint64_t norm_row_bytes(bool bf16, int64_t dim) {
  const uint64_t padded = ((uint64_t)dim + 127) / 128 * 128;
  return 4 * (bf16 ? padded + padded / 8 : padded);
}

// Partial sums of the weight gradient (rows of `partial`) that the backward pass writes at most.
constexpr int kNormPartials = 296;
struct RmsnormBackwardArgs {
  const void *dy, *h, *weight, *dres;
  void* dh;
  float* dweight;
  float* partial;   // [kNormPartials x dim]
  float2* stats;    // [rows]
  int64_t rows, dim;
  float eps;
  int w_bf16, dtype;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_rmsnorm_backward(const RmsnormBackwardArgs& a);

struct RouteArgs {
  const void* logits;
  const float* bias;
  const float* dweights;  // backward only
  int32_t* ids;           // written forward, read backward
  float* weights;
  void* dlogits;
  int64_t tokens, experts;
  mx_route_t route;
  int dtype;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_route(const RouteArgs& a);
cudaError_t launch_route_backward(const RouteArgs& a);

constexpr int kPlanChunk = 1024;  // choices that one CTA of the plan sorts
struct MoePlanArgs {
  const int32_t* ids;
  int32_t *offsets, *counts, *row_of, *src_of, *hist;  // hist: [chunks + 1 x experts]
  int64_t n, experts, align, rows;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_moe_plan(const MoePlanArgs& a);

struct MoeMoveArgs {
  const void *src, *y;       // rows of the tokens (MX codes or floats); combine: src unused
  const uint8_t* scales_in;
  const float* weights;
  const int32_t *offsets, *counts, *row_of, *src_of;
  void* dst;
  uint8_t* scales_out;
  float* dweights;
  int64_t tokens, topk, dim, experts, rows;
  int bits, dtype, layout;
  int sm_count;
  cudaStream_t stream;
};
cudaError_t launch_moe_gather(const MoeMoveArgs& a);
cudaError_t launch_moe_combine(const MoeMoveArgs& a);
cudaError_t launch_moe_combine_backward(const MoeMoveArgs& a);

// The experts' products (see mx_gemm_grouped() and mx_gemm_grouped_k()).  W is the operand on the
// M side of the MMA, X the ragged one on its N side; C is [.. x X rows x W rows].
struct GroupedArgs {
  const void *W, *X;
  const uint8_t *sW, *sX;
  const int32_t* offsets;
  void* C;
  int c_bf16;
  int k_groups;  // 0: groups of X rows, each with w_rows rows of W; 1: groups along K
  int64_t groups, w_rows, x_rows, K;
  int fmtW, fmtX;
  int64_t wait_cycles;  // budget of a wait in clocks; 0: the library's
  int drop_fill;        // failure drill: the operand copies leave out this fill of a stage; < 0: off
  int sm_count;
  cudaStream_t stream;
};
int launch_gemm_grouped(const GroupedArgs& a, cudaError_t* cuda_err);
int gemm_grouped_status(cudaStream_t stream, unsigned int* status, cudaError_t* cuda_err);

// The paged cache (see mx_kv_t).  A row is a token's codes for one head; rows are numbered
// (page * heads + head) * page_size + offset.
struct KvArgs {
  uint8_t *k_elems, *k_scales, *v_elems, *v_scales;
  int64_t pages, page_size, heads, dim;
  int fmt;
};
struct KvMoveArgs {
  KvArgs kv;
  const void *k, *v;       // append: rows to quantize
  void *k_out, *v_out;     // read: rows as numbers
  int64_t k_stride, v_stride;
  const int32_t* slots;
  int64_t tokens;
  int rounding, dtype;
  cudaStream_t stream;
};
cudaError_t launch_kv_append(const KvMoveArgs& a);
cudaError_t launch_kv_read(const KvMoveArgs& a);

struct KvAttentionArgs {
  KvArgs kv;
  const void* q;
  const int32_t *table, *lengths;
  void* out;
  float* lse;              // may be null
  void* workspace;
  int64_t batch, new_tokens, q_heads, max_pages, q_stride, window;
  float scale;
  int dtype;
  int sm_count;
  cudaStream_t stream;
};
size_t kv_attention_workspace(const KvArgs& kv);
cudaError_t launch_kv_attention(const KvAttentionArgs& a);

}  // namespace mx
