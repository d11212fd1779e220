// Paged key-value cache of MX rows: quantizing the rows of new tokens into their slots, and reading slots
// back as numbers (see mx_kv_t in mx.h).
//
// Both are streams: append reads 2 or 4 bytes and writes bits / 8 + 1 / 32 per element, read does the
// reverse.  A thread moves 16 elements of a key and of a value, so that what finding a slot's row costs (a division and a few
// multiplications) is paid once for both, and every store is whole sectors: 8192 tokens of 8 heads of 128, BF16 to E4M3, 11.7 us with 8
// elements of either, 9.7 with 8 of both, 7.3 so (inputs that change from call to call: 9.4, 5.4 of the 6.55 TB/s that a copy reaches);
// 16384 tokens back to BF16 24, 21 with half sectors, 13.4 (17.8, 5.7 TB/s).  A whole block a thread: 22.
#include <cuda_fp16.h>

#include "mx_device.cuh"
#include "mx_launch.h"
#include "mx_rows.cuh"

namespace mx {
namespace {

constexpr int kThreads = 256;

struct KvShape {
  int64_t slots;        // pages * page_size
  uint32_t heads, page_size, units, per_token;  // units of a row that threads move, units of a token
  FastDiv by_token, by_row, by_page;
  uint32_t code_bytes, scale_bytes;  // of a row
};

// Row (page * heads + head) * page_size + offset of a slot's token.
__device__ __forceinline__ size_t kv_row(const KvShape& s, uint32_t slot, uint32_t head) {
  const uint32_t page = fastdiv(slot, s.by_page);
  return ((size_t)page * s.heads + head) * s.page_size + (slot - page * s.page_size);
}

// Algorithm 1 of the rows of k and v.  A thread converts 16 elements of either, two neighbours a block; the scale bytes beyond the
// row's blocks are written by the lane of the last block.
template <int FMT, int ROUND, int DTYPE>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(
    const void* __restrict__ k, const void* __restrict__ v, int64_t k_stride, int64_t v_stride, uint8_t* k_elems,
    uint8_t* k_scales, uint8_t* v_elems, uint8_t* v_scales, const int32_t* __restrict__ slots, uint32_t total, KvShape s) {
  pdl_prologue();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  const uint32_t at = i < total ? i : total - 1;  // (two lanes share a block: both of them stay)
  const uint32_t token = fastdiv(at, s.by_token), in_token = at - token * s.per_token;
  Raw8<DTYPE> raw[2][2];
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      raw[n][h] = load_raw8<DTYPE>(n ? v : k, (size_t)token * (size_t)(n ? v_stride : k_stride) + (size_t)in_token * 16 + 8 * h);
  const int64_t slot = slots[token];
  const uint32_t head = fastdiv(in_token, s.by_row), unit = in_token - head * s.units;
  const bool there = i < total && slot >= 0 && slot < s.slots;
  const size_t row = there ? kv_row(s, (uint32_t)slot, head) : 0;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    float x[2][8], amax[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      widen(raw[n][h], x[h]);
      amax[h] = absmax_nan(absmax_nan(absmax_nan(x[h][0], x[h][1]), absmax_nan(x[h][2], x[h][3])),
                           absmax_nan(absmax_nan(x[h][4], x[h][5]), absmax_nan(x[h][6], x[h][7])));
    }
    amax[0] = absmax_nan(amax[0], amax[1]);
    amax[0] = absmax_nan(amax[0], __shfl_xor_sync(0xFFFFFFFFu, amax[0], 1));
    const BlockScale b = block_scale<FMT>(amax[0]);
    uint32_t lo[2], hi[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) cast8<FMT, ROUND>(x[h], b, lo[h], hi[h]);
    if (!there) continue;
    uint8_t* codes = (n ? v_elems : k_elems) + row * s.code_bytes;
    if (FmtTraits<FMT>::bits == 8) reinterpret_cast<uint4*>(codes)[unit] = make_uint4(lo[0], hi[0], lo[1], hi[1]);
    else reinterpret_cast<uint2*>(codes)[unit] = make_uint2(lo[0], lo[1]);
    if (unit % 2 == 0) {
      uint8_t* scales = (n ? v_scales : k_scales) + row * s.scale_bytes;
      scales[unit / 2] = (uint8_t)b.byte;
      if (unit + 2 == s.units)
        for (uint32_t j = unit / 2 + 1; j < s.scale_bytes; ++j) scales[j] = 0;
    }
  }
}

// Two codes as FP32 values; pair = code0 | code1 << 8 (4-bit: both in the low byte).
template <int FMT>
__device__ __forceinline__ float2 decode2(uint32_t pair) {
  if (FMT == MX_INT8)
    return make_float2((float)(int8_t)(pair & 0xFFu) * 0.015625f, (float)(int8_t)(pair >> 8 & 0xFFu) * 0.015625f);
  uint32_t h2;
  const uint16_t p = (uint16_t)pair;
  if (FMT == MX_E4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(p));
  else if (FMT == MX_E5M2) asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h2) : "h"(p));
  else asm("{ .reg .b8 lo, hi; mov.b16 {lo, hi}, %1; cvt.rn.f16x2.e2m1x2 %0, lo; }" : "=r"(h2) : "h"(p));
  return __half22float2(*reinterpret_cast<const __half2*>(&h2));
}

// The rows of a slot as numbers.  A thread reads 16 codes of the key and of the value.
template <int FMT, int DTYPE>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(
    const uint8_t* __restrict__ k_elems, const uint8_t* __restrict__ k_scales, const uint8_t* __restrict__ v_elems,
    const uint8_t* __restrict__ v_scales, const int32_t* __restrict__ slots, uint32_t total, KvShape s, void* k_out, void* v_out) {
  constexpr int kWords = FmtTraits<FMT>::bits / 2;
  pdl_prologue();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= total) return;
  const uint32_t token = fastdiv(i, s.by_token), in_token = i - token * s.per_token;
  const uint32_t head = fastdiv(in_token, s.by_row), unit = in_token - head * s.units;
  const int64_t slot = slots[token];
  uint32_t w[2][kWords] = {}, sb[2] = {0, 0};
  if (slot >= 0 && slot < s.slots) {
    const size_t row = kv_row(s, (uint32_t)slot, head);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint8_t* codes = (n ? v_elems : k_elems) + row * s.code_bytes;
      if (kWords == 4) {
        const uint4 c = ld_16(codes + (size_t)unit * 16);
        w[n][0] = c.x; w[n][1] = c.y; w[n][2 % kWords] = c.z; w[n][3 % kWords] = c.w;
      } else {
        const uint2 c = reinterpret_cast<const uint2*>(codes)[unit];
        w[n][0] = c.x; w[n][1] = c.y;
      }
      sb[n] = ((n ? v_scales : k_scales) + row * s.scale_bytes)[unit / 2];
    }
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const float X = __uint_as_float(sb[n] == 0 ? 0x00400000u : (sb[n] == 255 ? 0x7FC00000u : sb[n] << 23));  // 2^-127, NaN
    float x[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 p = decode2<FMT>(kWords == 4 ? w[n][(2 * h + j / 2) % kWords] >> 16 * (j & 1) : (w[n][h] >> 8 * j) & 0xFFu);
        x[h][2 * j] = p.x * X;
        x[h][2 * j + 1] = p.y * X;
      }
    void* out = n ? v_out : k_out;
    uint16_t* at = (uint16_t*)out + (size_t)i * 16;
    if (DTYPE == MX_BF16 && ((uintptr_t)at & 31u) == 0) {  // a whole sector: two stores would each write half of every one
      uint32_t o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = pack_bf16(x[j / 4][2 * (j % 4)], x[j / 4][2 * (j % 4) + 1]);
      st_32(at, o);
    } else {
      store8<DTYPE>(out, (size_t)i * 16, x[0]);
      store8<DTYPE>(out, (size_t)i * 16 + 8, x[1]);
    }
  }
}

// Shape of the cache with rows cut into units of so many elements.
KvShape shape_of(const KvArgs& kv, uint32_t unit) {
  KvShape s;
  const uint32_t bits = kv.fmt == MX_E2M1 ? 4 : 8;
  s.slots = kv.pages * kv.page_size;
  s.heads = (uint32_t)kv.heads;
  s.page_size = (uint32_t)kv.page_size;
  s.units = (uint32_t)kv.dim / unit;
  s.per_token = s.units * s.heads;
  s.by_token = make_fastdiv(s.per_token);
  s.by_row = make_fastdiv(s.units);
  s.by_page = make_fastdiv(s.page_size);
  s.code_bytes = (uint32_t)kv.dim * bits / 8;
  s.scale_bytes = ((uint32_t)kv.dim + 127) / 128 * 4;
  return s;
}

template <int FMT, int ROUND>
cudaError_t append_by_dtype(const KvMoveArgs& a, const KvShape& s, uint32_t total) {
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((total + kThreads - 1) / kThreads), dim3(kThreads), 0, a.stream, a.k, a.v, a.k_stride, a.v_stride,
                      a.kv.k_elems, a.kv.k_scales, a.kv.v_elems, a.kv.v_scales, a.slots, total, s);
  };
  return a.dtype == MX_BF16 ? go(kv_append_kernel<FMT, ROUND, MX_BF16>) : go(kv_append_kernel<FMT, ROUND, MX_F32>);
}
template <int FMT>
cudaError_t append_by_rounding(const KvMoveArgs& a, const KvShape& s, uint32_t total) {
  return a.rounding == MX_RNE ? append_by_dtype<FMT, MX_RNE>(a, s, total) : append_by_dtype<FMT, MX_RHAZ>(a, s, total);
}
template <int FMT>
cudaError_t read_by_dtype(const KvMoveArgs& a, const KvShape& s, uint32_t total) {
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((total + kThreads - 1) / kThreads), dim3(kThreads), 0, a.stream, a.kv.k_elems, a.kv.k_scales,
                      a.kv.v_elems, a.kv.v_scales, a.slots, total, s, a.k_out, a.v_out);
  };
  return a.dtype == MX_BF16 ? go(kv_read_kernel<FMT, MX_BF16>) : go(kv_read_kernel<FMT, MX_F32>);
}

}  // namespace

cudaError_t launch_kv_append(const KvMoveArgs& a) {
  const KvShape s = shape_of(a.kv, 16);
  const uint32_t total = (uint32_t)(a.tokens * a.kv.heads * (a.kv.dim / 16));  // below 2^31
  switch (a.kv.fmt) {
    case MX_E4M3: return append_by_rounding<MX_E4M3>(a, s, total);
    case MX_E5M2: return append_by_rounding<MX_E5M2>(a, s, total);
    case MX_E2M1: return append_by_rounding<MX_E2M1>(a, s, total);
    default: return append_by_rounding<MX_INT8>(a, s, total);
  }
}

cudaError_t launch_kv_read(const KvMoveArgs& a) {
  const KvShape s = shape_of(a.kv, 16);
  const uint32_t total = (uint32_t)(a.tokens * a.kv.heads * (a.kv.dim / 16));
  switch (a.kv.fmt) {
    case MX_E4M3: return read_by_dtype<MX_E4M3>(a, s, total);
    case MX_E5M2: return read_by_dtype<MX_E5M2>(a, s, total);
    case MX_E2M1: return read_by_dtype<MX_E2M1>(a, s, total);
    default: return read_by_dtype<MX_INT8>(a, s, total);
  }
}

}  // namespace mx
