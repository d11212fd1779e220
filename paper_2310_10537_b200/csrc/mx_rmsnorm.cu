// RMS norm with the residual's addition and MX output, and its backward pass.
//
//   h = x + residual;  s = rsqrt(mean(h^2) + eps);  y = h s w;  (P, X) = Algorithm 1 (y)
//
// Forward: one CTA per row.  The row is read once and stays in registers (FP32) while its sum of
// squares is formed, so that the traffic is x, residual in and h, codes, scales out; a thread holds
// groups of 8 consecutive elements, four neighbouring lanes an MX block, whose maximum takes two
// shuffles.  y is never rounded before Algorithm 1.  Bound by memory: 8192 x 8192 BF16 with residual, E4M3 out, 77.7 to 84.1 us,
// 5.6 to 6.07 TB/s of those bytes (a copy: 6.46); 8192 x 4096 40.7 us; 16 x 4096 2.6 us, of which launch, two barriers and one latency of memory.
#include <cuda_runtime.h>

#include "mx.h"
#include "mx_device.cuh"
#include "mx_launch.h"
#include "mx_rows.cuh"

namespace mx {
namespace {

struct NormParams {
  const void *x, *residual, *weight;
  void *h_out, *y_out;
  uint8_t *elems, *scales;
  uint32_t rows, dim, kblocks;
  float eps, inv_dim;
  uint32_t w_bf16, sticky, layout;
};

// 8 weights; the weights are shared by all rows and stay in the L1
__device__ __forceinline__ void load_weight8(const void* w, uint32_t w_bf16, uint32_t elem, float (&f)[8]) {
  if (w_bf16) {
    widen4(__ldg(reinterpret_cast<const uint4*>((const char*)w + (size_t)elem * 2)), f);
  } else {
    const float4 a = __ldg(reinterpret_cast<const float4*>((const char*)w + (size_t)elem * 4));
    const float4 b = __ldg(reinterpret_cast<const float4*>((const char*)w + (size_t)elem * 4) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
}
__device__ __forceinline__ float weight1(const void* w, uint32_t w_bf16, uint32_t c) {
  return w_bf16 ? __uint_as_float((uint32_t)__ldg((const uint16_t*)w + c) << 16) : __ldg((const float*)w + c);
}

// The elements at .. at + 7 of a BF16 tensor of `all` elements; those past its end are zero.
__device__ __forceinline__ uint4 load_part8(const void* base, size_t at, size_t all) {
  uint32_t w[4] = {};
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e)
    if (at + e < all) w[e >> 1] |= (uint32_t)((const uint16_t*)base)[at + e] << (16 * (e & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Sum over the CTA; every thread gets it.  `red` holds a float per warp and is not read again by
// the caller before its next barrier.
__device__ __forceinline__ float cta_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const uint32_t warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = lane < warps ? red[lane] : 0.0f;
#pragma unroll
  for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  return t;
}

template <int FMT>
__device__ __forceinline__ void cast8_sticky(const float (&v)[8], const BlockScale& s, uint32_t sticky, uint32_t& lo,
                                             uint32_t& hi) {
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = mul_ftz(v[2 * i], s.m1), b = mul_ftz(v[2 * i + 1], s.m1);
    if (FMT == MX_INT8) { a *= s.m2; b *= s.m2; }
    // ties away from zero: the last mantissa bit set moves a tie past the half-way point (see cast_pair)
    a = __uint_as_float(__float_as_uint(a) | sticky);
    b = __uint_as_float(__float_as_uint(b) | sticky);
    p[i] = cast_pair<FMT, MX_RNE>(a, b);
  }
  pack8<FMT>(p, lo, hi);
  if (!s.finite) { lo = 0; hi = 0; }
}

__device__ __forceinline__ size_t scale_at(const NormParams& p, uint32_t row, uint32_t kb) {
  return p.layout == MX_SCALES_LINEAR ? scale_offset<MX_SCALES_LINEAR>(row, kb, p.kblocks)
                                      : scale_offset<MX_SCALES_SWIZZLED>(row, kb, p.kblocks);
}

// The scale words of the rows that pad a swizzled scale tensor to 128 rows, spread over the grid.
__device__ __forceinline__ void zero_pad_rows(const NormParams& p) {
  if (p.layout != MX_SCALES_SWIZZLED) return;
  const uint32_t pad = (0u - p.rows) & 127u, kchunks = (p.kblocks + 3) >> 2;
  for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < pad * kchunks; i += gridDim.x * blockDim.x) {
    const uint32_t r = i / kchunks, c = i - r * kchunks;
    *reinterpret_cast<uint32_t*>(p.scales + scale_offset<MX_SCALES_SWIZZLED>(p.rows + r, 4 * c, p.kblocks)) = 0u;
  }
}

// Quantizes the group g of 8 values of a row whose blocks are four neighbouring lanes' groups, and stores its codes
// and the block's scale (with the swizzled layout also the zero bytes up to whole words).
template <int FMT>
__device__ __forceinline__ void store_group(const NormParams& p, uint32_t row, uint8_t* out_row, uint32_t g,
                                            const float (&v)[8]) {
  constexpr uint32_t bits = FmtTraits<FMT>::bits;
  const uint32_t lane = threadIdx.x & 31, groups_stored = p.kblocks * 4;
  float m[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) m[e] = absmax_nan(v[2 * e], v[2 * e + 1]);
  float am = absmax_nan(absmax_nan(m[0], m[1]), absmax_nan(m[2], m[3]));
  am = absmax_nan(am, __shfl_xor_sync(0xffffffffu, am, 1));
  am = absmax_nan(am, __shfl_xor_sync(0xffffffffu, am, 2));
  const BlockScale bs = block_scale<FMT>(am);
  uint32_t lo, hi;
  cast8_sticky<FMT>(v, bs, p.sticky, lo, hi);
  if constexpr (bits == 6) {  // two lanes' 48 bits each fill three words
    const uint32_t lo_next = __shfl_down_sync(0xffffffffu, lo, 1);
    if (g < groups_stored) {
      uint32_t* d = reinterpret_cast<uint32_t*>(out_row + 12 * (size_t)(g >> 1));
      if ((lane & 1) == 0) {
        d[0] = lo;
        d[1] = __byte_perm(hi, lo_next, 0x5410);
      } else {
        d[2] = __byte_perm(lo, hi, 0x5432);
      }
    }
  } else if (g < groups_stored) {
    if constexpr (bits == 8) *reinterpret_cast<uint2*>(out_row + 8 * (size_t)g) = make_uint2(lo, hi);
    else *reinterpret_cast<uint32_t*>(out_row + 4 * (size_t)g) = lo;
  }
  const uint32_t kb = g >> 2;
  if ((lane & 3) == 0) {
    if (kb < p.kblocks) p.scales[scale_at(p, row, kb)] = (uint8_t)bs.byte;
    else if (p.layout == MX_SCALES_SWIZZLED && kb < ((p.kblocks + 3) & ~3u)) p.scales[scale_at(p, row, kb)] = 0;
  }
}

// dim % 8 == 0 and dim <= 8 * V * blockDim: the row in registers.
template <int DTYPE, int FMT, int V>
__global__ void __launch_bounds__(V == 4 ? 512 : 1024) rmsnorm_kernel(const NormParams p) {
  constexpr uint32_t bits = FmtTraits<FMT>::bits;
  __shared__ float red[32];
  pdl_prologue();
  const uint32_t T = blockDim.x, row = blockIdx.x;
  const size_t base = (size_t)row * p.dim;
  const uint32_t groups = p.dim >> 3;                 // of 8 elements that exist
  const uint32_t groups_stored = p.kblocks * 4;       // whole blocks: the last one padded with zeros
  float v[V][8];
  float ss = 0.0f;
  {
    Raw8<DTYPE> a[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t g = i * T + threadIdx.x;
      if (g < groups) {
        a[i] = load_raw8<DTYPE>(p.x, base + 8 * (size_t)g);
        if (p.residual) b[i] = load_raw8<DTYPE>(p.residual, base + 8 * (size_t)g);
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t g = i * T + threadIdx.x;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
      if (g < groups) {
        widen<DTYPE>(a[i], v[i]);
        if (p.residual) {
          float r[8];
          widen<DTYPE>(b[i], r);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e] += r[e];
        }
        if (p.h_out) store8<DTYPE>(p.h_out, base + 8 * (size_t)g, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
      }
    }
  }
  const float s = rsqrtf(cta_sum(ss, red) * p.inv_dim + p.eps);
  uint8_t* out_row = p.elems + (size_t)row * p.kblocks * (4 * bits);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t g = i * T + threadIdx.x;
    if (i * T + (threadIdx.x & ~31u) >= ((groups_stored + 15) & ~15u)) break;  // warp-uniform
    if (g < groups) {
      float w[8];
      load_weight8(p.weight, p.w_bf16, 8 * g, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * s * w[e];
      if (p.y_out) store8<DTYPE>(p.y_out, base + 8 * (size_t)g, v[i]);
    }
    store_group<FMT>(p, row, out_row, g, v[i]);
  }
  zero_pad_rows(p);
}

// Any dim that fits shared memory: rows start anywhere.  h is formed once, stored, and waits in shared memory as FP32,
// from where it is quantized in groups of 8 like the rows above (both types sum the squares in the same order).  x, residual and h_out lie alike relative to 16 bytes, so BF16 rows move in the
// aligned vectors that cover them -- only the first and the last of a row go by elements -- and shared memory skips a
// word after every 8, which keeps both the shifted writes and the groups' reads free of bank conflicts.  FP32 rows move an
// element per lane, whole sectors (in vectors of 8 the registers leave too few threads: 8192 x 4001 104 us instead of 73).
// (8192 x 4001 BF16: 69 us; 114 an element per lane, 165 with a second pass over memory.)
template <int DTYPE> __host__ __device__ constexpr uint32_t any_at(uint32_t c) { return DTYPE == MX_BF16 ? c + (c >> 3) : c; }

template <int DTYPE>
__device__ __forceinline__ void any_group(const float* h, uint32_t g, float (&v)[8]) {
  if constexpr (DTYPE == MX_BF16) {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) v[e] = h[9 * g + e];
  } else {
    const float4 a = reinterpret_cast<const float4*>(h)[2 * g], b = reinterpret_cast<const float4*>(h)[2 * g + 1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

template <int DTYPE, int FMT, uint32_t T>
__global__ void __launch_bounds__(T) rmsnorm_any_kernel(const NormParams p) {
  constexpr uint32_t bits = FmtTraits<FMT>::bits;
  extern __shared__ float4 row_smem[];
  __shared__ float red[32];
  float* h = reinterpret_cast<float*>(row_smem);  // element c at any_at(c), up to dim rounded up to 128
  pdl_prologue();
  const uint32_t row = blockIdx.x, groups = (p.kblocks + 3) / 4 * 16;
  const size_t base = (size_t)row * p.dim;
  float ss = 0.0f;
  if constexpr (DTYPE == MX_BF16) {
    const uint32_t shift = (uint32_t)(base & 7u), vecs = (p.dim + shift + 7) >> 3;
    const size_t first = base - shift, all = (size_t)p.rows * p.dim;  // element 0 of vector 0; of the tensor
    constexpr uint32_t U = 4;
    for (uint32_t j0 = threadIdx.x; j0 < vecs; j0 += U * T) {
      uint4 v[U], q[U];  // (loads first: h_out may be x or residual)
#pragma unroll
      for (uint32_t k = 0; k < U; ++k) {
        const uint32_t j = j0 + T * k;
        const size_t at = first + 8 * (size_t)j;
        v[k] = q[k] = make_uint4(0, 0, 0, 0);
        if (j < vecs && at + 8 <= all) {
          v[k] = ld_16((const uint16_t*)p.x + at);
          if (p.residual) q[k] = ld_16((const uint16_t*)p.residual + at);
        } else if (j < vecs) {  // the last row's end
          v[k] = load_part8(p.x, at, all);
          if (p.residual) q[k] = load_part8(p.residual, at, all);
        }
      }
#pragma unroll
      for (uint32_t k = 0; k < U; ++k) {
        const uint32_t j = j0 + T * k;
        if (j >= vecs) break;
        float f[8], g[8];
        widen4(v[k], f);
        if (p.residual) {
          widen4(q[k], g);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] += g[e];
        }
        const uint32_t c0 = 8 * j - shift;  // (wraps in vector 0 of a shifted row)
        if (8 * j >= shift && c0 + 8 <= p.dim) {
          if (p.h_out) store8<MX_BF16>(p.h_out, base + c0, f);
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) h[any_at<DTYPE>(c0 + e)] = f[e];
        } else {
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) {
            const uint32_t c = c0 + e;
            if (c < p.dim) {  // (a neighbour's element wraps to a large number)
              if (p.h_out) store1<DTYPE>(p.h_out, base + c, f[e]);
              h[any_at<DTYPE>(c)] = f[e];
            }
          }
        }
      }
    }
  } else {
    for (uint32_t c0 = threadIdx.x; c0 < p.dim; c0 += 8 * T) {
      float v[8], r[8];
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k) {
        const uint32_t c = c0 + T * k;
        v[k] = c < p.dim ? load1<DTYPE>(p.x, base + c) : 0.0f;
        r[k] = c < p.dim && p.residual ? load1<DTYPE>(p.residual, base + c) : 0.0f;
      }
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k) {
        const uint32_t c = c0 + T * k;
        if (c < p.dim) {
          if (p.residual) v[k] += r[k];
          if (p.h_out) store1<DTYPE>(p.h_out, base + c, v[k]);
          h[c] = v[k];
          ss = fmaf(v[k], v[k], ss);
        }
      }
    }
  }
  for (uint32_t c = p.dim + threadIdx.x; c < 8 * groups; c += T) h[any_at<DTYPE>(c)] = 0.0f;
  if constexpr (DTYPE == MX_BF16) {  // the squares in the order of the FP32 rows
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < p.dim; c += T) {
      const float v = h[any_at<DTYPE>(c)];
      ss = fmaf(v, v, ss);
    }
  }
  const float s = rsqrtf(cta_sum(ss, red) * p.inv_dim + p.eps);  // (its barrier: the row is in shared memory)
  uint8_t* out_row = p.elems + (size_t)row * p.kblocks * (4 * bits);
  for (uint32_t g0 = threadIdx.x & ~31u; g0 < groups; g0 += T) {  // (warps stay whole for the shuffles)
    const uint32_t g = g0 + (threadIdx.x & 31);
    float v[8] = {}, w[8] = {};
    if (g < groups) any_group<DTYPE>(h, g, v);
    if (8 * g + 8 <= p.dim) {
      load_weight8(p.weight, p.w_bf16, 8 * g, w);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (8 * g + e < p.dim) w[e] = weight1(p.weight, p.w_bf16, 8 * g + e);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * s * w[e];
    if (8 * g >= p.dim) {  // padding stays zero whatever s is
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    } else if (8 * g + 8 > p.dim) {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (8 * g + e >= p.dim) v[e] = 0.0f;
    }
    if (p.y_out && g < groups) {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) h[any_at<DTYPE>(8 * g) + e] = v[e];
    }
    store_group<FMT>(p, row, out_row, g, v);
  }
  if (p.y_out) {
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < p.dim; c += T) store1<DTYPE>(p.y_out, base + c, h[any_at<DTYPE>(c)]);
  }
  zero_pad_rows(p);
}

// Rows longer than shared memory: an element per lane, an MX block per warp and step; the row is read twice.
template <int DTYPE, int FMT>
__global__ void __launch_bounds__(1024) rmsnorm_long_kernel(const NormParams p) {
  constexpr uint32_t bits = FmtTraits<FMT>::bits;
  __shared__ float red[32];
  pdl_prologue();
  const uint32_t row = blockIdx.x, lane = threadIdx.x & 31;
  const size_t base = (size_t)row * p.dim;
  float ss = 0.0f;
  for (uint32_t c = threadIdx.x; c < p.dim; c += blockDim.x) {
    float v = load1<DTYPE>(p.x, base + c);
    if (p.residual) v += load1<DTYPE>(p.residual, base + c);
    ss = fmaf(v, v, ss);
  }
  const float s = rsqrtf(cta_sum(ss, red) * p.inv_dim + p.eps);  // (its barrier also orders the reads above before the stores below)
  uint8_t* out_row = p.elems + (size_t)row * p.kblocks * (4 * bits);
  for (uint32_t kb = threadIdx.x >> 5; kb < ((p.kblocks + 3) & ~3u); kb += blockDim.x >> 5) {
    const uint32_t c = kb * 32 + lane;
    float y = 0.0f;
    if (c < p.dim) {
      float v = load1<DTYPE>(p.x, base + c);
      if (p.residual) v += load1<DTYPE>(p.residual, base + c);
      if (p.h_out) store1<DTYPE>(p.h_out, base + c, v);
      y = v * s * weight1(p.weight, p.w_bf16, c);
      if (p.y_out) store1<DTYPE>(p.y_out, base + c, y);
    }
    if (kb >= p.kblocks) {
      if (p.layout == MX_SCALES_SWIZZLED && lane == 0) p.scales[scale_at(p, row, kb)] = 0;
      continue;
    }
    float am = absmax_nan(y, 0.0f);
#pragma unroll
    for (int o = 16; o; o >>= 1) am = absmax_nan(am, __shfl_xor_sync(0xffffffffu, am, o));
    const BlockScale bs = block_scale<FMT>(am);
    float a = mul_ftz(y, bs.m1);
    if (FMT == MX_INT8) a *= bs.m2;
    a = __uint_as_float(__float_as_uint(a) | p.sticky);
    uint32_t code = cast_pair<FMT, MX_RNE>(a, 0.0f) & ((1u << bits) - 1u);
    if (!bs.finite) code = 0;
    // four lanes' codes are 32, 24 or 16 bits of the row's stream
    uint32_t w = code | (__shfl_down_sync(0xffffffffu, code, 1) << bits);
    w |= __shfl_down_sync(0xffffffffu, w, 2) << (2 * bits);
    if ((lane & 3) == 0) {
      uint8_t* d = out_row + (size_t)kb * (4 * bits) + (lane >> 2) * (bits / 2);
#pragma unroll
      for (uint32_t i = 0; i < bits / 2; ++i) d[i] = (uint8_t)(w >> (8 * i));
    }
    if (lane == 0) p.scales[scale_at(p, row, kb)] = (uint8_t)bs.byte;
  }
  zero_pad_rows(p);
}

// ---------------------------------------------------------------------------------------------------
// Backward.  Both row sums are taken over what is read anyway,
//   s1 = sum h^2,  s2 = sum dy h w,   s = rsqrt(s1 / D + eps),   dh = s (dy w - h s^2 s2 / D) + dres,
// so a row is read once and needs one reduction.  The grid stays resident; a thread keeps its columns
// from row to row and sums its share of the weight gradient, dy h s, in registers.  Every CTA writes
// one row of partial sums and a second kernel adds those in a fixed order.  Bound by memory: 8192 x 4096 BF16 with
// dres 51 us, 5.25 TB/s of the rows' bytes, 44 of them the first kernel; 1023 x 1000 FP32 6.3 us, where the first and
// last rows' latencies and the second launch stand against 1.9 us of traffic.
// ---------------------------------------------------------------------------------------------------
struct NormBackParams {
  const void *dy, *h, *weight, *dres;
  void* dh;
  float* partial;
  float2* stats;
  uint32_t rows, dim, w_bf16, row_chunk;
  float eps, inv_dim;
};

// Pairs of FP32 numbers: one instruction for both.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
template <int DTYPE>
__device__ __forceinline__ void widen2(const Raw8<DTYPE>& r, uint64_t (&v)[4]) {
  float f[8];
  widen<DTYPE>(r, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2(f[2 * i], f[2 * i + 1]);
}

// A group's share of the row sums: s1 += h^2, s2 += (dy h) w.
template <int DTYPE>
__device__ __forceinline__ void sum_group(const Raw8<DTYPE>& hr, const Raw8<DTYPE>& gr, const uint64_t (&w)[4],
                                          uint64_t& s1, uint64_t& s2) {
  uint64_t h[4], g[4];
  widen2<DTYPE>(hr, h);
  widen2<DTYPE>(gr, g);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s1 = fma2(h[i], h[i], s1);
    s2 = fma2(mul2(g[i], h[i]), w[i], s2);
  }
}

// The second half of a row, with k = s c: dh = s dy w + dres - h k, and dw += s dy h.
template <int DTYPE>
__device__ __forceinline__ void finish_group(const NormBackParams& p, size_t at, const Raw8<DTYPE>& hr, const Raw8<DTYPE>& gr,
                                             const Raw8<DTYPE>& qr, const uint64_t (&w)[4], float s, float k,
                                             uint64_t (&dw)[4]) {
  uint64_t h[4], g[4], q[4];
  widen2<DTYPE>(hr, h);
  widen2<DTYPE>(gr, g);
  if (p.dres) {
    widen2<DTYPE>(qr, q);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = 0;
  }
  const uint64_t ss = pack2(s, s), kk = pack2(-k, -k);
  float o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t gs = mul2(g[i], ss);
    unpack2(fma2(h[i], kk, fma2(gs, w[i], q[i])), o[2 * i], o[2 * i + 1]);
    dw[i] = fma2(gs, h[i], dw[i]);
  }
  store8<DTYPE>(p.dh, at, o);
}

__device__ __forceinline__ void load_weight2(const NormBackParams& p, uint32_t elem, uint64_t (&w)[4]) {
  float f[8];
  load_weight8(p.weight, p.w_bf16, elem, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack2(f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ float sum2(uint64_t v) {
  float lo, hi;
  unpack2(v, lo, hi);
  return lo + hi;
}
__device__ __forceinline__ void spread2(const uint64_t (&v)[4], float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2(v[i], f[2 * i], f[2 * i + 1]);
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// dim % 8 == 0, 1024 < dim <= 8 V blockDim: a row per CTA at a time.  The next NS rows are on their way to shared memory
// meanwhile -- a thread copies just the elements that it will take itself, so the ring needs no
// barrier.  (One row ahead in registers left 48 KB an SM in flight: 8192 x 4096 BF16 52.7 us.)
template <int DTYPE, int V, int NS>
__global__ void __launch_bounds__(512) rmsnorm_backward_kernel(const NormBackParams p) {
  constexpr uint32_t kGroup = DTYPE == MX_BF16 ? 16 : 32;  // bytes of 8 elements
  extern __shared__ uint4 ring[];
  __shared__ float2 red[2][16];
  pdl_prologue();
  const uint32_t T = blockDim.x, lane = threadIdx.x & 31, warps = T >> 5, groups = p.dim >> 3;
  const uint32_t slot = V * T * kGroup, stage_bytes = 3 * slot;  // h, dy, dres
  const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(ring);
  uint64_t dw[V][4], w[V][4];  // a thread's columns, and so its weights, are the same in every row
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t g = i * T + threadIdx.x;
#pragma unroll
    for (int e = 0; e < 4; ++e) { dw[i][e] = 0; w[i][e] = 0; }
    if (g < groups) load_weight2(p, 8 * g, w[i]);
  }
  auto request = [&](uint32_t row, uint32_t stage) {
    if (row < p.rows) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const uint32_t g = i * T + threadIdx.x;
        if (g < groups) {
          const size_t at = ((size_t)row * p.dim + 8 * (size_t)g) * (kGroup / 8);
          const uint32_t dst = ring0 + stage * stage_bytes + g * kGroup;
#pragma unroll
          for (uint32_t k = 0; k < kGroup; k += 16) {
            cp_async16(dst + k, (const char*)p.h + at + k);
            cp_async16(dst + slot + k, (const char*)p.dy + at + k);
            if (p.dres) cp_async16(dst + 2 * slot + k, (const char*)p.dres + at + k);
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto take = [&](uint32_t stage, uint32_t tensor, uint32_t g) {
    Raw8<DTYPE> r;
    const uint4* q = ring + (stage * stage_bytes + tensor * slot + g * kGroup) / 16;
    r.v[0] = q[0];
    if constexpr (DTYPE == MX_F32) r.v[1] = q[1];
    return r;
  };
#pragma unroll
  for (int i = 0; i < NS; ++i) request(blockIdx.x + i * gridDim.x, i);
  uint32_t side = 0, stage = 0;
  for (uint32_t row = blockIdx.x; row < p.rows; row += gridDim.x, side ^= 1) {
    asm volatile("cp.async.wait_group %0;" ::"n"(NS - 1) : "memory");
    uint64_t a1 = 0, a2 = 0;
    Raw8<DTYPE> h[V], d[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t g = i * T + threadIdx.x;
      if (g < groups) {
        h[i] = take(stage, 0, g);
        d[i] = take(stage, 1, g);
        if (p.dres) q[i] = take(stage, 2, g);
        sum_group<DTYPE>(h[i], d[i], w[i], a1, a2);
      }
    }
    float s1 = sum2(a1), s2 = sum2(a2);
    request(row + NS * gridDim.x, stage);  // into the slots just read
    if (++stage == NS) stage = 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    if (lane == 0) red[side][threadIdx.x >> 5] = make_float2(s1, s2);
    __syncthreads();
    float2 t = red[side][lane & 15];
    if ((lane & 15) >= warps) t = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int o = 8; o; o >>= 1) {
      t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
      t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
    }
    const float s = rsqrtf(t.x * p.inv_dim + p.eps), k = s * (s * s * (t.y * p.inv_dim));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t g = i * T + threadIdx.x;
      if (g < groups) finish_group<DTYPE>(p, (size_t)row * p.dim + 8 * (size_t)g, h[i], d[i], q[i], w[i], s, k, dw[i]);
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t g = i * T + threadIdx.x;
    if (g < groups) {
      float f[8];
      spread2(dw[i], f);
      store8<MX_F32>(p.partial, (size_t)blockIdx.x * p.dim + 8 * (size_t)g, f);
    }
  }
}

// dim % 8 == 0, dim <= 256 V <= 1024: a row per warp, so that a reduction is five shuffles and eight rows are under way
// in a CTA; the warps' weight gradients meet in shared memory at the end, in warp order.
constexpr uint32_t kRowWarps = 8;
template <int DTYPE, int V>
__global__ void __launch_bounds__(32 * kRowWarps) rmsnorm_backward_warp_kernel(const NormBackParams p) {
  extern __shared__ float sums[];  // [warps][dim]
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, groups = p.dim >> 3;
  uint64_t dw[V][4], w[V][4];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t g = i * 32 + lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) { dw[i][e] = 0; w[i][e] = 0; }
    if (g < groups) load_weight2(p, 8 * g, w[i]);
  }
  for (uint32_t row = blockIdx.x * kRowWarps + warp; row < p.rows; row += gridDim.x * kRowWarps) {
    Raw8<DTYPE> h[V], d[V], q[V];
    const size_t base = (size_t)row * p.dim;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t g = i * 32 + lane;
      if (g < groups) {
        h[i] = load_raw8<DTYPE>(p.h, base + 8 * (size_t)g);
        d[i] = load_raw8<DTYPE>(p.dy, base + 8 * (size_t)g);
        if (p.dres) q[i] = load_raw8<DTYPE>(p.dres, base + 8 * (size_t)g);
      }
    }
    uint64_t a1 = 0, a2 = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i * 32 + lane < groups) sum_group<DTYPE>(h[i], d[i], w[i], a1, a2);
    float s1 = sum2(a1), s2 = sum2(a2);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    const float s = rsqrtf(s1 * p.inv_dim + p.eps), k = s * (s * s * (s2 * p.inv_dim));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t g = i * 32 + lane;
      if (g < groups) finish_group<DTYPE>(p, base + 8 * (size_t)g, h[i], d[i], q[i], w[i], s, k, dw[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t g = i * 32 + lane;
    if (g < groups) {
      float f[8];
      spread2(dw[i], f);
      float4* d = reinterpret_cast<float4*>(sums + (size_t)warp * p.dim + 8 * g);
      d[0] = make_float4(f[0], f[1], f[2], f[3]);
      d[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
  }
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < p.dim; c += blockDim.x) {
    float t = sums[c];
#pragma unroll
    for (uint32_t w = 1; w < kRowWarps; ++w) t += sums[w * p.dim + c];
    p.partial[(size_t)blockIdx.x * p.dim + c] = t;
  }
}

// Rows that start anywhere, dim <= 32 V <= 1024: a row per warp, an element per lane; the weights wait in shared memory.
template <int DTYPE, int V>
__global__ void __launch_bounds__(32 * kRowWarps) rmsnorm_backward_warp_any_kernel(const NormBackParams p) {
  extern __shared__ float sums[];  // [warps][dim], then the weights
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* weight = sums + kRowWarps * p.dim;
  for (uint32_t c = threadIdx.x; c < p.dim; c += blockDim.x) weight[c] = weight1(p.weight, p.w_bf16, c);
  __syncthreads();
  float dw[V];
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = 0.0f;
  for (uint32_t row = blockIdx.x * kRowWarps + warp; row < p.rows; row += gridDim.x * kRowWarps) {
    const size_t base = (size_t)row * p.dim + lane;
    float h[V], g[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool live = 32 * i + lane < p.dim;
      h[i] = live ? load1<DTYPE>(p.h, base + 32 * i) : 0.0f;
      g[i] = live ? load1<DTYPE>(p.dy, base + 32 * i) : 0.0f;
      q[i] = live && p.dres ? load1<DTYPE>(p.dres, base + 32 * i) : 0.0f;
    }
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s1 = fmaf(h[i], h[i], s1);
      if (32 * i + lane < p.dim) s2 = fmaf(g[i] * weight[32 * i + lane], h[i], s2);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    const float s = rsqrtf(s1 * p.inv_dim + p.eps), k = s * (s * s * (s2 * p.inv_dim));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (32 * i + lane >= p.dim) continue;
      const float gs = g[i] * s;
      dw[i] = fmaf(gs, h[i], dw[i]);
      store1<DTYPE>(p.dh, base + 32 * i, fmaf(gs, weight[32 * i + lane], fmaf(-k, h[i], q[i])));
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (32 * i + lane < p.dim) sums[warp * p.dim + 32 * i + lane] = dw[i];
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < p.dim; c += blockDim.x) {
    float t = sums[c];
#pragma unroll
    for (uint32_t w = 1; w < kRowWarps; ++w) t += sums[w * p.dim + c];
    p.partial[(size_t)blockIdx.x * p.dim + c] = t;
  }
}

// Any dim up to 512 V: the ring above for rows that start anywhere.  The 16-byte vectors that cover a row are copied
// by whichever thread comes to them, so a barrier stands between copy and use; a thread takes every 512th
// element, twice from shared memory.  (8192 x 4001 BF16: 150 us with the two kernels below.)
__device__ __forceinline__ void cp_async16_part(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <int DTYPE> __host__ __device__ constexpr uint32_t elem_bytes() { return DTYPE == MX_BF16 ? 2u : 4u; }
// bytes of a tensor's slot: a row, up to 15 bytes before it, whole vectors
template <int DTYPE>
__host__ __device__ inline uint32_t any_slot(uint32_t dim) { return (dim * elem_bytes<DTYPE>() + 15 + 15) / 16 * 16; }

template <int DTYPE, int V, int NS>
__global__ void __launch_bounds__(512) rmsnorm_backward_any_kernel(const NormBackParams p) {
  constexpr uint32_t esz = elem_bytes<DTYPE>();
  extern __shared__ uint4 ring[];
  __shared__ float2 red[2][16];
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, slot = any_slot<DTYPE>(p.dim), stage_bytes = 3 * slot;
  const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(ring);
  const size_t row_bytes = (size_t)p.dim * esz, all_bytes = row_bytes * p.rows;
  float dw[V], w[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t c = i * 512 + threadIdx.x;
    dw[i] = 0.0f;
    w[i] = c < p.dim ? weight1(p.weight, p.w_bf16, c) : 0.0f;
  }
  auto request = [&](uint32_t row, uint32_t stage) {
    if (row < p.rows) {
      const size_t b0 = row * row_bytes, a0 = b0 & ~(size_t)15;
      const uint32_t vecs = (uint32_t)((b0 + row_bytes - a0 + 15) / 16);
      for (uint32_t j = threadIdx.x; j < vecs; j += 512) {
        const size_t at = a0 + 16 * (size_t)j;
        const uint32_t n = all_bytes - at < 16 ? (uint32_t)(all_bytes - at) : 16u;  // nothing behind the tensor is read
        const uint32_t dst = ring0 + stage * stage_bytes + 16 * j;
        cp_async16_part(dst, (const char*)p.h + at, n);
        cp_async16_part(dst + slot, (const char*)p.dy + at, n);
        if (p.dres) cp_async16_part(dst + 2 * slot, (const char*)p.dres + at, n);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) request(blockIdx.x + i * gridDim.x, i);
  uint32_t side = 0, stage = 0;
  for (uint32_t row = blockIdx.x; row < p.rows; row += gridDim.x, side ^= 1) {
    asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
    __syncthreads();  // the row has landed, and everybody is done with the row before: its stage is free
    request(row + (NS - 1) * gridDim.x, stage == 0 ? NS - 1 : stage - 1);
    const size_t base = (size_t)row * p.dim;
    const char* at = (const char*)ring + stage * stage_bytes + (uint32_t)(row * row_bytes & 15);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t c = i * 512 + threadIdx.x;
      if (c < p.dim) {
        const float h = load1<DTYPE>(at, c), g = load1<DTYPE>(at + slot, c);
        s1 = fmaf(h, h, s1);
        s2 = fmaf(g * h, w[i], s2);
      }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    if (lane == 0) red[side][threadIdx.x >> 5] = make_float2(s1, s2);
    __syncthreads();
    float2 t = red[side][lane & 15];
#pragma unroll
    for (int o = 8; o; o >>= 1) {
      t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
      t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
    }
    const float s = rsqrtf(t.x * p.inv_dim + p.eps), k = s * (s * s * (t.y * p.inv_dim));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t c = i * 512 + threadIdx.x;
      if (c < p.dim) {
        const float h = load1<DTYPE>(at, c), gs = load1<DTYPE>(at + slot, c) * s;
        const float q = p.dres ? load1<DTYPE>(at + 2 * slot, c) : 0.0f;
        dw[i] = fmaf(gs, h, dw[i]);
        store1<DTYPE>(p.dh, base + c, fmaf(-k, h, fmaf(gs, w[i], q)));
      }
    }
    if (++stage == NS) stage = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t c = i * 512 + threadIdx.x;
    if (c < p.dim) p.partial[(size_t)blockIdx.x * p.dim + c] = dw[i];
  }
}

// Longer rows, in two kernels: the row sums first (a CTA per row), then a thread per column goes down a chunk
// of rows, writes dh and sums the column's weight gradient.  h and dy are read twice; dh may lie on dy.
template <int DTYPE>
__global__ void __launch_bounds__(256) rmsnorm_row_sums_kernel(const NormBackParams p) {
  __shared__ float red[2][32];
  pdl_prologue();
  const uint32_t row = blockIdx.x;
  const size_t base = (size_t)row * p.dim;
  float s1 = 0.0f, s2 = 0.0f;
  for (uint32_t c = threadIdx.x; c < p.dim; c += blockDim.x) {
    const float h = load1<DTYPE>(p.h, base + c);
    s1 = fmaf(h, h, s1);
    s2 = fmaf(load1<DTYPE>(p.dy, base + c) * weight1(p.weight, p.w_bf16, c), h, s2);
  }
  s1 = cta_sum(s1, red[0]);
  s2 = cta_sum(s2, red[1]);
  if (threadIdx.x == 0) {
    const float s = rsqrtf(s1 * p.inv_dim + p.eps);
    p.stats[row] = make_float2(s, s * s * (s2 * p.inv_dim));
  }
}

template <int DTYPE>
__global__ void __launch_bounds__(256) rmsnorm_columns_kernel(const NormBackParams p) {
  pdl_prologue();
  const uint32_t c = blockIdx.x * 256 + threadIdx.x;
  if (c >= p.dim) return;
  const uint32_t r0 = blockIdx.y * p.row_chunk, r1 = min(p.rows, r0 + p.row_chunk);
  const float w = weight1(p.weight, p.w_bf16, c);
  float dw = 0.0f;
#pragma unroll 4
  for (uint32_t r = r0; r < r1; ++r) {
    const size_t at = (size_t)r * p.dim + c;
    const float2 st = __ldg(p.stats + r);
    const float h = load1<DTYPE>(p.h, at), d = load1<DTYPE>(p.dy, at);
    float o = st.x * (d * w - h * st.y);
    if (p.dres) o += load1<DTYPE>(p.dres, at);
    dw = fmaf(d, h * st.x, dw);
    store1<DTYPE>(p.dh, at, o);
  }
  p.partial[(size_t)blockIdx.y * p.dim + c] = dw;
}

// dweight[c] = sum over the partial rows, always in the same order: 32 strands of rows per column, all of a
// thread's loads in flight at once (as chains of dependent batches they took 8 us).
__global__ void __launch_bounds__(1024) rmsnorm_dweight_kernel(const float* __restrict__ partial, float* __restrict__ dweight,
                                                               uint32_t parts, uint32_t dim) {
  __shared__ float sum[32][33];
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, strand = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float t = 0.0f;
  constexpr uint32_t kEach = (kNormPartials + 31) / 32;
  float v[kEach];
#pragma unroll
  for (uint32_t k = 0; k < kEach; ++k) {
    const uint32_t r = strand + 32 * k;
    v[k] = c < dim && r < parts ? partial[(size_t)r * dim + c] : 0.0f;
  }
#pragma unroll
  for (uint32_t k = 0; k < kEach; ++k) t += v[k];
  sum[strand][lane] = t;
  __syncthreads();
  // warp w sums column w's strands
  t = sum[lane][strand];
#pragma unroll
  for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  const uint32_t col = blockIdx.x * 32 + strand;
  if (lane == 0 && col < dim) dweight[col] = t;
}

// ---- host side ---------------------------------------------------------------

struct Shape {
  uint32_t threads;
  int v;     // groups of 8 per thread; 0: the kernels for any dim
  bool few;  // rows: each has an SM to itself
};

template <int DTYPE, int FMT, uint32_t T>
cudaError_t launch_any_forward(const NormParams& p, uint32_t smem, cudaStream_t stream) {
  static bool attr_set[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(rmsnorm_any_kernel<DTYPE, FMT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)kNormRowBytes);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  return launch_pdl(rmsnorm_any_kernel<DTYPE, FMT, T>, dim3(p.rows), dim3(T), smem, stream, p);
}

template <int DTYPE, int FMT>
cudaError_t launch_forward(const NormParams& p, Shape s, cudaStream_t stream) {
  const dim3 grid(p.rows);
  switch (s.v) {
    case 1: return launch_pdl(rmsnorm_kernel<DTYPE, FMT, 1>, grid, dim3(s.threads), 0, stream, p);
    case 2: return launch_pdl(rmsnorm_kernel<DTYPE, FMT, 2>, grid, dim3(s.threads), 0, stream, p);
    case 4: return launch_pdl(rmsnorm_kernel<DTYPE, FMT, 4>, grid, dim3(s.threads), 0, stream, p);
    default: break;
  }
  const uint64_t row_bytes = norm_row_bytes(DTYPE == MX_BF16, p.dim);
  if (row_bytes > kNormRowBytes) return launch_pdl(rmsnorm_long_kernel<DTYPE, FMT>, grid, dim3(1024), 0, stream, p);
  const uint32_t smem = (uint32_t)row_bytes;
  // few threads where rows are short, so that more of them are under way (8192 x 257 BF16: 13.6 us with 64, 25 with 256); their
  // number is a constant of the kernel, which halves its registers (8192 x 4001 FP32: 94 us otherwise, 73)
  if (!s.few && p.dim <= 768) return launch_any_forward<DTYPE, FMT, 64>(p, smem, stream);
  if (!s.few && p.dim <= 2048) return launch_any_forward<DTYPE, FMT, 128>(p, smem, stream);
  return launch_any_forward<DTYPE, FMT, 256>(p, smem, stream);
}

template <int DTYPE>
cudaError_t launch_forward_fmt(int fmt, const NormParams& p, Shape s, cudaStream_t stream) {
  switch (fmt) {
    case MX_E4M3: return launch_forward<DTYPE, MX_E4M3>(p, s, stream);
    case MX_E5M2: return launch_forward<DTYPE, MX_E5M2>(p, s, stream);
    case MX_E3M2: return launch_forward<DTYPE, MX_E3M2>(p, s, stream);
    case MX_E2M3: return launch_forward<DTYPE, MX_E2M3>(p, s, stream);
    case MX_E2M1: return launch_forward<DTYPE, MX_E2M1>(p, s, stream);
    default: return launch_forward<DTYPE, MX_INT8>(p, s, stream);
  }
}

template <int DTYPE, int V, int NS>
cudaError_t launch_ring(const NormBackParams& p, uint32_t threads, uint32_t grid, cudaStream_t stream) {
  const uint32_t smem = NS * 3 * V * threads * (DTYPE == MX_BF16 ? 16 : 32);
  static bool attr_set[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(rmsnorm_backward_kernel<DTYPE, V, NS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             NS * 3 * V * 512 * (DTYPE == MX_BF16 ? 16 : 32));
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  return launch_pdl(rmsnorm_backward_kernel<DTYPE, V, NS>, dim3(grid), dim3(threads), smem, stream, p);
}

template <int DTYPE, int V, int NS>
cudaError_t launch_any(const NormBackParams& p, uint32_t smem, int sms, uint32_t* parts, cudaStream_t stream) {
  static bool attr_set[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(rmsnorm_backward_any_kernel<DTYPE, V, NS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  uint32_t grid = (smem <= 112 * 1024 ? 2u : 1u) * (uint32_t)sms;
  if (grid > (uint32_t)kNormPartials) grid = (uint32_t)kNormPartials;
  *parts = p.rows < grid ? p.rows : grid;
  return launch_pdl(rmsnorm_backward_any_kernel<DTYPE, V, NS>, dim3(*parts), dim3(512), smem, stream, p);
}
// Rows of any length up to 8192: many short ones a warp each, else three of them in the ring (two where three do not fit).
template <int DTYPE>
cudaError_t launch_backward_any(const NormBackParams& p, int sms, uint32_t* parts, cudaStream_t stream) {
  const uint32_t stage = 3 * any_slot<DTYPE>(p.dim);
  if (3 * stage > 220 * 1024) return launch_any<DTYPE, 16, 2>(p, 2 * stage, sms, parts, stream);
  if (p.dim <= 1024 && p.rows >= 1024) {
    // (1001 BF16: 8192 rows 38 us, 55 in the ring; 64 rows 8.4, 4.4; 257: 13, 45)
    const uint32_t need = (p.rows + kRowWarps - 1) / kRowWarps, most = 2u * (uint32_t)sms;
    *parts = need < most ? need : most;
    if (*parts > (uint32_t)kNormPartials) *parts = (uint32_t)kNormPartials;
    const dim3 grid(*parts), block(32 * kRowWarps);
    const size_t smem = (kRowWarps + 1) * (size_t)p.dim * 4;
    if (p.dim <= 256) return launch_pdl(rmsnorm_backward_warp_any_kernel<DTYPE, 8>, grid, block, smem, stream, p);
    if (p.dim <= 512) return launch_pdl(rmsnorm_backward_warp_any_kernel<DTYPE, 16>, grid, block, smem, stream, p);
    return launch_pdl(rmsnorm_backward_warp_any_kernel<DTYPE, 32>, grid, block, smem, stream, p);
  }
  if (p.dim <= 1024) return launch_any<DTYPE, 2, 3>(p, 3 * stage, sms, parts, stream);
  if (p.dim <= 2048) return launch_any<DTYPE, 4, 3>(p, 3 * stage, sms, parts, stream);
  if (p.dim <= 4096) return launch_any<DTYPE, 8, 3>(p, 3 * stage, sms, parts, stream);
  return launch_any<DTYPE, 16, 3>(p, 3 * stage, sms, parts, stream);
}

// Writes *parts rows of partial sums.
template <int DTYPE>
cudaError_t launch_backward(const NormBackParams& p, int sms, uint32_t* parts, cudaStream_t stream) {
  const uint32_t groups = p.dim / 8;
  auto at_most = [&](uint32_t ctas, uint32_t rows_each) {
    const uint32_t need = (p.rows + rows_each - 1) / rows_each;
    const uint32_t cap = ctas < (uint32_t)kNormPartials ? ctas : (uint32_t)kNormPartials;
    return need < cap ? need : cap;
  };
  if (groups <= 128) {
    *parts = at_most(2u * (uint32_t)sms, kRowWarps);
    const dim3 grid(*parts), block(32 * kRowWarps);
    const size_t smem = kRowWarps * (size_t)p.dim * 4;
    if (groups <= 32) return launch_pdl(rmsnorm_backward_warp_kernel<DTYPE, 1>, grid, block, smem, stream, p);
    if (groups <= 64) return launch_pdl(rmsnorm_backward_warp_kernel<DTYPE, 2>, grid, block, smem, stream, p);
    return launch_pdl(rmsnorm_backward_warp_kernel<DTYPE, 4>, grid, block, smem, stream, p);
  }
  const uint32_t threads = groups < 512 ? (groups + 31) / 32 * 32 : 512;
  if (groups <= threads) {  // up to 4096 elements: two CTAs an SM, 96 KB of rows each (FP32: two rows)
    *parts = at_most(2u * (uint32_t)sms, 1);
    return launch_ring<DTYPE, 1, DTYPE == MX_BF16 ? 4 : 2>(p, threads, *parts, stream);
  }
  *parts = at_most((uint32_t)sms, 1);  // up to 8192: one CTA, 192 KB
  return launch_ring<DTYPE, 2, DTYPE == MX_BF16 ? 4 : 2>(p, threads, *parts, stream);
}

}  // namespace

cudaError_t launch_rmsnorm_quantize(const RmsnormArgs& a) {
  NormParams p;
  p.x = a.x; p.residual = a.residual; p.weight = a.weight; p.h_out = a.h_out; p.y_out = a.y_out;
  p.elems = a.elems; p.scales = a.scales;
  p.rows = (uint32_t)a.rows; p.dim = (uint32_t)a.dim; p.kblocks = (uint32_t)((a.dim + 31) / 32);
  p.eps = a.eps; p.inv_dim = 1.0f / (float)a.dim;
  p.w_bf16 = (uint32_t)a.w_bf16; p.sticky = a.rounding == MX_RHAZ ? 1u : 0u; p.layout = (uint32_t)a.layout;
  // Groups of 8 that a row stores, whole 16-group runs (the four scale bytes of a swizzled word).
  const uint32_t groups = (p.kblocks + 3) / 4 * 16;
  Shape s = {256, 0, a.rows <= a.sm_count};
  if (a.dim % 8 == 0 && groups <= 2048) {
    if (s.few) {  // a row per SM: as many threads as the row has groups, the shortest chain
      s.threads = groups < 1024 ? (groups + 31) / 32 * 32 : 1024;
    } else {
      s.threads = (groups / 4 + 31) / 32 * 32;
      if (s.threads < 64) s.threads = 64;
    }
    const uint32_t v = (groups + s.threads - 1) / s.threads;
    s.v = v <= 1 ? 1 : v <= 2 ? 2 : 4;
  }
  return a.dtype == MX_BF16 ? launch_forward_fmt<MX_BF16>(a.fmt, p, s, a.stream)
                            : launch_forward_fmt<MX_F32>(a.fmt, p, s, a.stream);
}

cudaError_t launch_rmsnorm_backward(const RmsnormBackwardArgs& a) {
  NormBackParams p;
  p.dy = a.dy; p.h = a.h; p.weight = a.weight; p.dres = a.dres; p.dh = a.dh; p.partial = a.partial; p.stats = a.stats;
  p.rows = (uint32_t)a.rows; p.dim = (uint32_t)a.dim; p.w_bf16 = (uint32_t)a.w_bf16;
  p.eps = a.eps; p.inv_dim = 1.0f / (float)a.dim; p.row_chunk = 0;
  uint32_t parts;
  cudaError_t e;
  if (a.dim <= 8192) {
    if (a.dim % 8 == 0)
      e = a.dtype == MX_BF16 ? launch_backward<MX_BF16>(p, a.sm_count, &parts, a.stream)
                             : launch_backward<MX_F32>(p, a.sm_count, &parts, a.stream);
    else
      e = a.dtype == MX_BF16 ? launch_backward_any<MX_BF16>(p, a.sm_count, &parts, a.stream)
                             : launch_backward_any<MX_F32>(p, a.sm_count, &parts, a.stream);
  } else {
    e = a.dtype == MX_BF16 ? launch_pdl(rmsnorm_row_sums_kernel<MX_BF16>, dim3(p.rows), dim3(256), 0, a.stream, p)
                           : launch_pdl(rmsnorm_row_sums_kernel<MX_F32>, dim3(p.rows), dim3(256), 0, a.stream, p);
    if (e != cudaSuccess) return e;
    p.row_chunk = (p.rows + 63) / 64;
    parts = (p.rows + p.row_chunk - 1) / p.row_chunk;
    const dim3 grid((p.dim + 255) / 256, parts);
    e = a.dtype == MX_BF16 ? launch_pdl(rmsnorm_columns_kernel<MX_BF16>, grid, dim3(256), 0, a.stream, p)
                           : launch_pdl(rmsnorm_columns_kernel<MX_F32>, grid, dim3(256), 0, a.stream, p);
  }
  if (e != cudaSuccess) return e;
  return launch_pdl(rmsnorm_dweight_kernel, dim3((p.dim + 31) / 32), dim3(1024), 0, a.stream, (const float*)a.partial,
                    a.dweight, parts, p.dim);
}

}  // namespace mx
