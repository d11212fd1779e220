// Rows of FP32 or BF16 numbers: groups of 8 consecutive elements as vectors, and single elements.
#pragma once

#include "mx_device.cuh"

namespace mx {

__device__ __forceinline__ uint4 ld_16(const void* p) {  // rows are read once: not kept in the L1
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// 8 consecutive elements as they lie in memory.
template <int DTYPE> struct Raw8 { uint4 v[DTYPE == MX_BF16 ? 1 : 2]; };

template <int DTYPE>
__device__ __forceinline__ Raw8<DTYPE> load_raw8(const void* base, size_t elem) {
  Raw8<DTYPE> r;
  const char* p = (const char*)base + elem * (DTYPE == MX_BF16 ? 2 : 4);
  if constexpr (DTYPE == MX_F32) {
    if (((uintptr_t)p & 31u) == 0) {
      asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(r.v[0].x), "=r"(r.v[0].y), "=r"(r.v[0].z), "=r"(r.v[0].w), "=r"(r.v[1].x), "=r"(r.v[1].y),
                     "=r"(r.v[1].z), "=r"(r.v[1].w) : "l"(p));
      return r;
    }
    r.v[1] = ld_16(p + 16);
  }
  r.v[0] = ld_16(p);
  return r;
}
__device__ __forceinline__ void widen4(const uint4& u, float (&f)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
template <int DTYPE>
__device__ __forceinline__ void widen(const Raw8<DTYPE>& r, float (&f)[8]) {
  if constexpr (DTYPE == MX_BF16) {
    widen4(r.v[0], f);
  } else {
    f[0] = __uint_as_float(r.v[0].x); f[1] = __uint_as_float(r.v[0].y);
    f[2] = __uint_as_float(r.v[0].z); f[3] = __uint_as_float(r.v[0].w);
    f[4] = __uint_as_float(r.v[1].x); f[5] = __uint_as_float(r.v[1].y);
    f[6] = __uint_as_float(r.v[1].z); f[7] = __uint_as_float(r.v[1].w);
  }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
template <int DTYPE>
__device__ __forceinline__ void store8(void* base, size_t elem, const float (&f)[8]) {
  if constexpr (DTYPE == MX_BF16) {
    *reinterpret_cast<uint4*>((char*)base + elem * 2) =
        make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  } else {
    // whole sectors: two 16-byte stores would each write half of every sector they touch
    float4* p = reinterpret_cast<float4*>((char*)base + elem * 4);
    if (((uintptr_t)p & 31u) == 0) {
      const uint32_t w[8] = {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]),
                             __float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])};
      st_32(p, w);
      return;
    }
    p[0] = make_float4(f[0], f[1], f[2], f[3]);
    p[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
}
template <int DTYPE>
__device__ __forceinline__ float load1(const void* base, size_t elem) {
  if constexpr (DTYPE == MX_BF16) return __uint_as_float((uint32_t)((const uint16_t*)base)[elem] << 16);
  else return ((const float*)base)[elem];
}
template <int DTYPE>
__device__ __forceinline__ void store1(void* base, size_t elem, float v) {
  if constexpr (DTYPE == MX_BF16) ((uint16_t*)base)[elem] = (uint16_t)pack_bf16(v, 0.0f);
  else ((float*)base)[elem] = v;
}

}  // namespace mx
