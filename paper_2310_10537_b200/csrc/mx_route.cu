// Routing to experts: scores, group choice, top-k and weights of each token, and the gradient of the
// weights.  One warp per token, or a few lanes (below); a lane holds consecutive experts in registers (read as
// vectors), so that a lower lane always means a lower expert and ties fall to the lowest index by themselves.
#include <cuda_runtime.h>

#include "mx.h"
#include "mx_device.cuh"
#include "mx_launch.h"

namespace mx {
namespace {

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kRouteWarps = 4;  // tokens per CTA

struct RouteParams {
  const void* logits;
  const float *bias, *dweights;
  int32_t* ids;
  float* weights;
  void* dlogits;
  uint32_t tokens, experts, topk, score, groups, topk_groups, group_score, renormalize, group_size, group_lanes;
  FastDiv by_group_size;
  float scale;
};

// Floats as unsigned integers of the same order; -0 counts as +0, and NaN ranks above everything (the
// addition makes every NaN the canonical one, 0x7fffffff).  0 is below the key of every float: "not a candidate".
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_key(uint32_t k) {
  return k == 0u ? -INFINITY : __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// 1 / (1 + exp(-x)) without a branch: t = exp(-|x|), and 1 / (1 + t) by one Newton-Raphson step from the approximate
// reciprocal (1 + t is in [1, 2]: neither end of the range of floats is near).
__device__ __forceinline__ float sigmoid(float x) {
  const float t = expf(-fabsf(x)), d = 1.0f + t;
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
  r = fmaf(r, fmaf(-d, r, 1.0f), r);
  return x >= 0.0f ? r : t * r;
}

template <int DTYPE>
__device__ __forceinline__ float load_logit(const RouteParams& p, size_t at) {
  return DTYPE == MX_BF16 ? __uint_as_float((uint32_t)__ldg((const uint16_t*)p.logits + at) << 16)
                          : __ldg((const float*)p.logits + at);
}

// The lane's NV logits; experts past the end read as -Inf.
template <int DTYPE, int NV>
__device__ __forceinline__ void load_logits(const RouteParams& p, uint32_t token, uint32_t lane, float (&x)[NV]) {
  const uint32_t e0 = lane * NV;
  const size_t at = (size_t)token * p.experts + e0;
  // vectors where every row starts on one and the lane's experts all exist
  if constexpr (DTYPE == MX_F32 && NV % 4 == 0) {
    if ((p.experts & 3u) == 0 && e0 + NV <= p.experts) {
      const float4* q = reinterpret_cast<const float4*>((const float*)p.logits + at);
#pragma unroll
      for (int i = 0; i < NV / 4; ++i) {
        const float4 v = __ldg(q + i);
        x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
      }
      return;
    }
  }
  if constexpr (DTYPE == MX_BF16 && NV % 4 == 0) {
    if ((p.experts & 3u) == 0 && e0 + NV <= p.experts) {
      const uint2* q = reinterpret_cast<const uint2*>((const uint16_t*)p.logits + at);
#pragma unroll
      for (int i = 0; i < NV / 4; ++i) {
        const uint2 v = __ldg(q + i);
        x[4 * i] = __uint_as_float(v.x << 16); x[4 * i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[4 * i + 2] = __uint_as_float(v.y << 16); x[4 * i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
      }
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    x[j] = -INFINITY;
    if (e0 + j < p.experts) x[j] = load_logit<DTYPE>(p, at + j);
  }
}

// The lane's NV biases.
template <int NV>
__device__ __forceinline__ void load_bias(const RouteParams& p, uint32_t e0, float (&b)[NV]) {
  if constexpr (NV % 4 == 0) {
    if ((reinterpret_cast<uintptr_t>(p.bias) & 15u) == 0 && e0 + NV <= p.experts) {
#pragma unroll
      for (int i = 0; i < NV / 4; ++i) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(p.bias + e0) + i);
        b[4 * i] = v.x; b[4 * i + 1] = v.y; b[4 * i + 2] = v.z; b[4 * i + 3] = v.w;
      }
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) b[j] = e0 + j < p.experts ? __ldg(p.bias + e0 + j) : 0.0f;
}

__device__ __forceinline__ float warp_max(float v) {  // NaN wins
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float w = __shfl_xor_sync(kFull, v, o);
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(v), "f"(w));
  }
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

// Maximum and sum of exponentials of a row of logits (softmax).
template <int NV>
__device__ __forceinline__ void softmax_stats(const float (&x)[NV], float& m, float& sum) {
  m = x[0];
#pragma unroll
  for (int j = 1; j < NV; ++j) asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(x[j]));
  m = warp_max(m);
  if (m == -INFINITY) m = 0.0f;  // nothing to choose: every exponential is 0, and the sum
  sum = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) sum += expf(x[j] - m);
  sum = warp_sum(sum);
}
__device__ __forceinline__ float softmax_of(float x, float m, float sum) {
  const float e = expf(x - m);
  return sum == 0.0f ? 0.0f : e / sum;
}

// The value that a group is ranked by, from its two largest keys.
__device__ __forceinline__ float group_value(const RouteParams& p, bool by_score, float m, float sum, uint32_t a, uint32_t b) {
  if (p.group_score != MX_GROUP_TOP2) return from_key(a);
  float va = from_key(a), vb = from_key(b);
  if (!by_score) {  // the keys are those of logits, and scores are added
    va = softmax_of(va, m, sum);
    vb = b ? softmax_of(vb, m, sum) : 0.0f;
  }
  return b ? va + vb : va;  // (a group of one expert has one score)
}

// The two largest keys of a set, a >= b.
__device__ __forceinline__ void top2_add(uint32_t& a, uint32_t& b, uint32_t k) {
  b = max(b, min(a, k));
  a = max(a, k);
}

// The topk best keys of the warp, in descending order, equal ones in the order of the experts: lane i gets
// the i-th one's expert.  `smem`: 64 words of the warp.
//
// Taking the best of all keys topk times costs a pass over a lane's NV keys each time.  So the field is cut down
// first: the topk-th largest of the lanes' own maxima is a floor under the topk-th largest key, and what is not
// below it -- little more than topk keys -- is laid out one per lane, where taking the best is a reduction and
// a vote.  More than 32 of them (many equal keys), or fewer lanes with candidates than topk: key by key.
// (16384 tokens, 8 of 256 experts in groups: 1432 instructions per token key by key.)
template <int NV>
__device__ __forceinline__ void top_k(const RouteParams& p, uint32_t (&key)[NV], uint32_t e0, uint32_t lane,
                                      uint32_t* smem, uint32_t& my_id) {
  uint32_t best = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) best = max(best, key[j]);
  if constexpr (NV > 1) {
    uint32_t floor_key = 0, rest = best;
    for (uint32_t i = 0; i < p.topk; ++i) {
      floor_key = __reduce_max_sync(kFull, rest);
      if (lane == __ffs(__ballot_sync(kFull, rest == floor_key)) - 1) rest = 0;
    }
    uint32_t n = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) n += key[j] >= floor_key ? 1u : 0u;
    uint32_t upto = n;
#pragma unroll
    for (uint32_t o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(kFull, upto, o);
      if (lane >= o) upto += v;
    }
    const uint32_t all = __shfl_sync(kFull, upto, 31);
    if (floor_key != 0 && all <= 32) {
      uint32_t at = upto - n;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (key[j] >= floor_key) {
          smem[at] = key[j];
          smem[32 + at] = e0 + j;
          ++at;
        }
      }
      __syncwarp();
      uint32_t k = lane < all ? smem[lane] : 0u;
      const uint32_t id = lane < all ? smem[32 + lane] : 0u;
      uint32_t place = 32;  // of this lane's key in the order
      for (uint32_t i = 0; i < p.topk; ++i) {
        const uint32_t top = __reduce_max_sync(kFull, k);
        if (lane == __ffs(__ballot_sync(kFull, k == top)) - 1) {
          place = i;
          k = 0;
        }
      }
      __syncwarp();
      if (place < 32) smem[place] = id;
      __syncwarp();
      my_id = lane < p.topk ? smem[lane] : 0u;
      return;
    }
  }
  for (uint32_t i = 0; i < p.topk; ++i) {
    const uint32_t top = __reduce_max_sync(kFull, best);
    const uint32_t winner = __ffs(__ballot_sync(kFull, best == top)) - 1;
    uint32_t at = 0;
    if (lane == winner) {
      best = 0;
      bool found = false;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const bool hit = !found && key[j] == top;
        if (hit) { at = e0 + j; key[j] = 0u; found = true; }
        best = max(best, key[j]);
      }
    }
    at = __shfl_sync(kFull, at, winner);
    if (lane == i) my_id = at;
  }
}

template <int DTYPE, int NV>
__global__ void __launch_bounds__(32 * kRouteWarps) route_kernel(const RouteParams p) {
  extern __shared__ uint32_t keys_smem[];
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t token = blockIdx.x * kRouteWarps + warp;
  if (token >= p.tokens) return;
  const uint32_t e0 = lane * NV;
  const bool soft = p.score == MX_SCORE_SOFTMAX;
  float x[NV];
  load_logits<DTYPE, NV>(p, token, lane, x);
  float m = 0.0f, sum = 1.0f;
  if (soft) softmax_stats<NV>(x, m, sum);
  uint32_t key[NV];
  const bool by_score = !soft || p.bias != nullptr;
  // a group's two best values are added: softmax without a bias needs the scores there too
  if (by_score) {
    float b[NV];
    if (p.bias) {
      load_bias<NV>(p, e0, b);
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) b[j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) key[j] = order_key((soft ? softmax_of(x[j], m, sum) : sigmoid(x[j])) + b[j]);
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) key[j] = order_key(x[j]);
  }
  if (e0 + NV > p.experts) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (e0 + j >= p.experts) key[j] = 0u;
  }
  if (p.groups > 1) {
    uint32_t rank_key = 0;  // of group `lane`
    const uint32_t lanes_per_group = p.group_size / NV;
    const bool aligned = p.group_size % NV == 0 && (lanes_per_group & (lanes_per_group - 1)) == 0;
    if (aligned) {  // a group is a power of two of whole lanes
      uint32_t a = 0, b = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) top2_add(a, b, key[j]);
      for (uint32_t o = 1; o < lanes_per_group; o <<= 1) {
        const uint32_t a2 = __shfl_xor_sync(kFull, a, o), b2 = __shfl_xor_sync(kFull, b, o);
        b = max(max(b, b2), min(a, a2));
        a = max(a, a2);
      }
      const uint32_t k = order_key(group_value(p, by_score, m, sum, a, b));
      rank_key = __shfl_sync(kFull, k, (lane * lanes_per_group) & 31);
    } else {        // through shared memory, a lane per group
      uint32_t* mine = keys_smem + warp * (64 + NV * 32) + 64;
#pragma unroll
      for (int j = 0; j < NV; ++j) mine[e0 + j] = key[j];
      __syncwarp();
      if (lane < p.groups) {
        uint32_t a = 0, b = 0;
        for (uint32_t i = 0; i < p.group_size; ++i) top2_add(a, b, mine[lane * p.group_size + i]);
        rank_key = order_key(group_value(p, by_score, m, sum, a, b));
      }
    }
    // the topk_groups best groups, the lower one among equals (every group has a key above 0)
    uint32_t kept = 0, rest = lane < p.groups ? rank_key : 0u;
    for (uint32_t i = 0; i < p.topk_groups; ++i) {
      const uint32_t top = __reduce_max_sync(kFull, rest);
      const uint32_t who = __ffs(__ballot_sync(kFull, rest == top)) - 1;
      kept |= 1u << who;
      if (lane == who) rest = 0u;
    }
    if (aligned) {
      const bool mine_kept = e0 < p.experts && ((kept >> fastdiv(e0, p.by_group_size)) & 1u);
#pragma unroll
      for (int j = 0; j < NV; ++j) key[j] = mine_kept ? key[j] : 0u;
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (e0 + j < p.experts && !((kept >> fastdiv(e0 + j, p.by_group_size)) & 1u)) key[j] = 0u;
      __syncwarp();  // the keys in shared memory have been read
    }
  }
  uint32_t my_id = 0;
  top_k<NV>(p, key, e0, lane, keys_smem + warp * (64 + NV * 32), my_id);
  float my_s;
  const bool live = lane < p.topk;
  const float my_x = live ? load_logit<DTYPE>(p, (size_t)token * p.experts + my_id) : 0.0f;
  my_s = live ? (soft ? softmax_of(my_x, m, sum) : sigmoid(my_x)) : 0.0f;
  float w = my_s;
  if (p.renormalize) {
    const float total = warp_sum(my_s);
    w = total == 0.0f ? 0.0f : my_s / total;
  }
  if (live) {
    p.ids[(size_t)token * p.topk + lane] = (int32_t)my_id;
    p.weights[(size_t)token * p.topk + lane] = w * p.scale;
  }
}

// ---- a few lanes per token ---------------------------------------------------------------------------
// With many tokens the instructions of a warp per token bound the call: most of them are steps of a reduction, done
// by 32 lanes for one token.  Here L lanes share a token, kPartKeys consecutive experts each, and a warp
// takes 32 / L tokens.  The best kPartK keys come out of sorting networks -- eight keys at a time, merged into
// the lane's list, then the lanes' lists in pairs.  What is not below the topk-th goes to shared memory, where each
// finds its place by counting those before it.  (16384 tokens, 8 of 256 in groups, sigmoid and bias: 12.6 us, 16.6
// with a warp per token; 262144 tokens, 6 of 64: 36 us, 106.  Comparisons and selections bound it, which issue
// at half rate.)

constexpr int kPartKeys = 16;        // experts per lane
constexpr uint32_t kPartK = 8;       // most choices
constexpr uint32_t kPartField = 24;  // candidates that are counted against each other; more (equal keys): one by one

__device__ __forceinline__ void descend(uint32_t& a, uint32_t& b) {
  const uint32_t hi = max(a, b);
  b = min(a, b);
  a = hi;
}
__device__ __forceinline__ void sort8(uint32_t (&k)[8]) {  // odd-even merge sort
  descend(k[0], k[1]); descend(k[2], k[3]); descend(k[4], k[5]); descend(k[6], k[7]);
  descend(k[0], k[2]); descend(k[1], k[3]); descend(k[4], k[6]); descend(k[5], k[7]);
  descend(k[1], k[2]); descend(k[5], k[6]);
  descend(k[0], k[4]); descend(k[1], k[5]); descend(k[2], k[6]); descend(k[3], k[7]);
  descend(k[2], k[4]); descend(k[3], k[5]);
  descend(k[1], k[2]); descend(k[3], k[4]); descend(k[5], k[6]);
}
__device__ __forceinline__ void bitonic8(uint32_t (&k)[8]) {  // a bitonic sequence in descending order
#pragma unroll
  for (int d = 4; d; d >>= 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((i & d) == 0) descend(k[i], k[i + d]);
  }
}

// The eight best of two descending lists, into the first.
__device__ __forceinline__ void merge8(uint32_t (&k)[8], const uint32_t (&other)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) k[i] = max(k[i], other[7 - i]);
  bitonic8(k);
}

// The lane's kPartKeys numbers, in fours: number e0 and the next three, then those `step` fours further on; past the
// end of the row -Inf.  No load depends on a branch, and all are in flight at once.  Rows of a multiple of four numbers.
template <int DTYPE, int step = 1>
__device__ __forceinline__ void load_part(const void* row, size_t at, uint32_t experts, uint32_t e0, float (&x)[kPartKeys]) {
  constexpr int V = kPartKeys / 4;
  if constexpr (DTYPE == MX_F32) {
    float4 v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t e = e0 + 4 * step * i;
      v[i] = __ldg(reinterpret_cast<const float4*>((const float*)row + at + (e < experts ? e : 0u)));
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[4 * i] = v[i].x; x[4 * i + 1] = v[i].y; x[4 * i + 2] = v[i].z; x[4 * i + 3] = v[i].w;
    }
  } else {
    uint2 v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t e = e0 + 4 * step * i;
      v[i] = __ldg(reinterpret_cast<const uint2*>((const uint16_t*)row + at + (e < experts ? e : 0u)));
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[4 * i] = __uint_as_float(v[i].x << 16); x[4 * i + 1] = __uint_as_float(v[i].x & 0xFFFF0000u);
      x[4 * i + 2] = __uint_as_float(v[i].y << 16); x[4 * i + 3] = __uint_as_float(v[i].y & 0xFFFF0000u);
    }
  }
  if (e0 + 4 * step * (V - 1) >= experts) {
#pragma unroll
    for (int j = 0; j < kPartKeys; ++j)
      if (e0 + 4 * step * (j / 4) >= experts) x[j] = -INFINITY;
  }
}

// Maximum and sum of exponentials of a token's logits; `keep`: x becomes the exponentials.
template <int L>
__device__ __forceinline__ void part_softmax(float (&x)[kPartKeys], float& m, float& sum, bool keep) {
  m = x[0];
#pragma unroll
  for (int j = 1; j < kPartKeys; ++j) asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(x[j]));
#pragma unroll
  for (int o = 1; o < L; o <<= 1) {
    const float w = __shfl_xor_sync(kFull, m, o);
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(w));
  }
  if (m == -INFINITY) m = 0.0f;  // nothing to choose: every exponential is 0, and the sum
  sum = 0.0f;
#pragma unroll
  for (int j = 0; j < kPartKeys; ++j) {
    const float e = expf(x[j] - m);
    sum += e;
    if (keep) x[j] = e;
  }
#pragma unroll
  for (int o = 1; o < L; o <<= 1) sum += __shfl_xor_sync(kFull, sum, o);
}

// Needs experts % 4 == 0, experts <= kPartKeys L, topk <= kPartK, and the bias on a 16-byte boundary.
template <int DTYPE, int L>
__global__ void __launch_bounds__(32 * kRouteWarps) route_part_kernel(const RouteParams p) {
  constexpr uint32_t kTokens = 32 / L;  // of a warp
  __shared__ uint4 keys[kRouteWarps][kPartKeys / 4][32];
  __shared__ uint2 fields[kRouteWarps][kTokens][kPartField];
  __shared__ uint32_t chosen[kRouteWarps][kTokens][kPartK];
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, q = lane % L, part = lane / L, e0 = kPartKeys * q;
  const uint32_t token0 = (blockIdx.x * kRouteWarps + warp) * kTokens;
  if (token0 >= p.tokens) return;
  const uint32_t token = min(token0 + part, p.tokens - 1);  // (past the end: computed, not written)
  const bool soft = p.score == MX_SCORE_SOFTMAX, by_score = !soft || p.bias != nullptr;
  float m = 0.0f, sum = 1.0f;
  uint32_t key[kPartKeys];
  {
    float x[kPartKeys], b[kPartKeys];
    load_part<DTYPE>(p.logits, (size_t)token * p.experts, p.experts, e0, x);
    if (p.bias) {
      load_part<MX_F32>(p.bias, 0, p.experts, e0, b);
    } else {
#pragma unroll
      for (int j = 0; j < kPartKeys; ++j) b[j] = 0.0f;
    }
    if (soft) part_softmax<L>(x, m, sum, false);
    if (by_score) {
#pragma unroll
      for (int j = 0; j < kPartKeys; ++j) x[j] = (soft ? softmax_of(x[j], m, sum) : sigmoid(x[j])) + b[j];
    }
#pragma unroll
    for (int j = 0; j < kPartKeys; ++j) key[j] = order_key(x[j]);
    if (e0 + kPartKeys > p.experts) {
#pragma unroll
      for (int j = 0; j < kPartKeys; ++j)
        if (e0 + j >= p.experts) key[j] = 0u;
    }
  }
  auto lay_down = [&]() {  // the keys where they can be read by number
#pragma unroll
    for (int i = 0; i < kPartKeys / 4; ++i) keys[warp][i][lane] = make_uint4(key[4 * i], key[4 * i + 1], key[4 * i + 2], key[4 * i + 3]);
  };
  if (p.groups > 1 && p.group_lanes) {  // a group is a power of two of whole lanes
    const uint32_t lanes = p.group_lanes;  // of a group
    uint32_t a = 0, b = 0;
#pragma unroll
    for (int j = 0; j < kPartKeys; ++j) top2_add(a, b, key[j]);
#pragma unroll
    for (uint32_t o = 1; o < L; o <<= 1) {
      if (o < lanes) {
        const uint32_t a2 = __shfl_xor_sync(kFull, a, o), b2 = __shfl_xor_sync(kFull, b, o);
        b = max(max(b, b2), min(a, a2));
        a = max(a, a2);
      }
    }
    const uint32_t mine = order_key(group_value(p, by_score, m, sum, a, b)), first = e0 < p.experts ? q & ~(lanes - 1) : q;
    uint32_t before = 0;  // the better groups, and the equal ones of lower experts
    for (uint32_t g = 0; g < p.groups; ++g) {
      const uint32_t other = __shfl_sync(kFull, mine, g * lanes, L);
      before += other > mine || (other == mine && g * lanes < first) ? 1u : 0u;
    }
#pragma unroll
    for (int j = 0; j < kPartKeys; ++j) key[j] = before < p.topk_groups ? key[j] : 0u;
  } else if (p.groups > 1) {  // through shared memory, L groups at a time
    lay_down();
    __syncwarp();
    uint32_t* value = reinterpret_cast<uint32_t*>(fields[warp][part]);  // 32 groups at most
    for (uint32_t g = q; g < p.groups; g += L) {
      uint32_t a = 0, b = 0;
      for (uint32_t e = g * p.group_size; e < (g + 1) * p.group_size; ++e)
        top2_add(a, b, reinterpret_cast<const uint32_t*>(&keys[warp][(e % kPartKeys) >> 2][part * L + e / kPartKeys])[e & 3]);
      value[g] = order_key(group_value(p, by_score, m, sum, a, b));
    }
    __syncwarp();
    uint32_t kept = 0;
    for (uint32_t g = q; g < p.groups; g += L) {
      uint32_t before = 0;
      for (uint32_t o = 0; o < p.groups; ++o) before += value[o] > value[g] || (value[o] == value[g] && o < g) ? 1u : 0u;
      kept |= before < p.topk_groups ? 1u << g : 0u;
    }
#pragma unroll
    for (int o = 1; o < L; o <<= 1) kept |= __shfl_xor_sync(kFull, kept, o);
    uint32_t g = fastdiv(e0, p.by_group_size), at = e0 - g * p.group_size;
#pragma unroll
    for (int j = 0; j < kPartKeys; ++j) {
      key[j] = g < p.groups && ((kept >> g) & 1u) ? key[j] : 0u;
      if (++at == p.group_size) { at = 0; ++g; }
    }
  }
  lay_down();
  auto key_at = [&](uint32_t s) { return reinterpret_cast<const uint32_t*>(&keys[warp][s >> 2][lane])[s & 3]; };
  // A floor under the topk-th best: with up to 4 lanes that key itself, else the topk-th of the best of every four
  // keys, which lets few more through and is cheaper (4 lanes: 16384 tokens, 6 of 64: 5.8 us; 6.6 with fours)
  uint32_t best[8], k[8];
  if constexpr (L < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) { best[j] = key[j]; k[j] = key[8 + j]; }
    sort8(best);
    sort8(k);
    merge8(best, k);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) best[j] = max(max(key[4 * j], key[4 * j + 1]), max(key[4 * j + 2], key[4 * j + 3]));
    descend(best[0], best[1]); descend(best[2], best[3]);
    descend(best[0], best[2]); descend(best[1], best[3]);
    descend(best[1], best[2]);
    if constexpr (L < 32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) best[7 - j] = __shfl_xor_sync(kFull, best[j], 1);
      bitonic8(best);
    }
  }
  uint32_t floor_key;
  if constexpr (L < 32) {
#pragma unroll
    for (int o = L < 8 ? 1 : 2; o < L; o <<= 1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) k[j] = __shfl_xor_sync(kFull, best[j], o);
      merge8(best, k);
    }
    floor_key = best[0];
#pragma unroll
    for (uint32_t j = 1; j < kPartK; ++j) floor_key = j < p.topk ? best[j] : floor_key;
  } else {  // the whole warp: its best, taken off the lane that has it, topk times
    floor_key = 0;
    for (uint32_t i = 0; i < p.topk; ++i) {
      floor_key = __reduce_max_sync(kFull, best[0]);
      if (lane == __ffs(__ballot_sync(kFull, best[0] == floor_key)) - 1) {
        best[0] = best[1]; best[1] = best[2]; best[2] = best[3]; best[3] = 0;
      }
    }
  }
  floor_key = max(floor_key, 1u);  // (no candidate has 0)
  uint32_t hits = 0;
#pragma unroll
  for (int s = 0; s < kPartKeys; ++s) hits |= key[s] >= floor_key ? 1u << s : 0u;
  const uint32_t n = __popc(hits);
  uint32_t upto = n;
#pragma unroll
  for (uint32_t o = 1; o < L; o <<= 1) {
    const uint32_t v = __shfl_up_sync(kFull, upto, o, L);
    if (q >= o) upto += v;
  }
  const uint32_t all = __shfl_sync(kFull, upto, L - 1, L);
  if (!__any_sync(kFull, all > kPartField)) {
    uint2* field = fields[warp][part];  // in the order of the experts
    for (uint32_t at = upto - n; hits; ++at, hits &= hits - 1) {
      const uint32_t s = __ffs(hits) - 1;
      field[at] = make_uint2(key_at(s), e0 + s);
    }
    __syncwarp();
    for (uint32_t c = q; c < all; c += L) {
      const uint2 me = field[c];
      uint32_t place = 0;
#pragma unroll 4
      for (uint32_t j = 0; j < all; ++j) place += field[j].x > me.x || (field[j].x == me.x && j < c) ? 1u : 0u;
      if (place < p.topk) chosen[warp][part][place] = me.y;
    }
  } else {  // the next in the order, topk times
    uint32_t last_key = 0xffffffffu;
    int32_t last = -1;
    for (uint32_t r = 0; r < p.topk; ++r) {
      uint32_t top = 0, id = 0;
      for (uint32_t s = 0; s < (uint32_t)kPartKeys; ++s) {
        const uint32_t k = key_at(s), e = e0 + s;
        if (k > top && (k < last_key || (k == last_key && (int32_t)e > last))) { top = k; id = e; }
      }
#pragma unroll
      for (int o = 1; o < L; o <<= 1) {
        const uint32_t k2 = __shfl_xor_sync(kFull, top, o), id2 = __shfl_xor_sync(kFull, id, o);
        if (k2 > top || (k2 == top && id2 < id)) { top = k2; id = id2; }
      }
      last_key = top;
      last = (int32_t)id;
      if (q == 0) chosen[warp][part][r] = id;
    }
  }
  __syncwarp();
  constexpr int R = L < (int)kPartK ? kPartK / L : 1;  // choices per lane
  float s[R], total = 0.0f;
  uint32_t id[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool live = q + L * r < p.topk;
    id[r] = live ? chosen[warp][part][q + L * r] : 0u;
    const float x = load_logit<DTYPE>(p, (size_t)token * p.experts + id[r]);
    s[r] = live ? (soft ? softmax_of(x, m, sum) : sigmoid(x)) : 0.0f;
    total += s[r];
  }
#pragma unroll
  for (int o = 1; o < L; o <<= 1) total += __shfl_xor_sync(kFull, total, o);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (q + L * r < p.topk && token0 + part < p.tokens) {
      const size_t at = (size_t)token * p.topk + q + L * r;
      p.ids[at] = (int32_t)id[r];
      p.weights[at] = (p.renormalize ? (total == 0.0f ? 0.0f : s[r] / total) : s[r]) * p.scale;
    }
  }
}

// With S = sum of the chosen scores and d = dweights: renormalised weights w_j = scale s_j / S give
// ds_j = scale (d_j - sum_i d_i s_i / S) / S, others ds_j = scale d_j; then
//   softmax: dx_e = s_e (ds_e - sum_i ds_i s_i),   sigmoid: dx_e = ds_e s_e (1 - s_e).
template <int DTYPE, int NV>
__global__ void __launch_bounds__(32 * kRouteWarps) route_backward_kernel(const RouteParams p) {
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t token = blockIdx.x * kRouteWarps + warp;
  if (token >= p.tokens) return;
  const uint32_t e0 = lane * NV;
  const bool soft = p.score == MX_SCORE_SOFTMAX;
  float x[NV];
  load_logits<DTYPE, NV>(p, token, lane, x);
  float m = 0.0f, sum = 1.0f;
  if (soft) softmax_stats<NV>(x, m, sum);
  int32_t id = -1;
  float d = 0.0f, s = 0.0f;
  if (lane < p.topk) {
    id = __ldg(p.ids + (size_t)token * p.topk + lane);
    d = __ldg(p.dweights + (size_t)token * p.topk + lane);
    if ((uint32_t)id < p.experts) {
      const size_t at = (size_t)token * p.experts + (uint32_t)id;
      const float xs = load_logit<DTYPE>(p, at);
      s = soft ? softmax_of(xs, m, sum) : sigmoid(xs);
    } else {
      id = -1;
      d = 0.0f;
    }
  }
  float ds = p.scale * d;
  if (p.renormalize) {
    const float total = warp_sum(s), dot = warp_sum(d * s);
    ds = total == 0.0f || id < 0 ? 0.0f : p.scale * (d - dot / total) / total;
  }
  const float inner = soft ? warp_sum(ds * s) : 0.0f;
  // ds spread over the experts by way of shared memory
  extern __shared__ float ds_smem[];
  float* mine = ds_smem + warp * (NV * 32);
#pragma unroll
  for (int j = 0; j < NV; ++j) mine[j * 32 + lane] = 0.0f;
  __syncwarp();
  if (id >= 0) atomicAdd(mine + ((uint32_t)id % NV) * 32 + (uint32_t)id / NV, ds);
  __syncwarp();
  float o[NV];
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    o[j] = mine[j * 32 + lane];
    if (soft) {
      o[j] = expf(x[j] - m) * inv * (o[j] - inner);
    } else if (o[j] != 0.0f) {
      const float t = expf(-fabsf(x[j]));  // s (1 - s) without the difference: t / (1 + t)^2
      o[j] *= t / ((1.0f + t) * (1.0f + t));
    }
  }
  const size_t at = (size_t)token * p.experts + e0;
  if constexpr (NV % 4 == 0) {
    if ((p.experts & 3u) == 0 && e0 + NV <= p.experts) {
#pragma unroll
      for (int i = 0; i < NV / 4; ++i) {
        if constexpr (DTYPE == MX_F32) {
          reinterpret_cast<float4*>((float*)p.dlogits + at)[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        } else {
          uint2 v;
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v.x) : "f"(o[4 * i + 1]), "f"(o[4 * i]));
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v.y) : "f"(o[4 * i + 3]), "f"(o[4 * i + 2]));
          reinterpret_cast<uint2*>((uint16_t*)p.dlogits + at)[i] = v;
        }
      }
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (e0 + j < p.experts) {
      if constexpr (DTYPE == MX_F32) {
        ((float*)p.dlogits)[at + j] = o[j];
      } else {
        uint32_t v;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(0.0f), "f"(o[j]));
        ((uint16_t*)p.dlogits)[at + j] = (uint16_t)v;
      }
    }
  }
}

// The same with L lanes per token and up to kPartKeys L experts, for the reason given above route_part_kernel: the
// reductions of a warp per token.  Order does not matter here, and a lane holds every L-th four experts, so that
// the lanes' vectors meet in whole sectors.  Needs experts % 4 == 0 and topk <= kPartK.
template <int DTYPE, int L>
__global__ void __launch_bounds__(32 * kRouteWarps) route_backward_part_kernel(const RouteParams p) {
  constexpr uint32_t kTokens = 32 / L;
  constexpr int V = kPartKeys / 4;
  __shared__ float4 ds_of[kRouteWarps][V][32];
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, q = lane % L, part = lane / L;
  const uint32_t token0 = (blockIdx.x * kRouteWarps + warp) * kTokens;
  if (token0 >= p.tokens) return;
  const bool live = token0 + part < p.tokens;
  const size_t token = min(token0 + part, p.tokens - 1), row = token * p.experts;
  const bool soft = p.score == MX_SCORE_SOFTMAX;
  constexpr int R = L < (int)kPartK ? kPartK / L : 1;  // choices per lane
  int32_t id[R];
  float d[R], xs[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t c = q + L * r;
    id[r] = c < p.topk ? __ldg(p.ids + token * p.topk + c) : -1;
    d[r] = c < p.topk ? __ldg(p.dweights + token * p.topk + c) : 0.0f;
    if ((uint32_t)id[r] >= p.experts) { id[r] = -1; d[r] = 0.0f; }
    xs[r] = load_logit<DTYPE>(p, row + (id[r] < 0 ? 0u : (uint32_t)id[r]));
  }
#pragma unroll
  for (int i = 0; i < V; ++i) ds_of[warp][i][lane] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float x[kPartKeys];  // (a sigmoid's gradient is that of the chosen logits alone)
  float m = 0.0f, sum = 1.0f;
  if (soft) {
    load_part<DTYPE, L>(p.logits, row, p.experts, 4 * q, x);
    part_softmax<L>(x, m, sum, true);
  }
  float s[R], ds[R], total = 0.0f, dot = 0.0f, inner = 0.0f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    s[r] = id[r] < 0 ? 0.0f : soft ? softmax_of(xs[r], m, sum) : sigmoid(xs[r]);
    total += s[r];
    dot += d[r] * s[r];
  }
  if (p.renormalize) {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
      total += __shfl_xor_sync(kFull, total, o);
      dot += __shfl_xor_sync(kFull, dot, o);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    ds[r] = p.scale * d[r];
    if (p.renormalize) ds[r] = total == 0.0f || id[r] < 0 ? 0.0f : p.scale * (d[r] - dot / total) / total;
    inner += ds[r] * s[r];
    if (!soft && ds[r] != 0.0f) {
      const float t = expf(-fabsf(xs[r]));  // s (1 - s) without the difference: t / (1 + t)^2
      ds[r] *= t / ((1.0f + t) * (1.0f + t));
    }
  }
  if (soft) {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) inner += __shfl_xor_sync(kFull, inner, o);
  }
  __syncwarp();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (id[r] >= 0) {
      const uint32_t unit = (uint32_t)id[r] >> 2;
      atomicAdd(reinterpret_cast<float*>(&ds_of[warp][unit / L][part * L + unit % L]) + (id[r] & 3), ds[r]);
    }
  }
  __syncwarp();
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float4 v = ds_of[warp][i][lane];
    float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (soft) o[j] = x[4 * i + j] * inv * (o[j] - inner);
    const uint32_t e0 = 4 * (L * i + q);
    if (live && e0 < p.experts) {
      if constexpr (DTYPE == MX_F32) {
        *reinterpret_cast<float4*>((float*)p.dlogits + row + e0) = make_float4(o[0], o[1], o[2], o[3]);
      } else {
        uint2 w;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.x) : "f"(o[1]), "f"(o[0]));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.y) : "f"(o[3]), "f"(o[2]));
        *reinterpret_cast<uint2*>((uint16_t*)p.dlogits + row + e0) = w;
      }
    }
  }
}

RouteParams route_params(const RouteArgs& a, bool backward) {
  RouteParams p;
  p.logits = a.logits; p.bias = a.bias; p.dweights = a.dweights; p.ids = a.ids; p.weights = a.weights;
  p.dlogits = a.dlogits; p.tokens = (uint32_t)a.tokens; p.experts = (uint32_t)a.experts;
  p.topk = (uint32_t)a.route.topk; p.score = (uint32_t)a.route.score;
  p.groups = backward ? 1u : (uint32_t)a.route.groups;  // (the gradient has no groups: nobody has checked that field)
  p.topk_groups = (uint32_t)a.route.topk_groups; p.group_score = (uint32_t)a.route.group_score;
  p.renormalize = a.route.renormalize ? 1u : 0u; p.scale = a.route.scale;
  p.group_size = p.experts / p.groups;
  p.by_group_size = make_fastdiv(p.group_size);
  const uint32_t lanes = p.group_size / kPartKeys;
  p.group_lanes = p.group_size % kPartKeys == 0 && (lanes & (lanes - 1)) == 0 ? lanes : 0u;
  return p;
}

template <int DTYPE, int NV>
cudaError_t launch_nv(const RouteParams& p, bool backward, cudaStream_t stream) {
  const dim3 grid((p.tokens + kRouteWarps - 1) / kRouteWarps), block(32 * kRouteWarps);
  if (backward) return launch_pdl(route_backward_kernel<DTYPE, NV>, grid, block, sizeof(float) * 32 * NV * kRouteWarps, stream, p);
  return launch_pdl(route_kernel<DTYPE, NV>, grid, block, sizeof(uint32_t) * (64 + NV * 32) * kRouteWarps, stream, p);
}

template <int DTYPE, int L>
cudaError_t launch_part(const RouteParams& p, bool backward, cudaStream_t stream) {
  const uint32_t per_cta = 32 / L * kRouteWarps;
  return launch_pdl(backward ? route_backward_part_kernel<DTYPE, L> : route_part_kernel<DTYPE, L>,
                    dim3((p.tokens + per_cta - 1) / per_cta), dim3(32 * kRouteWarps), 0, stream, p);
}

template <int DTYPE>
cudaError_t launch_dtype(const RouteParams& p, bool backward, cudaStream_t stream) {
  // A few lanes per token, or a warp (in parentheses; us).  Few tokens are a matter of one token's latency, which is
  // the warp's: 8 experts, top-2, 2048 tokens 2.7 (2.3), 4096 2.7 (2.9); 64, top-8, 1024 3.2 (2.8), 2048 3.3 (3.9); 256, top-8,
  // 16 2.9 (2.8), in 8 groups, sigmoid and bias 1024 3.8 (3.7), 2048 5.5 (6.1), 65536 40 (52).  (Top-2 gains less: 256, sigmoid and bias
  // 4096 6.4 (5.1), 65536 32.5 (32.8).)  With more than 256 a lane of the warp has 16 keys either way, and what is left is
  // the sorting networks': 512, top-8, 16 2.8 (3.0), 16384 14.8 (15.7); 384 in 8 groups, 1024 6.2 (8.1); it loses at most 5 % where the
  // groups are no power of two of whole lanes (320 in 8, 65536 99 (95)).
  // Gradient: 64 experts, 1024 tokens 2.4 (2.2), 2048 2.4 (2.5); 128, 16 2.1 (2.2), 16384 5.0 (6.8).
  const bool enough = backward ? p.experts > 64 || p.tokens >= 2048u
                               : p.experts > 256 || p.tokens >= (p.experts > 32 ? 2048u : 4096u);
  if (enough && p.topk <= kPartK && p.experts % 4 == 0 && p.experts <= 32 * kPartKeys &&
      (backward || (reinterpret_cast<uintptr_t>(p.bias) & 15u) == 0)) {
    if (p.experts <= 2 * kPartKeys) return launch_part<DTYPE, 2>(p, backward, stream);
    if (p.experts <= 4 * kPartKeys) return launch_part<DTYPE, 4>(p, backward, stream);
    if (p.experts <= 8 * kPartKeys) return launch_part<DTYPE, 8>(p, backward, stream);
    if (p.experts <= 16 * kPartKeys) return launch_part<DTYPE, 16>(p, backward, stream);
    return launch_part<DTYPE, 32>(p, backward, stream);
  }
  if (p.experts <= 32) return launch_nv<DTYPE, 1>(p, backward, stream);
  if (p.experts <= 64) return launch_nv<DTYPE, 2>(p, backward, stream);
  if (p.experts <= 128) return launch_nv<DTYPE, 4>(p, backward, stream);
  if (p.experts <= 256) return launch_nv<DTYPE, 8>(p, backward, stream);
  if (p.experts <= 512) return launch_nv<DTYPE, 16>(p, backward, stream);
  return launch_nv<DTYPE, 32>(p, backward, stream);
}

}  // namespace

cudaError_t launch_route(const RouteArgs& a) {
  const RouteParams p = route_params(a, false);
  return a.dtype == MX_BF16 ? launch_dtype<MX_BF16>(p, false, a.stream) : launch_dtype<MX_F32>(p, false, a.stream);
}

cudaError_t launch_route_backward(const RouteArgs& a) {
  const RouteParams p = route_params(a, true);
  return a.dtype == MX_BF16 ? launch_dtype<MX_BF16>(p, true, a.stream) : launch_dtype<MX_F32>(p, true, a.stream);
}

}  // namespace mx
