// Rows of tokens to their experts and back: the plan (a stable counting sort of the choices by expert),
// the gather of MX rows into expert order, the weighted sum back to the tokens and its backward pass.
// Everything here is bound by the rows it moves: each is read once and written once.
#include <cuda_runtime.h>

#include "mx.h"
#include "mx_device.cuh"
#include "mx_launch.h"
#include "mx_rows.cuh"

namespace mx {
namespace {

constexpr uint32_t kFull = 0xffffffffu;
constexpr uint32_t kPlanThreads = 512, kPlanWarps = 16, kPlanPerWarp = kPlanChunk / kPlanWarps;

// ---- plan ------------------------------------------------------------------------------------------
// A CTA sorts a chunk of kPlanChunk choices.  Ranks are exact and independent of timing: a warp takes
// 64 consecutive choices, lanes with the same expert find each other by a vote per bit of its number
// (match.any takes 45 clocks of a unit that the SM's warps share), and the warps' counts are added up in warp
// order.  With more than one chunk the chunks' histograms come first, in a launch of their own, and every
// CTA adds up those before its own; where that is more than kPlanDirect numbers a third launch does it once
// for all of them.  (65536 choices of 64 experts: 6.9 us, two launches' latencies mostly; 10.1 with chunks of 2048,
// match.any and a warp per expert.)

struct PlanParams {
  const int32_t* ids;
  int32_t *offsets, *counts, *row_of, *src_of, *hist;
  uint32_t n, experts, align, chunks, rows, scanned;
};
constexpr uint32_t kPlanDirect = 64 * kPlanThreads;  // histogram entries a CTA adds up by itself

__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const PlanParams p) {
  extern __shared__ uint32_t count[];
  pdl_prologue();
  for (uint32_t e = threadIdx.x; e < p.experts; e += kPlanThreads) count[e] = 0;
  __syncthreads();
  const uint32_t c0 = blockIdx.x * kPlanChunk;
  for (uint32_t i = c0 + threadIdx.x; i < min(p.n, c0 + kPlanChunk); i += kPlanThreads) {
    const uint32_t e = (uint32_t)__ldg(p.ids + i);
    if (e < p.experts) atomicAdd(&count[e], 1u);
  }
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < p.experts; e += kPlanThreads)
    p.hist[(size_t)blockIdx.x * p.experts + e] = (int32_t)count[e];
}

__device__ __forceinline__ uint32_t warp_prefix(uint32_t v, uint32_t lane) {  // inclusive
#pragma unroll
  for (uint32_t o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(kFull, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// hist[c][e] becomes the choices of expert e before chunk c; row `chunks` the totals.  A block per 32
// experts (lanes), the chunks in 32 runs (warps).
__global__ void __launch_bounds__(1024) plan_scan_kernel(const PlanParams p) {
  __shared__ uint32_t run[32][33];
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
  const uint32_t per = (p.chunks + 31) / 32, c0 = min(p.chunks, warp * per), c1 = min(p.chunks, c0 + per);
  uint32_t t = 0;
  if (e < p.experts) {
#pragma unroll 8
    for (uint32_t c = c0; c < c1; ++c) t += (uint32_t)p.hist[(size_t)c * p.experts + e];
  }
  run[warp][lane] = t;
  __syncthreads();
  // warp w: the runs of expert w
  const uint32_t v = run[lane][warp], upto = warp_prefix(v, lane);
  run[lane][warp] = upto - v;
  if (lane == 31 && blockIdx.x * 32 + warp < p.experts)
    p.hist[(size_t)p.chunks * p.experts + blockIdx.x * 32 + warp] = (int32_t)upto;
  __syncthreads();
  t = run[warp][lane];
  if (e < p.experts) {
    for (uint32_t c = c0; c < c1; ++c) {
      int32_t* h = p.hist + (size_t)c * p.experts + e;
      const uint32_t x = (uint32_t)*h;
      *h = (int32_t)t;
      t += x;
    }
  }
}

// Shared memory of plan_place_kernel per expert: first row, choices (then the end of its group), rows without
// a choice, and the warps' counts.
inline size_t plan_smem(uint32_t experts) { return (size_t)experts * (3 * sizeof(uint32_t) + kPlanWarps * sizeof(uint16_t)); }

__global__ void __launch_bounds__(kPlanThreads) plan_place_kernel(const PlanParams p) {
  extern __shared__ uint32_t smem[];
  const uint32_t E = p.experts;
  uint32_t* first = smem;               // [E] row of the chunk's first choice
  uint32_t* total_of = smem + E;        // [E] choices of the expert; then the end of its group
  uint32_t* pad_rows = smem + 2 * E;    // [E]
  uint16_t* count = reinterpret_cast<uint16_t*>(smem + 3 * E);  // [warps][E]
  __shared__ uint32_t warp_total[kPlanWarps];
  pdl_prologue();
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t expert[kPlanPerWarp / 32], rank[kPlanPerWarp / 32];
  const uint32_t i0 = blockIdx.x * kPlanChunk + warp * kPlanPerWarp + lane;
#pragma unroll
  for (uint32_t k = 0; k < kPlanPerWarp / 32; ++k) {
    const uint32_t e = i0 + 32 * k < p.n ? (uint32_t)__ldg(p.ids + i0 + 32 * k) : 0xffffffffu;
    expert[k] = e < E ? e : 0xffffffffu;
  }
  for (uint32_t i = threadIdx.x; i < kPlanWarps * E; i += kPlanThreads) count[i] = 0;
  for (uint32_t i = threadIdx.x; i < E; i += kPlanThreads) { first[i] = 0; total_of[i] = 0; }
  __syncthreads();
  uint16_t* mine = count + warp * E;
#pragma unroll
  for (uint32_t k = 0; k < kPlanPerWarp / 32; ++k) {
    const bool live = expert[k] < E;
    uint32_t peers = __ballot_sync(kFull, live);
    for (uint32_t b = 1; b < E; b <<= 1) {
      const uint32_t set = __ballot_sync(kFull, expert[k] & b);
      peers &= expert[k] & b ? set : ~set;
    }
    const uint32_t before = live ? mine[expert[k]] : 0u;
    __syncwarp();
    if (live && (peers & ((1u << lane) - 1u)) == 0) mine[expert[k]] = (uint16_t)(before + __popc(peers));
    __syncwarp();
    rank[k] = before + __popc(peers & ((1u << lane) - 1u));
  }
  // the chunks before this one, and all of them (integers: the order of the additions does not matter)
  if (p.scanned) {
    for (uint32_t e = threadIdx.x; e < E; e += kPlanThreads) {
      first[e] = (uint32_t)p.hist[(size_t)blockIdx.x * E + e];
      total_of[e] = (uint32_t)p.hist[(size_t)p.chunks * E + e];
    }
  } else if (p.chunks > 1) {
    const uint32_t strands = E < kPlanThreads ? kPlanThreads / E : 1u, strand = threadIdx.x / E;
    if (strand < strands) {
      for (uint32_t e = threadIdx.x - strand * E; e < E; e += kPlanThreads) {
        uint32_t all = 0, before = 0;
#pragma unroll 8
        for (uint32_t c = strand; c < p.chunks; c += strands) {
          const uint32_t h = (uint32_t)p.hist[(size_t)c * E + e];
          all += h;
          before += c < blockIdx.x ? h : 0u;
        }
        atomicAdd(&total_of[e], all);
        atomicAdd(&first[e], before);
      }
    }
  }
  __syncthreads();
  // the warps' counts become ranks
  for (uint32_t e = threadIdx.x; e < E; e += kPlanThreads) {
    uint32_t c[kPlanWarps], t = 0;
#pragma unroll
    for (uint32_t w = 0; w < kPlanWarps; ++w) c[w] = count[w * E + e];
#pragma unroll
    for (uint32_t w = 0; w < kPlanWarps; ++w) {
      count[w * E + e] = (uint16_t)t;
      t += c[w];
    }
    if (p.chunks <= 1) total_of[e] = t;
  }
  // groups one after the other, kPlanThreads experts at a time
  uint32_t start = 0;
  for (uint32_t e0 = 0; e0 < E; e0 += kPlanThreads) {
    const uint32_t e = e0 + threadIdx.x, total = e < E ? total_of[e] : 0u;  // (written by this thread, or before the barrier)
    const uint32_t padded = (total + p.align - 1) / p.align * p.align;
    uint32_t scan = warp_prefix(padded, lane);
    if (lane == 31) warp_total[warp] = scan;
    __syncthreads();
    const uint32_t w = lane < kPlanWarps ? warp_total[lane] : 0u;
    scan += start + __reduce_add_sync(kFull, lane < warp ? w : 0u);
    start += __reduce_add_sync(kFull, w);
    if (e < E) {
      first[e] += scan - padded;
      total_of[e] = scan;
      pad_rows[e] = padded - total;
      if (blockIdx.x == 0) {
        p.counts[e] = (int32_t)total;
        p.offsets[e] = (int32_t)(scan - padded);
      }
    }
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[E] = (int32_t)start;
#pragma unroll
  for (uint32_t k = 0; k < kPlanPerWarp / 32; ++k) {
    const uint32_t i = i0 + 32 * k;
    if (i < p.n) {
      const int32_t row = expert[k] < E ? (int32_t)(first[expert[k]] + mine[expert[k]] + rank[k]) : -1;
      p.row_of[i] = row;
      if (row >= 0) p.src_of[row] = (int32_t)i;
    }
  }
  // rows without a choice: the last ones of every group (a warp per group, spread over the blocks), and
  // those behind the last group
  for (uint32_t g = blockIdx.x * kPlanWarps + warp; g < E; g += gridDim.x * kPlanWarps) {
    const uint32_t r1 = total_of[g], n_pad = pad_rows[g];
    for (uint32_t r = r1 - n_pad + lane; r < r1; r += 32) p.src_of[r] = -1;
  }
  for (uint32_t r = start + blockIdx.x * kPlanThreads + threadIdx.x; r < p.rows; r += gridDim.x * kPlanThreads)
    p.src_of[r] = -1;
}

// ---- rows that no choice maps to ---------------------------------------------------------------------
// The blocks behind the tokens' blocks of a launch write them as zeros: `split` blocks per expert for
// the rows that pad its group, then kTailBlocks blocks for the rows behind the last group.
constexpr uint32_t kTailBlocks = 256;

struct ZeroRows {
  const int32_t *offsets, *counts;
  uint32_t experts, rows, split;
};
// About 1024 blocks, since those without rows cost their launch (8 tokens x 512, 8 of 256 experts: gradient 5.4 us; 10.8 with
// 4096).  Where the rows hold more, one for 64 KB up to 4096, over the experts that can be chosen at all (42 tokens x 5408
// FP32, 1 of 128 experts, 115 MB of padding: 26.9 us with 1024 over all of them, 19.8).
inline uint32_t zero_split(int64_t experts, int64_t choices, int64_t rows, int64_t row_bytes) {
  const double bytes = (double)(rows > choices ? rows - choices : 0) * (double)row_bytes;
  const double blocks = bytes / 65536 < 1024 ? 1024 : bytes / 65536 > 4096 ? 4096 : bytes / 65536;
  const int64_t spread = bytes > 32e6 && choices < experts ? (choices ? choices : 1) : experts;
  const int64_t split = (int64_t)blocks / spread;
  return split < 1 ? 1u : split > 32 ? 32u : (uint32_t)split;
}
inline uint32_t zero_blocks(const ZeroRows& z) { return z.experts * z.split + kTailBlocks; }

// Calls f(row) for the rows that block `z` of the zero blocks owns.
template <typename F>
__device__ __forceinline__ void for_zero_rows(const ZeroRows& q, uint32_t z, F f) {
  int64_t r0, r1;
  uint32_t step, at;
  if (z < q.experts * q.split) {
    const uint32_t e = z / q.split;
    r0 = (int64_t)__ldg(q.offsets + e) + __ldg(q.counts + e);
    r1 = __ldg(q.offsets + e + 1);
    step = q.split;
    at = z - e * q.split;
  } else {
    r0 = __ldg(q.offsets + q.experts);
    r1 = q.rows;
    step = kTailBlocks;
    at = z - q.experts * q.split;
  }
  if (r0 < 0) r0 = 0;
  if (r1 > (int64_t)q.rows) r1 = q.rows;
  for (int64_t r = r0 + at; r < r1; r += step) f((uint32_t)r);
}

// ---- gather ------------------------------------------------------------------------------------------

struct GatherParams {
  const uint8_t *elems_in, *scales_in;
  const int32_t *row_of, *src_of;
  uint8_t *elems_out, *scales_out;
  uint32_t tokens, topk, kblocks, row_bytes, layout, scale_blocks, token_blocks;
  FastDiv by_topk;
  ZeroRows zero;
};

constexpr uint32_t kMoveWarps = 8;

// Codes: a warp per token, the row passes through registers once and goes to every row it is chosen for.
// Swizzled scales: a block per 128 output rows, which writes their 512-byte chunks whole -- a row's scale
// words lie 512 bytes apart, and written row by row each is an eighth of a sector (8192 tokens x 4096, 8 of
// 64 experts: 65 us instead of 56.4, which is 5.8 TB/s of rows read once and written eight times; a memset of the
// output runs at 3.9, a copy at 6.5).
template <typename Vec>
__global__ void __launch_bounds__(32 * kMoveWarps) gather_kernel(const GatherParams p) {
  constexpr uint32_t U = 8;  // vectors in flight per lane
  pdl_prologue();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t vecs = p.row_bytes / sizeof(Vec), kchunks = (p.kblocks + 3) >> 2;
  const bool swizzled = p.layout == MX_SCALES_SWIZZLED;
  if (blockIdx.x < p.scale_blocks) {
    // thread u of each half writes word u of a chunk: row u / 4 + 32 (u % 4) of the 128
    const uint32_t u = threadIdx.x & 127u, half = threadIdx.x >> 7, row = blockIdx.x * 128 + (u >> 2) + 32 * (u & 3u);
    const uint32_t i = row < p.zero.rows ? (uint32_t)__ldg(p.src_of + row) : 0xffffffffu;
    const bool live = i < p.tokens * p.topk;
    const uint32_t t = live ? fastdiv(i, p.by_topk) : 0u;
    const uint32_t* src = reinterpret_cast<const uint32_t*>(p.scales_in + scale_offset<MX_SCALES_SWIZZLED>(t, 0, p.kblocks));
    uint32_t* dst = reinterpret_cast<uint32_t*>(p.scales_out) + (size_t)blockIdx.x * kchunks * 128 + u;
    for (uint32_t c0 = half; c0 < kchunks; c0 += 2 * U) {
      uint32_t w[U];
#pragma unroll
      for (uint32_t k = 0; k < U; ++k) w[k] = live && c0 + 2 * k < kchunks ? __ldg(src + (size_t)(c0 + 2 * k) * 128) : 0u;
#pragma unroll
      for (uint32_t k = 0; k < U; ++k)
        if (c0 + 2 * k < kchunks) dst[(size_t)(c0 + 2 * k) * 128] = w[k];
    }
    return;
  }
  const uint32_t block = blockIdx.x - p.scale_blocks;
  if (block < p.token_blocks) {
    const uint32_t t = block * kMoveWarps + warp;
    if (t >= p.tokens) return;
    const int32_t* rows = p.row_of + (size_t)t * p.topk;
    const Vec* src = reinterpret_cast<const Vec*>(p.elems_in + (size_t)t * p.row_bytes);
    for (uint32_t v0 = lane; v0 < vecs; v0 += 32 * U) {
      Vec v[U];
#pragma unroll
      for (uint32_t u = 0; u < U; ++u)
        if (v0 + 32 * u < vecs) v[u] = __ldg(src + v0 + 32 * u);
      for (uint32_t j = 0; j < p.topk; ++j) {
        const uint32_t r = (uint32_t)__ldg(rows + j);
        if (r >= p.zero.rows) continue;
        Vec* dst = reinterpret_cast<Vec*>(p.elems_out + (size_t)r * p.row_bytes);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
          if (v0 + 32 * u < vecs) dst[v0 + 32 * u] = v[u];
      }
    }
    if (!swizzled) {
      for (uint32_t k = lane; k < p.kblocks; k += 32) {
        const uint8_t b = __ldg(p.scales_in + (size_t)t * p.kblocks + k);
        for (uint32_t j = 0; j < p.topk; ++j) {
          const uint32_t r = (uint32_t)__ldg(rows + j);
          if (r < p.zero.rows) p.scales_out[(size_t)r * p.kblocks + k] = b;
        }
      }
    }
    return;
  }
  for_zero_rows(p.zero, block - p.token_blocks, [&](uint32_t r) {
    Vec* dst = reinterpret_cast<Vec*>(p.elems_out + (size_t)r * p.row_bytes);
    for (uint32_t v = threadIdx.x; v < vecs; v += blockDim.x) dst[v] = Vec{};
    if (!swizzled)
      for (uint32_t k = threadIdx.x; k < p.kblocks; k += blockDim.x) p.scales_out[(size_t)r * p.kblocks + k] = 0;
  });
}

// ---- combine -----------------------------------------------------------------------------------------

struct CombineParams {
  const void *y, *dout;
  const float* weights;
  const int32_t* row_of;
  void *out, *dy;
  float* dweights;
  uint32_t tokens, topk, dim, rows, token_blocks;
  ZeroRows zero;
};

// Several CTAs per token, each with a part of the columns.  VEC: 8 elements at a time (dim % 8 == 0), else one.
// Bound by memory: 8192 tokens x 4096 BF16, top-8, 98 us, 6.2 TB/s.
template <int DTYPE, bool VEC>
__global__ void __launch_bounds__(128) combine_kernel(const CombineParams p) {
  pdl_prologue();
  const uint32_t t = blockIdx.x;
  const int32_t* rows = p.row_of + (size_t)t * p.topk;
  const float* wt = p.weights ? p.weights + (size_t)t * p.topk : nullptr;
  if constexpr (VEC) {
    for (uint32_t g = blockIdx.y * blockDim.x + threadIdx.x; g < p.dim / 8; g += gridDim.y * blockDim.x) {
      float acc[8] = {};
#pragma unroll 4
      for (uint32_t j = 0; j < p.topk; ++j) {
        const uint32_t r = (uint32_t)__ldg(rows + j);
        if (r >= p.rows) continue;
        const float w = wt ? __ldg(wt + j) : 1.0f;
        float f[8];
        widen<DTYPE>(load_raw8<DTYPE>(p.y, (size_t)r * p.dim + 8 * (size_t)g), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, f[e], acc[e]);
      }
      store8<DTYPE>(p.out, (size_t)t * p.dim + 8 * (size_t)g, acc);
    }
  } else {
    for (uint32_t c = blockIdx.y * blockDim.x + threadIdx.x; c < p.dim; c += gridDim.y * blockDim.x) {
      float acc = 0.0f;
      for (uint32_t j = 0; j < p.topk; ++j) {
        const uint32_t r = (uint32_t)__ldg(rows + j);
        if (r < p.rows) acc = fmaf(wt ? __ldg(wt + j) : 1.0f, load1<DTYPE>(p.y, (size_t)r * p.dim + c), acc);
      }
      store1<DTYPE>(p.out, (size_t)t * p.dim + c, acc);
    }
  }
}

// A CTA per token, kJ of its choices at a time: every choice's row of dy is written while its dot
// product with dout is formed; the warps' partial products meet in shared memory in warp order.  kJ is the
// number of y rows in flight per thread and costs registers: no more than the token has choices.
// Bound by memory: 8192 tokens x 4096 BF16, top-4, 112.6 us, 5.95 TB/s.
constexpr uint32_t kBackWarps = 8;

template <int DTYPE, bool VEC, uint32_t kJ>
__global__ void __launch_bounds__(32 * kBackWarps) combine_backward_kernel(const CombineParams p) {
  pdl_prologue();
  constexpr uint32_t G = VEC ? 8 : 1;
  const uint32_t units = p.dim / G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x >= p.token_blocks) {
    for_zero_rows(p.zero, blockIdx.x - p.token_blocks, [&](uint32_t r) {
      for (uint32_t g = threadIdx.x; g < units; g += blockDim.x) {
        if constexpr (VEC) {
          const float zero[8] = {};
          store8<DTYPE>(p.dy, (size_t)r * p.dim + 8 * (size_t)g, zero);
        } else {
          store1<DTYPE>(p.dy, (size_t)r * p.dim + g, 0.0f);
        }
      }
    });
    return;
  }
  __shared__ float dots[kBackWarps][kJ];
  const uint32_t t = blockIdx.x;
  for (uint32_t j0 = 0; j0 < p.topk; j0 += kJ) {
    const uint32_t nj = min(kJ, p.topk - j0);
    uint32_t row[kJ];
    float w[kJ], dot[kJ];
#pragma unroll
    for (uint32_t j = 0; j < kJ; ++j) {
      row[j] = j < nj ? (uint32_t)__ldg(p.row_of + (size_t)t * p.topk + j0 + j) : 0xffffffffu;
      w[j] = j < nj && p.weights ? __ldg(p.weights + (size_t)t * p.topk + j0 + j) : 1.0f;
      dot[j] = 0.0f;
    }
    for (uint32_t g = threadIdx.x; g < units; g += blockDim.x) {
      if constexpr (VEC) {
        float d[8];
        widen<DTYPE>(load_raw8<DTYPE>(p.dout, (size_t)t * p.dim + 8 * (size_t)g), d);
        Raw8<DTYPE> raw[kJ];
        if (p.y) {
#pragma unroll
          for (uint32_t j = 0; j < kJ; ++j)
            if (row[j] < p.rows) raw[j] = load_raw8<DTYPE>(p.y, (size_t)row[j] * p.dim + 8 * (size_t)g);
        }
#pragma unroll
        for (uint32_t j = 0; j < kJ; ++j) {
          if (row[j] >= p.rows) continue;
          float o[8];
          if (p.y) {
            widen<DTYPE>(raw[j], o);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot[j] = fmaf(d[e], o[e], dot[j]);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = w[j] * d[e];
          store8<DTYPE>(p.dy, (size_t)row[j] * p.dim + 8 * (size_t)g, o);
        }
      } else {
        const float d = load1<DTYPE>(p.dout, (size_t)t * p.dim + g);
#pragma unroll
        for (uint32_t j = 0; j < kJ; ++j) {
          if (row[j] >= p.rows) continue;
          if (p.y) dot[j] = fmaf(d, load1<DTYPE>(p.y, (size_t)row[j] * p.dim + g), dot[j]);
          store1<DTYPE>(p.dy, (size_t)row[j] * p.dim + g, w[j] * d);
        }
      }
    }
    if (!p.dweights) continue;
#pragma unroll
    for (uint32_t j = 0; j < kJ; ++j) {
#pragma unroll
      for (int o = 16; o; o >>= 1) dot[j] += __shfl_xor_sync(kFull, dot[j], o);
      if (lane == 0) dots[warp][j] = dot[j];
    }
    __syncthreads();
    if (threadIdx.x < nj) {
      float s = 0.0f;
#pragma unroll
      for (uint32_t i = 0; i < kBackWarps; ++i) s += dots[i][threadIdx.x];
      p.dweights[(size_t)t * p.topk + j0 + threadIdx.x] = s;
    }
    __syncthreads();
  }
}

template <int DTYPE, bool VEC>
cudaError_t launch_backward_vec(const MoeMoveArgs& a, const CombineParams& p) {
  const dim3 grid(p.token_blocks + zero_blocks(p.zero)), block(32 * kBackWarps);
  if (p.topk <= 2) return launch_pdl(combine_backward_kernel<DTYPE, VEC, 2>, grid, block, 0, a.stream, p);
  if (p.topk <= 4) return launch_pdl(combine_backward_kernel<DTYPE, VEC, 4>, grid, block, 0, a.stream, p);
  return launch_pdl(combine_backward_kernel<DTYPE, VEC, 8>, grid, block, 0, a.stream, p);
}
template <int DTYPE>
cudaError_t launch_backward_dtype(const MoeMoveArgs& a, const CombineParams& p) {
  return a.dim % 8 == 0 ? launch_backward_vec<DTYPE, true>(a, p) : launch_backward_vec<DTYPE, false>(a, p);
}

ZeroRows zero_rows(const MoeMoveArgs& a, int64_t row_bytes) {
  ZeroRows z;
  z.offsets = a.offsets; z.counts = a.counts; z.experts = (uint32_t)a.experts; z.rows = (uint32_t)a.rows;
  z.split = zero_split(a.experts, a.tokens * a.topk, a.rows, row_bytes);
  return z;
}

}  // namespace

cudaError_t launch_moe_plan(const MoePlanArgs& a) {
  PlanParams p;
  p.ids = a.ids; p.offsets = a.offsets; p.counts = a.counts; p.row_of = a.row_of; p.src_of = a.src_of; p.hist = a.hist; p.rows = (uint32_t)a.rows;
  p.n = (uint32_t)a.n; p.experts = (uint32_t)a.experts; p.align = (uint32_t)a.align;
  p.chunks = (uint32_t)((a.n + kPlanChunk - 1) / kPlanChunk);
  p.scanned = p.chunks > 1 && (uint64_t)p.chunks * p.experts > kPlanDirect ? 1u : 0u;
  static bool attr_set[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(plan_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan_smem(1024));
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  if (p.chunks > 1) {
    e = launch_pdl(plan_count_kernel, dim3(p.chunks), dim3(kPlanThreads), sizeof(uint32_t) * a.experts, a.stream, p);
    if (e != cudaSuccess) return e;
  }
  if (p.scanned) {
    e = launch_pdl(plan_scan_kernel, dim3((p.experts + 31) / 32), dim3(1024), 0, a.stream, p);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(plan_place_kernel, dim3(p.chunks ? p.chunks : 1), dim3(kPlanThreads), plan_smem(p.experts), a.stream, p);
}

cudaError_t launch_moe_gather(const MoeMoveArgs& a) {
  GatherParams p;
  p.elems_in = (const uint8_t*)a.src; p.scales_in = a.scales_in; p.row_of = a.row_of; p.src_of = a.src_of;
  p.elems_out = (uint8_t*)a.dst; p.scales_out = a.scales_out;
  p.tokens = (uint32_t)a.tokens; p.topk = (uint32_t)a.topk; p.kblocks = (uint32_t)(a.dim / 32);
  p.row_bytes = (uint32_t)(a.dim * a.bits / 8); p.layout = (uint32_t)a.layout;
  p.token_blocks = (p.tokens + kMoveWarps - 1) / kMoveWarps;
  p.scale_blocks = a.layout == MX_SCALES_SWIZZLED ? (uint32_t)((a.rows + 127) / 128) : 0u;
  p.by_topk = make_fastdiv((uint32_t)a.topk);
  p.zero = zero_rows(a, p.row_bytes);
  const dim3 grid(p.scale_blocks + p.token_blocks + zero_blocks(p.zero)), block(32 * kMoveWarps);
  // rows of 6-bit codes are multiples of 24 bytes: 8-byte vectors unless dim is a multiple of 64
  return p.row_bytes % 16 == 0 ? launch_pdl(gather_kernel<uint4>, grid, block, 0, a.stream, p)
                               : launch_pdl(gather_kernel<uint2>, grid, block, 0, a.stream, p);
}

static CombineParams combine_params(const MoeMoveArgs& a) {
  CombineParams p;
  p.y = a.y; p.dout = a.src; p.weights = a.weights; p.row_of = a.row_of; p.out = a.dst; p.dy = a.dst;
  p.dweights = a.dweights; p.tokens = (uint32_t)a.tokens; p.topk = (uint32_t)a.topk; p.dim = (uint32_t)a.dim;
  p.rows = (uint32_t)a.rows; p.token_blocks = p.tokens;
  p.zero = {};
  return p;
}

cudaError_t launch_moe_combine(const MoeMoveArgs& a) {
  const CombineParams p = combine_params(a);
  // Two steps of columns per CTA, so that the last round of CTAs is a small part of all (4817 tokens x 7520, top-4: 66 us,
  // 77 with a CTA per token; one step: 66, but 8192 x 4096, top-2, 37 instead of 33).  One step where that leaves an SM
  // less than 16 of them (239 x 6144, top-6: 4.9 us, 6.8; 64 x 4096, top-4: 3.5, 7.2 with a CTA per token).
  const uint32_t units = a.dim % 8 == 0 ? p.dim / 8 : p.dim, two = (units + 255) / 256;
  const bool enough = (uint64_t)p.tokens * two >= 16u * (uint64_t)a.sm_count;
  const uint32_t parts = enough ? two : (units + 127) / 128;
  const dim3 grid(p.tokens, parts < 65535u ? parts : 65535u), block(128);
  if (a.dtype == MX_BF16)
    return a.dim % 8 == 0 ? launch_pdl(combine_kernel<MX_BF16, true>, grid, block, 0, a.stream, p)
                          : launch_pdl(combine_kernel<MX_BF16, false>, grid, block, 0, a.stream, p);
  return a.dim % 8 == 0 ? launch_pdl(combine_kernel<MX_F32, true>, grid, block, 0, a.stream, p)
                        : launch_pdl(combine_kernel<MX_F32, false>, grid, block, 0, a.stream, p);
}

cudaError_t launch_moe_combine_backward(const MoeMoveArgs& a) {
  CombineParams p = combine_params(a);
  p.zero = zero_rows(a, a.dim * (a.dtype == MX_BF16 ? 2 : 4));
  return a.dtype == MX_BF16 ? launch_backward_dtype<MX_BF16>(a, p) : launch_backward_dtype<MX_F32>(a, p);
}

}  // namespace mx
