// Attention of the newest tokens over a paged cache of MX rows (see mx_kv_attention in mx.h).
//
// Mathematics.  For the query rows r of one sequence that share a key-value head, with s in units of log2 e,
//   s[j, r] = sum_b KX[j, b] * c[r, b] * (sum_{d in block b} KP[j, d] * q'[r, d])        scale * q = c[r, b] * q'
//   out[r, d] = sum_j 2^{s[j, r]} VX[j, b(d)] VP[j, d] / sum_j 2^{s[j, r]}
// Both inner sums are tensor-core products of FP16 operands with FP32 accumulators: codes of every format are exact in
// FP16 (INT8 as the integer), queries are scaled into its range by a power of two for each row and block, so that a block whose queries are
// small and whose keys are large counts like any other.  Its factor c (from shared memory, two rows in one multiplication) comes before the key's
// block scale: the products stay in FP32's range where the score does.  (One power for a row, applied after the sum, lost such blocks
// and overflowed; the factors cost 64 sequences to 8192 1 %.)  A value's scale depends on the token, the axis that its product sums over, so it joins the
// softmax weight: w[j, r, b] = 2^{s - m[r]} VX[j, b] F[r, b], with the reference m[r] of a row's scores and a power of two F[r, b]
// that holds the row's largest w of the block so far in FP16's range.  A row's m, and a row and block's F, move only when a tile breaks their own
// bound (looked at after a vote of the warp), and what has been summed moves with them: no row depends on what else its tile of rows holds.
// (F's room goes up to FP16's largest number: with a bound of 2^15 rows of 256 elements took 227 us for 217, 4-bit ones 86 for 82.)
// Rounded to FP16: w, half a step 2^-11 of a weight (BF16 results, whose own rounding is 2^-8), or two FP16 terms, 2^-22 (FP32
// results; the queries too).  BF16 queries are exact down to 2^-31 of their block's largest element, and off by 2^-39 of that below; FP32 ones
// by 2^-22 of themselves or 2^-50 of that.  Scores, maxima, sums and accumulators are FP32.
//
// Layout.  A warp takes kTokens tokens at a time: S^T = K Q^T has the tokens on the M side of the MMA and the query rows
// on its N side, 8 of them (a group of 4 query heads wastes half of 8, not three quarters of 16), then
// O^T = V^T W^T with the row's elements on the M side.  W^T comes out of S^T's accumulators by 8 x 8 transposes
// in registers.  The order of the elements within a block and of the tokens within a tile is free in these sums, and chosen
// such that a lane's codes are consecutive bytes: no shuffling of codes but the pairing of neighbouring tokens' values.
// (The tensor core's block-scaled instructions do not fit the values, whose scales change along the axis that is summed over.  They would fit the
// scores, with queries in several terms of 8 bits; that is not tried.  The plain FP8 form, mma.sync of the codes as they are by queries in three E5M2
// terms, runs at a fraction of the FP16 one's rate here: 110 -> 162 us.)
// The warps of a block have their own tiles and their own asynchronous copies, kStages tiles deep, and meet only at the
// end of a sequence.
//
// Split.  The tiles of all sequences, heads and groups of rows, one after the other, are dealt out in equal runs to
// two or three blocks per SM, whatever the lengths.  A block that holds the whole of a sequence's tiles for a head writes the result,
// otherwise it leaves a part (its weighted mean and the log of its weight) and a second kernel joins the parts, in the
// order of the tiles: results do not depend on timing.  Where the table holds few tokens a block takes one sequence and head as a whole, and
// nothing is joined (one sequence of 333 tokens: 10.6 -> 7.2 us).
//
// What bounds it.  Large batches the cache's bytes: 64 sequences of up to 8192 tokens, 8 heads of 128 with 4 queries each, E4M3, 111 us (5.6 of
// the 6.55 TB/s that a copy reaches; 121 us where every call has inputs of its own; further sequences add theirs at 6.4), one of 131072 tokens 54 to 56.
// What is left there: 2 us until the first tile, the flush of a block's last sequence, 4 us of the join, and blocks that finish 10 % apart.  Below 30 us
// these fixed parts count for more than the bytes.  Rows of 4 bits and groups of more than 8 queries: instructions (about 700 a tile of 32
// tokens, of which the conversion of the codes 160 and the weights 170, issued at 60 % of the rate): 4-bit rows reach 2.9 TB/s, 16 queries
// a head 2.9.
#pragma once

#include <cuda_fp16.h>

#include "mx_device.cuh"
#include "mx_kv_attention_args.h"
#include "mx_rows.cuh"

namespace mx {
namespace attn {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;  // the reference before any score
constexpr float kRoom = 2.0f;                       // a moved m leaves the new maximum up to a factor 2^3 below it
constexpr float kTop = 65504.0f;                    // weights stay at or below FP16's largest number,
constexpr float kPast = 65520.0f;                   // .. to which it rounds what is below this
constexpr int kAim = 12;                            // log2 of the largest weight after F has moved
constexpr float kMost = 8.507059173023462e37f;      // 2^126, F's largest value

constexpr uint32_t kOneByLower = 0x3A000000u;       // 2^-11
constexpr float kLower = 2048.0f;                   // of a query's second FP16 term, which would else be among FP16's smallest numbers

// Shape of a kernel instance.
constexpr int kSharedOfSm = 228 * 1024;
constexpr int kJoinPitch = 36;  // words of a block of 32 elements in the buffer that joins the warps: rows 2 t in different banks
template <int FMT, int DIM, bool WIDE>
struct Cfg {
  static constexpr int kResident = blocks_per_sm(DIM, WIDE);
  static constexpr int kBits = FmtTraits<FMT>::bits;
  static constexpr bool kOdd = FMT == MX_E4M3 || FMT == MX_E5M2;  // formats with codes of NaN or Inf
  static constexpr int kBlocks = DIM / 32;
  static constexpr int kRow = DIM * kBits / 8;             // bytes of a row's codes
  static constexpr int kGroup = 4 * kBits;                 // bytes of a block's codes
  // rows in shared memory: whole powers of two, so that the 16-byte units can be permuted within lines of 128 bytes
  static constexpr int kPitch = kRow <= 32 ? 32 : kRow <= 64 ? 64 : kRow <= 128 ? 128 : 256;
  static constexpr int kTokens = 1 << tile_log2(DIM, kBits);
  static constexpr int kTiles = kTokens / 16;              // MMA tiles of 16 tokens
  static constexpr int kMine = kTokens <= 32 ? 1 : kTokens / 32;  // tokens whose place in the cache a lane looks up
  static constexpr int kScale = (kBlocks + 3) / 4 * 4;     // bytes of a row's scales
  static constexpr int kUnits = kRow / 16;                 // 16-byte units of a row
  static constexpr int kCopies = kTokens * kUnits / 32;    // of these a lane copies
  static constexpr int kCodes = kTokens * kPitch;
  static constexpr int kStage = 2 * kCodes + 2 * kTokens * kScale + 128;  // codes, scales, the mask of seen tokens
  static constexpr int kNotes = kOdd ? 8 * DIM / 16 * 4 : 0;  // odd elements of values, two bits a row and element
  static constexpr int kJoin = kWarps * 8 * kJoinPitch * 4 + 2 * kWarps * 16 * 4 + kNotes;
  static constexpr int kFit = (kSharedOfSm / kResident - 1024 - kJoin) / (kWarps * kStage);
  static constexpr int kStages = kFit < 4 ? kFit : 4;
  static constexpr int kShared = kWarps * kStages * kStage + kJoin;
  static_assert(kStages >= 2 && kTokens * kUnits % 32 == 0, "tiles in flight");
  // the integer n of an INT8 code stands for n / 64
  static constexpr float kUnit = FMT == MX_INT8 ? 0.015625f : 1.0f;
};

// 2^n for -149 <= n <= 127, 0 below.
__device__ __forceinline__ float pow2(int n) {
  return __uint_as_float(n >= -126 ? (uint32_t)(127 + n) << 23 : n >= -149 ? 1u << (149 + n) : 0u);
}
// The power of two that a block with the largest magnitude `bits` (not 0) is divided by, which puts that in [2^14, 2^15): -127 .. 113 (Inf and NaN: 114).
// (Below 2^-113 it stays smaller: FP32's smallest numbers are whole multiples of FP16's then.)
__device__ __forceinline__ int block_exp(uint32_t bits) { return max((int)(bits >> 23), 14) - 141; }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mul2(float& x, float& y, const uint2& by) {  // in one instruction
  asm("{ .reg .b64 a, b; mov.b64 a, {%0, %1}; mov.b64 b, {%2, %3}; mul.rn.f32x2 a, a, b; mov.b64 {%0, %1}, a; }"
      : "+f"(x), "+f"(y) : "r"(by.x), "r"(by.y));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float2 unpack_half(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }
__device__ __forceinline__ uint32_t max_half2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Transpose of an 8 x 8 matrix of 16-bit elements held as two of a row per lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two scale bytes of a word as FP32 (0: 2^-127, 255: NaN).
__device__ __forceinline__ void scales2(uint32_t word, bool upper, float& a, float& b) {
  uint32_t d;
  if (!upper) asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.bf16x2.ue8m0x2 %0, lo; }" : "=r"(d) : "r"(word));
  else asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.bf16x2.ue8m0x2 %0, hi; }" : "=r"(d) : "r"(word));
  a = __uint_as_float(d << 16);
  b = __uint_as_float(d & 0xFFFF0000u);
}

// The scales of a token (as many as its row has blocks).
template <class C>
__device__ __forceinline__ void load_scales(uint32_t at, float (&s)[C::kScale]) {
#pragma unroll
  for (int c = 0; c < C::kScale; c += 4) {
    uint32_t w;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at + c));
    scales2(w, false, s[c], s[c + 1]);
    if (c + 2 < C::kBlocks) scales2(w, true, s[c + 2], s[c + 3]);
  }
}

// Codes as FP16 pairs.  `w` holds four 8-bit codes (4-bit: all eight of the lane's): pair 0 are codes 0, 1.
template <int FMT>
__device__ __forceinline__ uint32_t half_pair(uint32_t w, int pair) {
  uint32_t h;
  if constexpr (FMT == MX_E4M3) {
    if (pair == 0) asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(h) : "r"(w));
    else asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, hi; }" : "=r"(h) : "r"(w));
  } else if constexpr (FMT == MX_E5M2) {
    h = __byte_perm(w, 0, pair ? 0x3424 : 0x1404);  // E5M2 is FP16's upper byte
  } else if constexpr (FMT == MX_E2M1) {
    // (unpacked from the whole word: taken from a half of it, byte 2 came out as byte 0)
#define MX_E2M1_PAIR(byte) asm("{ .reg .b8 b0, b1, b2, b3; mov.b32 {b0, b1, b2, b3}, %1; cvt.rn.f16x2.e2m1x2 %0, " byte "; }" : "=r"(h) : "r"(w))
    if (pair == 0) MX_E2M1_PAIR("b0");
    else if (pair == 1) MX_E2M1_PAIR("b1");
    else if (pair == 2) MX_E2M1_PAIR("b2");
    else MX_E2M1_PAIR("b3");
#undef MX_E2M1_PAIR
  } else {  // 0x6400 | u = 1024 + u; u = n + 128
    const uint32_t u = __byte_perm(w ^ 0x80808080u, 0x64646464u, pair ? 0x4342 : 0x4140);
    const uint32_t bias = 0x64806480u;  // 1152
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h) : "r"(u), "r"(bias));
  }
  return h;
}

// The upper bit of every byte of four FP8 codes that is NaN or Inf: E4M3 0x7F, E5M2 0x7C .. 0x7F, of either sign.
template <int FMT>
__device__ __forceinline__ uint32_t odd_codes(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + (FMT == MX_E4M3 ? 0x01010101u : 0x04040404u)) & 0x80808080u;
}

// Byte offset of a row (0 .. kTokens - 1) in a tile's codes, its 16-byte units permuted such that the four or eight rows that a
// warp reads at a time lie in different banks; byte x of the row is at offset ^ x (+ 128 for the second line of a row of 256).
template <class C>
__device__ __forceinline__ uint32_t row_at(uint32_t r) {
  if (C::kPitch >= 128) return r * C::kPitch + (C::kBits == 8 ? ((r ^ (r >> 2)) & 3) << 5 : (r & 7) << 4);
  if (C::kPitch == 64) return (r >> 1) * 128 + (((r & 1) << 6) ^ (C::kBits == 8 ? ((r >> 1) & 3) << 5 : ((r >> 1) & 3) << 4));
  return (r >> 2) * 128 + (((r & 3) << 5) ^ (((r >> 2) & 1) << 4));
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_small(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(there ? N : 0) : "memory");
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds2(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}

// NaN and Inf codes among a tile's values that some rows see and others do not, those of its tokens 0 .. head - 1 and tail .. end - 1, become 0
// in the tile, and are noted for each row and element that sees them: two bits in odd[row * DIM / 16 + element / 16], 1 for Inf, 2 for -Inf,
// 3 for NaN (or both infinities).  Codes of tokens that are not there are 0.  (Where the two ranges meet, what is done twice does no harm.)
template <int FMT, int DIM, bool WIDE>
__device__ __forceinline__ void take_out_odd(const Args& a, uint32_t codes, uint32_t* odd, int head, int tail, int end, int j0, uint32_t group0, int length,
                                             uint32_t lane) {
  using C = Cfg<FMT, DIM, WIDE>;
#pragma unroll 1
  for (int n = (int)lane; n < (head + end - tail) * C::kUnits; n += 32) {
    const int m = n / C::kUnits;
    const uint32_t k = (uint32_t)(m < head ? m : tail + m - head), u = (uint32_t)n % C::kUnits;
    const uint32_t at = codes + (row_at<C>(k) ^ ((u & 7) << 4)) + (u >> 3) * 128;
    const uint4 v = lds16(at);
    if ((odd_codes<FMT>(v.x) | odd_codes<FMT>(v.y) | odd_codes<FMT>(v.z) | odd_codes<FMT>(v.w)) == 0) continue;
#pragma unroll 1
    for (uint32_t w = 0; w < 4; ++w) {
      const uint32_t c = lds4(at + 4 * w);
#pragma unroll 1
      for (uint32_t mask = odd_codes<FMT>(c); mask; mask &= mask - 1) {
        const uint32_t e = (__ffs(mask) - 1) / 8, code = c >> 8 * e & 0xFFu;
        const uint32_t bits = FMT == MX_E5M2 && (code & 0x7Fu) == 0x7Cu ? (code & 0x80u ? 2 : 1) : 3;
#pragma unroll 1
        for (uint32_t r = 0; r < 8 && group0 + r < a.rows; ++r) {
          const int hi = length - (int)(a.new_tokens - 1 - fastdiv(group0 + r, a.by_group)), j = j0 + (int)k;
          if (j < hi && (a.window == 0 || j >= hi - (int)a.window)) atomicOr(odd + r * (DIM / 16) + u, bits << 2 * (4 * w + e));
        }
      }
      asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + 4 * w), "r"(c & ~((odd_codes<FMT>(c) >> 7) * 0xFFu)) : "memory");
    }
  }
}

// The instance for rows of DIM elements in format FMT; WIDE: FP32 queries and results; NOTES: several new tokens, which see different tokens, of a
// format with NaN and Inf codes (an instance of its own: what it does beside the rest costs 1 to 3 % also where a condition keeps it from running).
template <int FMT, int DIM, bool WIDE, bool NOTES>
__global__ void __launch_bounds__(kWarps * 32, blocks_per_sm(DIM, WIDE)) kv_attention_kernel(const Args a) {
  using C = Cfg<FMT, DIM, WIDE>;
  constexpr int B = C::kBlocks, TL = C::kTiles, W = WIDE ? 2 : 1;
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem) + warp * (C::kStages * C::kStage);
  float* join = reinterpret_cast<float*>(smem + kWarps * C::kStages * C::kStage);  // [kWarps][8][kJoinPitch]
  float2* join_ml = reinterpret_cast<float2*>(join + kWarps * 8 * kJoinPitch);     // [kWarps][16]
  uint32_t* odd = reinterpret_cast<uint32_t*>(join_ml + kWarps * 16);              // [8][DIM / 16] (see take_out_odd)
  if (NOTES) {
    for (uint32_t i = threadIdx.x; i < DIM / 2; i += kWarps * 32) odd[i] = 0;
    __syncthreads();
  }

  // The lengths come from the kernels before this one.  The join may be scheduled only after this point, so that it, too,
  // finds them written.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // Powers of two of this warp's queries by block and row, in its part of the buffer that joins the warps (in use only between two
  // sequences): [B][8], of which a lane reads rows 2 t, 2 t + 1.
  float* q_by = join + warp * 8 * kJoinPitch;
  const int scale_exp = a.scale_exp + (FMT == MX_INT8 ? -6 : 0);  // (the integer n of an INT8 code stands for n / 64)
  const uint32_t q_by_at = (uint32_t)__cvta_generic_to_shared(q_by) + t * 8;

  Share share;
  Segment s;
  uint32_t first = 0, last;  // this block's tiles are first .. last - 1
  if (a.whole) {
    s.b = blockIdx.x / (a.heads * a.row_tiles);
    s.hr = blockIdx.x - s.b * (a.heads * a.row_tiles);
    s.start = 0;
    a.fill(s, a.length(s.b));
    last = s.end;
    if (last == 0) {  // no token to see
      for (uint32_t i = threadIdx.x; i < 8 * (DIM / 8); i += kWarps * 32) {
        const uint32_t r = s.row_tile(a) * 8 + i / (DIM / 8);
        if (r >= a.rows) break;
        const size_t row = a.out_row(s, r);
        const float zero[8] = {};
        store8<WIDE ? MX_F32 : MX_BF16>(a.out, row * DIM + i % (DIM / 8) * 8, zero);
        if (a.lse && i % (DIM / 8) == 0) a.lse[row] = -INFINITY;
      }
      return;
    }
  } else {
    share = a.share(lane);
    first = blockIdx.x * share.per;
    last = min(first + share.per, share.total);
    if (first >= share.total) {
      if (threadIdx.x == 0 && !a.by_segment) a.unfinished[blockIdx.x] = {0, 0, 0, 0};
      return;
    }
    s = a.find(share, first, lane);
  }

  // ---- the copies' side: which tokens the next tile to copy holds -------------------------------------------
  Segment ls = s;
  uint32_t unit = first + warp, lu = unit;  // the tiles to work on and to copy next
  uint32_t page[C::kMine], off[C::kMine];   // of this lane's tokens in the tile to copy: tokens lane, 32 + lane
  bool there[C::kMine];
  auto look_up = [&] {
    if (lu >= last) return;
#pragma unroll 1
    while (lu >= ls.end) a.next(ls);
#pragma unroll
    for (int i = 0; i < C::kMine; ++i) {
      const uint32_t j = (ls.first_tile + (lu - ls.start)) * C::kTokens + 32 * i + (lane % C::kTokens);
      there[i] = j < ls.length && j >= ls.begin;
      const uint32_t p = fastdiv(j, a.by_page);
      off[i] = j - p * a.page_size;
      page[i] = 0;
      if (there[i]) page[i] = (uint32_t)a.table[(size_t)ls.b * a.max_pages + p];
    }
  };
  uint32_t fill = 0;  // the stage to fill next
  auto copy_tile = [&] {
    if (lu < last) {
      const uint32_t stage = base + fill * C::kStage, scales = stage + 2 * C::kCodes;
      uint32_t row[C::kMine], seen[C::kMine];
      bool all = true;
#pragma unroll
      for (int i = 0; i < C::kMine; ++i) {
        const bool ok = there[i] && page[i] < a.pages;  // (a negative entry is a large one)
        row[i] = ok ? (page[i] * a.heads + ls.head(a)) * a.page_size + off[i] : 0;
        seen[i] = __ballot_sync(0xFFFFFFFFu, ok);
        all = all && seen[i] == 0xFFFFFFFFu;
        if (C::kTokens >= 32) {
          copy_small<C::kScale>(scales + (32 * i + lane) * C::kScale, a.k_scales + (size_t)row[i] * C::kScale, ok);
          copy_small<C::kScale>(scales + (C::kTokens + 32 * i + lane) * C::kScale, a.v_scales + (size_t)row[i] * C::kScale, ok);
        } else {  // keys' by the lower half of the warp, values' by the upper
          copy_small<C::kScale>(scales + lane * C::kScale, (lane < 16 ? a.k_scales : a.v_scales) + (size_t)row[i] * C::kScale, ok);
        }
        if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(scales + 2 * C::kTokens * C::kScale + 4 * i), "r"(seen[i]) : "memory");
      }
      // 16-byte units lane, 32 + lane, .. of the tile, and where they go: the lane's part of that, and (where a row is a power of two of
      // them) a constant one, which meet in an exclusive or within a line
      constexpr bool kEven = (C::kUnits & (C::kUnits - 1)) == 0;
      const uint32_t u0 = lane % C::kUnits, to0 = stage + (row_at<C>(lane / C::kUnits) ^ ((u0 & 7) << 4)) + (u0 >> 3) * 128;
      auto place = [&](int i) {
        if (kEven) {
          const uint32_t c = row_at<C>(32 * i / C::kUnits);
          return (to0 ^ (c & 127)) + (c & ~127u);
        }
        const uint32_t r = (lane + 32 * i) / C::kUnits, u = (lane + 32 * i) % C::kUnits;
        return stage + (row_at<C>(r) ^ ((u & 7) << 4)) + (u >> 3) * 128;
      };
      // (every lane takes part in the exchange and the vote: no condition stands before them)
      const uint32_t row0 = __shfl_sync(0xFFFFFFFFu, row[0], 0);
      bool run = all;  // tokens one after the other in memory, as within a page
#pragma unroll
      for (int i = 0; i < C::kMine; ++i) run = run & (row[i] == row0 + 32 * i + lane % C::kTokens);
      run = __all_sync(0xFFFFFFFFu, run);
      if (run) {
        const size_t at = (size_t)row0 * C::kRow + lane * 16;
        const uint8_t *k = a.k_elems + at, *v = a.v_elems + at;
#pragma unroll
        for (int i = 0; i < C::kCopies; ++i) {
          const uint32_t to = place(i);
          copy16(to, k + i * 512);
          copy16(to + C::kCodes, v + i * 512);
        }
      } else {
#pragma unroll
        for (int i = 0; i < C::kCopies; ++i) {
          const uint32_t n = lane + 32 * i, r = n / C::kUnits, u = n % C::kUnits;
          // (which of a lane's two tokens: known at compile time where the units of 32 tokens are whole rounds of the warp)
          const int mine = C::kMine == 1 ? 0 : 32 * i / (32 * C::kUnits);
          const size_t at = (size_t)__shfl_sync(0xFFFFFFFFu, row[mine], r % 32) * C::kRow + u * 16;
          const bool has = seen[mine] >> (r % 32) & 1;
          const uint32_t to = place(i);
          copy16(to, a.k_elems + at, has);
          copy16(to + C::kCodes, a.v_elems + at, has);
        }
      }
      lu += kWarps;
      fill = fill + 1 == C::kStages ? 0 : fill + 1;
      look_up();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  look_up();
  uint32_t ahead = C::kStages - 1;  // copies to start before the first tile

  // lane offsets of the codes: keys of tokens g, g + 8; values of tokens 2 t, 2 t + 1 (and 8 further on)
  const uint32_t k_at[2] = {row_at<C>(g) + t * (C::kGroup / 4), row_at<C>(g + 8) + t * (C::kGroup / 4)};
  uint32_t v_at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v_at[i] = row_at<C>(2 * t + (i & 1) + (i & 2) * 4) + g * (C::kGroup / 8);

  uint32_t use = 0;
  for (;;) {
    // ---- one sequence and head: the queries ------------------------------------------------------------------
    const uint32_t seg_end = min(s.end, last);
    const uint32_t group0 = s.row_tile(a) * 8;  // first query row of this tile of rows
    uint32_t q[W][B][2][2];
    int lo[2], hi[2];  // tokens that the lane's rows 2 t, 2 t + 1 see
    Raw8<WIDE ? MX_F32 : MX_BF16> raw[B];
    const uint32_t q_row = group0 + g, q_token = fastdiv(q_row, a.by_group), q_head = s.head(a) * a.group + (q_row - q_token * a.group);
    const size_t q_at = ((size_t)s.b * a.new_tokens + q_token) * a.q_stride + (size_t)q_head * DIM + t * 8;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      raw[b] = {};
      if (q_row < a.rows) raw[b] = load_raw8<WIDE ? MX_F32 : MX_BF16>(a.q, q_at + b * 32);
    }
#pragma unroll 1
    for (; ahead > 0; --ahead) copy_tile();  // (the first copies are under way while the queries are prepared)
    float x[B][8];
    uint32_t ab[B];     // largest magnitude of a block, its bits
    int most = -1024;   // largest power of two in a factor of the row
#pragma unroll
    for (int b = 0; b < B; ++b) {
      widen(raw[b], x[b]);
      float amax = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = absmax_nan(amax, x[b][j]);
      amax = absmax_nan(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
      amax = absmax_nan(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
      ab[b] = __float_as_uint(amax) & 0x7FFFFFFFu;
      if (ab[b]) most = max(most, block_exp(ab[b]) + scale_exp);
    }
    // Products by a factor of 2^60 or less, and not much less, leave the range of FP32 only where the score does.
    const int rest = most > 60 ? min(most - 60, 127) : most < -60 && most > -1024 ? max(most + 60, -126) : 0;
    // q' = q * 2^-e with a block's largest element in [2^14, 2^15): FP16 then holds what is 2^-28 of it to full precision.  Inf or NaN make
    // the row NaN.
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int e = ab[b] ? block_exp(ab[b]) : 0;
      const float into = ab[b] >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float u = x[b][4 * k + 2 * j] * into, v = x[b][4 * k + 2 * j + 1] * into;
          q[0][b][k][j] = pack_half(u, v);
          if (WIDE) {
            const float2 h = unpack_half(q[0][b][k][j]);
            q[W - 1][b][k][j] = pack_half((u - h.x) * kLower, (v - h.y) * kLower);
          }
        }
    }
#pragma unroll
    for (int b0 = 0; b0 < B; b0 += 4) {  // the factors of four blocks, one of them a lane
      uint32_t bits = ab[b0];
#pragma unroll
      for (int b = b0 + 1; b < b0 + 4 && b < B; ++b) bits = t == b - b0 ? ab[b] : bits;
      const float by = a.scale_mant * pow2(min((bits ? block_exp(bits) : 0) + scale_exp - rest, 127));
      if (b0 + t < B) q_by[(b0 + t) * 8 + g] = by;
    }
    if (t == 0) q_by[B * 8 + g] = pow2(rest);
    const bool extreme = __any_sync(0xFFFFFFFFu, rest != 0);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t row = group0 + 2 * t + j;
      const int i = row < a.rows ? (int)fastdiv(row, a.by_group) : (int)a.new_tokens - 1;
      hi[j] = (int)s.length - ((int)a.new_tokens - 1 - i);
      lo[j] = a.window ? max(hi[j] - (int)a.window, 0) : 0;
    }
    // tiles between these are seen by all rows
    const int all_lo = a.window ? max((int)s.length - (int)a.window, 0) : 0, all_hi = (int)s.length - ((int)a.new_tokens - 1);

    float m[2], l[2], F[B][2], acc[B][2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      m[j] = kLowest;
      l[j] = 0.0f;
#pragma unroll
      for (int b = 0; b < B; ++b) F[b][j] = kMost;
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[b][h][i] = 0.0f;

    bool fresh = true;  // m and F have not been set by a tile of this sequence

    // ---- its tiles ----------------------------------------------------------------------------------------
#pragma unroll 1
    for (; unit < seg_end; unit += kWarps) {
      copy_tile();
      asm volatile("cp.async.wait_group %0;" ::"n"(C::kStages - 1) : "memory");
      __syncwarp();
      const uint32_t stage = base + use * C::kStage, scales = stage + 2 * C::kCodes;
      const uint32_t k_of[2] = {stage + k_at[0], stage + k_at[1]};  // (stages begin at whole lines)
      const uint32_t v_of[4] = {stage + v_at[0], stage + v_at[1], stage + v_at[2], stage + v_at[3]};
      use = use + 1 == C::kStages ? 0 : use + 1;
      uint32_t seen[C::kMine];
      const int j0 = (int)(s.first_tile + (unit - s.start)) * C::kTokens;
      bool edge = j0 < all_lo || j0 + C::kTokens > all_hi;
#pragma unroll
      for (int i = 0; i < C::kMine; ++i) {
        seen[i] = lds4(scales + 2 * C::kTokens * C::kScale + 4 * i);
        edge = edge || seen[i] != 0xFFFFFFFFu;
      }

      // scores of tokens 16 x + g, 16 x + g + 8 for rows 2 t, 2 t + 1
      float p[TL][4];
#pragma unroll
      for (int x = 0; x < TL; ++x) {
        float ks[2][C::kScale];
#pragma unroll
        for (int h = 0; h < 2; ++h) load_scales<C>(scales + (16 * x + 8 * h + g) * C::kScale, ks[h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[x][i] = 0.0f;
#pragma unroll
        for (int b = 0; b < B; ++b) {
          uint32_t ka[2][4];  // two steps of 16 elements
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t at = (k_of[h] ^ ((b * C::kGroup) & 127)) + x * 16 * C::kPitch + (b * C::kGroup) / 128 * 128;
            if (C::kBits == 8) {
              const uint2 c = lds8(at);
              ka[0][h] = half_pair<FMT>(c.x, 0);
              ka[0][2 + h] = half_pair<FMT>(c.x, 1);
              ka[1][h] = half_pair<FMT>(c.y, 0);
              ka[1][2 + h] = half_pair<FMT>(c.y, 1);
            } else {
              const uint32_t c = lds4(at);
              ka[0][h] = half_pair<FMT>(c, 0);
              ka[0][2 + h] = half_pair<FMT>(c, 1);
              ka[1][h] = half_pair<FMT>(c, 2);
              ka[1][2 + h] = half_pair<FMT>(c, 3);
            }
          }
          float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int w = W - 1; w >= 0; --w) {
#pragma unroll
            for (int k = 0; k < 2; ++k) mma(d, ka[k], q[w][b][k][0], q[w][b][k][1]);
            if (w > 0) {
              const uint2 lower = make_uint2(kOneByLower, kOneByLower);
              mul2(d[0], d[1], lower);
              mul2(d[2], d[3], lower);
            }
          }
          const uint2 by = lds8(q_by_at + b * 32);
          mul2(d[0], d[1], by);
          mul2(d[2], d[3], by);
#pragma unroll
          for (int i = 0; i < 4; ++i) p[x][i] = fmaf(d[i], ks[i >> 1][b], p[x][i]);
        }
      }
      if (extreme) {
        const uint2 by = lds8(q_by_at + B * 32);
#pragma unroll
        for (int x = 0; x < TL; ++x) {
          mul2(p[x][0], p[x][1], by);
          mul2(p[x][2], p[x][3], by);
        }
      }
      uint32_t hidden = 0;  // bit: this score is of a token that the row does not see
      if (edge) {
        // A weight of zero does not keep a NaN or Inf code of a value out of the product.  Those of tokens that some rows see and others do
        // not, the oldest and the newest ones, are taken out and noted.  (What is hidden from all is not copied.)
        if (NOTES) {
          const int end = min((int)s.length - j0, C::kTokens);
          take_out_odd<FMT, DIM, WIDE>(a, stage + C::kCodes, odd, min(max(all_lo - j0, 0), end), min(max(all_hi - j0, 0), end), end, j0, group0, (int)s.length, lane);
          __syncwarp();
        }
#pragma unroll
        for (int x = 0; x < TL; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = 16 * x + 8 * (i >> 1) + (int)g, j = j0 + k;
            if (!(seen[x / 2 % C::kMine] >> (k % 32) & 1) || j < lo[i & 1] || j >= hi[i & 1]) hidden |= 1u << (x * 4 + i);
          }
      }

      // Weights without the values' scales: m moves when a score passes it, once at most.  (The scores are rounded numbers here, the same ones as
      // where the largest is found: nothing can be above m in one place and not in the other.)
      float y[TL][4];
      for (bool moved = false, move = fresh;; move = false) {
        if (!move) {
          float most = -1.0f;
#pragma unroll
          for (int x = 0; x < TL; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[x][i] = p[x][i] - m[i & 1];
          if (edge) {
#pragma unroll
            for (int x = 0; x < TL; ++x)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (hidden >> (x * 4 + i) & 1) y[x][i] = -INFINITY;
          }
#pragma unroll
          for (int x = 0; x < TL; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, y[x][i]);
          if (moved || !__any_sync(0xFFFFFFFFu, most > 0.0f)) break;
        }
        moved = true;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float top = -INFINITY;
#pragma unroll
          for (int x = 0; x < TL; ++x)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (!(hidden >> (x * 4 + 2 * h + j) & 1)) top = fmaxf(top, p[x][2 * h + j]);
#pragma unroll
          for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
          const float next = top > m[j] ? ceilf(top) + kRoom : m[j], up = top > m[j] ? next - m[j] : 0.0f;
          m[j] = next;
          l[j] *= ex2(-up);
          // F takes the move, as far as it can, so that what is summed keeps its size: a large value that a larger score has made
          // small does not hold F down
#pragma unroll
          for (int b = 0; b < B; ++b) {
            const float want = (float)((int)(__float_as_uint(F[b][j]) >> 23) - 127) + up, have = fminf(want, 126.0f), by = ex2(have - want);
            F[b][j] = __uint_as_float((uint32_t)((int)have + 127) << 23);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              acc[b][h][j] *= by;
              acc[b][h][2 + j] *= by;
            }
          }
        }
      }
#pragma unroll
      for (int x = 0; x < TL; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[x][i] = ex2(y[x][i]);
          l[i & 1] += p[x][i];
        }

      // weights with the values' scales: F moves when one passes kTop, once at most
      uint32_t w[W][B][TL][2];
      for (bool moved = false, move = fresh;; move = false) {
        if (!move) {
          uint32_t most = 0;
#pragma unroll
          for (int x = 0; x < TL; ++x) {
            float vs[2][C::kScale];
#pragma unroll
            for (int h = 0; h < 2; ++h) load_scales<C>(scales + (C::kTokens + 16 * x + 8 * h + g) * C::kScale, vs[h]);
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                // p is at most 1 and VX at most 2^127, F follows their product
                const float u = p[x][2 * h] * vs[h][b] * F[b][0], v = p[x][2 * h + 1] * vs[h][b] * F[b][1];
                const uint32_t c = pack_half(u, v);
                w[0][b][x][h] = c;
                most = max_half2(most, c);
                if (WIDE) {
                  const float2 r = unpack_half(c);
                  w[W - 1][b][x][h] = pack_half(u - r.x, v - r.y);
                }
              }
          }
          const float2 top2 = unpack_half(most);
          if (moved || !__any_sync(0xFFFFFFFFu, fmaxf(top2.x, top2.y) > kTop)) break;
        }
        moved = true;
        // F moves down to where the largest is in [2^kAim, 2^(kAim + 1)), for rows and blocks that broke the bound themselves; up only with m
        float top[B][2];
#pragma unroll
        for (int x = 0; x < TL; ++x)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v[C::kScale];
            load_scales<C>(scales + (C::kTokens + 16 * x + 8 * h + g) * C::kScale, v);
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
              for (int j = 0; j < 2; ++j) top[b][j] = fmaxf(x + h == 0 ? 0.0f : top[b][j], p[x][2 * h + j] * v[b]);
          }
#pragma unroll
        for (int d = 4; d < 32; d *= 2)
#pragma unroll
          for (int b = 0; b < B; ++b)
#pragma unroll
            for (int j = 0; j < 2; ++j) top[b][j] = fmaxf(top[b][j], __shfl_xor_sync(0xFFFFFFFFu, top[b][j], d));
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int e = (int)(__float_as_uint(top[b][j]) >> 23) - 127, have = (int)(__float_as_uint(F[b][j]) >> 23) - 127;
            const int next = top[b][j] * F[b][j] >= kPast ? kAim - e : have;
            const float by = ex2((float)(next - have));  // 1 where F stays
            F[b][j] = __uint_as_float((uint32_t)(127 + next) << 23);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              acc[b][h][j] *= by;
              acc[b][h][2 + j] *= by;
            }
          }
      }
      fresh = false;
      if (edge) {  // a token that is not seen weighs nothing, whatever its scale
#pragma unroll
        for (int x = 0; x < TL; ++x)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t two = hidden >> (x * 4 + 2 * h) & 3, keep = (two & 1 ? 0u : 0xFFFFu) | (two & 2 ? 0u : 0xFFFF0000u);
#pragma unroll
            for (int k = 0; k < W; ++k)
#pragma unroll
              for (int b = 0; b < B; ++b) w[k][b][x][h] &= keep;
          }
      }
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int x = 0; x < TL; ++x) {
          uint32_t va[2][4];
          const uint32_t blk = (b * C::kGroup) & 127, at = C::kCodes + x * 16 * C::kPitch + (b * C::kGroup) / 128 * 128;
          if (C::kBits == 8) {
            uint32_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = lds4((v_of[i] ^ blk) + at);
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // elements 0, 1 and 2, 3 of the lane's four
              const uint32_t y0 = __byte_perm(c[0], c[1], h ? 0x7362 : 0x5140), y1 = __byte_perm(c[2], c[3], h ? 0x7362 : 0x5140);
              va[h][0] = half_pair<FMT>(y0, 0);
              va[h][1] = half_pair<FMT>(y0, 1);
              va[h][2] = half_pair<FMT>(y1, 0);
              va[h][3] = half_pair<FMT>(y1, 1);
            }
          } else {
            const uint32_t c0 = lds2((v_of[0] ^ blk) + at) | lds2((v_of[2] ^ blk) + at) << 16;
            const uint32_t c1 = lds2((v_of[1] ^ blk) + at) | lds2((v_of[3] ^ blk) + at) << 16;
            // bytes: elements 0, 2 (and 1, 3) of tokens 2 t, 2 t + 1, then of those 8 further on
            const uint32_t y0 = (c0 & 0x0F0F0F0Fu) | (c1 & 0x0F0F0F0Fu) << 4, y1 = (c0 >> 4 & 0x0F0F0F0Fu) | (c1 & 0xF0F0F0F0u);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              va[h][0] = half_pair<FMT>(y0, h);
              va[h][1] = half_pair<FMT>(y1, h);
              va[h][2] = half_pair<FMT>(y0, 2 + h);
              va[h][3] = half_pair<FMT>(y1, 2 + h);
            }
          }
          uint32_t wb[W][2];
#pragma unroll
          for (int k = 0; k < W; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) wb[k][h] = transpose8(w[k][b][x][h]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (WIDE) {  // the sum over tokens in FP32 additions, which round to nearest
              float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
              mma(d, va[h], wb[W - 1][0], wb[W - 1][1]);
              mma(d, va[h], wb[0][0], wb[0][1]);
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[b][h][i] += d[i];
            } else {
              mma(acc[b][h], va[h], wb[0][0], wb[0][1]);
            }
          }
        }
      __syncwarp();  // the stage may be filled again
    }

    // ---- the block's warps joined: sum of acc 2^(m - M) / F over sum of l 2^(m - M) -------------------------------
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int d = 4; d < 32; d *= 2) l[j] += __shfl_xor_sync(0xFFFFFFFFu, l[j], d);
      if (g == 0) join_ml[warp * 16 + 2 * t + j] = make_float2(m[j], l[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float top = kLowest, sum = 0.0f;
      float2 ml[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        ml[w] = join_ml[w * 16 + 2 * t + j];
        top = fmaxf(top, ml[w].x);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum = fmaf(ml[w].y, ex2(ml[w].x - top), sum);
      const float mine = sum == 0.0f ? 0.0f : ex2(m[j] - top) * C::kUnit * rcp(sum);
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const float by = __uint_as_float((254u << 23) - __float_as_uint(F[b][j]));  // 1 / F, a power of two
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          acc[b][h][j] = acc[b][h][j] * mine * by;
          acc[b][h][2 + j] = acc[b][h][2 + j] * mine * by;
        }
      }
    }
    const bool whole = s.start >= first && s.end <= last;
    // a thread puts out two elements of one row of each block, row tid / 16 of the eight
    const uint32_t out_row = threadIdx.x / 16, out_at = threadIdx.x % 16 * 2;
    const uint32_t r = group0 + out_row;
    const size_t row = a.out_row(s, r);
    const size_t part = (size_t)(blockIdx.x * 2 + (s.start >= first ? 1 : 0)) * 8 + out_row;
    if (out_at == 0 && r < a.rows && (!whole || a.lse)) {
      float top = kLowest, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, join_ml[w * 16 + out_row].x);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum = fmaf(join_ml[w * 16 + out_row].y, ex2(join_ml[w * 16 + out_row].x - top), sum);
      const float lse2 = sum == 0.0f ? -INFINITY : top + lg2(sum);
      if (whole) a.lse[row] = lse2 * kLn2;
      else a.part_lse[part] = lse2;
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *reinterpret_cast<float4*>(join + (warp * 8 + 2 * t + j) * kJoinPitch + 4 * g) =
            make_float4(acc[b][0][j], acc[b][0][2 + j], acc[b][1][j], acc[b][1][2 + j]);
      __syncthreads();
      float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 u = *reinterpret_cast<const float2*>(join + (w * 8 + out_row) * kJoinPitch + out_at);
        v.x += u.x;
        v.y += u.y;
      }
      if (NOTES) {
        const uint32_t bits = odd[out_row * (DIM / 16) + b * 2 + out_at / 16] >> out_at % 16 * 2;
        const float inf = INFINITY;
        if (bits & 1) v.x += inf;
        if (bits & 2) v.x -= inf;
        if (bits & 4) v.y += inf;
        if (bits & 8) v.y -= inf;
      }
      if (r < a.rows) {
        if (!whole) *reinterpret_cast<float2*>(a.parts + part * DIM + b * 32 + out_at) = v;
        else if (WIDE) *reinterpret_cast<float2*>((float*)a.out + row * DIM + b * 32 + out_at) = v;
        else *reinterpret_cast<uint32_t*>((uint16_t*)a.out + row * DIM + b * 32 + out_at) = pack_bf16(v.x, v.y);
      }
      __syncthreads();  // before the buffer is used again
    }
    // the sequence that begins here and goes on is joined from this block's part and those of the blocks behind it
    if (threadIdx.x == 0 && !a.whole && (a.by_segment ? s.start >= first : s.end >= last)) {
      const uint32_t parts = s.start >= first && s.end > last ? (s.end - 1) / share.per - blockIdx.x + 1 : 0;
      a.unfinished[a.by_segment ? s.b * a.heads * a.row_tiles + s.hr : blockIdx.x] = {s.b, s.hr, parts, blockIdx.x};
    }
    if (s.end >= last) break;
    if (NOTES) {  // (all have read them: the barrier above)
      for (uint32_t i = threadIdx.x; i < DIM / 2; i += kWarps * 32) odd[i] = 0;
      __syncthreads();
    }
    a.next(s);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <int FMT, int DIM, bool WIDE>
cudaError_t launch_instance(const Args& a, uint32_t ctas, cudaStream_t stream) {
  using C = Cfg<FMT, DIM, WIDE>;
  auto kernel = kv_attention_kernel<FMT, DIM, WIDE, false>;
  if constexpr (C::kOdd) {
    if (a.new_tokens > 1) kernel = kv_attention_kernel<FMT, DIM, WIDE, true>;
  }
  // (a function attribute per device: set on every call, it costs less than a microsecond)
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kShared);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(ctas), dim3(kWarps * 32), C::kShared, stream, a);
}
template <int FMT>
cudaError_t launch_format(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream) {
  switch (dim) {
    case 64: return wide ? launch_instance<FMT, 64, true>(a, ctas, stream) : launch_instance<FMT, 64, false>(a, ctas, stream);
    case 96: return wide ? launch_instance<FMT, 96, true>(a, ctas, stream) : launch_instance<FMT, 96, false>(a, ctas, stream);
    case 128: return wide ? launch_instance<FMT, 128, true>(a, ctas, stream) : launch_instance<FMT, 128, false>(a, ctas, stream);
    case 192: return wide ? launch_instance<FMT, 192, true>(a, ctas, stream) : launch_instance<FMT, 192, false>(a, ctas, stream);
    default: return wide ? launch_instance<FMT, 256, true>(a, ctas, stream) : launch_instance<FMT, 256, false>(a, ctas, stream);
  }
}

}  // namespace attn
}  // namespace mx
