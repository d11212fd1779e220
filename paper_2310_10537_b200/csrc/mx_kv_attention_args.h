// What the kernels of mx_kv_attention share: their arguments, and how the tiles of all sequences are dealt out.
#pragma once

#include "mx_device.cuh"

namespace mx {
namespace attn {

constexpr int kWarps = 4;         // of a block
constexpr uint32_t kRows = 8;     // query rows of a unit, the N side of an MMA
constexpr uint32_t kCtas = 444;   // blocks at most: three on each of 148 SMs
// Blocks per SM of an instance, by its registers.
__host__ __device__ constexpr int blocks_per_sm(int dim, bool wide) { return dim <= 128 && !wide ? 3 : 2; }
// A block's fewest tiles: one per warp.
constexpr uint32_t kLeast = kWarps;

// Tokens of a tile: 64 of 64 elements, so that what a tile costs whatever its size counts less (their weights for every block still fit the
// registers); 16 for rows above 128 bytes, for the shared memory.
__host__ __device__ constexpr int tile_log2(int dim, int bits) { return dim <= 64 ? 6 : dim * bits <= 1024 ? 5 : 4; }

// The tiles first .. of one sequence b for one key-value head and one tile of query rows: units start .. end - 1 of the
// whole list, which runs over sequences, then heads and tiles of rows, then tiles of tokens.
struct Segment {
  uint32_t b, hr;            // hr: head * row tiles + row tile
  uint32_t start, end;
  uint32_t first_tile;       // tile number (of all the sequence's tokens) of unit `start`
  uint32_t begin, length;    // tokens that some query sees: begin .. length - 1
  template <class A> __device__ uint32_t head(const A& a) const { return fastdiv(hr, a.by_row_tiles); }
  template <class A> __device__ uint32_t row_tile(const A& a) const { return hr - head(a) * a.row_tiles; }
};

// What a warp keeps of all lengths: lane i has the units of sequences i * chunk .. (i + 1) * chunk - 1.
struct Share {
  uint32_t total, per;       // units in all, and of a block
  uint32_t before;           // units before this lane's sequences
  uint32_t mine;
  uint32_t length;           // of this lane's only sequence, where lanes have one
};

// A sequence and head whose tiles go on behind the block that they begin in: that block, and how many parts there are (0: none,
// it is finished).
struct Unfinished {
  uint32_t b, hr, parts, block;
};

struct Args {
  const uint8_t *k_elems, *k_scales, *v_elems, *v_scales;
  const void* q;
  const int32_t *table, *lengths;
  void* out;
  float *lse, *parts, *part_lse;  // parts: [2 * blocks][kRows][dim]
  Unfinished* unfinished;         // of each block, or (by_segment) of each sequence, head and tile of rows that has tiles
  int64_t q_stride;
  uint32_t pages, page_size, heads, batch, new_tokens, q_heads, max_pages, window;
  uint32_t group, rows;           // query heads of a key-value head; query rows of one: new_tokens * group
  uint32_t row_tiles;             // units of kRows query rows
  uint32_t tile_log2, chunk;      // log2 of a tile's tokens; sequences of a lane
  FastDiv by_page, by_group, by_row_tiles, by_grid;
  float scale_mant;               // scale * log2 e = scale_mant * 2^scale_exp
  int scale_exp;
  bool by_segment, whole;         // whole: block i takes the i-th sequence, head and tile of rows as a whole

  __device__ __forceinline__ uint32_t length(uint32_t b) const {
    const int n = lengths[b];
    return n < 0 ? 0 : min((uint32_t)n, max_pages * page_size);
  }
  // Row of out (and lse) of query row r of a segment's key-value head.
  __device__ __forceinline__ size_t out_row(const Segment& s, uint32_t r) const {
    const uint32_t i = fastdiv(r, by_group);
    return ((size_t)s.b * new_tokens + i) * q_heads + s.head(*this) * group + (r - i * group);
  }
  // First token that the earliest query sees.
  __device__ __forceinline__ uint32_t begin(uint32_t length) const {
    const int64_t e = (int64_t)length - (new_tokens - 1) - window;
    return window == 0 || e < 0 ? 0 : (uint32_t)e;
  }
  __device__ __forceinline__ uint32_t tiles(uint32_t length) const {
    return length == 0 ? 0 : ((length - 1) >> tile_log2) + 1 - (begin(length) >> tile_log2);
  }
  __device__ __forceinline__ void fill(Segment& s, uint32_t length) const {
    s.length = length;
    s.begin = begin(s.length);
    s.first_tile = s.begin >> tile_log2;
    s.end = s.start + tiles(s.length);
  }
  // The next segment that has units.  (There is one, unless somebody writes the lengths meanwhile: then one without tokens, without end.)
  __device__ __forceinline__ void next(Segment& s) const {
    const uint32_t n = s.end - s.start;
    s.start = s.end;
    if (s.hr + 1 < heads * row_tiles) {
      ++s.hr;
      s.end = s.start + n;
      return;
    }
    s.hr = 0;
#pragma unroll 1
    do {
      if (s.b + 1 >= batch) {
        s.end = 0xFFFFFFFFu;
        s.length = 0;
        return;
      }
      ++s.b;
      fill(s, length(s.b));
    } while (s.end == s.start);
  }
  __device__ __forceinline__ static uint32_t scan(uint32_t v, uint32_t lane) {  // inclusive sums over the lanes
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, v, d);
      if (lane >= (uint32_t)d) v += u;
    }
    return v;
  }
  __device__ __forceinline__ Share share(uint32_t lane) const {
    Share r;
    uint32_t n = 0;
    r.length = 0;
    if (chunk == 1) {
      if (lane < batch) r.length = length(lane);
      n = tiles(r.length);
    } else {
      const uint32_t e = min((lane + 1) * chunk, batch);
#pragma unroll 1
      for (uint32_t b = lane * chunk; b < e; b += 4) {  // (four lengths in flight)
        uint32_t v[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = b + i < e ? length(b + i) : 0;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) n += tiles(v[i]);
      }
    }
    r.mine = n * heads * row_tiles;
    const uint32_t sum = scan(r.mine, lane);
    r.before = sum - r.mine;
    r.total = __shfl_sync(0xFFFFFFFFu, sum, 31);
    r.per = max(fastdiv(r.total + gridDim.x - 1, by_grid), kLeast);
    return r;
  }
  // The segment of a unit below total.
  __device__ __forceinline__ Segment find(const Share& share, uint32_t unit, uint32_t lane) const {
    const uint32_t who = __ffs(__ballot_sync(0xFFFFFFFFu, unit >= share.before && unit - share.before < share.mine)) - 1;
    uint32_t at = __shfl_sync(0xFFFFFFFFu, share.before, who);
    Segment s;
    s.b = min(who, batch - 1);
    uint32_t tokens = __shfl_sync(0xFFFFFFFFu, share.length, who);
    if (chunk > 1) {
#pragma unroll 1
      for (uint32_t b0 = who * chunk; b0 < batch; b0 += 32) {  // its sequences, 32 at a time
        const uint32_t b = b0 + lane;
        const uint32_t mine = b < min((who + 1) * chunk, batch) ? tiles(length(b)) * heads * row_tiles : 0, sum = scan(mine, lane);
        const uint32_t hit = __ballot_sync(0xFFFFFFFFu, unit - at < sum);
        if (hit) {
          const uint32_t w = __ffs(hit) - 1;
          s.b = b0 + w;
          at += __shfl_sync(0xFFFFFFFFu, sum - mine, w);
          break;
        }
        at += __shfl_sync(0xFFFFFFFFu, sum, 31);
      }
    }
    if (chunk > 1) tokens = length(s.b);
    s.start = 0;
    fill(s, tokens);
    const uint32_t n = max(s.end, 1u);
    s.hr = min((unit - at) / n, heads * row_tiles - 1);
    s.start = at + s.hr * n;
    s.end = s.start + n;
    return s;
  }
};

cudaError_t launch_e4m3(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream);
cudaError_t launch_e5m2(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream);
cudaError_t launch_e2m1(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream);
cudaError_t launch_int8(const Args& a, int dim, bool wide, uint32_t ctas, cudaStream_t stream);

}  // namespace attn
}  // namespace mx
