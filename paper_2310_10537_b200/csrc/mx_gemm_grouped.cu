// The experts' products of a mixture-of-experts layer on MX operands, tcgen05 block-scaled MMA.
//
//   row groups   C[r, n]    = sum_k X[r, k] W[g(r), n, k]          X: the tokens' rows, sorted by group
//   K groups     C[g, m, n] = sum_{k in group g} X[m, k] W[n, k]   (weight gradients)
//
// The group sizes are known on the device only, and they are ragged.  Therefore the regular operand W
// takes the M side of the MMA -- a CTA pair multiplies 256 of its rows -- and the ragged operand X its
// N side, whose extent is a run-time field of the instruction: a tile has as many columns as the
// group has rows left (a multiple of 32, at most max_n), and no MMA work is spent on rows that are not
// there.  With X on the M side a group of 300 rows would cost 512.  The accumulator holds C transposed
// (lane = column of C, TMEM column = row of C); a warp stores 32 consecutive columns of one row at a time.
//
// One pair of CTAs per two SMs, persistent over the items (group, W tile, X tile) in that order, which
// every role of the kernel walks by itself from a table of the groups' first items that each CTA
// makes in shared memory.  Per CTA:
//   warp 0      copies 128 rows of W and its half of the X rows -> the stage's barrier (the leader's)
//   warp 1      (leader) four MMAs per stage
//   warp 2      (leader) scale chunks shared -> tensor memory, ahead of the MMAs
//   warp 3      copies the stage's scale chunks -> a barrier of their own
//   warps 4-11  epilogue, under the next item's MMAs: tiles of up to 128 columns have two accumulators;
//               wider ones alternate between columns 0..255 and 128..383 of tensor memory (two
//               whole ones and the scales do not fit), and the half both use is drained first
// (Scale copies issued by the MMA thread right before their MMAs wait in line behind the MMAs of the
// stage before and then hold up their own: 65536 x 4096 x 4096 over 32 groups took 1155 us that way.)
// What bounds it: large groups the power limit -- 65536 x 4096 x 4096 over 32 groups 820 to 1012 us by the state of the
// board, 2.2 to 2.7 PFLOP/s, at 1.29 GHz; of its cycles 86 % are MMAs, 2 % the hand-over of accumulators, and a stage takes 573
// clocks instead of 512.  Weight gradients 4096 x 2048 over 16 groups of 2048 rows, BF16 out: 207 to 273 us; an item has half as many
// stages, so the hand-overs and the epilogue's stores count twice: 81 % MMAs at the same clock (FP32 out 67 to 69 %, at 1.36).  128 rows on
// 56 experts of 2048 x 4096, FP4 weights: 55.7 to 60.7 us, 4.1 to 4.5 TB/s of weights; 448 tiles on 74 pairs are seven rounds of which the
// last holds 4, and a stage's copies and hand-overs take longer than its bytes.
// Every wait is bounded (see mbar_wait); on expiry a status word is set and all roles fall through to
// the common exit.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "mx.h"
#include "mx_device.cuh"
#include "mx_launch.h"
#include "mx_tcgen05.cuh"
#include "mx_tmap.h"

namespace mx {
namespace {

constexpr int kBK = 128;               // K elements per stage: 4 MX blocks, 4 MMAs
constexpr uint32_t kThreads = 384;     // 12 warps
constexpr uint32_t kTmemCols = 512;
constexpr long long kSpinLimit = 2000000000LL;  // budget of a wait in cycles (~1 s)
constexpr uint32_t kMaxStages = 10;
constexpr uint32_t kWBytes = 128 * kBK;         // one byte per element in shared memory
constexpr uint32_t kSortedGroups = 128;
constexpr uint32_t kXBoxRows = 16;              // rows of X per copy (half a 32-row step per CTA)
constexpr uint32_t kNoDrop = 0xFFFFFFFFu;       // failure drill off

enum : unsigned int {
  ST_PRODUCER_WAIT = 1,   // a stage never became empty
  ST_MMA_WAIT_FULL = 2,   // a stage never became full
  ST_MMA_WAIT_ACC = 3,    // an accumulator was never drained
  ST_EPILOGUE_WAIT = 4,   // an accumulator never became full
  ST_SCALE_WAIT = 5,      // a stage's scales never landed
};
// What an expired wait leaves behind: a word per stream (see status_word), so that a checked call learns of its own
// stream's products alone.
constexpr uint32_t kStatusWords = 128;
__device__ unsigned int g_grouped_status[kStatusWords];

struct GroupedParams {
  const int32_t* offsets;
  void* C;
  uint32_t c_bf16, groups, w_rows, x_rows, k_len, k_chunks, k_stages;  // the whole K axis in elements, chunks, stages
  uint32_t max_n, acc_step, shared_half, band, stages, sf_per_stage, x_stage_bytes, idesc, w_box_bytes, x_box_bytes;
  uint32_t drop_fill, status_word;
  long long spin_limit;
};

// One tile of C for a pair: W rows w0 .. w0 + 255, X rows x0 .. x0 + n - 1 (n a multiple of 32, those
// from x_end on are not stored), nk stages from K chunk k0 on.
struct Item {
  uint32_t group, w0, x0, n, x_end, k0, nk;
};

// Tables in shared memory: groups' offsets (rows, or K chunks) and first items.
struct Tables {
  const uint32_t* offset;
  const uint32_t* first;  // K groups: in the order of `order`
  const uint32_t* order;
};

// X rows of a group in tiles of at most max_n, as even as whole steps of 64 allow, starting at
// multiples of 64 (where the scale bytes of a tile's first row may lie in their TMEM columns).  Every tile has rows (an MMA
// of N = 0 would be a bad one): rows / tiles is at most max_n, a multiple of 64, and so is the step it is rounded up
// to; the tiles before the last then hold at most (tiles - 1) max_n rows, which is less than all.
__host__ __device__ constexpr uint32_t x_tiles(uint32_t rows, uint32_t max_n) { return (rows + max_n - 1) / max_n; }
__host__ __device__ constexpr uint32_t x_step(uint32_t rows, uint32_t tiles) { return ((rows + tiles - 1) / tiles + 63u) & ~63u; }
constexpr bool tiles_have_rows(uint32_t max_n) {
  for (uint32_t rows = 1; rows <= 4096; ++rows) {
    const uint32_t tiles = x_tiles(rows, max_n), step = x_step(rows, tiles);
    if (step > max_n || (tiles - 1) * step >= rows) return false;
  }
  return true;
}
static_assert(tiles_have_rows(64) && tiles_have_rows(128) && tiles_have_rows(256), "a tile without rows");

template <bool KG>
__device__ __forceinline__ bool next_item(const GroupedParams& p, const Tables& tb, uint32_t t, uint32_t& slot, Item& it) {
  while (slot < p.groups && t >= tb.first[slot + 1]) ++slot;
  if (slot >= p.groups) return false;
  const uint32_t g = KG ? tb.order[slot] : slot;
  const uint32_t o = tb.offset[g], len = tb.offset[g + 1] > o ? tb.offset[g + 1] - o : 0u;
  const uint32_t rows = KG ? p.x_rows : len;
  const uint32_t tiles = x_tiles(rows, p.max_n), step = x_step(rows, tiles);
  // bands of X tiles: every W tile meets a band before the next band begins, so that the tiles which
  // all pairs work on at a time share both operands in the L2
  const uint32_t j = t - tb.first[slot], w_tiles = (p.w_rows + 255) / 256, per_band = p.band * w_tiles;
  const uint32_t b = j / per_band, in_band = j - b * per_band, bx = min(p.band, tiles - b * p.band);
  const uint32_t wt = in_band / bx, xt = b * p.band + (in_band - wt * bx);
  it.group = g;
  it.w0 = wt * 256;
  it.x0 = xt * step;
  it.n = min(step, (rows - it.x0 + 31u) & ~31u);
  it.x_end = min(rows, it.x0 + it.n);
  if (KG) {
    it.k0 = o;
    it.nk = len;
  } else {
    it.x0 += o;
    it.x_end += o;
    it.k0 = 0;
    it.nk = p.k_stages;
  }
  // Every lane holds the same item, but it comes out of shared memory and the compiler does not know; a
  // broadcast says so, and the copies' and MMAs' operands stay in uniform registers.
  auto same = [](uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); };
  it.group = same(it.group); it.w0 = same(it.w0); it.x0 = same(it.x0); it.n = same(it.n);
  it.x_end = same(it.x_end); it.k0 = same(it.k0); it.nk = same(it.nk);
  return true;
}

// Offsets as the kernel may use them: the end of the tensor, or on the grid; in units of rows (KG: of K chunks, of which
// the last one may be a part: the copies fill it up with zeros).
template <bool KG>
__device__ __forceinline__ uint32_t sane_offset(const GroupedParams& p, int32_t raw) {
  const uint32_t v = raw > 0 ? (uint32_t)raw : 0u;
  if (KG) return v >= p.k_len ? p.k_chunks : v / (uint32_t)kBK;
  return v >= p.x_rows ? p.x_rows : (v & ~63u);
}

__device__ __forceinline__ void raise_abort(const GroupedParams& p, volatile uint32_t* abort_flag, unsigned int code) {
  atomicCAS(&g_grouped_status[p.status_word], 0u, code);
  *abort_flag = 1u;
}

template <bool KG, uint32_t KCH>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
mx_gemm_grouped_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
                       const __grid_constant__ CUtensorMap tmap_xf, const __grid_constant__ CUtensorMap tmap_sw,
                       const __grid_constant__ CUtensorMap tmap_sx, const GroupedParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  // a stage holds kch K chunks of 128 elements, each with its W, X and scale bytes
  const uint32_t chunk_bytes = kWBytes + p.x_stage_bytes, stage_bytes = KCH * chunk_bytes;  // multiples of 1024
  const uint32_t sf_chunk = 512u * p.sf_per_stage, sf_bytes = KCH * sf_chunk;
  const uint32_t off_sf = p.stages * stage_bytes, off_bar = off_sf + p.stages * sf_bytes;
  constexpr uint32_t kBars = 4 * kMaxStages + 4;
  const uint32_t bar0 = smem_base + off_bar;
  auto full_bar = [&](uint32_t s) { return bar0 + 8 * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8 * (kMaxStages + s); };
  auto sf_full_bar = [&](uint32_t s) { return bar0 + 8 * (2 * kMaxStages + s); };
  auto sf_ready_bar = [&](uint32_t s) { return bar0 + 8 * (3 * kMaxStages + s); };
  auto acc_full_bar = [&](uint32_t a) { return bar0 + 8 * (4 * kMaxStages + a); };
  auto acc_empty_bar = [&](uint32_t a) { return bar0 + 8 * (4 * kMaxStages + 2 + a); };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_gen + off_bar + kBars * 8);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  uint32_t* offset = reinterpret_cast<uint32_t*>(smem_gen + off_bar + kBars * 8 + 16);
  uint32_t* first = offset + p.groups + 1;
  uint32_t* order = first + p.groups + 1;  // (K groups)

  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const uint32_t bar0_leader = map_to_cta(bar0, 0);
  auto leader_bar = [&](uint32_t local_bar) { return bar0_leader + (local_bar - bar0); };

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < p.stages; ++s) {
      mbar_init(full_bar(s), 1);      // used in the leader: its producer's arrive + the bytes of both CTAs
      mbar_init(empty_bar(s), 1);     // a tcgen05.commit, delivered to both
      mbar_init(sf_full_bar(s), 1);   // as full
      mbar_init(sf_ready_bar(s), 1);  // used in the leader: the copier's tcgen05.commit
    }
    for (uint32_t a = 0; a < 2; ++a) {
      mbar_init(acc_full_bar(a), 1);
      mbar_init(acc_empty_bar(a), 16);  // used in the leader: eight epilogue warps in each CTA
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_w)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_x)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_sw)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_sx)) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  // Programmatic stream serialization: all above overlapped the kernel before; from here on its
  // results are read (the offsets first).
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (uint32_t g = threadIdx.x; g <= p.groups; g += kThreads) offset[g] = sane_offset<KG>(p, __ldg(p.offsets + g));
  __syncthreads();
  if (KG) {
    // The longest groups first, the empty ones last: pairs that take a second item then take a short one.  (4 of 8 groups
    // empty, 21831 rows, 512 x 1920: 28.6 us; 38.7 in the groups' order.)  Many groups make many items, and even out by themselves.
    for (uint32_t g = threadIdx.x; g < p.groups; g += kThreads) {
      uint32_t place = g;
      if (p.groups <= kSortedGroups) {
        auto len = [&](uint32_t i) { return offset[i + 1] > offset[i] ? offset[i + 1] - offset[i] : 0u; };
        const uint32_t mine = len(g);
        place = 0;
        for (uint32_t i = 0; i < p.groups; ++i) place += len(i) > mine || (len(i) == mine && i < g) ? 1u : 0u;
      }
      order[place] = g;
    }
  }
  if (warp == 0) {  // first item of every group: a running sum, 32 groups at a time
    const uint32_t w_tiles = (p.w_rows + 255) / 256;
    uint32_t run = 0;
    for (uint32_t g0 = 0; g0 <= p.groups; g0 += 32) {
      const uint32_t g = g0 + lane;
      uint32_t items = 0;
      if (g < p.groups) {
        const uint32_t len = offset[g + 1] > offset[g] ? offset[g + 1] - offset[g] : 0u;
        items = w_tiles * x_tiles(KG ? p.x_rows : len, p.max_n);
      }
      uint32_t scan = items;
#pragma unroll
      for (uint32_t o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += v;
      }
      if (g <= p.groups) first[g] = run + scan - items;
      run += __shfl_sync(0xffffffffu, scan, 31);
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // the peer's barriers exist before anything is signalled remotely
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const Tables tb = {offset, first, order};
  const uint32_t sf_col0 = p.acc_step + p.max_n;
  // The accumulator of a pair's i-th item lies at column acc_step * (i & 1).  Two separate ones: the item
  // waits until the one before the last is drained, each with a barrier of its own.  Overlapping ones
  // (shared_half): until the last item's part of columns 128..255 is; one barrier, a phase per item.
  auto acc_bar_index = [&](uint32_t i) { return p.shared_half ? 0u : i & 1u; };
  auto acc_parity = [&](uint32_t i) { return (p.shared_half ? i : i >> 1) & 1u; };

  if (warp == 0 || warp == 3) {
    // ------------------- copies (both CTAs): warp 0 operands, warp 3 scale chunks -------------------
    // Failure drill (drop_fill != kNoDrop): the operands' fill with that running number is left out in both CTAs -- no copy
    // is issued and its barrier is not armed -- so that the MMA issuer's wait for it runs out.
    const bool scales = warp == 3;
    const uint32_t drop = scales ? kNoDrop : p.drop_fill;
    uint32_t stage = 0, phase = 0, g = 0, fill = 0;
    bool ok = true;
    Item it;
    for (uint32_t t = pair; ok && next_item<KG>(p, tb, t, g, it); t += num_pairs) {
      const uint32_t wrow = (KG ? 0u : it.group * p.w_rows) + it.w0 + rank * 128u;
      const uint32_t half = it.n >> 1, xrow = it.x0 + rank * half, boxes = half / kXBoxRows;
      const bool whole = it.n == p.max_n;  // a full tile's X rows are one copy
      const uint32_t sx0 = it.x0 >> 7;
      const uint32_t tx = 2u * KCH * (scales ? sf_chunk : p.w_box_bytes + boxes * p.x_box_bytes);
      for (uint32_t kc = 0; kc < it.nk; ++kc) {
        ok = mbar_wait_warp(empty_bar(stage), phase ^ 1u, abort_flag, p.spin_limit);
        if (!ok) {
          raise_abort(p, abort_flag, ST_PRODUCER_WAIT);
          break;
        }
        if (fill++ != drop && elect_one()) {
          const uint32_t bar = scales ? sf_full_bar(stage) : full_bar(stage), fb = leader_bar(bar);
          if (rank == 0) mbar_arrive_expect_tx(bar, tx);
#pragma unroll
          for (uint32_t c = 0; c < KCH; ++c) {  // (a chunk past the end of K is filled with zeros)
            const uint32_t chunk = it.k0 + kc * KCH + c;
            const int kx = (int)(chunk * kBK), kz = (int)chunk;
            if (scales) {
              const uint32_t ds = smem_base + off_sf + stage * sf_bytes + c * sf_chunk;
              tma_load_3d_pair(ds, &tmap_sw, 0, kz, (int)(wrow >> 7), fb);
              tma_load_3d_pair(ds + 512u, &tmap_sx, 0, kz, (int)sx0, fb);
            } else {
              const uint32_t dw = smem_base + stage * stage_bytes + c * chunk_bytes, dx = dw + kWBytes;
              tma_load_3d_pair(dw, &tmap_w, kx, (int)wrow, 0, fb);
              if (whole) {
                tma_load_3d_pair(dx, &tmap_xf, kx, (int)xrow, 0, fb);
              } else {
                for (uint32_t j = 0; j < boxes; ++j)
                  tma_load_3d_pair(dx + j * (kXBoxRows * 128u), &tmap_x, kx, (int)(xrow + j * kXBoxRows), 0, fb);
              }
            }
          }
        }
        __syncwarp();
        if (++stage == p.stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) {  // let copies that are still in flight land before the CTA goes away
      const long long t0 = clock64();
      while (clock64() - t0 < 2000000LL) {}
    }
  } else if (warp == 2) {
    // ------------------------------ scale copier (leader) ------------------------------
    if (rank == 0) {
      uint32_t stage = 0, phase = 0, g = 0;
      bool ok = true;
      Item it;
      for (uint32_t t = pair; ok && next_item<KG>(p, tb, t, g, it); t += num_pairs) {
        for (uint32_t kc = 0; kc < it.nk; ++kc) {
          ok = mbar_wait_warp(sf_full_bar(stage), phase, abort_flag, p.spin_limit);
          if (!ok) {
            raise_abort(p, abort_flag, ST_SCALE_WAIT);
            break;
          }
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (uint32_t c = 0; c < KCH; ++c) {
              const uint32_t sf_smem = smem_base + off_sf + stage * sf_bytes + c * sf_chunk;
              const uint32_t sf_tmem = tmem_base + sf_col0 + (stage * KCH + c) * (4u * p.sf_per_stage);
#pragma unroll
              for (uint32_t j = 0; j < 4; ++j)
                if (j < p.sf_per_stage) tc_cp_scales_pair(sf_tmem + 4 * j, scale_desc(sf_smem + 512 * j));
            }
            tc_commit_leader(sf_ready_bar(stage));  // arrives when the copies have completed in both CTAs
          }
          __syncwarp();
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------ MMA issuer (leader) ------------------------------
    if (rank == 0) {
      uint32_t stage = 0, phase = 0, i = 0, g = 0;
      bool ok = true;
      Item it;
      for (uint32_t t = pair; ok && next_item<KG>(p, tb, t, g, it); t += num_pairs, ++i) {
        if (!__all_sync(0xffffffffu, mbar_wait(acc_empty_bar(acc_bar_index(i)), acc_parity(i) ^ 1u, abort_flag,
                                               4 * p.spin_limit))) {
          raise_abort(p, abort_flag, ST_MMA_WAIT_ACC);
          break;
        }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (i & 1u) * p.acc_step;
        const uint32_t sx_col = 4 + ((it.x0 & 127u) >> 5);  // a tile starts on row 0 or 64 of a scale chunk
        const uint32_t idesc0 = p.idesc | ((it.n >> 3) << 17);
        for (uint32_t kc = 0; kc < it.nk; ++kc) {
          // half of the lanes wait for the scales, half for the operands: one wait's time for both
          ok = __all_sync(0xffffffffu, mbar_wait((lane & 1u) ? full_bar(stage) : sf_ready_bar(stage), phase, abort_flag,
                                                 p.spin_limit));
          if (!ok) {
            raise_abort(p, abort_flag, ST_MMA_WAIT_FULL);
            break;
          }
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (uint32_t c = 0; c < KCH; ++c) {
              const uint32_t sf_tmem = tmem_base + sf_col0 + (stage * KCH + c) * (4u * p.sf_per_stage);
              const uint64_t wdesc = operand_desc(smem_base + stage * stage_bytes + c * chunk_bytes);
              const uint64_t xdesc = operand_desc(smem_base + stage * stage_bytes + c * chunk_bytes + kWBytes);
#pragma unroll
              for (uint32_t k = 0; k < 4; ++k)  // byte k of each scale column belongs to MX block k of the chunk
                tc_mma_pair(d_tmem, wdesc + 2 * k, xdesc + 2 * k, idesc0 | (k << 4) | (k << 29), sf_tmem, sf_tmem + sx_col,
                            (kc | c | k) != 0 ? 1u : 0u);
            }
            tc_commit_pair(empty_bar(stage));
          }
          __syncwarp();
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
        if (ok && elect_one()) tc_commit_pair(acc_full_bar(i & 1u));
        __syncwarp();
      }
    }
  } else {
    // ------------------------------ epilogue (both CTAs) ------------------------------
    // Warps q and q + 4 share the TMEM lanes 32 q .. 32 q + 31 and take alternate steps of 32 X rows.
    const uint32_t quarter = warp & 3u, odd = (warp - 4u) >> 2;
    uint32_t i = 0, g = 0;
    Item it;
    for (uint32_t t = pair; next_item<KG>(p, tb, t, g, it); t += num_pairs, ++i) {
      if (!mbar_wait_warp(acc_full_bar(i & 1u), (i >> 1) & 1u, abort_flag, 4 * p.spin_limit)) {
        if (lane == 0) raise_abort(p, abort_flag, ST_EPILOGUE_WAIT);
        break;
      }
      tc_fence_after();
      const uint32_t n = it.w0 + rank * 128u + quarter * 32u + lane;  // this thread's column of C
      const size_t row_base = KG ? (size_t)it.group * p.x_rows : 0;
      const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + (i & 1u) * p.acc_step;
      // up to two steps (64 columns of the tile) from column c on, 64 apart, into registers
      auto load = [&](uint32_t c, uint32_t (&r)[2][32]) {
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
          if (c + 64 * h < it.n && it.nk != 0) {
            tc_ld32(taddr + c + 64 * h, r[h]);
          } else {  // an empty K group: no MMA has written the accumulator
#pragma unroll
            for (int j = 0; j < 32; ++j) r[h][j] = 0u;
          }
        }
        tc_wait_ld();
      };
      auto store = [&](uint32_t c, const uint32_t (&r)[2][32]) {
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
          const uint32_t r0 = it.x0 + c + 64 * h, live = it.x_end > r0 ? it.x_end - r0 : 0u;
          if (n >= p.w_rows || live == 0) continue;
          const size_t at = (row_base + r0) * p.w_rows + n;
          if (p.c_bf16) {
            uint16_t* dst = reinterpret_cast<uint16_t*>(p.C) + at;
#pragma unroll
            for (uint32_t j = 0; j < 32; ++j) {
              uint16_t v;
              asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(v) : "f"(__uint_as_float(r[h][j])));
              if (j < live) dst[(size_t)j * p.w_rows] = v;
            }
          } else {
            float* dst = reinterpret_cast<float*>(p.C) + at;
#pragma unroll
            for (uint32_t j = 0; j < 32; ++j)
              if (j < live) dst[(size_t)j * p.w_rows] = __uint_as_float(r[h][j]);
          }
        }
      };
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(leader_bar(acc_empty_bar(acc_bar_index(i))));
      };
      // columns 128..255 of tensor memory first where the next item uses them too
      const uint32_t c0 = (p.shared_half && !(i & 1u)) ? 128u : 0u, c1 = 128u - c0;
      uint32_t r[2][32];
      load(c0 + 32 * odd, r);
      release();
      store(c0 + 32 * odd, r);
      if (p.shared_half) {
        load(c1 + 32 * odd, r);
        store(c1 + 32 * odd, r);
      }
    }
  }

  // The next kernel may be launched: 0.5 to 1 us of a product of 10 us.  (Not earlier: blocks that wait on the SMs
  // took 2 % from a training step's products.)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // common exit: both CTAs leave together, then the pair's tensor memory is freed
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

// ---- host side ---------------------------------------------------------------

int fmt_bits(int f) { return f == MX_E2M1 ? 4 : ((f == MX_E3M2 || f == MX_E2M3) ? 6 : 8); }

uint32_t mma_fmt_code(int f) {  // format field of the instruction descriptor
  switch (f) {
    case MX_E4M3: return 0;
    case MX_E5M2: return 1;
    case MX_E2M3: return 3;
    case MX_E3M2: return 4;
    default: return 5;  // MX_E2M1
  }
}

bool encode(EncodeTiledFn fn, CUtensorMap* map, CUtensorMapDataType dt, const void* ptr, const cuuint64_t (&dims)[3],
            const cuuint64_t (&strides)[2], const cuuint32_t (&box)[3], CUtensorMapSwizzle swz) {
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, dt, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swz,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Packed K-major operand [rows x K], box 128 elements x box_rows, 128-byte swizzle; 6- and 4-bit codes
// are expanded to a byte each on the way in.
bool operand_map(EncodeTiledFn fn, CUtensorMap* map, const void* ptr, int fmt, uint64_t rows, uint64_t K, uint32_t box_rows) {
  const int bits = fmt_bits(fmt);
  const CUtensorMapDataType dt = bits == 8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                 : bits == 6 ? CU_TENSOR_MAP_DATA_TYPE_16U6_ALIGN16B
                                             : CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B;
  const cuuint64_t pitch = K * (uint64_t)bits / 8;
  return encode(fn, map, dt, ptr, {K, rows, 1}, {pitch, pitch * rows}, {(cuuint32_t)kBK, box_rows, 1},
                CU_TENSOR_MAP_SWIZZLE_128B);
}

// Swizzled scale tensor as [groups of 128 rows][K chunks][128 words], a box `chunks` 512-byte chunks of
// consecutive row groups.
bool scale_map(EncodeTiledFn fn, CUtensorMap* map, const void* ptr, uint64_t rows, uint64_t K, uint32_t chunks) {
  const uint64_t k_chunks = (K + kBK - 1) / kBK;
  return encode(fn, map, CU_TENSOR_MAP_DATA_TYPE_UINT32, ptr, {128, k_chunks, (rows + 127) / 128},
                {512, 512 * k_chunks}, {128, 1, chunks}, CU_TENSOR_MAP_SWIZZLE_NONE);
}

// The status word of a stream of device `dev`: a table of stream handles, entered without a lock.  When more streams
// have come than there are words, a word serves several of them, and a checked call may also report a
// failure of another of those.
uint32_t status_word(int dev, cudaStream_t stream) {
  static std::atomic<uintptr_t> table[64][kStatusWords];
  const uintptr_t key = (uintptr_t)stream + 1;  // (the default stream is 0)
  const uint32_t start = (uint32_t)((key >> 4) * 2654435761u >> 16) % kStatusWords;
  if (dev < 0 || dev >= 64) return start;
  for (uint32_t i = 0; i < kStatusWords; ++i) {
    std::atomic<uintptr_t>& slot = table[dev][(start + i) % kStatusWords];
    uintptr_t have = slot.load(std::memory_order_relaxed);
    if (have == 0 && slot.compare_exchange_strong(have, key, std::memory_order_relaxed)) have = key;
    if (have == key) return (start + i) % kStatusWords;
  }
  return start;
}

template <bool KG, uint32_t KCH>
cudaError_t launch_kernel(const GroupedArgs& a, EncodeTiledFn fn, uint32_t max_n) {
  CUtensorMap mw, mx_, mxf, msw, msx;
  const uint64_t w_all = (uint64_t)a.w_rows * (KG ? 1u : (uint64_t)a.groups);
  if (!operand_map(fn, &mw, a.W, a.fmtW, w_all, (uint64_t)a.K, 128) ||
      !operand_map(fn, &mx_, a.X, a.fmtX, (uint64_t)a.x_rows, (uint64_t)a.K, kXBoxRows) ||
      !scale_map(fn, &msw, a.sW, w_all, (uint64_t)a.K, 1))
    return cudaErrorInvalidValue;
  GroupedParams p;
  p.offsets = a.offsets; p.C = a.C; p.c_bf16 = (uint32_t)a.c_bf16; p.groups = (uint32_t)a.groups;
  p.w_rows = (uint32_t)a.w_rows; p.x_rows = (uint32_t)a.x_rows; p.k_len = (uint32_t)a.K;
  p.k_chunks = (uint32_t)((a.K + kBK - 1) / kBK);
  p.max_n = max_n;
  p.shared_half = p.max_n == 256 ? 1u : 0u;
  p.acc_step = p.shared_half ? 128 : p.max_n;
  // scale chunks per stage: one of W, and X rows 64 .. 64 + max_n - 1 of a chunk grid of 128
  p.sf_per_stage = 1 + (p.max_n == 64 ? 1 : p.max_n == 128 ? 2 : 3);
  if (!operand_map(fn, &mxf, a.X, a.fmtX, (uint64_t)a.x_rows, (uint64_t)a.K, p.max_n / 2) ||
      !scale_map(fn, &msx, a.sX, (uint64_t)a.x_rows, (uint64_t)a.K, p.sf_per_stage - 1))
    return cudaErrorInvalidValue;
  p.x_stage_bytes = p.max_n / 2 * 128;
  p.k_stages = (p.k_chunks + KCH - 1) / KCH;
  p.band = 16;
  const uint32_t fixed = 1024 + (4 * kMaxStages + 4) * 8 + 16 + (KG ? 3 : 2) * (p.groups + 1) * 4;
  const uint32_t per_stage = KCH * (kWBytes + p.x_stage_bytes + 512 * p.sf_per_stage);
  p.stages = (232448u - fixed) / per_stage;
  const uint32_t tmem_stages = (kTmemCols - p.acc_step - p.max_n) / (4 * p.sf_per_stage * KCH);
  if (p.stages > tmem_stages) p.stages = tmem_stages;
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  const uint32_t smem = fixed + p.stages * per_stage;
  // a_format [7,10), b_format [10,13), scale format E8M0 (bit 23), M = 256; N is set per item
  p.idesc = (mma_fmt_code(a.fmtW) << 7) | (mma_fmt_code(a.fmtX) << 10) | (1u << 23) | ((uint32_t)(256 >> 4) << 24);
  // bytes a copy reports: packed source bytes, rows past the end included
  p.w_box_bytes = (uint32_t)(128 * kBK * fmt_bits(a.fmtW) / 8);
  p.x_box_bytes = (uint32_t)(kXBoxRows * kBK * fmt_bits(a.fmtX) / 8);
  p.spin_limit = a.wait_cycles ? a.wait_cycles : kSpinLimit;
  p.drop_fill = a.drop_fill < 0 ? kNoDrop : (uint32_t)a.drop_fill;
  static bool attr_set[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(mx_gemm_grouped_kernel<KG, KCH>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  p.status_word = status_word(dev, a.stream);
  // no more pairs than items there can be: every group at most one tile more than its share of rows
  const int64_t w_tiles = (a.w_rows + 255) / 256;
  const int64_t most = KG ? a.groups * w_tiles * ((a.x_rows + p.max_n - 1) / p.max_n)
                          : w_tiles * (a.groups + a.x_rows / p.max_n);
  const uint32_t pairs = most < a.sm_count / 2 ? (uint32_t)most : (uint32_t)(a.sm_count / 2);
  return launch_pdl(mx_gemm_grouped_kernel<KG, KCH>, dim3(2 * pairs), dim3(kThreads), smem, a.stream, mw, mx_, mxf, msw, msx, p);
}

}  // namespace

int launch_gemm_grouped(const GroupedArgs& a, cudaError_t* cuda_err) {
  *cuda_err = cudaSuccess;
  EncodeTiledFn fn = encode_fn(cuda_err);
  if (!fn) return MX_ERR_CUDA;
  // The widest tile.  256 columns move the fewest operand bytes per MAC, which is what bounds large groups
  // (65536 x 4096 x 4096 over 32 groups: 943 us with 192, 835 with 256 on the same board; 820 to 1012 by the state of the board).  Groups that hold 64
  // rows on average take tiles of 64: a stage is then smaller and more of W is in flight, which is what
  // bounds a product with few rows; two K chunks share a stage there, since the hand-overs of a stage of
  // one chunk take as long as its copies (128 rows on 56 experts of 2048 x 4096: FP4 weights 66.9 -> 57.1 us
  // with two, FP8 88.9 -> 85.3).  A plan's row bound holds up to 63 rows of padding a group: hence 96 and 192.
  const int64_t avg = a.k_groups ? a.x_rows : a.x_rows / a.groups;
  const uint32_t max_n = avg <= 96 ? 64 : avg <= 192 ? 128 : 256;
  *cuda_err = a.k_groups ? launch_kernel<true, 1>(a, fn, max_n)
                         : max_n == 64 ? launch_kernel<false, 2>(a, fn, max_n) : launch_kernel<false, 1>(a, fn, max_n);
  return *cuda_err == cudaSuccess ? MX_OK : MX_ERR_CUDA;
}

// Reads and clears the stream's status word, after what has been launched on the stream.
int gemm_grouped_status(cudaStream_t stream, unsigned int* out, cudaError_t* cuda_err) {
  int dev = 0;
  *cuda_err = cudaGetDevice(&dev);
  const size_t at = sizeof(unsigned int) * status_word(dev, stream);
  const unsigned int zero = 0;
  if (*cuda_err == cudaSuccess)
    *cuda_err = cudaMemcpyFromSymbolAsync(out, g_grouped_status, sizeof(unsigned int), at, cudaMemcpyDeviceToHost, stream);
  if (*cuda_err == cudaSuccess) *cuda_err = cudaStreamSynchronize(stream);
  if (*cuda_err == cudaSuccess && *out != 0) {
    *cuda_err = cudaMemcpyToSymbolAsync(g_grouped_status, &zero, sizeof(unsigned int), at, cudaMemcpyHostToDevice, stream);
    if (*cuda_err == cudaSuccess) *cuda_err = cudaStreamSynchronize(stream);
  }
  return *cuda_err == cudaSuccess ? MX_OK : MX_ERR_CUDA;
}

}  // namespace mx
