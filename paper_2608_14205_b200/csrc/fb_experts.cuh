// The experts' side of a layer: products grouped by slot over the dispatch order (fb_expert_matmul), rows of 8-bit
// floats with block scales (fb_quantize_rows) and the weighted sum of a token's rows (fb_combine).
//
// fb_expert_matmul.  For the rows p of slot s (slot_offsets[s] <= p < slot_offsets[s + 1])
//     out[p] = act(x[row(p)] W_s^T),   row(p) = perm[p] / k  (or p),
// act none, or SwiGLU over W_s = [gate rows; up rows]: g / (1 + exp(-g)) * u.  With e4m3 operands the product is
//     sum over blocks b of 128 columns of  sx[row][b] * sw[i / 128][b] * (q_x[row][b] . q_w[i][b]),
// the inner products on the tensor cores, the scaled sum over the blocks in 32-bit registers.
//
// Two kernels, here for bf16 and in fb_experts_e4m3.cuh for e4m3.  Both have blocks that stay, each of which walks its
// tiles t, t + blocks, ...; the map from a number to (slot, rows of W, rows of x) is a prefix sum over the slots, made by
// every block from slot_offsets: nothing is handed from one launch to the next and no scratch is used, so calls may
// overlap on any streams.  In both, rows of x that lie one behind the other come by TMA, gathered ones by cp.async from
// four warps.  (The gathering TMA load, four rows per copy, took 16 cycles a row here, 2000 per k-block of 128 rows, while
// the MMAs of that block take 512: up projection of 8192 x 2048 with 128 experts of 768 in 890 us, 331 us with tiles of
// rows that were gathered before.)
//
// bf16.  A pair of blocks (tcgen05 cta_group::2) takes tiles of 256 rows of W by up to 256 rows of x.  The MMA's M side is
// W, whose size is a multiple of what a tile needs in all practice; its N side, which goes in steps of 32, is x, so that
// the ragged counts of the slots (a few rows in decode, any number in prefill) cost what they have, not what a tile holds:
// a slot with 300 rows is two tiles of 160, not two of 256.
// Warps: 0 loads by TMA, 1 issues the MMAs (even block), 2 passes on that gathered rows are there, 4-11 take the
// accumulators out while the next tile's MMAs run, 12-15 gather.  TMEM lanes are rows of W, columns rows of x; the
// 16x256b form of tcgen05.ld gives a thread the same columns of lanes r and r + 16, where W's tile has its gate row r and
// up row r side by side (the tensor map interleaves them 16 by 16), so SwiGLU needs no exchange.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/freebalance.h"
#include "fb_ptx.cuh"

namespace fb {

constexpr int kExpertThreads = 512;
constexpr int kExpertEpilogueWarps = 8;
constexpr int kExpertFirstEpilogueWarp = 4;
constexpr int kExpertFirstGatherWarp = 12;
constexpr int kGatherWarps = 4;
constexpr int kGatherRows = 8;                          // rows per thread: 128 rows / 4 warps / 4 rows per copy of a warp
constexpr int kTileLoadRows = 16;                       // rows of x per TMA load
constexpr int kNoRow = -2, kZeroRow = -1;
constexpr uint32_t kExpertRingBytes = 6 * 32768;         // stages of 128 rows of W and as many of x as the largest tile has
constexpr int kExpertTileM = 256;                       // rows of W per pair
constexpr int kExpertTileN = 256;                       // rows of x per tile at most
constexpr int kExpertStepN = 32;                        // (the MMA of a pair takes N in steps of 32)
constexpr uint32_t kExpertWBytes = 128 * 128;           // 128 rows of W, 128 bytes each
constexpr int kExpertStages = kExpertRingBytes / (kExpertWBytes + 64 * kExpertStepN);      // of the smallest tile
constexpr int kBand = 8;                                // tiles of x that share a walk over W (4, 8, 16, 64: 5.62, 5.64, 5.72, 5.94 ms for
                                                        // 131072 tokens of 128 experts; 16384 and fewer: no difference)

struct ExpertParams {
  const uint32_t* slot_offsets;    // [n_slots + 1] or NULL (one slot of `rows` rows)
  const int32_t* perm;             // or NULL
  const void* x;                   // [x_rows][row_bytes]
  const float* x_scale;            // [x_rows][scale_k]
  const float* w_scale;            // per slot [row blocks][scale_k]
  uint64_t w_scale_slot;           // words from one slot's scales to the next
  void* out;                       // [rows][n_out]
  float* out_scale;                // [rows][ceil(n_out / 128)]
  int32_t* status;
  int32_t n_slots, k, x_rows, rows;
  int32_t row_bytes;               // of x
  int32_t num_kb;                  // steps of 128 bytes of K
  int32_t n_out;                   // columns of out
  int32_t m_blocks;                // tiles of W per slot
  int32_t scale_k;                 // ceil(K / 128)
  int32_t max_tiles;               // tiles of x that rising offsets can give
  int32_t pieces;                  // split launches: blocks (pairs) of a cluster that share a tile's K
};

// Split launches.  A call with fewer tiles than the GPU has blocks (or pairs) for is latency: one tile's k-blocks one after the
// other.  There a cluster shares the tile, each block (pair) a range of K; the partial sums go through the rings, which
// are done with by then, and are added up in the order of the pieces by the block that stores the result.  (When: fb_expert_matmul.)
struct KRange {
  int begin, end;                  // k-blocks
};
__device__ __forceinline__ KRange k_range(const ExpertParams& p, int piece) {
  return {static_cast<int>(static_cast<long long>(p.num_kb) * piece / p.pieces), static_cast<int>(static_cast<long long>(p.num_kb) * (piece + 1) / p.pieces)};
}
// All threads of a cluster, warp by warp, wherever they are.
__device__ __forceinline__ void cluster_meet() {
  __syncwarp();
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ float4 ld_cluster_v4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

struct ExpertTiles {
  int32_t most;                                         // rows of x in the largest tile
  // A slot has several tiles, so W is read more than once.  Where none has, its loads go first when L2 needs room (decode, 64
  // tokens of 256 experts of 7168 x 2048 in e4m3: 906 -> 900 us; with it for prefill of 16384 tokens: 4900 -> 5250 us).
  int32_t several;
  int32_t warp_most[kExpertThreads / 32];
  int32_t warp_sums[kExpertThreads / 32];
  int32_t first_tile[FB_MAX_EXPERTS + 1];               // tiles of x before this slot's
  int32_t first_row[FB_MAX_EXPERTS];
  int32_t count[FB_MAX_EXPERTS];
};

struct ExpertShared {
  uint64_t full_bar[kExpertStages], empty_bar[kExpertStages];
  uint64_t x_bar[kExpertStages];                        // this block's gathered rows have arrived
  uint64_t acc_full[2], acc_empty[2];                   // per set of 256 columns
  uint64_t rows_bar[2];                                 // SwiGLU, per half of the warps: 32 rows of results are staged
  uint32_t tmem_base;
  int32_t abort_flag;
  ExpertTiles tiles;
};

// ---------------------------------------------------------------- copies
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1, int32_t c2, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_5d_pair(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1, int32_t c2,
                                                 int32_t c3, int32_t c4, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5, %6, %7}], [%2], %8;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_rows_pair(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
// 16 bytes to shared memory, zeros where bytes == 0.
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Ordinary writes to shared memory before it are seen by the tensor core.
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Arrive at the barrier at this offset in a block of the pair, for hand-overs whose data is no ordinary memory (TMEM), or
// has been made visible by a fence of its own.  (mbar_arrive_cluster's release at cluster scope waits about a microsecond.)
__device__ __forceinline__ void mbar_arrive_pair(uint32_t bar, uint32_t rank) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(map_to_cta(bar, rank)) : "memory");
}
// The same when pred != 0; a predicated copy, not a branch.
__device__ __forceinline__ void cp_async_16_if(uint32_t pred, uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %3, 0;\n@p cp.async.cg.shared.global [%0], [%1], 16, %2;\n}\n" ::"r"(dst), "l"(src), "r"(bytes), "r"(pred)
               : "memory");
}
// Arrives at the barrier once the thread's copies so far are complete.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// ---------------------------------------------------------------- tensor cores
// 16 lanes x 32 columns: register 4 g + 2 h + b of thread t is lane t / 4 + 8 h, column 8 g + 2 (t % 4) + b.
__device__ __forceinline__ void tmem_ld_16x256b(uint32_t taddr, float (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(taddr)
      : "memory");
}
// Four 8x8 matrices of 16-bit numbers, transposed: lane l's address is row l % 8 of matrix l / 8 as stored.
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}
// (__fdividef gives 0 for a divisor above 2^126: silu(g) is 0 for g below -87)
__device__ __forceinline__ float swiglu(float g, float u) { return __fdividef(g, 1.0f + __expf(-g)) * u; }

// ---------------------------------------------------------------- tiles
struct ExpertTile {
  int slot, m;                     // slot, tile of W
  int row, valid;                  // first row (a position counted from slot_offsets[0]) and rows of x
  int n;                           // valid rounded up to kExpertStepN
};

// Tiles of x of a slot with c rows: as few as possible; bf16: all but the last of equal size, in steps of kExpertStepN.
__device__ __forceinline__ int round_up_n(int rows) { return (rows + kExpertStepN - 1) / kExpertStepN * kExpertStepN; }
template <int kRows>
__device__ __forceinline__ int expert_tile_rows(int c, int tiles) { return kRows == kExpertTileN ? round_up_n((c + tiles - 1) / tiles) : kRows; }
template <int kRows>
__device__ __forceinline__ int expert_tiles(int c) {
  if (c <= 0) return 0;
  const int per = expert_tile_rows<kRows>(c, (c + kRows - 1) / kRows);
  return (c + per - 1) / per;
}

// All threads: the tiles of every slot; returns their number times the tiles of W.  Counts that are no prefix sums below
// `rows` are reported and their rows left out (all rows, where slots overlap so much that the launch was not sized for it).
template <int kRows>
__device__ __forceinline__ int expert_plan_tiles(ExpertTiles& sh, const ExpertParams& p, uint32_t& base) {
  const int e = threadIdx.x, lane = e & 31, warp = e >> 5;
  int tiles = 0, most = 0;
  base = p.slot_offsets != nullptr ? p.slot_offsets[0] : 0u;
  if (e < p.n_slots) {
    int first = 0, count = p.rows;
    if (p.slot_offsets != nullptr) {
      const uint32_t lo = p.slot_offsets[e], hi = p.slot_offsets[e + 1];
      const uint64_t positions = p.perm != nullptr ? static_cast<uint64_t>(p.x_rows) * static_cast<uint32_t>(p.k) : UINT32_MAX;
      if (base <= lo && lo <= hi && hi - base <= static_cast<uint32_t>(p.rows) && hi <= positions) {
        first = static_cast<int>(lo - base);
        count = static_cast<int>(hi - lo);
      } else {
        count = 0;
        atomicCAS(p.status, 0, FB_ERR_RANGE);
      }
    }
    tiles = expert_tiles<kRows>(count);
    if (tiles > 0) most = expert_tile_rows<kRows>(count, tiles);
    sh.first_row[e] = first;
    sh.count[e] = count;
  }
  int sum = tiles;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += v;
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 31) { sh.warp_sums[warp] = sum; sh.warp_most[warp] = most; }
  const int several = __syncthreads_or(tiles > 1);
  const int w = lane < kExpertThreads / 32 ? sh.warp_sums[lane] : 0;
  sum += __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
  if (e < p.n_slots) sh.first_tile[e + 1] = sum;
  if (e == 0) {
    sh.first_tile[0] = 0;
    most = 0;
    for (int i = 0; i < (p.n_slots + 31) / 32; ++i) most = max(most, sh.warp_most[i]);
    sh.most = most;
    sh.several = several;
  }
  __syncthreads();
  const int all = sh.first_tile[p.n_slots];
  if (all <= p.max_tiles) return all * p.m_blocks;
  if (e == 0) atomicCAS(p.status, 0, FB_ERR_RANGE);
  return 0;
}

// Tile number g: slot by slot; inside a slot bands of up to kBand tiles of x, which walk over W together (a tile of W is
// then read by the band's tiles at about the same time, and the band's rows of x stay in L2).  A whole warp asks, for
// numbers that rise: from_slot is the slot of the one before (0 at first), 32 slots are looked at at a time.
template <int kRows>
__device__ __forceinline__ ExpertTile expert_tile(const ExpertTiles& sh, const ExpertParams& p, int g, int& from_slot) {
  const int tile = g / p.m_blocks, lane = threadIdx.x & 31;
  int slot = from_slot;
  for (;;) {                                             // first_tile[slot] <= tile < first_tile[slot + 1]
    const int at = slot + 1 + lane;
    const unsigned past = __ballot_sync(0xffffffffu, at >= p.n_slots || sh.first_tile[at] > tile);
    if (past != 0) { slot += __ffs(past) - 1; break; }
    slot += 32;
  }
  from_slot = slot;
  ExpertTile t;
  t.slot = slot;
  const int first = sh.first_tile[slot], tiles = sh.first_tile[slot + 1] - first;
  int r = g - first * p.m_blocks, j = 0, width = tiles;
  if (tiles > kBand) {
    j = r / (kBand * p.m_blocks) * kBand;
    width = min(kBand, tiles - j);
    r -= j * p.m_blocks;
  }
  t.m = r;
  if (width > 1) {
    t.m = r / width;
    j += r - t.m * width;
  }
  const int count = sh.count[slot], per = expert_tile_rows<kRows>(count, tiles);
  t.row = sh.first_row[slot] + j * per;
  t.valid = min(per, count - j * per);
  t.n = round_up_n(t.valid);
  return t;
}

// The row of x that is row i of a tile, or kZeroRow behind the tile's last one.  (Zeros there, not whatever was there or a
// repeated row: the results are not stored, but products of zeros take less power, and the power limit sets the clock.)
__device__ __forceinline__ int expert_x_row(const ExpertParams& p, uint32_t base, const ExpertTile& t, int i) {
  int x = t.row + min(i, t.valid - 1);                   // counted from slot_offsets[0]; no branch: a thread's loads go out together
  if (p.perm != nullptr) {
    const int32_t entry = p.perm[static_cast<size_t>(base) + x];
    x = static_cast<int>(static_cast<uint32_t>(entry) / static_cast<uint32_t>(p.k)) | entry >> 31;      // (a negative entry: -1, not row 0)
  }
  if (static_cast<unsigned>(x) >= static_cast<unsigned>(p.x_rows)) {
    atomicCAS(p.status, 0, FB_ERR_RANGE);
    x = 0;
  }
  return i < t.valid ? x : kZeroRow;
}

template <bool kSwiglu>
struct ExpertLayout {
  // Rows with a pad that keeps eight of them in different banks.  SwiGLU: the 64 numbers of a block's part of a row, 32 rows, in
  // two buffers for each half of the warps; else the 32 numbers of a warp, 32 rows for each warp.
  static constexpr int kRowBytes = kSwiglu ? 144 : 80;
  static constexpr int kBuffer = 32 * kRowBytes;
  static constexpr uint32_t kStagingAt = kExpertRingBytes;
  static constexpr uint32_t kDynamic = kStagingAt + (kSwiglu ? 4 : kExpertEpilogueWarps) * kBuffer + 1024;
};

// The gather warps' part of a kernel: for every k-block of every tile, rows_of(g, row0, r) gives the row numbers of this
// thread's rows row0 + 16 i of the block's 128 (kNoRow: nothing is written, kZeroRow: zeros are), whose 16 bytes each go to
// the stage's tile of 128-byte rows in the 128-byte swizzle.  x_bar[s] counts the threads whose copies are complete and the warps.
template <typename Rows>
__device__ __forceinline__ void gather_rows(const ExpertParams& p, KRange k, int total, int first, int stride, uint32_t x_tiles, uint32_t stages,
                                            uint32_t stage_bytes, uint64_t* empty_bar,
                                            uint64_t* x_bar, volatile int* abort_flag, Rows rows_of) {
  const int lane = threadIdx.x & 31, unit = lane & 7;
  const int row0 = (static_cast<int>(threadIdx.x >> 5) - kExpertFirstGatherWarp) * 4 + (lane >> 3);
  const uint32_t row_bytes = static_cast<uint32_t>(p.row_bytes);
  const uint32_t to = x_tiles + static_cast<uint32_t>(row0 * 128 + ((unit ^ (row0 & 7)) << 4));        // (16 i rows on: same swizzle)
  // 16 bytes of the last k-block that lie behind the row's end are zeros
  const bool tail = static_cast<uint32_t>(p.num_kb - 1) * 128u + 16u * unit < row_bytes;
  uint32_t s = 0, phase = 0;
  bool ok = true;
  int32_t rows[kGatherRows];
#pragma unroll
  for (int i = 0; i < kGatherRows; ++i) rows[i] = kNoRow;
  if (first < total) rows_of(first, row0, rows);
  for (int g = first; g < total && ok; g += stride) {
    const uint8_t* src[kGatherRows];
    uint32_t some = 0, zero = 0;                         // rows i to copy, to clear
#pragma unroll
    for (int i = 0; i < kGatherRows; ++i) {
      src[i] = static_cast<const uint8_t*>(p.x) + static_cast<uint64_t>(static_cast<uint32_t>(max(rows[i], 0))) * row_bytes + 16u * unit;
      some |= (rows[i] >= 0 ? 1u : 0u) << i;
      zero |= (rows[i] == kZeroRow ? 1u : 0u) << i;
    }
    const bool whole = __all_sync(0xffffffffu, some == (1u << kGatherRows) - 1);
    for (int kb = k.begin; kb < k.end; ++kb) {
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&empty_bar[s]), phase ^ 1u, abort_flag));
      if (!ok) break;
      const bool inside = kb + 1 < p.num_kb || tail;
      const uint32_t bytes = inside ? 16u : 0u, at = inside ? static_cast<uint32_t>(kb) * 128u : 0u, dst = to + s * stage_bytes;
      if (whole) {
#pragma unroll
        for (int i = 0; i < kGatherRows; ++i) cp_async_16(dst + 2048u * i, src[i] + at, bytes);
      } else {
#pragma unroll
        for (int i = 0; i < kGatherRows; ++i)
          cp_async_16_if(some & (1u << i), dst + 2048u * i, src[i] + at, bytes);
        if (kb - k.begin < static_cast<int>(stages) && zero != 0) {      // zeros stay for the tile's later uses of the stage
#pragma unroll
          for (int i = 0; i < kGatherRows; ++i)
            if ((zero >> i) & 1u) st_shared_v4(dst + 2048u * i, 0u, 0u, 0u, 0u);
        }
        __syncwarp();
      }
      if (lane == 0) mbar_arrive(smem_u32(&x_bar[s]));   // (the zeros; the copies report for themselves)
      cp_async_arrive(smem_u32(&x_bar[s]));
      if (kb == k.begin && g + stride < total) rows_of(g + stride, row0, rows);      // these numbers arrive meanwhile
      if (++s == stages) { s = 0; phase ^= 1u; }
    }
  }
  cp_async_wait_all();
}

// The loading warp's end: every stage is free again.  A commit of the MMAs arrives at the barriers of both blocks of a pair, in no
// order with the other commit behind the same MMAs, so the results' barrier says nothing about these arrivals: without this wait
// a block could leave while one is on its way to its shared memory.  (A stage never used passes at once.)
__device__ __forceinline__ bool take_back_stages(uint64_t* empty_bar, uint32_t s, uint32_t phase, uint32_t stages, volatile int* abort_flag) {
  for (uint32_t i = 0; i < stages; ++i) {
    if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&empty_bar[s]), phase ^ 1u, abort_flag))) return false;
    if (++s == stages) { s = 0; phase ^= 1u; }
  }
  return true;
}

// One warp's part: gathered rows that have arrived are made visible to the tensor core and reported.
template <typename Arrive>
__device__ __forceinline__ void pass_on_rows(KRange k, int total, int first, int stride, uint32_t stages, uint64_t* x_bar,
                                             volatile int* abort_flag, Arrive arrive) {
  uint32_t s = 0, phase = 0;
  bool ok = true;
  for (int g = first; g < total && ok; g += stride)
    for (int kb = k.begin; kb < k.end; ++kb) {
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&x_bar[s]), phase, abort_flag));
      if (!ok) break;
      fence_proxy_async();
      if ((threadIdx.x & 31) == 0) arrive(s);
      __syncwarp();
      if (++s == stages) { s = 0; phase ^= 1u; }
    }
}

// Large calls are bound by the tensor cores under the power limit: 131072 x 2048 with 128 experts of 768, up projection with
// SwiGLU, 4.75 ms (1388 TFLOP/s) in short runs and 5.57 - 5.88 ms (1184 - 1122) at 1000 W; one 8192 x 8192 x 8192 product 855 us there,
// cuBLAS 860 - 900.  Ragged ones lose what small tiles and their fixed stride cost (8192 tokens, slots of 150 - 2000 rows: 353 us and
// 418 - 449, 1168 and 987 - 918; the busiest pair has 9 - 11 % more columns than the mean).  Few rows are bound by the stream of W: 40
// tokens, down projection, 56.5 us, 6.2 TB/s of 6.5 measured; one token, 50 MB, 13.4 us (13.7 where every pass reads other experts,
// from HBM), of which 8.6 are the stream (96 SMs have tiles), the rest launch, offsets, row numbers and the way out one after the other.
template <bool kSwiglu, bool kSplit>
__global__ void __launch_bounds__(kExpertThreads, 1)
fb_expert_matmul_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                        const __grid_constant__ ExpertParams p) {
  using L = ExpertLayout<kSwiglu>;
  constexpr int kStepK = 64;                             // numbers of K per stage
  extern __shared__ uint8_t smem_raw[];
  __shared__ ExpertShared sh;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  const int lane = threadIdx.x & 31;
  const uint32_t cluster_rank = cluster_ctarank(), leader_rank = cluster_rank & ~1u;
  const int rank = static_cast<int>(cluster_rank & 1u), piece = kSplit ? static_cast<int>(cluster_rank >> 1) : 0;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  volatile int* abort_flag = &sh.abort_flag;
  const bool gather = p.perm != nullptr;

  if (threadIdx.x == 0) {
    sh.abort_flag = 0;
    for (int s = 0; s < kExpertStages; ++s) {
      mbar_init(smem_u32(&sh.full_bar[s]), gather ? 3 : 1);        // the TMA loads; each block's gathered rows
      mbar_init(smem_u32(&sh.empty_bar[s]), 1);
      mbar_init(smem_u32(&sh.x_bar[s]), 33 * kGatherWarps);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(smem_u32(&sh.acc_full[a]), 1);
      mbar_init(smem_u32(&sh.acc_empty[a]), 2 * kExpertEpilogueWarps);
      mbar_init(smem_u32(&sh.rows_bar[a]), kExpertEpilogueWarps / 2);
    }
    fence_mbar_init();
    if (!gather) prefetch_tensormap(&map_x);           // (a gather has none)
    prefetch_tensormap(&map_w);
  }
  if (warp == 1) {
    tmem_alloc<2>(smem_u32(&sh.tmem_base), 512);
    tmem_relinquish<2>();
  }
  tcgen05_fence_before();
  __syncthreads();
  cluster_arrive_relaxed(); cluster_wait();              // the partner's barriers and tensor memory are ready too
  tcgen05_fence_after();
  pdl_wait();
  pdl_launch_dependents();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem_base, 0);      // (warp-uniform for the compiler as well)
  uint32_t base;
  int slot = 0;                                          // of the warp's last tile
  const int total = expert_plan_tiles<kExpertTileN>(sh.tiles, p, base);
  const int sharers = kSplit ? 2 * p.pieces : 2;         // blocks per tile
  const int stride = static_cast<int>(gridDim.x) / sharers, first = static_cast<int>(blockIdx.x) / sharers;
  const KRange kr = kSplit ? k_range(p, piece) : KRange{0, p.num_kb};
  // Few rows per tile leave room for more stages: what is under way is W, and a launch of few tiles has few blocks to ask for it.
  const uint32_t stage_bytes = kExpertWBytes + 64u * static_cast<uint32_t>(max(sh.tiles.most, kExpertStepN));
  const uint32_t stages = kExpertRingBytes / stage_bytes;      // (kExpertStages at most)

  if (warp == 0) {
    // -------------------------------------------------------------- TMA loads
    const bool leader = elect_one();
    const uint64_t policy = sh.tiles.several ? l2_policy_evict_normal() : l2_policy_evict_first();
    uint32_t s = 0, phase = 0, fills = 0;
    bool ok = true;
    for (int g = first; g < total && ok; g += stride) {
      const ExpertTile t = expert_tile<kExpertTileN>(sh.tiles, p, g, slot);
      const int half = t.n / 2, x_row = t.row + rank * half + kTileLoadRows * lane;
      const uint32_t bytes = 2u * kExpertWBytes + (gather ? 0u : 128u * static_cast<uint32_t>(t.n));
      for (int kb = kr.begin; kb < kr.end; ++kb) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.empty_bar[s]), phase ^ 1u, abort_flag));
        if (!ok) break;
        const uint32_t w_dst = smem + s * stage_bytes, x_dst = w_dst + kExpertWBytes;
        const uint32_t full = map_to_cta(smem_u32(&sh.full_bar[s]), leader_rank);
        if (leader) {
          if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh.full_bar[s]), bytes);
          if constexpr (kSwiglu)
            tma_load_5d_pair(w_dst, &map_w, full, kb * kStepK, 0, 0, (t.m * (kExpertTileM / 2) + rank * 64) / 16, t.slot, policy);
          else
            tma_load_3d_pair(w_dst, &map_w, full, kb * kStepK, t.m * kExpertTileM + rank * 128, t.slot, policy);
        }
        __syncwarp();
        if (!gather && kTileLoadRows * lane < half)
          tma_load_rows_pair(x_dst + 128u * kTileLoadRows * lane, &map_x, full, kb * kStepK, x_row);
        __syncwarp();
        ++fills;
        if (++s == stages) { s = 0; phase ^= 1u; }
      }
    }
    if (ok) ok = take_back_stages(sh.empty_bar, s, phase, stages, abort_flag);
    if (!ok && rank == 0) {                              // given up: the copies under way end before the block does
      volatile int never = 0;
      for (uint32_t f = fills > stages ? fills - stages : 0; f < fills; ++f)
        mbar_wait(smem_u32(&sh.full_bar[f % stages]), (f / stages) & 1u, &never);
    }
  } else if (warp == 1 && rank == 0) {
    // -------------------------------------------------------------- MMAs
    const bool leader = elect_one();
    uint32_t s = 0, phase = 0, used = 0;                 // accumulators begun
    bool ok = true;
    for (int g = first; g < total && ok; g += stride) {
      const ExpertTile t = expert_tile<kExpertTileN>(sh.tiles, p, g, slot);
      const uint32_t idesc = umma_idesc_bf16_f32(256, static_cast<uint32_t>(t.n)), a = used & 1u, acc = tmem + a * kExpertTileN;
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.acc_empty[a]), ((used >> 1) & 1u) ^ 1u, abort_flag));
      if (!ok) break;
      for (int kb = kr.begin; kb < kr.end; ++kb) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.full_bar[s]), phase, abort_flag));
        if (!ok) break;
        tcgen05_fence_after();
        const uint32_t w_addr = smem + s * stage_bytes;
        const uint64_t adesc = umma_smem_desc_sw128(w_addr), bdesc = umma_smem_desc_sw128(w_addr + kExpertWBytes);
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)                 // 32 bytes of K each
            umma_bf16<2>(acc, adesc + 2u * kk, bdesc + 2u * kk, idesc, (kk != 0 || kb != kr.begin) ? 1u : 0u);
          umma_commit_pair(smem_u32(&sh.empty_bar[s]), cluster_rank);
          if (kb == kr.end - 1) umma_commit_pair(smem_u32(&sh.acc_full[a]), cluster_rank);
        }
        __syncwarp();
        if (++s == stages) { s = 0; phase ^= 1u; }
      }
      ++used;
    }
  } else if (warp == 2 && gather) {
    pass_on_rows(kr, total, first, stride, stages, sh.x_bar, abort_flag, [&](uint32_t s) { mbar_arrive_pair(smem_u32(&sh.full_bar[s]), leader_rank); });
  } else if (warp >= kExpertFirstGatherWarp) {
    if (gather)
      gather_rows(p, kr, total, first, stride, smem + kExpertWBytes, stages, stage_bytes, sh.empty_bar, sh.x_bar, abort_flag,
                                                    [&](int g, int row0, int32_t (&r)[kGatherRows]) {
        const ExpertTile t = expert_tile<kExpertTileN>(sh.tiles, p, g, slot);
#pragma unroll
        for (int i = 0; i < kGatherRows; ++i)
          r[i] = 16 * i < t.n / 2 ? expert_x_row(p, base, t, rank * (t.n / 2) + row0 + 16 * i) : kNoRow;
      });
  } else if (warp >= kExpertFirstEpilogueWarp) {
    // -------------------------------------------------------------- results
    const int quarter = warp & 3, half = (warp - kExpertFirstEpilogueWarp) >> 2;     // TMEM lanes; chunks of 32 columns half, half + 2, ..
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t staging = smem + L::kStagingAt + static_cast<uint32_t>((kSwiglu ? 2 * half : warp - kExpertFirstEpilogueWarp) * L::kBuffer);
    // matrix i of an stmatrix: columns 8 (g + i / 2) .., rows 8 (i % 2) ..; SwiGLU: 16 of the row's 64 numbers are this warp's
    const uint32_t to = staging + static_cast<uint32_t>((8 * ((lane >> 4) & 1) + (lane & 7)) * L::kRowBytes + ((lane >> 3) & 1) * 16 + (kSwiglu ? 32 * quarter : 0));
    // what a warp stores: 16 bytes per lane; SwiGLU: 8 of the 32 rows, whole lines (131072 tokens: 5.75 -> 5.67 ms, in turn on one box;
    // a warp's own 16 numbers are 32 bytes of a line); else its own 32 numbers of each row
    constexpr int kUnits = kSwiglu ? 8 : 4;              // lanes per row
    const int unit = lane % kUnits;
    uint32_t passes = 0;
    uint32_t used = 0;
    bool ok = true, met = false;
    for (int g = first; g < total && ok; g += stride) {
      const ExpertTile t = expert_tile<kExpertTileN>(sh.tiles, p, g, slot);
      const int column = (kSwiglu ? t.m * 128 + rank * 64 : t.m * 256 + rank * 128 + quarter * 32) + unit * 8;
      const uint32_t a = used & 1u;
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.acc_full[a]), (used >> 1) & 1u, abort_flag));
      if (!ok) break;
      tcgen05_fence_after();
      // split: chunk c / 32 of the tile lies at [chunk][quarter][vector of 4][lane] of the block's ring
      const uint32_t parts = smem + static_cast<uint32_t>(quarter * 4096 + lane * 16);
      if constexpr (kSplit) {
        for (int c = 32 * half; c < t.n; c += 64) {
          float u[16], l[16];
          tmem_ld_16x256b(lanes + a * kExpertTileN + c, u);
          tmem_ld_16x256b(lanes + (16u << 16) + a * kExpertTileN + c, l);
          tmem_ld_wait();
#pragma unroll
          for (int v = 0; v < 8; ++v) {
            const float* f = v < 4 ? u + 4 * v : l + 4 * (v - 4);
            st_shared_v4(parts + 512u * c + 512u * v, __float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
          }
        }
        cluster_meet();
        met = true;
      }
      for (int c = 32 * half; c < t.n; c += 64) {
        float u[16], l[16];
        if constexpr (kSplit) {
          if ((c >> 6) % p.pieces != piece) continue;
#pragma unroll
          for (int i = 0; i < 16; ++i) u[i] = l[i] = 0.0f;
          for (int from = 0; from < p.pieces; ++from) {
            const uint32_t theirs = map_to_cta(parts + 512u * c, static_cast<uint32_t>(2 * from + rank));
#pragma unroll
            for (int v = 0; v < 8; ++v) {
              const float4 w = ld_cluster_v4(theirs + 512u * v);
              float* f = v < 4 ? u + 4 * v : l + 4 * (v - 4);
              f[0] += w.x; f[1] += w.y; f[2] += w.z; f[3] += w.w;
            }
          }
        } else {
          tmem_ld_16x256b(lanes + a * kExpertTileN + c, u);
          tmem_ld_16x256b(lanes + (16u << 16) + a * kExpertTileN + c, l);
          tmem_ld_wait();
        }
        if constexpr (kSwiglu) {
#pragma unroll
          for (int i = 0; i < 16; ++i) u[i] = swiglu(u[i], l[i]);
        }
        const uint32_t buffer = kSwiglu ? (passes & 1u) * L::kBuffer : 0u;
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          stmatrix_x4_trans(to + buffer + 8u * q * L::kRowBytes, pack_bf16(u[4 * q], u[4 * q + 1]), pack_bf16(u[4 * q + 2], u[4 * q + 3]),
                            pack_bf16(u[4 * q + 4], u[4 * q + 5]), pack_bf16(u[4 * q + 6], u[4 * q + 7]));
          if constexpr (!kSwiglu)
            stmatrix_x4_trans(to + 8u * q * L::kRowBytes + 32u, pack_bf16(l[4 * q], l[4 * q + 1]), pack_bf16(l[4 * q + 2], l[4 * q + 3]),
                              pack_bf16(l[4 * q + 4], l[4 * q + 5]), pack_bf16(l[4 * q + 6], l[4 * q + 7]));
        }
        __syncwarp();
        if constexpr (kSwiglu) {
          // the four quarters' numbers; who fills a buffer again has seen all of them at the barrier of the other one
          if (lane == 0) mbar_arrive(smem_u32(&sh.rows_bar[half]));
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.rows_bar[half]), passes & 1u, abort_flag));
          if (!ok) break;
          ++passes;
        }
        constexpr int kStores = kSwiglu ? 2 : 4;
#pragma unroll
        for (int i = 0; i < kStores; ++i) {
          const int r = (kSwiglu ? 8 * quarter : 0) + i * (32 / kUnits) + lane / kUnits;
          const uint4 v = ld_shared_v4(staging + buffer + static_cast<uint32_t>(r * L::kRowBytes + unit * 16));
          if (c + r < t.valid && column < p.n_out)
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + static_cast<size_t>(t.row + c + r) * p.n_out + column) = v;
        }
        __syncwarp();
      }
      if (!ok) break;
      tcgen05_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_pair(smem_u32(&sh.acc_empty[a]), leader_rank);
      ++used;
    }
    if constexpr (kSplit)
      if (!met) cluster_meet();
  }
  if constexpr (kSplit)
    if (warp < kExpertFirstEpilogueWarp || warp >= kExpertFirstGatherWarp) cluster_meet();

  // ---------------------------------------------------------------- teardown
  tcgen05_fence_before();
  __syncthreads();
  cluster_arrive(); cluster_wait();                      // nobody leaves while the partner may still signal it
  if (threadIdx.x == 0 && sh.abort_flag) atomicCAS(p.status, 0, FB_ERR_TIMEOUT);
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_dealloc<2>(tmem, 512);
  }
}

// ---------------------------------------------------------------- rows to e4m3 with block scales
// Half a warp per block of 128 columns: a = max(max |x|, 2^-100), s = a / 448, q = x * (448 / a) rounded to e4m3.
// HBM bound: 3 bytes per number; 16384 x 7168 in 54.1 us in a graph, 6.58 TB/s (a copy: 6.53), 57 - 59 us in calls one by one.  A thread has
// kQuantizeUnroll loads of 16 bytes, of consecutive blocks, under way together.
constexpr int kQuantizeThreads = 256;
constexpr int kQuantizeUnroll = 4;

// kWhole: n is a multiple of 128, so block b is the numbers 128 b .. 128 b + 127 of x, whatever its row.
template <bool kWhole>
__global__ void __launch_bounds__(kQuantizeThreads)
fb_quantize_rows_kernel(const __nv_bfloat16* __restrict__ x, long long rows, int n, int blocks_k, uint8_t* __restrict__ q,
                        float* __restrict__ scale) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 15;
  const long long items = rows * blocks_k;
  const long long item0 = (static_cast<long long>(blockIdx.x) * (kQuantizeThreads / 16) + (threadIdx.x >> 4)) * kQuantizeUnroll;
  uint4 v[kQuantizeUnroll];
  long long at[kQuantizeUnroll];
  long long row = 0;
  int block = 0;
  if constexpr (!kWhole) {
    row = item0 / blocks_k;
    block = static_cast<int>(item0 - row * blocks_k);
  }
#pragma unroll
  for (int i = 0; i < kQuantizeUnroll; ++i) {
    if constexpr (kWhole) {
      at[i] = item0 + i < items ? (item0 + i) * 128 + lane * 8 : -1;
    } else {
      const int column = block * 128 + lane * 8;
      at[i] = (item0 + i < items && column < n) ? row * n + column : -1;
      if (++block == blocks_k) { block = 0; ++row; }
    }
    v[i] = make_uint4(0, 0, 0, 0);
    if (at[i] >= 0) v[i] = __ldcs(reinterpret_cast<const uint4*>(x + at[i]));
  }
  float scales = 0.0f;                                   // lane i keeps that of block i
#pragma unroll
  for (int i = 0; i < kQuantizeUnroll; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
    float f[8], top = 0x1p-100f;
#pragma unroll
    for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(w[j] << 16); f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (lane == i) scales = top;
    const float inv = 448.0f / top;
    uint32_t packed[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) packed[j] = pack_e4m3(f[4 * j] * inv, f[4 * j + 1] * inv, f[4 * j + 2] * inv, f[4 * j + 3] * inv);
    if (at[i] >= 0) *reinterpret_cast<uint2*>(q + at[i]) = make_uint2(packed[0], packed[1]);
  }
  if (lane < kQuantizeUnroll && item0 + lane < items) scale[item0 + lane] = scales / 448.0f;
}

// ---------------------------------------------------------------- weighted sum of a token's rows
// y[t] = sum over j of w[t][j] * rows[inv_perm[t k + j]] (+ addend[t]), j ascending, in 32 bits, rounded once.
// HBM bound: k + 1 (+ 1) rows per token; a thread has its k loads of 16 bytes under way together.  16384 tokens of 8 rows of
// 7168: 314 - 318 us, 6.7 TB/s (a copy, half of whose bytes are written: 6.53).
constexpr int kCombineThreads = 128;

template <int kK>
__global__ void __launch_bounds__(kCombineThreads)
fb_combine_kernel(const __nv_bfloat16* __restrict__ rows, const float* __restrict__ w, const int32_t* __restrict__ inv_perm, int T, int n,
                  int pieces, const __nv_bfloat16* addend, __nv_bfloat16* out, int32_t* status) {      // (addend may be out)
  pdl_wait();
  pdl_launch_dependents();
  const int t = static_cast<int>(blockIdx.x) / pieces, piece = static_cast<int>(blockIdx.x) - t * pieces;
  const int vec = piece * kCombineThreads + threadIdx.x;
  if (vec * 8 >= n) return;
  float weight[kK];
  uint4 v[kK], more = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < kK; ++j) {
    const size_t a = static_cast<size_t>(t) * kK + j;
    int pos = inv_perm[a];
    weight[j] = w[a];
    if (static_cast<unsigned>(pos) >= static_cast<unsigned>(T) * kK) {
      atomicCAS(status, 0, FB_ERR_RANGE);
      pos = 0;
    }
    v[j] = __ldcs(reinterpret_cast<const uint4*>(rows + static_cast<size_t>(pos) * n) + vec);
  }
  const size_t at = static_cast<size_t>(t) * n / 8 + vec;
  if (addend != nullptr) more = reinterpret_cast<const uint4*>(addend)[at];
  float sum[8] = {};
#pragma unroll
  for (int j = 0; j < kK; ++j) {
    const uint32_t u[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[2 * i] = fmaf(weight[j], __uint_as_float(u[i] << 16), sum[2 * i]);
      sum[2 * i + 1] = fmaf(weight[j], __uint_as_float(u[i] & 0xffff0000u), sum[2 * i + 1]);
    }
  }
  if (addend != nullptr) {
    const uint32_t u[4] = {more.x, more.y, more.z, more.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[2 * i] += __uint_as_float(u[i] << 16);
      sum[2 * i + 1] += __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  reinterpret_cast<uint4*>(out)[at] = make_uint4(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]), pack_bf16(sum[4], sum[5]),
                                                 pack_bf16(sum[6], sum[7]));
}

}  // namespace fb
