// The experts' side of a layer: products grouped by slot over the dispatch order (fb_expert_matmul), rows of 8-bit
// floats with block scales (fb_quantize_rows) and the weighted sum of a token's rows (fb_combine).
//
// fb_expert_matmul.  For the rows p of slot s (slot_offsets[s] <= p < slot_offsets[s + 1])
//     out[p] = act(x[row(p)] W_s^T),   row(p) = perm[p] / k  (or p),
// act none, or SwiGLU over W_s = [gate rows; up rows]: g / (1 + exp(-g)) * u.  With e4m3 operands the product is
//     sum over blocks b of 128 columns of  sx[row][b] * sw[i / 128][b] * (q_x[row][b] . q_w[i][b]),
// the inner products on the tensor cores, the scaled sum over the blocks in 32-bit registers.
//
// Layout of the work.  A pair of blocks (tcgen05 cta_group::2) takes tiles of 256 rows of W by up to 256 rows of x.
// The MMA's M side is W, whose size is a multiple of what a tile needs in all practice; its N side, which goes in
// steps of 32, is x, so that the ragged counts of the slots (a few rows in decode, any number in prefill) cost what
// they have, not what a tile holds: a slot with 300 rows is two tiles of 160, not two of 256.
// The blocks of a launch stay, each pair walks the tiles t, t + pairs, ...; the map from a number to (slot, rows of W,
// rows of x) is a prefix sum over the slots, made by every block from slot_offsets: nothing is handed from one launch to
// the next and no scratch is used, so calls may overlap on any streams.
//
// Warps: 0 loads (one lane W by tiles of 16 KB; every lane four gathered rows of x per copy, its row numbers in
// registers for the whole tile), 1 issues the MMAs (even block), 2-3 bring the scales (e4m3), 4-11 take the
// accumulators out: TMEM lanes are rows of W, columns rows of x; the 16x256b form of tcgen05.ld gives a thread the
// same column of lanes r and r + 16, where W's tile has its gate row r and up row r side by side (the tensor map
// interleaves them 16 by 16), so SwiGLU needs no exchange.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/freebalance.h"
#include "fb_ptx.cuh"

namespace fb {

constexpr int kExpertThreads = 384;
constexpr int kExpertEpilogueWarps = 8;
constexpr int kExpertFirstEpilogueWarp = 4;
constexpr int kExpertStages = 6;
constexpr int kExpertTileM = 256;                       // rows of W per pair
constexpr int kExpertTileN = 256;                       // rows of x per tile at most
constexpr int kExpertStepN = 32;                        // (the MMA of a pair takes N in steps of 32)
constexpr uint32_t kExpertWBytes = 128 * 128;           // a block's part of a stage: 128 rows of W ..
constexpr uint32_t kExpertStageBytes = 2 * kExpertWBytes;   // .. and up to 128 rows of x, 128 bytes each
constexpr int kScaleSlots = 4;                          // k-blocks of scales in flight
constexpr int kScaleThreads = 64;
constexpr int kBand = 8;                                // tiles of x that share a walk over W

struct ExpertParams {
  const uint32_t* slot_offsets;    // [n_slots + 1] or NULL (one slot of `rows` rows)
  const int32_t* perm;             // or NULL
  const float* x_scale;            // [x_rows][scale_k]
  const float* w_scale;            // per slot [row blocks][scale_k]
  uint64_t w_scale_slot;           // words from one slot's scales to the next
  void* out;                       // [rows][n_out]
  float* out_scale;                // [rows][ceil(n_out / 128)]
  int32_t* status;
  int32_t n_slots, k, x_rows, rows;
  int32_t num_kb;                  // steps of 128 bytes of K
  int32_t n_out;                   // columns of out
  int32_t m_blocks;                // tiles of W per slot
  int32_t scale_k;                 // ceil(K / 128)
};

struct ExpertShared {
  uint64_t full_bar[kExpertStages], empty_bar[kExpertStages];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t scale_full[kScaleSlots], scale_empty[kScaleSlots];
  uint64_t top_bar;                                     // both blocks' column maxima are there
  uint32_t tmem_base;
  int32_t abort_flag;
  int32_t warp_sums[kExpertThreads / 32];
  int32_t first_tile[FB_MAX_EXPERTS + 1];               // tiles of x before this slot's
  int32_t first_row[FB_MAX_EXPERTS];
  int32_t count[FB_MAX_EXPERTS];
};

// ---------------------------------------------------------------- copies
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1, int32_t c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void tma_load_5d_pair(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1, int32_t c2,
                                                 int32_t c3, int32_t c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
// Four rows of a matrix (a tensor map with a box one row high) one behind the other.
__device__ __forceinline__ void tma_gather4_pair(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, const int32_t (&row)[4]) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(row[0]), "r"(row[1]), "r"(row[2]), "r"(row[3])
      : "memory");
}

// ---------------------------------------------------------------- tensor cores
// e4m3 x e4m3 -> fp32, both operands K-major.
__device__ __forceinline__ uint32_t umma_idesc_e4m3_f32(uint32_t M, uint32_t N) { return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24); }
__device__ __forceinline__ void umma_e4m3_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// 16 lanes x 32 columns: register 4 g + 2 h + b of thread t is lane t / 4 + 8 h, column 8 g + 2 (t % 4) + b.
__device__ __forceinline__ void tmem_ld_16x256b_x4(uint32_t taddr, float (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(taddr)
      : "memory");
}
// (d0, d1) += (a0, a1) * (s0, s1)
__device__ __forceinline__ void fma_two(float& d0, float& d1, float a0, float a1, float s0, float s1) {
  asm("{\n.reg .b64 a, s, d;\nmov.b64 a, {%2, %3};\nmov.b64 s, {%4, %5};\nmov.b64 d, {%0, %1};\n"
      "fma.rn.f32x2 d, a, s, d;\nmov.b64 {%0, %1}, d;\n}"
      : "+f"(d0), "+f"(d1)
      : "f"(a0), "f"(a1), "f"(s0), "f"(s1));
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
__device__ __forceinline__ void st_cluster_v4(uint32_t addr, float a, float b, float c, float d) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float swiglu(float g, float u) { return __fdividef(g, 1.0f + __expf(-g)) * u; }

// ---------------------------------------------------------------- tiles
struct ExpertTile {
  int slot, m;                     // slot, tile of W
  int row, valid;                  // first row (a position counted from slot_offsets[0]) and rows of x
  int n;                           // valid rounded up to kExpertStepN: the MMA's N
};

// Tiles of x of a slot with c rows: as few as possible, all but the last of equal size.
__device__ __forceinline__ int round_up_n(int rows) { return (rows + kExpertStepN - 1) / kExpertStepN * kExpertStepN; }
__device__ __forceinline__ int expert_tile_rows(int c, int tiles) { return round_up_n((c + tiles - 1) / tiles); }
__device__ __forceinline__ int expert_tiles(int c) {
  if (c <= 0) return 0;
  const int per = expert_tile_rows(c, (c + kExpertTileN - 1) / kExpertTileN);
  return (c + per - 1) / per;
}

// All threads: the tiles of every slot.  Counts that are no prefix sums below `rows` are reported and their rows left out.
__device__ __forceinline__ void expert_plan_tiles(ExpertShared& sh, const ExpertParams& p) {
  const int e = threadIdx.x, lane = e & 31, warp = e >> 5;
  int tiles = 0;
  if (e < p.n_slots) {
    int first = 0, count = p.rows;
    if (p.slot_offsets != nullptr) {
      const uint32_t base = p.slot_offsets[0], lo = p.slot_offsets[e], hi = p.slot_offsets[e + 1];
      if (base <= lo && lo <= hi && hi - base <= static_cast<uint32_t>(p.rows)) {
        first = static_cast<int>(lo - base);
        count = static_cast<int>(hi - lo);
      } else {
        count = 0;
        atomicCAS(p.status, 0, FB_ERR_RANGE);
      }
    }
    sh.first_row[e] = first;
    sh.count[e] = count;
    tiles = expert_tiles(count);
  }
  int sum = tiles;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += v;
  }
  if (lane == 31) sh.warp_sums[warp] = sum;
  __syncthreads();
  for (int w = 0; w < warp; ++w) sum += sh.warp_sums[w];
  if (e < p.n_slots) sh.first_tile[e + 1] = sum;
  if (e == 0) sh.first_tile[0] = 0;
  __syncthreads();
}

// Tile number g: slot by slot; inside a slot bands of up to kBand tiles of x, which walk over W together (a tile of W is
// then read by the band's tiles at about the same time, and the band's rows of x stay in L2).
__device__ __forceinline__ ExpertTile expert_tile(const ExpertShared& sh, const ExpertParams& p, int g) {
  int lo = 0, hi = p.n_slots;                            // first_tile[lo] * m_blocks <= g < first_tile[hi] * m_blocks
  const int tile = g / p.m_blocks;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sh.first_tile[mid] <= tile) lo = mid; else hi = mid;
  }
  ExpertTile t;
  t.slot = lo;
  const int first = sh.first_tile[lo], tiles = sh.first_tile[lo + 1] - first;
  int r = g - first * p.m_blocks;
  const int band = r / (kBand * p.m_blocks);
  const int width = min(kBand, tiles - band * kBand);
  r -= band * kBand * p.m_blocks;
  t.m = r / width;
  const int j = band * kBand + r - t.m * width;
  const int count = sh.count[lo], per = expert_tile_rows(count, tiles);
  t.row = sh.first_row[lo] + j * per;
  t.valid = min(per, count - j * per);
  t.n = round_up_n(t.valid);
  return t;
}

// The row of x at position `row` (counted from slot_offsets[0]); rows behind a tile's last repeat that one.
__device__ __forceinline__ int expert_x_row(const ExpertParams& p, uint32_t base, const ExpertTile& t, int i) {
  const int row = t.row + min(i, t.valid - 1);
  int x = row;
  if (p.perm != nullptr) x = p.perm[static_cast<size_t>(base) + row] / p.k;
  if (static_cast<unsigned>(x) >= static_cast<unsigned>(p.x_rows)) {
    atomicCAS(p.status, 0, FB_ERR_RANGE);
    x = 0;
  }
  return x;
}

// Where column n of a tile (a row of x) lies among 256 words: a thread's eight columns of a 32-column chunk side by side.
__device__ __forceinline__ int column_word(int n) { return (n & ~31) | ((n >> 1) & 3) * 8 | ((n >> 3) & 3) * 2 | (n & 1); }

template <bool kE4m3, bool kSwiglu, bool kQuantize>
struct ExpertLayout {
  // bf16 rows of 16 (SwiGLU) or 32 numbers with a pad that keeps eight rows in different banks; e4m3 rows of 16 bytes
  static constexpr int kRowBytes = kQuantize ? 16 : kSwiglu ? 48 : 80;
  static constexpr int kWarpStaging = 32 * kRowBytes;
  static constexpr int kScaleSlotBytes = kE4m3 ? (kSwiglu ? 2 : 1) * kExpertTileN * 4 : 0;
  static constexpr int kTopBytes = kQuantize ? 8 * kExpertTileN * 4 : 0;             // one of two sets
  static constexpr uint32_t kStagingAt = kExpertStages * kExpertStageBytes;
  static constexpr uint32_t kScalesAt = kStagingAt + kExpertEpilogueWarps * kWarpStaging;
  static constexpr uint32_t kTopAt = kScalesAt + kScaleSlots * kScaleSlotBytes;
  static constexpr uint32_t kDynamic = kTopAt + 2 * kTopBytes + 1024;
};

template <bool kE4m3, bool kSwiglu, bool kQuantize>
__global__ void __launch_bounds__(kExpertThreads, 1)
fb_expert_matmul_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                        const __grid_constant__ ExpertParams p) {
  using L = ExpertLayout<kE4m3, kSwiglu, kQuantize>;
  constexpr int kStepK = kE4m3 ? 128 : 64;               // numbers of K per stage
  extern __shared__ uint8_t smem_raw[];
  __shared__ ExpertShared sh;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  volatile int* abort_flag = &sh.abort_flag;

  if (threadIdx.x == 0) {
    sh.abort_flag = 0;
    for (int s = 0; s < kExpertStages; ++s) {
      mbar_init(smem_u32(&sh.full_bar[s]), 1);
      mbar_init(smem_u32(&sh.empty_bar[s]), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(smem_u32(&sh.acc_full[a]), 1);
      mbar_init(smem_u32(&sh.acc_empty[a]), 2 * kExpertEpilogueWarps);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      mbar_init(smem_u32(&sh.scale_full[s]), kScaleThreads / 32);
      mbar_init(smem_u32(&sh.scale_empty[s]), kExpertEpilogueWarps);
    }
    mbar_init(smem_u32(&sh.top_bar), 2 * kExpertEpilogueWarps);
    fence_mbar_init();
    prefetch_tensormap(&map_x);
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
  const uint32_t tmem = sh.tmem_base;
  expert_plan_tiles(sh, p);
  const int total = sh.first_tile[p.n_slots] * p.m_blocks;
  const int stride = static_cast<int>(gridDim.x) / 2, first = static_cast<int>(blockIdx.x) / 2;
  const uint32_t base = p.slot_offsets != nullptr ? p.slot_offsets[0] : 0u;

  if (warp < kExpertFirstEpilogueWarp) {
    if constexpr (kE4m3) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) {
      // ------------------------------------------------------------ loads
      const bool leader = elect_one();
      uint32_t s = 0, phase = 0, fills = 0;
      bool ok = true;
      ExpertTile t;
      int32_t rows[4], next_rows[4];
      auto fetch = [&](int g, ExpertTile& tile, int32_t (&r)[4]) {
        if (g >= total) return;
        tile = expert_tile(sh, p, g);
        const int at = static_cast<int>(rank) * (tile.n / 2) + 4 * lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = expert_x_row(p, base, tile, at + i);
      };
      fetch(first, t, rows);
      for (int g = first; g < total && ok; g += stride) {
        ExpertTile next = t;
        const int half = t.n / 2;
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (kb == 0) fetch(g + stride, next, next_rows);        // the next tile's row numbers arrive meanwhile
          ok = __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&sh.empty_bar[s]), phase ^ 1u, abort_flag));
          if (!ok) break;
          const uint32_t w_dst = smem + s * kExpertStageBytes, x_dst = w_dst + kExpertWBytes;
          const uint32_t full = map_to_cta(smem_u32(&sh.full_bar[s]), 0u);
          if (leader) {
            if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh.full_bar[s]), 2u * kExpertWBytes + 128u * static_cast<uint32_t>(t.n));
            if constexpr (kSwiglu)
              tma_load_5d_pair(w_dst, &map_w, full, kb * kStepK, 0, 0, (t.m * (kExpertTileM / 2) + static_cast<int>(rank) * 64) / 16, t.slot);
            else
              tma_load_3d_pair(w_dst, &map_w, full, kb * kStepK, t.m * kExpertTileM + static_cast<int>(rank) * 128, t.slot);
          }
          __syncwarp();
          if (4 * lane < half) tma_gather4_pair(x_dst + 512u * lane, &map_x, full, kb * kStepK, rows);
          __syncwarp();
          ++fills;
          if (++s == kExpertStages) { s = 0; phase ^= 1u; }
        }
        t = next;
#pragma unroll
        for (int i = 0; i < 4; ++i) rows[i] = next_rows[i];
      }
      if (!ok && rank == 0) {                            // given up: the copies under way end before the block does
        volatile int never = 0;
        for (uint32_t f = fills > kExpertStages ? fills - kExpertStages : 0; f < fills; ++f)
          mbar_wait<true>(smem_u32(&sh.full_bar[f % kExpertStages]), (f / kExpertStages) & 1u, &never);
      }
    } else if (warp == 1 && rank == 0) {
      // ------------------------------------------------------------ MMAs
      const bool leader = elect_one();
      uint32_t s = 0, phase = 0, buf = 0, use = 0;
      bool ok = true;
      for (int g = first; g < total && ok; g += stride) {
        const ExpertTile t = expert_tile(sh, p, g);
        const uint32_t N = static_cast<uint32_t>(t.n);
        const uint32_t idesc = kE4m3 ? umma_idesc_e4m3_f32(256, N) : umma_idesc_bf16_f32(256, N);
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (kE4m3 || kb == 0) {                        // the accumulators' previous contents have been read out
            ok = __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&sh.acc_empty[buf]), (use & 1u) ^ 1u, abort_flag));
            if (!ok) break;
          }
          ok = __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&sh.full_bar[s]), phase, abort_flag));
          if (!ok) break;
          tcgen05_fence_after();
          const uint32_t w_addr = smem + s * kExpertStageBytes;
          const uint64_t adesc = umma_smem_desc_sw128(w_addr), bdesc = umma_smem_desc_sw128(w_addr + kExpertWBytes);
          const uint32_t acc = tmem + buf * kExpertTileN;
          const bool last = kE4m3 || kb == p.num_kb - 1;
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {             // 32 bytes of K each
              const uint32_t add = (kk != 0 || (!kE4m3 && kb != 0)) ? 1u : 0u;
              if constexpr (kE4m3) umma_e4m3_pair(acc, adesc + 2u * kk, bdesc + 2u * kk, idesc, add);
              else umma_bf16<2>(acc, adesc + 2u * kk, bdesc + 2u * kk, idesc, add);
            }
            umma_commit_pair(smem_u32(&sh.empty_bar[s]), 0u);
            if (last) umma_commit_pair(smem_u32(&sh.acc_full[buf]), 0u);
          }
          __syncwarp();
          if (last) {
            buf ^= 1u;
            if (buf == 0) ++use;
          }
          if (++s == kExpertStages) { s = 0; phase ^= 1u; }
        }
      }
    } else if (kE4m3 && warp >= 2) {
      // ------------------------------------------------------------ scales: sx[row][kb] * sw[kb] for the tile's columns
      const int at = (warp - 2) * 32 + lane;
      uint32_t slot = 0, phase = 0;
      bool ok = true;
      for (int g = first; g < total && ok; g += stride) {
        const ExpertTile t = expert_tile(sh, p, g);
        const float* xs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) xs[i] = p.x_scale + static_cast<size_t>(expert_x_row(p, base, t, at + 64 * i)) * p.scale_k;
        const float* ws = p.w_scale + static_cast<size_t>(t.slot) * p.w_scale_slot;
        const float *w0, *w1 = nullptr;
        if constexpr (kSwiglu) {                         // gate blocks, then up blocks; a tile's 64 gate rows share one
          w0 = ws + static_cast<size_t>(t.m) * p.scale_k;
          w1 = w0 + static_cast<size_t>((p.n_out + 127) / 128) * p.scale_k;
        } else {
          // (the odd block of a pair may lie behind the last row of W: its results are not stored)
          w0 = ws + static_cast<size_t>(min(2 * t.m + static_cast<int>(rank), (p.n_out + 127) / 128 - 1)) * p.scale_k;
        }
        constexpr int kAhead = 4;
        float v[4][kAhead], a[kAhead], b[kAhead];
        auto load = [&](int kb0) {
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            const int kb = min(kb0 + j, p.num_kb - 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i][j] = xs[i][kb];
            a[j] = w0[kb];
            if constexpr (kSwiglu) b[j] = w1[kb];
          }
        };
        load(0);
        for (int kb0 = 0; kb0 < p.num_kb && ok; kb0 += kAhead) {
          float cv[4][kAhead], ca[kAhead], cb[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            ca[j] = a[j];
            if constexpr (kSwiglu) cb[j] = b[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) cv[i][j] = v[i][j];
          }
          load(kb0 + kAhead);
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            if (kb0 + j < p.num_kb && ok) {
              ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.scale_empty[slot]), phase ^ 1u, abort_flag));
              if (ok) {
                const uint32_t dst = smem + L::kScalesAt + slot * L::kScaleSlotBytes;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint32_t word = dst + 4u * column_word(at + 64 * i);
                  asm volatile("st.shared.f32 [%0], %1;" ::"r"(word), "f"(cv[i][j] * ca[j]) : "memory");
                  if constexpr (kSwiglu) asm volatile("st.shared.f32 [%0], %1;" ::"r"(word + 4u * kExpertTileN), "f"(cv[i][j] * cb[j]) : "memory");
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.scale_full[slot]));
                if (++slot == kScaleSlots) { slot = 0; phase ^= 1u; }
              }
            }
          }
        }
      }
    }
  } else {
    // -------------------------------------------------------------- results
    if constexpr (kE4m3) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int quarter = warp & 3, half = (warp - kExpertFirstEpilogueWarp) >> 2;     // TMEM lanes; chunks half, half + 2, ..
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t staging = smem + L::kStagingAt + static_cast<uint32_t>(warp - kExpertFirstEpilogueWarp) * L::kWarpStaging;
    uint32_t buf = 0, use = 0, slot = 0, slot_phase = 0, tiles_done = 0;
    constexpr int kChunks = kExpertTileN / 32 / 2;       // of a warp
    bool ok = true;
    // 32 columns of the tile from (upper, lower): lanes 0-15 and 16-31 of the quarter
    auto store_bf16 = [&](const ExpertTile& t, int chunk, float (&u)[16], float (&l)[16]) {
      // matrix i of a store: columns 8 (g + i / 2) .., rows 8 (i % 2) ..
      const uint32_t to = staging + static_cast<uint32_t>((8 * ((lane >> 4) & 1) + (lane & 7)) * L::kRowBytes + ((lane >> 3) & 1) * 16);
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        stmatrix_x4_trans(to + 8u * g * L::kRowBytes, pack_bf16(u[4 * g], u[4 * g + 1]), pack_bf16(u[4 * g + 2], u[4 * g + 3]),
                          pack_bf16(u[4 * g + 4], u[4 * g + 5]), pack_bf16(u[4 * g + 6], u[4 * g + 7]));
        if constexpr (!kSwiglu)
          stmatrix_x4_trans(to + 8u * g * L::kRowBytes + 32u, pack_bf16(l[4 * g], l[4 * g + 1]), pack_bf16(l[4 * g + 2], l[4 * g + 3]),
                            pack_bf16(l[4 * g + 4], l[4 * g + 5]), pack_bf16(l[4 * g + 6], l[4 * g + 7]));
      }
      __syncwarp();
      constexpr int kUnits = kSwiglu ? 2 : 4;            // of 16 bytes per row
      const int unit = lane % kUnits;
      const int column = (kSwiglu ? t.m * 128 + static_cast<int>(rank) * 64 + quarter * 16
                                  : t.m * 256 + static_cast<int>(rank) * 128 + quarter * 32) + unit * 8;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int r = i * (32 / kUnits) + lane / kUnits;
        const uint4 v = ld_shared_v4(staging + static_cast<uint32_t>(r * L::kRowBytes + unit * 16));
        if (chunk * 32 + r < t.valid && column < p.n_out)
          *reinterpret_cast<uint4*>(out + static_cast<size_t>(t.row + chunk * 32 + r) * p.n_out + column) = v;
      }
      __syncwarp();
    };
    auto release = [&]() {                               // this warp has read the accumulators
      tcgen05_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(smem_u32(&sh.acc_empty[buf]), 0u);
      buf ^= 1u;
      if (buf == 0) ++use;
    };
    for (int g = first; g < total && ok; g += stride) {
      const ExpertTile t = expert_tile(sh, p, g);
      const int chunks = (t.n + 31) / 32;
      if constexpr (!kE4m3) {
        ok = __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&sh.acc_full[buf]), use & 1u, abort_flag));
        if (!ok) break;
        tcgen05_fence_after();
        for (int c = half; c < chunks; c += 2) {
          float u[16], l[16];
          tmem_ld_16x256b_x4(lanes + buf * kExpertTileN + 32u * c, u);
          tmem_ld_16x256b_x4(lanes + (16u << 16) + buf * kExpertTileN + 32u * c, l);
          tmem_ld_wait();
          if constexpr (kSwiglu) {
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = swiglu(u[i], l[i]);
          }
          store_bf16(t, c, u, l);
        }
        release();
      } else {
        float u[kChunks][16], l[kChunks][16];
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) u[c][i] = l[c][i] = 0.0f;
        for (int kb = 0; kb < p.num_kb; ++kb) {
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.scale_full[slot]), slot_phase, abort_flag)) &&
               __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&sh.acc_full[buf]), use & 1u, abort_flag));
          if (!ok) break;
          tcgen05_fence_after();
          const uint32_t scales = smem + L::kScalesAt + slot * L::kScaleSlotBytes + 32u * (lane & 3);
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const int chunk = 2 * c + half;
            if (chunk < chunks) {
              float tu[16], tl[16], su[8], sl[8];
              tmem_ld_16x256b_x4(lanes + buf * kExpertTileN + 32u * chunk, tu);
              tmem_ld_16x256b_x4(lanes + (16u << 16) + buf * kExpertTileN + 32u * chunk, tl);
              ld_shared_floats<8>(scales + 128u * chunk, su);
              if constexpr (kSwiglu) ld_shared_floats<8>(scales + 4u * kExpertTileN + 128u * chunk, sl);
              tmem_ld_wait();
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const float s0 = kSwiglu ? sl[2 * q] : su[2 * q], s1 = kSwiglu ? sl[2 * q + 1] : su[2 * q + 1];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const int i = 4 * q + 2 * h;
                  fma_two(u[c][i], u[c][i + 1], tu[i], tu[i + 1], su[2 * q], su[2 * q + 1]);
                  fma_two(l[c][i], l[c][i + 1], tl[i], tl[i + 1], s0, s1);
                }
              }
            }
          }
          release();
          if (lane == 0) mbar_arrive(smem_u32(&sh.scale_empty[slot]));
          if (++slot == kScaleSlots) { slot = 0; slot_phase ^= 1u; }
        }
        if (!ok) break;
        if constexpr (kSwiglu) {
#pragma unroll
          for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) u[c][i] = swiglu(u[c][i], l[c][i]);
        }
        if constexpr (!kQuantize) {
#pragma unroll
          for (int c = 0; c < kChunks; ++c)
            if (2 * c + half < chunks) store_bf16(t, 2 * c + half, u[c], l[c]);
        } else {
          // The largest of a row's 128 outputs: 16 here, by shuffles; the four quarters' and the two blocks' through both
          // blocks' shared memory, in two sets in turn (a warp writes a set again after all warps have passed the other).
          // Rows of W behind the last one are zeros, so their outputs are and change no maximum.
          const uint32_t set = smem + L::kTopAt + (tiles_done & 1u) * L::kTopBytes;
          const uint32_t mine = set + 4u * kExpertTileN * (4u * rank + quarter) + 32u * (lane & 3);
          const uint32_t theirs = map_to_cta(mine, rank ^ 1u);
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const int chunk = 2 * c + half;
            if (chunk < chunks) {
              float top[8];
#pragma unroll
              for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  float m = fmaxf(fabsf(u[c][4 * q + b]), fabsf(u[c][4 * q + 2 + b]));
                  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                  top[2 * q + b] = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                }
              if (lane < 4) {
                st_cluster_v4(map_to_cta(mine, rank) + 128u * chunk, top[0], top[1], top[2], top[3]);
                st_cluster_v4(map_to_cta(mine, rank) + 128u * chunk + 16u, top[4], top[5], top[6], top[7]);
                st_cluster_v4(theirs + 128u * chunk, top[0], top[1], top[2], top[3]);
                st_cluster_v4(theirs + 128u * chunk + 16u, top[4], top[5], top[6], top[7]);
              }
            }
          }
          asm volatile("fence.acq_rel.cluster;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive_cluster(smem_u32(&sh.top_bar), 0u);
            mbar_arrive_cluster(smem_u32(&sh.top_bar), 1u);
          }
          ok = __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&sh.top_bar), tiles_done & 1u, abort_flag));
          if (!ok) break;
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const int chunk = 2 * c + half;
            if (chunk < chunks) {
              float top[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) top[i] = 0x1p-100f;       // smallest scale: see fb_quantize_rows
#pragma unroll
              for (int w = 0; w < 8; ++w) {
                float v[8];
                ld_shared_floats<8>(set + 4u * kExpertTileN * w + 128u * chunk + 32u * (lane & 3), v);
#pragma unroll
                for (int i = 0; i < 8; ++i) top[i] = fmaxf(top[i], v[i]);
              }
#pragma unroll
              for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  const int r = 8 * q + 2 * (lane & 3) + b;          // row of x within the chunk
                  const float m = top[2 * q + b], inv = 448.0f / m;
                  if (rank == 0 && quarter == 0 && lane < 4 && chunk * 32 + r < t.valid)
                    p.out_scale[static_cast<size_t>(t.row + chunk * 32 + r) * ((p.n_out + 127) / 128) + t.m] = m / 448.0f;
                  const __nv_fp8x2_storage_t two = __nv_cvt_float2_to_fp8x2(
                      make_float2(u[c][4 * q + b] * inv, u[c][4 * q + 2 + b] * inv), __NV_SATFINITE, __NV_E4M3);
                  const uint32_t to = staging + static_cast<uint32_t>(r * L::kRowBytes + (lane >> 2));
                  asm volatile("st.shared.u8 [%0], %1;" ::"r"(to), "r"(static_cast<uint32_t>(two) & 0xffu) : "memory");
                  asm volatile("st.shared.u8 [%0], %1;" ::"r"(to + 8u), "r"(static_cast<uint32_t>(two) >> 8) : "memory");
                }
              __syncwarp();
              const uint4 v = ld_shared_v4(staging + static_cast<uint32_t>(lane * L::kRowBytes));
              const int column = t.m * 128 + static_cast<int>(rank) * 64 + quarter * 16;
              if (chunk * 32 + lane < t.valid && column < p.n_out)
                *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.out) + static_cast<size_t>(t.row + chunk * 32 + lane) * p.n_out + column) = v;
              __syncwarp();
            }
          }
        }
      }
      ++tiles_done;
    }
  }

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
// HBM bound: 3 bytes per number.
constexpr int kQuantizeThreads = 256;
constexpr int kQuantizeUnroll = 4;

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
#pragma unroll
  for (int i = 0; i < kQuantizeUnroll; ++i) {
    const long long item = item0 + i, row = item / blocks_k;
    const int column = static_cast<int>(item - row * blocks_k) * 128 + lane * 8;
    at[i] = (item < items && column < n) ? row * n + column : -1;
    v[i] = make_uint4(0, 0, 0, 0);
    if (at[i] >= 0) v[i] = __ldcs(reinterpret_cast<const uint4*>(x + at[i]));
  }
#pragma unroll
  for (int i = 0; i < kQuantizeUnroll; ++i) {
    float f[8];
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(w[j] << 16); f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
    float top = 0x1p-100f;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float inv = 448.0f / top;
    uint32_t packed[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * j] * inv, f[4 * j + 1] * inv), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * j + 2] * inv, f[4 * j + 3] * inv), __NV_SATFINITE, __NV_E4M3);
      packed[j] = lo | hi << 16;
    }
    if (at[i] >= 0) *reinterpret_cast<uint2*>(q + at[i]) = make_uint2(packed[0], packed[1]);
    if (lane == 0 && item0 + i < items) scale[item0 + i] = top / 448.0f;
  }
}

// ---------------------------------------------------------------- weighted sum of a token's rows
// y[t] = sum over j of w[t][j] * rows[inv_perm[t k + j]] (+ addend[t]), j ascending, in 32 bits, rounded once.
// HBM bound: k + 1 (+ 1) rows per token; a thread has its k loads of 16 bytes under way together.
constexpr int kCombineThreads = 128;

template <int kK>
__global__ void __launch_bounds__(kCombineThreads)
fb_combine_kernel(const __nv_bfloat16* __restrict__ rows, const float* __restrict__ w, const int32_t* __restrict__ inv_perm, int T, int n,
                  int pieces, const __nv_bfloat16* __restrict__ addend, __nv_bfloat16* __restrict__ out, int32_t* status) {
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
