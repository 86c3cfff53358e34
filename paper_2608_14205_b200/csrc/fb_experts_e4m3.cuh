// fb_expert_matmul with e4m3 operands and block scales: for every row p of slot s
//     out[p][i] = act(sum over blocks b of 128 columns of  sx[row(p)][b] * sw_s[i / 128][b] * (q_x[row(p)][b] . q_w[i][b])).
// The inner product of a block is a k-block of MMAs (tcgen05 kind::f8f6f4) with an accumulator of its own; the scaled sum
// over the blocks is held in 32-bit registers, 128 rows x 256 columns in those of eight warps.
//
// Here the MMA's M side is x (128 rows) and its N side W (256 rows, with SwiGLU 16 of gate and 16 of up in turn): a TMEM
// lane is a row of x, so a thread of the results warps has one row, whose scale is a register, and 128 rows of W, which
// share one scale (with SwiGLU two).  The other way round - W on the M side in pairs of blocks, as for bf16, where counts
// that are no multiple of the tile cost less - every column has a scale of its own, which each warp has to read from
// shared memory for every k-block; that, tcgen05.ld in its 16-lane form and the way over two blocks at each hand-over took
// 880 cycles per k-block whose MMAs take 512.
//
// kPair: two blocks (cta_group::2) take 256 rows of x by 256 of W, each with its 128 rows of x and half of the rows of W
// in its shared memory; else one block takes 128 x 256.  The pair brings 32 KB into an SM per k-block, the single block
// 48 KB; the single block's tiles fit counts better that are no multiple of 256 (the rule is in fb_expert_matmul).
//
// One block per SM.  Warps: 0 loads by TMA, 1 issues the MMAs, 2 passes on that gathered rows are there, 4-11 add up and store, 12-15 gather rows of x.  Two
// accumulators of 256 columns: the MMAs fill one while the other is added up.
#pragma once
#include "fb_experts.cuh"

namespace fb {

constexpr uint32_t kE4m3XBytes = 128 * 128;             // a block's rows of x in a stage
constexpr uint32_t kE4m3WarpStaging = 32 * 64;          // 32 rows of 64 bytes, or 16 of 128
template <bool kPair>
struct ExpertE4m3Layout {
  static constexpr int kRows = kPair ? 256 : 128;       // of x per tile
  static constexpr int kStages = kPair ? 6 : 4;
  static constexpr uint32_t kWBytes = (kPair ? 128 : 256) * 128;        // a block's rows of W in a stage
  static constexpr uint32_t kStageBytes = kE4m3XBytes + kWBytes;
  static constexpr uint32_t kStagingAt = kStages * kStageBytes;
  static constexpr uint32_t kDynamic = kStagingAt + kExpertEpilogueWarps * kE4m3WarpStaging + 1024;
};
constexpr int kE4m3Ahead = 4;                           // k-blocks whose scales are on their way

struct ExpertE4m3Shared {
  uint64_t full_bar[6], empty_bar[6], x_bar[6];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t top_bar[4];                                  // per quarter: its two warps' maxima are there
  uint32_t tmem_base;
  int32_t abort_flag;
  float top[2][2][128];                                 // in turn; per half of the columns: a row's largest output
  ExpertTiles tiles;
};

__device__ __forceinline__ void tma_load_rows(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1)
               : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1, int32_t c2, uint64_t policy) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1, int32_t c2, int32_t c3, int32_t c4, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5, %6, %7}], [%2], %8;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "l"(policy)
      : "memory");
}
// e4m3 x e4m3 -> fp32, both operands K-major.
__device__ __forceinline__ uint32_t umma_idesc_e4m3_f32(uint32_t M, uint32_t N) { return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24); }
template <int kCtaGroup>
__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (kCtaGroup == 1)
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_d),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_d),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void umma_commit_one(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// (d0, d1) += (a0, a1) * s
__device__ __forceinline__ void fma_two(float& d0, float& d1, uint32_t a0, uint32_t a1, float s) {
  asm("{\n.reg .b64 a, s, d;\nmov.b64 a, {%2, %3};\nmov.b64 s, {%4, %4};\nmov.b64 d, {%0, %1};\n"
      "fma.rn.f32x2 d, a, s, d;\nmov.b64 {%0, %1}, d;\n}"
      : "+f"(d0), "+f"(d1)
      : "r"(a0), "r"(a1), "f"(s));
}
// What a k-block takes (cycles; 8192 x 8192 x 8192): its MMAs 516, with the hand-overs of the accumulators 588, with the loads
// 660, with the read-out of TMEM 666, with the multiply-adds 805 - the chain wait, read, add, release of the eight warps, whose pipe
// is 32 % busy.  Up projection with SwiGLU and quantised results, 256 experts of 7168 x 2048: 16384 tokens 4.3 ms (1796 TFLOP/s)
// in short runs, 4.9 - 5.25 ms at 1000 W; 64 tokens 900 us, 6.6 TB/s (a copy: 6.53), and 961 - 1034 us at 1000 W.
template <bool kPair, bool kSwiglu, bool kQuantize, bool kSplit>
__global__ void __launch_bounds__(kExpertThreads, 1)
fb_expert_matmul_e4m3_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                             const __grid_constant__ ExpertParams p) {
  static_assert(!(kPair && kSplit), "a call of few tiles has no pairs");
  using L = ExpertE4m3Layout<kPair>;
  constexpr int kGroup = kPair ? 2 : 1;                  // blocks per tile
  extern __shared__ uint8_t smem_raw[];
  __shared__ ExpertE4m3Shared sh;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  const int lane = threadIdx.x & 31;
  const int rank = kPair ? static_cast<int>(cluster_ctarank()) : 0;
  const int piece = kSplit ? static_cast<int>(cluster_ctarank()) : 0;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  volatile int* abort_flag = &sh.abort_flag;
  const bool gather = p.perm != nullptr;

  if (threadIdx.x == 0) {
    sh.abort_flag = 0;
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(smem_u32(&sh.full_bar[s]), gather ? 1 + kGroup : 1);    // the TMA loads; each block's gathered rows
      mbar_init(smem_u32(&sh.empty_bar[s]), 1);
      mbar_init(smem_u32(&sh.x_bar[s]), 33 * kGatherWarps);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(smem_u32(&sh.acc_full[a]), 1);
      mbar_init(smem_u32(&sh.acc_empty[a]), kGroup * kExpertEpilogueWarps);
    }
    for (int q = 0; q < 4; ++q) mbar_init(smem_u32(&sh.top_bar[q]), 2);
    fence_mbar_init();
    if (!gather) prefetch_tensormap(&map_x);
    prefetch_tensormap(&map_w);
  }
  if (warp == 1) {
    tmem_alloc<kGroup>(smem_u32(&sh.tmem_base), 512);
    tmem_relinquish<kGroup>();
  }
  tcgen05_fence_before();
  __syncthreads();
  if constexpr (kPair) { cluster_arrive_relaxed(); cluster_wait(); }      // the partner's barriers and tensor memory are ready too
  tcgen05_fence_after();
  pdl_wait();
  pdl_launch_dependents();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem_base, 0);      // (warp-uniform for the compiler as well)
  uint32_t base;
  int slot = 0;                                          // of the warp's last tile
  const int total = expert_plan_tiles<L::kRows>(sh.tiles, p, base);
  const int sharers = kSplit ? p.pieces : kGroup;        // blocks per tile
  const int stride = static_cast<int>(gridDim.x) / sharers, first = static_cast<int>(blockIdx.x) / sharers;
  const KRange kr = kSplit ? k_range(p, piece) : KRange{0, p.num_kb};

  // Registers: 256 threads with 208 and 256 with 48 are the 512 x 128 of the launch.
  if (warp < kExpertFirstEpilogueWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 0) {
      // ------------------------------------------------------------ TMA loads
      const bool leader = elect_one();
      const uint64_t policy = sh.tiles.several ? l2_policy_evict_normal() : l2_policy_evict_first();
      uint32_t s = 0, phase = 0, fills = 0;
      bool ok = true;
      for (int g = first; g < total && ok; g += stride) {
        const ExpertTile t = expert_tile<L::kRows>(sh.tiles, p, g, slot);
        // (loads without a row of the tile begin behind the last row of x and give zeros)
        const int i = rank * 128 + kTileLoadRows * lane, x_row = i < t.valid ? t.row + i : p.x_rows;
        const uint32_t bytes = kGroup * (L::kWBytes + (gather ? 0u : kE4m3XBytes));
        for (int kb = kr.begin; kb < kr.end; ++kb) {
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.empty_bar[s]), phase ^ 1u, abort_flag));
          if (!ok) break;
          const uint32_t x_dst = smem + s * L::kStageBytes, w_dst = x_dst + kE4m3XBytes;
          const uint32_t full = kPair ? map_to_cta(smem_u32(&sh.full_bar[s]), 0u) : smem_u32(&sh.full_bar[s]);
          if (leader) {
            if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh.full_bar[s]), bytes);
            if constexpr (kSwiglu) {
              const int w_group = t.m * (kExpertTileM / 2 / 16) + rank * 4;      // of 16 outputs
              if constexpr (kPair) tma_load_5d_pair(w_dst, &map_w, full, kb * 128, 0, 0, w_group, t.slot, policy);
              else tma_load_5d(w_dst, &map_w, full, kb * 128, 0, 0, w_group, t.slot, policy);
            } else {
              const int w_row = t.m * kExpertTileM + rank * 128;
              if constexpr (kPair) tma_load_3d_pair(w_dst, &map_w, full, kb * 128, w_row, t.slot, policy);
              else tma_load_3d(w_dst, &map_w, full, kb * 128, w_row, t.slot, policy);
            }
          }
          __syncwarp();
          if (!gather && lane < 128 / kTileLoadRows) {
            if constexpr (kPair) tma_load_rows_pair(x_dst + 128u * kTileLoadRows * lane, &map_x, full, kb * 128, x_row);
            else tma_load_rows(x_dst + 128u * kTileLoadRows * lane, &map_x, full, kb * 128, x_row);
          }
          __syncwarp();
          ++fills;
          if (++s == L::kStages) { s = 0; phase ^= 1u; }
        }
      }
      if (ok) ok = take_back_stages(sh.empty_bar, s, phase, L::kStages, abort_flag);
      if (!ok && rank == 0) {                            // given up: the copies under way end before the block does
        volatile int never = 0;
        for (uint32_t f = fills > L::kStages ? fills - L::kStages : 0; f < fills; ++f)
          mbar_wait(smem_u32(&sh.full_bar[f % L::kStages]), (f / L::kStages) & 1u, &never);
      }
    } else if (warp == 1 && rank == 0) {
      // ------------------------------------------------------------ MMAs
      const bool leader = elect_one();
      const uint32_t idesc = umma_idesc_e4m3_f32(128 * kGroup, 256);
      uint32_t s = 0, phase = 0, used = 0;               // accumulators begun
      bool ok = true;
      for (int g = first; g < total && ok; g += stride) {
        for (int kb = kr.begin; kb < kr.end; ++kb) {
          const uint32_t a = used & 1u, acc = tmem + a * 256u;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.full_bar[s]), phase, abort_flag));
          if (ok) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.acc_empty[a]), ((used >> 1) & 1u) ^ 1u, abort_flag));
          if (!ok) break;
          tcgen05_fence_after();
          const uint32_t x_addr = smem + s * L::kStageBytes;
          const uint64_t adesc = umma_smem_desc_sw128(x_addr), bdesc = umma_smem_desc_sw128(x_addr + kE4m3XBytes);
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) umma_e4m3<kGroup>(acc, adesc + 2u * kk, bdesc + 2u * kk, idesc, kk != 0 ? 1u : 0u);      // 32 of K each
            if constexpr (kPair) {
              umma_commit_pair(smem_u32(&sh.acc_full[a]), 0u);
              umma_commit_pair(smem_u32(&sh.empty_bar[s]), 0u);
            } else {
              umma_commit_one(smem_u32(&sh.acc_full[a]));
              umma_commit_one(smem_u32(&sh.empty_bar[s]));
            }
          }
          __syncwarp();
          ++used;
          if (++s == L::kStages) { s = 0; phase ^= 1u; }
        }
      }
    } else if (warp == 2 && gather) {
      pass_on_rows(kr, total, first, stride, L::kStages, sh.x_bar, abort_flag, [&](uint32_t s) {
        if constexpr (kPair) mbar_arrive_pair(smem_u32(&sh.full_bar[s]), 0u);
        else mbar_arrive(smem_u32(&sh.full_bar[s]));
      });
    }
  } else if (warp >= kExpertFirstGatherWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (gather)
      gather_rows(p, kr, total, first, stride, smem, L::kStages, L::kStageBytes, sh.empty_bar, sh.x_bar, abort_flag,
                                                [&](int g, int row0, int32_t (&r)[kGatherRows]) {
        const ExpertTile t = expert_tile<L::kRows>(sh.tiles, p, g, slot);
#pragma unroll
        for (int i = 0; i < kGatherRows; ++i) r[i] = expert_x_row(p, base, t, rank * 128 + row0 + 16 * i);
      });
  } else {
    // -------------------------------------------------------------- sums and results
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int quarter = warp & 3, half = (warp - kExpertFirstEpilogueWarp) >> 2;     // TMEM lanes (rows of x); 128 columns each
    const int row0 = rank * 128 + quarter * 32, row = row0 + lane;      // of the tile
    const uint32_t from = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + 128u * half;
    const uint32_t staging = smem + L::kStagingAt + static_cast<uint32_t>(warp - kExpertFirstEpilogueWarp) * kE4m3WarpStaging;
    uint32_t used = 0, tiles_done = 0;
    bool ok = true, met = false;
    // scales of the next k-blocks: this thread's row, and the blocks of W (gate and up; or this half's)
    const float *xs = nullptr, *w0 = nullptr, *w1 = nullptr;
    float v[kE4m3Ahead], a0[kE4m3Ahead], a1[kE4m3Ahead];
    auto load = [&](int j, int kb) {
      kb = min(kb, p.num_kb - 1);
      v[j] = xs[kb];
      a0[j] = w0[kb];
      if constexpr (kSwiglu) a1[j] = w1[kb];
    };
    auto begin = [&](const ExpertTile& t) {
      xs = p.x_scale + static_cast<size_t>(max(expert_x_row(p, base, t, row), 0)) * p.scale_k;
      const float* ws = p.w_scale + static_cast<size_t>(t.slot) * p.w_scale_slot;
      const int blocks = (p.n_out + 127) / 128;          // (the second half of a tile may lie behind the last row of W: not stored)
      w0 = ws + static_cast<size_t>(kSwiglu ? t.m : min(2 * t.m + half, blocks - 1)) * p.scale_k;
      if constexpr (kSwiglu) w1 = w0 + static_cast<size_t>(blocks) * p.scale_k;
#pragma unroll
      for (int j = 0; j < kE4m3Ahead; ++j) load(j, kr.begin + j);
    };
    // 64 bytes of each of the warp's 32 rows (64 results in e4m3)
    auto store_bytes = [&](const ExpertTile& t, int column, const uint32_t (&value)[16]) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        st_shared_v4(staging + static_cast<uint32_t>(lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)), value[4 * i], value[4 * i + 1],
                     value[4 * i + 2], value[4 * i + 3]);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2), unit = lane & 3;
        const uint4 w = ld_shared_v4(staging + static_cast<uint32_t>(r * 64 + ((unit ^ ((r >> 1) & 3)) << 4)));
        if (row0 + r < t.valid && column + 16 * unit < p.n_out)
          *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.out) + static_cast<size_t>(t.row + row0 + r) * p.n_out + column + 16 * unit) = w;
      }
      __syncwarp();
    };
    // 128 bytes of each row (64 results in bf16), 16 rows at a time: whole lines leave the SM.  (Down projection of 5003 tokens,
    // 256 experts of 2048 x 7168, at 1000 W, in turn on the coolest box: 1037 us; 64 bytes of 32 rows at a time 1090; straight from
    // the registers 1215.  On two other boxes it takes 1149 and 1162.)
    auto store_wide = [&](const ExpertTile& t, int column, const uint32_t (&value)[32]) {
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        if ((lane >> 4) == part) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            st_shared_v4(staging + static_cast<uint32_t>((lane & 15) * 128 + ((i ^ (lane & 7)) << 4)), value[4 * i], value[4 * i + 1], value[4 * i + 2], value[4 * i + 3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * i + (lane >> 3), unit = lane & 7, in_tile = row0 + 16 * part + r;
          const uint4 w = ld_shared_v4(staging + static_cast<uint32_t>(r * 128 + ((unit ^ (r & 7)) << 4)));
          if (in_tile < t.valid && column + 8 * unit < p.n_out)
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + static_cast<size_t>(t.row + in_tile) * p.n_out + column + 8 * unit) = w;
        }
        __syncwarp();
      }
    };
    auto release = [&](uint32_t a) {                     // this warp has read the accumulator
      tcgen05_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (kPair) mbar_arrive_pair(smem_u32(&sh.acc_empty[a]), 0u);
        else mbar_arrive(smem_u32(&sh.acc_empty[a]));
      }
    };
    ExpertTile t;
    if (first < total) {
      t = expert_tile<L::kRows>(sh.tiles, p, first, slot);
      begin(t);
    }
    for (int g = first; g < total && ok; g += stride) {
      float acc[128];                                    // SwiGLU: 16 gate, 16 up, ..
#pragma unroll
      for (int i = 0; i < 128; ++i) acc[i] = 0.0f;
      const bool any = row0 < t.valid;           // this warp has rows of x here
      for (int kb = any ? kr.end : kr.begin; kb < kr.end && ok; ++kb, ++used) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.acc_full[used & 1u]), (used >> 1) & 1u, abort_flag));
        if (ok) release(used & 1u);
      }
      for (int kb0 = any ? kr.begin : kr.end; kb0 < kr.end && ok; kb0 += kE4m3Ahead) {
#pragma unroll
        for (int j = 0; j < kE4m3Ahead; ++j) {
          if (kb0 + j >= kr.end || !ok) break;
          const float s0 = v[j] * a0[j], s1 = kSwiglu ? v[j] * a1[j] : s0;
          load(j, kb0 + j + kE4m3Ahead);
          const uint32_t a = used & 1u;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.acc_full[a]), (used >> 1) & 1u, abort_flag));
          if (!ok) break;
          tcgen05_fence_after();
          // 32 and 16 columns in turn are added while the next ones are on their way
          uint32_t wide[32], narrow[16];
          auto add = [&](int c, const uint32_t* r, int n) {
#pragma unroll
            for (int i = 0; i < 32; i += 2)
              if (i < n) fma_two(acc[c + i], acc[c + i + 1], r[i], r[i + 1], ((c + i) & 16) == 0 ? s0 : s1);
          };
          const uint32_t at = from + 256u * a;
          tmem_ld_32x32b_x32(at, wide);
          tmem_ld_wait();
          tmem_ld_32x32b_x16(at + 32u, narrow);
          add(0, wide, 32);
          tmem_ld_wait();
          tmem_ld_32x32b_x32(at + 48u, wide);
          add(32, narrow, 16);
          tmem_ld_wait();
          tmem_ld_32x32b_x16(at + 80u, narrow);
          add(48, wide, 32);
          tmem_ld_wait();
          tmem_ld_32x32b_x32(at + 96u, wide);
          add(80, narrow, 16);
          tmem_ld_wait();
          release(a);
          add(96, wide, 32);
          ++used;
        }
      }
      if (!ok) break;
      if constexpr (kSplit) {                            // (a split launch has one tile per cluster)
        // The sums of row `lane` lie at [warp][vector v of 4 columns][lane] of the ring.  A block adds up 32 / pieces rows of each
        // quarter; in a warp `pieces` lanes share such a row, each `share` vectors of its results (SwiGLU: gate and up of them).
        constexpr uint32_t kVector = 512 + 16;           // (the pad keeps the sharers of a row in different banks)
        const uint32_t parts = smem + static_cast<uint32_t>(warp - kExpertFirstEpilogueWarp) * 32u * kVector;
        if (any) {
#pragma unroll
          for (int v = 0; v < 32; ++v)
            st_shared_v4(parts + kVector * v + 16u * lane, __float_as_uint(acc[4 * v]), __float_as_uint(acc[4 * v + 1]),
                         __float_as_uint(acc[4 * v + 2]), __float_as_uint(acc[4 * v + 3]));
        }
        cluster_meet();
        met = true;
        constexpr int kVectors = kSwiglu ? 16 : 32;      // of results in this half of the columns
        const int rows = 32 / p.pieces, mine = piece * rows + lane % rows, share = kVectors / p.pieces, v0 = lane / rows * share;
        const bool stored = row0 + mine < t.valid;
        float a[kVectors / 2][4], b[kSwiglu ? kVectors / 2 : 1][4];
#pragma unroll
        for (int i = 0; i < kVectors / 2; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) { a[i][c] = 0.0f; if constexpr (kSwiglu) b[i][c] = 0.0f; }
        if (stored) {
          for (int from = 0; from < p.pieces; ++from) {
            const uint32_t theirs = map_to_cta(parts, static_cast<uint32_t>(from)) + 16u * mine;
#pragma unroll
            for (int i = 0; i < kVectors / 2; ++i) {
              if (i < share) {
                const int q = v0 + i, v = kSwiglu ? (q >> 2) * 8 + (q & 3) : q;
                const float4 x = ld_cluster_v4(theirs + kVector * v);
                a[i][0] += x.x; a[i][1] += x.y; a[i][2] += x.z; a[i][3] += x.w;
                if constexpr (kSwiglu) {
                  const float4 y = ld_cluster_v4(theirs + kVector * (v + 4));
                  b[i][0] += y.x; b[i][1] += y.y; b[i][2] += y.z; b[i][3] += y.w;
                }
              }
            }
          }
        }
        if constexpr (kSwiglu) {
#pragma unroll
          for (int i = 0; i < kVectors / 2; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) a[i][c] = swiglu(a[i][c], b[i][c]);
        }
        const size_t at = static_cast<size_t>(t.row + row0 + mine);
        const int column = t.m * (kSwiglu ? 128 : 256) + half * 4 * kVectors + 4 * v0;
        float inv = 0.0f;
        if constexpr (kQuantize) {
          float top = 0x1p-100f;
#pragma unroll
          for (int i = 0; i < kVectors / 2; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) top = fmaxf(top, fabsf(a[i][c]));      // (zeros where i >= share)
          for (int d = rows; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          if (lane < rows) sh.top[0][half][quarter * 32 + lane] = top;
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sh.top_bar[quarter]));
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.top_bar[quarter]), 0u, abort_flag));
          if (!ok) break;
          top = fmaxf(top, sh.top[0][half ^ 1][quarter * 32 + lane % rows]);
          inv = 448.0f / top;
          if (stored && half == 0 && lane < rows) p.out_scale[at * ((p.n_out + 127) / 128) + t.m] = top / 448.0f;
        }
#pragma unroll
        for (int i = 0; i < kVectors / 2; ++i) {
          const int c = column + 4 * i;
          if (i < share && stored && c < p.n_out) {
            if constexpr (kQuantize)
              *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p.out) + at * p.n_out + c) =
                  pack_e4m3(a[i][0] * inv, a[i][1] * inv, a[i][2] * inv, a[i][3] * inv);
            else
              *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at * p.n_out + c) =
                  make_uint2(pack_bf16(a[i][0], a[i][1]), pack_bf16(a[i][2], a[i][3]));
          }
        }
        break;
      }
      const ExpertTile done = t;
      if (g + stride < total) {                          // the next tile's first scales arrive under the stores
        t = expert_tile<L::kRows>(sh.tiles, p, g + stride, slot);
        begin(t);
      }
      if constexpr (kSwiglu) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[16 * c + i] = swiglu(acc[32 * c + i], acc[32 * c + 16 + i]);
      }
      if constexpr (!kQuantize) {
        constexpr int kPasses = kSwiglu ? 1 : 2;         // of 64 columns
#pragma unroll
        for (int c = 0; c < kPasses; ++c) {
          uint32_t value[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) value[i] = pack_bf16(acc[64 * c + 2 * i], acc[64 * c + 2 * i + 1]);
          store_wide(done, done.m * 128 * kPasses + half * 64 * kPasses + 64 * c, value);
        }
      } else {
        uint32_t value[16];
        // A row's 128 outputs are in the two warps of its quarter.  Two sets in turn: who writes a set again has seen the
        // other warp at the barrier of the set between.
        float top = 0x1p-100f;                           // smallest scale: see fb_quantize_rows
#pragma unroll
        for (int i = 0; i < 64; ++i) top = fmaxf(top, fabsf(acc[i]));
        float (&tops)[2][128] = sh.top[tiles_done & 1u];
        tops[half][quarter * 32 + lane] = top;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.top_bar[quarter]));
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.top_bar[quarter]), tiles_done & 1u, abort_flag));
        if (!ok) break;
        top = fmaxf(top, tops[half ^ 1][quarter * 32 + lane]);
        const float inv = 448.0f / top;
        if (half == 0 && row < done.valid) p.out_scale[static_cast<size_t>(done.row + row) * ((p.n_out + 127) / 128) + done.m] = top / 448.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) value[i] = pack_e4m3(acc[4 * i] * inv, acc[4 * i + 1] * inv, acc[4 * i + 2] * inv, acc[4 * i + 3] * inv);
        store_bytes(done, done.m * 128 + half * 64, value);
      }
      ++tiles_done;
    }
    if constexpr (kSplit)
      if (!met) cluster_meet();
  }
  if constexpr (kSplit)
    if (warp < kExpertFirstEpilogueWarp || warp >= kExpertFirstGatherWarp) cluster_meet();

  // ---------------------------------------------------------------- teardown
  tcgen05_fence_before();
  __syncthreads();
  if constexpr (kPair || kSplit) { cluster_arrive(); cluster_wait(); }    // nobody leaves while another may still signal it or read its sums
  if (threadIdx.x == 0 && sh.abort_flag) atomicCAS(p.status, 0, FB_ERR_TIMEOUT);
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_dealloc<kGroup>(tmem, 512);
  }
}

}  // namespace fb
