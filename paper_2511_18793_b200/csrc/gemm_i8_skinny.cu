// C = A W^T of 8-bit integers for at most 128 rows: the weight-streaming form (see gemm_skinny.cu), bound by reading W once.
// 128 rows of W are the MMA's 128-row operand and the rows of A its N (MT = 32, 64 or 128); an output tile is 128 columns of C.  The K range of a
// tile is split over the CTAs of a cluster so that every SM streams a share of W.  Each CTA leaves its 32-bit sums in its own shared memory, where
// the ring was; behind a cluster barrier the rows of the tile are dealt out to the warps of the cluster, which add the parts (whole
// numbers: in any order the same) and store 128 neighbouring elements per row.  20 x 16,384 x 2,048: 11.5 us from HBM (W alone 5.3 at the copy's rate),
// 5.8 from a warm L2.  Its 128 tiles are a CTA each, so nothing is split or joined: 20 of the SMs have none, and the others have a ring of 100 KB, of which
// 80 are W, because two CTAs per SM have to have room.
#include "gemm_i8.cuh"

namespace nz {

int sm_count();

namespace {

using namespace gemm_detail;
using namespace i8_detail;

template <int MT> struct SkCfg {
  static constexpr int kTileW = 128 * kStepK, kTileX = MT * kStepK, kStage = kTileW + kTileX;
  static constexpr int kStages = MT == 32 ? 5 : MT == 64 ? 4 : 3;
  static constexpr int kBar = 192;
  static constexpr int kSmem = kStages * kStage + 1024 + kBar;
  static constexpr int kTmemCols = MT;
  static_assert(MT * 128 * 4 <= kStages * kStage, "the sums do not fit in the ring");
  static_assert(2 * (kSmem + 1024) <= 228 * 1024, "two CTAs per SM");
};
constexpr int kSkEpiWarps = 8, kSkThreads = 64 + 32 * kSkEpiWarps;

__device__ __forceinline__ int4 ld_peer(uint32_t local, uint32_t rank) {
  uint32_t ra;
  int4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(local), "r"(rank));
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(ra) : "memory");
  return v;
}

// grid = tiles x splits, clusters of `splits` CTAs.  Warp 0: TMA; warp 1: TMEM and MMA; warps 2 to 9: sums and stores.
template <int MT, int OUT>
__global__ void __launch_bounds__(kSkThreads, 2) gemm_i8_skinny_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, GemmI8Args a,
                                                                      int splits) {
  using C = SkCfg<MT>;
  constexpr int STAGES = C::kStages;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar_base = base + STAGES * C::kStage;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  const uint32_t acc_full = bar_base + 16u * STAGES;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + STAGES * C::kStage + 16 * STAGES + 8);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tile = blockIdx.x / splits, split = blockIdx.x - tile * splits, n0 = tile * 128;
  const int k_iters = (a.K + kStepK - 1) / kStepK, k_base = k_iters / splits, k_rem = k_iters - k_base * splits;
  const int k_begin = split * k_base + min(split, k_rem), k_count = k_base + (split < k_rem ? 1 : 0);
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(acc_full, 1);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_map(&tmW);
    tma_prefetch_map(&tmX);
  }
  // The first of this CTA's weights into the L2 while the launch before is still running (a copy there is no older than memory: what that launch writes
  // is in it).
  if (threadIdx.x == 64)
    for (int k = 0; k < min(STAGES, k_count); ++k)
      asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&tmW), "r"((k_begin + k) * kStepK), "r"(n0) : "memory");
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(C::kTmemCols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  pdl_launch();
  // A row of the sums goes to one of the cluster's epilogue warps: this one's i-th is split + splits * (warp - 2 + 8 i); lane i has its scale.
  float sw[4], bias[4], sa_mine = 0.f;
  if (warp == 0) {
    const uint32_t leader = elect_one();
    int s = 0, k = 0;
    uint32_t round = 0;
    bool ok = true;
    for (; k < k_count; ++k) {
      if (!warp_wait_uniform(empty_bar(s), round ^ 1u, abort_flag)) { ok = false; break; }
      const uint32_t fb = full_bar(s), dst = base + s * C::kStage;
      mbar_expect_tx_if(fb, C::kStage, leader);
      tma_load_2d_if(dst, &tmW, (k_begin + k) * kStepK, n0, fb, leader);
      tma_load_2d_if(dst + C::kTileW, &tmX, (k_begin + k) * kStepK, 0, fb, leader);
      if (++s == STAGES) { s = 0; round ^= 1u; }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      for (int j = max(0, k - STAGES); j < k; ++j) mbar_wait(full_bar(j % STAGES), (j / STAGES) & 1);
    }
  } else if (warp == 1) {
    const uint32_t leader = elect_one();
    const uint64_t dw0 = smem_desc(base), dx0 = smem_desc(base + C::kTileW);
    int s = 0;
    uint32_t round = 0;
    bool ok = true;
    for (int k = 0; k < k_count; ++k) {
      if (!warp_wait_uniform(full_bar(s), round, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const uint64_t so = (uint64_t)(s * (C::kStage >> 4));
      mma_step(tmem_base, dw0 + so, dx0 + so, instr_desc(128, MT), k > 0 ? 1u : 0u, leader);
      tc_commit_if(empty_bar(s), leader);
      if (++s == STAGES) { s = 0; round ^= 1u; }
    }
    if (ok) tc_commit_if(acc_full, leader);
    else if (leader) *abort_flag = 1;
  } else {
    cols4(a, n0 + 4 * lane, sw, bias);
    const int r = split + splits * (warp - 2 + kSkEpiWarps * lane);
    if (r < a.M) sa_mine = a.a_scale[r];
    const bool ok = warp_wait_uniform(acc_full, 0, abort_flag);
    tc_fence_after();
    if (ok) {
      // TMEM lane = column n0 + 32 q + lane of C, TMEM column = row: [row][128 columns] in shared memory (the ring is idle: all products are done)
      const int q = warp & 3;
      int* img = reinterpret_cast<int*>(gen_base) + q * 32 + lane;
#pragma unroll 1
      for (int r0 = (warp - 2) / 4 * 16; r0 < min(MT, a.M); r0 += 32) {      // (the two warps of a lane quarter take 16 rows each in turn)
        int v[16];
        tmem_ld16_int(tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)r0, v);
#pragma unroll
        for (int j = 0; j < 16; ++j) img[(r0 + j) * 128] = v[j];
      }
    } else if (lane == 0) {
      *abort_flag = 1;
    }
  }
  tc_fence_before();
  if (splits > 1) cluster_sync_all();
  else __syncthreads();
  if (warp >= 2 && !*abort_flag) {
    const bool wide = wide_rows<OUT>(a) && n0 + 4 * lane + 3 < a.N;
    const uint32_t at = base + lane * 16;
    int i = 0;
#pragma unroll 2
    for (int r = split + splits * (warp - 2); r < a.M; r += splits * kSkEpiWarps, ++i) {
      const float sa = __shfl_sync(0xffffffffu, sa_mine, i);
      int4 part[8];
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p < splits) part[p] = splits > 1 ? ld_peer(at + r * 512, p) : *reinterpret_cast<const int4*>(gen_base + lane * 16 + r * 512);
      int acc[4] = {part[0].x, part[0].y, part[0].z, part[0].w};
#pragma unroll
      for (int p = 1; p < 8; ++p)
        if (p < splits) { acc[0] += part[p].x; acc[1] += part[p].y; acc[2] += part[p].z; acc[3] += part[p].w; }
      if (n0 + 4 * lane < a.N) store4<OUT>(a, r, n0 + 4 * lane, acc, sa, sw, bias, wide);
    }
  }
  if (splits > 1) cluster_sync_all();                // no CTA leaves while a peer may still read its sums
  else __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::kTmemCols));
  }
  if (threadIdx.x == 0 && *abort_flag) atomicOr(a.status, kStInternal);
}

template <int MT, int OUT>
bool launch(const GemmI8Args& a, cudaStream_t st) {
  using C = SkCfg<MT>;
  CUtensorMap tw, tx;
  if (!map_i8(a.W, a.N, a.K, 128, &tw) || !map_i8(a.A, a.M, a.K, MT, &tx)) return false;
  static PerDeviceOnce configured;
  configured.run([] { cudaFuncSetAttribute(gemm_i8_skinny_kernel<MT, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem); });
  const int tiles = (a.N + 127) / 128, k_iters = (a.K + kStepK - 1) / kStepK;
  // as many CTAs as bring the grid to one per SM (two: 20 x 6144 x 4096 13.6 instead of 10.4 us), at most 8 per tile, each with at least two steps (32 KB of W)
  int splits = sm_count() / tiles;
  if (splits > k_iters / 2) splits = k_iters / 2;
  if (splits > 8) splits = 8;
  if (splits < 1) splits = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(tiles * splits); cfg.blockDim = dim3(kSkThreads); cfg.dynamicSmemBytes = C::kSmem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = splits; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = pdl_enabled() ? 2 : 1;
  cudaLaunchKernelEx(&cfg, gemm_i8_skinny_kernel<MT, OUT>, tw, tx, a, splits);
  return true;
}
template <int OUT>
bool launch_mt(const GemmI8Args& a, cudaStream_t st) {
  return a.M <= 32 ? launch<32, OUT>(a, st) : a.M <= 64 ? launch<64, OUT>(a, st) : launch<128, OUT>(a, st);
}

}  // namespace

bool launch_gemm_i8_skinny(const GemmI8Args& a, bool bf16_out, cudaStream_t st) {
  return bf16_out ? launch_mt<kBf16>(a, st) : a.epilogue == kEpiAddF32 ? launch_mt<kF32Add>(a, st) : launch_mt<kF32>(a, st);
}

}  // namespace nz
