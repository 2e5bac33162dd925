// C = A W^T of 8-bit integers on the tensor cores (tcgen05 kind::i8, 32-bit integer accumulators in TMEM): tiles of 128 x BN, and of 256 x 256 on CTA
// pairs.  The roles, rings and waits are those of gemm_tc.cu and gemm_tc2.cu: a TMA warp, an issuing warp, eight epilogue warps, persistent
// over tiles with two accumulators.  A k-step moves the bytes of a bf16 step and holds twice the products, so their cost model gives the tiling.
// The sums are whole numbers: no order of summation, tiling or kernel changes a bit of C.  16,008 x 4,096 x 11,008: 428 us, 3.37e15 operations a second, twice
// what bf16 products reach here; with few k-steps a tile (971 x 9,728 x 896 to fp32: 16 us, floor 7) the first loads, the last epilogue and whole waves of tiles count.
#include <stdlib.h>

#include "gemm_i8.cuh"

namespace nz {

int sm_count();
int gemm_tc_plan(int M, int N, int K);
bool launch_gemm_i8_skinny(const GemmI8Args& a, bool bf16_out, cudaStream_t st);
void launch_gemm_i8_simt(const GemmI8Args& a, bool bf16, cudaStream_t st);

namespace {

using namespace gemm_detail;
using namespace i8_detail;

constexpr int kTileA = 128 * kStepK;

template <int BN> struct I8Cfg {
  static constexpr int kTileB = BN * kStepK;
  static constexpr int kStage = kTileA + kTileB;
  static constexpr int kStages = BN >= 192 ? 4 : BN == 160 ? 5 : BN == 128 ? 6 : 8;
  static constexpr int kSmem = kStages * kStage + 1024 + 256 + kTransposeBytes;
  static constexpr uint32_t kDesc = instr_desc(128, BN);
};

template <int BN, int OUT>
__global__ void __launch_bounds__(kThreads) gemm_i8_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, GemmI8Args a) {
  using C = I8Cfg<BN>;
  constexpr int STAGES = C::kStages, kAcc = 2 * BN;
  constexpr int kTmemCols = kAcc <= 64 ? 64 : kAcc <= 128 ? 128 : kAcc <= 256 ? 256 : 512;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bar_base = base + STAGES * C::kStage;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  auto acc_full = [&](int b) { return bar_base + 8u * (2 * STAGES + b); };
  auto acc_empty = [&](int b) { return bar_base + 8u * (2 * STAGES + 2 + b); };
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + STAGES * C::kStage + 8 * (2 * STAGES + 4));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int k_iters = (a.K + kStepK - 1) / kStepK;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), kEpiWarps); }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_map(&tmA);
    tma_prefetch_map(&tmB);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(kTmemCols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  pdl_launch();
  const int tiles_m = (a.M + 127) / 128, tiles_n = (a.N + BN - 1) / BN, n_tiles = tiles_m * tiles_n;

  if (warp == 0) {
    const uint32_t leader = elect_one();
    int it = 0, s = 0;
    uint32_t round = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x) {
      const int m0 = (tile % tiles_m) * 128, n0 = (tile / tiles_m) * BN;
      for (int k = 0; k < k_iters; ++k, ++it) {
        if (!warp_wait_uniform(empty_bar(s), round ^ 1u, abort_flag)) { ok = false; break; }
        const uint32_t fb = full_bar(s), dst = base + s * C::kStage;
        mbar_expect_tx_if(fb, C::kStage, leader);
        tma_load_2d_if(dst, &tmA, k * kStepK, m0, fb, leader);
        tma_load_2d_if(dst + kTileA, &tmB, k * kStepK, n0, fb, leader);
        if (++s == STAGES) { s = 0; round ^= 1u; }
      }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      for (int j = max(0, it - STAGES); j < it; ++j) mbar_wait(full_bar(j % STAGES), (j / STAGES) & 1);
    }
  } else if (warp == 1) {
    const uint32_t leader = elect_one();
    int t_local = 0, s = 0;
    uint32_t round = 0;
    bool ok = true;
    const uint64_t da0 = smem_desc(base), db0 = smem_desc(base + kTileA);
    for (int tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x, ++t_local) {
      const int b = t_local & 1;
      if (t_local >= 2 && !warp_wait_uniform(acc_empty(b), ((t_local >> 1) - 1) & 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      for (int k = 0; k < k_iters; ++k) {
        if (!warp_wait_uniform(full_bar(s), round, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint64_t so = (uint64_t)(s * (C::kStage >> 4));
        mma_step(tmem_base + (uint32_t)(b * BN), da0 + so, db0 + so, C::kDesc, k > 0 ? 1u : 0u, leader);
        tc_commit_if(empty_bar(s), leader);
        if (++s == STAGES) { s = 0; round ^= 1u; }
      }
      if (ok) tc_commit_if(acc_full(b), leader);
    }
    if (!ok && leader) *abort_flag = 1;
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;
    int4* stg = reinterpret_cast<int4*>(gen_base + STAGES * C::kStage + 256) + (warp - 2) * (32 * 8);
    const bool wide = wide_rows<OUT>(a);
    int t_local = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x, ++t_local) {
      const int b = t_local & 1, m0 = (tile % tiles_m) * 128, n0 = (tile / tiles_m) * BN;
      TileScales<BN> ts;
      ts.get(a, q, half, lane, m0, n0);
      ok = warp_wait_uniform(acc_full(b), (t_local >> 1) & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      drain<BN, OUT>(a, tmem_base + (uint32_t)(b * BN), q, half, lane, stg, m0, n0, wide, ts);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(acc_empty(b));
    }
    if (!ok && lane == 0) *abort_flag = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols));
  }
  if (threadIdx.x == 0 && *abort_flag) atomicOr(a.status, kStInternal);
}

// ---------------------------------------------------------------------------------------------------
// 256 x 256 tiles on CTA pairs
// ---------------------------------------------------------------------------------------------------
constexpr int kPairN = 256, kTileHalfB = 128 * kStepK, kPairStage = kTileA + kTileHalfB, kPairStages = 6;
constexpr int kPairSmem = kPairStages * kPairStage + 1024 + 256 + kTransposeBytes;
constexpr uint32_t kLeaderMask = 0xFEFFFFFFu;

__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t leader_bar, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
      ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(leader_bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar, uint32_t leader) {
  const uint16_t both = 3;
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
      ::"r"(bar), "h"(both), "r"(leader) : "memory");
}

template <int OUT>
__global__ void __launch_bounds__(kThreads) gemm_i8_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, GemmI8Args a) {
  constexpr int STAGES = kPairStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bar_base = base + STAGES * kPairStage;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  auto acc_full = [&](int b) { return bar_base + 8u * (2 * STAGES + b); };
  auto acc_empty = [&](int b) { return bar_base + 8u * (2 * STAGES + 2 + b); };
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + STAGES * kPairStage + 8 * (2 * STAGES + 4));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int k_iters = (a.K + kStepK - 1) / kStepK;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), 2 * kEpiWarps); }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_map(&tmA);
    tma_prefetch_map(&tmB);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(2 * kPairN));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  pdl_launch();
  const int tiles_m = (a.M + 255) / 256, tiles_n = (a.N + kPairN - 1) / kPairN, n_tiles = tiles_m * tiles_n;
  const int band = tiles_n >= 16 ? 16 : 8;           // (see gemm_tc2.cu)
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (warp == 0) {
    const uint32_t leader = elect_one();
    int it = 0, s = 0;
    uint32_t round = 0;
    bool ok = true;
    for (int tile = pair; tile < n_tiles && ok; tile += n_pairs) {
      const TileMN tt = tile_of(tile, tiles_m, tiles_n, band);
      const int m0 = tt.m * 256 + (int)rank * 128, nb0 = tt.n * kPairN + (int)rank * 128;
      for (int k = 0; k < k_iters; ++k, ++it) {
        if (!warp_wait_uniform(empty_bar(s), round ^ 1u, abort_flag)) { ok = false; break; }
        const uint32_t dst = base + s * kPairStage, fb = full_bar(s) & kLeaderMask;
        mbar_expect_tx_if(full_bar(s), 2 * kPairStage, rank == 0 ? leader : 0u);
        tma_load_pair(dst, &tmA, k * kStepK, m0, fb, leader);
        tma_load_pair(dst + kTileA, &tmB, k * kStepK, nb0, fb, leader);
        if (++s == STAGES) { s = 0; round ^= 1u; }
      }
    }
    // (both CTAs' copies arrive on the leader's barriers: it waits for those in flight, and the other for it, at the cluster's barrier)
    if (!ok && lane == 0) {
      *abort_flag = 1;
      if (rank == 0)
        for (int j = max(0, it - STAGES); j < it; ++j) mbar_wait(full_bar(j % STAGES), (j / STAGES) & 1);
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t leader = elect_one();
      int t_local = 0, s = 0;
      uint32_t round = 0;
      bool ok = true;
      const uint64_t da0 = smem_desc(base), db0 = smem_desc(base + kTileA);
      for (int tile = pair; tile < n_tiles && ok; tile += n_pairs, ++t_local) {
        const int b = t_local & 1;
        if (t_local >= 2 && !warp_wait_uniform(acc_empty(b), ((t_local >> 1) - 1) & 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        for (int k = 0; k < k_iters; ++k) {
          if (!warp_wait_uniform(full_bar(s), round, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t so = (uint64_t)(s * (kPairStage >> 4));
          mma_step_pair(tmem_base + (uint32_t)(b * kPairN), da0 + so, db0 + so, instr_desc(256, kPairN), k > 0 ? 1u : 0u, leader);
          commit_pair(empty_bar(s), leader);
          if (++s == STAGES) { s = 0; round ^= 1u; }
        }
        if (ok) commit_pair(acc_full(b), leader);
      }
      if (!ok && lane == 0) *abort_flag = 1;
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;
    int4* stg = reinterpret_cast<int4*>(gen_base + STAGES * kPairStage + 256) + (warp - 2) * (32 * 8);
    const bool wide = wide_rows<OUT>(a);
    int t_local = 0;
    bool ok = true;
    for (int tile = pair; tile < n_tiles && ok; tile += n_pairs, ++t_local) {
      const TileMN tt = tile_of(tile, tiles_m, tiles_n, band);
      const int b = t_local & 1, m0 = tt.m * 256 + (int)rank * 128, n0 = tt.n * kPairN;
      TileScales<kPairN> ts;
      ts.get(a, q, half, lane, m0, n0);
      ok = warp_wait_uniform(acc_full(b), (t_local >> 1) & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      drain<kPairN, OUT>(a, tmem_base + (uint32_t)(b * kPairN), q, half, lane, stg, m0, n0, wide, ts);
      tc_fence_before();
      __syncwarp();
      // (relaxed: nothing in memory is handed over, and a release would wait for the stores of C.  What the products behind it rest on is that the
      // accumulator is in registers: tcgen05.wait::ld in the drain, and the fence before this.  16,008 x 16,384 x 512: 240 us with a release, 191
      // without; 8,634 x 2,336 x 832: 26.5, 22.5)
      if (lane == 0) asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(acc_empty(b) & kLeaderMask) : "memory");
    }
    if (!ok && lane == 0) *abort_flag = 1;
  }
  tc_fence_before();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(2 * kPairN));
  }
  if (threadIdx.x == 0 && *abort_flag) atomicOr(a.status, kStInternal);
}

// ---------------------------------------------------------------------------------------------------
// host side; false = not launched (a tensor map was refused)
// ---------------------------------------------------------------------------------------------------
template <int BN, int OUT>
bool launch(const GemmI8Args& a, cudaStream_t st) {
  CUtensorMap ta, tb;
  if (!map_i8(a.A, a.M, a.K, 128, &ta) || !map_i8(a.W, a.N, a.K, BN, &tb)) return false;
  static PerDeviceOnce configured;
  configured.run([] { cudaFuncSetAttribute(gemm_i8_kernel<BN, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, I8Cfg<BN>::kSmem); });
  const long long tiles = (long long)((a.M + 127) / 128) * ((a.N + BN - 1) / BN);
  const int grid = (int)(tiles < sm_count() ? tiles : sm_count());
  launch_pdl(gemm_i8_kernel<BN, OUT>, dim3(grid), dim3(kThreads), I8Cfg<BN>::kSmem, st, ta, tb, a);
  return true;
}
template <int OUT>
bool launch_pair(const GemmI8Args& a, cudaStream_t st) {
  CUtensorMap ta, tb;
  if (!map_i8(a.A, a.M, a.K, 128, &ta) || !map_i8(a.W, a.N, a.K, 128, &tb)) return false;
  static PerDeviceOnce configured;
  configured.run([] { cudaFuncSetAttribute(gemm_i8_pair_kernel<OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem); });
  const long long tiles = (long long)((a.M + 255) / 256) * ((a.N + kPairN - 1) / kPairN);
  const int pairs = (int)(tiles < sm_count() / 2 ? tiles : sm_count() / 2);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(2 * pairs); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = kPairSmem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = pdl_enabled() ? 2 : 1;
  cudaLaunchKernelEx(&cfg, gemm_i8_pair_kernel<OUT>, ta, tb, a);
  return true;
}

template <int OUT>
bool launch_tiles(const GemmI8Args& a, cudaStream_t st) {
  switch (gemm_tc_plan(a.M, a.N, (a.K + kStepK - 1) / kStepK * 64)) {      // a step is a bf16 step's bytes: 64 of its elements
    case 512: return launch_pair<OUT>(a, st);
    case 256: return launch<256, OUT>(a, st);
    case 192: return launch<192, OUT>(a, st);
    case 160: return launch<160, OUT>(a, st);
    case 128: return launch<128, OUT>(a, st);
    case 64: return launch<64, OUT>(a, st);
    default: return launch<32, OUT>(a, st);
  }
}

}  // namespace

void launch_gemm_i8(const GemmI8Args& a, bool bf16, cudaStream_t st) {
  LaunchScope ls(kcGemm, st);
  const bool bf16_out = bf16 && a.epilogue == kEpiStoreAct;
  const bool tc = a.K % 16 == 0 && ((uintptr_t)a.A & 15) == 0 && ((uintptr_t)a.W & 15) == 0 && tma_encode_fn();
  if (tc) {
    // Few rows stream the weights with W as the 128-row operand; beyond 32 of them only where that splits the K range three ways or more, which is what the
    // general kernel's wider tiles then lose by.  us, streaming / general, 48 rows: 6144 x 4096 11.4 / 10.8, 22016 x 4096 25.6 / 24.5, 2048 x 8192 10.3 / 13.3,
    // 4096 x 11008 16.4 / 19.4; 100 rows: 13.6 / 11.0, 29.4 / 24.9, 12.2 / 13.5, 18.1 / 19.7; 20 rows: 10.4 / 15.6, 23.3 / 26.9, 8.9 / 13.2, 14.8 / 19.1.
    const bool streams = a.M <= 32 || (a.M <= 128 && sm_count() / ((a.N + 127) / 128) >= 3);
    if (streams && launch_gemm_i8_skinny(a, bf16_out, st)) return;
    if (bf16_out ? launch_tiles<kBf16>(a, st) : a.epilogue == kEpiAddF32 ? launch_tiles<kF32Add>(a, st) : launch_tiles<kF32>(a, st)) return;
  }
  launch_gemm_i8_simt(a, bf16, st);
}

}  // namespace nz
