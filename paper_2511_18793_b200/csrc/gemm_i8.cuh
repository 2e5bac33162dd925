// tcgen05 pieces of the 8-bit products.  A k-step is 128 bytes of a row, which is 128 elements here: tiles, swizzle, descriptors and copies are
// byte for byte those of the bf16 kernels, and a step has twice the products.
#pragma once

#include "gemm_epilogue.cuh"
#include "operators.cuh"

namespace nz {
namespace i8_detail {

constexpr int kStepK = 128;                        // elements (= bytes) of K per step

// kind::i8 instruction descriptor: D = s32, A = B = signed 8-bit, both K-major.
constexpr uint32_t instr_desc(int m, int n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

// The four MMAs (32 elements of K each) of a step in one statement (see tc_mma_kstep).
__device__ __forceinline__ void mma_step(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate_first, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, t, q;\n\t.reg .b64 a1, b1, a2, b2, a3, b3;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.eq.b32 t, %4, %4;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "add.s64 a1, %1, 2;\n\tadd.s64 b1, %2, 2;\n\t"
      "add.s64 a2, %1, 4;\n\tadd.s64 b2, %2, 4;\n\t"
      "add.s64 a3, %1, 6;\n\tadd.s64 b3, %2, 6;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::i8 [%0], a1, b1, %3, t;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::i8 [%0], a2, b2, %3, t;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::i8 [%0], a3, b3, %3, t;\n\t}"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate_first), "r"(leader) : "memory");
}
__device__ __forceinline__ void mma_step_pair(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate_first, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, t, q;\n\t.reg .b64 a1, b1, a2, b2, a3, b3;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.eq.b32 t, %4, %4;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "add.s64 a1, %1, 2;\n\tadd.s64 b1, %2, 2;\n\t"
      "add.s64 a2, %1, 4;\n\tadd.s64 b2, %2, 4;\n\t"
      "add.s64 a3, %1, 6;\n\tadd.s64 b3, %2, 6;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::i8 [%0], a1, b1, %3, t;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::i8 [%0], a2, b2, %3, t;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::i8 [%0], a3, b3, %3, t;\n\t}"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate_first), "r"(leader) : "memory");
}

// 32 columns of the warp's TMEM lanes as integers.
__device__ __forceinline__ void tmem_ld32_ask(uint32_t taddr, int* v) {      // v is there after the next tmem_ld_wait
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
        "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait(int* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(v[i]));      // (not moved in front of the wait)
}

__device__ __forceinline__ void tmem_ld16_int(uint32_t taddr, int* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(v[i]));
}

// int8 row-major [rows, K] with dense rows; box = 128 columns x box_rows rows, 128-byte swizzle.  What lies outside reads as zeros.
inline bool map_i8(const void* ptr, long long rows, long long K, int box_rows, CUtensorMap* out) {
  if (!tma_encode_fn()) return false;
  cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)K};
  cuuint32_t box[2] = {128u, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return tma_encode_fn()(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

enum Out { kBf16 = 0, kF32 = 1, kF32Add = 2 };

// Four neighbouring elements of a row of C.  `wide`: C can be written in vectors of four elements there.
template <int OUT>
__device__ __forceinline__ void store4(const GemmI8Args& a, int row, int n, const int* acc, float sa, const float* sw, const float* bias, bool wide) {
  float x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = i8_value(acc[e], sa, sw[e], bias[e]);
  const long long at = (long long)row * a.N + n;
  if constexpr (OUT == kBf16) {
    __nv_bfloat16* c = (__nv_bfloat16*)a.C + at;
    if (wide) *reinterpret_cast<uint2*>(c) = gemm_detail::pack_bf16x4(x[0], x[1], x[2], x[3]);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) c[e] = __float2bfloat16_rn(x[e]);
  } else {
    float* c = (float*)a.C + at;
    if (wide) {
      float4 y = make_float4(x[0], x[1], x[2], x[3]);
      if constexpr (OUT == kF32Add) {
        const float4 old = *reinterpret_cast<const float4*>(c);
        y = make_float4(__fadd_rn(old.x, x[0]), __fadd_rn(old.y, x[1]), __fadd_rn(old.z, x[2]), __fadd_rn(old.w, x[3]));
      }
      *reinterpret_cast<float4*>(c) = y;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) c[e] = OUT == kF32Add ? __fadd_rn(c[e], x[e]) : x[e];
    }
  }
}
// Vectors of four elements: every row of C begins on their boundary.
template <int OUT>
__device__ __forceinline__ bool wide_rows(const GemmI8Args& a) {
  constexpr uintptr_t kVec = OUT == kBf16 ? 8 : 16;
  return a.N % 4 == 0 && ((uintptr_t)a.C & (kVec - 1)) == 0;
}
__device__ __forceinline__ void cols4(const GemmI8Args& a, int n, float* sw, float* bias) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = n + e < a.N;
    sw[e] = in ? a.w_scale[n + e] : 0.f;
    bias[e] = in && a.bias ? a.bias[n + e] : 0.f;
  }
}

// What an epilogue warp needs from memory for a tile, asked for while the tile's products run: its row's scale, and the scales and biases of the lane's four
// columns in each of the warp's 32-column groups (asked for group by group behind them: 971 x 9728 x 896 18.1 us).
template <int BN>
struct TileScales {
  static constexpr int kGroups = (BN / 32 + 1) / 2;
  float sa, sw[kGroups][4], bias[kGroups][4];
  __device__ __forceinline__ void get(const GemmI8Args& a, int q, int half, int lane, int m0, int n0) {
    const int row = m0 + q * 32 + lane;
    sa = row < a.M ? a.a_scale[row] : 0.f;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) cols4(a, n0 + (half + 2 * i) * 32 + 4 * (lane & 7), sw[i], bias[i]);
  }
};

// The same as `drain` below for a bf16 C whose rows are in 16-byte pieces.  A lane has its own row's accumulators, so it scales and rounds them before they
// are turned, which is half the bytes through shared memory, and the next group's are on their way meanwhile.  The columns' scales and biases lie in the
// upper half of the warp's staging area.  16,008 x 16,384 x 512, where the epilogue is the bound: 240 us, 267 through `drain`.
template <int BN>
__device__ __forceinline__ void drain_bf16(const GemmI8Args& a, uint32_t tmem_acc, int q, int half, int lane, int4* stg, int m0, int n0, const TileScales<BN>& ts) {
  constexpr int kG = TileScales<BN>::kGroups;
  const int m_warp = m0 + q * 32;
  if (m_warp >= a.M) return;
  float4 *sws = reinterpret_cast<float4*>(stg + 128), *bs = sws + 8 * kG;
  static_assert(2 * 8 * kG <= 128, "staging area");
  if (lane < 8)
#pragma unroll
    for (int i = 0; i < kG; ++i) {
      sws[8 * i + lane] = make_float4(ts.sw[i][0], ts.sw[i][1], ts.sw[i][2], ts.sw[i][3]);
      bs[8 * i + lane] = make_float4(ts.bias[i][0], ts.bias[i][1], ts.bias[i][2], ts.bias[i][3]);
    }
  const uint32_t t0 = tmem_acc + ((uint32_t)(q * 32) << 16);
  auto there = [&](int i) { return half + 2 * i < BN / 32 && n0 + (half + 2 * i) * 32 < a.N; };      // (warp-uniform)
  int v[32];
  if (!there(0)) return;
  tmem_ld32_ask(t0 + (uint32_t)(half * 32), v);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kG; ++i) {
    if (!there(i)) break;
    const int n = n0 + (half + 2 * i) * 32;
    uint32_t w[16];
    tmem_ld_wait(v);
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const float4 sw = sws[8 * i + c], b = bs[8 * i + c];
      const uint2 y = gemm_detail::pack_bf16x4(i8_value(v[4 * c], ts.sa, sw.x, b.x), i8_value(v[4 * c + 1], ts.sa, sw.y, b.y),
                                               i8_value(v[4 * c + 2], ts.sa, sw.z, b.z), i8_value(v[4 * c + 3], ts.sa, sw.w, b.w));
      w[2 * c] = y.x; w[2 * c + 1] = y.y;
    }
    if (i + 1 < kG && there(i + 1)) tmem_ld32_ask(t0 + (uint32_t)((half + 2 * (i + 1)) * 32), v);
#pragma unroll
    for (int p = 0; p < 4; ++p) stg[lane * 4 + (p ^ ((lane >> 1) & 3))] = make_int4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 8 * j + (lane >> 2), p = lane & 3;
      const int4 x = stg[r * 4 + (p ^ ((r >> 1) & 3))];
      if (m_warp + r < a.M && n + 8 * p < a.N) *reinterpret_cast<int4*>((__nv_bfloat16*)a.C + (long long)(m_warp + r) * a.N + n + 8 * p) = x;
    }
    __syncwarp();
  }
}

// Drains the BN columns of a 128-row accumulator: epilogue warp (lane quarter q, half) takes every second 32-column group, turns its 32 x 32 blocks
// through shared memory so that 8 lanes have 32 neighbouring columns of a row, and stores four rows at a time.
template <int BN, int OUT>
__device__ __forceinline__ void drain(const GemmI8Args& a, uint32_t tmem_acc, int q, int half, int lane, int4* stg, int m0, int n0, bool wide, const TileScales<BN>& ts) {
  if constexpr (OUT == kBf16)
    if (a.N % 8 == 0 && ((uintptr_t)a.C & 15) == 0) { drain_bf16<BN>(a, tmem_acc, q, half, lane, stg, m0, n0, ts); return; }
  const int k8 = lane & 7, rsub = lane >> 3;
  const int m_warp = m0 + q * 32;
  if (m_warp >= a.M) return;
  const uint32_t t0 = tmem_acc + ((uint32_t)(q * 32) << 16);
#pragma unroll
  for (int i = 0; i < TileScales<BN>::kGroups; ++i) {
    const int g = half + 2 * i, n = n0 + g * 32;
    if (g >= BN / 32 || n >= a.N) break;             // (warp-uniform)
    int v[32];
    tmem_ld32_ask(t0 + (uint32_t)(g * 32), v);
    tmem_ld_wait(v);
#pragma unroll
    for (int c = 0; c < 8; ++c) stg[lane * 8 + (c ^ (lane & 7))] = make_int4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 4 * j + rsub;
      const int4 x = stg[r * 8 + (k8 ^ (r & 7))];
      const int acc[4] = {x.x, x.y, x.z, x.w};
      const float sa = __shfl_sync(0xffffffffu, ts.sa, r);
      if (m_warp + r < a.M && n + 4 * k8 < a.N) store4<OUT>(a, m_warp + r, n + 4 * k8, acc, sa, ts.sw[i], ts.bias[i], wide);
    }
    __syncwarp();
  }
}

}  // namespace i8_detail
}  // namespace nz
