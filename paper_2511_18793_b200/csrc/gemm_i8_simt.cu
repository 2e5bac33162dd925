// C = A W^T of 8-bit integers on the CUDA cores (four products per instruction): the sizes and alignments that the tensor-core kernels do
// not take.  64 x 64 tiles of C, 64 bytes of K at a time.
#include "operators.cuh"

namespace nz {

namespace {

constexpr int kT = 64, kKB = 64, kLd = kKB / 4 + 1;

template <typename OUT, bool ADD>
__global__ void __launch_bounds__(256) gemm_i8_simt_kernel(GemmI8Args a, int tiles_n) {
  __shared__ int as[kT * kLd], ws[kT * kLd];
  pdl_wait();
  pdl_launch();
  const int m0 = blockIdx.x / tiles_n * kT, n0 = blockIdx.x % tiles_n * kT;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  int acc[4][4] = {};
  for (int k0 = 0; k0 < a.K; k0 += kKB) {
    __syncthreads();
    for (int i = threadIdx.x; i < kT * (kKB / 4); i += 256) {
      const int r = i / (kKB / 4), c = i % (kKB / 4) * 4;
      uint32_t wa = 0, ww = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k0 + c + e < a.K) {
          if (m0 + r < a.M) wa |= (uint32_t)(uint8_t)a.A[(long long)(m0 + r) * a.K + k0 + c + e] << (8 * e);
          if (n0 + r < a.N) ww |= (uint32_t)(uint8_t)a.W[(long long)(n0 + r) * a.K + k0 + c + e] << (8 * e);
        }
      as[r * kLd + c / 4] = (int)wa;
      ws[r * kLd + c / 4] = (int)ww;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kKB / 4; ++c) {
      int x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = as[(ty + 16 * i) * kLd + c]; y[i] = ws[(tx + 16 * i) * kLd + c]; }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(x[i], y[j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m >= a.M || n >= a.N) continue;
      const float x = i8_value(acc[i][j], a.a_scale[m], a.w_scale[n], a.bias ? a.bias[n] : 0.f);
      OUT* c = (OUT*)a.C + (long long)m * a.N + n;
      if (ADD) *c = from_f32<OUT>(__fadd_rn(to_f32(*c), x));
      else *c = from_f32<OUT>(x);
    }
}

}  // namespace

void launch_gemm_i8_simt(const GemmI8Args& a, bool bf16, cudaStream_t st) {
  const int tiles_n = (a.N + kT - 1) / kT;
  const dim3 grid((unsigned)((long long)((a.M + kT - 1) / kT) * tiles_n));
  if (a.epilogue == kEpiAddF32) launch_pdl(gemm_i8_simt_kernel<float, true>, grid, dim3(256), 0, st, a, tiles_n);
  else if (a.epilogue == kEpiStoreF32 || !bf16) launch_pdl(gemm_i8_simt_kernel<float, false>, grid, dim3(256), 0, st, a, tiles_n);
  else launch_pdl(gemm_i8_simt_kernel<__nv_bfloat16, false>, grid, dim3(256), 0, st, a, tiles_n);
}

}  // namespace nz
