// Rows to 8-bit integers with a scale each:  scale = max|x| / 127,  q = 127 x / max|x| to the nearest, halves to even.
//
// One read of x and one write of q bound it: a row's chunks stay in registers between the two (up to kKeep per thread; what a longer row
// has beyond is read again, from the L2).  The maximum is taken over the bit patterns of |x|, in which a NaN is above
// infinity and that above all numbers.  x * (127 / max) is off by less than 1e-4 of a step, so a quotient that near to a border
// is divided in 64 bits, where a half is a half: a value half as large as the row's largest lies on the border 63.5 exactly.
#include <type_traits>

#include "operators.cuh"

namespace nz {

namespace {

template <typename T> struct Chunk;                // 16 bytes of x
template <> struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(const uint4& u, int i) { return __uint_as_float(i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w); }
  static __device__ __forceinline__ uint32_t top(const uint4& u) { return max(max(u.x & 0x7fffffffu, u.y & 0x7fffffffu), max(u.z & 0x7fffffffu, u.w & 0x7fffffffu)); }
};
template <> struct Chunk<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(const uint4& u, int i) {
    const uint32_t w = (i >> 1) == 0 ? u.x : (i >> 1) == 1 ? u.y : (i >> 1) == 2 ? u.z : u.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  // (16-bit patterns of |x| are ordered as their values are: two maxima per instruction, a NaN stays one)
  static __device__ __forceinline__ uint32_t top(const uint4& u) {
    const uint32_t m = __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu));
    return max(m & 0xffff0000u, m << 16);
  }
};

struct RowScale { float top, inv; bool bad; };
__device__ __forceinline__ RowScale row_scale_of(uint32_t top_bits) {
  RowScale r;
  r.bad = top_bits >= 0x7f800000u;
  r.top = __uint_as_float(top_bits);
  r.inv = 127.f / r.top;                           // (rows whose largest value is below 1e-30: the 64-bit division throughout)
  return r;
}
__device__ __forceinline__ int to_i8_exact(float x, const RowScale& s) {
  return s.bad || s.top == 0.f ? 0 : (int)rint((double)x * 127.0 / (double)s.top);
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Four values: rounded by adding 1.5 x 2^23, whose last byte is then the 8-bit integer; what is left over tells how near a border they were.
template <typename T>
__device__ __forceinline__ uint32_t four(const uint4& u, int g, const RowScale& s) {
  constexpr float kMagic = 12582912.f;
  uint32_t b[4];
  float off = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = Chunk<T>::get(u, 4 * g + e), r = fmaf(x, s.inv, kMagic);
    off = fmaxf(off, fabsf(fmaf(x, s.inv, kMagic - r)));
    b[e] = __float_as_uint(r);
  }
  // (also where inv is no number, or infinite, or the row has NaNs: the comparison is false)
  if (!(off <= 0.4999f) || s.top < 1e-30f || s.bad)
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = (uint32_t)to_i8_exact(Chunk<T>::get(u, 4 * g + e), s);
  return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}

constexpr int kKeep = 8;                           // chunks of a row that a thread keeps

// TPR threads per row; a warp per row: eight rows per block.  VEC: rows of x and q in 16- and 8- (4-) byte pieces.
template <int TPR> constexpr int kBlock = TPR == 32 ? 256 : TPR;
template <typename T, int TPR, bool VEC>
__global__ void __launch_bounds__(kBlock<TPR>) quantize_rows_kernel(const T* __restrict__ x, long long x_stride, int M, int K, int8_t* __restrict__ q,
                                                            float* __restrict__ scale) {
  __shared__ uint32_t warp_top[TPR / 32];
  pdl_wait();
  pdl_launch();
  const int row = blockIdx.x * (kBlock<TPR> / TPR) + threadIdx.x / TPR, t = threadIdx.x % TPR;
  const bool live = row < M;
  const T* xr = x + (long long)row * x_stride;
  int8_t* qr = q + (long long)row * K;
  constexpr int N = VEC ? Chunk<T>::N : 1;
  const int chunks = live ? K / N : 0;
  uint4 keep[VEC ? kKeep : 1];
  uint32_t top = 0;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (t + i * TPR < chunks) keep[i] = reinterpret_cast<const uint4*>(xr)[t + i * TPR];
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (t + i * TPR < chunks)
        top = max(top, Chunk<T>::top(keep[i]));
    for (int c = t + kKeep * TPR; c < chunks; c += TPR) {
      const uint4 u = reinterpret_cast<const uint4*>(xr)[c];
      top = max(top, Chunk<T>::top(u));
    }
  } else {
    for (int c = t; c < chunks; c += TPR) top = max(top, abs_bits(to_f32(xr[c])));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if (TPR > 32) {
    if ((threadIdx.x & 31) == 0) warp_top[threadIdx.x >> 5] = top;
    __syncthreads();
    top = warp_top[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; ++w) top = max(top, warp_top[w]);
  }
  if (!live) return;
  const RowScale s = row_scale_of(top);
  if (t == 0) scale[row] = s.bad ? __uint_as_float(0x7fc00000u) : s.top / 127.f;
  if constexpr (VEC) {
    auto store = [&](int c, const uint4& u) {
      uint32_t w[N / 4];
#pragma unroll
      for (int g = 0; g < N / 4; ++g) w[g] = four<T>(u, g, s);
      if constexpr (N == 8) reinterpret_cast<uint2*>(qr)[c] = make_uint2(w[0], w[1]);
      else reinterpret_cast<uint32_t*>(qr)[c] = w[0];
    };
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (t + i * TPR < chunks) store(t + i * TPR, keep[i]);
    for (int c = t + kKeep * TPR; c < chunks; c += TPR) store(c, reinterpret_cast<const uint4*>(xr)[c]);
  } else {
    for (int c = t; c < chunks; c += TPR) {
      const float x = to_f32(xr[c]), r = fmaf(x, s.inv, 12582912.f);
      const bool near = !(fabsf(fmaf(x, s.inv, 12582912.f - r)) <= 0.4999f) || s.top < 1e-30f || s.bad;
      qr[c] = (int8_t)(near ? to_i8_exact(x, s) : __float_as_int(r));
    }
  }
}

template <typename T>
void launch_t(const T* x, long long x_stride, int M, int K, int8_t* q, float* scale, cudaStream_t st) {
  constexpr int N = Chunk<T>::N;
  const bool vec = K % N == 0 && x_stride % N == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)q & (N - 1)) == 0;
  // threads per row: as few as have four chunks each, at most 256 (16,008 rows of 11,008: 110 us with 256 threads, 132 with 512); what a row has
  // beyond kKeep chunks per thread is read again
  const int chunks = K / (vec ? N : 1);
  const auto go = [&](auto tpr, auto v) {
    constexpr int TPR = decltype(tpr)::value;
    constexpr int kRows = kBlock<TPR> / TPR;
    launch_pdl(quantize_rows_kernel<T, TPR, decltype(v)::value>, dim3((M + kRows - 1) / kRows), dim3(kBlock<TPR>), 0, st, x, x_stride, M, K, q, scale);
  };
  const auto pick = [&](auto v) {
    if (chunks <= 32 * 4) go(std::integral_constant<int, 32>{}, v);
    else if (chunks <= 128 * 4) go(std::integral_constant<int, 128>{}, v);
    else go(std::integral_constant<int, 256>{}, v);
  };
  if (vec) pick(std::true_type{});
  else pick(std::false_type{});
}

}  // namespace

void launch_quantize_rows(const void* x, long long x_stride, int M, int K, int8_t* q, float* scale, bool bf16, cudaStream_t st) {
  LaunchScope ls(kcMisc, st);
  if (bf16) launch_t((const __nv_bfloat16*)x, x_stride, M, K, q, scale, st);
  else launch_t((const float*)x, x_stride, M, K, q, scale, st);
}

}  // namespace nz
