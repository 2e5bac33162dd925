// Rows to 8-bit integers with a scale each:  scale = max|x| / 127,  q = 127 x / max|x| to the nearest, halves to even.
//
// One read of x and one write of q bound it: a row's chunks stay in registers between the two (up to kKeep per thread; what a longer row
// has beyond is read again, from the L2), or, of many rows, in shared memory.  The maximum is taken over the bit patterns of |x|, in which a NaN is above
// infinity and that above all numbers.  x * (127 / max) is off by less than 1e-4 of a step, so a quotient that near to a border
// is divided in 64 bits, where a half is a half: a value half as large as the row's largest lies on the border 63.5 exactly.
#include <algorithm>
#include <type_traits>

#include "operators.cuh"
#include "tma.cuh"

namespace nz {

int sm_count();

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

// Many rows: a CTA per SM, whose groups of TPR threads take a row each in turn.  A group has a ring of `stages` rows in shared memory that bulk copies fill ahead
// of it, so that loads are in flight all the time (in the kernel above a CTA's loads, its maximum and its stores follow one another, with a new CTA for every
// row), and reads a row there twice.  16,008 rows of 11,008 values of 16 bits: 86 us, 94 % of the copy bandwidth (110 above); of 8,192 68 (94), of 2,048 28 (34).
// Below kStreamMin bytes its start costs more than it saves: 8,000 rows of 2,048 16 us (19 above), 2,000 of 4,096 11 (10).
constexpr int kStreamThreads = 1024, kStreamBytes = 200 * 1024, kMaxStages = 8;
constexpr long long kStreamMin = 32000000;          // bytes of x
template <int TPR> constexpr int kGroups = kStreamThreads / TPR;
template <int TPR> constexpr int kStreamHead = kGroups<TPR> * (2 * kMaxStages + 1) * 8 + 2 * (kStreamThreads / 32) * 4 + 16;      // barriers, maxima, flag

template <typename T, int TPR>
__global__ void __launch_bounds__(kStreamThreads, 1) quantize_stream_kernel(const T* __restrict__ x, long long x_stride, int M, int K, int8_t* __restrict__ q,
                                                                            float* __restrict__ scale, int stages, int* status) {
  constexpr int N = Chunk<T>::N, kWarps = TPR / 32, G = kGroups<TPR>;
  extern __shared__ __align__(128) uint8_t smem[];
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, lane = threadIdx.x & 31;
  const uint32_t bars = smem_u32(smem) + (uint32_t)(group * (2 * kMaxStages + 1)) * 8u;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kMaxStages + s); };
  const uint32_t top_bar = bars + 8u * (2 * kMaxStages);      // the group's maxima are written
  uint32_t* tops = reinterpret_cast<uint32_t*>(smem + G * (2 * kMaxStages + 1) * 8) + group * 2 * kWarps;
  volatile uint32_t* abort_flag = reinterpret_cast<uint32_t*>(smem + G * (2 * kMaxStages + 1) * 8) + 2 * (kStreamThreads / 32);
  const uint32_t row_bytes = (uint32_t)K * sizeof(T);
  uint8_t* ring = smem + (kStreamHead<TPR> + 127) / 128 * 128 + (size_t)group * stages * row_bytes;
  if (threadIdx.x == 0) *abort_flag = 0;
  if (t == 0) {
    for (int s = 0; s < stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), kWarps); }
    mbar_init(top_bar, kWarps);
    mbar_fence_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_launch();
  const int first = blockIdx.x * G + group, step = gridDim.x * G, rows = first < M ? (M - 1 - first) / step + 1 : 0;
  auto bring = [&](int i) {
    const uint32_t bar = full_bar(i % stages);
    mbar_expect_tx(bar, row_bytes);
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(ring + (size_t)(i % stages) * row_bytes)),
                 "l"(x + (long long)(first + (long long)i * step) * x_stride), "r"(row_bytes), "r"(bar) : "memory");
  };
  int brought = min(stages, rows), i = 0;
  if (t == 0)
    for (int k = 0; k < brought; ++k) bring(k);
  bool ok = true;
  const int chunks = K / N;
  for (; i < rows; ++i) {
    const int s = i % stages, row = first + i * step;
    ok = warp_wait_uniform(full_bar(s), (uint32_t)(i / stages) & 1u, abort_flag);
    if (!ok) break;
    const uint4* xs = reinterpret_cast<const uint4*>(ring + (size_t)s * row_bytes);
    uint32_t top = 0;
#pragma unroll 4
    for (int c = t; c < chunks; c += TPR) top = max(top, Chunk<T>::top(xs[c]));
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (kWarps > 1) {
      uint32_t* mine = tops + (i & 1) * kWarps;      // (two sets: a warp that is a row ahead does not overwrite what others still read)
      if (lane == 0) {
        mine[t / 32] = top;
        mbar_arrive(top_bar);
      }
      __syncwarp();
      ok = warp_wait_uniform(top_bar, (uint32_t)i & 1u, abort_flag);
      if (!ok) break;
      top = __reduce_max_sync(0xffffffffu, lane < kWarps ? mine[lane] : 0u);
    }
    const RowScale rs = row_scale_of(top);
    if (t == 0) scale[row] = rs.bad ? __uint_as_float(0x7fc00000u) : rs.top / 127.f;
    int8_t* qr = q + (long long)row * K;
#pragma unroll 2
    for (int c = t; c < chunks; c += TPR) {
      const uint4 u = xs[c];
      if constexpr (N == 8) reinterpret_cast<uint2*>(qr)[c] = make_uint2(four<T>(u, 0, rs), four<T>(u, 1, rs));
      else reinterpret_cast<uint32_t*>(qr)[c] = four<T>(u, 0, rs);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty_bar(s));
    if (t < 32 && brought < rows) {                  // the next row into the place of this one
      ok = warp_wait_uniform(empty_bar(s), (uint32_t)(i / stages) & 1u, abort_flag);
      if (!ok) break;
      if (t == 0) bring(brought);
      ++brought;
    }
  }
  if (!ok && lane == 0) {
    *abort_flag = 1;
    atomicOr(status, kStInternal);
    if (t == 0)                                      // the copies in flight land before the CTA's memory goes away
      for (int k = i; k < brought; ++k) mbar_wait(full_bar(k % stages), (uint32_t)(k / stages) & 1u);
  }
}

// Rows that the ring has room for, two per group and more; false: not launched.
template <typename T, int TPR>
bool launch_stream(const T* x, long long x_stride, int M, int K, int8_t* q, float* scale, int* status, cudaStream_t st) {
  const size_t row_bytes = (size_t)K * sizeof(T);
  const int stages = (int)std::min<size_t>(kMaxStages, kStreamBytes / (kGroups<TPR> * row_bytes));
  if (stages < 2) return false;
  static PerDeviceOnce configured;
  configured.run([] { cudaFuncSetAttribute(quantize_stream_kernel<T, TPR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamBytes + kStreamHead<TPR> + 128); });
  launch_pdl(quantize_stream_kernel<T, TPR>, dim3((unsigned)std::min(sm_count(), (M - 1) / kGroups<TPR> + 1)), dim3(kStreamThreads),
             (size_t)stages * kGroups<TPR> * row_bytes + kStreamHead<TPR> + 128, st, x, x_stride, M, K, q, scale, stages, status);
  return true;
}

template <typename T>
void launch_t(const T* x, long long x_stride, int M, int K, int8_t* q, float* scale, int* status, cudaStream_t st) {
  constexpr int N = Chunk<T>::N;
  const bool vec = K % N == 0 && x_stride % N == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)q & (N - 1)) == 0;
  // threads per row: as few as have four chunks each, at most 256 (16,008 rows of 11,008: 110 us with 256 threads, 132 with 512); what a row has
  // beyond kKeep chunks per thread is read again
  const int chunks = K / (vec ? N : 1);
  // (in the ring: as few threads per row as leave every group two rows; rows of more than 100 KiB have no room)
  const auto stream = [&](auto tpr) { return launch_stream<T, decltype(tpr)::value>(x, x_stride, M, K, q, scale, status, st); };
  if (vec && (long long)M * K * (long long)sizeof(T) >= kStreamMin &&
      (stream(std::integral_constant<int, 32>{}) || stream(std::integral_constant<int, 128>{}) || stream(std::integral_constant<int, 256>{}) ||
       stream(std::integral_constant<int, 512>{}) || stream(std::integral_constant<int, 1024>{})))
    return;
  const auto go = [&](auto tpr, auto v) {
    constexpr int TPR = decltype(tpr)::value;
    constexpr int kRows = kBlock<TPR> / TPR;
    launch_pdl(quantize_rows_kernel<T, TPR, decltype(v)::value>, dim3((M - 1) / kRows + 1), dim3(kBlock<TPR>), 0, st, x, x_stride, M, K, q, scale);
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

void launch_quantize_rows(const void* x, long long x_stride, int M, int K, int8_t* q, float* scale, bool bf16, int* status, cudaStream_t st) {
  LaunchScope ls(kcMisc, st);
  if (bf16) launch_t((const __nv_bfloat16*)x, x_stride, M, K, q, scale, status, st);
  else launch_t((const float*)x, x_stride, M, K, q, scale, status, st);
}

}  // namespace nz
