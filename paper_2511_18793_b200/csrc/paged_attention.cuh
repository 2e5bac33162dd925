// What the two tensor-core kernels over a paged cache share: the copy of a tile of pages into shared memory, and the scores' forms.
#pragma once

#include "operators.cuh"
#include "tma.cuh"

namespace nz {

// K and V pools as 4-D tensors {head_dim, page_size, KV heads, pages}; box = 64 columns x `box_rows` positions, 128-byte swizzle.
// A box lies within a page: box_rows is the largest power of two, at most 64, that divides the page size (at least 8, which is where
// the swizzle repeats).  Coordinates outside the pool read as zeros.
inline int paged_box_rows(int page_size) {
  int r = 1;
  while (r < 64 && page_size % (2 * r) == 0) r *= 2;
  return r;
}
inline bool paged_map(const PagedView& p, const void* pool, int box_rows, CUtensorMap* out) {
  if (!tma_encode_fn()) return false;
  cuuint64_t dims[4] = {(cuuint64_t)p.hd, (cuuint64_t)p.page_size, (cuuint64_t)p.Hkv, (cuuint64_t)p.n_pages};
  // (an extent of one step may come with any stride: 16 bytes stand in for it)
  cuuint64_t strides[3] = {p.page_size == 1 ? 16 : (cuuint64_t)p.pos_stride * 2, p.Hkv == 1 ? 16 : (cuuint64_t)p.head_stride * 2,
                           p.n_pages == 1 ? 16 : (cuuint64_t)p.page_stride * 2};
  for (cuuint64_t s : strides)
    if (s >= 1ull << 40) return false;
  cuuint32_t box[4] = {64u, (cuuint32_t)box_rows, 1, 1}, estr[4] = {1, 1, 1, 1};
  return tma_encode_fn()(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace paged_detail {

__device__ __forceinline__ void tma_load_4d_if(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, int w, uint32_t bar, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %7, 0;\n\t"
      "@q cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
      ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "r"(leader) : "memory");
}
// A barrier's phase, asked for once without waiting.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {       // zeros where there is nothing to read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {      // counts as one arrival once this thread's copies have landed
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {      // 2^x, flushing; ex2(-inf) = 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The page of position t of sequence b where some row of the CTA sees it (lo <= t < hi), else one outside the pool, whose positions
// read as zeros; so does a bad one, which is reported.
__device__ __forceinline__ int page_of(const PagedView& kv, int b, int t, int n, int lo, int hi) {
  if (t + n <= lo || t >= hi) return kv.n_pages;
  const int page = kv.table[(long long)b * kv.table_stride + t / kv.page_size];
  if (page < 0 || page >= kv.n_pages) { atomicOr(kv.status, kStBadPage); return kv.n_pages; }
  return page;
}

// Eight bf16 values: is one of them infinite or not a number; and with zeros in the place of those.  (An exponent of ones is the only one that a further
// step carries into the sign's bit.)
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ bool any_odd(const uint4& x) { return (odd_bits(x.x) | odd_bits(x.y) | odd_bits(x.z) | odd_bits(x.w)) != 0u; }
__device__ __forceinline__ uint32_t without_odd(uint32_t w) {
  const uint32_t o = odd_bits(w);
  return w & ~((o >> 15) * 0xffffu);
}
__device__ __forceinline__ uint4 without_odd(const uint4& x) { return make_uint4(without_odd(x.x), without_odd(x.y), without_odd(x.z), without_odd(x.w)); }

// tanh to about 2e-7 absolute (relative below 1/4, by its series: a cap far above the scores must not cost them digits).
__device__ __forceinline__ float tanh_fast(float y) {
  const float z = y * y;
  const float small = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
  const float e = ex2(2.f * 1.4426950408889634f * y);
  const float large = 1.f - __fdividef(2.f, 1.f + e);
  return fabsf(y) < 0.25f ? small : large;
}

}  // namespace paged_detail
}  // namespace nz
