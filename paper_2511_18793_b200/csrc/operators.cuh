// The operators over a paged context cache and the 8-bit projections: argument structs, launchers, and what their kernels share.
#pragma once

#include "common.cuh"

namespace nz {

// --------------------------------------------------------------------------------------------------
// paged context cache
// --------------------------------------------------------------------------------------------------
// nezha_paged_kv as the kernels take it.
struct PagedView {
  void *k, *v;
  long long page_stride, head_stride, pos_stride;
  int n_pages, page_size, Hkv, hd;
  const int* table; long long table_stride;
  int max_pages, batch;
  const int *row_start, *kv_len;
  int rows, max_new, max_kv;
  int* status;
};

// One sequence of a call: its first new row, how many there are, and its positions.  Contents that the caller's bounds do not
// cover are reported and make it a sequence without rows.
struct PagedSeq { int row0, n, len; };
__device__ __forceinline__ PagedSeq paged_seq(const PagedView& p, int b, bool report) {
  const int r0 = p.row_start[b], r1 = p.row_start[b + 1], len = p.kv_len[b];
  if (r0 < 0 || r1 < r0 || r1 > p.rows || r1 - r0 > p.max_new || len < 0 || len > p.max_kv) {
    if (report) atomicOr(p.status, kStBadPage);
    return PagedSeq{0, 0, 0};
  }
  return PagedSeq{r0, r1 - r0, len};
}

struct AppendArgs {
  PagedView kv;
  const void* q; long long q_stride; int Hq; void* q_out; long long q_out_stride;
  const void* k; long long k_stride; const void* v; long long v_stride;
  int rot, interleaved; const float* table; int n_table; const int* positions;
};
void launch_kv_append(const AppendArgs& a, bool bf16, cudaStream_t st);

// Rotary frequencies of a nezha_rope (rot_dim / 2 of them, at most 64) and the magnitude of cosine and sine.
struct RopeFrequencies { double f[64]; double magnitude; int half; };
void launch_rope_table(const RopeFrequencies& f, float* table, int n_positions, cudaStream_t st);

struct PagedAttnArgs {
  PagedView kv;
  const void* q; long long q_stride; void* out; long long out_stride; float* lse;
  int Hq, G;                        // query heads, and query heads per KV head
  float scale, softcap; const float* slopes;
  int causal, window;
  // A context split over CTAs: split s has the tiles [s, s + 1) * split_tiles of its sequence (tiles of kAttnTile positions) and leaves
  // its normalised fp32 output [splits][rows * Hq][hd] and the base-2 log of its sum [splits][rows * Hq] (-inf: it saw nothing).
  int splits, split_tiles;
  float *part_o, *part_lse;
};
constexpr int kAttnTile = 64;       // positions per unit of a split

// Positions [lo, hi) that the row at position p sees of a sequence of len positions.
struct Visible { int lo, hi; };
__device__ __forceinline__ Visible visible(const PagedAttnArgs& a, int p, int len) {
  Visible v{0, len};
  if (a.causal) {
    v.hi = min(len, p + 1);
    if (a.window > 0) v.lo = max(0, max(p, 0) - a.window + 1);      // (p may be far below 0: p - window would wrap round)
  }
  if (v.hi < v.lo) v.hi = v.lo;
  return v;
}

// A CTA's place in a launch of Hkv x row tiles x splits x sequences CTAs: KV heads fastest, so that neighbours share a sequence's pages' table.
struct AttnCta { int kvh, tile, split, b; };
__device__ __forceinline__ AttnCta attn_cta(const PagedAttnArgs& a, int row_tiles) {
  unsigned i = blockIdx.x;
  AttnCta c;
  c.kvh = (int)(i % (unsigned)a.kv.Hkv); i /= (unsigned)a.kv.Hkv;
  c.tile = (int)(i % (unsigned)row_tiles); i /= (unsigned)row_tiles;
  c.split = (int)(i % (unsigned)a.splits);
  c.b = (int)(i / (unsigned)a.splits);
  return c;
}

// How a call is served; a function of its sizes alone (the workspace's too).
struct PagedAttnPlan { int kernel; int splits, split_tiles; size_t bytes; };
PagedAttnPlan paged_attn_plan(const PagedAttnArgs& a, bool bf16);
void launch_paged_attention(const PagedAttnArgs& a, const PagedAttnPlan& plan, bool bf16, cudaStream_t st);

// --------------------------------------------------------------------------------------------------
// 8-bit projections
// --------------------------------------------------------------------------------------------------
void launch_quantize_rows(const void* x, long long x_stride, int M, int K, int8_t* q, float* scale, bool bf16, int* status, cudaStream_t st);

struct GemmI8Args {
  const int8_t *A, *W; const float *a_scale, *w_scale, *bias;
  void* C;
  int M, N, K, epilogue;            // kEpiStoreAct, kEpiStoreF32, kEpiAddF32
  int* status;
};
// One element of C before it is stored: the same roundings in every kernel.
__device__ __forceinline__ float i8_value(int acc, float sa, float sw, float bias) {
  return __fadd_rn(__fmul_rn(__fmul_rn((float)acc, sa), sw), bias);
}
void launch_gemm_i8(const GemmI8Args& a, bool bf16, cudaStream_t st);

}  // namespace nz
