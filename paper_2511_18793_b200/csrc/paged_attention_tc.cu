// Attention over a paged cache on mma.sync (bf16, heads of 64 and 128): calls of few query rows, which are bound by reading keys and values
// once, and what the tcgen05 kernel does not take (page sizes that are no multiple of 8, caps that its series does not bear).
//
// A CTA has one (sequence, KV head), a tile of 16 RW query rows (tokens times the heads of the group) and a share of the context.  A producer
// warp brings tiles of 64 positions into a ring: by TMA, one box of 64 columns per page or piece of a page, where the page size is a
// multiple of 8, else 16 bytes at a time (cp.async), positions that no row sees as zeros.  RW row warps x KW position groups compute
// S = Q K^T and O += P V in registers with a running maximum and sum; the KW groups take every KW-th tile and are merged at the end.
// 9 to 16 rows: RW = 1, KW = 2, 64 KB of ring; three CTAs per SM with heads of 64, two with heads of 128, whose 208 registers a thread (plain; 247 capped or
// biased) leave room for eight warps.  One token of 16 heads of 128 on one, 64 sequences on up to 4,000 positions: 31 us, floor 13 (the bytes).
// 17 to 64 rows: RW = 4, KW = 1.  Ten tokens of 32 heads on 8, 32 sequences on up to 4,000 positions: heads of 128 130 us, floor 55; heads of 64 64, 28.
// At most 8 rows (the last kernel here): three CTAs per SM -- a warp's chain (scores, softmax, second product) takes about as long as a tile's way from HBM,
// so six or more of them per SM keep the memory busy.  64 tokens of 32 heads of 128 on 8, on up to 4,000 positions in pages of 16: 126 us, 5.5 TB/s of the
// copy's 6.5 (113 with a warm L2; pages of 20, by 16-byte copies: 212); one token on 32k positions, heads of 64: 24 us with the join, of which the stream is 10.
//
// What a row does not see has no part in its sums: scores are replaced, not added to; values at positions outside what the CTA's rows see
// are zeroed in the tile, and where only some of its rows see a position, values that are not finite are taken out of the tile and added to
// the rows that see them at the end (what 0 x infinity would spread to the others).  Waits are bounded as everywhere.
#include <math.h>
#include <stdlib.h>

#include "paged_attention.cuh"

namespace nz {

namespace {

using namespace paged_detail;

constexpr int kPos = kAttnTile;

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr));
}
__device__ __forceinline__ void mma_bf16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
// 16-byte chunk `chunk` of position `pos` of a tile made of HD / 64 sub-tiles of 64 positions x 128 bytes, 128-byte swizzle.
__device__ __forceinline__ uint32_t kv_off(int pos, int chunk) { return (chunk >> 3) * (kPos * 128) + pos * 128 + (((chunk & 7) ^ (pos & 7)) << 4); }

// A tile of V on the edge of what the CTA's rows see, by the warp that is about to use it: positions that no row sees become zeros, and where some rows do not
// see a position (outside [c_lo, c_hi)) its values that are not finite do, which odd_flag tells.
template <int HD>
__device__ __forceinline__ void clear_values(uint8_t* v, int p0, int u_lo, int u_hi, int c_lo, int c_hi, volatile uint32_t* odd_flag) {
  constexpr int CH = HD / 8;
  for (int i = threadIdx.x & 31; i < kPos * CH; i += 32) {
    const int p = p0 + i / CH;
    if (p >= c_lo && p < c_hi) continue;
    uint4* at = reinterpret_cast<uint4*>(v + kv_off(i / CH, i % CH));
    if (p < u_lo || p >= u_hi) { *at = make_uint4(0u, 0u, 0u, 0u); continue; }
    if (any_odd(*at)) { *at = without_odd(*at); *odd_flag = 1; }
  }
  __syncwarp();
}

// The producer warp of a CTA: the NT tiles of sequence b and KV head kvh from tile t_begin on, S slots of {K, V}; `full` and `empty` barriers as in the kernels.
template <int HD, int S, bool PAGES>
__device__ __forceinline__ void produce(const CUtensorMap& tmK, const CUtensorMap& tmV, const PagedAttnArgs& a, int b, int kvh, uint32_t base, uint32_t bar_base,
                                        volatile uint32_t* abort_flag, int t_begin, int NT, int u_lo, int u_hi, int box_rows) {
  constexpr int kTileBytes = kPos * HD * 2, NH = HD / 64, CH = HD / 8;
  const int lane = threadIdx.x & 31;
  auto full_bar = [&](int kv, int s) { return bar_base + 8u * (2 * s + kv); };
  auto empty_bar = [&](int kv, int s) { return bar_base + 8u * (2 * (S + s) + kv); };
  // Two rings, whichever has a free slot is served: a K slot is free again after the scores, its V slot only at the end of the tile (one ring of
  // pairs: 64 tokens on up to 4,000 positions 142 us).  The boxes of all tiles are numbered through; a lane looks up the page of one box in 32, for each ring,
  // 32 boxes ahead (looked up tile by tile, a page's way from memory was in every tile's: 64 tokens, heads of 64, 4,000 positions 120 us).
  const uint32_t leader = elect_one();
  const int nb = PAGES ? kPos / box_rows : 0;
  int t[2] = {0, 0}, y[2], page[2] = {0, 0}, next[2] = {0, 0};      // the next tile of each ring, its place in its page; pages of this and the next 32 boxes
  auto look_up = [&](int box) {
    box += lane;
    return box < NT * nb ? page_of(a.kv, b, t_begin * kPos + box * box_rows, box_rows, u_lo, u_hi) : 0;
  };
  if constexpr (PAGES) {
    y[0] = y[1] = t_begin * kPos % a.kv.page_size;
    page[0] = page[1] = look_up(0);
    next[0] = next[1] = look_up(32);
  }
  bool ok = true;
  long long since = clock64();
  while (t[0] < NT || t[1] < NT) {
    bool served = false;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const int s = t[kv] % S;
      if (t[kv] >= NT || (t[kv] >= S && !__all_sync(0xffffffffu, mbar_test(empty_bar(kv, s), ((t[kv] / S) - 1) & 1)))) continue;
      const uint32_t dst = base + s * 2 * kTileBytes + kv * kTileBytes, bar = full_bar(kv, s);
      if constexpr (PAGES) {
        mbar_expect_tx_if(bar, kTileBytes, leader);
        const int first = t[kv] * nb;
        if (t[kv] > 0 && (first & 31) == 0) { page[kv] = next[kv]; next[kv] = look_up(first + 32); }      // (nb divides 32)
        for (int i = 0; i < nb; ++i) {
          const int pg = __shfl_sync(0xffffffffu, page[kv], (first + i) & 31);
#pragma unroll
          for (int h = 0; h < NH; ++h) tma_load_4d_if(dst + h * (kPos * 128) + i * box_rows * 128, kv ? &tmV : &tmK, h * 64, y[kv], kvh, pg, bar, leader);
          y[kv] += box_rows;
          if (y[kv] >= a.kv.page_size) y[kv] -= a.kv.page_size;
        }
      } else {
        for (int i = 0; i < kPos; i += 32) {       // a lane looks a position up, the warp copies the 32 of them
          const int p = (t_begin + t[kv]) * kPos + i + lane;
          const int pg = page_of(a.kv, b, p, 1, u_lo, u_hi);
          const long long at = pg * a.kv.page_stride + kvh * a.kv.head_stride + (long long)(p % a.kv.page_size) * a.kv.pos_stride;
          const __nv_bfloat16* pool = (const __nv_bfloat16*)(kv ? a.kv.v : a.kv.k);
          for (int j = 0; j < 32; j += 32 / CH) {
            const int from = j + lane / CH, c = lane % CH;
            const long long src = __shfl_sync(0xffffffffu, at, from) + c * 8;
            const bool real = __shfl_sync(0xffffffffu, pg, from) < a.kv.n_pages;
            cp_async16(dst + kv_off(i + from, c), pool + (real ? src : 0), real);
          }
        }
        cp_async_arrive(bar);
      }
      ++t[kv];
      served = true;
    }
    if (served) since = clock64();
    else if (__any_sync(0xffffffffu, *abort_flag || clock64() - since > kWaitCycles)) { ok = false; break; }
  }
  if (!ok) {                                       // the copies in flight land before the CTA's memory goes away
    if (lane == 0) *abort_flag = 1;
    for (int kv = 0; kv < 2; ++kv)
      for (int j = max(0, t[kv] - S); j < t[kv]; ++j) mbar_wait(full_bar(kv, j % S), (j / S) & 1);
  }
}

template <int HD, int RW, int KW>
struct Cfg {
  static constexpr int kTileBytes = kPos * HD * 2;
  static constexpr int kStages = KW == 1 ? (HD == 64 ? 4 : 3) : (HD == 64 ? 4 : 2);    // a multiple of KW
  static constexpr int kThreads = (RW * KW + 1) * 32;
  static constexpr int kMergeFloats = (HD / 8) * 4 + 4;
  static constexpr int kRingBytes = kStages * 2 * kTileBytes;
  static constexpr int kSmemBytes = kRingBytes + 1024 + 256;
  static_assert((KW - 1) * RW * kMergeFloats * 32 * 4 <= kRingBytes, "the merge uses the ring");
};

// FORM: capped scores or a distance bias.  PAGES: TMA (else cp.async).  a.splits parts of the context in workspace if above 1.
template <int HD, int RW, int KW, bool FORM, bool PAGES>
__global__ void __launch_bounds__(Cfg<HD, RW, KW>::kThreads) paged_attn_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                                 PagedAttnArgs a, int row_tiles, int box_rows) {
  using C = Cfg<HD, RW, KW>;
  constexpr int S = C::kStages, KS = HD / 16, NB = HD / 8, NH = HD / 64, CH = HD / 8;
  constexpr int kRows = 16 * RW;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar_base = base + C::kRingBytes;
  // slot s of the K ring (kv 0) and of the V ring (kv 1)
  auto full_bar = [&](int kv, int s) { return bar_base + 8u * (2 * s + kv); };
  auto empty_bar = [&](int kv, int s) { return bar_base + 8u * (2 * (S + s) + kv); };
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(gen_base + C::kRingBytes + 32 * S);
  volatile uint32_t* odd_flag = abort_flag + 1;      // a value that is not finite was taken out of a tile
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s)
      for (int kv = 0; kv < 2; ++kv) { mbar_init(full_bar(kv, s), PAGES ? 1 : 32); mbar_init(empty_bar(kv, s), RW); }
    *abort_flag = 0; *odd_flag = 0;
    mbar_fence_init();
    if (PAGES) { tma_prefetch_map(&tmK); tma_prefetch_map(&tmV); }
  }
  __syncthreads();
  pdl_wait();
  pdl_launch();
  const AttnCta cta = attn_cta(a, row_tiles);
  const int kvh = cta.kvh, b = cta.b, split = cta.split;
  const PagedSeq sq = paged_seq(a.kv, b, kvh == 0 && cta.tile == 0 && split == 0 && threadIdx.x == 0);
  const int G = a.G, R = sq.n * G, r0 = cta.tile * kRows;
  if (r0 >= R) return;
  const int first_p = sq.len - sq.n;
  // what the tile's rows see between them (u_lo, u_hi), and what all of them see (the part between c_lo and c_hi)
  const Visible v0 = visible(a, first_p + r0 / G, sq.len), v1 = visible(a, first_p + min(r0 + kRows - 1, R - 1) / G, sq.len);
  const int u_lo = v0.lo, u_hi = v1.hi, c_lo = v1.lo, c_hi = v0.hi;
  int t_begin = u_lo / kPos, t_end = (u_hi + kPos - 1) / kPos;
  if (a.splits > 1) {
    t_begin = max(t_begin, split * a.split_tiles);
    t_end = min(t_end, (split + 1) * a.split_tiles);
  }
  const int NT = max(0, t_end - t_begin);

  float o[NB][4];
  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};   // m in the scaled log2 domain
  const int qr = lane >> 2, qc = lane & 3;
  const int rw = warp % RW, g = warp / RW;
  int tok[2] = {0, 0}, head[2] = {0, 0}, pos[2] = {0, 0};
  Visible vis[2];
  bool live[2] = {false, false};
  const float sc = a.scale * 1.4426950408889634f;

  if (warp == RW * KW) {
    // ------------------------------------------------------------------ producer
    produce<HD, S, PAGES>(tmK, tmV, a, b, kvh, base, bar_base, abort_flag, t_begin, NT, u_lo, u_hi, box_rows);
  } else {
    // ------------------------------------------------------------------ consumers
    float slope[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = r0 + rw * 16 + qr + i * 8;
      live[i] = row < R;
      const int rr = live[i] ? row : r0;             // dead rows shadow the tile's first row (never stored)
      tok[i] = sq.row0 + rr / G;
      head[i] = kvh * G + rr % G;
      pos[i] = first_p + rr / G;
      vis[i] = visible(a, pos[i], sq.len);
      if (FORM && a.slopes) slope[i] = a.slopes[head[i]];
    }
    uint32_t qf[KS][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __nv_bfloat16* qp = (const __nv_bfloat16*)a.q + (long long)tok[i] * a.q_stride + (long long)head[i] * HD + qc * 2;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks][i] = *reinterpret_cast<const uint32_t*>(qp + ks * 16);
        qf[ks][i + 2] = *reinterpret_cast<const uint32_t*>(qp + ks * 16 + 8);
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) { o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f; }
    for (int tl = g; tl < NT; tl += KW) {
      const int s = tl % S, p0 = (t_begin + tl) * kPos;
      if (!warp_wait_uniform(full_bar(0, s), (tl / S) & 1, abort_flag)) { if (lane == 0) *abort_flag = 1; break; }
      const uint32_t kt = base + s * 2 * C::kTileBytes, vt = kt + C::kTileBytes;
      const bool edge = p0 < c_lo || p0 + kPos > c_hi;    // some row does not see all of the tile
      // ---- S = Q K^T (16 rows x 64 positions per warp); rows qr and qr + 8, columns j * 8 + qc * 2 + {0, 1}
      float x[8][4];
#pragma unroll
      for (int j = 0; j < 8; ++j) { x[j][0] = x[j][1] = x[j][2] = x[j][3] = 0.f; }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int jp = 0; jp < 4; ++jp) {
          const int m = lane >> 3;
          uint32_t b0, b1, b2, b3;
          ldsm_x4(kt + kv_off(jp * 16 + (m >> 1) * 8 + (lane & 7), ks * 2 + (m & 1)), b0, b1, b2, b3);
          mma_bf16(x[jp * 2], qf[ks], b0, b1);
          mma_bf16(x[jp * 2 + 1], qf[ks], b2, b3);
        }
      // what this warp read is in its registers when the slot is given back
      __threadfence_block();
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(0, s));
      if constexpr (FORM) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = x[j][e] * a.scale;
            if (a.softcap > 0.f) v = a.softcap * tanh_fast(__fdividef(v, a.softcap));
            v -= slope[e >> 1] * fabsf((float)(pos[e >> 1] - (p0 + j * 8 + qc * 2 + (e & 1))));
            x[j][e] = v * 1.4426950408889634f;
          }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j][e] *= sc;
      }
      if (edge) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int p = p0 + j * 8 + qc * 2 + (e & 1);
            if (p < vis[e >> 1].lo || p >= vis[e >> 1].hi) x[j][e] = -INFINITY;
          }
      }
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        mx[0] = fmaxf(mx[0], fmaxf(x[j][0], x[j][1]));
        mx[1] = fmaxf(mx[1], fmaxf(x[j][2], x[j][3]));
      }
      float corr[2], neg_m[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
        const float m_new = fmaxf(m_run[i], mx[i]);
        const float m_safe = m_new == -INFINITY ? 0.f : m_new;
        corr[i] = ex2(m_run[i] - m_safe);
        m_run[i] = m_new;
        neg_m[i] = -m_safe;
      }
      float rs[2] = {0.f, 0.f};
      uint32_t pf[4][4];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float p0_ = ex2(x[j][0] + neg_m[0]), p1_ = ex2(x[j][1] + neg_m[0]), p2_ = ex2(x[j][2] + neg_m[1]), p3_ = ex2(x[j][3] + neg_m[1]);
        rs[0] += p0_ + p1_; rs[1] += p2_ + p3_;
        pf[j >> 1][(j & 1) * 2] = pack_bf16(p0_, p1_);
        pf[j >> 1][(j & 1) * 2 + 1] = pack_bf16(p2_, p3_);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) l_run[i] = l_run[i] * corr[i] + rs[i];
#pragma unroll
      for (int j = 0; j < NB; ++j) { o[j][0] *= corr[0]; o[j][1] *= corr[0]; o[j][2] *= corr[1]; o[j][3] *= corr[1]; }
      if (!warp_wait_uniform(full_bar(1, s), (tl / S) & 1, abort_flag)) { if (lane == 0) *abort_flag = 1; break; }
      if (edge) clear_values<HD>(gen_base + (vt - base), p0, u_lo, u_hi, c_lo, c_hi, odd_flag);
      // ---- O += P V
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int np = 0; np < NB / 2; ++np) {
          const int m = lane >> 3;
          uint32_t b0, b1, b2, b3;
          ldsm_x4_t(vt + kv_off(ks * 16 + (m & 1) * 8 + (lane & 7), np * 2 + (m >> 1)), b0, b1, b2, b3);
          mma_bf16(o[np * 2], pf[ks], b0, b1);
          mma_bf16(o[np * 2 + 1], pf[ks], b2, b3);
        }
      // (and what it wrote ordered before the next copy)
      __threadfence_block();
      if (edge && PAGES) fence_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(1, s));
    }
    // every lane has summed its own columns: the row's sum is four lanes'
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l_run[i] += __shfl_xor_sync(0xffffffffu, l_run[i], 1);
      l_run[i] += __shfl_xor_sync(0xffffffffu, l_run[i], 2);
    }
  }
  __syncthreads();                                   // the ring is idle
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicOr(a.kv.status, kStInternal);
    return;
  }
  float* merge = reinterpret_cast<float*>(gen_base);
  if constexpr (KW > 1) {
    if (warp >= RW && warp < RW * KW) {
      float* dst = merge + (((g - 1) * RW + rw) * C::kMergeFloats) * 32 + lane;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) dst[(j * 4 + e) * 32] = o[j][e];
      dst[(NB * 4 + 0) * 32] = m_run[0]; dst[(NB * 4 + 1) * 32] = m_run[1];
      dst[(NB * 4 + 2) * 32] = l_run[0]; dst[(NB * 4 + 3) * 32] = l_run[1];
    }
    __syncthreads();
  }
  if (warp >= RW) return;
  if constexpr (KW > 1) {
#pragma unroll 1
    for (int og = 1; og < KW; ++og) {
      const float* src = merge + (((og - 1) * RW + rw) * C::kMergeFloats) * 32 + lane;
      float c_s[2], c_o[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float m_o = src[(NB * 4 + i) * 32], l_o = src[(NB * 4 + 2 + i) * 32];
        const float m_new = fmaxf(m_run[i], m_o), m_safe = m_new == -INFINITY ? 0.f : m_new;
        c_s[i] = ex2(m_run[i] - m_safe); c_o[i] = ex2(m_o - m_safe);
        l_run[i] = l_run[i] * c_s[i] + l_o * c_o[i];
        m_run[i] = m_new;
      }
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = o[j][e] * c_s[e >> 1] + src[(j * 4 + e) * 32] * c_o[e >> 1];
    }
  }
  if (*odd_flag) {
    // the values that were taken out, to the rows that see them
    for (int p = max(u_lo, t_begin * kPos); p < min(u_hi, t_end * kPos); ++p) {
      if (p >= c_lo && p < c_hi) { p = c_hi - 1; continue; }
      const int page = page_of(a.kv, b, p, 1, u_lo, u_hi);
      if (page >= a.kv.n_pages) continue;
      const __nv_bfloat16* v = (const __nv_bfloat16*)a.kv.v + page * a.kv.page_stride + kvh * a.kv.head_stride + (long long)(p % a.kv.page_size) * a.kv.pos_stride;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = __bfloat162float(v[j * 8 + qc * 2 + (e & 1)]);
          if (!(fabsf(y) < INFINITY) && p >= vis[e >> 1].lo && p < vis[e >> 1].hi) o[j][e] += y;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (!live[i]) continue;
    const bool none = l_run[i] == 0.f;
    const float inv = none ? 0.f : 1.f / l_run[i];
    if (a.splits > 1) {
      const long long at = ((long long)split * a.kv.rows + tok[i]) * a.Hq + head[i];
      if (qc == 0) a.part_lse[at] = none ? -INFINITY : m_run[i] + log2f(l_run[i]);
      if (none) continue;                            // (a part without weight is not read)
      float* op = a.part_o + at * HD + qc * 2;
#pragma unroll
      for (int j = 0; j < NB; ++j) *reinterpret_cast<float2*>(op + j * 8) = make_float2(o[j][i * 2] * inv, o[j][i * 2 + 1] * inv);
    } else {
      if (a.lse && qc == 0) a.lse[(long long)tok[i] * a.Hq + head[i]] = none ? -INFINITY : (m_run[i] + log2f(l_run[i])) * 0.6931471805599453f;
      __nv_bfloat16* op = (__nv_bfloat16*)a.out + (long long)tok[i] * a.out_stride + (long long)head[i] * HD + qc * 2;
#pragma unroll
      for (int j = 0; j < NB; ++j) *reinterpret_cast<__nv_bfloat162*>(op + j * 8) = __floats2bfloat162_rn(o[j][i * 2] * inv, o[j][i * 2 + 1] * inv);
    }
  }
}

// ---------------------------------------------------------------------------------------------------
// At most 8 query rows (a token of up to 8 heads per KV head): the products turned round, positions and dimensions as the 16 rows of m16n8k16 and the queries
// as its 8 columns -- S^T = K Q^T, O^T += V^T P^T, P^T through movmatrix -- which is half the instructions and half the registers.
// ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <int HD, int KW>
struct TokCfg {
  static constexpr int kTileBytes = kPos * HD * 2, kStages = KW == 2 ? 2 : 4, kThreads = (KW + 1) * 32;
  static constexpr int kRingBytes = kStages * 2 * kTileBytes, kSmemBytes = kRingBytes + 1024 + 256;
  static constexpr int kMergeFloats = 8 * HD + 16;             // a group's O [query][dim], maxima, sums
  static_assert(KW * kMergeFloats * 4 <= kRingBytes, "the merge uses the ring");
};

template <int HD, int KW, bool FORM, bool PAGES>
__global__ void __launch_bounds__(TokCfg<HD, KW>::kThreads, 3) paged_attn_token_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                                      PagedAttnArgs a, int box_rows) {
  using C = TokCfg<HD, KW>;
  constexpr int S = C::kStages, KS = HD / 16, DT = HD / 16, CH = HD / 8;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar_base = base + C::kRingBytes;
  auto full_bar = [&](int kv, int s) { return bar_base + 8u * (2 * s + kv); };
  auto empty_bar = [&](int kv, int s) { return bar_base + 8u * (2 * (S + s) + kv); };
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(gen_base + C::kRingBytes + 32 * S);
  volatile uint32_t* odd_flag = abort_flag + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s)
      for (int kv = 0; kv < 2; ++kv) { mbar_init(full_bar(kv, s), PAGES ? 1 : 32); mbar_init(empty_bar(kv, s), 1); }
    *abort_flag = 0; *odd_flag = 0;
    mbar_fence_init();
    if (PAGES) { tma_prefetch_map(&tmK); tma_prefetch_map(&tmV); }
  }
  __syncthreads();
  pdl_wait();
  pdl_launch();
  const AttnCta cta = attn_cta(a, 1);
  const int kvh = cta.kvh, b = cta.b, split = cta.split;
  const PagedSeq sq = paged_seq(a.kv, b, kvh == 0 && split == 0 && threadIdx.x == 0);
  const int G = a.G, R = sq.n * G;
  if (R == 0) return;
  const int first_p = sq.len - sq.n;
  const Visible v0 = visible(a, first_p, sq.len), v1 = visible(a, first_p + sq.n - 1, sq.len);
  const int u_lo = v0.lo, u_hi = v1.hi, c_lo = v1.lo, c_hi = v0.hi;      // what some of the rows see; what all of them see
  int t_begin = u_lo / kPos, t_end = (u_hi + kPos - 1) / kPos;
  if (a.splits > 1) {
    t_begin = max(t_begin, split * a.split_tiles);
    t_end = min(t_end, (split + 1) * a.split_tiles);
  }
  const int NT = max(0, t_end - t_begin);
  float* merge = reinterpret_cast<float*>(gen_base);

  if (warp == KW) {
    produce<HD, S, PAGES>(tmK, tmV, a, b, kvh, base, bar_base, abort_flag, t_begin, NT, u_lo, u_hi, box_rows);
    __syncthreads();                                 // (the consumers' two barriers)
    __syncthreads();
  } else {
    const int qr = lane >> 2, qc = lane & 3;         // fragment row (and + 8) / pair of columns: this lane's queries are 2 qc, 2 qc + 1
    float o[DT][4];
    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
    Visible vis[2];
    int pos[2];
    float slope[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = min(2 * qc + i, R - 1);        // queries that do not exist shadow the last (never stored)
      pos[i] = first_p + row / G;
      vis[i] = visible(a, pos[i], sq.len);
      if (FORM && a.slopes) slope[i] = a.slopes[kvh * G + row % G];
    }
    uint32_t qf[KS][2];
    {
      const int row = min(qr, R - 1);
      const __nv_bfloat16* qp = (const __nv_bfloat16*)a.q + (long long)(sq.row0 + row / G) * a.q_stride + (long long)(kvh * G + row % G) * HD + qc * 2;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks][0] = *reinterpret_cast<const uint32_t*>(qp + ks * 16);
        qf[ks][1] = *reinterpret_cast<const uint32_t*>(qp + ks * 16 + 8);
      }
    }
#pragma unroll
    for (int j = 0; j < DT; ++j) { o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f; }
    const float sc = a.scale * 1.4426950408889634f;
    for (int tl = warp; tl < NT; tl += KW) {
      const int s = tl % S, p0 = (t_begin + tl) * kPos;
      if (!warp_wait_uniform(full_bar(0, s), (tl / S) & 1, abort_flag)) { if (lane == 0) *abort_flag = 1; break; }
      const uint32_t kt = base + s * 2 * C::kTileBytes, vt = kt + C::kTileBytes;
      const bool edge = p0 < c_lo || p0 + kPos > c_hi;
      // ---- S^T = K Q^T: x[mt] = positions 16 mt + qr (and + 8), queries 2 qc (and + 1)
      float x[4][4];
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) { x[mt][0] = x[mt][1] = x[mt][2] = x[mt][3] = 0.f; }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
          const int m = lane >> 3;
          uint32_t f[4];
          ldsm_x4(kt + kv_off(mt * 16 + (m & 1) * 8 + (lane & 7), ks * 2 + (m >> 1)), f[0], f[1], f[2], f[3]);
          mma_bf16(x[mt], f, qf[ks][0], qf[ks][1]);
        }
      // what this warp read is in its registers when the slot is given back
      __threadfence_block();
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(0, s));
#pragma unroll
      for (int mt = 0; mt < 4; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = p0 + mt * 16 + qr + (e >> 1) * 8, i = e & 1;
          if constexpr (FORM) {
            float v = x[mt][e] * a.scale;
            if (a.softcap > 0.f) v = a.softcap * tanh_fast(__fdividef(v, a.softcap));
            v -= slope[i] * fabsf((float)(pos[i] - p));
            x[mt][e] = v * 1.4426950408889634f;
          } else {
            x[mt][e] *= sc;
          }
          if (edge && (p < vis[i].lo || p >= vis[i].hi)) x[mt][e] = -INFINITY;
        }
      float corr[2], neg_m[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float mx = fmaxf(fmaxf(fmaxf(x[0][i], x[0][i + 2]), fmaxf(x[1][i], x[1][i + 2])), fmaxf(fmaxf(x[2][i], x[2][i + 2]), fmaxf(x[3][i], x[3][i + 2])));
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float m_new = fmaxf(m_run[i], mx), m_safe = m_new == -INFINITY ? 0.f : m_new;
        corr[i] = ex2(m_run[i] - m_safe);
        m_run[i] = m_new;
        neg_m[i] = -m_safe;
      }
      float rs[2] = {0.f, 0.f};
      uint32_t pf[4][2];
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[mt][e] = ex2(x[mt][e] + neg_m[e & 1]);
        rs[0] += x[mt][0] + x[mt][2]; rs[1] += x[mt][1] + x[mt][3];
        pf[mt][0] = transpose8(pack_bf16(x[mt][0], x[mt][1]));
        pf[mt][1] = transpose8(pack_bf16(x[mt][2], x[mt][3]));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) l_run[i] = l_run[i] * corr[i] + rs[i];
#pragma unroll
      for (int j = 0; j < DT; ++j) { o[j][0] *= corr[0]; o[j][1] *= corr[1]; o[j][2] *= corr[0]; o[j][3] *= corr[1]; }
      if (!warp_wait_uniform(full_bar(1, s), (tl / S) & 1, abort_flag)) { if (lane == 0) *abort_flag = 1; break; }
      if (edge) clear_values<HD>(gen_base + (vt - base), p0, u_lo, u_hi, c_lo, c_hi, odd_flag);
      // ---- O^T += V^T P^T
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int j = 0; j < DT; ++j) {
          const int m = lane >> 3;
          uint32_t f[4];
          ldsm_x4_t(vt + kv_off(ks * 16 + (m >> 1) * 8 + (lane & 7), j * 2 + (m & 1)), f[0], f[1], f[2], f[3]);
          mma_bf16(o[j], f, pf[ks][0], pf[ks][1]);
        }
      __threadfence_block();
      if (edge && PAGES) fence_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(1, s));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) l_run[i] += __shfl_xor_sync(0xffffffffu, l_run[i], w);
    __syncthreads();                                 // the ring is idle
    // the groups' states, for all threads to merge
    float* mine = merge + warp * C::kMergeFloats;
#pragma unroll
    for (int j = 0; j < DT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[(2 * qc + (e & 1)) * HD + j * 16 + qr + (e >> 1) * 8] = o[j][e];
    if (qr == 0)
#pragma unroll
      for (int i = 0; i < 2; ++i) { mine[8 * HD + 2 * qc + i] = m_run[i]; mine[8 * HD + 8 + 2 * qc + i] = l_run[i]; }
    __syncthreads();
  }
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicOr(a.kv.status, kStInternal);
    return;
  }
  // a thread has two neighbouring dimensions of a query
  for (int i = threadIdx.x; i < R * (HD / 2); i += C::kThreads) {
    const int row = i / (HD / 2), d = 2 * (i - row * (HD / 2));
    float m = -INFINITY;
#pragma unroll
    for (int g = 0; g < KW; ++g) m = fmaxf(m, merge[g * C::kMergeFloats + 8 * HD + row]);
    const float m_safe = m == -INFINITY ? 0.f : m;
    float l = 0.f, y[2] = {0.f, 0.f};
#pragma unroll
    for (int g = 0; g < KW; ++g) {
      const float* st = merge + g * C::kMergeFloats;
      const float w = ex2(st[8 * HD + row] - m_safe);
      l = fmaf(w, st[8 * HD + 8 + row], l);
      const float2 v = *reinterpret_cast<const float2*>(st + row * HD + d);
      y[0] = fmaf(w, v.x, y[0]); y[1] = fmaf(w, v.y, y[1]);
    }
    const int tok = sq.row0 + row / G, head = kvh * G + row % G;
    if (*odd_flag) {
      const Visible v = visible(a, first_p + row / G, sq.len);
      for (int p = max(u_lo, t_begin * kPos); p < min(u_hi, t_end * kPos); ++p) {
        if (p >= c_lo && p < c_hi) { p = c_hi - 1; continue; }
        const int page = page_of(a.kv, b, p, 1, u_lo, u_hi);
        if (page >= a.kv.n_pages || p < v.lo || p >= v.hi) continue;
        const __nv_bfloat16* vp = (const __nv_bfloat16*)a.kv.v + page * a.kv.page_stride + kvh * a.kv.head_stride + (long long)(p % a.kv.page_size) * a.kv.pos_stride + d;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float z = __bfloat162float(vp[e]);
          if (!(fabsf(z) < INFINITY)) y[e] += z;
        }
      }
    }
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    if (a.splits > 1) {
      const long long at = ((long long)split * a.kv.rows + tok) * a.Hq + head;
      if (d == 0) a.part_lse[at] = none ? -INFINITY : m + log2f(l);
      if (!none) *reinterpret_cast<float2*>(a.part_o + at * HD + d) = make_float2(y[0] * inv, y[1] * inv);
    } else {
      if (a.lse && d == 0) a.lse[(long long)tok * a.Hq + head] = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      *reinterpret_cast<__nv_bfloat162*>((__nv_bfloat16*)a.out + (long long)tok * a.out_stride + (long long)head * HD + d) = __floats2bfloat162_rn(y[0] * inv, y[1] * inv);
    }
  }
}

template <int HD, int KW, bool FORM, bool PAGES>
void launch_token(const PagedAttnArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, int box_rows, cudaStream_t st) {
  using C = TokCfg<HD, KW>;
  static PerDeviceOnce configured;
  configured.run([] { cudaFuncSetAttribute(paged_attn_token_kernel<HD, KW, FORM, PAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes); });
  launch_pdl(paged_attn_token_kernel<HD, KW, FORM, PAGES>, dim3((unsigned)((long long)a.kv.Hkv * a.splits * a.kv.batch)), dim3(C::kThreads), C::kSmemBytes, st, tk, tv, a,
             box_rows);
}

template <int HD, int RW, int KW, bool FORM, bool PAGES>
void launch(const PagedAttnArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, int box_rows, cudaStream_t st) {
  using C = Cfg<HD, RW, KW>;
  static PerDeviceOnce configured;
  configured.run([] { cudaFuncSetAttribute(paged_attn_tc_kernel<HD, RW, KW, FORM, PAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes); });
  const int row_tiles = (int)(((long long)a.kv.max_new * a.G + 16 * RW - 1) / (16 * RW));
  launch_pdl(paged_attn_tc_kernel<HD, RW, KW, FORM, PAGES>, dim3((unsigned)((long long)a.kv.Hkv * row_tiles * a.splits * a.kv.batch)), dim3(C::kThreads),
             C::kSmemBytes, st, tk, tv, a, row_tiles, box_rows);
}
template <int HD, int RW, int KW>
void launch_form(const PagedAttnArgs& a, cudaStream_t st) {
  CUtensorMap tk{}, tv{};
  const int box = paged_box_rows(a.kv.page_size);
  const bool pages = box >= 8 && paged_map(a.kv, a.kv.k, box, &tk) && paged_map(a.kv, a.kv.v, box, &tv);
  const bool form = a.softcap > 0.f || a.slopes;
  if (form && pages) launch<HD, RW, KW, true, true>(a, tk, tv, box, st);
  else if (form) launch<HD, RW, KW, true, false>(a, tk, tv, box, st);
  else if (pages) launch<HD, RW, KW, false, true>(a, tk, tv, box, st);
  else launch<HD, RW, KW, false, false>(a, tk, tv, box, st);
}

template <int HD, int KW>
void launch_token_form(const PagedAttnArgs& a, cudaStream_t st) {
  CUtensorMap tk{}, tv{};
  const int box = paged_box_rows(a.kv.page_size);
  const bool pages = box >= 8 && paged_map(a.kv, a.kv.k, box, &tk) && paged_map(a.kv, a.kv.v, box, &tv);
  const bool form = a.softcap > 0.f || a.slopes;
  if (form && pages) launch_token<HD, KW, true, true>(a, tk, tv, box, st);
  else if (form) launch_token<HD, KW, true, false>(a, tk, tv, box, st);
  else if (pages) launch_token<HD, KW, false, true>(a, tk, tv, box, st);
  else launch_token<HD, KW, false, false>(a, tk, tv, box, st);
}

}  // namespace

// rows: at most 8 in all; or 16 (one row warp, two position groups) or 64 per CTA.
void launch_paged_attn_tc(const PagedAttnArgs& a, int rows, cudaStream_t st) {
  if (rows == 8) { if (a.kv.hd == 64) launch_token_form<64, 4>(a, st); else launch_token_form<128, 2>(a, st); return; }
  if (a.kv.hd == 64) { if (rows == 16) launch_form<64, 1, 2>(a, st); else launch_form<64, 4, 1>(a, st); }
  else { if (rows == 16) launch_form<128, 1, 2>(a, st); else launch_form<128, 4, 1>(a, st); }
}

}  // namespace nz
