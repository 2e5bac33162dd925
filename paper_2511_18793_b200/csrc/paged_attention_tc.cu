// Attention over a paged cache on mma.sync (bf16, heads of 64 and 128): calls of few query rows, which are bound by reading keys and values
// once, and page sizes that the tcgen05 kernel does not take.
//
// A CTA has one (sequence, KV head), a tile of 16 RW query rows (tokens times the heads of the group) and a share of the context.  A producer
// warp brings tiles of 64 positions into a ring: by TMA, one box of 64 columns per page or piece of a page, where the page size is a
// multiple of 8, else 16 bytes at a time (cp.async), positions that no row sees as zeros.  RW row warps x KW position groups compute
// S = Q K^T and O += P V in registers with a running maximum and sum; the KW groups take every KW-th tile and are merged at the end.
// One token per sequence: RW = 1, KW = 2, 64 KB of ring, three CTAs per SM -- a warp's chain (scores, softmax, second product) takes about
// as long as a tile's way from HBM, so six of them per SM keep the memory busy.
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

template <int HD, int RW, int KW>
struct Cfg {
  static constexpr int kTileBytes = kPos * HD * 2;
  static constexpr int kStages = KW == 1 ? (HD == 64 ? 4 : 3) : (HD == 64 ? 4 : 2);    // a multiple of KW
  static constexpr int kThreads = (RW * KW + 1) * 32;
  static constexpr int kMergeFloats = (HD / 8) * 4 + 4;
  static constexpr int kRingBytes = kStages * 2 * kTileBytes;
  static constexpr int kSmemBytes = kRingBytes + 1024 + 128;
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
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(gen_base + C::kRingBytes + 16 * S);
  volatile uint32_t* odd_flag = abort_flag + 1;      // a value that is not finite was taken out of a tile
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(full_bar(s), PAGES ? 1 : 32); mbar_init(empty_bar(s), RW); }
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
    bool ok = true;
    int t = 0;
    if constexpr (PAGES) {
      const uint32_t leader = elect_one();
      const int nb = kPos / box_rows;
      // lane i looks box i of the next tile up while this one's copies are issued
      auto look_up = [&](int tile) { return lane < nb ? page_of(a.kv, b, tile * kPos + lane * box_rows, box_rows, u_lo, u_hi) : 0; };
      int page = NT > 0 ? look_up(t_begin) : 0;
      for (; t < NT; ++t) {
        const int s = t % S;
        const int next = t + 1 < NT ? look_up(t_begin + t + 1) : 0;
        if (t >= S && !warp_wait_uniform(empty_bar(s), ((t / S) - 1) & 1, abort_flag)) { ok = false; break; }
        mbar_expect_tx_if(full_bar(s), 2 * C::kTileBytes, leader);
        const uint32_t kd = base + s * 2 * C::kTileBytes, vd = kd + C::kTileBytes;
        const int p0 = (t_begin + t) * kPos;
        for (int i = 0; i < nb; ++i) {
          const int pg = __shfl_sync(0xffffffffu, page, i), y = (p0 + i * box_rows) % a.kv.page_size;
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            tma_load_4d_if(kd + h * (kPos * 128) + i * box_rows * 128, &tmK, h * 64, y, kvh, pg, full_bar(s), leader);
            tma_load_4d_if(vd + h * (kPos * 128) + i * box_rows * 128, &tmV, h * 64, y, kvh, pg, full_bar(s), leader);
          }
        }
        page = next;
      }
    } else {
      for (; t < NT; ++t) {
        const int s = t % S;
        if (t >= S && !warp_wait_uniform(empty_bar(s), ((t / S) - 1) & 1, abort_flag)) { ok = false; break; }
        const uint32_t kd = base + s * 2 * C::kTileBytes, vd = kd + C::kTileBytes;
        for (int i = 0; i < kPos; i += 32) {         // a lane looks a position up, the warp copies the 32 of them
          const int p = (t_begin + t) * kPos + i + lane;
          const int page = page_of(a.kv, b, p, 1, u_lo, u_hi);
          const long long at = page * a.kv.page_stride + kvh * a.kv.head_stride + (long long)(p % a.kv.page_size) * a.kv.pos_stride;
          for (int j = 0; j < 32; j += 32 / CH) {
            const int from = j + lane / CH, c = lane % CH;
            const long long src = __shfl_sync(0xffffffffu, at, from) + c * 8;
            const bool real = __shfl_sync(0xffffffffu, page, from) < a.kv.n_pages;
            const uint32_t off = kv_off(i + from, c);
            cp_async16(kd + off, (const __nv_bfloat16*)a.kv.k + (real ? src : 0), real);
            cp_async16(vd + off, (const __nv_bfloat16*)a.kv.v + (real ? src : 0), real);
          }
        }
        cp_async_arrive(full_bar(s));
      }
    }
    if (!ok && lane == 0) *abort_flag = 1;
    if (!ok)                                         // the copies in flight land before the CTA's memory goes away
      for (int j = max(0, t - S); j < t; ++j) mbar_wait(full_bar(j % S), (j / S) & 1);
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
      if (!warp_wait_uniform(full_bar(s), (tl / S) & 1, abort_flag)) { if (lane == 0) *abort_flag = 1; break; }
      const uint32_t kt = base + s * 2 * C::kTileBytes, vt = kt + C::kTileBytes;
      const bool edge = p0 < c_lo || p0 + kPos > c_hi;    // some row does not see all of the tile
      if (edge) {
        // values that no row of the CTA sees: zeros.  Those that some do not see: finite ones stay.
        uint8_t* vg = gen_base + (vt - base);
        for (int i = lane; i < kPos * CH; i += 32) {
          const int p = p0 + i / CH;
          uint4* at = reinterpret_cast<uint4*>(vg + kv_off(i / CH, i % CH));
          if (p < u_lo || p >= u_hi) { *at = make_uint4(0u, 0u, 0u, 0u); continue; }
          if (p >= c_lo && p < c_hi) continue;
          uint4 x = *at;
          uint32_t* w = reinterpret_cast<uint32_t*>(&x);
          bool odd = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; odd = true; }
            if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; odd = true; }
          }
          if (odd) { *at = x; *odd_flag = 1; }
        }
        __syncwarp();
      }
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
      // what this warp read is in its registers, and what it wrote ordered before the next copy, when the slot is given back
      __threadfence_block();
      if (edge && PAGES) fence_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(s));
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

}  // namespace

// rows: 16 (one row warp, two position groups) or 64 per CTA.
void launch_paged_attn_tc(const PagedAttnArgs& a, int rows, cudaStream_t st) {
  if (a.kv.hd == 64) { if (rows == 16) launch_form<64, 1, 2>(a, st); else launch_form<64, 4, 1>(a, st); }
  else { if (rows == 16) launch_form<128, 1, 2>(a, st); else launch_form<128, 4, 1>(a, st); }
}

}  // namespace nz
