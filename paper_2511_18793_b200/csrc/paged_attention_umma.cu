// Attention over a paged cache on the Blackwell tensor path (tcgen05 + TMEM, bf16, heads of 64 and 128): calls of many query rows, which are bound by
// the two products and the exponentials between them.
//
// A CTA has one (sequence, KV head), up to NX tiles of 128 query rows (tokens times the heads of the group; below A, B, ...), and a share of the context in tiles
// of 128 positions (NX = 4: 64).  Warp 0 brings K and V tiles into one ring by TMA (a box of 64 columns per page or piece of a page), warp 1 issues the
// products, warps 2 and 3 look after V tiles on the edge of what the rows see, and from warp 4 each row tile has a warpgroup for its softmax, one thread per
// row (a TMEM lane is a row).  TMEM: S of each row tile, then O of each.
//   S_X = Q_X K^T, then the row's scores through registers: running reference maximum (raised only when the true one has grown by more
//   than 8 in log2, when O is rescaled in TMEM), base-2 exponentials, P as bf16 over the columns that its scores came from;
//   O_X += P V with P read from TMEM; S_X of the next tile is issued right behind it.
// While one tile's rows go through softmax, the tensor core runs the other tiles' products: P_A V, S_A', P_B V, S_B', ...  At 128 positions by 128 rows the
// products of heads of 128 take as many cycles as the exponentials (1,024 a row tile), those of 64 half; what is left over is the chain of one softmax thread.
//   NX = 1, calls of at most 128 rows: A has two buffers of S, so S of the next tile is there before the softmax of this one ends (148 such CTAs, heads of
//     128 over 16k positions: 380 us, the rate of the memory; 459 with one buffer).
//   NX = 2: 4,096 tokens of 32 heads of 128 behind 16k positions 1,055 us, 1,170 TFLOP/s, 71 % of the tensor cores' measured rate.  A third buffer of S,
//     or a second issuing warp, made A and B fall into step, where they want the same unit at the same time (heads of 64: 977 and 1,056 us for 919).
//   NX = 4, heads of 64 (four tiles of heads of 128 do not fit in TMEM): four warps per scheduler hide one another's latencies.  The same call with heads of 64
//     859 us (917 with NX = 2), a ragged batch of 32 with caps, biases and a window 280 (about 350).
// What a row does not see has no part in its sums (see paged_attention_tc.cu).  Waits are bounded as everywhere.
#include <math.h>
#include <stdlib.h>

#include "gemm_epilogue.cuh"
#include "paged_attention.cuh"

namespace nz {

int sm_count();

namespace {

using namespace gemm_detail;
using namespace paged_detail;

constexpr float kRaise = 8.f;

// NX: row tiles of a CTA (1, 2, 4)
template <int HD, int NX> struct UCfg {
  static constexpr int kPos = NX == 4 ? 64 : 128;              // positions per tile
  static constexpr int kGroups = NX == 4 ? 4 : 2;              // softmax warpgroups (of one row tile the second is idle)
  static constexpr int kThreads = 128 + 128 * kGroups;         // warps 0 to 3: copies, products, edges; from 4: the row tiles, four each
  // registers a thread; together what the threads have at the launch (168 of 384, 96 of 640)
  static constexpr int kRegsRest = NX == 4 ? 64 : 88, kRegsSoftmax = NX == 4 ? 104 : 208;
  static constexpr int kQBytes = 128 * HD * 2;                 // one row tile
  static constexpr int kTileBytes = kPos * HD * 2;             // one K or V tile
  static constexpr int kSlots = NX == 4 ? 16 : HD == 128 ? 5 : 8;
  static constexpr int kBarBytes = 512;
  static constexpr int kSmemBytes = kGroups * kQBytes + kSlots * kTileBytes + kBarBytes + 1024;
  static constexpr uint32_t kColO = 256;                       // TMEM: kPos columns of S for each row tile (of one: two buffers), then O of each
  static constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kPos >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
  static constexpr uint32_t kIdescPV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) /* B is N-major */ | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
  static_assert(kSmemBytes <= 227 * 1024 && 2 * kSmemBytes > 227 * 1024, "one CTA per SM");
  static_assert(kColO + kGroups * HD <= 512, "TMEM");
};

__device__ __forceinline__ void mma_a_tmem(uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accumulate, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
// N-major operand tile with the 128-byte swizzle: 8-row groups along K 1024 B apart, 64-element groups along N `lbo` bytes apart.
__device__ __forceinline__ uint64_t desc_nmajor(uint32_t addr, uint32_t lbo) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)((lbo >> 4) & 0x3FFF) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// tanh(y) / y as a polynomial in y^2, |y| <= 0.6: fitted to tanh for the least relative error, 8e-8.
constexpr float kTanhRange = 0.6f;
constexpr float kTanhNear = 0.2f, kTanhShort[3] = {0.99999988f, -0.3332859f, 0.13015407f};      // and for |y| <= 0.2: 1.1e-7
constexpr float kTanh[5] = {0.99999994f, -0.33332309f, 0.13310173f, -0.052101482f, 0.015475428f};

// FORM, a sum of: scores capped; scores biased by their distance (or a scale that is not positive).  0: neither.
enum { kCap = 1, kBias = 2 };

template <int HD, int FORM, int NX>
__global__ void __launch_bounds__(UCfg<HD, NX>::kThreads, 1) paged_attn_umma_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                      PagedAttnArgs a, int row_tiles, int box_rows) {
  using C = UCfg<HD, NX>;
  constexpr int SR = C::kSlots, NH = HD / 64, KS = HD / 16, kPosP = C::kPos;
  constexpr bool ONE = NX == 1;
  constexpr bool kHalves = NX < 4;      // P V begins when half of P is there
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t ring = base + C::kGroups * C::kQBytes, bar_base = ring + SR * C::kTileBytes;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (SR + s); };
  auto s_full = [&](int x) { return bar_base + 8u * (2 * SR + x); };          // S_X of tile j is in TMEM (and O_X holds the tiles before it)
  auto p_full = [&](int x) { return bar_base + 8u * (2 * SR + 4 + x); };      // P_X of tile j is
  auto o_full = [&](int x) { return bar_base + 8u * (2 * SR + 8 + x); };      // (ONE: O_A holds tile j, x = j % 2)
  auto p_half = [&](int x) { return bar_base + 8u * (2 * SR + 12 + x); };      // its first 64 positions are
  auto q_full = [&](int x) { return bar_base + 8u * (2 * SR + 16 + x); };      // Q_X is in shared memory
  const uint32_t edge_bar = bar_base + 8u * (2 * SR + 20), clean_bar = edge_bar + 8u;      // the next V tile on the edge is in its slot; what no row sees is out of it
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + (bar_base - base) + 8 * (2 * SR + 22));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  volatile uint32_t* odd_flag = tmem_slot + 2;      // a value that is not finite was taken out of a tile
  static_assert(8 * (2 * SR + 22) + 12 <= C::kBarBytes, "barrier area");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_wait();
  pdl_launch();
  AttnCta cta = attn_cta(a, row_tiles);
  cta.tile = row_tiles - 1 - cta.tile;              // the rows that see the most context go first
  const int kvh = cta.kvh, b = cta.b;
  const PagedSeq sq = paged_seq(a.kv, b, kvh == 0 && cta.tile == 0 && cta.split == 0 && threadIdx.x == 0);
  const int G = a.G, R = sq.n * G, r0 = cta.tile * (128 * C::kGroups);
  if (r0 >= R) return;                              // (the grid is made for the longest sequence)
  const int first_p = sq.len - sq.n;
  const int nx = ONE ? 1 : min(NX, (R - r0 + 127) / 128);      // row tiles that there are
  const Visible v0 = visible(a, first_p + r0 / G, sq.len), v1 = visible(a, first_p + min(r0 + 128 * C::kGroups - 1, R - 1) / G, sq.len);
  const int u_lo = v0.lo, u_hi = v1.hi, c_lo = v1.lo, c_hi = v0.hi;      // what some of the rows see; what all of them see
  int t_begin = u_lo / kPosP, t_end = (u_hi + kPosP - 1) / kPosP;
  if (a.splits > 1) {
    t_begin = max(t_begin, cta.split * (a.split_tiles * kAttnTile / kPosP));
    t_end = min(t_end, (cta.split + 1) * (a.split_tiles * kAttnTile / kPosP));
  }
  const int NT = max(0, t_end - t_begin);
  // The j-th tile of the CTA's share.  With a bias by distance the near positions, whose scores are large, go first: else the reference maximum would be raised tile by tile.
  constexpr bool kBack = (FORM & kBias) != 0;
  auto tile_at = [&](int j) { return kBack ? t_end - 1 - j : t_begin + j; };
  auto on_edge = [&](int tile) { return tile * kPosP < c_lo || (tile + 1) * kPosP > c_hi; };      // some of the rows do not see all of it
  // ONE: the columns of S_B are a second buffer for rows A, tile j uses x = j % 2, and S of the next tile is there before the softmax of this one ends.
  // K is then needed two tiles ahead of V, otherwise one; the ring's order is K_0 .. K_{lead - 1}, V_0, K_lead, V_1, K_{lead + 1}, ...
  constexpr int lead = ONE ? 2 : 1;
  auto k_at = [&](int t) { return t < lead ? t : 2 * t - lead + 1; };
  auto v_at = [&](int t) { return lead + 2 * t; };

  // The boxes of all tiles are numbered through; a lane has the page of one in 32 of them, looked up 32 boxes ahead.
  const int nb = kPosP / box_rows;
  auto look_up = [&](int box) {
    box += lane;
    const int j = box / nb;
    return j < NT ? page_of(a.kv, b, tile_at(j) * kPosP + (box - j * nb) * box_rows, box_rows, u_lo, u_hi) : 0;
  };
  int first_pages[2] = {0, 0};
  if (warp == 0) { first_pages[0] = look_up(0); first_pages[1] = look_up(32); }
  if (threadIdx.x == 64) {
    for (int s = 0; s < SR; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int x = 0; x < 4; ++x) { mbar_init(s_full(x), 1); mbar_init(p_full(x), 4); mbar_init(o_full(x), 1); mbar_init(p_half(x), 4); mbar_init(q_full(x), 4); }
    mbar_init(edge_bar, 1); mbar_init(clean_bar, 2);
    *abort_flag = 0; *odd_flag = 0;
    mbar_fence_init();
    tma_prefetch_map(&tmK);
    tma_prefetch_map(&tmV);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsRest));
    if (warp == 0) {
      // ------------------------------------------------------------------ copies: K_0, V_0, K_1, V_1, ... through one ring
      const uint32_t leader = elect_one();
      // (of each of K and V: the pages of its present 32 boxes and of the next)
      int page[2] = {first_pages[0], first_pages[0]}, next[2] = {first_pages[1], first_pages[1]}, last = -1;
      auto bring = [&](int kv, int t, int i) {
        const int s = i % SR, first = t * nb;        // (nb divides 32)
        if (i >= SR && !warp_wait_uniform(empty_bar(s), (uint32_t)(i / SR - 1) & 1u, abort_flag)) return false;
        if (t > 0 && (first & 31) == 0) { page[kv] = next[kv]; next[kv] = look_up(first + 32); }
        int y = tile_at(t) * kPosP % a.kv.page_size;
        mbar_expect_tx_if(full_bar(s), C::kTileBytes, leader);
        for (int n = 0; n < nb; ++n) {
          const int pg = __shfl_sync(0xffffffffu, page[kv], (first + n) & 31);
#pragma unroll
          for (int h = 0; h < NH; ++h)
            tma_load_4d_if(ring + s * C::kTileBytes + h * (kPosP * 128) + n * box_rows * 128, kv ? &tmV : &tmK, h * 64, y, kvh, pg, full_bar(s), leader);
          y += box_rows;
          if (y >= a.kv.page_size) y -= a.kv.page_size;
        }
        last = i;
        return true;
      };
      bool ok = true;
      for (int t = 0; t < min(lead, NT) && ok; ++t) ok = bring(0, t, k_at(t));
      for (int t = 0; t < NT && ok; ++t) {
        ok = bring(1, t, v_at(t));
        if (ok && t + lead < NT) ok = bring(0, t + lead, k_at(t + lead));
      }
      if (!ok && lane == 0) {                        // the copies in flight land before the CTA's memory goes away
        *abort_flag = 1;
        for (int j = max(0, last - SR + 1); j <= last; ++j) mbar_wait(full_bar(j % SR), (j / SR) & 1);
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ products
      const uint32_t leader = elect_one();
      bool ok = true;
      auto slot_ready = [&](int i) { return warp_wait_uniform(full_bar(i % SR), (uint32_t)(i / SR) & 1u, abort_flag); };
      auto issue_s = [&](int u, int xx, int i) {     // S of buffer u = Q_X K^T, K at place i of the ring's order
        const uint32_t kt = ring + (i % SR) * C::kTileBytes, qt = base + xx * C::kQBytes;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          tc_mma(tmem_base + (uint32_t)(kPosP * u), smem_desc(qt + (ks >> 2) * (128 * 128) + (ks & 3) * 32), smem_desc(kt + (ks >> 2) * (kPosP * 128) + (ks & 3) * 32),
                 C::kIdescS, ks > 0 ? 1u : 0u, leader);
        tc_commit_if(s_full(u), leader);
      };
      auto issue_pv = [&](int u, int xx, int i, int half, bool first) {      // O_X += P V, P of buffer u, 64 of the positions
        const uint32_t vt = ring + (i % SR) * C::kTileBytes;
#pragma unroll
        for (int kk = 0; kk < kPosP / 32; ++kk) {
          const int ks = half * (kPosP / 32) + kk;
          mma_a_tmem(tmem_base + C::kColO + (uint32_t)(HD * xx), tmem_base + (uint32_t)(kPosP * u) + 8u * ks, desc_nmajor(vt + ks * (16 * 128), kPosP * 128), C::kIdescPV,
                     !first || ks > 0 ? 1u : 0u, leader);
        }
      };
      uint32_t edges = 0;
      auto clean = [&](int j) {                      // (V is in its slot)
        if (!on_edge(tile_at(j))) return true;
        if (leader) mbar_arrive(edge_bar);
        return warp_wait_uniform(clean_bar, edges++ & 1u, abort_flag);
      };
      auto add_pv = [&](int u, int xx, int j, uint32_t parity) {             // O_X += P V of tile j, as P comes
        if constexpr (kHalves) {
          if (!warp_wait_uniform(p_half(u), parity, abort_flag)) return false;
          tc_fence_after();
          issue_pv(u, xx, v_at(j), 0, j == 0);
        }
        if (!warp_wait_uniform(p_full(u), parity, abort_flag)) return false;
        tc_fence_after();
        if constexpr (!kHalves) issue_pv(u, xx, v_at(j), 0, j == 0);
        issue_pv(u, xx, v_at(j), 1, false);
        return true;
      };
      if constexpr (!ONE) {
        if (NT > 0) {
          ok = slot_ready(0);
          for (int xx = 0; xx < nx && ok; ++xx) ok = warp_wait_uniform(q_full(xx), 0u, abort_flag);
          if (ok) {
            tc_fence_after();
            for (int xx = 0; xx < nx; ++xx) issue_s(xx, xx, 0);
            tc_commit_if(empty_bar(0), leader);      // K_0 may be overwritten
          }
        }
        for (int j = 0; j < NT && ok; ++j) {
          const bool more = j + 1 < NT;
          if (!slot_ready(2 * j + 1) || !clean(j) || (more && !slot_ready(2 * j + 2))) { ok = false; break; }
          for (int xx = 0; xx < nx; ++xx) {
            const bool last = xx == nx - 1;
            ok = add_pv(xx, xx, j, (uint32_t)j & 1u);
            if (!ok) break;
            if (last) tc_commit_if(empty_bar((2 * j + 1) % SR), leader);
            if (more) {                              // (behind P_X V_j, whose P lies where this goes: a CTA's products run in order)
              issue_s(xx, xx, 2 * j + 2);
              if (last) tc_commit_if(empty_bar((2 * j + 2) % SR), leader);
            } else {
              tc_commit_if(o_full(xx), leader);
            }
          }
        }
      } else {
        if (NT > 0) ok = warp_wait_uniform(q_full(0), 0u, abort_flag);
        for (int j = 0; j < min(2, NT) && ok; ++j) {
          ok = slot_ready(j);
          if (!ok) break;
          tc_fence_after();
          issue_s(j, 0, j);
          tc_commit_if(empty_bar(j), leader);
        }
        for (int j = 0; j < NT && ok; ++j) {
          const bool more = j + 2 < NT;
          ok = slot_ready(v_at(j)) && clean(j) && (!more || slot_ready(k_at(j + 2))) && add_pv(j & 1, 0, j, (uint32_t)(j >> 1) & 1u);
          if (!ok) break;
          tc_commit_if(o_full(j & 1), leader);
          tc_commit_if(empty_bar(v_at(j) % SR), leader);
          if (more) {
            issue_s(j & 1, 0, k_at(j + 2));
            tc_commit_if(empty_bar(k_at(j + 2) % SR), leader);
          }
        }
      }
      if (!ok && leader) *abort_flag = 1;
    } else {
      // ------------------------------------------------------------------ V tiles on the edge: zeros where no row of the CTA sees a position; where some do not, finite values stay
      bool ok = true;
      uint32_t edges = 0;
      for (int j = 0; j < NT && ok; ++j) {
        if (!on_edge(tile_at(j))) continue;
        const int i = v_at(j), s = i % SR;
        // (full_bar alone would not do: it may be phases behind or ahead of a warp that passes over the tiles between)
        // (the issuing warp may be all tiles away from the edge, each of which it waits for in bounds: so many times the bound)
        int tries = 0;
        do ok = warp_wait_uniform(edge_bar, edges & 1u, abort_flag);
        while (!ok && ++tries <= NT && !__any_sync(0xffffffffu, *abort_flag));
        ok = ok && warp_wait_uniform(full_bar(s), (uint32_t)(i / SR) & 1u, abort_flag);
        if (!ok) break;
        ++edges;
        for (int row = threadIdx.x - 64; row < kPosP; row += 64) {
          uint8_t* vg = gen_base + (ring - base) + s * C::kTileBytes + row * 128;
          const int p = tile_at(j) * kPosP + row;
          if (p >= c_lo && p < c_hi) continue;
          const bool unseen = p < u_lo || p >= u_hi;
#pragma unroll 8
          for (int i = 0; i < HD / 8; ++i) {         // (neighbouring threads take a row's pieces in different orders: 16 bytes of each of 8 rows are 128 of the banks)
            const int c = i ^ (row & 7);
            uint4* at = reinterpret_cast<uint4*>(vg + (c >> 3) * (kPosP * 128) + ((c & 7) << 4));
            if (unseen) *at = make_uint4(0u, 0u, 0u, 0u);
            else if (any_odd(*at)) { *at = without_odd(*at); *odd_flag = 1; }
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(clean_bar);
      }
      if (!ok && lane == 0) *abort_flag = 1;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsSoftmax));
    // ------------------------------------------------------------------ softmax, one thread per row
    // a warp brings its query rows into shared memory (K-major, 128-byte swizzle), zeros for rows that do not exist, while the first tiles are on their way
    const int x = (warp >> 2) - 1;                    // row tile of a softmax thread
    const int row = (warp & 3) * 32 + lane;           // = the TMEM lane this thread may read
    const bool live = r0 + x * 128 + row < R;
    const int rr = live ? r0 + x * 128 + row : r0;
    const int tok = sq.row0 + rr / G, head = kvh * G + rr % G, pos = first_p + rr / G;
    const Visible vis = live ? visible(a, pos, sq.len) : Visible{0, 0};
    const long long src = live ? (long long)tok * a.q_stride + (long long)head * HD : -1;
    constexpr int kPieces = HD / 8;                   // of 16 bytes; neighbouring lanes take those of one row (each its own row's: 32 cache lines a load, 5,700 cycles)
    uint4 qv[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const long long from = __shfl_sync(0xffffffffu, src, i * (32 / kPieces) + lane / kPieces);
      qv[i] = from >= 0 ? *reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.q + from + lane % kPieces * 8) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r = (warp & 3) * 32 + i * (32 / kPieces) + lane / kPieces, c = lane % kPieces;
      *reinterpret_cast<uint4*>(gen_base + x * C::kQBytes + (c >> 3) * (128 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = qv[i];
    }
    fence_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(q_full(x));
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_o = tmem_base + lane_addr + C::kColO + (uint32_t)(HD * x);
    const float sc = a.scale * 1.4426950408889634f;       // scores in base 2
    const float slope = (FORM & kBias) && a.slopes ? a.slopes[head] * 1.4426950408889634f : 0.f;
    // capped: cap2 tanh(s inv_cap) = s (k_0 + k_1 s^2 + ...) while no score of the warp's rows is beyond kTanhRange
    const float cap2 = (FORM & kCap) ? a.softcap * 1.4426950408889634f : 0.f, inv_cap = (FORM & kCap) ? a.scale / a.softcap : 0.f;
    const int pos_min = (FORM & kBias) ? __reduce_min_sync(0xffffffffu, pos) : 0;
    float m_ref = -INFINITY, l_run = 0.f;
    bool ok = true;
    if (x < nx) {
      for (int j = 0; j < NT; ++j) {
        const int p0 = tile_at(j) * kPosP;
        const int u = ONE ? j & 1 : x;               // its buffer of S
        const uint32_t t_s = tmem_base + lane_addr + (uint32_t)(kPosP * u);
        ok = warp_wait_uniform(s_full(u), (uint32_t)(ONE ? j >> 1 : j) & 1u, abort_flag);
        if (!ok) break;
        tc_fence_after();
        float sv[kPosP];
        {
          uint32_t r[kPosP];
#pragma unroll
          for (int c = 0; c < kPosP / 32; ++c) tmem_ld32_async(t_s + 32u * c, r + 32 * c);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < kPosP; ++c) { asm volatile("" : "+r"(r[c])); sv[c] = __uint_as_float(r[c]); }
        }
        if constexpr ((FORM & kCap) != 0) {
          float mb[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < kPosP; c += 8)
#pragma unroll
            for (int q = 0; q < 4; ++q) mb[q] = max3(mb[q], fabsf(sv[c + 2 * q]), fabsf(sv[c + 2 * q + 1]));
          // (positions that nobody sees may be beyond; a NaN among them is not noticed here and stays one below)
          const float top = fmaxf(fmaxf(mb[0], mb[1]), fmaxf(mb[2], mb[3])) * fabsf(inv_cap), i2 = inv_cap * inv_cap, lead = cap2 * inv_cap;
          if (__all_sync(0xffffffffu, top <= kTanhNear)) {
            const float c0 = kTanhShort[0] * lead, c1 = kTanhShort[1] * lead * i2, c2 = kTanhShort[2] * lead * i2 * i2;
            const f32x2 k0 = pack2(c0, c0), k1 = pack2(c1, c1), k2 = pack2(c2, c2);
#pragma unroll
            for (int c = 0; c < kPosP; c += 2) {
              const f32x2 v = pack2(sv[c], sv[c + 1]), z = mul2(v, v);
              unpack2(mul2(v, fma2(z, fma2(z, k2, k1), k0)), sv[c], sv[c + 1]);
            }
          } else if (__all_sync(0xffffffffu, top <= kTanhRange)) {
            const f32x2 k0 = pack2(kTanh[0] * lead, kTanh[0] * lead), i22 = pack2(i2, i2);
            const f32x2 k1 = pack2(kTanh[1] * lead, kTanh[1] * lead), k2 = pack2(kTanh[2] * lead, kTanh[2] * lead);
            const f32x2 k3 = pack2(kTanh[3] * lead, kTanh[3] * lead), k4 = pack2(kTanh[4] * lead, kTanh[4] * lead);
#pragma unroll
            for (int c = 0; c < kPosP; c += 2) {
              const f32x2 v = pack2(sv[c], sv[c + 1]), z = mul2(mul2(v, v), i22);
              unpack2(mul2(v, fma2(z, fma2(z, fma2(z, fma2(z, k4, k3), k2), k1), k0)), sv[c], sv[c + 1]);
            }
          } else {
#pragma unroll
            for (int c = 0; c < kPosP; ++c) sv[c] = cap2 * tanh_fast(sv[c] * inv_cap);
          }
        } else if constexpr (FORM != 0) {
          const f32x2 sc2 = pack2(sc, sc);
#pragma unroll
          for (int c = 0; c < kPosP; c += 2) unpack2(mul2(pack2(sv[c], sv[c + 1]), sc2), sv[c], sv[c + 1]);
        }
        float bias = 0.f;                            // of the whole row: its scores are off by it until the exponential
        if constexpr ((FORM & kBias) != 0) {
          const float rel = (float)(pos - p0);
          if (p0 + kPosP - 1 <= pos_min) {           // counted from the tile's last position, so that no product is larger than the position's own distance makes it
            bias = -slope * (rel - (float)(kPosP - 1));
#pragma unroll
            for (int c = 0; c < kPosP; ++c) sv[c] = fmaf(slope, (float)(c - (kPosP - 1)), sv[c]);
          } else {
#pragma unroll
            for (int c = 0; c < kPosP; ++c) sv[c] = fmaf(-slope, fabsf(rel - (float)c), sv[c]);
          }
        }
        if (p0 < c_lo) {                              // (a tile is seldom on both edges)
          const int from = vis.lo - p0;
#pragma unroll
          for (int c = 0; c < kPosP; ++c)
            if (c < from) sv[c] = -INFINITY;
        }
        if (p0 + kPosP > c_hi) {
          const int to = vis.hi - p0;
#pragma unroll
          for (int c = 0; c < kPosP; ++c)
            if (c >= to) sv[c] = -INFINITY;
        }
        float mq[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < kPosP; c += 8)
#pragma unroll
          for (int q = 0; q < 4; ++q) mq[q] = max3(mq[q], sv[c + 2 * q], sv[c + 2 * q + 1]);
        const float mx = FORM ? max3(fmaxf(mq[0], mq[1]), mq[2], mq[3]) + bias : max3(fmaxf(mq[0], mq[1]), mq[2], mq[3]) * sc;
        const bool raise = mx > m_ref + kRaise || (m_ref == -INFINITY && mx > -INFINITY);
        const float m_new = raise ? mx : m_ref;
        const float m_safe = m_new == -INFINITY ? 0.f : m_new;
        const float corr = raise ? ex2(m_ref - m_safe) : 1.f;
        m_ref = m_new;
        if (j > 0 && __any_sync(0xffffffffu, raise)) {      // rescale O (its products so far are complete: S_j was issued behind them)
          if constexpr (ONE) {                       // (or, with two buffers, are waited for)
            ok = warp_wait_uniform(o_full(u ^ 1), (uint32_t)((j - 1) >> 1) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
          }
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t ov[32];
            tmem_ld32_async(t_o + 32u * c, ov);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) { asm volatile("" : "+r"(ov[i])); ov[i] = __float_as_uint(__uint_as_float(ov[i]) * corr); }
            tmem_st16(t_o + 32u * c, ov);
            tmem_st16(t_o + 32u * c + 16u, ov + 16);
          }
        }
        const f32x2 sc2 = pack2(sc, sc), neg_m2 = pack2(bias - m_safe, bias - m_safe);
        f32x2 rs2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
        for (int h = 0; h < kPosP / 32; ++h) {       // P over the first half of the columns its scores came from
          uint32_t pk[16];
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            float x0, x1;
            const f32x2 v = pack2(sv[32 * h + c], sv[32 * h + c + 1]);
            unpack2(FORM ? add2(v, neg_m2) : fma2(v, sc2, neg_m2), x0, x1);
            const float e0 = ex2(x0), e1 = ex2(x1);
            rs2[(c >> 1) & 1] = add2(rs2[(c >> 1) & 1], pack2(e0, e1));
            const __nv_bfloat162 pb = __floats2bfloat162_rn(e0, e1);
            pk[c >> 1] = *reinterpret_cast<const uint32_t*>(&pb);
          }
          tmem_st16(t_s + 16u * h, pk);
          if (kHalves && h == kPosP / 64 - 1) {                 // half of P is there: its product may begin
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_half(u));
          }
        }
        float rs_lo, rs_hi;
        unpack2(add2(rs2[0], rs2[1]), rs_lo, rs_hi);
        l_run = l_run * corr + (rs_lo + rs_hi);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(u));
      }
      if (ok && NT > 0) {
        ok = !ONE ? warp_wait_uniform(o_full(x), 0u, abort_flag) : warp_wait_uniform(o_full((NT - 1) & 1), (uint32_t)((NT - 1) >> 1) & 1u, abort_flag);
        tc_fence_after();
      }
    }
    if (!ok && lane == 0) *abort_flag = 1;
    // (a wait that gave up leaves the others of the CTA to theirs: all softmax warps come here)
    asm volatile("barrier.sync.aligned 1, %0;" ::"n"(128 * C::kGroups) : "memory");
    if (!*abort_flag && x < nx) {
      const bool odd = *odd_flag, none = l_run == 0.f;
      const float inv = none ? 0.f : 1.f / l_run;
      const long long at = ((long long)cta.split * a.kv.rows + tok) * a.Hq + head;
      // where this thread's row goes (elements of the output or of the parts), -1: nowhere
      const long long mine = !live || (a.splits > 1 && none) ? -1 : a.splits > 1 ? at * HD : (long long)tok * a.out_stride + (long long)head * HD;
      // Turned in shared memory, where Q_X was, so that neighbouring lanes have neighbouring pieces of a row (each its own row's: 2,800 cycles)
      uint8_t* turn = gen_base + x * C::kQBytes + (warp & 3) * (32 * HD * 2);
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {
        float ov[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) ov[i] = 0.f;
        if (NT > 0) tmem_ld32(t_o + 32u * c, ov);    // warp-collective: rows that do not exist take part
        if (odd) {
          // the values that were taken out, to the rows that see them
          for (int p = max(u_lo, t_begin * kPosP); p < min(u_hi, t_end * kPosP); ++p) {
            if (p >= c_lo && p < c_hi) { p = c_hi - 1; continue; }
            const int page = page_of(a.kv, b, p, 1, u_lo, u_hi);
            if (page >= a.kv.n_pages || p < vis.lo || p >= vis.hi) continue;
            const __nv_bfloat16* v = (const __nv_bfloat16*)a.kv.v + page * a.kv.page_stride + kvh * a.kv.head_stride + (long long)(p % a.kv.page_size) * a.kv.pos_stride + 32 * c;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const float y = __bfloat162float(v[i]);
              if (!(fabsf(y) < INFINITY)) ov[i] += y;
            }
          }
          __syncwarp();
        }
        if (a.splits == 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint2 lo = pack_bf16x4(ov[8 * i] * inv, ov[8 * i + 1] * inv, ov[8 * i + 2] * inv, ov[8 * i + 3] * inv);
            const uint2 hi = pack_bf16x4(ov[8 * i + 4] * inv, ov[8 * i + 5] * inv, ov[8 * i + 6] * inv, ov[8 * i + 7] * inv);
            *reinterpret_cast<uint4*>(turn + lane * (HD * 2) + (((4 * c + i) ^ (lane & 7)) << 4)) = none ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(lo.x, lo.y, hi.x, hi.y);
          }
        } else {                                     // parts are in 32 bits, 32 columns at a time
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<float4*>(turn + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_float4(ov[4 * i] * inv, ov[4 * i + 1] * inv, ov[4 * i + 2] * inv, ov[4 * i + 3] * inv);
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 3);       // row of the warp's 32
            const float4 v = *reinterpret_cast<const float4*>(turn + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
            const long long to = __shfl_sync(0xffffffffu, mine, r);
            if (to >= 0) *reinterpret_cast<float4*>(a.part_o + to + 32 * c + 4 * (lane & 7)) = v;
          }
          __syncwarp();
        }
      }
      if (a.splits == 1) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int r = i * (32 / kPieces) + lane / kPieces, piece = lane % kPieces;
          const uint4 v = *reinterpret_cast<const uint4*>(turn + r * (HD * 2) + ((piece ^ (r & 7)) << 4));
          const long long to = __shfl_sync(0xffffffffu, mine, r);
          if (to >= 0) *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + to + 8 * piece) = v;
        }
      }
      if (live) {
        const float lse2 = none ? -INFINITY : m_ref + log2f(l_run);
        if (a.splits > 1) a.part_lse[at] = lse2;
        else if (a.lse) a.lse[(long long)tok * a.Hq + head] = lse2 * 0.6931471805599453f;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512));
  }
  if (threadIdx.x == 0 && *abort_flag) atomicOr(a.kv.status, kStInternal);
}

// The softmax warpgroups take more registers a thread and leave the other fewer: the launch has to have them all (else they would wait).
template <int HD, int FORM, int NX>
bool registers_add_up() {
  using C = UCfg<HD, NX>;
  cudaFuncAttributes at{};
  return cudaFuncGetAttributes(&at, paged_attn_umma_kernel<HD, FORM, NX>) == cudaSuccess && at.numRegs * C::kThreads >= C::kRegsRest * 128 + C::kRegsSoftmax * 128 * C::kGroups;
}

template <int HD, int FORM, int NX>
bool launch(const PagedAttnArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, int box_rows, cudaStream_t st) {
  using C = UCfg<HD, NX>;
  static const bool fits = registers_add_up<HD, FORM, NX>();
  if (!fits) return false;
  static PerDeviceOnce configured;
  configured.run([] { cudaFuncSetAttribute(paged_attn_umma_kernel<HD, FORM, NX>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes); });
  const int row_tiles = (int)(((long long)a.kv.max_new * a.G + 128 * C::kGroups - 1) / (128 * C::kGroups));
  launch_pdl(paged_attn_umma_kernel<HD, FORM, NX>, dim3((unsigned)((long long)a.kv.Hkv * row_tiles * a.splits * a.kv.batch)), dim3(C::kThreads), C::kSmemBytes, st, tk, tv, a,
             row_tiles, box_rows);
  return true;
}

template <int HD, int NX>
bool launch_form(const PagedAttnArgs& a, int form, const CUtensorMap& tk, const CUtensorMap& tv, int box, cudaStream_t st) {
  switch (form) {
    case 0: return launch<HD, 0, NX>(a, tk, tv, box, st);
    case kCap: return launch<HD, kCap, NX>(a, tk, tv, box, st);
    case kBias: return launch<HD, kBias, NX>(a, tk, tv, box, st);
    default: return launch<HD, kCap + kBias, NX>(a, tk, tv, box, st);
  }
}

}  // namespace

// The series of a capped score goes in powers of the unscaled q.k, with coefficients down to scale (scale / softcap)^4: they have to be normal numbers, or terms
// that count are lost (or are infinity times zero).  A cap of ordinary scores is far from that (scale 1/8: caps up to 1e8).
static bool series_holds(const PagedAttnArgs& a) {
  const double ratio = (double)a.scale / a.softcap, last = (double)kTanhShort[2] * a.scale * 1.4426950408889634 * ratio * ratio * ratio * ratio;
  return fabs(last) >= 2e-38;
}

// false: not launched (no tensor map, or a cap that the series does not bear).
bool launch_paged_attn_umma(const PagedAttnArgs& a, cudaStream_t st) {
  CUtensorMap tk{}, tv{};
  const int box = paged_box_rows(a.kv.page_size);
  if (a.softcap > 0.f && !series_holds(a)) return false;
  if (box < 8 || !paged_map(a.kv, a.kv.k, box, &tk) || !paged_map(a.kv, a.kv.v, box, &tv)) return false;
  const int form = (a.softcap > 0.f ? kCap : 0) + (a.slopes || !(a.scale > 0.f) ? kBias : 0);
  const long long rows = (long long)a.kv.max_new * a.G;
  // (512 rows a CTA only where 256 would be more CTAs than SMs: with fewer, halves on two SMs are done sooner)
  const bool many = rows > 256 && a.splits == 1 && (long long)a.kv.Hkv * a.kv.batch * ((rows + 255) / 256) > sm_count();
  if (a.kv.hd == 64) {
    if (rows <= 128) return launch_form<64, 1>(a, form, tk, tv, box, st);
    return many ? launch_form<64, 4>(a, form, tk, tv, box, st) : launch_form<64, 2>(a, form, tk, tv, box, st);
  }
  return rows <= 128 ? launch_form<128, 1>(a, form, tk, tv, box, st) : launch_form<128, 2>(a, form, tk, tv, box, st);
}

}  // namespace nz
