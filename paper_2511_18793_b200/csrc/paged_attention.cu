// Attention of new rows over a paged context cache: the plan of a call, the CUDA-core kernel (fp32, and heads of 16 and 32
// dimensions), and the kernel that joins the parts of a split context.
//
//   s_t = scale q.k_t, capped: c tanh(s / c), biased: - slope |p - t|;   o = sum_t e^{s_t - m} v_t / sum_t e^{s_t - m}  over the visible t
//
// The rows of a (sequence, KV head) pair are its new tokens times the G query heads of the group, so keys and values are read once per
// row tile and not once per head.  A context is split over CTAs where sequences, heads and row tiles leave SMs idle; the parts
// (their own maximum and sum: o and log2 of the sum) are joined by attn_join_kernel in the order of the splits.
#include <math.h>

#include <algorithm>

#include "operators.cuh"

namespace nz {

int sm_count();
bool launch_paged_attn_umma(const PagedAttnArgs& a, cudaStream_t st);
void launch_paged_attn_tc(const PagedAttnArgs& a, int rows, cudaStream_t st);

namespace {

enum { kSimt = 0, kTc16 = 1, kTc64 = 2, kUmma = 3, kToken = 4 };
constexpr int kMaxSplits = 64;
constexpr int kRowsS = 16, kPosS = 32, kWarpsS = 4, kRowsWarp = kRowsS / kWarpsS;
constexpr float kLog2e = 1.4426950408889634f;

// One CTA per (KV head, row tile, split, sequence), in this order, KV heads fastest.  A warp has 4 rows; scores: a lane is a position; second product: a
// lane is a dimension (heads of 16: two positions at a time).
template <typename T, int HD>
__global__ void __launch_bounds__(32 * kWarpsS) paged_attn_simt_kernel(PagedAttnArgs a, int row_tiles) {
  constexpr int LD = HD + 4;                        // floats per row: lanes on different rows meet different banks
  constexpr int DL = HD >= 32 ? HD / 32 : 1;        // dimensions per lane
  __shared__ __align__(16) float ks[kPosS * LD], vs[kPosS * LD], qs[kRowsS * LD];
  pdl_wait();
  pdl_launch();
  const AttnCta c = attn_cta(a, row_tiles);
  const int kvh = c.kvh, b = c.b, split = c.split;
  const PagedSeq s = paged_seq(a.kv, b, kvh == 0 && c.tile == 0 && split == 0 && threadIdx.x == 0);
  const int R = s.n * a.G, r0 = c.tile * kRowsS;
  if (r0 >= R) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first_p = s.len - s.n;
  // what any row of the tile sees, cut to the split's share
  int lo = visible(a, first_p + r0 / a.G, s.len).lo, hi = visible(a, first_p + min(r0 + kRowsS - 1, R - 1) / a.G, s.len).hi;
  if (a.splits > 1) {      // (the last share of the longest contexts ends at 2^31)
    lo = (int)max((long long)lo, (long long)split * a.split_tiles * kAttnTile);
    hi = (int)min((long long)hi, (long long)(split + 1) * a.split_tiles * kAttnTile);
  }
  for (int i = threadIdx.x; i < kRowsS * HD; i += blockDim.x) {
    const int r = i / HD, d = i - r * HD, row = min(r0 + r, R - 1);
    qs[r * LD + d] = to_f32(((const T*)a.q)[(long long)(s.row0 + row / a.G) * a.q_stride + (long long)(kvh * a.G + row % a.G) * HD + d]);
  }
  Visible vis[kRowsWarp];
  float slope[kRowsWarp], m[kRowsWarp], l[kRowsWarp], o[kRowsWarp][DL];
  int p[kRowsWarp];
#pragma unroll
  for (int i = 0; i < kRowsWarp; ++i) {
    const int row = min(r0 + warp * kRowsWarp + i, R - 1);
    p[i] = first_p + row / a.G;
    vis[i] = visible(a, p[i], s.len);
    slope[i] = a.slopes ? a.slopes[kvh * a.G + row % a.G] : 0.f;
    m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < DL; ++d) o[i][d] = 0.f;
  }
  for (int t0 = lo / kPosS * kPosS; t0 < hi; t0 += kPosS) {
    __syncthreads();
    // a tile of positions; those outside [lo, hi), whose pages may have been given back, and those on bad pages are zeros
    constexpr int V = 16 / sizeof(T);
    for (int i = threadIdx.x; i < kPosS * (HD / V); i += blockDim.x) {
      const int j = i / (HD / V), c = (i - j * (HD / V)) * V, t = t0 + j;
      T kk[V], vv[V];
#pragma unroll
      for (int e = 0; e < V; ++e) kk[e] = vv[e] = from_f32<T>(0.f);
      if (t >= lo && t < hi) {
        const int page = a.kv.table[(long long)b * a.kv.table_stride + t / a.kv.page_size];
        if (page >= 0 && page < a.kv.n_pages) {
          const long long at = page * a.kv.page_stride + kvh * a.kv.head_stride + (long long)(t % a.kv.page_size) * a.kv.pos_stride + c;
          *reinterpret_cast<uint4*>(kk) = *reinterpret_cast<const uint4*>((const T*)a.kv.k + at);
          *reinterpret_cast<uint4*>(vv) = *reinterpret_cast<const uint4*>((const T*)a.kv.v + at);
        } else {
          atomicOr(a.kv.status, kStBadPage);
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) { ks[j * LD + c + e] = to_f32(kk[e]); vs[j * LD + c + e] = to_f32(vv[e]); }
    }
    __syncthreads();
    float x[kRowsWarp];
#pragma unroll
    for (int i = 0; i < kRowsWarp; ++i) x[i] = 0.f;
    for (int d = 0; d < HD; d += 4) {
      const float4 k4 = *reinterpret_cast<const float4*>(ks + lane * LD + d);
#pragma unroll
      for (int i = 0; i < kRowsWarp; ++i) {
        const float4 q4 = *reinterpret_cast<const float4*>(qs + (warp * kRowsWarp + i) * LD + d);
        x[i] = fmaf(q4.x, k4.x, fmaf(q4.y, k4.y, fmaf(q4.z, k4.z, fmaf(q4.w, k4.w, x[i]))));
      }
    }
    const int t = t0 + lane;
#pragma unroll
    for (int i = 0; i < kRowsWarp; ++i) {
      x[i] *= a.scale;
      if (a.softcap > 0.f) x[i] = a.softcap * tanhf(x[i] / a.softcap);
      x[i] -= slope[i] * fabsf((float)(p[i] - t));
      if (t < max(lo, vis[i].lo) || t >= min(hi, vis[i].hi)) x[i] = -INFINITY;
      const float mx = fmaxf(m[i], warp_max(x[i])), base = mx == -INFINITY ? 0.f : mx;
      const float corr = expf(m[i] - base);
      x[i] = expf(x[i] - base);
      l[i] = l[i] * corr + x[i];                    // a lane's own share: added up at the end
      m[i] = mx;
#pragma unroll
      for (int d = 0; d < DL; ++d) o[i][d] *= corr;
    }
    // (weights of positions that a row does not see are left out, not multiplied by zero: they may hold anything)
    const int j_step = HD >= 32 ? 1 : 2, j_first = HD >= 32 ? 0 : lane >> 4;
    for (int j = 0; j < kPosS; j += j_step) {
      float v[DL];
#pragma unroll
      for (int d = 0; d < DL; ++d) v[d] = vs[(j + j_first) * LD + (HD >= 32 ? lane + 32 * d : (lane & 15))];
#pragma unroll
      for (int i = 0; i < kRowsWarp; ++i) {
        const float w = __shfl_sync(0xffffffffu, x[i], j + j_first);
        const int tj = t0 + j + j_first;
        if (tj >= vis[i].lo && tj < vis[i].hi)
#pragma unroll
          for (int d = 0; d < DL; ++d) o[i][d] = fmaf(w, v[d], o[i][d]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsWarp; ++i) {
    l[i] = warp_sum(l[i]);
    if (HD < 32) o[i][0] += __shfl_xor_sync(0xffffffffu, o[i][0], 16);
    const int row = r0 + warp * kRowsWarp + i;
    if (row >= R) continue;
    const float inv = l[i] > 0.f || l[i] != l[i] ? 1.f / l[i] : 0.f;
    const long long token = s.row0 + row / a.G;
    const int head = kvh * a.G + row % a.G;
    if (a.splits > 1) {
      const long long at = ((long long)split * a.kv.rows + token) * a.Hq + head;
      if (lane == 0) a.part_lse[at] = l[i] == 0.f ? -INFINITY : m[i] * kLog2e + log2f(l[i]);
#pragma unroll
      for (int d = 0; d < DL; ++d)
        if (HD >= 32 || lane < 16) a.part_o[at * HD + lane + 32 * d] = o[i][d] * inv;
    } else {
      if (a.lse && lane == 0) a.lse[token * a.Hq + head] = l[i] == 0.f ? -INFINITY : m[i] + logf(l[i]);
      T* out = (T*)a.out + token * a.out_stride + (long long)head * HD;
#pragma unroll
      for (int d = 0; d < DL; ++d)
        if (HD >= 32 || lane < 16) out[lane + 32 * d] = from_f32<T>(o[i][d] * inv);
    }
  }
}

// JW warps per (row, head): the parts weighted by their sums.  Warp w adds the parts w, w + JW, ... in their order, all of whose loads are under way
// together (a warp that skipped empty parts by a branch: one load at a time, 57 parts 20 us), the warps' sums are added in order.  Four warps where there
// are many parts, one, and four rows and heads per block, where there are few (8,352 of them in 3 parts: 12 us with a block each).
constexpr int kJoinWarps = 4;
template <typename T, int HD, int JW>
__global__ void __launch_bounds__(32 * kJoinWarps) attn_join_kernel(PagedAttnArgs a) {
  __shared__ float sums[kJoinWarps][HD];
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) % JW, group = (threadIdx.x >> 5) / JW;
  const long long rh = (long long)blockIdx.x * (kJoinWarps / JW) + group, all = (long long)a.kv.rows * a.Hq;
  if (JW < kJoinWarps && rh >= all) return;         // (a whole warp; nothing is waited for below)
  const int row = (int)(rh / a.Hq), head = (int)(rh - (long long)row * a.Hq);
  // a lane looks after two parts' weights (kMaxSplits of them at most)
  const long long n = all;
  float w[2], m = -INFINITY;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = lane + 32 * h;
    w[h] = i < a.splits ? a.part_lse[i * n + rh] : -INFINITY;
  }
  m = warp_max(fmaxf(w[0], w[1]));
  const bool none = m == -INFINITY && !__any_sync(0xffffffffu, w[0] != w[0] || w[1] != w[1]);
  unsigned seen[2];
  float sum = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    seen[h] = __ballot_sync(0xffffffffu, w[h] != -INFINITY);
    w[h] = w[h] == -INFINITY ? 0.f : exp2f(w[h] - m);      // (a NaN stays one)
    sum += w[h];
  }
  sum = warp_sum(sum);
  constexpr int DL = HD >= 32 ? HD / 32 : 1;
  float o[DL];
#pragma unroll
  for (int d = 0; d < DL; ++d) o[d] = 0.f;
  const int col = HD >= 32 ? lane * DL : lane & 15;
#pragma unroll(JW == 1 ? 8 : kMaxSplits / JW)
  for (int j = 0; j < kMaxSplits / JW; ++j) {
    const int i = warp + JW * j;
    if (i >= a.splits) break;
    const float wi = __shfl_sync(0xffffffffu, i < 32 ? w[0] : w[1], i & 31);
    const bool on = (i < 32 ? seen[0] : seen[1]) >> (i & 31) & 1u;          // (else nothing was written for it)
    const float* part = a.part_o + (i * n + rh) * HD + col;
    float x[DL];
    if constexpr (DL == 4) { const float4 v = on ? *reinterpret_cast<const float4*>(part) : make_float4(0.f, 0.f, 0.f, 0.f); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    else if constexpr (DL == 2) { const float2 v = on ? *reinterpret_cast<const float2*>(part) : make_float2(0.f, 0.f); x[0] = v.x; x[1] = v.y; }
    else x[0] = on ? *part : 0.f;
#pragma unroll
    for (int d = 0; d < DL; ++d) o[d] = fmaf(wi, x[d], o[d]);
  }
  if (HD >= 32 || lane < 16)
#pragma unroll
    for (int d = 0; d < DL; ++d) sums[group * JW + warp][col + d] = o[d];
  // rows that no sequence has are left alone (no split wrote anything for them; looked up while the parts are on their way)
  int lo = 0, hi = a.kv.batch + 1;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const int c = __popc(__ballot_sync(0xffffffffu, at < hi && a.kv.row_start[at] <= row));
    if (c == 0) break;
    hi = min(hi, lo + c * step);
    lo += (c - 1) * step + 1;
  }
  if (lo < 1 || lo > a.kv.batch) return;
  const PagedSeq s = paged_seq(a.kv, lo - 1, false);
  if (row < s.row0 || row >= s.row0 + s.n) return;
  if (JW > 1) __syncthreads();                       // (all warps of a row and head return above, or none)
  else __syncwarp();
  const float inv = none ? 0.f : 1.f / sum;
  T* out = (T*)a.out + row * a.out_stride + (long long)head * HD;
  for (int d = warp * 32 + lane; d < HD; d += 32 * JW) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < JW; ++i) x += sums[group * JW + i][d];
    out[d] = from_f32<T>(x * inv);
  }
  if (a.lse && warp == 0 && lane == 0) a.lse[rh] = none ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
}

template <typename T>
void launch_simt(const PagedAttnArgs& a, cudaStream_t st) {
  const int row_tiles = (int)(((long long)a.kv.max_new * a.G + kRowsS - 1) / kRowsS);
  const dim3 grid((unsigned)((long long)a.kv.Hkv * row_tiles * a.splits * a.kv.batch));
  switch (a.kv.hd) {
    case 16: launch_pdl(paged_attn_simt_kernel<T, 16>, grid, dim3(32 * kWarpsS), 0, st, a, row_tiles); break;
    case 32: launch_pdl(paged_attn_simt_kernel<T, 32>, grid, dim3(32 * kWarpsS), 0, st, a, row_tiles); break;
    case 64: launch_pdl(paged_attn_simt_kernel<T, 64>, grid, dim3(32 * kWarpsS), 0, st, a, row_tiles); break;
    default: launch_pdl(paged_attn_simt_kernel<T, 128>, grid, dim3(32 * kWarpsS), 0, st, a, row_tiles); break;
  }
}
template <typename T, int JW>
void launch_join(const PagedAttnArgs& a, cudaStream_t st) {
  constexpr int kRows = kJoinWarps / JW;
  const dim3 grid((unsigned)(((long long)a.kv.rows * a.Hq + kRows - 1) / kRows)), block(32 * kJoinWarps);
  switch (a.kv.hd) {
    case 16: launch_pdl(attn_join_kernel<T, 16, JW>, grid, block, 0, st, a); break;
    case 32: launch_pdl(attn_join_kernel<T, 32, JW>, grid, block, 0, st, a); break;
    case 64: launch_pdl(attn_join_kernel<T, 64, JW>, grid, block, 0, st, a); break;
    default: launch_pdl(attn_join_kernel<T, 128, JW>, grid, block, 0, st, a); break;
  }
}

}  // namespace

// Tiles of kAttnTile positions that a CTA of `rows` query rows goes through at most: all of a sequence's, or what a window lets them see.
static long long tiles_seen(const PagedAttnArgs& a, int rows) {
  long long span = a.kv.max_kv;
  if (a.window > 0) span = std::min(span, (long long)a.window + rows / a.G + 1 + kAttnTile);
  return (span + kAttnTile - 1) / kAttnTile;
}

PagedAttnPlan paged_attn_plan(const PagedAttnArgs& a, bool bf16) {
  PagedAttnPlan p{kSimt, 1, 0, 0};
  const long long rows = (long long)a.kv.max_new * a.G, tiles = (a.kv.max_kv + kAttnTile - 1) / kAttnTile;
  const long long pairs = (long long)a.kv.Hkv * a.kv.batch;
  long long s = 1;
  if (bf16 && a.kv.hd >= 64 && rows > 64 && a.kv.page_size % 8 == 0) {
    // Many rows: one CTA per SM.  A context is split where that gives idle SMs something to do, but not to even out the last wave of many: 512 CTAs (3.5
    // waves) as they are 1,094 us, in halves 1,158 (the parts' way through memory, and less idle silicon to leave the others its power).
    p.kernel = kUmma;
    const long long units = pairs * ((rows + 255) / 256);
    s = std::min(sm_count() / std::max(units, 1ll), (tiles_seen(a, 256) + 3) / 4);
  } else {
    int tile_rows = kRowsS, per_sm = 4, least = 2;
    if (bf16 && a.kv.hd >= 64) {
      p.kernel = rows <= 8 ? kToken : rows <= 16 ? kTc16 : kTc64;
      // (three waves of the three CTAs that an SM holds; of 9 to 16 rows with heads of 128 it holds two, which makes it four and a half)
      tile_rows = rows <= 8 ? 8 : rows <= 16 ? 16 : 64;
      per_sm = rows <= 16 ? 9 : 2;
      least = rows <= 16 ? 8 : 4;
    }
    const long long ctas = pairs * ((rows + tile_rows - 1) / tile_rows);
    s = std::min((per_sm * (long long)sm_count() + ctas - 1) / std::max(ctas, 1ll), tiles_seen(a, tile_rows) / least);
  }
  s = std::min(s, (long long)kMaxSplits);
  if (s > 1) {
    // (a window moves along the sequence, so all its positions are dealt out, in shares of what a row tile sees of them)
    const long long share = (tiles_seen(a, p.kernel == kUmma ? 256 : 16) + s - 1) / s;
    p.split_tiles = (int)((share + 1) / 2 * 2);
    p.splits = (int)((tiles + p.split_tiles - 1) / p.split_tiles);
    if (p.splits > kMaxSplits) { p.split_tiles = (int)((tiles + kMaxSplits - 1) / kMaxSplits + 1) / 2 * 2; p.splits = (int)((tiles + p.split_tiles - 1) / p.split_tiles); }
  }
  if (p.splits > 1) p.bytes = (size_t)p.splits * a.kv.rows * a.Hq * (a.kv.hd + 1) * sizeof(float);
  else { p.splits = 1; p.split_tiles = 0; }
  return p;
}

void launch_paged_attention(const PagedAttnArgs& args, const PagedAttnPlan& plan, bool bf16, cudaStream_t st) {
  PagedAttnArgs a = args;
  a.splits = plan.splits; a.split_tiles = plan.split_tiles;
  if (plan.splits > 1) a.part_lse = a.part_o + (long long)plan.splits * a.kv.rows * a.Hq * a.kv.hd;
  LaunchScope ls(kcAttention, st, plan.splits > 1 ? 2 : 1);
  if (plan.kernel == kUmma && launch_paged_attn_umma(a, st)) {}
  else if (plan.kernel == kToken) launch_paged_attn_tc(a, 8, st);
  else if (plan.kernel == kTc16) launch_paged_attn_tc(a, 16, st);
  else if (plan.kernel == kTc64 || plan.kernel == kUmma) launch_paged_attn_tc(a, 64, st);
  else if (bf16) launch_simt<__nv_bfloat16>(a, st);
  else launch_simt<float>(a, st);
  if (plan.splits > 1) {
    const bool few = plan.splits <= 8;
    if (bf16) few ? launch_join<__nv_bfloat16, 1>(a, st) : launch_join<__nv_bfloat16, 4>(a, st);
    else few ? launch_join<float, 1>(a, st) : launch_join<float, 4>(a, st);
  }
}

}  // namespace nz
