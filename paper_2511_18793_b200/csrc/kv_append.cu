// Rotary positions and the append to a paged cache, in one pass over the new rows.
//
//   (x_a, x_b) -> (x_a cos - x_b sin, x_b cos + x_a sin), pairs (i, i + rot / 2) or (2 i, 2 i + 1) of the first `rot` dimensions
//
// Nothing is computed to speak of: the launch reads q, k and v once and writes them once.  A block takes R rows whole (all heads of q, k and v), a
// thread the same 16-byte chunks of each, so the loads of R rows are in flight while the rows' places are looked up: which
// sequence a row is of (a 32-way search of row_start by one warp per row), its position, page and table row.
#include "operators.cuh"

namespace nz {

namespace {

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& u, float* x) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Where a row goes: its place in the pool (elements, KV head 0) and its row of the table; place -1: nowhere.
struct RowPlace { long long place; int turn; };

// By a whole warp.
__device__ RowPlace place_of(const AppendArgs& a, int row) {
  const PagedView& kv = a.kv;
  const RowPlace none{-1, 0};
  if (row >= kv.rows) return none;
  // the number of entries of row_start that are at most `row`
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = kv.batch + 1;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const int c = __popc(__ballot_sync(0xffffffffu, at < hi && kv.row_start[at] <= row));
    if (c == 0) break;
    hi = min(hi, lo + c * step);
    lo += (c - 1) * step + 1;
  }
  const int b = lo - 1;
  if (b < 0 || b >= kv.batch) return none;
  const PagedSeq s = paged_seq(kv, b, false);
  if (row < s.row0 || row >= s.row0 + s.n) return none;
  const int pos = s.len - s.n + row - s.row0;
  const int turn = a.rot == 0 ? 0 : a.positions ? a.positions[row] : pos;
  int page = -1;
  if (pos >= 0) page = kv.table[(long long)b * kv.table_stride + pos / kv.page_size];
  if (page < 0 || page >= kv.n_pages || turn < 0 || (a.rot > 0 && turn >= a.n_table)) {
    if (lane == 0) atomicOr(kv.status, kStBadPage);
    return none;
  }
  return RowPlace{page * kv.page_stride + (long long)(pos % kv.page_size) * kv.pos_stride, turn};
}

// The batch's row ranges and lengths, looked over once per launch (a row that no sequence claims would not show what is wrong with it).
__device__ __forceinline__ void look_over(const PagedView& kv) {
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < kv.batch; b += blockDim.x) paged_seq(kv, b, true);
}

// A thread's work on a row: which of q, k and v, the element offset inside the source row and behind the destination's start, the second chunk of a
// rotated pair of halves, and its columns of the table.
struct Unit { int kind; long long src, dst; int second, col; };   // kind 0: q, 1: k, 2: v; second 0: one chunk; col -1: copied

// Units of a head: the chunks that are rotated (of the half layout two at a time), then those that are copied.
template <int N, bool HALVES>
__device__ __forceinline__ Unit unit_of(const AppendArgs& a, int u, int per_turned, int per_copied) {
  const int hd = a.kv.hd;
  Unit r{};
  int head, w;
  const int n_turned = (a.Hq + a.kv.Hkv) * per_turned;
  if (u < n_turned) {
    head = u / per_turned; w = u - head * per_turned;
    const int turned = HALVES ? a.rot / 2 / N : a.rot / N;
    if (w < turned) { r.second = HALVES ? a.rot / 2 : 0; r.col = HALVES ? w * N : w * (N / 2); w *= N; }
    else { r.col = -1; w = a.rot + (w - turned) * N; }
    r.kind = head < a.Hq ? 0 : 1;
    if (r.kind) head -= a.Hq;
  } else {
    u -= n_turned;
    head = u / per_copied; w = (u - head * per_copied) * N;
    r.kind = 2; r.col = -1;
  }
  r.src = (long long)head * hd + w;
  r.dst = r.kind == 0 ? r.src : (long long)head * a.kv.head_stride + w;
  return r;
}

template <typename T, bool HALVES, int R>
__global__ void kv_append_kernel(AppendArgs a, int units, int per_turned, int per_copied) {
  constexpr int N = Vec<T>::N;
  __shared__ long long place[R];
  __shared__ int turn[R];
  pdl_wait();
  pdl_launch();
  const int row0 = blockIdx.x * R, warp = threadIdx.x >> 5;
  const T* const src[3] = {(const T*)a.q, (const T*)a.k, (const T*)a.v};
  const long long stride[3] = {a.q_stride, a.k_stride, a.v_stride};
  bool first = true;
  for (int u = threadIdx.x; u < units || first; u += blockDim.x) {      // (every thread comes through once: the barrier)
    const bool mine = u < units;
    Unit t{};
    uint4 x[R][2];
    if (mine) {
      t = unit_of<N, HALVES>(a, u, per_turned, per_copied);
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (row0 + i < a.kv.rows) {
          const T* p = src[t.kind] + (row0 + i) * stride[t.kind] + t.src;
          x[i][0] = *reinterpret_cast<const uint4*>(p);
          if (HALVES && t.second) x[i][1] = *reinterpret_cast<const uint4*>(p + t.second);
        }
    }
    if (first) {
      for (int i = warp; i < R; i += blockDim.x >> 5) {
        const RowPlace p = place_of(a, row0 + i);
        if ((threadIdx.x & 31) == 0) { place[i] = p.place; turn[i] = p.turn; }
      }
      __syncthreads();
      first = false;
    }
    if (!mine) break;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (place[i] < 0) continue;
      T* out = t.kind == 0 ? (T*)a.q_out + (row0 + i) * a.q_out_stride : (T*)(t.kind == 1 ? a.kv.k : a.kv.v) + place[i];
      out += t.dst;
      if (t.col < 0) { *reinterpret_cast<uint4*>(out) = x[i][0]; continue; }
      const float* tab = a.table + (long long)turn[i] * a.rot + t.col;
      float xa[N];
      Vec<T>::get(x[i][0], xa);
      if (HALVES) {
        float xb[N], ya[N], yb[N];
        Vec<T>::get(x[i][1], xb);
#pragma unroll
        for (int c = 0; c < N; c += 4) {
          const float4 co = *reinterpret_cast<const float4*>(tab + c), si = *reinterpret_cast<const float4*>(tab + a.rot / 2 + c);
          const float cs[4] = {co.x, co.y, co.z, co.w}, sn[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ya[c + e] = xa[c + e] * cs[e] - xb[c + e] * sn[e];
            yb[c + e] = xb[c + e] * cs[e] + xa[c + e] * sn[e];
          }
        }
        *reinterpret_cast<uint4*>(out) = Vec<T>::put(ya);
        *reinterpret_cast<uint4*>(out + t.second) = Vec<T>::put(yb);
      } else {
        float y[N];
#pragma unroll
        for (int c = 0; c < N / 2; c += 2) {
          const float2 co = *reinterpret_cast<const float2*>(tab + c), si = *reinterpret_cast<const float2*>(tab + a.rot / 2 + c);
          y[2 * c] = xa[2 * c] * co.x - xa[2 * c + 1] * si.x;
          y[2 * c + 1] = xa[2 * c + 1] * co.x + xa[2 * c] * si.x;
          y[2 * c + 2] = xa[2 * c + 2] * co.y - xa[2 * c + 3] * si.y;
          y[2 * c + 3] = xa[2 * c + 3] * co.y + xa[2 * c + 2] * si.y;
        }
        *reinterpret_cast<uint4*>(out) = Vec<T>::put(y);
      }
    }
  }
  look_over(a.kv);
}

// Any even `rot`: a block per row, a pair (or a copied element) at a time.
template <typename T>
__global__ void kv_append_any_kernel(AppendArgs a) {
  __shared__ long long place;
  __shared__ int turn;
  pdl_wait();
  pdl_launch();
  const int row = blockIdx.x, hd = a.kv.hd, half = a.rot / 2, per_head = half + (hd - a.rot);
  if (threadIdx.x < 32) {
    const RowPlace p = place_of(a, row);
    if (threadIdx.x == 0) { place = p.place; turn = p.turn; }
  }
  __syncthreads();
  look_over(a.kv);
  if (place < 0) return;
  const float* tab = a.table + (long long)turn * a.rot;
  for (int u = threadIdx.x; u < (a.Hq + 2 * a.kv.Hkv) * per_head; u += blockDim.x) {
    int head = u / per_head;
    const int w = u - head * per_head;
    const int kind = head < a.Hq ? 0 : head < a.Hq + a.kv.Hkv ? 1 : 2;
    head -= kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.kv.Hkv;
    const T* x = kind == 0 ? (const T*)a.q + row * a.q_stride : kind == 1 ? (const T*)a.k + row * a.k_stride : (const T*)a.v + row * a.v_stride;
    T* y = kind == 0 ? (T*)a.q_out + row * a.q_out_stride : (T*)(kind == 1 ? a.kv.k : a.kv.v) + place;
    x += (long long)head * hd;
    y += kind == 0 ? (long long)head * hd : (long long)head * a.kv.head_stride;
    if (w >= half) { y[a.rot + w - half] = x[a.rot + w - half]; continue; }
    const int ia = a.interleaved ? 2 * w : w, ib = a.interleaved ? 2 * w + 1 : w + half;
    if (kind == 2) {
      const T xa = x[ia], xb = x[ib];
      y[ia] = xa; y[ib] = xb;
      continue;
    }
    const float xa = to_f32(x[ia]), xb = to_f32(x[ib]), c = tab[w], s = tab[half + w];
    y[ia] = from_f32<T>(xa * c - xb * s);
    y[ib] = from_f32<T>(xb * c + xa * s);
  }
}

__global__ void rope_table_kernel(const __grid_constant__ RopeFrequencies f, float* table, int n) {
  pdl_wait();
  pdl_launch();
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (long long)n * f.half) return;
  const int p = (int)(i / f.half), c = (int)(i - (long long)p * f.half);
  double sn, cs;
  sincos((double)p * f.f[c], &sn, &cs);
  table[(long long)p * 2 * f.half + c] = (float)(cs * f.magnitude);
  table[(long long)p * 2 * f.half + f.half + c] = (float)(sn * f.magnitude);
}

template <typename T, bool HALVES>
void launch_vec(const AppendArgs& a, cudaStream_t st) {
  constexpr int N = Vec<T>::N;
  const int per_turned = (HALVES ? a.rot / 2 / N : a.rot / N) + (a.kv.hd - a.rot) / N, per_copied = a.kv.hd / N;
  const int units = (a.Hq + a.kv.Hkv) * per_turned + a.kv.Hkv * per_copied;
  const int threads = units >= 1024 ? 1024 : (units + 31) / 32 * 32;
  // rows per block: as many as keep the grid above two waves of blocks
  if (a.kv.rows > 4 * 148 * 4)
    launch_pdl(kv_append_kernel<T, HALVES, 4>, dim3((a.kv.rows + 3) / 4), dim3(threads), 0, st, a, units, per_turned, per_copied);
  else
    launch_pdl(kv_append_kernel<T, HALVES, 1>, dim3(a.kv.rows), dim3(threads), 0, st, a, units, per_turned, per_copied);
}

template <typename T>
void launch_t(const AppendArgs& a, cudaStream_t st) {
  constexpr int N = Vec<T>::N;
  if (a.rot % (a.interleaved ? N : 2 * N) == 0) {
    if (a.interleaved) launch_vec<T, false>(a, st);
    else launch_vec<T, true>(a, st);
  } else {
    launch_pdl(kv_append_any_kernel<T>, dim3(a.kv.rows), dim3(256), 0, st, a);
  }
}

}  // namespace

void launch_kv_append(const AppendArgs& a, bool bf16, cudaStream_t st) {
  LaunchScope ls(kcRope, st);
  if (bf16) launch_t<__nv_bfloat16>(a, st);
  else launch_t<float>(a, st);
}

void launch_rope_table(const RopeFrequencies& f, float* table, int n_positions, cudaStream_t st) {
  LaunchScope ls(kcMisc, st);
  const long long n = (long long)n_positions * f.half;
  launch_pdl(rope_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, f, table, n_positions);
}

}  // namespace nz
