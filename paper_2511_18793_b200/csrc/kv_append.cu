// Rotary positions and the append to a paged cache, in one pass over the new rows.
//
//   (x_a, x_b) -> (x_a cos - x_b sin, x_b cos + x_a sin), pairs (i, i + rot / 2) or (2 i, 2 i + 1) of the first `rot` dimensions
//
// Nothing is computed to speak of: the launch reads q, k and v once and writes them once.  A block takes whole rows (all heads of q, k and v), whose
// loads are in flight while the rows' places are looked up: which sequence a row is of (a 32-way search of row_start by one
// warp per row), its position, page and table row.  16,008 rows of 32 + 8 + 8 heads of 128: 68 us, 5.8 TB/s; 64 rows: 6 us, a launch and those look-ups.
#include "operators.cuh"

namespace nz {

int sm_count();

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

// A row takes `units` x `lanes` threads: a thread has one unit of a head's columns (16 bytes, or the two pieces of a pair of halves) in every
// `lanes`-th head of q, then k, then v, so that it reads its cosines and sines once per row and its loads of up to kHeads heads are under way together.
// (A thread per piece of one head, its table columns read again for each: 120 us for 16,008 rows of 32 + 8 + 8 heads of 128.)
constexpr int kHeads = 6;
// Threads of a block at most: they have to fit with kMaxRegs registers each (rows of more heads take further passes).  A few registers more cost a block per
// SM: 16,008 rows of 32 + 8 + 8 heads of 128, half of a head rotated, 91 us with 96 and 114 with 98; pairs side by side 74 with 64 and 81 with 68.
constexpr int kMaxThreads = 512;
template <bool HALVES> constexpr int kMaxRegs = HALVES ? 96 : 64;
static_assert(kMaxThreads * kMaxRegs<true> <= 65536, "registers of an SM");

template <typename T, bool HALVES>
__global__ void __maxnreg__(kMaxRegs<HALVES>) kv_append_kernel(AppendArgs a, int units, int turned, int lanes, int rows_per_block) {
  constexpr int N = Vec<T>::N;
  __shared__ long long place[16];
  __shared__ int turn[16];
  pdl_wait();
  pdl_launch();
  const int per_row = units * lanes, r = threadIdx.x / per_row, t = threadIdx.x - r * per_row;
  const int row = blockIdx.x * rows_per_block + r, w = t % units, lane_h = t / units;
  const bool live = r < rows_per_block && row < a.kv.rows;
  const int heads = a.Hq + 2 * a.kv.Hkv, hd = a.kv.hd;
  // the unit's columns: a turned pair of halves, a turned piece, or a piece that is copied
  const bool turns = w < turned, two = HALVES && turns;
  const int c0 = turns ? w * N : a.rot + (w - turned) * N, c1 = c0 + a.rot / 2;
  auto source = [&](int h) {
    return h < a.Hq ? (const T*)a.q + row * a.q_stride + (long long)h * hd
                    : h < a.Hq + a.kv.Hkv ? (const T*)a.k + row * a.k_stride + (long long)(h - a.Hq) * hd
                                          : (const T*)a.v + row * a.v_stride + (long long)(h - a.Hq - a.kv.Hkv) * hd;
  };
  float cs[N], sn[N];
  long long at = -1;
  bool first = true;
  for (int h0 = lane_h; first || (live && h0 < heads); h0 += kHeads * lanes) {
    uint4 x[kHeads][HALVES ? 2 : 1];
    if (live) {
#pragma unroll
      for (int i = 0; i < kHeads; ++i)
        if (h0 + i * lanes < heads) {
          const T* p = source(h0 + i * lanes);
          x[i][0] = *reinterpret_cast<const uint4*>(p + c0);
          if (HALVES && two) x[i][HALVES ? 1 : 0] = *reinterpret_cast<const uint4*>(p + c1);
        }
    }
    if (first) {                                     // where the rows go, while their loads are on their way
      for (int i = threadIdx.x >> 5; i < rows_per_block; i += blockDim.x >> 5) {
        const RowPlace p = place_of(a, blockIdx.x * rows_per_block + i);
        if ((threadIdx.x & 31) == 0) { place[i] = p.place; turn[i] = p.turn; }
      }
      __syncthreads();
      first = false;
      if (!live || (at = place[r]) < 0) break;
      if (turns) {
        const float* tab = a.table + (long long)turn[r] * a.rot + (HALVES ? c0 : c0 / 2);
        constexpr int P = HALVES ? N : N / 2;        // pairs of the unit
#pragma unroll
        for (int c = 0; c < P; c += 2) {
          const float2 co = *reinterpret_cast<const float2*>(tab + c), si = *reinterpret_cast<const float2*>(tab + a.rot / 2 + c);
          cs[c] = co.x; cs[c + 1] = co.y; sn[c] = si.x; sn[c + 1] = si.y;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const int h = h0 + i * lanes;
      if (h >= heads) continue;
      const bool is_v = h >= a.Hq + a.kv.Hkv;
      T* out = h < a.Hq ? (T*)a.q_out + row * a.q_out_stride + (long long)h * hd
                        : (T*)(is_v ? a.kv.v : a.kv.k) + at + (long long)(h - a.Hq - (is_v ? a.kv.Hkv : 0)) * a.kv.head_stride;
      if (!turns || is_v) {
        *reinterpret_cast<uint4*>(out + c0) = x[i][0];
        if (HALVES && two) *reinterpret_cast<uint4*>(out + c1) = x[i][HALVES ? 1 : 0];
        continue;
      }
      float xa[N];
      Vec<T>::get(x[i][0], xa);
      if constexpr (HALVES) {
        float xb[N], ya[N], yb[N];
        Vec<T>::get(x[i][1], xb);
#pragma unroll
        for (int c = 0; c < N; ++c) { ya[c] = xa[c] * cs[c] - xb[c] * sn[c]; yb[c] = xb[c] * cs[c] + xa[c] * sn[c]; }
        *reinterpret_cast<uint4*>(out + c0) = Vec<T>::put(ya);
        *reinterpret_cast<uint4*>(out + c1) = Vec<T>::put(yb);
      } else {
        float y[N];
#pragma unroll
        for (int c = 0; c < N; c += 2) {
          y[c] = xa[c] * cs[c / 2] - xa[c + 1] * sn[c / 2];
          y[c + 1] = xa[c + 1] * cs[c / 2] + xa[c] * sn[c / 2];
        }
        *reinterpret_cast<uint4*>(out + c0) = Vec<T>::put(y);
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
  const int turned = HALVES ? a.rot / 2 / N : a.rot / N, units = turned + (a.kv.hd - a.rot) / N, heads = a.Hq + 2 * a.kv.Hkv;
  // heads side by side: as few as keep all of a row's loads under way at once, and few rows' threads together a block of 128 or more
  int lanes = (heads + kHeads - 1) / kHeads;
  if (lanes * units > kMaxThreads) lanes = kMaxThreads / units;
  int rows = 1;
  if (a.kv.rows > 8 * sm_count())
    while (rows < 16 && 2 * rows * lanes * units <= 256) rows *= 2;
  const int threads = (rows * lanes * units + 31) / 32 * 32;
  launch_pdl(kv_append_kernel<T, HALVES>, dim3((a.kv.rows + rows - 1) / rows), dim3(threads), 0, st, a, units, turned, lanes, rows);
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
