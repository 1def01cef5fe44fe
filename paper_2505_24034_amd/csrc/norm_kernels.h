// norm_kernels.h -- the root-mean-square norm in front of the head, forward and backward.
//
//   s = x + residual (stored in x's type, and normalised as stored)      r = 1 / sqrt(mean(s^2) + eps)      h = s r w
//   with n = s r, g = dh w:      dx = r (g - n mean(g n)) + dsum         dw = sum over rows of dh n
//
//   k_rms_norm       h in x's type, in e4m3 with a power of two for each 128 entries, or in int8 with a scale for each row
//   k_rms_norm_bwd   dx, and the rows' share of dw in one partial row a workgroup
//   k_norm_dw        those summed, in order
//
// Bound by memory: a row is read once, kept in registers until its norm is known, and written once.  16384 x 4096 bf16 with a residual: forward 80 us (6.7
// TB/s), backward 105 - 111 (4.9) and 5 for dw; 1900 x 8192 to e4m3 19 us; one row of 4096 2.5.  Squares are summed in 64 bits: none overflows or
// vanishes, and no order of the sum shows.
#pragma once
#include "block_kernels.h"
#include "row_kernels.h"

namespace llamarl {

constexpr int64_t NORM_MOST_COLS = 16384;            // 1024 threads with two units of eight entries each
enum NormOut { OUT_SAME = 0, OUT_BLOCKS = 1, OUT_ROWS = 2 };

struct NormArgs {
  const void* x;
  const void* residual;    // null: none
  const void* w;
  int64_t N;
  int d;
  int w_bf16;
  float eps;
  void* sum;               // null where there is no residual
  void* h;                 // [N][d]: T, e4m3 or int8
  void* scale;             // OUT_BLOCKS: words, see block_kernels.h;  OUT_ROWS: float [N]
  float* rstd;             // [N] or null
};

// `left` entries of eight exist: all, none or (fp32) four
__device__ __forceinline__ void load_unit(Raw8<uint16_t>& u, const void* p, int64_t at, int left) {
  if (left >= OPT_ITEMS) u.load(static_cast<const uint16_t*>(p) + at);
  else u.clear();
}
__device__ __forceinline__ void load_unit(Raw8<float>& u, const void* p, int64_t at, int left) {
  const float* f = static_cast<const float*>(p) + at;
  u.clear();
  if (left > 0) u.a = *reinterpret_cast<const f32x4_t*>(f);
  if (left >= OPT_ITEMS) u.b = *reinterpret_cast<const f32x4_t*>(f + 4);
}
// STREAM: past the caches, for s and dx, which nothing reads soon; h is read next and stays in them.  rms_norm with a residual and then a product with h, s cached
// / past the caches / h past them as well: 16384 x 4096 181 / 176 / 184 us, 1900 x 8192 73 / 68 / 73, 64 x 4096 15.7 / 15.7 / 18.5.
template <bool STREAM, typename V>
__device__ __forceinline__ void store_word(void* p, const V& v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<V*>(p));
  else *static_cast<V*>(p) = v;
}
template <bool STREAM = false>
__device__ __forceinline__ void store_unit(uint16_t* p, int64_t at, int left, const float (&o)[OPT_ITEMS]) {
  if (left < OPT_ITEMS) return;
  i32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (int)pack_bf16(o[2 * i], o[2 * i + 1]);
  store_word<STREAM>(p + at, w);
}
template <bool STREAM = false>
__device__ __forceinline__ void store_unit(float* p, int64_t at, int left, const float (&o)[OPT_ITEMS]) {
  if (left > 0) store_word<STREAM>(p + at, f32x4_t{o[0], o[1], o[2], o[3]});
  if (left >= OPT_ITEMS) store_word<STREAM>(p + at + 4, f32x4_t{o[4], o[5], o[6], o[7]});
}
__device__ __forceinline__ void load_weights(const void* w, int bf16, int at, int left, float (&o)[OPT_ITEMS]) {
  if (bf16) {                                        // uniform
    Raw8<uint16_t> u;
    if (left >= OPT_ITEMS) {
      u.load(static_cast<const uint16_t*>(w) + at);
    } else {
      u.clear();                                     // four of them: fp32 rows beside bf16 weights
      if (left > 0) {
        const u32x2 two = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(w) + at);
        u.w[0] = (int)two[0];
        u.w[1] = (int)two[1];
      }
    }
    u.get(o);
  } else {
    Raw8<float> u;
    load_unit(u, w, at, left);
    u.get(o);
  }
}
// 1 / sqrt(v) of a mean in 64 bits: the hardware's estimate and two steps of Newton's; 0 for an infinite mean
__device__ __forceinline__ float inverse_root(double v) {
  double y = __builtin_amdgcn_rsq(v);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = y * fma(-0.5 * v * y, y, 1.5);
  return v == (double)INFINITY ? 0.f : (float)y;
}

// TH threads a row, UNITS units of eight entries a thread (unit i of thread t: columns 8 (i TH + t) ..); a block of 256 threads has four
// rows of 64, others one.
template <int TH>
constexpr int NORM_THREADS_OF = TH < 256 ? 256 : TH;
template <typename T, int OUT, int TH, int UNITS>
__global__ __launch_bounds__(NORM_THREADS_OF<TH>) void k_rms_norm(NormArgs a) {
  constexpr int ROWS = NORM_THREADS_OF<TH> / TH, WAVES = TH / 64;
  __shared__ double s_sum[WAVES];
  __shared__ uint32_t s_top[WAVES];
  const int tid = threadIdx.x % TH, lane = threadIdx.x & 63, wave = tid / 64;
  const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? wave_id() : 0);
  if (row >= a.N) return;                            // TH 64: of a wavefront, and there is no barrier;  else never
  const int64_t first = row * a.d;
  Raw8<T> x[UNITS], y[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const int col = (i * TH + tid) * OPT_ITEMS;
    load_unit(x[i], a.x, first + col, a.d - col);
  }
  if (a.residual != nullptr) {                       // uniform
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      load_unit(y[i], a.residual, first + col, a.d - col);
    }
  }
  float s[UNITS][OPT_ITEMS], w[UNITS][OPT_ITEMS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const int col = (i * TH + tid) * OPT_ITEMS;
    load_weights(a.w, a.w_bf16, col, a.d - col, w[i]);
  }
  double sq = 0.0;
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const int col = (i * TH + tid) * OPT_ITEMS;
    x[i].get(s[i]);
    if (a.residual != nullptr) {
      float t[OPT_ITEMS];
      y[i].get(t);
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) s[i][e] += t[e];
      store_unit<true>(static_cast<T*>(a.sum), first + col, a.d - col, s[i]);
      if constexpr (sizeof(T) == 2) {                // as it is stored
#pragma unroll
        for (int e = 0; e < OPT_ITEMS; e += 2) {
          const uint32_t p = pack_bf16(s[i][e], s[i][e + 1]);
          s[i][e] = __uint_as_float(p << 16);
          s[i][e + 1] = __uint_as_float(p & 0xffff0000u);
        }
      }
    }
    sq = add_squares(s[i], sq);
  }
  sq = wave_sum(sq);
  if constexpr (WAVES > 1) {
    if (lane == 0) s_sum[wave] = sq;
    __syncthreads();
    sq = s_sum[0];
#pragma unroll
    for (int q = 1; q < WAVES; ++q) sq += s_sum[q];
  }
  const float r = inverse_root(sq / (double)a.d + (double)a.eps);
  if (tid == 0 && a.rstd != nullptr) a.rstd[row] = r;
#pragma unroll
  for (int i = 0; i < UNITS; ++i)
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) s[i][e] = s[i][e] * r * w[i][e];
  if constexpr (OUT == OUT_SAME) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      store_unit(static_cast<T*>(a.h), first + col, a.d - col, s[i]);
    }
  } else if constexpr (OUT == OUT_BLOCKS) {         // 16 lanes a block, a wavefront's unit a word of four
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS, group = i * WAVES + wave;
      if (group * SCALE_GROUP >= a.d) break;         // wave-uniform
      if (col >= a.d) {
#pragma unroll
        for (int e = 0; e < OPT_ITEMS; ++e) s[i][e] = 0.f;      // past the row: whatever came of no weights
      }
      const int e = block_exponent(row_max(magnitude8(s[i])));
      if (col < a.d) *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.h) + first + col) = quantise8(s[i], e);
      const uint32_t word = scale_word(e);
      if (lane == 0) static_cast<uint32_t*>(a.scale)[(int64_t)group * a.N + row] = word;
    }
  } else {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      if (col < a.d) top = top_magnitude(s[i], top);
    }
    top = wave_top(top);
    if constexpr (WAVES > 1) {
      if (lane == 0) s_top[wave] = top;
      __syncthreads();
      top = s_top[0];
#pragma unroll
      for (int q = 1; q < WAVES; ++q) top = max(top, s_top[q]);
    }
    const float scale = int8_scale(top);
    const Int8Quotient by(scale);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      if (col < a.d) *reinterpret_cast<u32x2*>(static_cast<int8_t*>(a.h) + first + col) = by(s[i]);
    }
    if (tid == 0) static_cast<float*>(a.scale)[row] = scale;
  }
}

struct NormBwdArgs {
  const void* dh;
  const void* s;
  const void* w;
  const float* rstd;
  const void* dsum;        // null: none
  int64_t N;
  int d;
  int w_bf16;
  void* dx;
  float* part;             // [row_blocks][d]; null: dw is not asked for, or
  int row_blocks;
  void* dw;                // ... the workgroups behind the row_blocks sum up a few columns each
  int dw_bf16;
};
// dw of few rows: NORM_COLUMNS columns a workgroup, dh and s read a second time (from L2), where partial sums would take a launch more: 333 x 520
// 3.8 + 3.1 us.
constexpr int64_t NORM_FEW_ROWS = 512;
constexpr int NORM_COLUMNS = 64;
template <typename T, int THREADS>
__device__ __forceinline__ void norm_columns(const NormBwdArgs& a, int block) {
  constexpr int LANES = NORM_COLUMNS / OPT_ITEMS, SLICES = THREADS / LANES;
  __shared__ float s_dw[SLICES][NORM_COLUMNS + 1];
  const int slice = threadIdx.x / LANES, col = block * NORM_COLUMNS + threadIdx.x % LANES * OPT_ITEMS;
  float dw[OPT_ITEMS] = {};
#pragma unroll 4
  for (int64_t row = slice; row < a.N; row += SLICES) {
    Raw8<T> g, x;
    load_unit(g, a.dh, row * a.d + col, a.d - col);
    load_unit(x, a.s, row * a.d + col, a.d - col);
    const float r = a.rstd[row];
    float dh[OPT_ITEMS], s[OPT_ITEMS];
    g.get(dh);
    x.get(s);
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) dw[e] = fmaf(dh[e], s[e] * r, dw[e]);
  }
#pragma unroll
  for (int e = 0; e < OPT_ITEMS; ++e) s_dw[slice][threadIdx.x % LANES * OPT_ITEMS + e] = dw[e];
  __syncthreads();
  const int c = threadIdx.x;
  if (c >= NORM_COLUMNS || block * NORM_COLUMNS + c >= a.d) return;
  float t = 0.f;
  for (int q = 0; q < SLICES; ++q) t += s_dw[q][c];
  if (a.dw_bf16) static_cast<uint16_t*>(a.dw)[block * NORM_COLUMNS + c] = float_to_bf16_bits(t);
  else static_cast<float*>(a.dw)[block * NORM_COLUMNS + c] = t;
}
// Workgroups of 256 to 1024 threads walk over the rows, TH threads a row, the next row on its way (1900 x 8192: 34 -> 24 us, with 256 workgroups for 1024), the columns' share of dw in registers; its sums of a workgroup meet in LDS.
// Two workgroups a CU (one of 1024 threads): what a workgroup leaves of dw is written and read again, 4 d bytes each.
constexpr int NORM_BWD_BLOCKS = 512;
template <typename T, int TH, int UNITS>
__global__ __launch_bounds__(NORM_THREADS_OF<TH>) void k_rms_norm_bwd(NormBwdArgs a) {
  constexpr int ROWS = NORM_THREADS_OF<TH> / TH, WAVES = TH / 64;
  __shared__ float s_dot[2][WAVES];
  __shared__ float s_dw[ROWS > 1 ? ROWS * TH * UNITS * OPT_ITEMS : 1];
  if ((int)blockIdx.x >= a.row_blocks) return norm_columns<T, NORM_THREADS_OF<TH>>(a, blockIdx.x - a.row_blocks);
  const int tid = threadIdx.x % TH, lane = threadIdx.x & 63, wave = tid / 64, own = ROWS > 1 ? wave_id() : 0;
  constexpr bool ROOMY = TH * UNITS < 2048;                // 1024 threads have 128 registers each: w comes from L2 row by row, dsum late
  float w[UNITS][OPT_ITEMS], dw[UNITS][OPT_ITEMS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const int col = (i * TH + tid) * OPT_ITEMS;
    if constexpr (ROOMY) load_weights(a.w, a.w_bf16, col, a.d - col, w[i]);
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) dw[i][e] = 0.f;
  }
  const float inv_d = 1.f / (float)a.d;
  int turn = 0;
  Raw8<T> g[UNITS], x[UNITS], u[UNITS];
  float r = 0.f;
  const int64_t stride = (int64_t)a.row_blocks * ROWS;
  auto load_sums = [&](int64_t row) {
    if (a.dsum != nullptr) {                         // uniform
#pragma unroll
      for (int i = 0; i < UNITS; ++i) load_unit(u[i], a.dsum, row * a.d + (i * TH + tid) * OPT_ITEMS, a.d - (i * TH + tid) * OPT_ITEMS);
    }
  };
  auto load_row = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      load_unit(g[i], a.dh, row * a.d + col, a.d - col);
      load_unit(x[i], a.s, row * a.d + col, a.d - col);
    }
    r = a.rstd[row];
    if constexpr (ROOMY) load_sums(row);
  };
  int64_t row = (int64_t)blockIdx.x * ROWS + own;
  if (ROOMY && row < a.N) load_row(row);
  for (; row < a.N; row += stride, turn ^= 1) {
    const int64_t first = row * a.d;
    if constexpr (!ROOMY) load_row(row);
    float dh[UNITS][OPT_ITEMS], s[UNITS][OPT_ITEMS];
    Raw8<T> more[UNITS];
    const float rs = r;
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      g[i].get(dh[i]);
      x[i].get(s[i]);
      if constexpr (ROOMY) more[i] = u[i];
    }
    if constexpr (ROOMY) {                           // the next row on its way while this one is reduced and stored
      if (row + stride < a.N) load_row(row + stride);
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      if constexpr (!ROOMY) load_weights(a.w, a.w_bf16, col, a.d - col, w[i]);
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) {
        const float n = s[i][e] * rs;
        dot = fmaf(dh[i][e] * w[i][e], n, dot);
        dw[i][e] = fmaf(dh[i][e], n, dw[i][e]);
      }
    }
    dot = wave_sum(dot);
    if constexpr (WAVES > 1) {                       // two rows' sums in turn: one barrier a row
      if (lane == 0) s_dot[turn][wave] = dot;
      __syncthreads();
      dot = s_dot[turn][0];
#pragma unroll
      for (int q = 1; q < WAVES; ++q) dot += s_dot[turn][q];
    }
    const float mean = dot * inv_d;
    if constexpr (!ROOMY) load_sums(row);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      float o[OPT_ITEMS];
      if constexpr (!ROOMY) {
        load_weights(a.w, a.w_bf16, col, a.d - col, w[i]);
        more[i] = u[i];
      }
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) o[e] = rs * fmaf(-(s[i][e] * rs), mean, dh[i][e] * w[i][e]);
      if (a.dsum != nullptr) {
        float t[OPT_ITEMS];
        more[i].get(t);
#pragma unroll
        for (int e = 0; e < OPT_ITEMS; ++e) o[e] += t[e];
      }
      store_unit<true>(static_cast<T*>(a.dx), first + col, a.d - col, o);
    }
  }
  if (a.part == nullptr) return;                     // uniform
  float* out = a.part + (int64_t)blockIdx.x * a.d;
  if constexpr (ROWS > 1) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) s_dw[own * (TH * UNITS * OPT_ITEMS) + (i * TH + tid) * OPT_ITEMS + e] = dw[i][e];
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += NORM_THREADS_OF<TH>) {
      float t = s_dw[c];
#pragma unroll
      for (int q = 1; q < ROWS; ++q) t += s_dw[q * (TH * UNITS * OPT_ITEMS) + c];
      out[c] = t;
    }
  } else {
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      store_unit(out, col, a.d - col, dw[i]);
    }
  }
}

// dw of 32 columns: 32 slices of the partial rows, summed in order
constexpr int NORM_DW_COLS = 32, NORM_DW_SLICES = 32;
__global__ __launch_bounds__(NORM_DW_COLS* NORM_DW_SLICES) void k_norm_dw(const float* part, int rows, int d, void* dw, int bf16) {
  __shared__ float s[NORM_DW_SLICES][NORM_DW_COLS];
  const int c = threadIdx.x % NORM_DW_COLS, slice = threadIdx.x / NORM_DW_COLS;
  const int64_t col = (int64_t)blockIdx.x * NORM_DW_COLS + c;
  float t = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int q = slice; q < rows; q += NORM_DW_SLICES) t += part[(int64_t)q * d + col];
  }
  s[slice][c] = t;
  __syncthreads();
  if (slice == 0 && col < d) {
    for (int q = 1; q < NORM_DW_SLICES; ++q) t += s[q][c];
    if (bf16) static_cast<uint16_t*>(dw)[col] = float_to_bf16_bits(t);
    else static_cast<float*>(dw)[col] = t;
  }
}

}  // namespace llamarl
