// optim_kernels.h -- what a trainer does with the gradients: their norm over all tensors, and one AdamW step over all tensors.
//
//   k_grad_squares   sum of squares of each block of entries, in 64 bits
//   k_grad_norm      norm = sqrt(sum), scale = the factor that brings a norm above max_norm down to it
//   k_adamw          m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p -= lr (wd p + (m / c1) / (sqrt(v / c2) + eps)),
//                    c = 1 - b^t, g times the scale; states in fp32 or in 8 bits
//
// Both passes are bound by memory: every entry is read once, what changes is written once, and nothing is kept between the passes
// (the norm has to be known before the first entry moves).  A launch takes up to OPT_TENSORS tensors, described in its arguments:
// no table in memory that a caller would have to keep, or a captured graph could find changed.
//
// States in 8 bits: STATE_BLOCK neighbouring entries of a tensor share one fp32 factor, their largest magnitude / 448, and each
// is held as e4m3 times that.  The second moment is held as its square root, which halves the exponents it spans.  m is rounded
// to nearest: an update moves it by (1 - b1) |g - m|, a tenth of the difference, and half a step is 3 - 6 % of it.  What is below
// that is lost, so that m can stay up to 0.63 of itself away from a constant gradient (b1 = 0.9), but not on the other side of
// zero: b1 <= STATE_BETA1 takes more than half a step off any code above 2^-6 when the gradient is zero (1.125 -> 1.0547, nearer
// to 1).  sqrt(v) moves by less than a rounding step in one update (0.05 % at b2 = 0.999, a step is 6 - 12 %): rounded to nearest
// it would stay where it is however long the gradients say otherwise, so it is rounded up or down with the probability that keeps
// its mean, by bits hashed out of (step, tensor, entry) -- the same call gives the same bits.  A second moment that is not zero
// is never rounded to zero, where its entry would next be divided by eps: below the smallest code it counts as that.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm_nt.h"
#include "loss_kernels.h"

namespace llamarl {

constexpr int OPT_TENSORS = 48;              // tensors of a launch: 3.5 of the 4 KB of kernel arguments
// 512 threads against 256, in turn on one card: 8-bit states of the 8B head 1576 -> 1544 us, 32-bit ones and the norm 3362 -> 3338
constexpr int OPT_THREADS = 512, OPT_ITEMS = 8, OPT_UNIT = OPT_THREADS * OPT_ITEMS;
constexpr int STATE_BLOCK = 128;             // 16 lanes of eight entries: one row of a wavefront's cross-lane moves
constexpr float E4M3_MAX = 448.f;
constexpr double STATE_BETA1 = 0.9375;       // largest b1 of first moments in 8 bits
constexpr float STATE_TINY = 0x1p-100f;      // a block whose largest magnitude is below this is held as zeros (its inverse overflows)
constexpr int NORM_BLOCKS = 8192;            // partial sums of a gradient norm: at most so many and one a tensor

enum OptFlags { OPT_P_BF16 = 1, OPT_G_BF16 = 2, OPT_8BIT = 4, OPT_WIDE = 8 /* 16-byte accesses of every array are aligned */ };
struct OptTensor {
  void* p;
  float* master;
  const void* g;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  int64_t n;
  int flags;
  uint32_t place;                            // in the caller's list: part of the rounding bits' hash
};
struct OptList {
  OptTensor t[OPT_TENSORS];
  int first[OPT_TENSORS + 1];                // first workgroup of each tensor
  int count;
  int units;                                 // of OPT_UNIT entries that a workgroup takes (k_adamw: one)
};
// Tensor of this workgroup: the last whose first workgroup is not past it.  A lane looks at a tensor: one load, where a search would
// be a chain of them, which a list of small tensors waits for.
static_assert(OPT_TENSORS <= 64, "a lane a tensor");
__device__ __forceinline__ int opt_tensor_of(const OptList& l) {
  const int lane = threadIdx.x & 63;
  const uint64_t past = __ballot(lane < l.count && l.first[lane < OPT_TENSORS ? lane : 0] <= (int)blockIdx.x);
  return 63 - __builtin_clzll(past);
}

// Eight neighbouring entries from `at` on: 16-byte accesses where all eight exist and the tensor is aligned.
__device__ __forceinline__ void load8(const float* x, int64_t at, int left, bool wide, float (&o)[OPT_ITEMS]) {
  if (wide && left >= OPT_ITEMS) {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(x + at), b = *reinterpret_cast<const f32x4_t*>(x + at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] = a[i];
      o[i + 4] = b[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i) o[i] = i < left ? x[at + i] : 0.f;
  }
}
__device__ __forceinline__ void load8(const uint16_t* x, int64_t at, int left, bool wide, float (&o)[OPT_ITEMS]) {
  if (wide && left >= OPT_ITEMS) {
    const i32x4_t a = *reinterpret_cast<const i32x4_t*>(x + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float((uint32_t)a[i] << 16);
      o[2 * i + 1] = __uint_as_float((uint32_t)a[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i) o[i] = i < left ? bf16_bits_to_float(x[at + i]) : 0.f;
  }
}
__device__ __forceinline__ void load8(const void* x, bool bf16, int64_t at, int left, bool wide, float (&o)[OPT_ITEMS]) {
  if (bf16) load8(static_cast<const uint16_t*>(x), at, left, wide, o);
  else load8(static_cast<const float*>(x), at, left, wide, o);
}
__device__ __forceinline__ void store8(float* x, int64_t at, int left, bool wide, const float (&o)[OPT_ITEMS]) {
  if (wide && left >= OPT_ITEMS) {
    *reinterpret_cast<f32x4_t*>(x + at) = f32x4_t{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4_t*>(x + at + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i)
      if (i < left) x[at + i] = o[i];
  }
}
__device__ __forceinline__ void store8(uint16_t* x, int64_t at, int left, bool wide, const float (&o)[OPT_ITEMS]) {
  uint16_t b[OPT_ITEMS];
#pragma unroll
  for (int i = 0; i < OPT_ITEMS; ++i) b[i] = float_to_bf16_bits(o[i]);
  if (wide && left >= OPT_ITEMS) {
    i32x4_t a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = (int)((uint32_t)b[2 * i] | (uint32_t)b[2 * i + 1] << 16);
    *reinterpret_cast<i32x4_t*>(x + at) = a;
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i)
      if (i < left) x[at + i] = b[i];
  }
}

// ---- norm ------------------------------------------------------------------------------------------------------------------
// Squares and sums in 64 bits: no entry's square overflows or vanishes, and the order of half a billion additions does not show.
__device__ __forceinline__ double add_squares(const float (&x)[OPT_ITEMS], double s) {
#pragma unroll
  for (int i = 0; i < OPT_ITEMS; ++i) s = fma((double)x[i], (double)x[i], s);
  return s;
}
// Whole units of an aligned tensor, NORM_LOADS of them asked for before the first is used: one at a time leaves few
// bytes in flight where the gradients are bf16.  109 tensors of a 170 M model, bf16 79.7 -> 69.4 us, fp32 132 -> 127; 525 M entries 185 -> 183, 358 -> 349.
constexpr int NORM_LOADS = 4;
template <typename T>
__device__ __forceinline__ double unit_squares(const T* g, int64_t at, double s) {
  constexpr int WORDS = OPT_ITEMS * (int)sizeof(T) / 16;
  i32x4_t w[NORM_LOADS][WORDS];
#pragma unroll
  for (int q = 0; q < NORM_LOADS; ++q)
#pragma unroll
    for (int c = 0; c < WORDS; ++c) w[q][c] = *reinterpret_cast<const i32x4_t*>(g + at + (int64_t)q * OPT_UNIT + c * (16 / sizeof(T)));
#pragma unroll
  for (int q = 0; q < NORM_LOADS; ++q) {
    float x[OPT_ITEMS];
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __uint_as_float((uint32_t)w[q][i / 4][i % 4]);
      else x[i] = __uint_as_float(i % 2 == 0 ? (uint32_t)w[q][0][i / 2] << 16 : (uint32_t)w[q][0][i / 2] & 0xffff0000u);
    }
    s = add_squares(x, s);
  }
  return s;
}
__global__ __launch_bounds__(OPT_THREADS) void k_grad_squares(OptList l, double* part) {
  const int t = opt_tensor_of(l);
  const int64_t n = l.t[t].n, from = (int64_t)((int)blockIdx.x - l.first[t]) * l.units * OPT_UNIT;
  const bool bf16 = (l.t[t].flags & OPT_G_BF16) != 0, wide = (l.t[t].flags & OPT_WIDE) != 0;
  const void* g = l.t[t].g;
  double s = 0.0;
  int u = 0;
  if (wide)                                          // uniform, as is the loop's end
    for (; u + NORM_LOADS <= l.units && from + (int64_t)(u + NORM_LOADS) * OPT_UNIT <= n; u += NORM_LOADS) {
      const int64_t at = from + (int64_t)u * OPT_UNIT + threadIdx.x * OPT_ITEMS;
      s = bf16 ? unit_squares(static_cast<const uint16_t*>(g), at, s) : unit_squares(static_cast<const float*>(g), at, s);
    }
  for (; u < l.units; ++u) {
    const int64_t at = from + (int64_t)u * OPT_UNIT + threadIdx.x * OPT_ITEMS;
    if (at >= n) break;
    float x[OPT_ITEMS];
    load8(g, bf16, at, (int)min(n - at, (int64_t)OPT_ITEMS), wide, x);
    s = add_squares(x, s);
  }
  __shared__ double s_w[OPT_THREADS / 64];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = s_w[0];
#pragma unroll
    for (int w = 1; w < OPT_THREADS / 64; ++w) s += s_w[w];
    part[blockIdx.x] = s;
  }
}
// One workgroup; the sums in the order of the list.
constexpr int NORM_THREADS = 1024;
__global__ __launch_bounds__(NORM_THREADS) void k_grad_norm(const double* part, int64_t count, float max_norm, float* norm, float* scale) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < count; i += NORM_THREADS) s += part[i];
  __shared__ double s_w[NORM_THREADS / 64];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < NORM_THREADS / 64; ++w) s += s_w[w];
    const double r = sqrt(s);
    *norm = (float)r;
    *scale = !isfinite(r) ? __builtin_nanf("") : r > (double)max_norm ? (float)((double)max_norm / r) : 1.f;
  }
}

// ---- AdamW -----------------------------------------------------------------------------------------------------------------
struct AdamwArgs {
  OptList l;
  float lr, b1, one_b1, b2, one_b2, eps, decay;
  float inv_c1, inv_sqrt_c2;                 // 1 / (1 - b1^t), 1 / sqrt(1 - b2^t)
  double beta1, beta2;                       // for a step that is on the device
  int64_t step;
  const float* scale;                        // null: 1
  const float* lr_device;                    // null: lr
  const int64_t* step_device;                // null: step
};

__device__ __forceinline__ double power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}
// Rounded correctly: the estimate of 1 / sqrt(v), one step of Newton's iteration whose residual is exact.  v_rsq_f32 alone loses what
// lies below the normal numbers.
__device__ __forceinline__ float root(float v) {
  const bool small = v < 0x1p-96f;
  const float x = small ? v * 0x1p64f : v, e = __builtin_amdgcn_rsqf(x);
  const float s = x * e, r = fmaf(fmaf(-s, s, x), 0.5f * e, s);
  return !(x > 0.f && x < INFINITY) ? x : small ? r * 0x1p-32f : r;
}
// x / s for several x, rounded correctly: the reciprocal is made once, and a quotient's residual is exact
struct Quotient {
  float s, inv;
  __device__ __forceinline__ explicit Quotient(float s_) : s(s_) {
    const float e = __builtin_amdgcn_rcpf(s_);
    inv = fmaf(fmaf(-s_, e, 1.f), e, e);
  }
  __device__ __forceinline__ float operator()(float x) const {
    const float q = x * inv;
    return fmaf(fmaf(-q, s, x), inv, q);
  }
};
// over the 16 lanes of a block's row, in every lane; a NaN is passed over
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __uint_as_float(dpp_move<ROW_ROR(8)>(__float_as_uint(x))));
  x = fmaxf(x, __uint_as_float(dpp_move<ROW_ROR(4)>(__float_as_uint(x))));
  x = fmaxf(x, __uint_as_float(dpp_move<ROW_ROR(2)>(__float_as_uint(x))));
  return fmaxf(x, __uint_as_float(dpp_move<ROW_ROR(1)>(__float_as_uint(x))));
}
// 16 random bits for each of the entries 2 pair (low half) and 2 pair + 1 of a tensor.  Multiplicative hashing of a counter; the
// odd factors are 2^32 / golden ratio and 2^30, 2^31 times roots of 2, 3, 5.
__device__ __forceinline__ uint32_t rounding_bits(uint32_t pair, uint32_t step, uint32_t place) {
  uint32_t x = pair + step * 0x9E3779B9u + place * 0xB504F333u;
  x = (x ^ x >> 16) * 0xDDB3D743u;
  x = (x ^ x >> 15) * 0x8F1BBCDDu;
  return x ^ x >> 16;
}
// y in [0, 448] up to a rounding: the e4m3 value below or above it, above with the probability of its distance from below in 2^-16.  e4m3
// has three mantissa bits: of fp32's 23 the last 20 go.  Below the normal numbers (2^-6) the steps are those just above.
__device__ __forceinline__ float round_by(float y, uint32_t bits16) {
  const float lift = y < 0x1p-6f ? 0x1p-6f : 0.f;
  const float z = __uint_as_float((__float_as_uint(y + lift) + (bits16 << 4)) & 0xfff00000u) - lift;
  return y > 0.f ? fminf(fmaxf(z, 0x1p-9f), E4M3_MAX) : y;
}
__device__ __forceinline__ void from_e4m3(uint32_t w, float scale, float* o) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  o[0] = a[0] * scale;
  o[1] = a[1] * scale;
  o[2] = b[0] * scale;
  o[3] = b[1] * scale;
}
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// eight states of a thread; `left` of them exist
__device__ __forceinline__ void load_states(const uint8_t* q, float scale, int64_t at, int left, bool wide, float (&o)[OPT_ITEMS]) {
  u32x2 w = {0u, 0u};
  if (wide && left >= OPT_ITEMS) {
    w = *reinterpret_cast<const u32x2*>(q + at);
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i)
      if (i < left) w[i / 4] |= (uint32_t)q[at + i] << 8 * (i % 4);
  }
  from_e4m3(w[0], scale, o);
  from_e4m3(w[1], scale, o + 4);
}
__device__ __forceinline__ void store_states(uint8_t* q, int64_t at, int left, bool wide, u32x2 w) {
  if (wide && left >= OPT_ITEMS) {
    *reinterpret_cast<u32x2*>(q + at) = w;
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i)
      if (i < left) q[at + i] = (uint8_t)(w[i / 4] >> 8 * (i % 4));
  }
}

__global__ __launch_bounds__(OPT_THREADS) void k_adamw(AdamwArgs a) {
  const float gs = a.scale != nullptr ? *a.scale : 1.f;
  const float lr = a.lr_device != nullptr ? *a.lr_device : a.lr;
  float inv_c1 = a.inv_c1, inv_sqrt_c2 = a.inv_sqrt_c2;
  int64_t step = a.step;
  if (a.step_device != nullptr) {
    step = max(*a.step_device, (int64_t)1);
    inv_c1 = (float)(1.0 / (1.0 - power(a.beta1, step)));
    inv_sqrt_c2 = (float)(1.0 / sqrt(1.0 - power(a.beta2, step)));
  }
  const int ti = opt_tensor_of(a.l);
  const OptTensor& t = a.l.t[ti];
  const int64_t at = (int64_t)((int)blockIdx.x - a.l.first[ti]) * OPT_UNIT + threadIdx.x * OPT_ITEMS;
  // lanes past the end stay: a block's row finds its maximum together
  const int left = (int)max((int64_t)0, min(t.n - at, (int64_t)OPT_ITEMS));
  const int flags = t.flags;
  const bool wide = (flags & OPT_WIDE) != 0, p_bf16 = (flags & OPT_P_BF16) != 0, g_bf16 = (flags & OPT_G_BF16) != 0;
  const bool bits8 = (flags & OPT_8BIT) != 0;
  float g[OPT_ITEMS], p[OPT_ITEMS], m[OPT_ITEMS], r[OPT_ITEMS];  // r: sqrt(v)
  load8(t.g, g_bf16, at, left, wide, g);
  // A step whose scale is not finite is not taken.  Asked here, not before the loads: the scale is a load itself.
  const bool taken = fabsf(gs) < INFINITY; // uniform
  if (t.master != nullptr) load8(t.master, at, left, wide, p);
  else load8(t.p, p_bf16, at, left, wide, p);
  if (!bits8) {
    float v[OPT_ITEMS];
    load8(static_cast<const float*>(t.m), at, left, wide, m);
    load8(static_cast<const float*>(t.v), at, left, wide, v);
    if (!taken) return;
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i) {
      const float x = g[i] * gs;
      m[i] = fmaf(a.b1, m[i], a.one_b1 * x);
      v[i] = fmaf(a.b2, v[i], a.one_b2 * x * x);
      r[i] = root(v[i]);
    }
    store8(static_cast<float*>(t.m), at, left, wide, m);
    store8(static_cast<float*>(t.v), at, left, wide, v);
  } else {
    const int64_t block = at / STATE_BLOCK;
    float ms = 0.f, rs = 0.f;
    if (left > 0) {
      ms = t.m_scale[block];
      rs = t.v_scale[block];
    }
    load_states(static_cast<const uint8_t*>(t.m), ms, at, left, wide, m);
    load_states(static_cast<const uint8_t*>(t.v), rs, at, left, wide, r);
    if (!taken) return;
    float top_m = 0.f, top_r = 0.f;
    {
      // Every operation rounded by itself, so that the codes are what the formula gives in any other program: a last bit can turn a code,
      // a code turn the block's next largest magnitude, and two runs of a model then part.
#pragma clang fp contract(off)
#pragma unroll
      for (int i = 0; i < OPT_ITEMS; ++i) {
        const float x = g[i] * gs;
        m[i] = m[i] * a.b1 + x * a.one_b1;
        r[i] = root(r[i] * r[i] * a.b2 + x * x * a.one_b2);
        top_m = fmaxf(top_m, fabsf(m[i]));
        top_r = fmaxf(top_r, r[i]);
      }
    }
    top_m = row_max(top_m);
    top_r = row_max(top_r);
    const float sm = top_m < STATE_TINY ? 0.f : top_m * (1.f / E4M3_MAX), sr = top_r < STATE_TINY ? 0.f : top_r * (1.f / E4M3_MAX);
    const Quotient by_m(sm > 0.f ? sm : 1.f), by_r(sr > 0.f ? sr : 1.f);
    const float keep_m = sm > 0.f ? 1.f : 0.f, keep_r = sr > 0.f ? 1.f : 0.f;
    u32x2 qm, qr;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e = 4 * h;
      qm[h] = to_e4m3(by_m(m[e] * keep_m), by_m(m[e + 1] * keep_m), by_m(m[e + 2] * keep_m), by_m(m[e + 3] * keep_m));
      const uint32_t pair = (uint32_t)(at >> 1) + 2 * h;
      const uint32_t x = rounding_bits(pair, (uint32_t)step, t.place), y = rounding_bits(pair + 1, (uint32_t)step, t.place);
      qr[h] = to_e4m3(round_by(by_r(r[e] * keep_r), x & 0xffffu), round_by(by_r(r[e + 1] * keep_r), x >> 16),
                      round_by(by_r(r[e + 2] * keep_r), y & 0xffffu), round_by(by_r(r[e + 3] * keep_r), y >> 16));
    }
    store_states(static_cast<uint8_t*>(t.m), at, left, wide, qm);
    store_states(static_cast<uint8_t*>(t.v), at, left, wide, qr);
    if (left > 0 && (threadIdx.x & 15) == 0) {
      t.m_scale[block] = sm;
      t.v_scale[block] = sr;
    }
  }
  // the change is summed before it is taken off: lr wd is below the last bit of 1 for the learning rates in use
#pragma unroll
  for (int i = 0; i < OPT_ITEMS; ++i)
    p[i] -= lr * fmaf(a.decay, p[i], m[i] * inv_c1 * __builtin_amdgcn_rcpf(fmaf(r[i], inv_sqrt_c2, a.eps)));
  if (t.master != nullptr) store8(t.master, at, left, wide, p);
  if (p_bf16) store8(static_cast<uint16_t*>(t.p), at, left, wide, p);
  else store8(static_cast<float*>(t.p), at, left, wide, p);
}

}  // namespace llamarl
