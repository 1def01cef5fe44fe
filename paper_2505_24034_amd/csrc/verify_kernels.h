// verify_kernels.h -- drafted tokens against the target's distribution.
//
// Sequence b has drafts x_0 .. x_{n-1}, target logits for each of their places and the one behind, numbers u_0 .. u_K in [0, 1).  With
// p_i = softmax(target logits / T) and q_i = softmax(draft logits / T), or all of it on x_i where drafts have no distribution:
//
//   draft i is accepted while u_i q_i(x_i) < p_i(x_i);     the first that is not is replaced by a token of max(p_i - q_i, 0), normalised;
//   behind n accepted drafts comes a token of p_n.         Either is the first v with  sum_{w <= v} r(w) > u_K sum_w r(w).
//
// so what leaves is distributed as p whatever q is.  T = 0: p is all on the first of the largest logits.
//
//   k_verify_rows    every row's largest logit and sum of exponentials, in chunks
//   k_verify_sums    accepted drafts; the chunks' sums of r, one row a sequence
//   k_verify_pick    the chunk, then the token that u_K falls on; outputs
//
// Bound by memory (every row once, then one or two rows a sequence) and, for small batches, by the three launches.  Everything that decides is in 64
// bits: a token is one of V borders, and with fp32's 1e-7 in each of 128256 terms every tenth sample would have moved by a token.  fp64 runs at fp32's
// rate here; the exponential is a polynomial of degree 9.
#pragma once
#include "norm_kernels.h"

namespace llamarl {

constexpr int VERIFY_THREADS = 256, VERIFY_UNITS = 4, VERIFY_CHUNK = VERIFY_THREADS * VERIFY_UNITS * OPT_ITEMS;      // logits of a workgroup
constexpr int VERIFY_MOST_DRAFTS = 127;              // 2 K + 1 rows of a sequence: a thread each
constexpr int PICK_THREADS = VERIFY_CHUNK / OPT_ITEMS;

// e^x for x <= 0, within 3e-14 of it; 0 below e^-745.  x = n ln 2 + f, |f| <= ln 2 / 2; e^f interpolated at Chebyshev's nodes.
__device__ __forceinline__ double exp_below(double x) {
  x = fmax(x, -800.0);
  const double n = __builtin_rint(x * 0x1.71547652b82fep+0), f = fma(n, -0x1.62e42fefa39efp-1, x);
  double y = 0x1.72e12288ba07ep-19;
  y = fma(y, f, 0x1.a17e155b49e91p-16);
  y = fma(y, f, 0x1.a01994b1cb939p-13);
  y = fma(y, f, 0x1.6c162b99260a8p-10);
  y = fma(y, f, 0x1.11111123c4de7p-7);
  y = fma(y, f, 0x1.55555588c80e6p-5);
  y = fma(y, f, 0x1.5555555550d6ap-3);
  y = fma(y, f, 0x1.ffffffffe744fp-2);
  y = fma(y, f, 0x1.0000000000006p+0);
  y = fma(y, f, 0x1.000000000003dp+0);
  return __builtin_amdgcn_ldexp(y, (int)n);
}

struct VerifyArgs {
  const void* z;           // target logits [B][K+1][V]
  const void* y;           // draft logits [B][K][V], or null
  const int32_t* drafts;   // [B][K]
  const int32_t* lens;     // [B] or null: K
  const float* temps;      // [B] or null: 1
  const float* u;          // [B][K+1]
  int64_t V;
  int B, K, chunks;
  float* part_m;           // [rows][chunks], rows: B (K+1) of the target, then B K of the drafts
  double* part_s;
  int32_t* part_i;         // first place of part_m, T = 0 only
  double* sum_r;           // [B][chunks]
  double* sum_p;
  int32_t* tokens;         // [B][K+1]
  int32_t* accepted;       // [B]
  float* logp;             // [B][K+1]
};
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int b) { return a.lens == nullptr ? a.K : min(max(a.lens[b], 0), a.K); }
__device__ __forceinline__ float temperature_of(const VerifyArgs& a, int b) { return a.temps == nullptr ? 1.f : a.temps[b]; }

// eight logits from v on, rows start wherever V puts them; -inf past the row
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void load_logits(const float* row, int64_t v, int64_t V, float (&o)[OPT_ITEMS]) {
  if (v + OPT_ITEMS <= V) {
    const f32x4_any x = *reinterpret_cast<const f32x4_any*>(row + v), y = *reinterpret_cast<const f32x4_any*>(row + v + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] = x[i];
      o[i + 4] = y[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i) o[i] = v + i < V ? row[v + i] : -INFINITY;
  }
}
__device__ __forceinline__ void load_logits(const uint16_t* row, int64_t v, int64_t V, float (&o)[OPT_ITEMS]) {
  if (v + OPT_ITEMS <= V) {
    const i32x4_any x = *reinterpret_cast<const i32x4_any*>(row + v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float((uint32_t)x[i] << 16);
      o[2 * i + 1] = __uint_as_float((uint32_t)x[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < OPT_ITEMS; ++i) o[i] = v + i < V ? bf16_bits_to_float(row[v + i]) : -INFINITY;
  }
}
__device__ __forceinline__ float logit_at(const float* p) { return *p; }
__device__ __forceinline__ float logit_at(const uint16_t* p) { return bf16_bits_to_float(*p); }

__device__ __forceinline__ float wave_max(float x) {
  x = row_max(x);
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// A chunk of a row: largest logit, sum of exponentials relative to it (NaN where a logit is NaN or infinite); T = 0: where the largest is first.
template <typename T>
__global__ __launch_bounds__(VERIFY_THREADS) void k_verify_rows(VerifyArgs a) {
  constexpr int WAVES = VERIFY_THREADS / 64;
  __shared__ float s_m[WAVES];
  __shared__ double s_s[WAVES];
  __shared__ int s_i[WAVES];
  const int64_t row = blockIdx.x / a.chunks, targets = (int64_t)a.B * (a.K + 1);
  const int chunk = (int)(blockIdx.x - row * a.chunks);
  const bool draft = row >= targets;
  const int64_t at = draft ? row - targets : row;
  const int per = draft ? a.K : a.K + 1, b = (int)(at / per), i = (int)(at - (int64_t)b * per);
  const float temp = temperature_of(a, b);
  if (i >= drafts_of(a, b) + (draft ? 0 : 1) || !(temp >= 0.f && temp < INFINITY) || (draft && temp == 0.f)) return;      // uniform: nobody asks for it
  const T* z = static_cast<const T*>(draft ? a.y : a.z) + at * a.V;
  const int64_t v0 = (int64_t)chunk * VERIFY_CHUNK + threadIdx.x * OPT_ITEMS;
  float x[VERIFY_UNITS][OPT_ITEMS];
#pragma unroll
  for (int q = 0; q < VERIFY_UNITS; ++q) load_logits(z, v0 + q * (VERIFY_THREADS * OPT_ITEMS), a.V, x[q]);
  float m = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int q = 0; q < VERIFY_UNITS; ++q)
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) {
      m = fmaxf(m, x[q][e]);
      bad |= !(x[q][e] < INFINITY);
    }
  m = wave_max(m);
  const int lane = threadIdx.x & 63, wave = wave_id();
  if (lane == 0) s_m[wave] = m;
  bad = __syncthreads_or(bad);
  m = s_m[0];
#pragma unroll
  for (int q = 1; q < WAVES; ++q) m = fmaxf(m, s_m[q]);
  const int64_t out = row * a.chunks + chunk;
  if (temp == 0.f) {                                 // uniform
    int first = 0x7fffffff;
#pragma unroll
    for (int q = VERIFY_UNITS - 1; q >= 0; --q)
#pragma unroll
      for (int e = OPT_ITEMS - 1; e >= 0; --e)
        if (x[q][e] == m) first = (int)(v0 + q * (VERIFY_THREADS * OPT_ITEMS) + e);
    for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o));
    if (lane == 0) s_i[wave] = first;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int q = 1; q < WAVES; ++q) first = min(first, s_i[q]);
      a.part_m[out] = m;
      a.part_s[out] = bad ? __builtin_nan("") : 1.0;
      a.part_i[out] = first;
    }
    return;
  }
  const double inv = 1.0 / (double)temp;
  double s = 0.0;
  if (m > -INFINITY) {                               // uniform
#pragma unroll
    for (int q = 0; q < VERIFY_UNITS; ++q)
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) s += exp_below(((double)x[q][e] - (double)m) * inv);
  }
  s = wave_sum(s);
  if (lane == 0) s_s[wave] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 1; q < WAVES; ++q) s += s_s[q];
    a.part_m[out] = m;
    a.part_s[out] = bad ? __builtin_nan("") : s;
  }
}

// What becomes of a sequence.  The same in every workgroup that asks.
struct Verdict {
  int n, accepted;
  bool none;               // the row that the last token comes from has no distribution
  int first;               // T = 0: the token
  float temp;
  double inv;              // 1 / T
  float mp, mq;            // of that row: largest logits, 1 / sums; mq, iq: only where the draft there was refused
  double ip, iq;
};
constexpr int VERIFY_ROWS = 2 * VERIFY_MOST_DRAFTS + 1;
struct VerdictMemory {
  float m[VERIFY_ROWS];
  double s[VERIFY_ROWS];
  int first[VERIFY_MOST_DRAFTS + 1];
  uint8_t ok[VERIFY_MOST_DRAFTS + 1];
};
// All threads of the workgroup; 16 lanes a row.  Rows 0 .. n: the target's; K + 1 + i: the i-th draft's.
template <typename T>
__device__ __forceinline__ Verdict verdict_of(const VerifyArgs& a, int b, VerdictMemory& s) {
  Verdict d;
  d.n = drafts_of(a, b);
  d.temp = temperature_of(a, b);
  const bool valid = d.temp >= 0.f && d.temp < INFINITY, greedy = d.temp == 0.f;
  d.inv = greedy ? 1.0 : 1.0 / (double)d.temp;
  const int K = a.K, lane16 = threadIdx.x & 15, rows = valid ? (a.y != nullptr && !greedy ? 2 * d.n + 1 : d.n + 1) : 0;
  const int64_t targets = (int64_t)a.B * (K + 1);
  for (int r = threadIdx.x / 16; r < rows; r += blockDim.x / 16) {
    const bool draft = r > d.n;
    const int i = draft ? r - d.n - 1 : r;
    const int64_t at = (draft ? targets + (int64_t)b * K + i : (int64_t)b * (K + 1) + i) * a.chunks;
    float m = -INFINITY;
    for (int c = lane16; c < a.chunks; c += 16) m = fmaxf(m, a.part_m[at + c]);
    m = row_max(m);
    double sum = 0.0;
    int first = 0x7fffffff;
    for (int c = lane16; c < a.chunks; c += 16) {
      const float mc = a.part_m[at + c];
      const double sc = a.part_s[at + c];
      if (!(sc == sc)) sum = sc;                     // a chunk with a NaN may have m = -inf
      else if (mc > -INFINITY) sum += greedy ? 1.0 : sc * exp_below(((double)mc - (double)m) * d.inv);
      if (greedy && mc == m) first = min(first, a.part_i[at + c]);
    }
    for (int o = 8; o > 0; o >>= 1) {
      sum += __shfl_xor(sum, o, 16);
      first = min(first, __shfl_xor(first, o, 16));
    }
    if (lane16 == 0) {
      const int to = draft ? K + 1 + i : i;
      s.m[to] = m;
      s.s[to] = m > -INFINITY ? sum : __builtin_nan("");
      if (!draft) s.first[i] = first;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < d.n; i += blockDim.x) {
    const int x = a.drafts[(int64_t)b * K + i];
    bool ok = false;
    if (valid && x >= 0 && x < a.V) {
      const float given = a.u[(int64_t)b * (K + 1) + i];
      const double u = given < 0.f ? 0.f : given, S = s.s[i];
      if (greedy) {
        ok = S == S && x == s.first[i] && u < 1.0;
      } else if (S == S) {
        const double p = exp_below(((double)logit_at(static_cast<const T*>(a.z) + ((int64_t)b * (K + 1) + i) * a.V + x) - (double)s.m[i]) * d.inv) / S;
        double q = 1.0;
        if (a.y != nullptr)
          q = exp_below(((double)logit_at(static_cast<const T*>(a.y) + ((int64_t)b * K + i) * a.V + x) - (double)s.m[K + 1 + i]) * d.inv) / s.s[K + 1 + i];
        ok = u * q < p;                              // false where q is NaN
      }
    }
    s.ok[i] = ok;
  }
  __syncthreads();
  int k = 0;
  while (k < d.n && s.ok[k]) ++k;
  d.accepted = k;
  d.none = !valid || !(s.s[k] == s.s[k]);
  d.first = 0;
  d.mp = d.mq = 0.f;
  d.ip = d.iq = 0.0;
  if (!d.none) {
    if (greedy) d.first = s.first[k];
    d.mp = s.m[k];
    d.ip = 1.0 / s.s[k];
    if (k < d.n && a.y != nullptr && !greedy) {
      d.none = !(s.s[K + 1 + k] == s.s[K + 1 + k]);
      d.mq = s.m[K + 1 + k];
      d.iq = 1.0 / s.s[K + 1 + k];
    }
  }
  return d;
}
// p and r of eight tokens from v on
template <typename T>
__device__ __forceinline__ void rest_of(const VerifyArgs& a, int b, const Verdict& d, int64_t v, double (&p)[OPT_ITEMS], double (&r)[OPT_ITEMS]) {
  float z[OPT_ITEMS];
  load_logits(static_cast<const T*>(a.z) + ((int64_t)b * (a.K + 1) + d.accepted) * a.V, v, a.V, z);
#pragma unroll
  for (int e = 0; e < OPT_ITEMS; ++e) r[e] = p[e] = exp_below(((double)z[e] - (double)d.mp) * d.inv) * d.ip;
  if (d.accepted == d.n) return;                     // uniform
  if (a.y != nullptr) {
    float y[OPT_ITEMS];
    load_logits(static_cast<const T*>(a.y) + ((int64_t)b * a.K + d.accepted) * a.V, v, a.V, y);
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) {
#pragma clang fp contract(off)
      const double q = exp_below(((double)y[e] - (double)d.mq) * d.inv) * d.iq;      // rounded as p is: equal logits leave nothing
      r[e] = fmax(p[e] - q, 0.0);
    }
  } else {
    const int x = a.drafts[(int64_t)b * a.K + d.accepted];
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) r[e] = v + e == x ? 0.0 : p[e];
  }
}

template <typename T>
__global__ __launch_bounds__(VERIFY_THREADS) void k_verify_sums(VerifyArgs a) {
  constexpr int WAVES = VERIFY_THREADS / 64;
  __shared__ VerdictMemory memory;
  __shared__ double s_r[WAVES], s_p[WAVES];
  const int b = blockIdx.x / a.chunks, chunk = blockIdx.x - b * a.chunks;
  const Verdict d = verdict_of<T>(a, b, memory);
  if (d.none || d.temp == 0.f) return;               // uniform
  double sr = 0.0, sp = 0.0;
#pragma unroll
  for (int q = 0; q < VERIFY_UNITS; ++q) {
    const int64_t v = (int64_t)chunk * VERIFY_CHUNK + (q * VERIFY_THREADS + threadIdx.x) * OPT_ITEMS;
    double p[OPT_ITEMS], r[OPT_ITEMS];
    rest_of<T>(a, b, d, v, p, r);
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) {
      sr += r[e];
      sp += p[e];
    }
  }
  sr = wave_sum(sr);
  sp = wave_sum(sp);
  if ((threadIdx.x & 63) == 0) {
    s_r[threadIdx.x / 64] = sr;
    s_p[threadIdx.x / 64] = sp;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 1; q < WAVES; ++q) {
      sr += s_r[q];
      sp += s_p[q];
    }
    a.sum_r[(int64_t)b * a.chunks + chunk] = sr;
    a.sum_p[(int64_t)b * a.chunks + chunk] = sp;
  }
}

template <typename T>
__global__ __launch_bounds__(PICK_THREADS) void k_verify_pick(VerifyArgs a) {
  constexpr int WAVES = PICK_THREADS / 64;
  __shared__ VerdictMemory memory;
  __shared__ double s_w[WAVES], s_left;
  __shared__ int s_chunk, s_empty, s_last[WAVES], s_token;
  __shared__ float s_logit;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = wave_id();
  const Verdict d = verdict_of<T>(a, b, memory);
  int token = -1;
  if (!d.none && d.temp == 0.f) {
    token = d.first;
  } else if (!d.none) {                              // uniform
    if (threadIdx.x == 0) {
      // the chunk: sums one after the other, as few as V / 8192
      const double* sums = a.sum_r + (int64_t)b * a.chunks;
      double total = 0.0;
      for (int c = 0; c < a.chunks; ++c) total += sums[c];
      s_empty = !(total > 0.0);                      // p = q: any token of p
      if (s_empty) {
        sums = a.sum_p + (int64_t)b * a.chunks;
        total = 0.0;
        for (int c = 0; c < a.chunks; ++c) total += sums[c];
      }
      const double u = fmin(fmax((double)a.u[(int64_t)b * (a.K + 1) + a.K], 0.0), 0x1.fffffep-1), at = u * total;
      double before = 0.0, from = 0.0;
      int chunk = 0;
      for (int c = 0; c < a.chunks; ++c) {           // the first whose end lies behind `at`; past rounding, the last with anything in it
        if (!(sums[c] > 0.0)) continue;
        chunk = c;
        from = before;
        before += sums[c];
        if (before > at) break;
      }
      s_chunk = chunk;
      s_left = at - from;
      s_token = 0x7fffffff;
    }
    __syncthreads();
    const int64_t v = (int64_t)s_chunk * VERIFY_CHUNK + threadIdx.x * OPT_ITEMS;
    double p[OPT_ITEMS], r[OPT_ITEMS], own = 0.0;
    rest_of<T>(a, b, d, v, p, r);
    int last = -1;
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) {
      if (s_empty) r[e] = p[e];
      if (r[e] > 0.0) last = (int)v + e;
      own += r[e];
      r[e] = own;
    }
    // sums before this thread's
    double up = own;
    for (int o = 1; o < 64; o <<= 1) {
      const double t = __shfl_up(up, o);
      if (lane >= o) up += t;
    }
    for (int o = 32; o > 0; o >>= 1) last = max(last, __shfl_xor(last, o));
    if (lane == 63) s_w[wave] = up;
    if (lane == 0) s_last[wave] = last;
    __syncthreads();
    double before = up - own;
    for (int q = 0; q < wave; ++q) before += s_w[q];
    int found = 0x7fffffff;
#pragma unroll
    for (int e = OPT_ITEMS - 1; e >= 0; --e)
      if (before + r[e] > s_left && (e == 0 ? own > 0.0 && r[0] > 0.0 : r[e] > r[e > 0 ? e - 1 : 0])) found = (int)v + e;
    for (int o = 32; o > 0; o >>= 1) found = min(found, __shfl_xor(found, o));
    if (lane == 0 && found != 0x7fffffff) atomicMin(&s_token, found);
    __syncthreads();
    token = s_token;
    if (token == 0x7fffffff) {                       // past the chunk's end by a rounding
      token = -1;
      for (int q = 0; q < WAVES; ++q) token = max(token, s_last[q]);
    }
  }
  if (threadIdx.x == 0) {
    a.accepted[b] = d.accepted;
    s_logit = token >= 0 ? logit_at(static_cast<const T*>(a.z) + ((int64_t)b * (a.K + 1) + d.accepted) * a.V + token) : 0.f;
  }
  __syncthreads();
  for (int i = threadIdx.x; i <= a.K; i += PICK_THREADS) {
    const int64_t at = (int64_t)b * (a.K + 1) + i;
    int t = -1;
    float lp = 0.f;
    if (i <= d.accepted) {
      t = i < d.accepted ? a.drafts[(int64_t)b * a.K + i] : token;
      if (t < 0) {
        lp = __builtin_nanf("");
      } else if (d.temp > 0.f) {
        const float z = i < d.accepted ? logit_at(static_cast<const T*>(a.z) + at * a.V + t) : s_logit;
        lp = (float)(((double)z - (double)memory.m[i]) * d.inv - log(memory.s[i]));
      }
    }
    a.tokens[at] = t;
    a.logp[at] = lp;
  }
}

}  // namespace llamarl
