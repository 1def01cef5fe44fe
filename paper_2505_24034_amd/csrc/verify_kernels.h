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
//   k_verify_pick    accepted drafts; sums of r, one row a sequence, in parts; the workgroup that is done last finds the token
//
// Everything that decides is in 64 bits: a token is one of V borders, and with fp32's 1e-7 in each of 128256 terms every tenth sample would have
// moved by a token.  fp64 runs at fp32's rate here, so a logit costs what its instructions are, whatever their width: see PowersOf.
// 64 sequences with up to five drafts over 128256 bf16 logits: 46 - 48 + 29 - 30 us, half of the first at the rate of vector instructions (memory: 17); one sequence with
// four: 4.8 + 9.7, trips to memory.
#pragma once
#include "norm_kernels.h"

namespace llamarl {

constexpr int VERIFY_THREADS = 256, VERIFY_UNITS = 4, VERIFY_CHUNK = VERIFY_THREADS * VERIFY_UNITS * OPT_ITEMS;      // logits of a workgroup
constexpr int VERIFY_MOST_DRAFTS = 127;              // 2 K + 1 rows of a sequence
constexpr int VERIFY_PART = 64 * OPT_ITEMS;          // ... of a wavefront's unit: what the sums that a token is looked up in are of
// An entry of p is a power, times its row's scale, over a sum of powers times their chunk's two scales: five powers, each within 1.06e-12 of itself (exp2_parts).
// So of equal distributions max(p - q, 0) leaves up to ten times that, 1.06e-11 (logits and the same plus a constant: 2.2e-12 seen), and what it leaves below
// 2^-36 = 1.46e-11 is no distribution.  A draft of q is refused with the probability of that remainder, so p is drawn from instead.
constexpr double REST_LEAST = 0x1p-36;

// 2^f for |f| <= 1/2, within 1.1e-12 of it: interpolated at Chebyshev's nodes.  A token moves with the probability of its border's, 1e-7 over a vocabulary.
// Several at once, operation by operation: a chain of dependent ones takes twice the time of its instructions where a SIMD has one or two wavefronts.
template <int N>
__device__ __forceinline__ void exp2_parts(const double (&f)[N], double (&y)[N]) {
  constexpr double C[] = {0x1.63d1443896e27p-20, 0x1.00dc56f4f275bp-16, 0x1.4308ac7b284d8p-13,
                          0x1.5d874594355b1p-10, 0x1.3b2ab7181fd6bp-7, 0x1.c6b08dd70cedep-5,
                          0x1.ebfbdff823cd1p-3, 0x1.62e42fef84c8bp-1, 0x1.0000000000000p+0};
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] = C[0];
#pragma unroll
  for (int k = 1; k < 9; ++k)
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = fma(y[e], f[e], C[k]);
}
__device__ __forceinline__ double exp2_part(double f) {
  double x[1] = {f}, y[1];
  exp2_parts(x, y);
  return y[0];
}
constexpr double LOG2E_64 = 0x1.71547652b82fep+0;
// 2^y for y <= 0; exactly 0 far below
__device__ __forceinline__ double exp2_below(double y) {
  y = fmax(y, -1200.0);
  const double n = __builtin_rint(y);
  return __builtin_amdgcn_ldexp(exp2_part(y - n), (int)n);
}
// e^(z / T) for the logits z of a row, relative to 2^M, M the integer nearest to (largest logit / T) log2 e: fifteen instructions a logit.
// With c = log2 e / T the sum t = z c + (1.5 2^52 - M) is rounded to an integer whose low word is n = rint(z c) - M; the fraction is z c less that integer,
// in one operation and so without loss however large z c is.  Below `least` (z c < M - 1150, -inf among it) the power is 0 whatever z is.  Where c |m| is
// beyond 2^30 (neighbouring fp32 numbers are 2^6 powers apart there) or T beyond 2^96, where M or `least` leave their types, it is z - m that is taken.
struct PowersOf {
  double c, shift, m;
  float least;
  bool far;                // uniform
  __device__ __forceinline__ PowersOf(float largest, float temp, double inv_t) : c(LOG2E_64 * inv_t), m((double)largest) {
    const double x = m * c;
    far = !(fabs(x) < 0x1p30 && inv_t > 0x1p-96);
    shift = 0x1.8p52 - __builtin_rint(x);
    least = (float)((__builtin_rint(x) - 1150.0) * ((double)temp * 0x1.62e42fefa39efp-1));
  }
  __device__ __forceinline__ void near(const float (&z)[OPT_ITEMS], double (&y)[OPT_ITEMS]) const {
    constexpr int N = 4;
#pragma unroll
    for (int first = 0; first < OPT_ITEMS; first += N) {
      double d[N], t[N], part[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float at;
        asm("v_max_f32 %0, %1, %2" : "=v"(at) : "v"(z[first + e]), "v"(least));      // fmaxf quiets its operands first: one instruction more
        d[e] = (double)at;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) t[e] = fma(d[e], c, shift);
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = fma(d[e], c, -(t[e] - shift));
      exp2_parts(d, part);
#pragma unroll
      for (int e = 0; e < N; ++e) y[first + e] = __builtin_amdgcn_ldexp(part[e], (int)(uint32_t)__builtin_bit_cast(uint64_t, t[e]));
      LLAMARL_FENCE();                               // the next four want the same registers
    }
  }
  __device__ __forceinline__ double any(float z) const { return exp2_below(((double)z - m) * c) / to_largest(); }
  // 2^M over e^(m / T): what a sum of powers is to be multiplied with to be one relative to the largest
  __device__ __forceinline__ double to_largest() const { return far ? 1.0 : exp2_part(-fma(m, c, -(0x1.8p52 - shift))); }
};

struct VerifyPart {        // of a row's chunk
  double sum;              // of e^((z - largest) / T); NaN where a logit is NaN or +inf
  float largest;
  int first;               // T = 0: the first place of the largest
};
struct VerifyArgs {
  const void* z;           // target logits [B][K+1][V]
  const void* y;           // draft logits [B][K][V], or null
  const int32_t* drafts;   // [B][K]
  const int32_t* lens;     // [B] or null: K
  const float* temps;      // [B] or null: 1
  const float* u;          // [B][K+1]
  int64_t V;
  int B, K, chunks;
  VerifyPart* part;        // [rows][chunks], rows: B (K+1) of the target, then B K of the drafts
  float* at;               // [rows] logit of the row's draft
  double* sums;            // [B][chunks][VERIFY_CHUNK / VERIFY_PART] of r
  unsigned int* ticket;    // [B] workgroups of k_verify_pick that have stored theirs (zeroed by k_verify_rows)
  int32_t* tokens;         // [B][K+1]
  int32_t* accepted;       // [B]
  float* logp;             // [B][K+1]
};
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int b) { return a.lens == nullptr ? a.K : min(max(a.lens[b], 0), a.K); }
__device__ __forceinline__ float temperature_of(const VerifyArgs& a, int b) { return a.temps == nullptr ? 1.f : a.temps[b]; }

// Eight neighbouring logits as they lie in memory; rows start wherever V puts them.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
struct Logits8;
template <>
struct Logits8<float> {
  f32x4_t a, b;
  __device__ __forceinline__ void load(const float* p) {
    const f32x4_any x = *reinterpret_cast<const f32x4_any*>(p), y = *reinterpret_cast<const f32x4_any*>(p + 4);
    a = f32x4_t{x[0], x[1], x[2], x[3]};
    b = f32x4_t{y[0], y[1], y[2], y[3]};
  }
  __device__ __forceinline__ void get(float (&o)[OPT_ITEMS]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] = a[i];
      o[i + 4] = b[i];
    }
  }
  __device__ __forceinline__ void leave_out(int first) {      // the first so many are -inf
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = i < first ? -INFINITY : a[i];
      b[i] = i + 4 < first ? -INFINITY : b[i];
    }
  }
};
template <>
struct Logits8<uint16_t> {
  i32x4_t w;
  __device__ __forceinline__ void load(const uint16_t* p) {
    const i32x4_any x = *reinterpret_cast<const i32x4_any*>(p);
    w = i32x4_t{x[0], x[1], x[2], x[3]};
  }
  __device__ __forceinline__ void get(float (&o)[OPT_ITEMS]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float((uint32_t)w[i] << 16);
      o[2 * i + 1] = __uint_as_float((uint32_t)w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void leave_out(int first) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = 2 * i < first ? 0xff80u : (uint32_t)w[i] & 0xffffu, hi = 2 * i + 1 < first ? 0xff800000u : (uint32_t)w[i] & 0xffff0000u;
      w[i] = (int)(lo | hi);
    }
  }
};
__device__ __forceinline__ float logit_at(const float* p) { return *p; }
__device__ __forceinline__ float logit_at(const uint16_t* p) { return bf16_bits_to_float(*p); }
// A lane's eight logits from v on.  Past the row's end it takes the row's last eight, of which those before v count as -inf: one load for all, no lane by itself.
template <typename T>
struct Window {
  Logits8<T> x;
  __device__ __forceinline__ static int64_t start(int64_t v, int64_t V) { return min(v, max(V - OPT_ITEMS, (int64_t)0)); }
  __device__ __forceinline__ void load(const T* row, int64_t v, int64_t V) {
    if (V >= OPT_ITEMS) x.load(row + start(v, V));   // uniform
  }
  // behind the load: those before v
  __device__ __forceinline__ void settle(int64_t v, int64_t V) { x.leave_out((int)min(v - start(v, V), (int64_t)OPT_ITEMS)); }
  // ... and a row of up to seven, which is the first lane's
  __device__ __forceinline__ void get(const T* row, int64_t v, int64_t V, float (&o)[OPT_ITEMS]) {
    if (V < OPT_ITEMS) {                             // uniform
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) o[e] = -INFINITY;
#pragma unroll 1
      for (int at = 0; at < V; ++at) {
        const float z = v == 0 ? logit_at(row + at) : -INFINITY;
#pragma unroll
        for (int e = 0; e < OPT_ITEMS; ++e) o[e] = e == at ? z : o[e];
      }
      return;
    }
    if (__any(v > start(v, V))) settle(v, V);        // wave-uniform
    x.get(o);
  }
};

// The larger of two, NaN where one is.
__device__ __forceinline__ float top_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_top_of(float x) {
  x = top_of(x, __uint_as_float(dpp_move<ROW_ROR(8)>(__float_as_uint(x))));
  x = top_of(x, __uint_as_float(dpp_move<ROW_ROR(4)>(__float_as_uint(x))));
  x = top_of(x, __uint_as_float(dpp_move<ROW_ROR(2)>(__float_as_uint(x))));
  x = top_of(x, __uint_as_float(dpp_move<ROW_ROR(1)>(__float_as_uint(x))));
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = top_of(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return top_of(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// A workgroup takes `each` neighbouring chunks of a row, the next one's logits on their way while it adds up this one's.  (One chunk each: workgroups
// came and went at 200 a microsecond, the half that nobody asks for among them, and a SIMD had three wavefronts of the seven that it holds.  A fixed grid
// that walks over all: which rows are asked for is known on the device only, and some workgroups had twice as many of them as others.)
template <typename T>
constexpr int VERIFY_ROWS_PER_CU = sizeof(T) == 2 ? 4 : 3;      // two chunks' logits in registers: as many as these leave
template <typename T>
__global__ __launch_bounds__(VERIFY_THREADS, VERIFY_ROWS_PER_CU<T>) void k_verify_rows(VerifyArgs a, int each, int eager) {
  constexpr int WAVES = VERIFY_THREADS / 64;
  __shared__ float s_m[2][WAVES];
  __shared__ double s_s[WAVES];
  __shared__ int s_i[WAVES];
  const int lane = threadIdx.x & 63, wave = wave_id(), groups = (a.chunks + each - 1) / each;
  const int row = blockIdx.x / (unsigned)groups, targets = a.B * (a.K + 1), group = blockIdx.x - row * groups;
  const bool draft = row >= targets;
  const int at = draft ? row - targets : row, per = draft ? a.K : a.K + 1, b = at / per, i = at - b * per;
  if (!draft && i == 0 && group == 0 && threadIdx.x == 0) a.ticket[b] = 0;
  const T* row_z = static_cast<const T*>(draft ? a.y : a.z) + (int64_t)at * a.V;
  const int first_chunk = group * each, end = min(first_chunk + each, a.chunks);
  Window<T> raw[VERIFY_UNITS];
  auto place = [&](int64_t v0, int q) { return v0 + (q * VERIFY_THREADS + (int)threadIdx.x) * OPT_ITEMS; };
  auto load_chunk = [&](int64_t v0) {
#pragma unroll
    for (int q = 0; q < VERIFY_UNITS; ++q) raw[q].load(row_z, place(v0, q), a.V);
  };
  if (eager) load_chunk((int64_t)first_chunk * VERIFY_CHUNK);
  const int x = i < a.K ? a.drafts[(int64_t)b * a.K + i] : -1;
  const float temp = temperature_of(a, b);
  if (i >= drafts_of(a, b) + (draft ? 0 : 1) || !(temp >= 0.f && temp < INFINITY) || (draft && temp == 0.f)) return;      // uniform: nobody asks for it
  if (!eager) load_chunk((int64_t)first_chunk * VERIFY_CHUNK);
  if (threadIdx.x == 0 && x >= first_chunk * VERIFY_CHUNK && x < min((int64_t)end * VERIFY_CHUNK, a.V)) a.at[row] = logit_at(row_z + x);
  const double inv = 1.0 / (double)temp;
  if (a.V < OPT_ITEMS) {                             // uniform: no eight logits to load
    if (threadIdx.x != 0) return;
    VerifyPart out = {0.0, -INFINITY, 0x7fffffff};
    for (int v = 0; v < a.V; ++v) out.largest = top_of(out.largest, logit_at(row_z + v));
    for (int v = (int)a.V - 1; v >= 0; --v) {
      const float z = logit_at(row_z + v);
      if (z == out.largest) out.first = v;
      if (out.largest > -INFINITY) out.sum += temp == 0.f ? 1.0 : exp2_below(((double)z - (double)out.largest) * (LOG2E_64 * inv));
    }
    if (!(out.largest < INFINITY)) out.sum = __builtin_nan("");
    a.part[row] = out;
    return;
  }
  // A chunk has one barrier that every wavefront passes, between the maxima's writing and their reading; the second one only chunks with a sum or a first
  // place have (none: nothing but -inf, a NaN, +inf).  So two chunks' maxima lie in turn in s_m: a wavefront writes a buffer again two chunks on, behind the
  // barrier of the chunk between, which the others reach when they have read it.  s_s and s_i are written behind a chunk's first barrier, and so when all
  // have read what the chunks before left there.
  for (int chunk = first_chunk; chunk < end; ++chunk) {
    const int64_t v0 = (int64_t)chunk * VERIFY_CHUNK;
    float(&top)[WAVES] = s_m[chunk & 1];
    Logits8<T> x[VERIFY_UNITS];
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < VERIFY_UNITS; ++q) {
      x[q] = raw[q].x;
      if (v0 + VERIFY_CHUNK > a.V) {                 // uniform
        raw[q].settle(place(v0, q), a.V);
        x[q] = raw[q].x;
      }
      float z[OPT_ITEMS];
      x[q].get(z);
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) m = top_of(m, z[e]);
    }
    if (chunk + 1 < end) load_chunk(v0 + VERIFY_CHUNK);      // uniform
    m = wave_top_of(m);
    if (lane == 0) top[wave] = m;
    __syncthreads();
    m = top[0];
#pragma unroll
    for (int q = 1; q < WAVES; ++q) m = top_of(m, top[q]);
    VerifyPart out = {__builtin_nan(""), m, 0x7fffffff};
    if (m < INFINITY) {                              // uniform; NaN is not
      out.sum = 0.0;
      if (temp == 0.f) {
#pragma unroll
        for (int q = VERIFY_UNITS - 1; q >= 0; --q) {
          float z[OPT_ITEMS];
          x[q].get(z);
#pragma unroll
          for (int e = OPT_ITEMS - 1; e >= 0; --e)
            if (z[e] == m) out.first = (int)Window<T>::start(place(v0, q), a.V) + e;
        }
        for (int o = 32; o > 0; o >>= 1) out.first = min(out.first, __shfl_xor(out.first, o));
        if (lane == 0) s_i[wave] = out.first;
        __syncthreads();
        for (int q = 0; q < WAVES; ++q) out.first = min(out.first, s_i[q]);
        out.sum = 1.0;
      } else if (m > -INFINITY) {
        const PowersOf power(m, temp, inv);
        double s = 0.0;
        if (!power.far) {
#pragma unroll
          for (int q = 0; q < VERIFY_UNITS; ++q) {
            float z[OPT_ITEMS];
            double y[OPT_ITEMS];
            x[q].get(z);
            power.near(z, y);
            s += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
          }
        } else {                                     // rare, and kept short
#pragma unroll 1
          for (int64_t v = v0 + threadIdx.x; v < min(v0 + VERIFY_CHUNK, a.V); v += VERIFY_THREADS) s += power.any(logit_at(row_z + v));
        }
        s = wave_sum(s);
        if (lane == 0) s_s[wave] = s;
        __syncthreads();
        s = s_s[0];
        for (int q = 1; q < WAVES; ++q) s += s_s[q];
        out.sum = s * power.to_largest();
      }
    }
    if (threadIdx.x == 0) a.part[(int64_t)row * a.chunks + chunk] = out;
  }
}

// What becomes of a sequence.  The same in every workgroup that asks.
struct Verdict {
  int n, accepted;
  bool none;               // the row that the last token comes from has no distribution
  int draft;               // of this thread's place, and its logit
  float logit;
  int first;               // T = 0: the token
  float temp;
  double inv;              // 1 / T
  float mp, mq;            // of that row: largest logits, sums; mq, sq: only where the draft there was refused
  double sp, sq;
};
constexpr int VERIFY_ROWS = 2 * VERIFY_MOST_DRAFTS + 1;
struct VerdictMemory {
  float m[VERIFY_ROWS];
  double s[VERIFY_ROWS];
  int first[VERIFY_MOST_DRAFTS + 1];
  uint8_t ok[VERIFY_MOST_DRAFTS + 1];
};
// All threads of the workgroup: 16 lanes a row, then a thread a draft.  Rows 0 .. K: the target's; K + 1 + i: the i-th draft's.  Bound by trips to memory, so
// everything is asked for at once, also of rows that turn out not to count (whatever the scratch holds there).
__device__ __forceinline__ Verdict verdict_of(const VerifyArgs& a, int b, VerdictMemory& s) {
  Verdict d;
  static_assert(VERIFY_MOST_DRAFTS <= VERIFY_THREADS, "a thread each");
  const int K = a.K, lane16 = threadIdx.x & 15, mine = threadIdx.x, rows = a.y != nullptr ? 2 * K + 1 : K + 1;
  const int64_t targets = (int64_t)a.B * (K + 1);
  auto part_of = [&](int r) { return a.part + (r > K ? targets + (int64_t)b * K + r - K - 1 : (int64_t)b * (K + 1) + r) * a.chunks; };
  VerifyPart ahead = {0.0, -INFINITY, 0x7fffffff};   // of the first 16 chunks, which are most often all
  if (mine / 16 < rows && lane16 < a.chunks) ahead = part_of(mine / 16)[lane16];
  int x = -1;
  float u = 0.f, zx = 0.f, yx = 0.f;
  if (mine < K) {
    x = a.drafts[(int64_t)b * K + mine];
    u = a.u[(int64_t)b * (K + 1) + mine];
    zx = a.at[(int64_t)b * (K + 1) + mine];
    if (a.y != nullptr) yx = a.at[targets + (int64_t)b * K + mine];
  }
  d.n = drafts_of(a, b);
  d.temp = temperature_of(a, b);
  const bool valid = d.temp >= 0.f && d.temp < INFINITY, greedy = d.temp == 0.f;
  d.inv = greedy ? 1.0 : 1.0 / (double)d.temp;
  const double c = LOG2E_64 * d.inv;
  for (int r = mine / 16; r < rows; r += VERIFY_THREADS / 16) {
    const VerifyPart* part = part_of(r);
    VerifyPart own = ahead;
    if (r != mine / 16) {
      own = {0.0, -INFINITY, 0x7fffffff};
      if (lane16 < a.chunks) own = part[lane16];
    }
    const bool counts = valid && (r > K ? r - K - 1 < d.n && !greedy : r <= d.n);
    float m = own.largest;
    for (int i = lane16 + 16; i < a.chunks; i += 16) m = top_of(m, part[i].largest);
    m = top_of(m, __uint_as_float(dpp_move<ROW_ROR(8)>(__float_as_uint(m))));
    m = top_of(m, __uint_as_float(dpp_move<ROW_ROR(4)>(__float_as_uint(m))));
    m = top_of(m, __uint_as_float(dpp_move<ROW_ROR(2)>(__float_as_uint(m))));
    m = top_of(m, __uint_as_float(dpp_move<ROW_ROR(1)>(__float_as_uint(m))));
    double sum = 0.0;
    int first = 0x7fffffff;
    auto add = [&](const VerifyPart& p) {
      if (p.largest > -INFINITY) sum += greedy ? 1.0 : p.sum * exp2_below(((double)p.largest - (double)m) * c);
      if (p.largest == m) first = min(first, p.first);
    };
    add(own);
    for (int i = lane16 + 16; i < a.chunks; i += 16) add(part[i]);
    sum += move_words(sum, [](uint32_t w) { return dpp_move<ROW_ROR(8)>(w); });
    sum += move_words(sum, [](uint32_t w) { return dpp_move<ROW_ROR(4)>(w); });
    sum += move_words(sum, [](uint32_t w) { return dpp_move<ROW_ROR(2)>(w); });
    sum += move_words(sum, [](uint32_t w) { return dpp_move<ROW_ROR(1)>(w); });
    first = min(first, (int)dpp_move<ROW_ROR(8)>((uint32_t)first));
    first = min(first, (int)dpp_move<ROW_ROR(4)>((uint32_t)first));
    first = min(first, (int)dpp_move<ROW_ROR(2)>((uint32_t)first));
    first = min(first, (int)dpp_move<ROW_ROR(1)>((uint32_t)first));
    if (lane16 == 0 && counts) {
      s.m[r] = m;
      s.s[r] = m > -INFINITY && m < INFINITY ? sum : __builtin_nan("");
      if (r <= K) s.first[r] = first;
    }
  }
  __syncthreads();
  bool ok = false;
  d.draft = x;
  d.logit = zx;
  if (mine < d.n) {
    if (valid && x >= 0 && x < a.V) {
      const double given = u < 0.f ? 0.f : u, S = s.s[mine];
      if (greedy) {
        ok = S == S && x == s.first[mine] && given < 1.0;
      } else if (S == S) {
        // u q < p with both sums on the other side: no division
        double p = exp2_below(((double)zx - (double)s.m[mine]) * c), q = S;
        if (a.y != nullptr) {
          q *= exp2_below(((double)yx - (double)s.m[K + 1 + mine]) * c);
          p *= s.s[K + 1 + mine];
        }
        ok = given * q < p;                          // false where one is NaN
      }
    }
    s.ok[mine] = ok;
  }
  __syncthreads();
  int k = 0;
  while (k < d.n && s.ok[k]) ++k;
  d.accepted = k;
  d.none = !valid || !(s.s[k] == s.s[k]);
  d.first = 0;
  d.mp = d.mq = 0.f;
  d.sp = d.sq = 1.0;
  if (!d.none) {
    if (greedy) d.first = s.first[k];
    d.mp = s.m[k];
    d.sp = s.s[k];
    if (k < d.n && a.y != nullptr && !greedy) {
      d.none = !(s.s[K + 1 + k] == s.s[K + 1 + k]);
      d.mq = s.m[K + 1 + k];
      d.sq = s.s[K + 1 + k];
    }
  }
  return d;
}
// What the last token of a sequence is drawn from: p - q times both their sums, p times its own.
template <typename T>
struct Rest {
  const T *z, *y;          // rows; y null: none
  int x;                   // the refused draft, where drafts have no distribution; -1
  PowersOf p, q;
  double by_p, by_q, least;
  __device__ __forceinline__ Rest(const VerifyArgs& a, int b, const Verdict& d)
      : z(static_cast<const T*>(a.z) + ((int64_t)b * (a.K + 1) + d.accepted) * a.V), y(nullptr), x(-1), p(d.mp, d.temp, d.inv), q(d.mq, d.temp, d.inv) {
    if (d.accepted < d.n) {                          // uniform
      if (a.y != nullptr) y = static_cast<const T*>(a.y) + ((int64_t)b * a.K + d.accepted) * a.V;
      else x = a.drafts[(int64_t)b * a.K + d.accepted];
    }
    by_p = p.to_largest() * d.sq;
    by_q = q.to_largest() * d.sp;
    least = REST_LEAST * d.sp * d.sq;
  }
  // r of a lane's eight tokens, `first` the first of them; t, s: their logits
  __device__ __forceinline__ void of(const float (&t)[OPT_ITEMS], const float (&s)[OPT_ITEMS], int64_t first, double (&r)[OPT_ITEMS]) const {
#pragma clang fp contract(off)                       // q is rounded as p is: equal logits leave nothing
    double o[OPT_ITEMS];
    if (!(p.far || (y != nullptr && q.far))) {       // uniform
      p.near(t, r);
      if (y != nullptr) q.near(s, o);
    } else {                                         // rare, and kept short
#pragma unroll 1
      for (int at = 0; at < OPT_ITEMS; ++at) {
        float u = 0.f, v = 0.f;
#pragma unroll
        for (int e = 0; e < OPT_ITEMS; ++e) {
          u = e == at ? t[e] : u;
          v = e == at ? s[e] : v;
        }
        const double x0 = p.any(u), x1 = y != nullptr ? q.any(v) : 0.0;
#pragma unroll
        for (int e = 0; e < OPT_ITEMS; ++e) {
          r[e] = e == at ? x0 : r[e];
          o[e] = e == at ? x1 : o[e];
        }
      }
    }
    const int64_t refused = x - first;
#pragma unroll
    for (int e = 0; e < OPT_ITEMS; ++e) {
      r[e] = r[e] * by_p;
      if (y != nullptr) {
        const double less = o[e] * by_q;
        r[e] = r[e] > less ? r[e] - less : 0.0;
      }
      r[e] = refused == e ? 0.0 : r[e];
    }
  }
};

// inclusive sums over the lanes
__device__ __forceinline__ double wave_scan(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll 1
  for (int o = 1; o < 64; o <<= 1) {
    const double t = __shfl_up(x, o);
    if (lane >= o) x += t;
  }
  return x;
}
// First lane whose inclusive sum lies behind `at` and whose own is not 0; past a rounding, the last that is not 0.  -1: none.
__device__ __forceinline__ int lane_behind(double sum, double own, double at) {
  const uint64_t some = __ballot(own > 0.0), behind = __ballot(own > 0.0 && sum > at);
  return behind != 0 ? (int)__builtin_ctzll(behind) : some != 0 ? 63 - (int)__builtin_clzll(some) : -1;
}

// Bound by latency: trips to memory one after the other, and the code itself, which a kernel this short fetches as it goes; so there is one place where
// logits become r, passed for each unit of a workgroup's and once more for the part that the token is in.  A sequence's units are dealt out to as many
// workgroups as run at once (one sequence: 63 of one unit, 16 of four took 4 us more).
template <typename T>
__global__ __launch_bounds__(VERIFY_THREADS, 2) void k_verify_pick(VerifyArgs a, int units, int some) {
  constexpr int WAVES = VERIFY_THREADS / 64, PARTS = VERIFY_CHUNK / VERIFY_PART;
  __shared__ VerdictMemory memory;
  __shared__ int s_token;
  __shared__ float s_logit;
  __shared__ double s_sums[PARTS];
  const int groups = (units + some - 1) / some, b = blockIdx.x / (unsigned)groups, group = blockIdx.x - b * groups, lane = threadIdx.x & 63, wave = wave_id();
  const Verdict d = verdict_of(a, b, memory);
  int token = -1;
  if (d.none || d.temp == 0.f) {                     // uniform
    if (group != 0) return;
    if (!d.none) token = d.first;
  } else {
    Rest<T> rest(a, b, d);
    const int parts = (int)((a.V + VERIFY_PART - 1) / VERIFY_PART), each = (parts + 63) / 64;
    const bool alone = groups == 1 && units <= VERIFY_UNITS;
    double* sums = a.sums + (int64_t)b * a.chunks * PARTS;
    auto sum_at = [&](int i) { return alone ? s_sums[i] : __hip_atomic_load(sums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    const float given = a.u[(int64_t)b * (a.K + 1) + a.K];
    const double u = fmin(fmax((double)given, 0.0), 0x1.fffffep-1);      // 1 and more count as the largest fp32 number below 1
    // unit `at` of the row, 2048 tokens: `some` of them, then (turn) every one, by one workgroup, where p - q leaves nothing and it is p that is drawn from
    int at = group * some, end = min(at + some, units);
    bool turn = false, last = false;
    double left = 0.0;
    int64_t v = ((int64_t)at * VERIFY_THREADS + threadIdx.x) * OPT_ITEMS;
    Window<T> z, y = {};
    z.load(rest.z, v, a.V);
    if (rest.y != nullptr) y.load(rest.y, v, a.V);
#pragma unroll 1
    while (true) {
      const int64_t first = Window<T>::start(v, a.V);
      float z8[OPT_ITEMS], y8[OPT_ITEMS] = {};
      double r[OPT_ITEMS];
      z.get(rest.z, v, a.V, z8);
      if (rest.y != nullptr) y.get(rest.y, v, a.V, y8);
      if (at + 1 < end) {                            // uniform: the next unit's logits, on their way
        v += VERIFY_THREADS * OPT_ITEMS;
        z.load(rest.z, v, a.V);
        if (rest.y != nullptr) y.load(rest.y, v, a.V);
      }
      rest.of(z8, y8, first, r);
      double own = 0.0;
#pragma unroll
      for (int e = 0; e < OPT_ITEMS; ++e) {
        own += r[e];
        r[e] = own;
      }
      if (last) {                                    // the part: its wavefront lane by lane, the lane token by token
        const double up = wave_scan(own);
        const int in = max(lane_behind(up, own, left), 0);
        left -= up - own;                            // of this lane; what counts is lane `in`
        int found = -1, some = 0;
        float logit = 0.f;
#pragma unroll
        for (int e = OPT_ITEMS - 1; e >= 0; --e) {
          const bool more = r[e] > (e > 0 ? r[e > 0 ? e - 1 : 0] : 0.0);
          if (more && some == 0) some = e;
          if (more && r[e] > left) found = e;
        }
        if (found < 0) found = some;                 // past the lane's end by a rounding
#pragma unroll
        for (int e = 0; e < OPT_ITEMS; ++e) logit = e == found ? z8[e] : logit;
        if (lane == in) {
          s_token = (int)first + found;
          s_logit = logit;
        }
        break;
      }
      // published as a loss's partial sums are: device-scope stores, complete when vmcnt is zero, then a ticket
      own = wave_sum(own);
      if (lane == 0 && alone) s_sums[at * WAVES + wave] = own;
      else if (lane == 0) __hip_atomic_store(sums + at * WAVES + wave, own, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (++at < end) continue;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (!turn && groups > 1) {
        if (threadIdx.x == 0) s_token = __hip_atomic_fetch_add(a.ticket + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)groups - 1u;
        __syncthreads();
        if (!s_token) return;                        // uniform
        __syncthreads();
      }
      // every wavefront finds the part, the first goes on: a lane `each` neighbouring parts, then the part
      constexpr int HELD = 4;                        // of a vocabulary of up to 131072 all
      double held[HELD] = {};
      own = 0.0;
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (i < each && lane * each + i < parts) held[i] = sum_at(lane * each + i);
#pragma unroll
      for (int i = 0; i < HELD; ++i) own += held[i];
#pragma unroll 1
      for (int i = HELD; i < each; ++i)
        if (lane * each + i < parts) own += sum_at(lane * each + i);
      const double sum = wave_scan(own), total = __shfl(sum, 63);
      if (!turn && !(total > rest.least)) {          // uniform: the same numbers everywhere
        __syncthreads();
        turn = true;
        rest.y = nullptr;
        rest.x = -1;
        at = 0;
        end = units;
        v = (int64_t)threadIdx.x * OPT_ITEMS;
        z.load(rest.z, v, a.V);
        continue;
      }
      if (wave != 0) break;
      left = u * total;
      const int of = max(lane_behind(sum, own, left), 0);
      left -= __shfl(sum, of) - __shfl(own, of);
      double before = 0.0, from = 0.0;
      int part = of * each;
      auto step = [&](int i, double s) {             // past the one that `left` falls into nothing changes
        if (!(s > 0.0) || before > left) return;
        part = of * each + i;
        from = before;
        before += s;
      };
#pragma unroll
      for (int i = 0; i < HELD; ++i) step(i, __shfl(held[i], of));
#pragma unroll 1
      for (int i = HELD; i < each; ++i) step(i, of * each + i < parts ? sum_at(of * each + i) : 0.0);
      left -= from;
      v = (int64_t)part * VERIFY_PART + lane * OPT_ITEMS;
      z.load(rest.z, v, a.V);
      if (rest.y != nullptr) y.load(rest.y, v, a.V);
      at = end;
      last = true;
    }
    __syncthreads();
    token = s_token;
  }
  const int i = threadIdx.x;
  if (i > a.K) return;
  int t = -1;
  float lp = 0.f;
  if (i <= d.accepted) {
    t = i < d.accepted ? d.draft : token;
    const float z = i < d.accepted ? d.logit : s_logit;
    if (t < 0) lp = __builtin_nanf("");
    else if (d.temp > 0.f) lp = (float)(((double)z - (double)memory.m[i]) * d.inv - log(memory.s[i]));
  }
  if (i == d.accepted) a.accepted[b] = i;
  a.tokens[(int64_t)b * (a.K + 1) + i] = t;
  a.logp[(int64_t)b * (a.K + 1) + i] = lp;
}

}  // namespace llamarl
