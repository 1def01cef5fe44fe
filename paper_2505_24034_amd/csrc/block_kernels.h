// block_kernels.h -- a head in 8 bits, as a generator holds it between two updates of the trainer's.
//
//   k_quantise_rows, k_quantise_tiles   e4m3 and a power of two for each 1 x 128 (activations) or 128 x 128 (weights) block
//   k_block_logits     z = H W^T of two such matrices, stored
//   k_block_partials   the same tiles reduced to (max, sum of exp, target logit) a token: token_logprobs without logits in memory
//   k_few_direct, k_few_tokens   both for up to 16 and 64 tokens and few rows, bound by the bytes of W
//
// A block's scale 2^e is the smallest power of two for which no finite entry exceeds 448 * 2^e, held as the byte e + 127;
// q = x / 2^e is exact before it is rounded to e4m3, and so are the products with the scales.  Entries that are not finite become NaN.
// Scale words: words[column / 512][row (or row / 128)], byte column / 128 % 4; bytes past the last column are 127 (1.0).
#pragma once
#include "gemm_blocks.h"
#include "head_kernels.h"
#include "optim_kernels.h"

namespace llamarl {

// ---- quantisation -------------------------------------------------------------------------------------------------------------
// Bound by memory: 2 (4) bytes in and one out an entry.
// exponent of a block whose largest finite magnitude is top
__device__ __forceinline__ int block_exponent(float top) {
  const int e = __builtin_amdgcn_frexp_expf(top);              // top = frac 2^e, frac in [0.5, 1);  448 = 0.875 * 2^9
  return top == 0.f ? 0 : max(__builtin_amdgcn_frexp_mantf(top) > 0.875f ? e - 8 : e - 9, -127);
}
__device__ __forceinline__ float finite_magnitude(float x) {
  const float m = fabsf(x);
  return m < INFINITY ? m : 0.f;
}
__device__ __forceinline__ float scaled_down(float x, int e) {
  return fabsf(x) < INFINITY ? __builtin_amdgcn_ldexpf(x, -e) : __builtin_nanf("");
}
__device__ __forceinline__ u32x2 quantise8(const float (&x)[OPT_ITEMS], int e) {
  float y[OPT_ITEMS];
#pragma unroll
  for (int i = 0; i < OPT_ITEMS; ++i) y[i] = scaled_down(x[i], e);
  return u32x2{to_e4m3(y[0], y[1], y[2], y[3]), to_e4m3(y[4], y[5], y[6], y[7])};
}
__device__ __forceinline__ float magnitude8(const float (&x)[OPT_ITEMS]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < OPT_ITEMS; ++i) top = fmaxf(top, finite_magnitude(x[i]));
  return top;
}

struct QuantiseArgs {
  const void* x;
  int64_t rows, cols;      // dense; cols a multiple of 16
  uint8_t* q;
  uint32_t* words;
  int groups;              // of 512 columns
};
// the wavefront's four exponents, one of each 16 lanes, as a word
__device__ __forceinline__ uint32_t scale_word(int e) {
  const int b = e + 127;
  return (uint32_t)__builtin_amdgcn_readlane(b, 0) | (uint32_t)__builtin_amdgcn_readlane(b, 16) << 8 |
         (uint32_t)__builtin_amdgcn_readlane(b, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane(b, 48) << 24;
}
// eight entries as they lie in memory
template <typename T>
struct Raw8;
template <>
struct Raw8<uint16_t> {
  i32x4_t w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const i32x4_t*>(p); }
  __device__ __forceinline__ void clear() { w = i32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ void get(float (&o)[OPT_ITEMS]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float((uint32_t)w[i] << 16);
      o[2 * i + 1] = __uint_as_float((uint32_t)w[i] & 0xffff0000u);
    }
  }
};
template <>
struct Raw8<float> {
  f32x4_t a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4_t*>(p);
    b = *reinterpret_cast<const f32x4_t*>(p + 4);
  }
  __device__ __forceinline__ void clear() { a = b = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void get(float (&o)[OPT_ITEMS]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] = a[i];
      o[i + 4] = b[i];
    }
  }
};
// A wavefront takes 512 columns of a row, QUANT_ROWS of those at a time: a block is 16 lanes of eight entries, the wavefront's four
// exponents are a word.
constexpr int QUANT_THREADS = 256, QUANT_ROWS = 4;
template <typename T>
__global__ __launch_bounds__(QUANT_THREADS) void k_quantise_rows(QuantiseArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t units = a.rows * a.groups, first = ((int64_t)blockIdx.x * (QUANT_THREADS / 64) + wave_id()) * QUANT_ROWS;
  Raw8<T> raw[QUANT_ROWS];
  int64_t at[QUANT_ROWS];                            // first entry of the lane; negative: none
#pragma unroll
  for (int i = 0; i < QUANT_ROWS; ++i) {
    const int64_t u = first + i, row = u / a.groups, col = (u - row * a.groups) * SCALE_GROUP + lane * OPT_ITEMS;
    at[i] = u < units && col < a.cols ? row * a.cols + col : -1;
    if (at[i] >= 0) raw[i].load(static_cast<const T*>(a.x) + at[i]);
    else raw[i].clear();
  }
#pragma unroll
  for (int i = 0; i < QUANT_ROWS; ++i) {
    const int64_t u = first + i, row = u / a.groups;
    if (u >= units) break;                           // wave-uniform
    float x[OPT_ITEMS];
    raw[i].get(x);
    const int e = block_exponent(row_max(magnitude8(x)));
    if (at[i] >= 0) *reinterpret_cast<u32x2*>(a.q + at[i]) = quantise8(x, e);
    const uint32_t word = scale_word(e);
    if (lane == 0) a.words[(u - row * a.groups) * a.rows + row] = word;
  }
}
// A workgroup takes one 128 x 128 block: 16 rows at a time, kept in registers, as they came, until the block's maximum is known.
template <typename T>
__global__ __launch_bounds__(QUANT_THREADS) void k_quantise_tiles(QuantiseArgs a) {
  constexpr int PASSES = SCALE_BLOCK / 16;
  const int64_t tile_rows = (a.rows + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const int blocks = a.groups * 4;
  const int64_t tr = blockIdx.x / blocks;
  const int cb = (int)(blockIdx.x - tr * blocks);
  const int64_t row0 = tr * SCALE_BLOCK + threadIdx.x / 16, col = (int64_t)cb * SCALE_BLOCK + (threadIdx.x & 15) * OPT_ITEMS;
  Raw8<T> raw[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (row0 + 16 * p < a.rows && col < a.cols) raw[p].load(static_cast<const T*>(a.x) + (row0 + 16 * p) * a.cols + col);
    else raw[p].clear();
  }
  float top = 0.f;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    float x[OPT_ITEMS];
    raw[p].get(x);
    top = fmaxf(top, magnitude8(x));
  }
  top = row_max(top);
  __shared__ float s_top[QUANT_THREADS / 16];
  if ((threadIdx.x & 15) == 0) s_top[threadIdx.x / 16] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QUANT_THREADS / 16; ++i) top = fmaxf(top, s_top[i]);
  const int e = block_exponent(top);
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    float x[OPT_ITEMS];
    raw[p].get(x);
    if (row0 + 16 * p < a.rows && col < a.cols) *reinterpret_cast<u32x2*>(a.q + (row0 + 16 * p) * a.cols + col) = quantise8(x, e);
  }
  if (threadIdx.x == 0) reinterpret_cast<uint8_t*>(a.words + (int64_t)(cb >> 2) * tile_rows + tr)[cb & 3] = (uint8_t)(e + 127);
}

// ---- logits and log-probabilities, many tokens ----------------------------------------------------------------------------------
struct BlockHead {
  const uint8_t* H;
  const uint8_t* W;
  const uint32_t* h_words;
  const uint32_t* w_words;
};
// The forward's tiles (fwd_tiles) on the 8-bit loop.
template <typename G>
__global__ __launch_bounds__(G::Shape::THREADS, MIN_WAVES<G>) void k_block_partials(FwdArgs a, const uint32_t* h_words, const uint32_t* w_words) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int n_act = *a.n_act;
  TileSchedule<PATCH_ROWS_LOGITS> sch;
  sch.init(a.tiles_v, (n_act + G::width() - 1) / G::width(), blockIdx.x, gridDim.x);
  if (!sch.has_tile()) return;                       // block-uniform
  G g;
  g.set_scales(w_words, a.V, h_words, a.N, a.d);
  fwd_tiles<G, G::NB>(a, g, sch, n_act, smem);
}

struct BlockLogitsArgs {
  BlockHead x;
  int64_t N, d, V;
  int64_t v_first, v_end;  // rows of W of this launch; v_first a multiple of 256
  int tiles_v, tiles_t;
  void* z;                 // [N][V]
};
// A tile's accumulators to z (its first logit), after(j) behind column block j.  Through a corner of LDS that the wavefront has for itself,
// 16 tokens x 128 bytes at a time, so that an instruction writes 128 bytes of a token: straight from the registers 32 of bf16, which took
// (2000, 65066, 528) 185 us instead of 173, (1714, 5653, 448) 28.4 instead of 24.8, and 64 of fp32: (2000, 65066, 528) 310
// instead of 295.
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(2)));      // rows of z start wherever V puts them
// PACK: bf16 by the conversion instruction (the same bits; a NaN's may differ).
template <typename S, typename Out, bool PACK = false>
struct TileStore {
  static constexpr bool BF16_OUT = sizeof(Out) == 2;
  // logits of a lane's store, and of 128 bytes (64 x 64 tiles: 64, all that four of them leave of a CU's LDS)
  static constexpr int PER = 16 / (int)sizeof(Out), MOST = (S::BM == 64 ? 4 : 8) * PER;
  static constexpr int PART = S::WAVE_M < MOST ? S::WAVE_M : MOST, BLOCKS = PART / 16;      // logits of a token, row blocks of a part
  static constexpr int PITCH = PART * (int)sizeof(Out) + 16, LANES = PART / PER;            // bytes of a token's row in LDS; lanes that store it
  static constexpr int EACH = 16 * LANES / 64;                             // stores of a part
  static constexpr int STORES = S::NB * (S::WAVE_M / PART) * EACH;         // of a wavefront of a whole tile, at least
  static constexpr int LDS_BYTES = S::WAVES * 16 * PITCH;                  // of a workgroup, behind the slabs
  template <typename F>
  __device__ __forceinline__ static void run(Out* z, int64_t V, const f32x4_t (&acc)[S::MB][S::NB], const LanePos<S>& lp, int rowsV, int rowsT,
                                             char* lds, F after) {
    char* own = lds + wave_id() * 16 * PITCH;
    const uint64_t p = reinterpret_cast<uint64_t>(z);
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p) |
                                                                             (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)) << 32),
                                                      (short)0, 0x7fffffff, 0x00020000);
    const int l16 = lp.lane & 15, g = lp.lane >> 4, token = lp.lane / LANES, chunk = lp.lane % LANES;
#pragma unroll
    for (int j = 0; j < S::NB; ++j) {
#pragma unroll
      for (int part = 0; part < S::WAVE_M / PART; ++part) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
          const f32x4_t x = acc[part * BLOCKS + i][j];
          char* at = own + l16 * PITCH + (16 * i + 4 * g) * (int)sizeof(Out);
          if constexpr (BF16_OUT && PACK) {
            *reinterpret_cast<u32x2*>(at) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
          } else if constexpr (BF16_OUT) {
            uint16_t b[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) b[r] = float_to_bf16_bits(x[r]);
            *reinterpret_cast<u32x2*>(at) = u32x2{(uint32_t)b[0] | (uint32_t)b[1] << 16, (uint32_t)b[2] | (uint32_t)b[3] << 16};
          } else {
            *reinterpret_cast<f32x4_t*>(at) = x;
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // a wavefront's LDS operations stay in order
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          const int t = e * (64 / LANES) + token, v = lp.wm * S::WAVE_M + part * PART + chunk * PER;
          const i32x4_t w = *reinterpret_cast<const i32x4_t*>(own + t * PITCH + chunk * 16);
          const int col = lp.wn * S::WAVE_N + 16 * j + t;
          if constexpr (BF16_OUT) {
            if (col < rowsT) {
              Out* at = z + (int64_t)col * V + v;
              if (v + PER <= rowsV) {
                *reinterpret_cast<i32x4_any*>(at) = i32x4_any{w[0], w[1], w[2], w[3]};
              } else {
#pragma unroll
                for (int r = 0; r < PER - 1; ++r)
                  if (v + r < rowsV) at[r] = (uint16_t)((uint32_t)w[r / 2] >> 16 * (r % 2));
              }
            }
          } else {                                   // lanes past the matrix out of bounds: one offset is all that the stores keep in registers
            const uint32_t at = col < rowsT ? ((uint32_t)col * (uint32_t)V + (uint32_t)v) * 4u : OOB_OFFSET;
            if (rowsV == S::BM) {                    // block-uniform
              __builtin_amdgcn_raw_buffer_store_b128(w, rs, (int)at, 0, 0);
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r) __builtin_amdgcn_raw_buffer_store_b32((uint32_t)w[r], rs, (int)(v + r < rowsV ? at : OOB_OFFSET), 4 * r, 0);
            }
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      LLAMARL_FENCE();
      after(j);
      LLAMARL_FENCE();
    }
  }
};
template <typename G, typename Out>
__global__ __launch_bounds__(G::Shape::THREADS, MIN_WAVES<G>) void k_block_logits(BlockLogitsArgs a) {
  typedef typename G::Shape S;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  TileSchedule<PATCH_ROWS_LOGITS> sch;
  sch.init(a.tiles_v, a.tiles_t, blockIdx.x, gridDim.x);
  if (!sch.has_tile()) return;                       // block-uniform
  G g;
  g.set_scales(a.x.w_words, a.V, a.x.h_words, a.N, a.d);
  const int last_row = (int)a.N - 1;
  auto setup = [&](const LogitsTile& t) {
    const int lane = threadIdx.x & 63, wave = wave_id(), t0 = t.tt * S::BN;
    const int64_t v0 = a.v_first + (int64_t)t.tv * S::BM;
    int grow[decltype(g.lb)::ITERS];
#pragma unroll
    for (int it = 0; it < decltype(g.lb)::ITERS; ++it)
      grow[it] = min(t0 + decltype(g.lb)::template lane_tile_row<false>(it, wave, lane, S::NB), last_row);
    g.template setup_gathered<false>(a.x.W + v0 * a.d, a.d, (int)min((int64_t)S::BM, a.v_end - v0), a.x.H,
                                     a.d, (int)min((int64_t)S::BN, a.N - t0), a.d, grow, a.N,
                                     a.N <= TURN_COLUMNS * S::BN ? t.tv / PATCH_ROWS_LOGITS : 0);
    g.set_scale_rows(v0, min(t0 + wave % (S::BN / 64) * 64 + lane, last_row));
  };
  LogitsTile cur;
  cur.take(sch);
  setup(cur);
#pragma unroll
  for (int q = 0; q < G::FIRST_PARTS; ++q) g.issue_first(smem, q);
  bool counted = false;
  while (true) {
    f32x4_t acc[S::MB][S::NB];
    const int64_t v0 = a.v_first + (int64_t)cur.tv * S::BM, t0 = (int64_t)cur.tt * S::BN;
    const int rowsV = (int)min((int64_t)S::BM, a.v_end - v0), rowsT = (int)min((int64_t)S::BN, a.N - t0);
    if (S::wave_col(wave_id()) * S::WAVE_N >= rowsT) {      // wave-uniform
      clear(acc);
      g.run_idle(smem);
    } else {
      g.template run<TileStore<S, Out>::STORES>(smem, acc, counted);
    }
    counted = rowsV == S::BM && rowsT == S::BN;      // every lane stores
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                    // as in fwd_tiles
    const LanePos<S> lp(tid);
    wait_vmcnt0();                                   // requests past K must not land in what is fetched next
    __syncthreads();                                 // every wave is done reading the slabs
    LLAMARL_FENCE();
    const bool last = !sch.has_tile();
    if (!last) {
      cur.take(sch);
      setup(cur);
      g.issue_first(smem, 0);
      g.issue_first(smem, 1);
    }
    LLAMARL_FENCE();
    TileStore<S, Out>::run(static_cast<Out*>(a.z) + t0 * a.V + v0, a.V, acc, lp, rowsV, rowsT, smem + G::LDS_BYTES, [&](int j) {
      if (!last && j < 2) g.issue_first(smem, 2 + j);
    });
    if (last) break;
  }
}

// ---- the target's logit ------------------------------------------------------------------------------------------------------------
// The 8-bit matrix pipe adds eight products at a time, each cut, towards zero, at 2^-13 of the largest of them (measured: beside 448 * 448, terms
// below 8 vanish and 12 counts as 8, for seven of the 127 others): seven lose less than that each, so a logit is off by less than 2^-10 of the sum of
// its terms' magnitudes, and by 1.5e-5 of the root of their sum of squares where their signs are random.  Over a flat distribution that averages out
// of the sum of exponentials (1e-7); where one token has nearly all of it, it does not.  The target's logit, which enters a log-probability by
// itself, is formed again from its widened entries, a wavefront a token, 2 d bytes, and so is its term of the sum (k_merge_logp).
__device__ __forceinline__ float e4m3_dot(uint32_t x, uint32_t y, float s) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)y, false);
  const auto c = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)y, true);
  return fmaf(c[1], e[1], fmaf(c[0], e[0], fmaf(a[1], b[1], fmaf(a[0], b[0], s))));
}
__device__ __forceinline__ int exponent_of(uint32_t word, int block) { return (int)(word >> 8 * (block & 3) & 0xffu) - 127; }
struct BlockTarget {       // for k_merge_logp
  static constexpr bool FORMED = true;
  BlockHead x;
  int64_t N, V;
  int d;
  // of token `row` and vocabulary row y, in every lane of a wavefront
  __device__ __forceinline__ float logit(int row, int y) const {
    const int lane = threadIdx.x & 63;
    const uint8_t *h = x.H + (int64_t)row * d, *w = x.W + (int64_t)y * d;
    const int64_t w_rows = (V + SCALE_BLOCK - 1) / SCALE_BLOCK;
    float z = 0.f;
    for (int k = lane * 16; k < d; k += 64 * 16) {
      const i32x4_t u = *reinterpret_cast<const i32x4_t*>(h + k), v = *reinterpret_cast<const i32x4_t*>(w + k);
      const int group = k / SCALE_GROUP, block = k / SCALE_BLOCK;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) s = e4m3_dot((uint32_t)u[i], (uint32_t)v[i], s);
      z += ldexpf(s, exponent_of(x.h_words[(int64_t)group * N + row], block) + exponent_of(x.w_words[(int64_t)group * w_rows + y / SCALE_BLOCK], block));
    }
    return wave_sum(z);
  }
};

// ---- few tokens ---------------------------------------------------------------------------------------------------------------------
// Every byte of W is used for a few products only, and the time is W's way from memory: W goes from there to the registers of the
// one wavefront that multiplies it.  The matrix pipe has time to spare, so the entries are widened to bf16, exactly, and multiplied
// there: full fp32 sums (see BlockTarget), the scales on a block's sum.
struct FewArgs {
  BlockHead x;
  int64_t N, d, V;
  int parts;               // k_few_direct: wavefronts that share rows of W, each with its groups of K
  void* z;                 // logits: [N][V]
  FwdArgs f;               // log-probs: rows, n_act, targets, n_pad, part_m, part_s, zt;  tile: the rows of a workgroup
};
constexpr int FEW_WAVES = DIRECT_WAVES, FEW_THREADS = 64 * FEW_WAVES;
// z of up to 64 rows of W (a lane each) and a token: stored, or reduced to the tile's partials
template <typename Out>
__device__ __forceinline__ void few_result(const FewArgs& a, int pos, int64_t first, int rows, int64_t tile, float z) {
  const int lane = threadIdx.x & 63;
  const int64_t v = first + lane;
  const bool there = lane < rows && v < a.V;
  if (first >= a.V) return;                          // wave-uniform
  if constexpr (std::is_void<Out>::value) {
    float m = there ? z : -INFINITY;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float base = m == -INFINITY ? 0.f : m * LOG2E;
    const float s = wave_sum(there ? fast_exp2(fmaf(z, LOG2E, -base)) : 0.f);
    if (lane == 0) {
      a.f.part_m[tile * a.f.n_pad + pos] = m;
      a.f.part_s[tile * a.f.n_pad + pos] = s;
    }
    if (there && v == a.f.targets[a.f.rows[pos]]) a.f.zt[pos] = z;
  } else if (there) {
    if constexpr (sizeof(Out) == 2) static_cast<uint16_t*>(a.z)[pos * a.V + v] = float_to_bf16_bits(z);
    else static_cast<float*>(a.z)[pos * a.V + v] = z;
  }
}
template <typename Out>
__device__ __forceinline__ int few_tokens(const FewArgs& a) {
  if constexpr (std::is_void<Out>::value) return *a.f.n_act;
  else return (int)a.N;
}
template <typename Out>
__device__ __forceinline__ int few_token(const FewArgs& a, int at, int n_act) {      // row of H
  const int t = min(at, n_act - 1);
  if constexpr (std::is_void<Out>::value) return a.f.rows[t];
  else return t;
}

// Up to 16 tokens.  A wavefront takes 16 rows of W and every parts-th group of 512 columns, all of it from memory to registers.
template <typename Out>
__global__ __launch_bounds__(FEW_THREADS, 4) void k_few_direct(FewArgs a) {
  constexpr int PITCH = 16 + 4;                      // floats of a token's row in LDS
  __shared__ float s_part[FEW_WAVES][DIRECT_TOKENS * PITCH];
  const int lane = threadIdx.x & 63, wave = wave_id(), l16 = lane & 15, g = lane >> 4;
  const int n_act = few_tokens<Out>(a);
  if (n_act == 0) return;                            // uniform
  const int ks = a.parts, kp = wave % ks, rows = FEW_WAVES / ks * 16;
  const int64_t first = (int64_t)blockIdx.x * rows;
  const int64_t row = min(first + wave / ks * 16 + l16, a.V - 1);
  const int d = (int)a.d, groups = (d + SCALE_GROUP - 1) / SCALE_GROUP;
  const int64_t w_rows = (a.V + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const uint32_t* w_words = a.x.w_words + row / SCALE_BLOCK;         // 16 rows share it
  const int token = few_token<Out>(a, l16, n_act);
  const uint8_t *w = a.x.W + row * a.d, *h = a.x.H + (int64_t)token * a.d;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const i32x4_t (&x)[2], const i32x4_t (&y)[2], uint32_t ww, uint32_t hw, int b) {
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      mma(widen(x[c][0], x[c][1]), widen(y[c][0], y[c][1]), sum);
      mma(widen(x[c][2], x[c][3]), widen(y[c][2], y[c][3]), sum);
    }
    const float s = scale_product(ww >> 8 * b, hw >> 8 * b);
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] = fmaf(sum[r], s, acc[r]);
  };
  for (int group = kp; group < groups; group += ks) {
    const uint32_t ww = w_words[(int64_t)group * w_rows], hw = a.x.h_words[(int64_t)group * a.N + token];
    const int k = group * SCALE_GROUP + g * 16;
    if ((group + 1) * SCALE_GROUP <= d) {            // uniform
      i32x4_t x[4][2], y[4][2];
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          x[b][c] = *reinterpret_cast<const i32x4_t*>(w + k + b * SCALE_BLOCK + c * 64);
          y[b][c] = *reinterpret_cast<const i32x4_t*>(h + k + b * SCALE_BLOCK + c * 64);
        }
#pragma unroll
      for (int b = 0; b < 4; ++b) multiply(x[b], y[b], ww, hw, b);
    } else {
      for (int b = 0; b < 4 && group * SCALE_GROUP + b * SCALE_BLOCK < d; ++b) {
        i32x4_t x[2], y[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int at = k + b * SCALE_BLOCK + c * 64, in = min(at, d - 16);
          x[c] = *reinterpret_cast<const i32x4_t*>(w + in);
          y[c] = *reinterpret_cast<const i32x4_t*>(h + in);
          if (at >= d) x[c] = y[c] = i32x4_t{0, 0, 0, 0};            // past K
        }
        multiply(x, y, ww, hw, b);
      }
    }
  }
  *reinterpret_cast<f32x4_t*>(&s_part[wave][l16 * PITCH + 4 * g]) = acc;
  __syncthreads();
  // a wavefront sums 64 rows of a token at a time, in the order of their parts
  const int per_token = (rows + 63) / 64;            // 1 or 2; rows are 16, 32, 64 or 128
  for (int at = wave; at < DIRECT_TOKENS * per_token; at += FEW_WAVES) {
    const int pos = at / per_token, sub = at - pos * per_token;
    if (pos >= n_act) break;                         // wave-uniform
    const int v = sub * 64 + lane;
    float z = 0.f;
    if (v < rows)
      for (int p = 0; p < ks; ++p) z += s_part[(v >> 4) * ks + p][pos * PITCH + (v & 15)];
    few_result<Out>(a, pos, first + sub * 64, min(rows, 64), (int64_t)blockIdx.x * per_token + sub, z);
  }
}

// Up to 64 tokens.  A workgroup takes 64 rows of W: a wavefront 16 rows and one half of the groups; the halves meet in LDS at the end, in order.  The
// tokens' part of a group is brought to LDS once for the four wavefronts of a half: read by each of them from L2 it was more traffic than W's (48
// tokens of a 128256 x 4096 head, which takes tiles by now: 217 - 250 us, 134 here).  W's registers are loaded again, for the next group, as soon as
// a block is multiplied.  Workgroups start at groups of their own: see SlabOrder.
constexpr int FEW_PITCH = FEW_ROWS + 4;              // floats of a token's row in LDS
template <int NB>
constexpr int FEW_SLAB = NB * 16 * SLAB_ROW_BYTES;   // a block of 128 columns of the tokens
template <int NB>
constexpr int FEW_LDS = 2 * 2 * 4 * FEW_SLAB<NB>;
// NB: column blocks of 16 tokens.  Out: float or uint16_t (bf16) logits; void: partials.
template <int NB, typename Out>
__global__ __launch_bounds__(FEW_THREADS, NB == 1 ? 4 : 2) void k_few_tokens(FewArgs a) {
  constexpr int ITEMS = 2 * NB;                      // 16-byte chunks of the tokens' part of a group that a thread brings
  extern __shared__ __attribute__((aligned(1024))) char smem[];      // [half][buffer][block][token][128 bytes, swizzled]
  const int lane = threadIdx.x & 63, wave = wave_id(), l16 = lane & 15, g = lane >> 4;
  const int n_act = few_tokens<Out>(a);
  if (n_act == 0) return;                            // uniform
  const int half = wave >> 2;
  const int64_t first = (int64_t)blockIdx.x * FEW_ROWS;
  const int64_t row = min(first + (wave & 3) * 16 + l16, a.V - 1);   // of this lane; past the last row the last again
  const int d = (int)a.d, groups = (d + SCALE_GROUP - 1) / SCALE_GROUP, turns = (groups + 1) / 2;
  const uint8_t* w = a.x.W + row * a.d;
  const int64_t w_rows = (a.V + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const uint32_t* w_words = a.x.w_words + first / SCALE_BLOCK;
  int token[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) token[j] = few_token<Out>(a, 16 * j + l16, n_act);
  const int in_half = threadIdx.x & 255, h_chunk = in_half % 32 * 16;
  uint32_t h_from[ITEMS];                            // chunk in_half % 32 of token 8 it + in_half / 32
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) h_from[it] = (uint32_t)few_token<Out>(a, 8 * it + in_half / 32, n_act) * (uint32_t)d;
  const int start = (int)(blockIdx.x % (unsigned)turns);
  auto group_of = [&](int turn) {                    // may be one past the last in the second half
    const int t = turn + start;
    return 2 * (t >= turns ? t - turns : t) + half;
  };
  i32x4_t x[4][2], y[ITEMS];
  uint32_t ww, hw[NB], ww_next = 0, hw_next[NB];
  // past K: from a place that exists; made zeros where they are used, a load is not waited for where it is asked for
  auto w_at = [&](int group, int b, int c) { return group * SCALE_GROUP + b * SCALE_BLOCK + c * 64 + g * 16; };
  auto load_w = [&](int group, int b) {
#pragma unroll
    for (int c = 0; c < 2; ++c) x[b][c] = *reinterpret_cast<const i32x4_t*>(w + min(w_at(group, b, c), d - 16));
  };
  auto load_h = [&](int group) {
    const uint32_t at = (uint32_t)min(group * SCALE_GROUP + h_chunk, d - 16);
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) y[it] = *reinterpret_cast<const i32x4_t*>(a.x.H + h_from[it] + at);
  };
  auto load_words = [&](int group, uint32_t& rw, uint32_t (&cw)[NB]) {
    const int64_t at = min(group, groups - 1);
    rw = w_words[at * w_rows];
#pragma unroll
    for (int j = 0; j < NB; ++j) cw[j] = a.x.h_words[at * a.N + token[j]];
  };
  auto bring = [&](int group, int buffer) {
    const bool past = group * SCALE_GROUP + h_chunk >= d;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      const int t = 8 * it + in_half / 32, b = in_half % 32 / 8, c = in_half % 8;
      if (past) y[it] = i32x4_t{0, 0, 0, 0};
      *reinterpret_cast<i32x4_t*>(smem + ((half * 2 + buffer) * 4 + b) * FEW_SLAB<NB> + t * SLAB_ROW_BYTES + (c ^ swizzle(t)) * 16) = y[it];
    }
  };
  f32x4_t acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  load_h(group_of(0));
  load_words(group_of(0), ww, hw);
#pragma unroll
  for (int b = 0; b < 4; ++b) load_w(group_of(0), b);
  bring(group_of(0), 0);
  __syncthreads();
  for (int turn = 0; turn < turns; ++turn) {
    const bool more = turn + 1 < turns;              // uniform
    const int now = group_of(turn), next = group_of(more ? turn + 1 : turn);
    load_h(next);
    load_words(next, ww_next, hw_next);
    const char* st = smem + (half * 2 + (turn & 1)) * 4 * FEW_SLAB<NB> + l16 * SLAB_ROW_BYTES;
    if ((now + 1) * SCALE_GROUP > d) {               // wave-uniform
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          if (w_at(now, b, c) >= d) x[b][c] = i32x4_t{0, 0, 0, 0};
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      f32x4_t sum[NB];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8_t w0 = widen(x[b][c][0], x[b][c][1]), w1 = widen(x[b][c][2], x[b][c][3]);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const i32x4_t v = *reinterpret_cast<const i32x4_t*>(st + b * FEW_SLAB<NB> + j * BLOCK_BYTES + ((4 * c + g) ^ swizzle(l16)) * 16);
          if (c == 0) sum[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          mma(w0, widen(v[0], v[1]), sum[j]);
          mma(w1, widen(v[2], v[3]), sum[j]);
        }
      }
      load_w(next, b);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const float s = scale_product(ww >> 8 * b, hw[j] >> 8 * b);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[j][r] = fmaf(sum[j][r], s, acc[j][r]);
      }
    }
    ww = ww_next;
#pragma unroll
    for (int j = 0; j < NB; ++j) hw[j] = hw_next[j];
    if (more) bring(next, (turn + 1) & 1);
    __syncthreads();
  }
  // 16 tokens at a time: both halves to LDS, then a wavefront a token sums them over the 64 rows
  float(*part)[16 * FEW_PITCH] = reinterpret_cast<float(*)[16 * FEW_PITCH]>(smem);
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    if (16 * j >= n_act) break;                      // uniform
    if (j > 0) __syncthreads();
    *reinterpret_cast<f32x4_t*>(&part[half][l16 * FEW_PITCH + 16 * (wave & 3) + 4 * g]) = acc[j];
    __syncthreads();
    for (int n = wave; n < 16 && 16 * j + n < n_act; n += FEW_WAVES)         // wave-uniform
      few_result<Out>(a, 16 * j + n, first, FEW_ROWS, blockIdx.x, part[0][n * FEW_PITCH + lane] + part[1][n * FEW_PITCH + lane]);
  }
}

}  // namespace llamarl
