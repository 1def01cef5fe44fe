// block_kernels.h -- a head in 8 bits, as a generator holds it between two updates of the trainer's.
//
//   k_quantise_rows, k_quantise_tiles   e4m3 and a power of two for each 1 x 128 (activations) or 128 x 128 (weights) block
//   k_block_logits     z = H W^T of two such matrices, stored
//   k_block_partials   the same tiles reduced to (max, sum of exp, target logit) a token: token_logprobs without logits in memory
//   k_few_tokens       both for up to 64 tokens, bound by the bytes of W
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
  int bf16;
  uint8_t* q;
  uint32_t* words;
  int groups;              // of 512 columns
};
// A wavefront takes 512 columns of a row: a block is 16 lanes of eight entries, the wavefront's four exponents are a word.
constexpr int QUANT_THREADS = 256;
__global__ __launch_bounds__(QUANT_THREADS) void k_quantise_rows(QuantiseArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t units = a.rows * a.groups, stride = (int64_t)gridDim.x * (QUANT_THREADS / 64);
  for (int64_t u = (int64_t)blockIdx.x * (QUANT_THREADS / 64) + wave_id(); u < units; u += stride) {
    const int64_t row = u / a.groups;
    const int group = (int)(u - row * a.groups);
    const int64_t col = (int64_t)group * SCALE_GROUP + lane * OPT_ITEMS;
    const int left = (int)max((int64_t)0, min(a.cols - col, (int64_t)OPT_ITEMS));      // eight or none
    float x[OPT_ITEMS];
    load8(a.x, a.bf16 != 0, row * a.cols + col, left, true, x);
    const int e = block_exponent(row_max(magnitude8(x)));
    if (left > 0) *reinterpret_cast<u32x2*>(a.q + row * a.cols + col) = quantise8(x, e);
    const uint32_t b = (uint32_t)(e + 127);
    const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)b, 0) | (uint32_t)__builtin_amdgcn_readlane((int)b, 16) << 8 |
                          (uint32_t)__builtin_amdgcn_readlane((int)b, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)b, 48) << 24;
    if (lane == 0) a.words[(int64_t)group * a.rows + row] = word;
  }
}
// A workgroup takes one 128 x 128 block: 16 rows at a time, kept in registers until the block's maximum is known.
__global__ __launch_bounds__(QUANT_THREADS) void k_quantise_tiles(QuantiseArgs a) {
  constexpr int PASSES = SCALE_BLOCK / 16;
  const int64_t tile_rows = (a.rows + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const int blocks = a.groups * 4;
  const int64_t tr = blockIdx.x / blocks;
  const int cb = (int)(blockIdx.x - tr * blocks);
  const int64_t row0 = tr * SCALE_BLOCK + threadIdx.x / 16, col = (int64_t)cb * SCALE_BLOCK + (threadIdx.x & 15) * OPT_ITEMS;
  float x[PASSES][OPT_ITEMS], top = 0.f;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const bool there = row0 + 16 * p < a.rows && col < a.cols;
    load8(a.x, a.bf16 != 0, (row0 + 16 * p) * a.cols + col, there ? OPT_ITEMS : 0, true, x[p]);
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) top = fmaxf(top, magnitude8(x[p]));
  top = row_max(top);
  __shared__ float s_top[QUANT_THREADS / 16];
  if ((threadIdx.x & 15) == 0) s_top[threadIdx.x / 16] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QUANT_THREADS / 16; ++i) top = fmaxf(top, s_top[i]);
  const int e = block_exponent(top);
#pragma unroll
  for (int p = 0; p < PASSES; ++p)
    if (row0 + 16 * p < a.rows && col < a.cols) *reinterpret_cast<u32x2*>(a.q + (row0 + 16 * p) * a.cols + col) = quantise8(x[p], e);
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
  int tiles_v, tiles_t;
  uint16_t* z;             // bf16 [N][V]
};
// A tile's accumulators to z (its first logit): four neighbouring logits of a token a store.
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));      // rows of z start wherever V puts them
template <typename S>
__device__ __forceinline__ void store_tile(uint16_t* z, int64_t V, const f32x4_t (&acc)[S::MB][S::NB], const LanePos<S>& lp, int rowsV, int rowsT) {
#pragma unroll
  for (int j = 0; j < S::NB; ++j) {
    if (lp.col(j) >= rowsT) continue;
    uint16_t* at = z + lp.col(j) * V + lp.row(0, 0);
#pragma unroll
    for (int i = 0; i < S::MB; ++i) {
      uint16_t b[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) b[r] = float_to_bf16_bits(acc[i][j][r]);
      if (lp.row(i, 3) < rowsV) {
        *reinterpret_cast<u32x2_any*>(at + 16 * i) = u32x2_any{(uint32_t)b[0] | (uint32_t)b[1] << 16, (uint32_t)b[2] | (uint32_t)b[3] << 16};
      } else {
#pragma unroll
        for (int r = 0; r < 3; ++r)
          if (lp.row(i, r) < rowsV) at[16 * i + r] = b[r];
      }
    }
  }
}
template <typename G>
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
    int grow[decltype(g.lb)::ITERS];
#pragma unroll
    for (int it = 0; it < decltype(g.lb)::ITERS; ++it)
      grow[it] = min(t0 + decltype(g.lb)::template lane_tile_row<false>(it, wave, lane, S::NB), last_row);
    g.template setup_gathered<false>(a.x.W + (int64_t)t.tv * S::BM * a.d, a.d, (int)min((int64_t)S::BM, a.V - (int64_t)t.tv * S::BM), a.x.H,
                                     a.d, (int)min((int64_t)S::BN, a.N - t0), a.d, grow, a.N,
                                     a.N <= TURN_COLUMNS * S::BN ? t.tv / PATCH_ROWS_LOGITS : 0);
    g.set_scale_rows((int64_t)t.tv * S::BM, min(t0 + wave % (S::BN / 64) * 64 + lane, last_row));
  };
  LogitsTile cur;
  cur.take(sch);
  setup(cur);
#pragma unroll
  for (int q = 0; q < G::FIRST_PARTS; ++q) g.issue_first(smem, q);
  while (true) {
    f32x4_t acc[S::MB][S::NB];
    const int64_t v0 = (int64_t)cur.tv * S::BM, t0 = (int64_t)cur.tt * S::BN;
    const int rowsV = (int)min((int64_t)S::BM, a.V - v0), rowsT = (int)min((int64_t)S::BN, a.N - t0);
    run_tile<G, S::NB>(g, smem, acc, S::wave_col(wave_id()) * S::WAVE_N >= rowsT);
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
#pragma unroll
      for (int q = 0; q < G::FIRST_PARTS; ++q) g.issue_first(smem, q);
    }
    LLAMARL_FENCE();
    store_tile<S>(a.z + t0 * a.V + v0, a.V, acc, lp, rowsV, rowsT);
    if (last) break;
  }
}

// ---- the target's logit ------------------------------------------------------------------------------------------------------------
// The 8-bit matrix pipe drops the low bits of products far below the largest it adds them to: a logit is good to 1.5e-5 of itself, a sum
// of exponentials over a vocabulary to 1e-7.  The one logit that enters a log-probability by itself is formed again from its
// widened entries: a wavefront a token, 2 d bytes.
__device__ __forceinline__ float e4m3_dot(uint32_t x, uint32_t y, float s) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)y, false);
  const auto c = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)y, true);
  return fmaf(c[1], e[1], fmaf(c[0], e[0], fmaf(a[1], b[1], fmaf(a[0], b[0], s))));
}
__device__ __forceinline__ int exponent_of(uint32_t word, int block) { return (int)(word >> 8 * (block & 3) & 0xffu) - 127; }
constexpr int TARGET_THREADS = 256;
__global__ __launch_bounds__(TARGET_THREADS) void k_target_logits(FwdArgs a, BlockHead x) {
  const int64_t p = (int64_t)blockIdx.x * (TARGET_THREADS / 64) + wave_id();
  if (p >= *a.n_act) return;
  const int row = a.rows[p], y = a.targets[row], lane = threadIdx.x & 63;
  const uint8_t *h = x.H + (int64_t)row * a.d, *w = x.W + (int64_t)y * a.d;
  const int64_t w_rows = (a.V + SCALE_BLOCK - 1) / SCALE_BLOCK;
  float z = 0.f;
  for (int k = lane * 16; k < (int)a.d; k += 64 * 16) {
    const i32x4_t u = *reinterpret_cast<const i32x4_t*>(h + k), v = *reinterpret_cast<const i32x4_t*>(w + k);
    const int group = k / SCALE_GROUP, block = k / SCALE_BLOCK;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = e4m3_dot((uint32_t)u[i], (uint32_t)v[i], s);
    z += ldexpf(s, exponent_of(x.h_words[(int64_t)group * a.N + row], block) + exponent_of(x.w_words[(int64_t)group * w_rows + y / SCALE_BLOCK], block));
  }
  z = wave_sum(z);
  if (lane == 0) a.zt[p] = z;
}

// ---- few tokens, and logits in fp32 ---------------------------------------------------------------------------------------------------
// With up to 64 tokens every byte of W is used for a few products only, and the time is W's way from memory: no LDS on it, many
// loads in flight.  A wavefront takes FEW_ROWS rows of W against all tokens, and one of KS interleaved parts of K (groups of 512
// columns: one word of scales); the parts meet in LDS, in order.  The matrix pipe has time to spare, so the entries are widened to
// bf16, exactly, and multiplied there: full fp32 sums (see k_target_logits), the scales on a block's sum.
// Logits in fp32 of more tokens are taken 64 at a time: the workgroups of one part of W follow each other on one XCD, whose L2 keeps it.
struct FewArgs {
  BlockHead x;
  int64_t N, d, V;
  int parts;               // KS: 1, 2, 4 or 8
  int row_blocks, chunks;  // workgroups' parts of W; chunks of FEW_MAX_TOKENS tokens
  void* z;                 // logits: [N][V]
  FwdArgs f;               // log-probs: rows, n_act, targets, n_pad, part_m, part_s, zt;  tile: FEW_ROWS rows of W
};
constexpr int FEW_WAVES = 8, FEW_THREADS = 64 * FEW_WAVES, FEW_MAX_TOKENS = 64;
template <int RB>
constexpr int FEW_PITCH = 16 * RB + 4;               // floats of a token's row in LDS
template <int RB, int NB>
struct FewBlock {                                    // the fragments of a block of 128 columns
  i32x8_t w[RB], h[NB];
};
// eight entries of a fragment as bf16: an operand of the 16x16x32 MFMA
__device__ __forceinline__ bf16x8_t widen(const i32x8_t& f, int quarter) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * quarter], 1.f, false),
                 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * quarter], 1.f, true),
                 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * quarter + 1], 1.f, false),
                 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * quarter + 1], 1.f, true);
  const i32x4_t w = {__builtin_bit_cast(int, a), __builtin_bit_cast(int, b), __builtin_bit_cast(int, c), __builtin_bit_cast(int, d)};
  return __builtin_bit_cast(bf16x8_t, w);
}
// NB: column blocks of 16 tokens.  Out: float or uint16_t (bf16) logits; void: partials.
template <int RB, int NB, typename Out>
__global__ __launch_bounds__(FEW_THREADS, 2) void k_few_tokens(FewArgs a) {
  constexpr bool STORE = !std::is_void<Out>::value;
  constexpr int RV = 16 * RB;
  __shared__ float s_part[FEW_WAVES][16 * FEW_PITCH<RB>];
  const int lane = threadIdx.x & 63, wave = wave_id(), l16 = lane & 15, g = lane >> 4;
  const int local = blockIdx.x >> 3, row_block = local / a.chunks * 8 + (blockIdx.x & 7);
  if (row_block >= a.row_blocks) return;             // uniform
  const int t0 = local % a.chunks * FEW_MAX_TOKENS;
  const int n_act = STORE ? (int)a.N : *a.f.n_act;
  if (n_act == 0) return;                            // uniform
  const int ks = a.parts, groups_of_rows = FEW_WAVES / ks;
  const int kp = wave % ks;
  const int64_t first = (int64_t)row_block * groups_of_rows * RV, row0 = first + (int64_t)(wave / ks) * RV;      // of this wavefront
  const int64_t row0_in = min(row0, (a.V - 1) / RV * RV);            // a wavefront past the last row repeats the last ones
  const int d = (int)a.d, blocks = (d + SCALE_BLOCK - 1) / SCALE_BLOCK, groups = (d + SCALE_GROUP - 1) / SCALE_GROUP;
  const uint8_t* w0 = a.x.W + row0_in * a.d;
  uint32_t woff[RB], hoff[NB];
  int token[NB];
#pragma unroll
  for (int i = 0; i < RB; ++i) woff[i] = (uint32_t)min((int64_t)(16 * i + l16), a.V - 1 - row0_in) * (uint32_t)d + 16u * g;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int at = min(t0 + 16 * j + l16, n_act - 1);
    token[j] = STORE ? at : a.f.rows[at];
    hoff[j] = (uint32_t)token[j] * (uint32_t)d + 16u * g;
  }
  const int64_t w_rows = (a.V + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const uint32_t* w_words = a.x.w_words + row0_in / SCALE_BLOCK;
  f32x4_t acc[RB][NB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  auto chunks = [](const uint8_t* p) {
    const i32x4_t x = *reinterpret_cast<const i32x4_t*>(p), y = *reinterpret_cast<const i32x4_t*>(p + 64);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto part_of = [&](const uint8_t* p, int k) {      // of a last block: chunks past K are zeros
    i32x4_t x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
    if (k + 16 * g < d) x = *reinterpret_cast<const i32x4_t*>(p);
    if (k + 64 + 16 * g < d) y = *reinterpret_cast<const i32x4_t*>(p + 64);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto multiply = [&](const FewBlock<RB, NB>& f, uint32_t ww, const uint32_t (&hw)[NB], int b) {
    f32x4_t sum[RB][NB];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x8_t w[RB];
#pragma unroll
      for (int i = 0; i < RB; ++i) w[i] = widen(f.w[i], q);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const bf16x8_t h = widen(f.h[j], q);
#pragma unroll
        for (int i = 0; i < RB; ++i) {
          if (q == 0) sum[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          mma(w[i], h, sum[i][j]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int e = exponent_of(ww, b) + exponent_of(hw[j], b);
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][j][r] += __builtin_amdgcn_ldexpf(sum[i][j][r], e);
    }
  };
  for (int group = kp; group < groups; group += ks) {
    const uint32_t ww = w_words[(int64_t)group * w_rows];
    uint32_t hw[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) hw[j] = a.x.h_words[(int64_t)group * a.N + token[j]];
    const int k = group * SCALE_GROUP;
    if (k + SCALE_GROUP <= d) {                      // uniform
      FewBlock<RB, NB> f[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int i = 0; i < RB; ++i) f[b].w[i] = chunks(w0 + k + b * SCALE_BLOCK + woff[i]);
#pragma unroll
        for (int j = 0; j < NB; ++j) f[b].h[j] = chunks(a.x.H + k + b * SCALE_BLOCK + hoff[j]);
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) multiply(f[b], ww, hw, b);
    } else {
      for (int b = 0; b < 4 && group * 4 + b < blocks; ++b) {
        FewBlock<RB, NB> f;
        const int kb = k + b * SCALE_BLOCK;
#pragma unroll
        for (int i = 0; i < RB; ++i) f.w[i] = part_of(w0 + kb + woff[i], kb);
#pragma unroll
        for (int j = 0; j < NB; ++j) f.h[j] = part_of(a.x.H + kb + hoff[j], kb);
        multiply(f, ww, hw, b);
      }
    }
  }
  // 16 tokens at a time: every wavefront's part to LDS, then RV lanes a token and group of rows sum them in order
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    if (t0 + 16 * j >= n_act) break;                 // uniform
    if (j > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < RB; ++i)
      *reinterpret_cast<f32x4_t*>(&s_part[wave][l16 * FEW_PITCH<RB> + 16 * i + 4 * g]) = acc[i][j];
    __syncthreads();
    for (int at = threadIdx.x; at < groups_of_rows * 16 * RV; at += FEW_THREADS) {      // whole wavefronts
      const int v = at % RV, n = at / RV % 16, rg = at / (RV * 16);
      float z = 0.f;
      for (int p = 0; p < ks; ++p) z += s_part[rg * ks + p][n * FEW_PITCH<RB> + v];
      const int64_t row = first + (int64_t)rg * RV + v;
      const int pos = t0 + 16 * j + n;
      if constexpr (STORE) {
        if (pos < n_act && row < a.V) {
          if constexpr (sizeof(Out) == 2) static_cast<uint16_t*>(a.z)[pos * a.V + row] = float_to_bf16_bits(z);
          else static_cast<float*>(a.z)[pos * a.V + row] = z;
        }
      } else {
        const bool there = row < a.V;
        float m = there ? z : -INFINITY;
#pragma unroll
        for (int o = RV / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        const float base = m == -INFINITY ? 0.f : m * LOG2E;
        float s = there ? fast_exp2(fmaf(z, LOG2E, -base)) : 0.f;
#pragma unroll
        for (int o = RV / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
        if (pos < n_act && first + (int64_t)rg * RV < a.V) {
          const int64_t tile = (first + (int64_t)rg * RV) / RV;
          if (v == 0) {
            a.f.part_m[tile * a.f.n_pad + pos] = m;
            a.f.part_s[tile * a.f.n_pad + pos] = s;
          }
          if (there && row == a.f.targets[a.f.rows[pos]]) a.f.zt[pos] = z;
        }
      }
    }
  }
}

}  // namespace llamarl
