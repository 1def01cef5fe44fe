// row_kernels.h -- a head in 8-bit integers: a scale for each token and each vocabulary row.
//
//   x[r,c] ~ scale[r] q[r,c]      scale[r] = max |x[r,.]| / 127      q = x / scale, to nearest even, in -127 .. 127
//   z[t,v] = (sum_k H[t,k] W[v,k]) W_scale[v] H_scale[t]             the sum in int32, exactly
//
//   k_quantise_int8    a matrix and its scales
//   k_row_logits       z of two such matrices, stored
//   k_row_partials     the same tiles reduced to (max, sum of exp, target logit) a token
//   k_row_direct       both for up to 16 tokens, bound by the bytes of W
//
// The int8 MFMA 16x16x64 takes 16 bytes a lane of either operand, as the bf16 one of 16x16x32 does, and as many cycles: the bf16 loops
// (gemm_nt.h, gemm_small.h) run on bytes as they are, with twice the k a slab.  Their accumulators hold the sums' bits until the epilogue
// makes logits of them.  (9216, 128256, 4096): 2.8 P operations/s sustained, bound by power; (1900, 33001, 2048) 32 us a round of 256 x 256 tiles, 14 of them
// products; few tokens are bound by W's way from memory, 5.2 - 5.9 TB/s: (1, 128256, 4096) 90 us, (48, 16032, 8192) 25.
#pragma once
#include "block_kernels.h"

namespace llamarl {

// a sum times its scales: three roundings in all
__device__ __forceinline__ float scaled_sum(int sum, float w, float h) { return (float)sum * w * h; }

// ---- quantisation -------------------------------------------------------------------------------------------------------------
constexpr uint32_t INT8_TINY = 0x0d800000u;          // 2^-100: a row below it is zeros, its scale 0
constexpr uint32_t FLOAT_INF = 0x7f800000u;
// bits of magnitudes are in the order of the magnitudes, infinities and NaN last
__device__ __forceinline__ uint32_t top_magnitude(const float (&x)[OPT_ITEMS], uint32_t top) {
#pragma unroll
  for (int i = 0; i < OPT_ITEMS; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  return top;
}
__device__ __forceinline__ uint32_t wave_top(uint32_t v) {
  v = max(v, dpp_move<ROW_ROR(8)>(v));
  v = max(v, dpp_move<ROW_ROR(4)>(v));
  v = max(v, dpp_move<ROW_ROR(2)>(v));
  v = max(v, dpp_move<ROW_ROR(1)>(v));
  const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(q[0], q[1]);
}
// NaN for a row with an entry that is not finite: all of its logits are NaN then
__device__ __forceinline__ float int8_scale(uint32_t top) {
  return top >= FLOAT_INF ? __builtin_nanf("") : top < INT8_TINY ? 0.f : __uint_as_float(top) / 127.f;
}
struct Int8Quotient {
  Quotient by;
  bool live;
  __device__ __forceinline__ explicit Int8Quotient(float scale) : by(scale > 0.f ? scale : 1.f), live(scale > 0.f) {}
  __device__ __forceinline__ u32x2 operator()(const float (&x)[OPT_ITEMS]) const {
    u32x2 w = {0u, 0u};
    if (live) {                                      // uniform over the row
#pragma unroll
      for (int i = 0; i < OPT_ITEMS; ++i) {
        const int q = (int)__builtin_rintf(by(x[i]));
        w[i / 4] |= ((uint32_t)q & 0xffu) << 8 * (i % 4);
      }
    }
    return w;
  }
};
struct QuantiseRowsArgs {
  const void* x;
  int64_t rows;
  int cols;                // dense, a multiple of 16
  int8_t* q;
  float* scale;
};
// TH threads a row, UNITS units of eight entries a thread, kept in registers until the row's largest is known; UNITS 0: any number, read twice.
template <typename T, int TH, int UNITS>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void k_quantise_int8(QuantiseRowsArgs a) {
  constexpr int ROWS = (TH < 256 ? 256 : TH) / TH, WAVES = TH / 64, HELD = UNITS > 0 ? UNITS : 1;
  __shared__ uint32_t s_top[WAVES];
  const int tid = threadIdx.x % TH;
  const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? wave_id() : 0);
  if (row >= a.rows) return;                         // as in k_rms_norm
  const T* x = static_cast<const T*>(a.x) + row * a.cols;
  int8_t* q = a.q + row * a.cols;
  Raw8<T> raw[HELD];
  float v[OPT_ITEMS];
  uint32_t top = 0;
  if constexpr (UNITS > 0) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      if (col < a.cols) raw[i].load(x + col);
      else raw[i].clear();
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      raw[i].get(v);
      top = top_magnitude(v, top);
    }
  } else {
    for (int col = tid * OPT_ITEMS; col < a.cols; col += TH * OPT_ITEMS) {
      raw[0].load(x + col);
      raw[0].get(v);
      top = top_magnitude(v, top);
    }
  }
  top = wave_top(top);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) s_top[tid / 64] = top;
    __syncthreads();
    top = s_top[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) top = max(top, s_top[i]);
  }
  const float scale = int8_scale(top);
  const Int8Quotient by(scale);
  if (tid == 0) a.scale[row] = scale;
  if constexpr (UNITS > 0) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int col = (i * TH + tid) * OPT_ITEMS;
      raw[i].get(v);
      if (col < a.cols) *reinterpret_cast<u32x2*>(q + col) = by(v);
    }
  } else {
    for (int col = tid * OPT_ITEMS; col < a.cols; col += TH * OPT_ITEMS) {
      raw[0].load(x + col);
      raw[0].get(v);
      *reinterpret_cast<u32x2*>(q + col) = by(v);
    }
  }
}

// ---- many tokens ----------------------------------------------------------------------------------------------------------------
struct RowHead {
  const int8_t* H;
  const int8_t* W;
  const float* h_scale;
  const float* w_scale;
};
// TileGemmSmall with its slabs taken round a ring (SlabRing), for W that streams from memory: workgroups start at slabs of their own.  From slab 0 / round a
// ring, us, logits of (64, 128256, 4096) 131 / 108, (100, 128256, 4096) 134 / 114, (64, 50000, 8192) 90 / 82, (48, 16032, 8192) on 64 x 64 31.0 / 26.  Eight slabs of
// 64 x 64 resident instead of four: (16, 16032, 8192) 24.8 for 24.2, (33, 128256, 4096) 117 for 117.
template <typename S_, int NSTAGE, int GROUPS_PER_CU_>
struct TileGemmRing : TileGemmSmall<I8, S_, NSTAGE, GROUPS_PER_CU_> {
  typedef TileGemmSmall<I8, S_, NSTAGE, GROUPS_PER_CU_> Base;
  typedef S_ S;
  using Base::BK;
  using Base::K;
  using Base::la;
  using Base::lb;
  SlabRing order;
  __device__ __forceinline__ void issue(char* stage, int kt) const {
    const int lane = threadIdx.x & 63, wave = wave_id(), k0 = kt * BK >= K ? kt * BK : order.template k<BK>(kt, K);      // past K: zeros, no traffic
    la.issue(stage, k0, K, wave, lane);
    lb.issue(stage + S::SLAB_A_BYTES, k0, K, wave, lane);
  }
  __device__ __forceinline__ void issue_first(char* smem, int) const {
#pragma unroll
    for (int i = 0; i < NSTAGE - 1; ++i) issue(smem + i * S::STAGE_BYTES, i);
  }
  template <bool NEAR>
  __device__ __forceinline__ void setup_gathered(const void* A_tile, int64_t lda, int rowsA, const void* B_base, int64_t ldb, int rowsB,
                                                 int64_t K_, const int (&grow)[Base::LoaderB::ITERS], int64_t b_total, int turn) {
    Base::template setup_gathered<NEAR>(A_tile, lda, rowsA, B_base, ldb, rowsB, K_, grow, b_total, turn);
    order.template init<BK>(K, turn);
  }
  __device__ __forceinline__ void run(char* smem, f32x4_t (&acc)[S::MB][S::NB]) {
    const int lane = threadIdx.x & 63, wave = wave_id();
    const int g = lane >> 4, l16 = lane & 15, sw = swizzle(l16);
    int a_addr[2], b_addr[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      a_addr[ks] = (S::wave_row(wave) * S::WAVE_M + l16) * SLAB_ROW_BYTES + (((4 * ks + g) ^ sw) * 16);
      b_addr[ks] = S::SLAB_A_BYTES + (S::wave_col(wave) * S::WAVE_N + l16) * SLAB_ROW_BYTES + (((4 * ks + g) ^ sw) * 16);
    }
    Base::clear(acc);
    const int nk = (K + BK - 1) / BK;
    wait_vmcnt0();
    __syncthreads();
    int st = 0;
    for (int kt = 0; kt < nk; ++kt) {                // see TileGemmSmall::run
      if (kt > 0) {
        wait_vmcnt<Base::LOADS * (NSTAGE - 2)>();
        __syncthreads();
      }
      issue(smem + (st == 0 ? NSTAGE - 1 : st - 1) * S::STAGE_BYTES, kt + NSTAGE - 1);
      Base::slab(smem + st * S::STAGE_BYTES, a_addr, b_addr, acc);
      st = st == NSTAGE - 1 ? 0 : st + 1;
    }
  }
};

// A loop of bf16's on bytes, and the scales of its tiles: a tile's rows' and columns' come to LDS with its first slabs, 64 words a
// wavefront, two tiles' in turn (an epilogue reads them while the next tile's are under way).
template <typename Loop>
struct RowScaled : Loop {
  typedef typename Loop::Shape Shape;
  static constexpr bool ROW_SCALES = true;
  static constexpr int ROW_WORDS = 0;                // HasScales: set_scale_rows is called
  static constexpr int PIECES = Shape::BM / 64, SCALES_BYTES = 2 * PIECES * 256;
  static constexpr int LDS_BYTES = Loop::LDS_BYTES + 2 * SCALES_BYTES;
  static_assert(Shape::BM == Shape::BN && Shape::WAVES >= 2 * PIECES, "a wavefront fetches 64 scales at most");
  const float* w_scale;
  const float* h_scale;
  int64_t V, N;
  char* scales;
  int turn, of_tile;
  __device__ __forceinline__ void set_scales(const RowHead& x, int64_t V_, int64_t N_, char* smem) {
    w_scale = x.w_scale;
    h_scale = x.h_scale;
    V = V_;
    N = N_;
    scales = smem + Loop::LDS_BYTES;
    turn = of_tile = 0;
  }
  // v0: the tile's first row of W; row: row of H of the tile's column wave % PIECES * 64 + lane
  __device__ __forceinline__ void set_scale_rows(int64_t v0, int row) {
    const int wave = wave_id(), lane = threadIdx.x & 63;
    turn ^= 1;
    if (wave >= 2 * PIECES) return;                  // wave-uniform
    const bool rows = wave < PIECES;
    const uint64_t p = reinterpret_cast<uint64_t>(rows ? w_scale : h_scale);
    const i32x4_t rs = {__builtin_amdgcn_readfirstlane((int)(uint32_t)p), __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xffffu)),
                        __builtin_amdgcn_readfirstlane((int)(rows ? V : N) * 4), 0x00020000};
    const uint32_t at = rows ? (uint32_t)min(v0 + wave * 64 + lane, V - 1) : (uint32_t)row;
    lds_dma4(lds_address(scales) + (uint32_t)(turn * SCALES_BYTES + wave * 256), at * 4u, rs);
  }
  __device__ __forceinline__ void run(char* smem, f32x4_t (&acc)[Shape::MB][Shape::NB], bool counted) {
    of_tile = turn;
    if constexpr (Loop::HAS_IDLE) Loop::run(smem, acc, counted);
    else Loop::run(smem, acc);
  }
  __device__ __forceinline__ void run_idle(char* smem) {
    of_tile = turn;
    Loop::run_idle(smem);
  }
  // sums to logits.  To be called behind the barrier that follows run(), before another tile's set_scale_rows but one.
  __device__ __forceinline__ void finish(f32x4_t (&acc)[Shape::MB][Shape::NB], const LanePos<Shape>& lp) const {
    const char* st = scales + of_tile * SCALES_BYTES;
    float h[Shape::NB];
#pragma unroll
    for (int j = 0; j < Shape::NB; ++j) h[j] = *reinterpret_cast<const float*>(st + PIECES * 256 + lp.col(j) * 4);
#pragma unroll
    for (int i = 0; i < Shape::MB; ++i) {
      const f32x4_t w = *reinterpret_cast<const f32x4_t*>(st + lp.row(i, 0) * 4);
#pragma unroll
      for (int j = 0; j < Shape::NB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][j][r] = scaled_sum(__float_as_int(acc[i][j][r]), w[r], h[j]);
    }
  }
};
typedef RowScaled<TileGemm<I8, 11, 2, true, SlabRing>> Rows256;            // counted: the two stores of a token's partials,
typedef RowScaled<TileGemm<I8, 11, 8, true, SlabRing>> Rows256Stored;      // ... the stores of the tile's last two column blocks
typedef RowScaled<TileGemmRing<Shape128, 2, 2>> Rows128;
typedef RowScaled<TileGemmRing<Shape64x64, 4, 2>> Rows64;

template <typename G>
__global__ __launch_bounds__(G::Shape::THREADS, MIN_WAVES<G>) void k_row_partials(FwdArgs a, RowHead x) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int n_act = *a.n_act;
  TileSchedule<PATCH_ROWS_LOGITS> sch;
  sch.init(a.tiles_v, (n_act + G::width() - 1) / G::width(), blockIdx.x, gridDim.x);
  if (!sch.has_tile()) return;                       // block-uniform
  G g;
  g.set_scales(x, a.V, a.N, smem);
  fwd_tiles<G, G::Shape::NB>(a, g, sch, n_act, smem);
}

struct RowLogitsArgs {
  RowHead x;
  int64_t N, d, V;
  int64_t v_first, v_end;  // rows of W of this launch; v_first a multiple of 256
  int tiles_v, tiles_t;
  void* z;                 // [N][V]
};
template <typename G, typename Out>
__global__ __launch_bounds__(G::Shape::THREADS, MIN_WAVES<G>) void k_row_logits(RowLogitsArgs a) {
  typedef typename G::Shape S;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  TileSchedule<PATCH_ROWS_LOGITS> sch;
  sch.init(a.tiles_v, a.tiles_t, blockIdx.x, gridDim.x);
  if (!sch.has_tile()) return;                       // block-uniform
  G g;
  g.set_scales(a.x, a.V, a.N, smem);
  const int last_row = (int)a.N - 1;
  auto setup = [&](const LogitsTile& t) {
    const int lane = threadIdx.x & 63, wave = wave_id(), t0 = t.tt * S::BN;
    const int64_t v0 = a.v_first + (int64_t)t.tv * S::BM;
    int grow[decltype(g.lb)::ITERS];
#pragma unroll
    for (int it = 0; it < decltype(g.lb)::ITERS; ++it)
      grow[it] = min(t0 + decltype(g.lb)::template lane_tile_row<false>(it, wave, lane, S::NB), last_row);
    g.template setup_gathered<false>(a.x.W + v0 * a.d, a.d, (int)min((int64_t)S::BM, a.v_end - v0), a.x.H, a.d,
                                     (int)min((int64_t)S::BN, a.N - t0), a.d, grow, a.N,
                                     a.N <= TURN_COLUMNS * S::BN ? t.tv / PATCH_ROWS_LOGITS : 0);
    g.set_scale_rows(v0, min(t0 + wave % G::PIECES * 64 + lane, last_row));
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
    run_tile<G, S::NB>(g, smem, acc, S::wave_col(wave_id()) * S::WAVE_N >= rowsT, counted);
    counted = rowsV == S::BM && rowsT == S::BN;      // every lane stores
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                    // as in fwd_tiles
    const LanePos<S> lp(tid);
    if constexpr (G::REQUESTS_PAST_K) wait_vmcnt0(); // they must not land in what is fetched next
    __syncthreads();                                 // every wave is done reading the slabs
    LLAMARL_FENCE();
    const bool last = !sch.has_tile();
    if (!last) {
      cur.take(sch);
      setup(cur);
      g.issue_first(smem, 0);
      if constexpr (G::FIRST_PARTS > 1) g.issue_first(smem, 1);
    }
    LLAMARL_FENCE();
    g.finish(acc, lp);
    TileStore<S, Out, true>::run(static_cast<Out*>(a.z) + t0 * a.V + v0, a.V, acc, lp, rowsV, rowsT, smem + G::LDS_BYTES, [&](int j) {
      if (!last && 2 + j < G::FIRST_PARTS) g.issue_first(smem, 2 + j);
    });
    if (last) break;
  }
}

// ---- up to 16 tokens ------------------------------------------------------------------------------------------------------------
// W goes from memory to the registers of the one wavefront that multiplies it.  A wavefront takes 16 rows of W and every parts-th group of
// 512 columns; the tokens' part comes from L2.
struct RowFewArgs {
  FewArgs few;             // N, d, V, parts, z, f (the operands there are not used)
  RowHead x;
};
constexpr int ROW_GROUP = 512;                       // columns: eight MFMAs
template <typename Out>
__global__ __launch_bounds__(FEW_THREADS, 4) void k_row_direct(RowFewArgs a) {
  constexpr int PITCH = 16 + 4;                      // sums of a token's row in LDS
  __shared__ int s_part[FEW_WAVES][DIRECT_TOKENS * PITCH];
  const int lane = threadIdx.x & 63, wave = wave_id(), l16 = lane & 15, g = lane >> 4;
  const int n_act = few_tokens<Out>(a.few);
  if (n_act == 0) return;                            // uniform
  const int ks = a.few.parts, kp = wave % ks, rows = FEW_WAVES / ks * 16;
  const int64_t first = (int64_t)blockIdx.x * rows, V = a.few.V;
  const int64_t row = min(first + wave / ks * 16 + l16, V - 1);
  const int d = (int)a.few.d, groups = (d + ROW_GROUP - 1) / ROW_GROUP;
  const int token = few_token<Out>(a.few, l16, n_act);
  const int8_t *w = a.x.W + row * d, *h = a.x.H + (int64_t)token * d;
  i32x4_t acc = {0, 0, 0, 0};
  for (int group = kp; group < groups; group += ks) {
    const int k = group * ROW_GROUP + g * 16;
    if ((group + 1) * ROW_GROUP <= d) {              // uniform
      i32x4_t x[8], y[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        x[c] = *reinterpret_cast<const i32x4_t*>(w + k + c * 64);
        y[c] = *reinterpret_cast<const i32x4_t*>(h + k + c * 64);
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) mma(x[c], y[c], acc);
    } else {
      for (int c = 0; c < 8 && group * ROW_GROUP + c * 64 < d; ++c) {
        const int at = k + c * 64, in = min(at, d - 16);
        i32x4_t x = *reinterpret_cast<const i32x4_t*>(w + in), y = *reinterpret_cast<const i32x4_t*>(h + in);
        if (at >= d) x = y = i32x4_t{0, 0, 0, 0};    // past K
        mma(x, y, acc);
      }
    }
  }
  *reinterpret_cast<i32x4_t*>(&s_part[wave][l16 * PITCH + 4 * g]) = acc;
  __syncthreads();
  const int per_token = (rows + 63) / 64;            // 1 or 2; rows are 16, 32, 64 or 128
  for (int at = wave; at < DIRECT_TOKENS * per_token; at += FEW_WAVES) {
    const int pos = at / per_token, sub = at - pos * per_token;
    if (pos >= n_act) break;                         // wave-uniform
    const int v = sub * 64 + lane;
    int sum = 0;
    float ws = 0.f;
    if (v < rows) {
      for (int p = 0; p < ks; ++p) sum += s_part[(v >> 4) * ks + p][pos * PITCH + (v & 15)];
      ws = a.x.w_scale[min(first + v, V - 1)];
    }
    const float z = scaled_sum(sum, ws, a.x.h_scale[few_token<Out>(a.few, pos, n_act)]);
    few_result<Out>(a.few, pos, first + sub * 64, min(rows, 64), (int64_t)blockIdx.x * per_token + sub, z);
  }
}

}  // namespace llamarl
