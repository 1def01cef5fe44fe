// gemm_blocks.h -- operands in 8 bits with a scale for each block of 128: the MFMA main loop of the large contractions.
//
// C[m,n] = sum_b 2^(ea[m,b] + eb[n,b]) sum_{k in block b} A[m,k] * B[n,k]      A, B e4m3, K-contiguous; fp32 accumulate
//
// A scale is a power of two (an 8-bit exponent, 2^(byte - 127)), so v_mfma_scale_f32_16x16x128_f8f6f4 applies both inside the matrix
// pipe: a k-step is one block, and no product is rescaled by vector instructions.  A slab of 128 bytes a row, the unit of
// gemm_nt.h's loops, is one block: the same LDS traffic and requests as bf16 at twice the products.
//   - workgroup tile, slab loads, swizzle, gather and bounds as in gemm_nt.h; a lane's 32-byte fragment is its row's 16-byte
//     chunks g and g + 4 (g = lane / 16), in both operands, so the reads are those of two bf16 k-steps.  Which k the pipe takes them for
//     does not matter: the operands agree, and the scale is the block's.
//   - scales come in words of four blocks, group-major: words[k / 512][row].  Every slab brings its words to LDS with its rows: one
//     request for the columns' (lane by lane) and one for the rows' (one word, a wavefront's rows share a block of 128).
#pragma once
#include "gemm_nt.h"

namespace llamarl {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr int SCALE_BLOCK = 128;              // columns (and rows of W) of a scale
constexpr int SCALE_GROUP = 4 * SCALE_BLOCK;  // columns of a word of scales

struct FP8 {
  typedef uint8_t store_t;
  typedef i32x8_t frag_t;
  static constexpr int EPC = 16;
};

__device__ __forceinline__ void mma_blocks(const i32x8_t& a, const i32x8_t& b, f32x4_t& c, int sa, int sb) {
  c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}
__device__ __forceinline__ i32x8_t both_chunks(const char* p0, const char* p1) {
  const i32x4_t x = *reinterpret_cast<const i32x4_t*>(p0), y = *reinterpret_cast<const i32x4_t*>(p1);
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// 64 words of LDS from the buffer `rsrc`, at byte offset voff (lane) + soff
__device__ __forceinline__ void lds_dma_words(uint32_t lds_addr, uint32_t voff, i32x4_t rsrc, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff)
               : "memory", "m0");
}

// Scale words of one operand of a tile.  desc: all words; a group of 512 columns is `pitch` bytes.  Rows and columns past the last
// (whose entries are zeros) get the last one's: every request lies inside.
struct ScaleWords {
  i32x4_t desc;
  uint32_t voff, pitch;
  int last_group;
  __device__ __forceinline__ void set_base(const uint32_t* words, int64_t rows, int64_t K) {
    const uint64_t p = reinterpret_cast<uint64_t>(words);
    pitch = (uint32_t)rows * 4u;
    last_group = (int)((K - 1) / SCALE_GROUP);
    desc = i32x4_t{__builtin_amdgcn_readfirstlane((int)(uint32_t)p), __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xffffu)),
                   __builtin_amdgcn_readfirstlane((int)(pitch * (uint32_t)(last_group + 1))), 0x00020000};
  }
  __device__ __forceinline__ void set_row(int64_t row) { voff = min((uint32_t)row * 4u, pitch - 4u); }
  __device__ __forceinline__ void issue(uint32_t lds_addr, int k0) const {
    lds_dma_words(lds_addr, voff, desc, (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)min(k0 / SCALE_GROUP, last_group) * pitch)));
  }
};

typedef TileShape<2, 2, 2, 2> Shape64x64;     // 4 wavefronts of 32 x 32
// What the loops share: operand streams, scale words, stages.  One workgroup of 256 x 256 tiles a CU, two of 128 x 128, four of 64 x 64.
template <typename S_, typename Order_>
struct BlockStreams {
  typedef FP8 Type;
  typedef S_ Shape;
  typedef i32x8_t frag_t;
  typedef SlabLoader<FP8, Shape::BM, Shape::WAVES, Shape::WAVE_M> LoaderA;
  typedef SlabLoader<FP8, Shape::BN, Shape::WAVES, Shape::WAVE_N> LoaderB;
  static constexpr int MB = Shape::MB, NB = Shape::NB;
  static constexpr bool KMAJOR = false, HAS_IDLE = true, HALVES = false, REQUESTS_PAST_K = true;
  static constexpr int BK = SCALE_BLOCK;
  static constexpr int COL_WORDS = Shape::STAGE_BYTES, ROW_WORDS = COL_WORDS + Shape::BN * 4;      // in a stage
  static constexpr int STAGE = ROW_WORDS + Shape::WAVES * 256;
  static constexpr int LDS_BYTES = 2 * STAGE;
  static constexpr int GROUPS_PER_CU = Shape::BM == 256 ? 1 : Shape::BM == 128 ? 2 : 4;
  static constexpr int FIRST_PARTS = 4;
  static constexpr int SLAB_REQUESTS = LoaderA::ITERS + LoaderB::ITERS + 2;
  static_assert(Shape::WAVE_M <= SCALE_BLOCK && Shape::BN % 64 == 0, "a wavefront's rows share their scales; words of 64 columns a request");
  LoaderA la;
  LoaderB lb;
  ScaleWords wa, wb;
  int K;
  Order_ order;
  __device__ __forceinline__ static constexpr int width() { return Shape::BN; }

  // words of all rows of A's matrix (a word for 128 rows) and of B's (one a row)
  __device__ __forceinline__ void set_scales(const uint32_t* a_words, int64_t a_rows, const uint32_t* b_words, int64_t b_rows, int64_t K_) {
    wa.set_base(a_words, (a_rows + SCALE_BLOCK - 1) / SCALE_BLOCK, K_);
    wb.set_base(b_words, b_rows, K_);
  }
  // a_row: the tile's first row of A's matrix; b_row: row of B's matrix of the tile's column (wave % (BN / 64)) * 64 + lane
  __device__ __forceinline__ void set_scale_rows(int64_t a_row, int b_row) {
    wa.set_row((a_row + Shape::wave_row(wave_id()) * Shape::WAVE_M) / SCALE_BLOCK);
    wb.set_row(b_row);
  }
  template <bool NEAR>
  __device__ __forceinline__ void setup_gathered(const void* A_tile, int64_t lda, int rowsA, const void* B_base, int64_t ldb, int rowsB,
                                                 int64_t K_, const int (&grow)[LoaderB::ITERS], int64_t b_total, int turn) {
    const int lane = threadIdx.x & 63, wave = wave_id();
    K = (int)K_;
    order.template init<BK>(K, turn);
    la.init(A_tile, lda, rowsA, wave, lane);
    lb.template init_gathered<NEAR>(B_base, ldb, b_total, grow, rowsB, wave, lane);
  }
  __device__ __forceinline__ void issue_words(char* st, int k0) const {
    const int wave = wave_id();
    wb.issue(lds_address(st) + COL_WORDS + (uint32_t)(wave % (Shape::BN / 64)) * 256u, k0);      // the second half of the wavefronts: the same again
    wa.issue(lds_address(st) + ROW_WORDS + (uint32_t)wave * 256u, k0);
  }
  __device__ __forceinline__ void issue_slab(char* st, int kt) const {
    const int lane = threadIdx.x & 63, wave = wave_id();
    const int k0 = slab_k(kt);
    la.issue(st, k0, K, wave, lane);
    lb.issue(st + Shape::SLAB_A_BYTES, k0, K, wave, lane);
    issue_words(st, k0);
  }
  // see TileGemm::issue_first
  __device__ __forceinline__ void issue_first(char* smem, int part) const {
    const int lane = threadIdx.x & 63, wave = wave_id();
    char* st = smem + (part >> 1) * STAGE;
    const int k0 = slab_k(part >> 1);
    if ((part & 1) == 0) {
      la.issue(st, k0, K, wave, lane);
    } else {
      lb.issue(st + Shape::SLAB_A_BYTES, k0, K, wave, lane);
      issue_words(st, k0);
    }
  }
  __device__ __forceinline__ int slabs() const { return (K + BK - 1) / BK; }
  // First k of the kt-th slab taken.  Slabs past K are requested like the others (zeros, no traffic), so that the loop needs no end of its own.
  __device__ __forceinline__ int slab_k(int kt) const { return kt * BK >= K ? kt * BK : order.template k<BK>(kt, K); }
  // see TileGemm::run_idle
  __device__ __forceinline__ void run_idle(char* smem) const {
    const int nk = slabs();
    wait_vmcnt0();
    __syncthreads();
    for (int kt = 0; kt < nk - 1; ++kt) {
      wait_vmcnt0();
      __syncthreads();
      issue_slab(smem + (kt & 1) * STAGE, kt + 2);
    }
  }

  struct Addresses {      // of a lane in a stage: the chunks of block 0 of either operand, and its column's word in column block 0
    int a[2], b[2], cw, rw;
  };
  // Of the rows and of each column block; words of four blocks until pick() has shifted the slab's byte to the bottom, where the
  // matrix pipe takes it from.
  struct Scales {
    uint32_t row, col[NB];
  };
  __device__ __forceinline__ static i32x8_t frag_a(const char* st, const Addresses& ad, int ib) {
    return both_chunks(st + ad.a[0] + ib * BLOCK_BYTES, st + ad.a[1] + ib * BLOCK_BYTES);
  }
  __device__ __forceinline__ static i32x8_t frag_b(const char* st, const Addresses& ad, int jb) {
    return both_chunks(st + ad.b[0] + jb * BLOCK_BYTES, st + ad.b[1] + jb * BLOCK_BYTES);
  }
  __device__ __forceinline__ static uint32_t word(const char* p) { return *reinterpret_cast<const uint32_t*>(p); }
  __device__ __forceinline__ static uint32_t pick(uint32_t w, int k0) { return w >> ((k0 / SCALE_BLOCK & 3) * 8); }
  __device__ __forceinline__ static Addresses addresses() {
    const int lane = threadIdx.x & 63, wave = wave_id(), g = lane >> 4, l16 = lane & 15, sw = swizzle(l16);
    Addresses ad;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      ad.a[c] = (Shape::wave_row(wave) * Shape::WAVE_M + l16) * SLAB_ROW_BYTES + (((4 * c + g) ^ sw) * 16);
      ad.b[c] = Shape::SLAB_A_BYTES + (Shape::wave_col(wave) * Shape::WAVE_N + l16) * SLAB_ROW_BYTES + (((4 * c + g) ^ sw) * 16);
    }
    ad.cw = COL_WORDS + (Shape::wave_col(wave) * Shape::WAVE_N + l16) * 4;
    ad.rw = ROW_WORDS + wave * 256 + lane * 4;
    return ad;
  }
};

// On the 8-bit matrix pipe.
template <typename S_, typename Order_>
struct TileGemmBlocks : BlockStreams<S_, Order_> {
  typedef BlockStreams<S_, Order_> Base;
  typedef S_ Shape;
  typedef typename Base::Addresses Addresses;
  typedef typename Base::Scales Scales;
  typedef i32x8_t frag_t;
  using Base::K;
  using Base::MB;
  using Base::NB;
  using Base::la;
  using Base::lb;
  using Base::frag_a;
  using Base::frag_b;
  using Base::issue_words;
  using Base::pick;
  using Base::slab_k;
  using Base::word;

  // Slot of the n-th load of a slab (the words' are the last, together), after TB.  Where no fragment is read, then every other slot: against
  // a load in each slot from TB on, 9216 tokens of a 128256 x 4096 head 3.66 -> 3.56 ms, (2048, 16032, 8192) 210 -> 202 us; two loads a
  // slot 3.71 ms; a barrier two or three slots later 3.61 - 3.66.
  __device__ __forceinline__ static constexpr int load_slot(int n) { return n < 4 ? n : n < 8 ? 2 * n - 4 : 11; }
  // One slab.  MB x 4 slots: pairs of row blocks, eight slots a pair, two a column block, the row operand snaking.  A fragment is
  // eight registers, so four row fragments are held, the pair's and the next's, and four column fragments once:
  //   - a pair's row fragments are read at the start of the pair before, into the registers of the one before that;
  //   - the slab's own reads so end at the start of its last pair but one; there is the barrier (TB), and behind it the slab after next
  //     is requested (load_slot);
  //   - the next slab's column block j is read when the last pair is done with this one's, seven slots ahead of its use, and
  //     its first row pair at the start of the last pair.
  // row_next: the rows' word of the next slab, whose byte is picked when this slab is done.
  template <bool BAR, bool FETCH>
  __device__ __forceinline__ void step(frag_t (&a)[4], frag_t (&b)[NB], Scales& sc, f32x4_t (&acc)[MB][NB], char* cur, const char* nxt,
                                       const Addresses& ad, int k_cur, int k_fetch) const {
    constexpr int PAIRS = MB / 2, LAST = 8 * (PAIRS - 1), TB = LAST - 5;
    constexpr int LA = Base::LoaderA::ITERS, LB = Base::LoaderB::ITERS;
    static_assert(NB == 4 && (MB == 8 || MB == 4) && LA + LB == 8 && TB + 1 + load_slot(8) < 8 * PAIRS, "every load has a slot");
    const int lane = threadIdx.x & 63, wave = wave_id();
    i32x4_t ra, rb;
    if (FETCH) {
      ra = la.rsrc();
      rb = lb.rsrc();
    }
    uint32_t row_next = 0;
    sc.row = pick(sc.row, k_cur);
#pragma unroll
    for (int t = 0; t < MB * NB; ++t) {
      const int p = t >> 3, jb = (t >> 1) & 3, ib = 2 * p + ((t ^ t >> 1) & 1);
      if (BAR && t == TB) {
        wait_vmcnt0();
        __syncthreads();
        LLAMARL_FENCE();
      }
      if (p == 0 && (t & 1) == 0) sc.col[jb] = pick(sc.col[jb], k_cur);
      mma_blocks(a[ib & 3], b[jb], acc[ib][jb], (int)sc.row, (int)sc.col[jb]);
      LLAMARL_FENCE();
      if (t < LAST && (t & 7) < 2) {
        const int next = 2 * (p + 1) + (t & 7);
        a[next & 3] = frag_a(cur, ad, next);
      }
      if (BAR) {
        if (t == LAST || t == LAST + 1) a[t - LAST] = frag_a(nxt, ad, t - LAST);
        if (t == LAST + 2) row_next = word(nxt + ad.rw);
        if (t > LAST && (t & 1) == 1) {
          b[jb] = frag_b(nxt, ad, jb);
          sc.col[jb] = word(nxt + ad.cw + jb * 64);
        }
      }
      LLAMARL_FENCE();
      if (FETCH) {
#pragma unroll
        for (int n = 0; n <= LA + LB; ++n)
          if (t == TB + 1 + load_slot(n)) {
            if (n < LA) la.issue_one(ra, cur, n, k_fetch, K, wave, lane);
            else if (n < LA + LB) lb.issue_one(rb, cur + Shape::SLAB_A_BYTES, n - LA, k_fetch, K, wave, lane);
            else issue_words(cur, k_fetch);
            LLAMARL_FENCE();
          }
      }
    }
    if (BAR) sc.row = row_next;
  }
  // counted (wave-uniform): the requests of the first slab were followed by those of the second and by STORES stores of the
  // previous tile at least: the first slab alone is waited for.
  template <int STORES = 0>
  __device__ __forceinline__ void run(char* smem, f32x4_t (&acc)[MB][NB], bool counted = false) {
    const int nk = this->slabs();
    const Addresses ad = Base::addresses();
    static_assert(STORES + Base::SLAB_REQUESTS < 64, "vmcnt counts to 63");
    if (counted) wait_vmcnt<STORES + Base::SLAB_REQUESTS>();
    else wait_vmcnt0();
    __syncthreads();
    frag_t a[4], b[NB];
    Scales sc;
    sc.row = word(smem + ad.rw);
#pragma unroll
    for (int i = 0; i < 2; ++i) a[i] = frag_a(smem, ad, i);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      b[j] = frag_b(smem, ad, j);
      sc.col[j] = word(smem + ad.cw + j * 64);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    LLAMARL_FENCE();
    char *s = smem, *o = smem + Base::STAGE;
    for (int kt = 0; kt < nk - 1; ++kt) {
      step<true, true>(a, b, sc, acc, s, o, ad, slab_k(kt), slab_k(kt + 2));
      char* x = s;
      s = o;
      o = x;
    }
    step<false, false>(a, b, sc, acc, s, o, ad, slab_k(nk - 1), 0);
  }
};

// eight entries of a fragment as bf16, exactly: an operand of the 16x16x32 MFMA
__device__ __forceinline__ bf16x8_t widen(int lo, int hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, 1.f, true),
                 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, 1.f, true);
  const i32x4_t w = {__builtin_bit_cast(int, a), __builtin_bit_cast(int, b), __builtin_bit_cast(int, c), __builtin_bit_cast(int, d)};
  return __builtin_bit_cast(bf16x8_t, w);
}
// 2^(sum of two scales), the ends of fp32's range for what lies beyond
__device__ __forceinline__ float scale_product(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_ldexpf(1.f, min((int)(a & 0xffu) + (int)(b & 0xffu) - 254, 127));
}

// Loops without an order of their own: a slab's fragments are read and multiplied as the compiler places them.
//   EXACT   fp32 sums (fp32 logits, and everything of up to 64 tokens): fragments are widened to bf16 and multiplied there, a block's sum is scaled
//           into the accumulators.  128 x 128: 128 widenings and 64 fused multiply-adds beside 64 MFMAs of 16 cycles a wavefront and slab; 1000
//           tokens of a 128256 x 4096 head run at 0.98 PFLOP/s.  (The three interleaved by hand, one MFMA and two or three of the others: the same
//           within 3 %.  256 x 128 tiles of four wavefronts of 128 x 64, a quarter less to widen: 0.81, one wavefront a SIMD leaves nothing to run
//           beside a wait.)
//   else    on the 8-bit pipe; 64 x 64 tiles, where few larger ones would leave CUs without work
template <typename S_, typename Order_, bool EXACT>
struct TileGemmBlocksSimple : BlockStreams<S_, Order_> {
  typedef BlockStreams<S_, Order_> Base;
  typedef S_ Shape;
  typedef typename Base::Addresses Addresses;
  using Base::K;
  using Base::MB;
  using Base::NB;
  using Base::slab_k;
  using Base::word;

  __device__ __forceinline__ static void slab(const char* st, const Addresses& ad, f32x4_t (&acc)[MB][NB], int k0) {
    const uint32_t row = Base::pick(word(st + ad.rw), k0);
    uint32_t col[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) col[j] = Base::pick(word(st + ad.cw + j * 64), k0);
    if constexpr (!EXACT) {
      i32x8_t b[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) b[j] = Base::frag_b(st, ad, j);
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const i32x8_t a = Base::frag_a(st, ad, i);
#pragma unroll
        for (int j = 0; j < NB; ++j) mma_blocks(a, b[j], acc[i][j], (int)row, (int)col[j]);
      }
    } else {
      f32x4_t sum[MB][NB];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        i32x4_t x[MB], y[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) y[j] = *reinterpret_cast<const i32x4_t*>(st + ad.b[c] + j * BLOCK_BYTES);
#pragma unroll
        for (int i = 0; i < MB; ++i) x[i] = *reinterpret_cast<const i32x4_t*>(st + ad.a[c] + i * BLOCK_BYTES);
#pragma unroll
        for (int h = 0; h < 2; ++h) {                // 32 of a block's columns: eight entries a lane
          bf16x8_t b[NB];
#pragma unroll
          for (int j = 0; j < NB; ++j) b[j] = widen(y[j][2 * h], y[j][2 * h + 1]);
#pragma unroll
          for (int i = 0; i < MB; ++i) {
            const bf16x8_t a = widen(x[i][2 * h], x[i][2 * h + 1]);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
              if (c == 0 && h == 0) sum[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
              mma(a, b[j], sum[i][j]);
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const float s = scale_product(row, col[j]);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(sum[i][j][r], s, acc[i][j][r]);
      }
    }
  }
  template <int STORES = 0>
  __device__ __forceinline__ void run(char* smem, f32x4_t (&acc)[MB][NB], bool counted = false) {      // see TileGemmBlocks::run
    const int nk = this->slabs();
    const Addresses ad = Base::addresses();
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    static_assert(STORES + Base::SLAB_REQUESTS < 64, "vmcnt counts to 63");
    if (counted) wait_vmcnt<STORES + Base::SLAB_REQUESTS>();
    else wait_vmcnt0();
    __syncthreads();
    char *s = smem, *o = smem + Base::STAGE;
    for (int kt = 0; kt < nk - 1; ++kt) {
      slab(s, ad, acc, slab_k(kt));
      wait_vmcnt0();                                 // the next slab, asked for one slab ago
      __syncthreads();
      this->issue_slab(s, kt + 2);
      char* x = s;
      s = o;
      o = x;
    }
    slab(s, ad, acc, slab_k(nk - 1));
  }
};

}  // namespace llamarl
