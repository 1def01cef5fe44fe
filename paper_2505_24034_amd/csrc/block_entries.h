// block_entries.h -- host side of llamarl_quantise_blocks, llamarl_logits_blocks and llamarl_token_logprobs_blocks.  Part of
// llamarl.hip.
#pragma once

namespace {

typedef TileGemmBlocks<Shape256, SlabRing> Blocks256;
typedef TileGemmBlocks<Shape128, SlabRing> Blocks128;
typedef TileGemmBlocksSimple<Shape64x64, SlabRing, false> Blocks64;
typedef TileGemmBlocksSimple<Shape128, SlabRing, true> Exact128;
typedef TileGemmBlocksSimple<Shape64x64, SlabRing, true> Exact64;

// As FwdWs; the planes: block_partials.
struct BlockWs {
  int64_t n_pad, plane;      // plane: floats
  size_t off_m, off_s, off_zt, off_rows, off_nact, total;
};
BlockWs block_ws(int64_t N, int64_t V) {
  BlockWs w;
  w.n_pad = round_up(N, 64);
  w.plane = block_partials(N, V);
  const int64_t plane = round_up(w.plane * 4, 256), per_token = round_up(w.n_pad * 4, 256);
  w.off_m = 0;
  w.off_s = (size_t)plane;
  w.off_zt = w.off_s + (size_t)plane;
  w.off_rows = w.off_zt + (size_t)per_token;
  w.off_nact = w.off_rows + (size_t)per_token;
  w.total = w.off_nact + 256;
  return w;
}

llamarl_status check_block_matrix(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0) return fail(LLAMARL_ERR_INVALID_ARG, "sizes must be positive (got %lld, %lld)", (long long)rows, (long long)cols);
  if (cols % 16 != 0) return fail(LLAMARL_ERR_UNSUPPORTED, "%lld columns: rows must be multiples of 16 bytes", (long long)cols);
  if (cols >= (int64_t)1 << 22 || rows >= (int64_t)1 << 31) return fail(LLAMARL_ERR_UNSUPPORTED, "matrix too large");
  return LLAMARL_OK;
}
constexpr int64_t BLOCK_MOST_H = (int64_t)1 << 31, BLOCK_MOST_ROWS = (int64_t)1 << 21;      // N d and V of a head are below these
llamarl_status check_block_head(const void* H, const uint8_t* H_scale, const void* W, const uint8_t* W_scale, int64_t N, int64_t d, int64_t V) {
  if (!H || !H_scale || !W || !W_scale) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  llamarl_status s = check_block_matrix(N, d);
  if (s == LLAMARL_OK) s = check_block_matrix(V, d);
  if (s != LLAMARL_OK) return s;
  if (N * d >= BLOCK_MOST_H) return fail(LLAMARL_ERR_UNSUPPORTED, "H must be smaller than 2 GiB (its rows are gathered with 32-bit offsets)");
  if (tile_count(N, V, 128) >= (int64_t)1 << 31 || V >= BLOCK_MOST_ROWS) return fail(LLAMARL_ERR_UNSUPPORTED, "too many tiles or logits of a token");
  if (!aligned16(H) || !aligned16(W)) return fail(LLAMARL_ERR_INVALID_ARG, "H and W must be 16-byte aligned");
  if (!aligned_to(H_scale, 4) || !aligned_to(W_scale, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "scales must be 4-byte aligned");
  return LLAMARL_OK;
}
BlockHead block_head(const void* H, const uint8_t* H_scale, const void* W, const uint8_t* W_scale) {
  return {static_cast<const uint8_t*>(H), static_cast<const uint8_t*>(W), reinterpret_cast<const uint32_t*>(H_scale),
          reinterpret_cast<const uint32_t*>(W_scale)};
}

template <int NB, typename Out>
llamarl_status launch_few_blocks(const FewArgs& a, hipStream_t st) {
  HIP_TRY(set_lds_if_large(k_few_tokens<NB, Out>, FEW_LDS<NB>));
  k_few_tokens<NB, Out><<<dim3((unsigned)((a.V + FEW_ROWS - 1) / FEW_ROWS)), dim3(FEW_THREADS), FEW_LDS<NB>, st>>>(a);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}
template <typename Out>
llamarl_status launch_few(FewArgs a, BlockTile tile, hipStream_t st) {
  if (tile == BLOCK_FEW)
    return (a.N <= 16   ? launch_few_blocks<1, Out>
            : a.N <= 32 ? launch_few_blocks<2, Out>
            : a.N <= 48 ? launch_few_blocks<3, Out>
                        : launch_few_blocks<4, Out>)(a, st);
  a.parts = direct_parts(a.d);
  const int rows = DIRECT_WAVES / a.parts * 16;
  k_few_direct<Out><<<dim3((unsigned)((a.V + rows - 1) / rows)), dim3(FEW_THREADS), 0, st>>>(a);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}
template <typename G, typename Out>
llamarl_status launch_block_logits(BlockLogitsArgs a, hipStream_t st) {
  a.tiles_v = (int)((a.v_end - a.v_first + G::Shape::BM - 1) / G::Shape::BM);
  a.tiles_t = (int)((a.N + G::Shape::BN - 1) / G::Shape::BN);
  constexpr int LDS = G::LDS_BYTES + TileStore<typename G::Shape, Out>::LDS_BYTES;
  static_assert(LDS * G::GROUPS_PER_CU <= 160 * 1024, "LDS of a CU");
  HIP_TRY(set_lds_if_large(k_block_logits<G, Out>, LDS));
  k_block_logits<G, Out><<<dim3((unsigned)persistent_grid((int64_t)a.tiles_v * a.tiles_t, G::GROUPS_PER_CU)), dim3(G::Shape::THREADS), LDS, st>>>(a);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}
template <typename G>
llamarl_status launch_block_partials(const FwdArgs& a, const BlockHead& x, hipStream_t st) {
  static_assert(fwd_bytes_of<G> * G::GROUPS_PER_CU <= 160 * 1024, "LDS of a CU");
  HIP_TRY(set_lds_if_large(k_block_partials<G>, fwd_bytes_of<G>));
  const int64_t tiles_t = (a.N + G::Shape::BN - 1) / G::Shape::BN;
  k_block_partials<G><<<dim3((unsigned)persistent_grid((int64_t)a.tiles_v * tiles_t, G::GROUPS_PER_CU)), dim3(G::Shape::THREADS),
                        fwd_bytes_of<G>, st>>>(a, x.h_words, x.w_words);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}

}  // namespace

extern "C" {

llamarl_status llamarl_quantise_blocks(const void* x, int64_t rows, int64_t cols, llamarl_dtype dt, int block_rows, void* q,
                                       uint8_t* scale, void* stream) {
  if (!x || !q || !scale) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if (!known(dt)) return fail(LLAMARL_ERR_INVALID_ARG, "unknown dtype %d", (int)dt);
  if (block_rows != 1 && block_rows != SCALE_BLOCK) return fail(LLAMARL_ERR_INVALID_ARG, "block_rows must be 1 or 128 (got %d)", block_rows);
  const llamarl_status s = check_block_matrix(rows, cols);
  if (s != LLAMARL_OK) return s;
  if (!aligned16(x) || !aligned16(q)) return fail(LLAMARL_ERR_INVALID_ARG, "x and q must be 16-byte aligned");
  if (!aligned_to(scale, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "scale must be 4-byte aligned");
  const int64_t groups = (cols + SCALE_GROUP - 1) / SCALE_GROUP, scale_rows = (rows + block_rows - 1) / block_rows;
  if (any_overlap({{q, rows * cols}, {scale, scale_rows * groups * 4}}, {{x, rows * cols * (int64_t)esize(dt)}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "x, q and scale must not overlap");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  QuantiseArgs a = {x, rows, cols, static_cast<uint8_t*>(q), reinterpret_cast<uint32_t*>(scale), (int)groups};
  const int64_t per = (QUANT_THREADS / 64) * QUANT_ROWS, blocks = block_rows == 1 ? (rows * groups + per - 1) / per : scale_rows * groups * 4;
  if (blocks >= (int64_t)1 << 24) return fail(LLAMARL_ERR_UNSUPPORTED, "matrix too large");
  const auto kernel = block_rows == 1 ? (dt == LLAMARL_BF16 ? k_quantise_rows<uint16_t> : k_quantise_rows<float>)
                                      : (dt == LLAMARL_BF16 ? k_quantise_tiles<uint16_t> : k_quantise_tiles<float>);
  kernel<<<dim3((unsigned)blocks), dim3(QUANT_THREADS), 0, st>>>(a);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}

llamarl_status llamarl_logits_blocks(const void* H, const uint8_t* H_scale, const void* W, const uint8_t* W_scale, int64_t N, int64_t d,
                                     int64_t V, llamarl_dtype z_dt, void* z, void* stream) {
  if (!z) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if (!known(z_dt)) return fail(LLAMARL_ERR_INVALID_ARG, "unknown dtype %d", (int)z_dt);
  const llamarl_status s = check_block_head(H, H_scale, W, W_scale, N, d, V);
  if (s != LLAMARL_OK) return s;
  if (!aligned16(z)) return fail(LLAMARL_ERR_INVALID_ARG, "z must be 16-byte aligned");
  const int64_t groups = (d + SCALE_GROUP - 1) / SCALE_GROUP;
  if (any_overlap({{z, N * V * (int64_t)esize(z_dt)}},
                  {{H, N * d}, {H_scale, groups * N * 4}, {W, V * d}, {W_scale, groups * ((V + SCALE_BLOCK - 1) / SCALE_BLOCK) * 4}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "z must not overlap an operand");
  const BlockHead x = block_head(H, H_scale, W, W_scale);
  const BlockLogits plan = z_dt == LLAMARL_F32 && N > FEW_TOKENS ? BlockLogits{block_tile(N, V, true), V, BLOCK_64} : block_logits(N, V, d);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (plan.tile <= BLOCK_FEW) {
    FewArgs f = {};
    f.x = x; f.N = N; f.d = d; f.V = V; f.z = z;
    return z_dt == LLAMARL_F32 ? launch_few<float>(f, plan.tile, st) : launch_few<uint16_t>(f, plan.tile, st);
  }
  BlockLogitsArgs a = {};
  a.x = x; a.N = N; a.d = d; a.V = V; a.z = z; a.v_end = plan.rows;
  if (z_dt == LLAMARL_F32) return (plan.tile == BLOCK_64 ? launch_block_logits<Exact64, float> : launch_block_logits<Exact128, float>)(a, st);
  if (N <= FEW_TOKENS) return (plan.tile == BLOCK_64 ? launch_block_logits<Exact64, uint16_t> : launch_block_logits<Exact128, uint16_t>)(a, st);
  const auto launch = [&](BlockTile t) {
    return (t == BLOCK_256   ? launch_block_logits<Blocks256, uint16_t>
            : t == BLOCK_128 ? launch_block_logits<Blocks128, uint16_t>
                             : launch_block_logits<Blocks64, uint16_t>)(a, st);
  };
  const llamarl_status first = launch(plan.tile);
  if (first != LLAMARL_OK || plan.rows == V) return first;
  a.v_first = plan.rows;
  a.v_end = V;
  return launch(plan.rest);
}

size_t llamarl_logprobs_blocks_workspace_bytes(int64_t N, int64_t V) {
  return N <= 0 || V <= 0 || N >= BLOCK_MOST_H / 16 || V >= BLOCK_MOST_ROWS ? 0 : block_ws(N, V).total;      // d >= 16
}

llamarl_status llamarl_token_logprobs_blocks(const void* H, const uint8_t* H_scale, const void* W, const uint8_t* W_scale,
                                             const int32_t* targets, const uint8_t* mask, int64_t N, int64_t d, int64_t V, float* logp,
                                             float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!targets || !logp || !lse) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  llamarl_status s = check_block_head(H, H_scale, W, W_scale, N, d, V);
  if (s != LLAMARL_OK) return s;
  if (!aligned_to(targets, 4) || !aligned_to(logp, 4) || !aligned_to(lse, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "misaligned targets, logp or lse");
  const BlockWs w = block_ws(N, V);
  if (!ws || ws_bytes < w.total)
    return fail(LLAMARL_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", ws ? ws_bytes : (size_t)0, w.total);
  if (!aligned16(ws)) return fail(LLAMARL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  const int64_t groups = (d + SCALE_GROUP - 1) / SCALE_GROUP;
  if (any_overlap({{logp, N * 4}, {lse, N * 4}, {ws, (int64_t)w.total}},
                  {{H, N * d}, {H_scale, groups * N * 4}, {W, V * d}, {W_scale, groups * ((V + SCALE_BLOCK - 1) / SCALE_BLOCK) * 4},
                   {targets, N * 4}, {mask, N}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "logp, lse and workspace must not overlap another array");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  char* base = reinterpret_cast<char*>(ws);
  int32_t *rows = reinterpret_cast<int32_t*>(base + w.off_rows), *n_act = reinterpret_cast<int32_t*>(base + w.off_nact);
  const BlockTile tile = block_tile(N, V, false);
  const BlockHead x = block_head(H, H_scale, W, W_scale);
  const int tile_rows = block_tile_rows(tile, d);
  FwdArgs a = {};
  a.H = H; a.W = W; a.targets = targets; a.N = N; a.d = d; a.V = V;
  a.tiles_v = (int)((V + tile_rows - 1) / tile_rows);
  a.n_pad = w.n_pad;
  if (a.tiles_v * w.n_pad > w.plane) return fail(LLAMARL_ERR_WORKSPACE, "partials of %d tiles do not fit", a.tiles_v);      // a mistake in the rules
  a.part_m = reinterpret_cast<float*>(base + w.off_m);
  a.part_s = reinterpret_cast<float*>(base + w.off_s);
  a.zt = reinterpret_cast<float*>(base + w.off_zt);
  a.rows = rows; a.n_act = n_act;
  k_compact_rows<<<dim3((unsigned)compact_blocks(N)), dim3(COMPACT_THREADS), 0, st>>>(
      compact_args({0, mask, targets, nullptr, V, N, 0, rows, n_act, logp, lse, nullptr, 0.f, nullptr, nullptr}));
  HIP_TRY(hipGetLastError());
  const bool exact = N <= FEW_TOKENS;
  if (tile <= BLOCK_FEW) {
    FewArgs f = {};
    f.x = x; f.N = N; f.d = d; f.V = V; f.f = a;
    s = launch_few<void>(f, tile, st);
  } else if (exact) {
    s = (tile == BLOCK_64 ? launch_block_partials<Exact64> : launch_block_partials<Exact128>)(a, x, st);
  } else {
    s = (tile == BLOCK_256   ? launch_block_partials<Blocks256>
         : tile == BLOCK_128 ? launch_block_partials<Blocks128>
                             : launch_block_partials<Blocks64>)(a, x, st);
  }
  if (s != LLAMARL_OK) return s;
  if (exact) return launch_merge(a, logp, lse, nullptr, 0, StoredTarget(), st);
  return launch_merge(a, logp, lse, nullptr, 0, BlockTarget{x, N, V, (int)d}, st);
}

}  // extern "C"
