// row_entries.h -- host side of llamarl_quantise_rows, llamarl_logits_rows and llamarl_token_logprobs_rows.  Part of llamarl.hip.
#pragma once

namespace {

// As BlockWs; the planes: row_partials.
BlockWs row_ws(int64_t N, int64_t V) {
  BlockWs w;
  w.n_pad = round_up(N, 64);
  w.plane = row_partials(N, V);
  const int64_t plane = round_up(w.plane * 4, 256), per_token = round_up(w.n_pad * 4, 256);
  w.off_m = 0;
  w.off_s = (size_t)plane;
  w.off_zt = w.off_s + (size_t)plane;
  w.off_rows = w.off_zt + (size_t)per_token;
  w.off_nact = w.off_rows + (size_t)per_token;
  w.total = w.off_nact + 256;
  return w;
}

constexpr int64_t ROW_MOST_COLS = (int64_t)1 << 17;  // columns are below this: 2^17 products of 2^14 would not fit an int32
llamarl_status check_row_matrix(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0) return fail(LLAMARL_ERR_INVALID_ARG, "sizes must be positive (got %lld, %lld)", (long long)rows, (long long)cols);
  if (cols % 16 != 0) return fail(LLAMARL_ERR_UNSUPPORTED, "%lld columns: rows must be multiples of 16 bytes", (long long)cols);
  if (cols >= ROW_MOST_COLS || rows >= (int64_t)1 << 31) return fail(LLAMARL_ERR_UNSUPPORTED, "matrix too large");
  return LLAMARL_OK;
}
llamarl_status check_row_head(const RowHead& x, int64_t N, int64_t d, int64_t V) {
  if (!x.H || !x.h_scale || !x.W || !x.w_scale) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  llamarl_status s = check_row_matrix(N, d);
  if (s == LLAMARL_OK) s = check_row_matrix(V, d);
  if (s != LLAMARL_OK) return s;
  if (N * d >= BLOCK_MOST_H) return fail(LLAMARL_ERR_UNSUPPORTED, "H must be smaller than 2 GiB (its rows are gathered with 32-bit offsets)");
  if (V >= BLOCK_MOST_ROWS || tile_count(N, V, 64) >= (int64_t)1 << 31) return fail(LLAMARL_ERR_UNSUPPORTED, "too many tiles or logits of a token");
  if (!aligned16(x.H) || !aligned16(x.W)) return fail(LLAMARL_ERR_INVALID_ARG, "H and W must be 16-byte aligned");
  if (!aligned_to(x.h_scale, 4) || !aligned_to(x.w_scale, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "scales must be 4-byte aligned");
  return LLAMARL_OK;
}

template <typename Out>
llamarl_status launch_row_direct(RowFewArgs a, hipStream_t st) {
  a.few.parts = direct_parts(a.few.d);
  const int rows = DIRECT_WAVES / a.few.parts * 16;
  k_row_direct<Out><<<dim3((unsigned)((a.few.V + rows - 1) / rows)), dim3(FEW_THREADS), 0, st>>>(a);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}
template <typename G, typename Out>
llamarl_status launch_row_logits(RowLogitsArgs a, hipStream_t st) {
  a.tiles_v = (int)((a.v_end - a.v_first + G::Shape::BM - 1) / G::Shape::BM);
  a.tiles_t = (int)((a.N + G::Shape::BN - 1) / G::Shape::BN);
  constexpr int LDS = G::LDS_BYTES + TileStore<typename G::Shape, Out>::LDS_BYTES;
  static_assert(LDS * G::GROUPS_PER_CU <= 160 * 1024, "LDS of a CU");
  HIP_TRY(set_lds_if_large(k_row_logits<G, Out>, LDS));
  k_row_logits<G, Out><<<dim3((unsigned)persistent_grid((int64_t)a.tiles_v * a.tiles_t, G::GROUPS_PER_CU)), dim3(G::Shape::THREADS), LDS, st>>>(a);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}
template <typename Out>
llamarl_status launch_row_tiles(const RowLogitsArgs& a, RowTile t, hipStream_t st) {
  return (t == ROW_256 ? launch_row_logits<Rows256Stored, Out> : t == ROW_128 ? launch_row_logits<Rows128, Out> : launch_row_logits<Rows64, Out>)(a, st);
}
template <typename G>
llamarl_status launch_row_partials(const FwdArgs& a, const RowHead& x, hipStream_t st) {
  static_assert(fwd_bytes_of<G> * G::GROUPS_PER_CU <= 160 * 1024, "LDS of a CU");
  HIP_TRY(set_lds_if_large(k_row_partials<G>, fwd_bytes_of<G>));
  const int64_t tiles_t = (a.N + G::Shape::BN - 1) / G::Shape::BN;
  k_row_partials<G><<<dim3((unsigned)persistent_grid((int64_t)a.tiles_v * tiles_t, G::GROUPS_PER_CU)), dim3(G::Shape::THREADS),
                      fwd_bytes_of<G>, st>>>(a, x);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}
constexpr int QUANTISE_MOST_THREADS = 1024;          // of rows longer than NORM_MOST_COLS
int quantise_threads(int64_t cols) {
  return cols > NORM_MOST_COLS ? QUANTISE_MOST_THREADS : with_quantise_shape(cols, [](auto s) { return decltype(s)::TH; });
}
template <typename T>
void launch_quantise_int8(const QuantiseRowsArgs& a, hipStream_t st) {
  if (a.cols > NORM_MOST_COLS) {
    k_quantise_int8<T, QUANTISE_MOST_THREADS, 0><<<dim3((unsigned)a.rows), dim3(QUANTISE_MOST_THREADS), 0, st>>>(a);
    return;
  }
  with_quantise_shape(a.cols, [&](auto s) {
    constexpr int TH = decltype(s)::TH;
    const int64_t per = rows_each(a.cols);
    k_quantise_int8<T, TH, decltype(s)::UNITS><<<dim3((unsigned)((a.rows + per - 1) / per)), dim3(NORM_THREADS_OF<TH>), 0, st>>>(a);
    return 0;
  });
}

}  // namespace

extern "C" {

llamarl_status llamarl_quantise_rows(const void* x, int64_t rows, int64_t cols, llamarl_dtype dt, int8_t* q, float* scale, void* stream) {
  if (!x || !q || !scale) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if (!known(dt)) return fail(LLAMARL_ERR_INVALID_ARG, "unknown dtype %d", (int)dt);
  llamarl_status s = check_row_matrix(rows, cols);
  if (s == LLAMARL_OK) s = check_row_launch(rows, quantise_threads(cols));
  if (s != LLAMARL_OK) return s;
  if (!aligned16(x) || !aligned16(q)) return fail(LLAMARL_ERR_INVALID_ARG, "x and q must be 16-byte aligned");
  if (!aligned_to(scale, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "scale must be 4-byte aligned");
  if (any_overlap({{q, rows * cols}, {scale, rows * 4}}, {{x, rows * cols * (int64_t)esize(dt)}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "x, q and scale must not overlap");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const QuantiseRowsArgs a = {x, rows, (int)cols, q, scale};
  if (dt == LLAMARL_BF16) launch_quantise_int8<uint16_t>(a, st);
  else launch_quantise_int8<float>(a, st);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}

llamarl_status llamarl_logits_rows(const int8_t* H, const float* H_scale, const int8_t* W, const float* W_scale, int64_t N, int64_t d,
                                   int64_t V, llamarl_dtype z_dt, void* z, void* stream) {
  if (!z) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if (!known(z_dt)) return fail(LLAMARL_ERR_INVALID_ARG, "unknown dtype %d", (int)z_dt);
  const RowHead x = {H, W, H_scale, W_scale};
  const llamarl_status s = check_row_head(x, N, d, V);
  if (s != LLAMARL_OK) return s;
  if (!aligned16(z)) return fail(LLAMARL_ERR_INVALID_ARG, "z must be 16-byte aligned");
  if (any_overlap({{z, N * V * (int64_t)esize(z_dt)}}, {{H, N * d}, {H_scale, N * 4}, {W, V * d}, {W_scale, V * 4}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "z must not overlap an operand");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const RowPlan plan = row_plan(N, V, d, false);
  if (plan.tile == ROW_DIRECT) {
    RowFewArgs f = {};
    f.x = x;
    f.few.N = N; f.few.d = d; f.few.V = V; f.few.z = z;
    return z_dt == LLAMARL_F32 ? launch_row_direct<float>(f, st) : launch_row_direct<uint16_t>(f, st);
  }
  RowLogitsArgs a = {x, N, d, V, 0, plan.rows, 0, 0, z};
  const auto launch = [&](RowTile t) { return z_dt == LLAMARL_F32 ? launch_row_tiles<float>(a, t, st) : launch_row_tiles<uint16_t>(a, t, st); };
  const llamarl_status first = launch(plan.tile);
  if (first != LLAMARL_OK || plan.rows == V) return first;
  a.v_first = plan.rows;
  a.v_end = V;
  return launch(plan.rest);
}

size_t llamarl_logprobs_rows_workspace_bytes(int64_t N, int64_t V) {
  return N <= 0 || V <= 0 || N >= BLOCK_MOST_H / 16 || V >= BLOCK_MOST_ROWS ? 0 : row_ws(N, V).total;      // d >= 16
}

llamarl_status llamarl_token_logprobs_rows(const int8_t* H, const float* H_scale, const int8_t* W, const float* W_scale,
                                           const int32_t* targets, const uint8_t* mask, int64_t N, int64_t d, int64_t V, float* logp,
                                           float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!targets || !logp || !lse) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  const RowHead x = {H, W, H_scale, W_scale};
  llamarl_status s = check_row_head(x, N, d, V);
  if (s != LLAMARL_OK) return s;
  if (!aligned_to(targets, 4) || !aligned_to(logp, 4) || !aligned_to(lse, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "misaligned targets, logp or lse");
  const BlockWs w = row_ws(N, V);
  if (!ws || ws_bytes < w.total)
    return fail(LLAMARL_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", ws ? ws_bytes : (size_t)0, w.total);
  if (!aligned16(ws)) return fail(LLAMARL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (any_overlap({{logp, N * 4}, {lse, N * 4}, {ws, (int64_t)w.total}},
                  {{H, N * d}, {H_scale, N * 4}, {W, V * d}, {W_scale, V * 4}, {targets, N * 4}, {mask, N}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "logp, lse and workspace must not overlap another array");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  char* base = reinterpret_cast<char*>(ws);
  int32_t *rows = reinterpret_cast<int32_t*>(base + w.off_rows), *n_act = reinterpret_cast<int32_t*>(base + w.off_nact);
  const RowPlan plan = row_plan(N, V, d, true);
  const int tile_rows = row_tile_rows(plan.tile, d), rest_rows = row_tile_rows(plan.rest, d);
  const int tiles = (int)((plan.rows + tile_rows - 1) / tile_rows), rest = (int)((V - plan.rows + rest_rows - 1) / rest_rows);
  FwdArgs a = {};
  a.H = H; a.W = W; a.targets = targets; a.N = N; a.d = d; a.V = V;
  a.tiles_v = tiles + rest;
  a.n_pad = w.n_pad;
  if (a.tiles_v * w.n_pad > w.plane) return fail(LLAMARL_ERR_WORKSPACE, "partials of %d tiles do not fit", a.tiles_v);      // a mistake in the rules
  a.part_m = reinterpret_cast<float*>(base + w.off_m);
  a.part_s = reinterpret_cast<float*>(base + w.off_s);
  a.zt = reinterpret_cast<float*>(base + w.off_zt);
  a.rows = rows; a.n_act = n_act;
  k_compact_rows<<<dim3((unsigned)compact_blocks(N)), dim3(COMPACT_THREADS), 0, st>>>(
      compact_args({0, mask, targets, nullptr, V, N, 0, rows, n_act, logp, lse, nullptr, 0.f, nullptr, nullptr}));
  HIP_TRY(hipGetLastError());
  if (plan.tile == ROW_DIRECT) {
    RowFewArgs f = {};
    f.x = x;
    f.few.N = N; f.few.d = d; f.few.V = V; f.few.f = a;
    s = launch_row_direct<void>(f, st);
  } else {
    // rows [first, first + count) of W, their partials from tile `at` on
    const auto launch = [&](RowTile t, int64_t first, int64_t count, int at, int n) {
      FwdArgs p = a;
      p.W = W + first * d; p.V = count; p.v_off = first; p.tiles_v = n;
      p.part_m += at * w.n_pad; p.part_s += at * w.n_pad;
      const RowHead y = {H, W + first * d, H_scale, W_scale + first};
      return (t == ROW_256 ? launch_row_partials<Rows256> : t == ROW_128 ? launch_row_partials<Rows128> : launch_row_partials<Rows64>)(p, y, st);
    };
    s = launch(plan.tile, 0, plan.rows, 0, tiles);
    if (s == LLAMARL_OK && rest > 0) s = launch(plan.rest, plan.rows, V - plan.rows, tiles, rest);
  }
  if (s != LLAMARL_OK) return s;
  return launch_merge(a, logp, lse, nullptr, 0, StoredTarget(), st);
}

}  // extern "C"
