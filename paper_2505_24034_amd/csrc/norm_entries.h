// norm_entries.h -- host side of llamarl_rms_norm and llamarl_rms_norm_bwd.  Part of llamarl.hip.
#pragma once

namespace {

template <int TH_, int UNITS_>
struct RowShape {
  static constexpr int TH = TH_, UNITS = UNITS_;
};
// f(RowShape) for rows of d entries: a wavefront a row up to 1024, then as many threads as have units of eight.  Forward of 16384 x 4096 bf16 rows on 256
// threads with two units each / 512 with one 91.9 / 89.9 us, 1900 x 8192 (four / 1024 with one) 20.8 / 19.7, 16384 x 2048 (64 with four / 256) 44.0 / 39.9.
template <typename F>
auto with_row_shape(int64_t d, F&& f) {
  const int64_t units = (d + OPT_ITEMS - 1) / OPT_ITEMS;
  if (units <= 64) return f(RowShape<64, 1>());
  if (units <= 128) return f(RowShape<64, 2>());
  if (units <= 256) return f(RowShape<256, 1>());
  if (units <= 512) return f(RowShape<512, 1>());
  if (units <= 1024) return f(RowShape<1024, 1>());
  return f(RowShape<1024, 2>());
}
// ... of quantise_rows, which holds less of a row: 16384 x 4096 on 256 threads / 512 29.2 / 32.3 us, 1900 x 8192 on 256 / 1024 8.3 / 9.9.
template <typename F>
auto with_quantise_shape(int64_t d, F&& f) {
  const int64_t units = (d + OPT_ITEMS - 1) / OPT_ITEMS;
  if (units <= 64) return f(RowShape<64, 1>());
  if (units <= 128) return f(RowShape<64, 2>());
  if (units <= 256) return f(RowShape<256, 1>());
  if (units <= 512) return f(RowShape<256, 2>());
  if (units <= 1024) return f(RowShape<256, 4>());
  return f(RowShape<1024, 2>());
}
int row_threads(int64_t d) {
  return with_row_shape(d, [](auto s) { return decltype(s)::TH; });
}
// rows of a workgroup
int64_t rows_each(int64_t d) { return row_threads(d) == 64 ? 4 : 1; }
// `rows` on `threads` threads each: a launch has fewer than 2^32
llamarl_status check_row_launch(int64_t rows, int threads) {
  const int64_t each = threads == 64 ? 4 : 1;
  return (rows + each - 1) / each * std::max(threads, 256) >= (int64_t)1 << 32 ? fail(LLAMARL_ERR_UNSUPPORTED, "too many rows") : LLAMARL_OK;
}

llamarl_status check_norm(int64_t N, int64_t d, llamarl_dtype dt, llamarl_dtype w_dt, const void* w) {
  if (N <= 0 || d <= 0) return fail(LLAMARL_ERR_INVALID_ARG, "sizes must be positive (got %lld, %lld)", (long long)N, (long long)d);
  if (!known(dt) || !known(w_dt)) return fail(LLAMARL_ERR_INVALID_ARG, "unknown dtype");
  if (d % (16 / (int64_t)esize(dt)) != 0) return fail(LLAMARL_ERR_UNSUPPORTED, "d = %lld: rows must be multiples of 16 bytes", (long long)d);
  if (d > NORM_MOST_COLS) return fail(LLAMARL_ERR_UNSUPPORTED, "d must be at most %lld", (long long)NORM_MOST_COLS);
  if (N >= (int64_t)1 << 31) return fail(LLAMARL_ERR_UNSUPPORTED, "too many rows");
  if (!aligned16(w)) return fail(LLAMARL_ERR_INVALID_ARG, "weight must be 16-byte aligned");
  return check_row_launch(N, row_threads(d));
}
// workgroups, and rows of partial sums; none for few rows, whose columns are summed up as they are
int64_t norm_bwd_blocks(int64_t N, int64_t d) {
  return std::min<int64_t>((N + rows_each(d) - 1) / rows_each(d), row_threads(d) == 1024 ? NORM_BWD_BLOCKS / 2 : NORM_BWD_BLOCKS);
}
bool norm_columns(int64_t N) { return N <= NORM_FEW_ROWS; }

template <typename T, int OUT>
llamarl_status launch_norm(const NormArgs& a, hipStream_t st) {
  with_row_shape(a.d, [&](auto s) {
    constexpr int TH = decltype(s)::TH;
    const int64_t per = rows_each(a.d);
    k_rms_norm<T, OUT, TH, decltype(s)::UNITS><<<dim3((unsigned)((a.N + per - 1) / per)), dim3(NORM_THREADS_OF<TH>), 0, st>>>(a);
    return 0;
  });
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}
template <typename T>
llamarl_status launch_norm_out(const NormArgs& a, llamarl_norm_out out, hipStream_t st) {
  return out == LLAMARL_NORM_SAME ? launch_norm<T, OUT_SAME>(a, st)
         : out == LLAMARL_NORM_E4M3_BLOCKS ? launch_norm<T, OUT_BLOCKS>(a, st) : launch_norm<T, OUT_ROWS>(a, st);
}
template <typename T>
void launch_norm_bwd(const NormBwdArgs& a, hipStream_t st) {
  const int columns = a.dw ? (a.d + NORM_COLUMNS - 1) / NORM_COLUMNS : 0;
  with_row_shape(a.d, [&](auto s) {
    constexpr int TH = decltype(s)::TH;
    k_rms_norm_bwd<T, TH, decltype(s)::UNITS><<<dim3((unsigned)(a.row_blocks + columns)), dim3(NORM_THREADS_OF<TH>), 0, st>>>(a);
    return 0;
  });
}

}  // namespace

extern "C" {

llamarl_status llamarl_rms_norm(const void* x, const void* residual, const void* weight, int64_t N, int64_t d, llamarl_dtype dt,
                                llamarl_dtype w_dt, float eps, llamarl_norm_out out, void* sum, void* h, void* h_scale, float* rstd,
                                void* stream) {
  if (!x || !weight || !h) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if ((residual == nullptr) != (sum == nullptr)) return fail(LLAMARL_ERR_INVALID_ARG, "residual and sum go together");
  if (out != LLAMARL_NORM_SAME && out != LLAMARL_NORM_E4M3_BLOCKS && out != LLAMARL_NORM_INT8_ROWS)
    return fail(LLAMARL_ERR_INVALID_ARG, "unknown output %d", (int)out);
  if ((out == LLAMARL_NORM_SAME) != (h_scale == nullptr)) return fail(LLAMARL_ERR_INVALID_ARG, "an output in 8 bits has scales, and no other");
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(LLAMARL_ERR_INVALID_ARG, "eps must be positive and finite");
  const llamarl_status s = check_norm(N, d, dt, w_dt, weight);
  if (s != LLAMARL_OK) return s;
  if (out != LLAMARL_NORM_SAME && d % 16 != 0) return fail(LLAMARL_ERR_UNSUPPORTED, "d = %lld: rows of 8 bits must be multiples of 16 bytes", (long long)d);
  if (!aligned16(x) || !aligned16(residual) || !aligned16(sum) || !aligned16(h)) return fail(LLAMARL_ERR_INVALID_ARG, "x, residual, sum and h must be 16-byte aligned");
  if (!aligned_to(h_scale, 4) || !aligned_to(rstd, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "h_scale and rstd must be 4-byte aligned");
  const int64_t bytes = N * d * (int64_t)esize(dt);
  const int64_t scales = out == LLAMARL_NORM_E4M3_BLOCKS ? (d + SCALE_GROUP - 1) / SCALE_GROUP * N * 4 : N * 4;
  if (any_overlap({{sum, bytes}, {h, out == LLAMARL_NORM_SAME ? bytes : N * d}, {h_scale, scales}, {rstd, N * 4}},
                  {{x, bytes}, {residual, bytes}, {weight, d * (int64_t)esize(w_dt)}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "outputs must not overlap another array");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const NormArgs a = {x, residual, weight, N, (int)d, w_dt == LLAMARL_BF16, eps, sum, h, h_scale, rstd};
  return dt == LLAMARL_BF16 ? launch_norm_out<uint16_t>(a, out, st) : launch_norm_out<float>(a, out, st);
}

size_t llamarl_rms_norm_bwd_workspace_bytes(int64_t N, int64_t d) {
  return N <= 0 || d <= 0 || d > NORM_MOST_COLS || norm_columns(N) ? 0 : (size_t)(norm_bwd_blocks(N, d) * d * 4);
}

llamarl_status llamarl_rms_norm_bwd(const void* dh, const void* s, const void* weight, const float* rstd, const void* dsum, int64_t N,
                                    int64_t d, llamarl_dtype dt, llamarl_dtype w_dt, void* dx, void* dweight, llamarl_dtype dw_dt,
                                    void* ws, size_t ws_bytes, void* stream) {
  if (!dh || !s || !weight || !rstd || !dx) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  const llamarl_status status = check_norm(N, d, dt, w_dt, weight);
  if (status != LLAMARL_OK) return status;
  if (!known(dw_dt)) return fail(LLAMARL_ERR_INVALID_ARG, "unknown dtype %d", (int)dw_dt);
  if (!aligned16(dh) || !aligned16(s) || !aligned16(dsum) || !aligned16(dx)) return fail(LLAMARL_ERR_INVALID_ARG, "dh, s, dsum and dx must be 16-byte aligned");
  if (!aligned_to(rstd, 4) || !aligned_to(dweight, esize(dw_dt))) return fail(LLAMARL_ERR_INVALID_ARG, "misaligned rstd or dweight");
  const size_t need = llamarl_rms_norm_bwd_workspace_bytes(N, d);
  if (dweight != nullptr && need > 0) {
    if (!ws || ws_bytes < need)
      return fail(LLAMARL_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", ws ? ws_bytes : (size_t)0, need);
    if (!aligned16(ws)) return fail(LLAMARL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  }
  const int64_t bytes = N * d * (int64_t)esize(dt);
  if (any_overlap({{dx, bytes}, {dweight, d * (int64_t)esize(dw_dt)}, {dweight && need > 0 ? ws : nullptr, (int64_t)need}},
                  {{dh, bytes}, {s, bytes}, {dsum, bytes}, {weight, d * (int64_t)esize(w_dt)}, {rstd, N * 4}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "outputs and workspace must not overlap another array");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const int64_t blocks = norm_bwd_blocks(N, d);
  const bool columns = dweight != nullptr && norm_columns(N);
  const NormBwdArgs a = {dh, s, weight, rstd, dsum, N, (int)d, w_dt == LLAMARL_BF16, dx, dweight && !columns ? static_cast<float*>(ws) : nullptr,
                         (int)blocks, columns ? dweight : nullptr, dw_dt == LLAMARL_BF16};
  if (dt == LLAMARL_BF16) launch_norm_bwd<uint16_t>(a, st);
  else launch_norm_bwd<float>(a, st);
  HIP_TRY(hipGetLastError());
  if (a.part == nullptr) return LLAMARL_OK;
  k_norm_dw<<<dim3((unsigned)((d + NORM_DW_COLS - 1) / NORM_DW_COLS)), dim3(NORM_DW_COLS * NORM_DW_SLICES), 0, st>>>(
      a.part, (int)blocks, (int)d, dweight, dw_dt == LLAMARL_BF16);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}

}  // extern "C"
