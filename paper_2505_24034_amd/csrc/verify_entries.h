// verify_entries.h -- host side of llamarl_verify_drafts.  Part of llamarl.hip.
#pragma once

namespace {

struct VerifyWs {
  int64_t rows, chunks;
  size_t off_at, off_sums, off_ticket, total;
};
VerifyWs verify_ws(int64_t B, int64_t K, int64_t V) {
  VerifyWs w;
  w.rows = B * (2 * K + 1);
  w.chunks = (V + VERIFY_CHUNK - 1) / VERIFY_CHUNK;
  w.off_at = (size_t)round_up(w.rows * w.chunks * (int64_t)sizeof(VerifyPart), 256);
  w.off_sums = w.off_at + (size_t)round_up(w.rows * 4, 256);
  w.off_ticket = w.off_sums + (size_t)round_up(B * w.chunks * (VERIFY_CHUNK / VERIFY_PART) * 8, 256);
  w.total = w.off_ticket + (size_t)round_up(B * 4, 256);
  return w;
}
bool verify_fits(int64_t B, int64_t K, int64_t V) {
  return B > 0 && K >= 0 && V > 0 && K <= VERIFY_MOST_DRAFTS && V < BLOCK_MOST_ROWS && B < (int64_t)1 << 20 &&
         B * (2 * K + 1) * ((V + VERIFY_CHUNK - 1) / VERIFY_CHUNK) < ((int64_t)1 << 32) / VERIFY_THREADS;
}
static_assert(VERIFY_ROW_CHUNK == VERIFY_CHUNK && VERIFY_PICK_UNIT == VERIFY_THREADS * OPT_ITEMS, "the rule's cuts");
template <typename T>
llamarl_status launch_verify(const VerifyArgs& a, int64_t rows, hipStream_t st) {
  const VerifyPlan p = verify_plan(rows, a.B, a.V, persistent_grid((int64_t)1 << 30));
  // a workgroup's only chunk is asked for before it knows whether somebody wants it
  k_verify_rows<T><<<dim3((unsigned)(rows * p.row_groups())), dim3(VERIFY_THREADS), 0, st>>>(a, (int)p.each, p.each == 1);
  HIP_TRY(hipGetLastError());
  k_verify_pick<T><<<dim3((unsigned)(a.B * p.pick_groups())), dim3(VERIFY_THREADS), 0, st>>>(a, (int)p.units, (int)p.some);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}

}  // namespace

extern "C" {

size_t llamarl_verify_drafts_workspace_bytes(int64_t B, int64_t K, int64_t V) { return verify_fits(B, K, V) ? verify_ws(B, K, V).total : 0; }

llamarl_status llamarl_verify_drafts(const void* logits, const void* draft_logits, const int32_t* drafts, const int32_t* draft_lens,
                                     const float* temperature, const float* uniforms, int64_t B, int64_t K, int64_t V, llamarl_dtype dt,
                                     int32_t* tokens, int32_t* accepted, float* logp, void* ws, size_t ws_bytes, void* stream) {
  if (!logits || !uniforms || !tokens || !accepted || !logp || (K > 0 && !drafts)) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if (B <= 0 || K < 0 || V <= 0) return fail(LLAMARL_ERR_INVALID_ARG, "bad sizes (B %lld, K %lld, V %lld)", (long long)B, (long long)K, (long long)V);
  if (!known(dt)) return fail(LLAMARL_ERR_INVALID_ARG, "unknown dtype %d", (int)dt);
  if (!verify_fits(B, K, V)) return fail(LLAMARL_ERR_UNSUPPORTED, "too many sequences, drafts (at most %d) or logits", VERIFY_MOST_DRAFTS);
  const size_t e = esize(dt);
  if (!aligned_to(logits, e) || !aligned_to(draft_logits, e) || !aligned_to(drafts, 4) || !aligned_to(draft_lens, 4) || !aligned_to(temperature, 4) ||
      !aligned_to(uniforms, 4) || !aligned_to(tokens, 4) || !aligned_to(accepted, 4) || !aligned_to(logp, 4))
    return fail(LLAMARL_ERR_INVALID_ARG, "arrays must have the alignment of their type");
  const VerifyWs w = verify_ws(B, K, V);
  if (!ws || ws_bytes < w.total)
    return fail(LLAMARL_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", ws ? ws_bytes : (size_t)0, w.total);
  if (!aligned16(ws)) return fail(LLAMARL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (K == 0) draft_logits = nullptr;
  const int64_t slots = B * (K + 1);
  if (any_overlap({{tokens, slots * 4}, {accepted, B * 4}, {logp, slots * 4}, {ws, (int64_t)w.total}},
                  {{logits, slots * V * (int64_t)e}, {draft_logits, B * K * V * (int64_t)e}, {K > 0 ? drafts : nullptr, B * K * 4}, {draft_lens, B * 4},
                   {temperature, B * 4}, {uniforms, slots * 4}}))
    return fail(LLAMARL_ERR_INVALID_ARG, "outputs and workspace must not overlap another array");
  char* base = static_cast<char*>(ws);
  const VerifyArgs a = {logits, draft_logits, drafts, draft_lens, temperature, uniforms, V, (int)B, (int)K, (int)w.chunks,
                        reinterpret_cast<VerifyPart*>(base), reinterpret_cast<float*>(base + w.off_at), reinterpret_cast<double*>(base + w.off_sums),
                        reinterpret_cast<unsigned int*>(base + w.off_ticket), tokens, accepted, logp};
  const int64_t rows = draft_logits ? w.rows : slots;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  return dt == LLAMARL_BF16 ? launch_verify<uint16_t>(a, rows, st) : launch_verify<float>(a, rows, st);
}

}  // extern "C"
