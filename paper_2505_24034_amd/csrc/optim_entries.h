// optim_entries.h -- host side of llamarl_grad_norm and llamarl_adamw_step: checks, the tensors of each launch, the launches.
// Part of llamarl.hip.
#pragma once

namespace {

constexpr int64_t OPT_MAX_ENTRIES = (int64_t)1 << 34;        // of a call: 2^22 workgroups of a unit

inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool known(llamarl_dtype dt) { return dt == LLAMARL_F32 || dt == LLAMARL_BF16; }

// f(list, workgroups) for each launch's tensors.  tensor(i, t): fills t (n among it) from the caller's i-th; tensors without entries
// take no part.
template <typename T, typename F>
llamarl_status for_each_launch(int64_t count, int units, OptList& l, T tensor, F launch) {
  const int64_t per = (int64_t)units * OPT_UNIT;
  constexpr int64_t MOST = ((int64_t)1 << 32) / OPT_THREADS - 1;      // a launch has fewer than 2^32 threads
  static_assert(OPT_MAX_ENTRIES / OPT_UNIT < MOST, "one tensor always fits a launch");
  l.units = units;
  l.count = 0;
  int64_t blocks = 0;
  auto flush = [&]() -> llamarl_status {
    if (l.count == 0) return LLAMARL_OK;
    l.first[l.count] = (int)blocks;
    const llamarl_status s = launch(l, (unsigned)blocks);
    l.count = 0;
    blocks = 0;
    return s;
  };
  for (int64_t i = 0; i < count; ++i) {
    OptTensor t = {};
    tensor(i, t);
    if (t.n == 0) continue;
    const int64_t need = (t.n + per - 1) / per;
    if (l.count == OPT_TENSORS || blocks + need > MOST) {
      const llamarl_status s = flush();
      if (s != LLAMARL_OK) return s;
    }
    l.t[l.count] = t;
    l.first[l.count++] = (int)blocks;
    blocks += need;
  }
  return flush();
}

// Whether a range of what a call writes lies over another of them, or over what it reads.
struct Span {
  const void* p;             // null: not given
  int64_t bytes;
};
bool any_overlap(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  auto meet = [](const Span& x, const Span& y) { return x.p != nullptr && y.p != nullptr && overlap(x.p, x.bytes, y.p, y.bytes); };
  for (const Span* w = written.begin(); w != written.end(); ++w) {
    for (const Span* o = w + 1; o != written.end(); ++o)
      if (meet(*w, *o)) return true;
    for (const Span& r : read)
      if (meet(*w, r)) return true;
  }
  return false;
}

struct Range {
  uintptr_t from, to;
  int64_t tensor;
  bool written;
};

// Whether anything that a step writes lies over something else that it reads or writes.
llamarl_status check_apart(const llamarl_adamw_tensor* t, int64_t count, const float* grad_scale, const float* lr_device, const int64_t* step_device) {
  const size_t most = (size_t)count * 7 + 3;
  Range* r = new (std::nothrow) Range[most];
  if (r == nullptr) return fail(LLAMARL_ERR_INVALID_ARG, "no host memory for a list of %lld tensors", (long long)count);
  size_t k = 0;
  for (int64_t i = 0; i < count; ++i) {
    const int64_t n = t[i].n, blocks = (n + STATE_BLOCK - 1) / STATE_BLOCK;
    if (n == 0) continue;
    const bool bits8 = t[i].m_scale != nullptr;
    auto add = [&](const void* p, int64_t bytes, bool written) {
      if (p != nullptr) r[k++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes, i, written};
    };
    add(t[i].param, n * (int64_t)esize(t[i].param_dt), true);
    add(t[i].master, n * 4, true);
    add(t[i].grad, n * (int64_t)esize(t[i].grad_dt), false);
    add(t[i].m, n * (bits8 ? 1 : 4), true);
    add(t[i].v, n * (bits8 ? 1 : 4), true);
    add(t[i].m_scale, blocks * 4, true);
    add(t[i].v_scale, blocks * 4, true);
  }
  auto word = [&](const void* p, uintptr_t bytes) {
    if (p != nullptr) r[k++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, count, false};
  };
  word(grad_scale, 4);
  word(lr_device, 4);
  word(step_device, 8);
  std::sort(r, r + k, [](const Range& x, const Range& y) { return x.from < y.from; });
  int64_t a = -1, b = -1;
  Range read = {0, 0, -1, false}, written = {0, 0, -1, true};        // those that reach furthest so far
  for (size_t i = 0; i < k && a < 0; ++i) {
    const Range* over = written.to > r[i].from ? &written : r[i].written && read.to > r[i].from ? &read : nullptr;
    if (over != nullptr) {
      a = over->tensor;
      b = r[i].tensor;
    }
    Range& far = r[i].written ? written : read;
    if (r[i].to > far.to) far = r[i];
  }
  delete[] r;
  if (a == count || b == count)
    return fail(LLAMARL_ERR_INVALID_ARG, "grad_scale, lr_device or step_device lies in tensor %lld", (long long)std::min(a, b));
  if (a >= 0) return fail(LLAMARL_ERR_INVALID_ARG, "arrays of tensors %lld and %lld overlap", (long long)a, (long long)b);
  return LLAMARL_OK;
}

llamarl_status check_adamw(const llamarl_adamw_tensor* tensors, int64_t count, const llamarl_adamw_params* p, const float* grad_scale,
                           const float* lr_device, const int64_t* step_device, int64_t& total) {
  if (p == nullptr || (tensors == nullptr && count > 0)) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if (count < 0 || count > (int64_t)1 << 24) return fail(LLAMARL_ERR_INVALID_ARG, "count must lie in [0, 2^24] (got %lld)", (long long)count);
  auto rate = [](double b) { return b >= 0.0 && b < 1.0; };
  auto weight = [](double x) { return x >= 0.0 && std::isfinite(x); };
  if (!rate(p->beta1) || !rate(p->beta2))
    return fail(LLAMARL_ERR_INVALID_ARG, "betas must lie in [0, 1) (got %g, %g)", p->beta1, p->beta2);
  if (!weight(p->eps) || !weight(p->weight_decay) || (lr_device == nullptr && !weight(p->lr)))
    return fail(LLAMARL_ERR_INVALID_ARG, "lr, eps and weight_decay must be finite and not negative (got %g, %g, %g)", p->lr, p->eps,
                p->weight_decay);
  if (step_device == nullptr && p->step < 1) return fail(LLAMARL_ERR_INVALID_ARG, "step counts from 1 (got %lld)", (long long)p->step);
  if (!aligned_to(grad_scale, 4) || !aligned_to(lr_device, 4) || !aligned_to(step_device, 8))
    return fail(LLAMARL_ERR_INVALID_ARG, "misaligned grad_scale, lr_device or step_device");
  total = 0;
  for (int64_t i = 0; i < count; ++i) {
    const llamarl_adamw_tensor& t = tensors[i];
    if (t.n < 0) return fail(LLAMARL_ERR_INVALID_ARG, "tensor %lld has %lld entries", (long long)i, (long long)t.n);
    if (t.n == 0) continue;
    if (!known(t.param_dt) || !known(t.grad_dt)) return fail(LLAMARL_ERR_INVALID_ARG, "tensor %lld: unknown dtype", (long long)i);
    if (!t.param || !t.grad || !t.m || !t.v) return fail(LLAMARL_ERR_INVALID_ARG, "tensor %lld: null pointer", (long long)i);
    if ((t.m_scale == nullptr) != (t.v_scale == nullptr))
      return fail(LLAMARL_ERR_INVALID_ARG, "tensor %lld: both m_scale and v_scale, or neither", (long long)i);
    if (t.m_scale != nullptr && p->beta1 > STATE_BETA1)
      return fail(LLAMARL_ERR_INVALID_ARG, "tensor %lld: first moments in 8 bits need beta1 <= %g (got %g)", (long long)i, STATE_BETA1, p->beta1);
    if (t.master != nullptr && t.param_dt == LLAMARL_F32)
      return fail(LLAMARL_ERR_INVALID_ARG, "tensor %lld: a master copy of fp32 parameters", (long long)i);
    if (!aligned_to(t.param, esize(t.param_dt)) || !aligned_to(t.grad, esize(t.grad_dt)) || !aligned_to(t.master, 4) ||
        !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4) || (t.m_scale == nullptr && (!aligned_to(t.m, 4) || !aligned_to(t.v, 4))))
      return fail(LLAMARL_ERR_INVALID_ARG, "tensor %lld: misaligned for its type", (long long)i);
    if (t.n > OPT_MAX_ENTRIES || (total += t.n) > OPT_MAX_ENTRIES)
      return fail(LLAMARL_ERR_UNSUPPORTED, "more than 2^34 entries");
  }
  return check_apart(tensors, count, grad_scale, lr_device, step_device);
}

}  // namespace

extern "C" {

size_t llamarl_grad_norm_workspace_bytes(int64_t count) {
  return count < 0 || count > (int64_t)1 << 24 ? 0 : (size_t)(NORM_BLOCKS + count) * sizeof(double);
}

llamarl_status llamarl_grad_norm(const llamarl_gradient* grads, int64_t count, float max_norm, float* norm, float* scale, void* ws,
                                 size_t ws_bytes, void* stream) {
  if (!norm || !scale || (grads == nullptr && count > 0)) return fail(LLAMARL_ERR_INVALID_ARG, "null pointer argument");
  if (count < 0 || count > (int64_t)1 << 24) return fail(LLAMARL_ERR_INVALID_ARG, "count must lie in [0, 2^24] (got %lld)", (long long)count);
  if (!(max_norm > 0.f)) return fail(LLAMARL_ERR_INVALID_ARG, "max_norm must be positive (got %g)", (double)max_norm);
  if (!aligned_to(norm, 4) || !aligned_to(scale, 4)) return fail(LLAMARL_ERR_INVALID_ARG, "misaligned norm or scale");
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (grads[i].n < 0) return fail(LLAMARL_ERR_INVALID_ARG, "gradient %lld has %lld entries", (long long)i, (long long)grads[i].n);
    if (grads[i].n == 0) continue;
    if (!known(grads[i].dt)) return fail(LLAMARL_ERR_INVALID_ARG, "gradient %lld: unknown dtype", (long long)i);
    if (!grads[i].grad) return fail(LLAMARL_ERR_INVALID_ARG, "gradient %lld: null pointer", (long long)i);
    if (!aligned_to(grads[i].grad, esize(grads[i].dt))) return fail(LLAMARL_ERR_INVALID_ARG, "gradient %lld: misaligned for its type", (long long)i);
    if (grads[i].n > OPT_MAX_ENTRIES || (total += grads[i].n) > OPT_MAX_ENTRIES)
      return fail(LLAMARL_ERR_UNSUPPORTED, "more than 2^34 entries");
  }
  const size_t need = llamarl_grad_norm_workspace_bytes(count);
  if (!ws || ws_bytes < need)
    return fail(LLAMARL_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", ws ? ws_bytes : (size_t)0, need);
  if (!aligned16(ws)) return fail(LLAMARL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (any_overlap({{norm, 4}, {scale, 4}, {ws, (int64_t)need}}, {})) return fail(LLAMARL_ERR_INVALID_ARG, "norm, scale and workspace must not overlap");
  for (int64_t i = 0; i < count; ++i) {
    const Span g = {grads[i].n > 0 ? grads[i].grad : nullptr, grads[i].n > 0 ? grads[i].n * (int64_t)esize(grads[i].dt) : 0};
    if (any_overlap({g}, {{norm, 4}, {scale, 4}, {ws, (int64_t)need}}))
      return fail(LLAMARL_ERR_INVALID_ARG, "norm, scale or workspace lies in gradient %lld", (long long)i);
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  double* part = reinterpret_cast<double*>(ws);
  // Whole units of at least total / NORM_BLOCKS, in turns of NORM_LOADS: at most NORM_BLOCKS workgroups, and one more for each tensor's end.  4096 /
  // 8192 / 16384 / 32768 of them: 170 M model in bf16 69 / 69 / 67 / 88 us, fp32 130 / 127 / 127 / 124; 525 M entries in fp32 360 / 349 / 352 / 372.
  int units = (int)std::max<int64_t>((total + (int64_t)NORM_BLOCKS * OPT_UNIT - 1) / ((int64_t)NORM_BLOCKS * OPT_UNIT), 1);
  if (units > 2) units = (units + NORM_LOADS - 1) / NORM_LOADS * NORM_LOADS;
  OptList l;
  int64_t done = 0;
  const llamarl_status s = for_each_launch(
      count, units, l,
      [&](int64_t i, OptTensor& t) {
        t.g = grads[i].grad;
        t.n = grads[i].n;
        t.flags = (grads[i].dt == LLAMARL_BF16 ? OPT_G_BF16 : 0) | (aligned16(t.g) ? OPT_WIDE : 0);
      },
      [&](const OptList& list, unsigned blocks) -> llamarl_status {
        k_grad_squares<<<dim3(blocks), dim3(OPT_THREADS), 0, st>>>(list, part + done);
        HIP_TRY(hipGetLastError());
        done += blocks;
        return LLAMARL_OK;
      });
  if (s != LLAMARL_OK) return s;
  k_grad_norm<<<dim3(1), dim3(NORM_THREADS), 0, st>>>(part, done, max_norm, norm, scale);
  HIP_TRY(hipGetLastError());
  return LLAMARL_OK;
}

llamarl_status llamarl_adamw_step(const llamarl_adamw_tensor* tensors, int64_t count, const llamarl_adamw_params* p,
                                  const float* grad_scale, const float* lr_device, const int64_t* step_device, void* stream) {
  int64_t total;
  llamarl_status s = check_adamw(tensors, count, p, grad_scale, lr_device, step_device, total);
  if (s != LLAMARL_OK) return s;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  AdamwArgs a;
  a.lr = (float)p->lr;
  a.b1 = (float)p->beta1;
  a.one_b1 = (float)(1.0 - p->beta1);
  a.b2 = (float)p->beta2;
  a.one_b2 = (float)(1.0 - p->beta2);
  a.eps = (float)p->eps;
  a.decay = (float)p->weight_decay;
  a.beta1 = p->beta1;
  a.beta2 = p->beta2;
  a.step = p->step;
  a.inv_c1 = step_device ? 1.f : (float)(1.0 / (1.0 - std::pow(p->beta1, (double)p->step)));
  a.inv_sqrt_c2 = step_device ? 1.f : (float)(1.0 / std::sqrt(1.0 - std::pow(p->beta2, (double)p->step)));
  a.scale = grad_scale;
  a.lr_device = lr_device;
  a.step_device = step_device;
  // One unit a workgroup: with more the chip's last round is longer.  Measured with units of 2048 entries (256 threads), 1 / 2 / 4 / 8 / 16 a workgroup:
  // 8B head, 32 bits 3.29 / 3.34 / 3.38 / 3.43 / 3.50 ms, 8 bits 1.56 / 1.60 / 1.64 / 1.67 / 1.70, 109 tensors of a 170 M model 983 / 1022 / 1047 / 1083 /
  // 1126 us.
  return for_each_launch(
      count, 1, a.l,
      [&](int64_t i, OptTensor& t) {
        const llamarl_adamw_tensor& c = tensors[i];
        t.p = c.param;
        t.master = c.master;
        t.g = c.grad;
        t.m = c.m;
        t.v = c.v;
        t.m_scale = c.m_scale;
        t.v_scale = c.v_scale;
        t.n = c.n;
        t.place = (uint32_t)i;
        t.flags = (c.param_dt == LLAMARL_BF16 ? OPT_P_BF16 : 0) | (c.grad_dt == LLAMARL_BF16 ? OPT_G_BF16 : 0) |
                  (c.m_scale != nullptr ? OPT_8BIT : 0) |
                  (aligned16(c.param) && aligned16(c.master) && aligned16(c.grad) && aligned16(c.m) && aligned16(c.v) ? OPT_WIDE : 0);
      },
      [&](const OptList&, unsigned blocks) -> llamarl_status {
        k_adamw<<<dim3(blocks), dim3(OPT_THREADS), 0, st>>>(a);
        HIP_TRY(hipGetLastError());
        return LLAMARL_OK;
      });
}

}  // extern "C"
