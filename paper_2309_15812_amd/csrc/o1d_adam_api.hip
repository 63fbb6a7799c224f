// C ABI of the AdamW step (declared in include/o1d.h).
#include <algorithm>
#include <new>
#include <vector>

#include "o1d_adam.h"
#include "o1d_rows_check.h"

namespace {

o1d_status_t check_rate(const char* fn, const char* what, double v, bool below_one) {
  if (!(v >= 0.) || isinf(v) || (below_one && v >= 1.))
    return fail(O1D_ERR_INVALID, "%s: %s=%g is out of range", fn, what, v);
  return O1D_OK;
}

}  // namespace

extern "C" {

size_t o1d_adamw_workspace_bytes(double max_norm) { return max_norm > 0. ? rows::kNormBlocks * sizeof(double) : kNoSpace; }

o1d_status_t o1d_adamw(const o1d_adamw_tensor_t* tensors, int count, o1d_dtype_t param_dtype, o1d_dtype_t grad_dtype,
                       const o1d_adamw_state_t* state, const o1d_adamw_options_t* options, float* norm, void* workspace,
                       size_t workspace_bytes, void* stream) {
  const char* fn = "o1d_adamw";
  for (o1d_dtype_t dt : {param_dtype, grad_dtype})
    if (dt != O1D_F32 && dt != O1D_BF16) return fail(O1D_ERR_INVALID, "%s: unknown dtype %d", fn, (int)dt);
  if (count < 0) return fail(O1D_ERR_INVALID, "%s: negative count %d", fn, count);
  if (!state || !options || (count && !tensors)) return fail(O1D_ERR_INVALID, "%s: NULL argument", fn);
  const o1d_adamw_state_t& S = *state;
  const o1d_adamw_options_t& H = *options;
  O1D_TRY(check_rate(fn, "lr", H.lr, false));
  O1D_TRY(check_rate(fn, "beta1", H.beta1, true));
  O1D_TRY(check_rate(fn, "beta2", H.beta2, true));
  O1D_TRY(check_rate(fn, "eps", H.eps, false));
  O1D_TRY(check_rate(fn, "weight_decay", H.weight_decay, false));
  O1D_TRY(check_rate(fn, "max_norm", H.max_norm, false));
  if (S.bits != 8 && S.bits != 32) return fail(O1D_ERR_INVALID, "%s: states have 8 or 32 bits, not %d", fn, S.bits);
  const bool clip = H.max_norm > 0.;
  O1D_TRY(check_null(fn, {S.step}));
  if (clip) O1D_TRY(check_null(fn, {norm}));
  for (const void* p : {(const void*)S.step, (const void*)norm, (const void*)H.lr_at})
    O1D_TRY(check_elem_aligned(fn, p, "a scalar", 4));
  O1D_TRY(check_workspace(fn, clip ? workspace : nullptr, workspace_bytes, clip ? o1d_adamw_workspace_bytes(H.max_norm) : 0));
  // The tensors with values; what a call reads and writes lies apart
  struct Piece {
    uintptr_t from, to;
    bool out;
  };
  const size_t ps = elem_size(param_dtype), gs = elem_size(grad_dtype), ss = S.bits == 8 ? 1 : 4;
  std::vector<rows::AdamTensor> list;
  std::vector<Piece> pieces, parts;
  try {
    list.reserve((size_t)count);
    pieces.reserve(2 * (size_t)count + 8);
    parts.reserve((size_t)count);
    long long end = 0;
    auto add = [&](const void* p, size_t bytes, bool out) {
      if (p && bytes) pieces.push_back({(uintptr_t)p, (uintptr_t)p + bytes, out});
    };
    for (int i = 0; i < count; ++i) {
      const o1d_adamw_tensor_t& t = tensors[i];
      if (t.n < 0 || t.at < 0) return fail(O1D_ERR_INVALID, "%s: tensor %d has a negative size or place", fn, i);
      if (t.n == 0) continue;
      if (t.n > (1ll << 37) || t.at > (1ll << 37)) return fail(O1D_ERR_UNSUPPORTED, "%s: tensor %d exceeds 2^37 values", fn, i);
      if (t.at % rows::kAdamGroup)
        return fail(O1D_ERR_INVALID, "%s: tensor %d's states start at %lld, no multiple of %d", fn, i, t.at, rows::kAdamGroup);
      O1D_TRY(check_null(fn, {t.p, t.g}));
      O1D_TRY(check_elem_aligned(fn, t.p, "a parameter", ps));
      O1D_TRY(check_elem_aligned(fn, t.g, "a gradient", gs));
      const long long to = t.at + rows::cdiv(t.n, rows::kAdamGroup) * rows::kAdamGroup;
      end = to > end ? to : end;
      add(t.p, (size_t)t.n * ps, true);
      add(t.g, (size_t)t.n * gs, false);
      parts.push_back({(uintptr_t)t.at, (uintptr_t)to, true});
      list.push_back({t.p, t.g, t.n, t.at});
    }
    if (!list.empty()) {
      O1D_TRY(check_null(fn, {S.m, S.v}));
      if (S.bits == 8) O1D_TRY(check_null(fn, {S.m_scale, S.v_scale}));
      for (const void* p : {(const void*)S.m, (const void*)S.v, (const void*)S.m_scale, (const void*)S.v_scale,
                            (const void*)S.master})
        O1D_TRY(check_elem_aligned(fn, p, "a state", 16));
      const size_t n = (size_t)end;
      add(S.m, n * ss, true);
      add(S.v, n * ss, true);
      if (S.bits == 8) {
        add(S.m_scale, n / rows::kAdamGroup * 4, true);
        add(S.v_scale, n / rows::kAdamGroup * 4, true);
      }
      add(S.master, n * 4, true);
    }
    add(S.step, 8, true);
    add(H.lr_at, 4, false);
    if (clip) {
      add(norm, 4, true);
      add(workspace, o1d_adamw_workspace_bytes(H.max_norm), true);
    }
    // in order of their start, one that is written may not reach into the next (gradients may be shared)
    auto apart_all = [&](std::vector<Piece>& v) {
      std::sort(v.begin(), v.end(), [](const Piece& a, const Piece& b) { return a.from < b.from; });
      uintptr_t out_end = 0, any_end = 0;
      for (const Piece& p : v) {
        if (p.from < out_end || (p.out && p.from < any_end)) return false;
        if (p.out && p.to > out_end) out_end = p.to;
        if (p.to > any_end) any_end = p.to;
      }
      return true;
    };
    if (!apart_all(parts)) return fail(O1D_ERR_INVALID, "%s: two tensors' parts of the states overlap", fn);
    if (!apart_all(pieces)) return fail(O1D_ERR_INVALID, "%s: a tensor that is written overlaps another", fn);
  } catch (const std::bad_alloc&) {
    return fail(O1D_ERR_UNSUPPORTED, "%s: no host memory for %d tensors", fn, count);
  }
  (void)hipGetLastError();
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Dtype pdt = (Dtype)param_dtype, gdt = (Dtype)grad_dtype;
  if (list.empty()) return clip ? hip_status(fn, o1d::launch_zero(Dtype::F32, norm, 1, s)) : ok();
  if (clip)
    O1D_TRY(hip_status(fn, rows::launch_grad_norm(gdt, list.data(), (int)list.size(), static_cast<double*>(workspace), S.step + 1, norm, s)));
  const rows::AdamState st{S.m, S.v, S.m_scale, S.v_scale, S.master, S.step, S.bits};
  rows::AdamHyper h{};
  h.lr = (float)H.lr;
  h.beta1 = (float)H.beta1;
  h.beta2 = (float)H.beta2;
  h.eps = (float)H.eps;
  h.decay = (float)H.weight_decay;
  h.beta1_64 = H.beta1;
  h.beta2_64 = H.beta2;
  h.rest1 = (float)(1. - H.beta1);
  h.rest2 = (float)(1. - H.beta2);
  h.keep = (float)(1. - H.lr * H.weight_decay);
  h.lr_at = H.lr_at;
  h.norm = clip ? norm : nullptr;
  h.max_norm = (float)H.max_norm;
  h.follow = H.follow != 0;
  return hip_status(fn, rows::launch_adam(pdt, gdt, list.data(), (int)list.size(), st, h, s));
}

}  // extern "C"
