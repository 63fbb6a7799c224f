// C ABI of the row operators (declared in include/o1d.h): layer norm, the
// matrix product with an epilogue and its gradients, 8-bit checkpoints.
// Argument checks and dispatch; no device memory is allocated here.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdio.h>

#include <initializer_list>

#include "o1d.h"
#include "o1d_rows.h"
#include "o1d_status.h"

namespace {

using o1d::Dtype;
using o1d::elem_size;
using o1d::fail;
using o1d::ok;
using o1d::overlaps;
namespace rows = o1d::rows;

// Rows and features below 2^31 with room for a tile; row strides such that a
// tile's offsets stay below 2^31 bytes.
constexpr int kMaxRows = 0x7fffffff - 1024;
constexpr int kMaxFeatures = 1 << 20;
constexpr long long kMaxStride = 1 << 21;

// What a call that needs no workspace asks for all the same, so that callers need not know which do.  One that
// writes to its workspace asks for more, however little that is: callers may share
// a workspace of kNoSpace bytes between calls that run at the same time.
constexpr size_t kNoSpace = 256, kLeastSpace = 2 * kNoSpace;
size_t space_for(size_t bytes) { return bytes < kLeastSpace ? kLeastSpace : bytes; }

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// One tensor of a call: where it lies and how far it reaches.
struct Span {
  const char* what;
  const void* p;
  size_t bytes;
  bool out;
};

size_t reach(long long M, long long ld, long long C, size_t es) {
  return M > 0 && C > 0 ? ((size_t)(M - 1) * (size_t)ld + (size_t)C) * es : 0;
}
size_t held_q_bytes(int M, int C) { return (size_t)M * (size_t)rows::held_ld(C); }
size_t held_scale_bytes(int M, int C) { return (size_t)M * (size_t)rows::held_groups(C) * sizeof(float); }

// No output overlaps an input or another output.
template <int N>
o1d_status_t apart(const char* fn, const Span (&s)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < N; ++j)
      if (i != j && s[i].out && s[i].p && s[j].p && s[i].bytes && s[j].bytes &&
          overlaps(s[i].p, s[i].bytes, s[j].p, s[j].bytes))
        return fail(O1D_ERR_INVALID, "%s: %s overlaps %s", fn, s[i].what, s[j].what);
  return O1D_OK;
}

o1d_status_t check_dims(const char* fn, int M, int C, const char* feature, o1d_dtype_t dt) {
  if (dt != O1D_F32 && dt != O1D_BF16) return fail(O1D_ERR_INVALID, "%s: unknown dtype %d", fn, (int)dt);
  if (M < 0) return fail(O1D_ERR_INVALID, "%s: negative rows M=%d", fn, M);
  if (C < 1) return fail(O1D_ERR_INVALID, "%s: %s=%d must be positive", fn, feature, C);
  if (M > kMaxRows) return fail(O1D_ERR_UNSUPPORTED, "%s: M=%d rows exceed %d", fn, M, kMaxRows);
  if (C > kMaxFeatures) return fail(O1D_ERR_UNSUPPORTED, "%s: %s=%d exceeds %d", fn, feature, C, kMaxFeatures);
  return O1D_OK;
}

o1d_status_t check_ld(const char* fn, const char* what, long long ld, int C) {
  if (ld < C) return fail(O1D_ERR_INVALID, "%s: row stride %lld of %s is below its %d features", fn, ld, what, C);
  if (ld >= kMaxStride) return fail(O1D_ERR_UNSUPPORTED, "%s: row stride %lld of %s exceeds %lld", fn, ld, what, kMaxStride);
  return O1D_OK;
}

o1d_status_t check_act(const char* fn, o1d_act_t act) {
  return (int)act >= 0 && (int)act < rows::kActs ? O1D_OK
                                                 : fail(O1D_ERR_INVALID, "%s: unknown activation %d", fn, (int)act);
}

// The integers are accessed eight at a time.
o1d_status_t check_held(const char* fn, const signed char* q, const float* scale) {
  if (!q || !scale) return fail(O1D_ERR_INVALID, "%s: a checkpoint needs its integers and its scales", fn);
  if ((uintptr_t)q % 16) return fail(O1D_ERR_INVALID, "%s: a checkpoint's integers must be 16-byte aligned", fn);
  return O1D_OK;
}

// A tensor (p) or a checkpoint (q), one of the two.
o1d_status_t check_either(const char* fn, const char* what, const void* p, long long ld, int C, const signed char* q,
                          const float* scale) {
  if (!p == !q) return fail(O1D_ERR_INVALID, "%s: %s is given as a tensor or as a checkpoint, one of the two", fn, what);
  return p ? check_ld(fn, what, ld, C) : check_held(fn, q, scale);
}

o1d_status_t check_elem_aligned(const char* fn, const void* p, const char* what, size_t es) {
  return (uintptr_t)p % es ? fail(O1D_ERR_INVALID, "%s: %s is not aligned to its elements", fn, what) : O1D_OK;
}

o1d_status_t hip_status(const char* fn, hipError_t e) {
  if (e != hipSuccess) return fail(O1D_ERR_HIP, "%s: kernel launch failed: %s", fn, hipGetErrorString(e));
  return ok();
}

#define O1D_TRY(expr)                         \
  do {                                        \
    const o1d_status_t st_ = (expr);          \
    if (st_ != O1D_OK) return st_;            \
  } while (0)

o1d_status_t check_null(const char* fn, std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!p) return fail(O1D_ERR_INVALID, "%s: NULL tensor pointer", fn);
  return O1D_OK;
}

o1d_status_t check_workspace(const char* fn, const void* workspace, size_t bytes, size_t need) {
  if (need && (bytes < need || !workspace))
    return fail(O1D_ERR_WORKSPACE, "%s: workspace of %zu bytes given, %zu needed", fn, bytes, need);
  if ((uintptr_t)workspace % 16) return fail(O1D_ERR_INVALID, "%s: workspace must be 16-byte aligned", fn);
  return O1D_OK;
}

o1d_status_t check_blocks(const char* fn, const rows::MmPlan& pl) {
  const long long blocks = (long long)pl.p.tm * pl.p.tn * pl.p.nsplit;
  return blocks > (1 << 24) - 8 ? fail(O1D_ERR_UNSUPPORTED, "%s: %lld workgroups exceed the grid", fn, blocks) : O1D_OK;
}

// The weight gradient's workspace: the partial results, then (where x is a
// checkpoint or has an activation) the product's operand act(x).
struct WgradSpace {
  rows::MmPlan plan;
  size_t part, operand;
  bool made;      // act(x) is made by the product
  long long ldx;  // of the operand
  size_t bytes() const { return part + operand; }
};

WgradSpace wgrad_space(int M, int I, int O, o1d_act_t act, bool held, o1d_dtype_t dt) {
  WgradSpace s;
  const bool rewritten = held || act != O1D_ACT_NONE;
  const int es = (int)elem_size(dt), run = 16 / es;
  s.plan = rows::plan_wgrad(O, I, M, es, held, (int)act, s.made);
  s.part = s.plan.p.nsplit > 1 ? space_for(round256((size_t)s.plan.p.nsplit * ((size_t)O * I + O) * sizeof(float)))
                               : kNoSpace;
  s.ldx = rows::cdiv(I, run) * run;
  s.operand = rewritten && !s.made ? round256((size_t)M * s.ldx * es) : 0;
  return s;
}

// ---- names

thread_local char g_name[128] = "";

const char* dt_name(o1d_dtype_t dt) { return dt == O1D_BF16 ? "bf16" : "f32"; }

// The product's launch, as launch_mm and the kernels' own launchers choose it.
void name_mm(char* out, size_t n, int kind, const rows::MmPlan& pl, o1d_dtype_t dt, bool whole, bool held) {
  const char *op = kind == rows::kFwd ? "fwd" : (kind == rows::kDgrad ? "dgrad" : "wgrad"), *d = dt_name(dt);
  const rows::Shape& s = rows::kShapes[pl.shape];
  const int bm = 32 * s.tm * s.wm, bn = 32 * s.tn * s.wn;
  if (pl.few)
    snprintf(out, n, "few/%s/%s/%d%s", op, d, pl.p.M <= 16 ? 16 : (pl.p.M <= 32 ? 32 : 64), held ? "/held" : "");
  else if (dt == O1D_BF16 && !pl.p.made && whole)
    snprintf(out, n, "mmf/%s/%s/%dx%d", op, d, bm, bn);
  else
    snprintf(out, n, "mm/%s/%s/%dx%d%s", op, d, bm, bn, pl.p.made ? "/made" : "");
}

}  // namespace

extern "C" {

const char* o1d_rows_kernel_name(int op, int M, int I, int O, o1d_act_t act, int held, o1d_dtype_t dtype, int aligned) {
  const char* fn = "o1d_rows_kernel_name";
  g_name[0] = '\0';
  if (op < 0 || op > 4 || check_dims(fn, M, I, "I", dtype) != O1D_OK || M == 0) return g_name;
  const int es = (int)elem_size(dtype);
  if (op >= 3) {
    const rows::LnMap m = op == 3 ? rows::ln_fwd_map(I, es) : rows::ln_bwd_map(I, es);
    char size[32] = "wide";
    if (m.lanes) snprintf(size, sizeof(size), "%dx%d", m.lanes, m.runs);
    if (op == 3)
      snprintf(g_name, sizeof(g_name), "ln_fwd/%s/%s", dt_name(dtype), size);
    else
      snprintf(g_name, sizeof(g_name), "ln_bwd/%s/%s%s%s", dt_name(dtype), size, held ? "/held" : "",
               rows::ln_bwd_blocks(M, I, es) > 1 ? "+col_sum" : "");
    return g_name;
  }
  if (check_dims(fn, M, O, "O", dtype) != O1D_OK || check_act(fn, act) != O1D_OK) return g_name;
  const auto whole = [&](int kind, int m, int n, int k) {
    return aligned && rows::whole_runs(kind, m, n, k, nullptr, 0, nullptr, 0, es);
  };
  if (op < 2) {
    const int kind = op == 0 ? rows::kFwd : rows::kDgrad, n = op == 0 ? O : I, k = op == 0 ? I : O;
    const bool w = whole(kind, M, n, k), writes = op == 0 && held;
    name_mm(g_name, sizeof(g_name), kind, rows::plan_mm(kind, M, n, k, es, writes, w), dtype, w, writes);
    return g_name;
  }
  WgradSpace s = wgrad_space(M, I, O, act, held != 0, dtype);
  s.plan.p.made = s.made;
  // (an operand from a pass of its own has whole rows)
  char mm[64];
  name_mm(mm, sizeof(mm), rows::kWgrad, s.plan, dtype, whole(rows::kWgrad, O, I, M), false);
  const int parts = s.plan.p.nsplit;
  snprintf(g_name, sizeof(g_name), "%s%s%s", s.operand ? "act+" : "", mm,
           parts == 1 ? "" : (rows::wide_sum(parts, (long long)O * I + O) ? "+mm_sum_wide" : "+mm_sum"));
  return g_name;
}

o1d_status_t o1d_ln_fwd(const void* x, long long ldx, const void* w, const void* b, void* y, long long ldy, float* mean,
                        float* rstd, int M, int C, float eps, o1d_dtype_t dtype, void* stream) {
  const char* fn = "o1d_ln_fwd";
  O1D_TRY(check_dims(fn, M, C, "C", dtype));
  O1D_TRY(check_ld(fn, "x", ldx, C));
  O1D_TRY(check_ld(fn, "y", ldy, C));
  if (!(eps >= 0.f) || isinf(eps)) return fail(O1D_ERR_INVALID, "%s: eps must be finite and not negative", fn);
  if (M == 0) return ok();
  O1D_TRY(check_null(fn, {x, w, b, y}));
  if (!mean != !rstd) return fail(O1D_ERR_INVALID, "%s: mean and rstd are given together or not at all", fn);
  const size_t es = elem_size(dtype);
  for (const void* p : {x, w, b, (const void*)y}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  const Span spans[] = {{"x", x, reach(M, ldx, C, es), false}, {"w", w, C * es, false}, {"b", b, C * es, false},
                        {"y", y, reach(M, ldy, C, es), true}, {"mean", mean, M * sizeof(float), true},
                        {"rstd", rstd, M * sizeof(float), true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  rows::LnParams p{};
  p.M = M;
  p.C = C;
  p.ldx = ldx;
  p.ldy = ldy;
  p.eps = eps;
  p.x = x;
  p.w = w;
  p.b = b;
  p.y = y;
  p.mean = mean;
  p.rstd = rstd;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(fn, dtype == O1D_F32 ? rows::launch_ln_fwd_f32(p, s) : rows::launch_ln_fwd_bf16(p, s));
}

size_t o1d_ln_bwd_workspace_bytes(int M, int C, o1d_dtype_t dtype) {
  if (check_dims("o1d_ln_bwd", M, C, "C", dtype) != O1D_OK || M == 0) return 0;
  const int blocks = rows::ln_bwd_blocks(M, C, (int)elem_size(dtype));
  return blocks > 1 ? space_for((size_t)blocks * 2 * C * sizeof(float)) : kNoSpace;
}

o1d_status_t o1d_ln_bwd(const void* x, long long ldx, const signed char* xq, const float* xscale, const void* dy,
                        long long lddy, const float* mean, const float* rstd, const void* w, void* dx, long long lddx,
                        void* dw, void* db, int M, int C, o1d_dtype_t dtype, void* workspace, size_t workspace_bytes,
                        void* stream) {
  const char* fn = "o1d_ln_bwd";
  O1D_TRY(check_dims(fn, M, C, "C", dtype));
  if (M > 0) O1D_TRY(check_either(fn, "x", x, ldx, C, xq, xscale));
  O1D_TRY(check_ld(fn, "dy", lddy, C));
  O1D_TRY(check_ld(fn, "dx", lddx, C));
  O1D_TRY(check_null(fn, {dw, db}));
  const size_t es = elem_size(dtype), need = o1d_ln_bwd_workspace_bytes(M, C, dtype);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (M > 0) O1D_TRY(check_null(fn, {dy, mean, rstd, w, dx}));
  O1D_TRY(check_workspace(fn, workspace, workspace_bytes, need));
  for (const void* p : {x, dy, w, (const void*)dx, (const void*)dw, (const void*)db})
    O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  const Span spans[] = {{"x", x, reach(M, ldx, C, es), false}, {"the checkpoint", xq, held_q_bytes(M, C), false},
                        {"its scales", xscale, held_scale_bytes(M, C), false}, {"dy", dy, reach(M, lddy, C, es), false},
                        {"mean", mean, M * sizeof(float), false}, {"rstd", rstd, M * sizeof(float), false},
                        {"w", w, C * es, false}, {"dx", dx, reach(M, lddx, C, es), true}, {"dw", dw, C * es, true},
                        {"db", db, C * es, true}, {"the workspace", workspace, need, true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  if (M == 0) {
    O1D_TRY(hip_status(fn, o1d::launch_zero((Dtype)dtype, dw, C, s)));
    return hip_status(fn, o1d::launch_zero((Dtype)dtype, db, C, s));
  }
  rows::LnParams p{};
  p.M = M;
  p.C = C;
  p.ldx = ldx;
  p.ldy = lddy;
  p.lddx = lddx;
  p.x = x;
  p.xq = reinterpret_cast<const int8_t*>(xq);
  p.xscale = xscale;
  p.w = w;
  p.dy = dy;
  p.dx = dx;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.dw = dw;
  p.db = db;
  p.part = static_cast<float*>(workspace);
  p.blocks = rows::ln_bwd_blocks(M, C, (int)es);
  O1D_TRY(hip_status(fn, dtype == O1D_F32 ? rows::launch_ln_bwd_f32(p, s) : rows::launch_ln_bwd_bf16(p, s)));
  return p.blocks > 1 ? hip_status(fn, rows::launch_col_sum((Dtype)dtype, p.part, p.blocks, 2ll * C, C, dw, db, s)) : ok();
}

o1d_status_t o1d_linear_fwd(const void* x, long long ldx, const void* w, const void* b, o1d_act_t act, const void* res,
                            long long ldres, void* y, long long ldy, void* pre, long long ldpre, signed char* q,
                            float* scale, int M, int I, int O, o1d_dtype_t dtype, void* stream) {
  const char* fn = "o1d_linear_fwd";
  O1D_TRY(check_dims(fn, M, I, "I", dtype));
  O1D_TRY(check_dims(fn, M, O, "O", dtype));
  O1D_TRY(check_act(fn, act));
  O1D_TRY(check_ld(fn, "x", ldx, I));
  O1D_TRY(check_ld(fn, "y", ldy, O));
  if (res) O1D_TRY(check_ld(fn, "the residual", ldres, O));
  if (pre) O1D_TRY(check_ld(fn, "pre", ldpre, O));
  if (q || scale) O1D_TRY(check_held(fn, q, scale));
  if (M == 0) return ok();
  O1D_TRY(check_null(fn, {x, w, y}));
  const size_t es = elem_size(dtype);
  for (const void* p : {x, w, b, res, (const void*)y, (const void*)pre}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  const Span spans[] = {{"x", x, reach(M, ldx, I, es), false}, {"w", w, (size_t)O * I * es, false}, {"b", b, O * es, false},
                        {"the residual", res, reach(M, ldres, O, es), false}, {"y", y, reach(M, ldy, O, es), true},
                        {"pre", pre, reach(M, ldpre, O, es), true}, {"the checkpoint", q, held_q_bytes(M, O), true},
                        {"its scales", scale, held_scale_bytes(M, O), true}};
  O1D_TRY(apart(fn, spans));
  rows::MmPlan pl = rows::plan_mm(rows::kFwd, M, O, I, (int)es, q != nullptr,
                                  rows::whole_runs(rows::kFwd, M, O, I, x, ldx, w, I, (int)es));
  O1D_TRY(check_blocks(fn, pl));
  (void)hipGetLastError();
  rows::MmParams& p = pl.p;
  p.a = x;
  p.lda = ldx;
  p.b = w;
  p.ldb = I;
  p.act = (int)act;
  p.bias = b;
  p.res = res;
  p.ldres = ldres;
  p.out = y;
  p.ldo = ldy;
  p.pre = pre;
  p.ldpre = ldpre;
  p.q = reinterpret_cast<int8_t*>(q);
  p.scale = scale;
  p.ldq = rows::held_ld(O);
  p.groups = rows::held_groups(O);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(fn, rows::launch_mm((Dtype)dtype, rows::kFwd, pl, s));
}

o1d_status_t o1d_linear_bwd_input(const void* dy, long long lddy, const void* w, o1d_act_t act, const void* pre,
                                  long long ldpre, const signed char* preq, const float* prescale, void* dx,
                                  long long lddx, int M, int I, int O, o1d_dtype_t dtype, void* stream) {
  const char* fn = "o1d_linear_bwd_input";
  O1D_TRY(check_dims(fn, M, I, "I", dtype));
  O1D_TRY(check_dims(fn, M, O, "O", dtype));
  O1D_TRY(check_act(fn, act));
  O1D_TRY(check_ld(fn, "dy", lddy, O));
  O1D_TRY(check_ld(fn, "dx", lddx, I));
  if (M > 0 && act != O1D_ACT_NONE) O1D_TRY(check_either(fn, "pre", pre, ldpre, I, preq, prescale));
  if (M == 0) return ok();
  O1D_TRY(check_null(fn, {dy, w, dx}));
  const size_t es = elem_size(dtype);
  for (const void* p : {dy, w, pre, (const void*)dx}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  const bool held = act != O1D_ACT_NONE && preq;
  const Span spans[] = {{"dy", dy, reach(M, lddy, O, es), false}, {"w", w, (size_t)O * I * es, false},
                        {"pre", act != O1D_ACT_NONE ? pre : nullptr, reach(M, ldpre, I, es), false},
                        {"the checkpoint", held ? preq : nullptr, held_q_bytes(M, I), false},
                        {"its scales", held ? prescale : nullptr, held_scale_bytes(M, I), false},
                        {"dx", dx, reach(M, lddx, I, es), true}};
  O1D_TRY(apart(fn, spans));
  rows::MmPlan pl = rows::plan_mm(rows::kDgrad, M, I, O, (int)es, false,
                                  rows::whole_runs(rows::kDgrad, M, I, O, dy, lddy, w, I, (int)es));
  O1D_TRY(check_blocks(fn, pl));
  (void)hipGetLastError();
  rows::MmParams& p = pl.p;
  p.a = dy;
  p.lda = lddy;
  p.b = w;
  p.ldb = I;
  p.act = (int)act;
  p.out = dx;
  p.ldo = lddx;
  p.pre = const_cast<void*>(pre);
  p.ldpre = ldpre;
  p.q = held ? reinterpret_cast<int8_t*>(const_cast<signed char*>(preq)) : nullptr;
  p.scale = const_cast<float*>(prescale);
  p.ldq = rows::held_ld(I);
  p.groups = rows::held_groups(I);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(fn, rows::launch_mm((Dtype)dtype, rows::kDgrad, pl, s));
}

size_t o1d_linear_bwd_weight_workspace_bytes(int M, int I, int O, o1d_act_t act, int held, o1d_dtype_t dtype) {
  const char* fn = "o1d_linear_bwd_weight";
  if (check_dims(fn, M, I, "I", dtype) != O1D_OK || check_dims(fn, M, O, "O", dtype) != O1D_OK || M == 0) return 0;
  return check_act(fn, act) == O1D_OK ? wgrad_space(M, I, O, act, held != 0, dtype).bytes() : 0;
}

o1d_status_t o1d_linear_bwd_weight(const void* x, long long ldx, const signed char* xq, const float* xscale, o1d_act_t act,
                                   const void* dy, long long lddy, void* dw, void* db, int M, int I, int O,
                                   o1d_dtype_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "o1d_linear_bwd_weight";
  O1D_TRY(check_dims(fn, M, I, "I", dtype));
  O1D_TRY(check_dims(fn, M, O, "O", dtype));
  O1D_TRY(check_act(fn, act));
  if (M > 0) O1D_TRY(check_either(fn, "x", x, ldx, I, xq, xscale));
  O1D_TRY(check_ld(fn, "dy", lddy, O));
  O1D_TRY(check_null(fn, {dw}));
  const size_t es = elem_size(dtype);
  const bool rewritten = xq || act != O1D_ACT_NONE;
  if (M > 0) O1D_TRY(check_null(fn, {dy}));
  for (const void* p : {x, dy, (const void*)dw, (const void*)db}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  hipStream_t s = static_cast<hipStream_t>(stream);
  WgradSpace space{};
  if (M > 0) {
    space = wgrad_space(M, I, O, act, xq != nullptr, dtype);
    O1D_TRY(check_blocks(fn, space.plan));
  }
  const size_t need = M > 0 ? space.bytes() : 0;
  O1D_TRY(check_workspace(fn, workspace, workspace_bytes, need));
  const Span spans[] = {{"x", x, reach(M, ldx, I, es), false}, {"the checkpoint", xq, held_q_bytes(M, I), false},
                        {"its scales", xscale, held_scale_bytes(M, I), false}, {"dy", dy, reach(M, lddy, O, es), false},
                        {"dw", dw, (size_t)O * I * es, true}, {"db", db, O * es, true},
                        {"the workspace", workspace, need, true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  if (M == 0) {
    O1D_TRY(hip_status(fn, o1d::launch_zero((Dtype)dtype, dw, (size_t)O * I, s)));
    return db ? hip_status(fn, o1d::launch_zero((Dtype)dtype, db, O, s)) : ok();
  }
  rows::MmParams& p = space.plan.p;
  p.a = dy;
  p.lda = lddy;
  p.b = x;
  p.ldb = ldx;
  p.part = static_cast<float*>(workspace);
  p.out = dw;
  p.db = db;
  p.want_db = db != nullptr;
  if (space.made) {
    p.made = 1;
    p.act = (int)act;
    p.bq = reinterpret_cast<const int8_t*>(xq);
    p.scale = const_cast<float*>(xscale);
    p.ldq = rows::held_ld(I);
    p.groups = rows::held_groups(I);
  } else if (rewritten) {
    void* operand = static_cast<char*>(workspace) + space.part;
    const rows::Operand in{x, ldx, reinterpret_cast<const int8_t*>(xq), xscale};
    O1D_TRY(hip_status(fn, rows::launch_act((Dtype)dtype, in, nullptr, 0, M, I, (int)act, operand, space.ldx, s)));
    p.b = operand;
    p.ldb = space.ldx;
  }
  O1D_TRY(hip_status(fn, rows::launch_mm((Dtype)dtype, rows::kWgrad, space.plan, s)));
  return p.nsplit > 1 ? hip_status(fn, rows::launch_mm_sum((Dtype)dtype, space.plan, dw, db, s)) : ok();
}

o1d_status_t o1d_act_bwd(const void* pre, long long ldpre, const signed char* preq, const float* prescale, o1d_act_t act,
                         const void* dy, long long lddy, void* dh, long long lddh, int M, int C, o1d_dtype_t dtype,
                         void* stream) {
  const char* fn = "o1d_act_bwd";
  O1D_TRY(check_dims(fn, M, C, "C", dtype));
  O1D_TRY(check_act(fn, act));
  if (M > 0) O1D_TRY(check_either(fn, "pre", pre, ldpre, C, preq, prescale));
  O1D_TRY(check_ld(fn, "dy", lddy, C));
  O1D_TRY(check_ld(fn, "dh", lddh, C));
  if (M == 0) return ok();
  O1D_TRY(check_null(fn, {dy, dh}));
  const size_t es = elem_size(dtype);
  for (const void* p : {pre, dy, (const void*)dh}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  const Span spans[] = {{"pre", pre, reach(M, ldpre, C, es), false}, {"the checkpoint", preq, held_q_bytes(M, C), false},
                        {"its scales", prescale, held_scale_bytes(M, C), false}, {"dy", dy, reach(M, lddy, C, es), false},
                        {"dh", dh, reach(M, lddh, C, es), true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  const rows::Operand in{pre, ldpre, reinterpret_cast<const int8_t*>(preq), prescale};
  return hip_status(fn, rows::launch_act((Dtype)dtype, in, dy, lddy, M, C, (int)act, dh, lddh,
                                         static_cast<hipStream_t>(stream)));
}

o1d_status_t o1d_pack(const void* x, long long ldx, signed char* q, float* scale, int M, int C, o1d_dtype_t dtype,
                      void* stream) {
  const char* fn = "o1d_pack";
  O1D_TRY(check_dims(fn, M, C, "C", dtype));
  O1D_TRY(check_ld(fn, "x", ldx, C));
  if (M == 0) return ok();
  O1D_TRY(check_null(fn, {x}));
  O1D_TRY(check_held(fn, q, scale));
  O1D_TRY(check_elem_aligned(fn, x, "x", elem_size(dtype)));
  const Span spans[] = {{"x", x, reach(M, ldx, C, elem_size(dtype)), false}, {"the checkpoint", q, held_q_bytes(M, C), true},
                        {"its scales", scale, held_scale_bytes(M, C), true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  return hip_status(fn, rows::launch_pack((Dtype)dtype, x, ldx, M, C, {reinterpret_cast<int8_t*>(q), scale},
                                          static_cast<hipStream_t>(stream)));
}

o1d_status_t o1d_unpack(const signed char* q, const float* scale, o1d_act_t act, void* y, long long ldy, int M, int C,
                        o1d_dtype_t dtype, void* stream) {
  const char* fn = "o1d_unpack";
  O1D_TRY(check_dims(fn, M, C, "C", dtype));
  O1D_TRY(check_act(fn, act));
  O1D_TRY(check_ld(fn, "y", ldy, C));
  if (M == 0) return ok();
  O1D_TRY(check_null(fn, {y}));
  O1D_TRY(check_held(fn, q, scale));
  O1D_TRY(check_elem_aligned(fn, y, "y", elem_size(dtype)));
  const Span spans[] = {{"the checkpoint", q, held_q_bytes(M, C), false}, {"its scales", scale, held_scale_bytes(M, C), false},
                        {"y", y, reach(M, ldy, C, elem_size(dtype)), true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  const rows::Operand in{nullptr, 0, reinterpret_cast<const int8_t*>(q), scale};
  return hip_status(fn, rows::launch_act((Dtype)dtype, in, nullptr, 0, M, C, (int)act, y, ldy,
                                         static_cast<hipStream_t>(stream)));
}

}  // extern "C"
