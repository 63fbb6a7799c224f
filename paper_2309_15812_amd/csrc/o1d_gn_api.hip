// C ABI of group norm (declared in include/o1d.h).
#include "o1d_gn.h"
#include "o1d_rows_check.h"

namespace {

o1d_status_t check_gn(const char* fn, int N, int P, int C, int groups, o1d_dtype_t dt) {
  if (N < 0 || P < 0) return fail(O1D_ERR_INVALID, "%s: negative size N=%d P=%d", fn, N, P);
  if (N > 0 && P < 1) return fail(O1D_ERR_INVALID, "%s: a sample has at least one pixel", fn);
  const long long M = (long long)N * P;
  O1D_TRY(check_dims(fn, M > kMaxRows ? kMaxRows : (int)M, C, "C", dt));
  if (M > kMaxRows) return fail(O1D_ERR_UNSUPPORTED, "%s: %lld rows exceed %d", fn, M, kMaxRows);
  if (groups < 1 || C % groups) return fail(O1D_ERR_INVALID, "%s: groups=%d do not divide C=%d", fn, groups, C);
  if (C / groups > rows::kGnMostChannels)
    return fail(O1D_ERR_UNSUPPORTED, "%s: a group of %d channels exceeds %d", fn, C / groups, rows::kGnMostChannels);
  return O1D_OK;
}

o1d_status_t check_pieces(const char* fn, const rows::GnPlan& pl, int N) {
  const long long n = (pl.held ? rows::cdiv(N, 8) * 8 : (long long)N * pl.chunks) * pl.bundles;
  // (a grid has fewer than 2^32 threads)
  return n * (pl.held ? pl.threads : 256) > 0xffffffffll ? fail(O1D_ERR_UNSUPPORTED, "%s: %lld workgroups exceed the grid", fn, n) : O1D_OK;
}

rows::GnParams gn_params(const rows::GnPlan& pl, int N, int P, int C, int groups, o1d_act_t act) {
  rows::GnParams p{};
  p.N = N;
  p.P = P;
  p.C = C;
  p.G = groups;
  p.D = C / groups;
  p.over_d = p.D > 1 ? (uint32_t)(((1ull << 32) + p.D - 1) / p.D) : 0;
  p.act = (int)act;
  p.gb = pl.gb;
  p.bundles = pl.bundles;
  p.chunks = pl.chunks;
  p.rows = pl.rows;
  return p;
}

}  // namespace

extern "C" {

size_t o1d_gn_fwd_workspace_bytes(int N, int P, int C, int groups, o1d_dtype_t dtype) {
  if (check_gn("o1d_gn_fwd", N, P, C, groups, dtype) != O1D_OK || N == 0) return 0;
  const long long n = rows::gn_fwd_floats(rows::plan_gn(false, N, P, C, groups, (int)elem_size(dtype)), N, groups);
  return n ? space_for((size_t)n * sizeof(float)) : kNoSpace;
}

o1d_status_t o1d_gn_fwd(const void* x, long long ldx, const void* w, const void* b, o1d_act_t act, void* y, long long ldy,
                        float* mean, float* rstd, int N, int P, int C, int groups, float eps, o1d_dtype_t dtype,
                        void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "o1d_gn_fwd";
  O1D_TRY(check_gn(fn, N, P, C, groups, dtype));
  O1D_TRY(check_act(fn, act));
  O1D_TRY(check_ld(fn, "x", ldx, C));
  O1D_TRY(check_ld(fn, "y", ldy, C));
  if (!(eps >= 0.f) || isinf(eps)) return fail(O1D_ERR_INVALID, "%s: eps must be finite and not negative", fn);
  if (N == 0) return ok();
  O1D_TRY(check_null(fn, {x, w, b, y, mean, rstd}));
  const size_t es = elem_size(dtype), need = o1d_gn_fwd_workspace_bytes(N, P, C, groups, dtype);
  const long long M = (long long)N * P;
  O1D_TRY(check_workspace(fn, workspace, workspace_bytes, need));
  for (const void* p : {x, w, b, (const void*)y}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  for (const void* p : {(const void*)mean, (const void*)rstd}) O1D_TRY(check_elem_aligned(fn, p, "a statistic", 4));
  const size_t stats = (size_t)N * groups * sizeof(float);
  const Span spans[] = {{"x", x, reach(M, ldx, C, es), false}, {"w", w, C * es, false}, {"b", b, C * es, false},
                        {"y", y, reach(M, ldy, C, es), true}, {"mean", mean, stats, true}, {"rstd", rstd, stats, true},
                        {"the workspace", workspace, need, true}};
  O1D_TRY(apart(fn, spans));
  const rows::GnPlan pl = rows::plan_gn(false, N, P, C, groups, (int)es);
  O1D_TRY(check_pieces(fn, pl, N));
  (void)hipGetLastError();
  rows::GnParams p = gn_params(pl, N, P, C, groups, act);
  p.ldx = ldx;
  p.ldy = ldy;
  p.eps = eps;
  p.x = x;
  p.w = w;
  p.b = b;
  p.out = y;
  p.mean = mean;
  p.rstd = rstd;
  p.part = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(fn, dtype == O1D_F32 ? rows::launch_gn_fwd_f32(pl, p, s) : rows::launch_gn_fwd_bf16(pl, p, s));
}

size_t o1d_gn_bwd_workspace_bytes(int N, int P, int C, int groups, o1d_dtype_t dtype) {
  if (check_gn("o1d_gn_bwd", N, P, C, groups, dtype) != O1D_OK || N == 0) return 0;
  return space_for((size_t)rows::gn_bwd_floats(rows::plan_gn(true, N, P, C, groups, (int)elem_size(dtype)), N, C, groups) *
                   sizeof(float));
}

o1d_status_t o1d_gn_bwd(const void* x, long long ldx, const void* dy, long long lddy, const float* mean, const float* rstd,
                        const void* w, const void* b, o1d_act_t act, void* dx, long long lddx, void* dw, void* db, int N,
                        int P, int C, int groups, o1d_dtype_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "o1d_gn_bwd";
  O1D_TRY(check_gn(fn, N, P, C, groups, dtype));
  O1D_TRY(check_act(fn, act));
  O1D_TRY(check_ld(fn, "x", ldx, C));
  O1D_TRY(check_ld(fn, "dy", lddy, C));
  O1D_TRY(check_ld(fn, "dx", lddx, C));
  O1D_TRY(check_null(fn, {dw, db}));
  const size_t es = elem_size(dtype), need = o1d_gn_bwd_workspace_bytes(N, P, C, groups, dtype);
  const long long M = (long long)N * P;
  if (N > 0) O1D_TRY(check_null(fn, {x, dy, mean, rstd, w, b, dx}));
  O1D_TRY(check_workspace(fn, workspace, workspace_bytes, need));
  for (const void* p : {x, dy, w, b, (const void*)dx, (const void*)dw, (const void*)db})
    O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  for (const void* p : {(const void*)mean, (const void*)rstd}) O1D_TRY(check_elem_aligned(fn, p, "a statistic", 4));
  const size_t stats = (size_t)N * groups * sizeof(float);
  const Span spans[] = {{"x", x, reach(M, ldx, C, es), false}, {"dy", dy, reach(M, lddy, C, es), false},
                        {"mean", mean, stats, false}, {"rstd", rstd, stats, false}, {"w", w, C * es, false},
                        {"b", b, C * es, false}, {"dx", dx, reach(M, lddx, C, es), true}, {"dw", dw, C * es, true},
                        {"db", db, C * es, true}, {"the workspace", workspace, need, true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (N == 0) {
    O1D_TRY(hip_status(fn, o1d::launch_zero((Dtype)dtype, dw, C, s)));
    return hip_status(fn, o1d::launch_zero((Dtype)dtype, db, C, s));
  }
  const rows::GnPlan pl = rows::plan_gn(true, N, P, C, groups, (int)es);
  O1D_TRY(check_pieces(fn, pl, N));
  rows::GnParams p = gn_params(pl, N, P, C, groups, act);
  p.ldx = ldx;
  p.ldd = lddy;
  p.ldy = lddx;
  p.x = x;
  p.dy = dy;
  p.w = w;
  p.b = b;
  p.out = dx;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.part = static_cast<float*>(workspace);
  p.dw = dw;
  p.db = db;
  return hip_status(fn, dtype == O1D_F32 ? rows::launch_gn_bwd_f32(pl, p, s) : rows::launch_gn_bwd_bf16(pl, p, s));
}

}  // extern "C"
