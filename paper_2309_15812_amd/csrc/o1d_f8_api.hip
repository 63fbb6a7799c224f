// C ABI of the products of 8-bit floating point operands (declared in include/o1d.h).
#include "o1d_f8.h"
#include "o1d_rows_check.h"

namespace {

o1d_status_t check_type(const char* fn, o1d_scaled_t type) {
  return type == O1D_E4M3 || type == O1D_E5M2 ? O1D_OK : fail(O1D_ERR_INVALID, "%s: unknown type %d", fn, (int)type);
}

o1d_status_t check_packed(const char* fn, const char* what, const unsigned char* q, const unsigned char* e) {
  if (!q || !e) return fail(O1D_ERR_INVALID, "%s: %s needs its values and its exponents", fn, what);
  if ((uintptr_t)q % 16 || (uintptr_t)e % 16)
    return fail(O1D_ERR_INVALID, "%s: values and exponents of %s must be 16-byte aligned", fn, what);
  return O1D_OK;
}

// Rows that a weight gradient sums: the offsets of a tile's 128 rows stay below 2^31 bytes.
constexpr int kMostSummed = 8 * (int)kMaxStride - 1024;

size_t q_bytes(int R, int K) { return (size_t)R * (size_t)rows::f8_ld(K); }
size_t e_bytes(int R, int K) { return (size_t)rows::f8_le(R) * (size_t)rows::f8_groups(K); }

// A product's plan with its operands: A of M rows, B of N rows, K values each.
rows::F8Plan planned(int kind, int M, int N, int K, const unsigned char* aq, const unsigned char* ae, o1d_scaled_t type,
                     const unsigned char* bq, const unsigned char* be, o1d_dtype_t dt) {
  rows::F8Plan pl = rows::plan_f8(kind, M, N, K, (int)elem_size(dt));
  pl.atype = (int)type;
  pl.p.mm.a = aq;
  pl.p.mm.b = bq;
  pl.p.mm.lda = pl.p.mm.ldb = rows::f8_ld(K);
  pl.p.ea = ae;
  pl.p.eb = be;
  pl.p.lea = rows::f8_le(M);
  pl.p.leb = rows::f8_le(N);
  return pl;
}

o1d_status_t check_tiles(const char* fn, const rows::F8Plan& pl) {
  const long long blocks = (long long)pl.p.mm.tm * pl.p.mm.tn * (pl.p.mm.nsplit ? pl.p.mm.nsplit : 1);
  return blocks > (1 << 24) - 8 ? fail(O1D_ERR_UNSUPPORTED, "%s: %lld workgroups exceed the grid", fn, blocks) : O1D_OK;
}

}  // namespace

extern "C" {

size_t o1d_pack_scaled_workspace_bytes(int M, int C, int sums) {
  if (check_dims("o1d_pack_scaled", M, C, "C", O1D_F32) != O1D_OK || M == 0) return 0;
  return sums ? space_for((size_t)rows::f8_groups(M) * C * sizeof(float)) : kNoSpace;
}

o1d_status_t o1d_pack_scaled(const void* x, long long ldx, o1d_scaled_t type, unsigned char* q, unsigned char* e,
                             unsigned char* qt, unsigned char* et, void* sums, int M, int C, o1d_dtype_t dtype,
                             void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "o1d_pack_scaled";
  O1D_TRY(check_dims(fn, M, C, "C", dtype));
  O1D_TRY(check_type(fn, type));
  O1D_TRY(check_ld(fn, "x", ldx, C));
  const size_t es = elem_size(dtype), need = sums ? o1d_pack_scaled_workspace_bytes(M, C, 1) : 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  O1D_TRY(check_elem_aligned(fn, sums, "the sums", es));
  if (M == 0) return sums ? hip_status(fn, o1d::launch_zero((Dtype)dtype, sums, C, s)) : ok();
  if (M > (1 << 30) - 64) return fail(O1D_ERR_UNSUPPORTED, "%s: M=%d rows exceed the grid", fn, M);
  O1D_TRY(check_null(fn, {x}));
  if (!q && !e && !qt && !et) return fail(O1D_ERR_INVALID, "%s: no operand is asked for", fn);
  if (q || e) O1D_TRY(check_packed(fn, "the operand", q, e));
  if (qt || et) O1D_TRY(check_packed(fn, "the transposed operand", qt, et));
  if (sums && !qt) return fail(O1D_ERR_INVALID, "%s: sums come with the transposed operand", fn);
  O1D_TRY(check_workspace(fn, sums ? workspace : nullptr, workspace_bytes, need));
  O1D_TRY(check_elem_aligned(fn, x, "x", es));
  const Span spans[] = {{"x", x, reach(M, ldx, C, es), false}, {"the operand", q, q_bytes(M, C), true},
                        {"its exponents", e, e_bytes(M, C), true}, {"the transposed operand", qt, q_bytes(C, M), true},
                        {"its exponents", et, e_bytes(C, M), true}, {"the sums", sums, C * es, true},
                        {"the workspace", sums ? workspace : nullptr, need, true}};
  O1D_TRY(apart(fn, spans));
  (void)hipGetLastError();
  rows::F8PackParams p{};
  p.x = x;
  p.ldx = ldx;
  p.M = M;
  p.C = C;
  p.type = (int)type;
  p.q = q;
  p.e = e;
  p.qt = qt;
  p.et = et;
  p.part = sums ? static_cast<float*>(workspace) : nullptr;
  O1D_TRY(hip_status(fn, rows::launch_f8_pack((Dtype)dtype, p, s)));
  if (!sums) return ok();
  return hip_status(fn, rows::launch_col_sum((Dtype)dtype, p.part, rows::f8_groups(M), C, C, sums, nullptr, s));
}

o1d_status_t o1d_scaled_linear_fwd(const unsigned char* xq, const unsigned char* xe, o1d_scaled_t type,
                                   const unsigned char* wq, const unsigned char* we, const void* b, o1d_act_t act,
                                   const void* res, long long ldres, void* y, long long ldy, void* pre, long long ldpre, int M,
                                   int I, int O, o1d_dtype_t dtype, void* stream) {
  const char* fn = "o1d_scaled_linear_fwd";
  O1D_TRY(check_dims(fn, M, I, "I", dtype));
  O1D_TRY(check_dims(fn, M, O, "O", dtype));
  O1D_TRY(check_type(fn, type));
  O1D_TRY(check_act(fn, act));
  O1D_TRY(check_ld(fn, "y", ldy, O));
  if (res) O1D_TRY(check_ld(fn, "the residual", ldres, O));
  if (pre) O1D_TRY(check_ld(fn, "pre", ldpre, O));
  if (M == 0) return ok();
  O1D_TRY(check_packed(fn, "x", xq, xe));
  O1D_TRY(check_packed(fn, "w", wq, we));
  O1D_TRY(check_null(fn, {y}));
  const size_t es = elem_size(dtype);
  for (const void* p : {b, res, (const void*)y, (const void*)pre}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  const Span spans[] = {{"x", xq, q_bytes(M, I), false}, {"x's exponents", xe, e_bytes(M, I), false},
                        {"w", wq, q_bytes(O, I), false}, {"w's exponents", we, e_bytes(O, I), false}, {"b", b, O * es, false},
                        {"the residual", res, reach(M, ldres, O, es), false}, {"y", y, reach(M, ldy, O, es), true},
                        {"pre", pre, reach(M, ldpre, O, es), true}};
  O1D_TRY(apart(fn, spans));
  rows::F8Plan pl = planned(rows::kFwd, M, O, I, xq, xe, type, wq, we, dtype);
  O1D_TRY(check_tiles(fn, pl));
  (void)hipGetLastError();
  rows::MmParams& p = pl.p.mm;
  p.act = (int)act;
  p.bias = b;
  p.res = res;
  p.ldres = ldres;
  p.out = y;
  p.ldo = ldy;
  p.pre = pre;
  p.ldpre = ldpre;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(fn, dtype == O1D_F32 ? rows::launch_f8_fwd_f32(pl, s) : rows::launch_f8_fwd_bf16(pl, s));
}

o1d_status_t o1d_scaled_linear_bwd_input(const unsigned char* dyq, const unsigned char* dye, o1d_scaled_t type,
                                         const unsigned char* wtq, const unsigned char* wte, o1d_act_t act, const void* pre,
                                         long long ldpre, void* dx, long long lddx, int M, int I, int O, o1d_dtype_t dtype,
                                         void* stream) {
  const char* fn = "o1d_scaled_linear_bwd_input";
  O1D_TRY(check_dims(fn, M, I, "I", dtype));
  O1D_TRY(check_dims(fn, M, O, "O", dtype));
  O1D_TRY(check_type(fn, type));
  O1D_TRY(check_act(fn, act));
  O1D_TRY(check_ld(fn, "dx", lddx, I));
  if (act != O1D_ACT_NONE) O1D_TRY(check_ld(fn, "pre", ldpre, I));
  if (M == 0) return ok();
  O1D_TRY(check_packed(fn, "dy", dyq, dye));
  O1D_TRY(check_packed(fn, "w", wtq, wte));
  O1D_TRY(check_null(fn, {dx}));
  const void* slope = act != O1D_ACT_NONE ? pre : nullptr;
  if (act != O1D_ACT_NONE) O1D_TRY(check_null(fn, {pre}));
  const size_t es = elem_size(dtype);
  for (const void* p : {slope, (const void*)dx}) O1D_TRY(check_elem_aligned(fn, p, "a tensor", es));
  const Span spans[] = {{"dy", dyq, q_bytes(M, O), false}, {"dy's exponents", dye, e_bytes(M, O), false},
                        {"w", wtq, q_bytes(I, O), false}, {"w's exponents", wte, e_bytes(I, O), false},
                        {"pre", slope, reach(M, ldpre, I, es), false}, {"dx", dx, reach(M, lddx, I, es), true}};
  O1D_TRY(apart(fn, spans));
  rows::F8Plan pl = planned(rows::kDgrad, M, I, O, dyq, dye, type, wtq, wte, dtype);
  O1D_TRY(check_tiles(fn, pl));
  (void)hipGetLastError();
  rows::MmParams& p = pl.p.mm;
  p.act = (int)act;
  p.out = dx;
  p.ldo = lddx;
  p.pre = const_cast<void*>(slope);
  p.ldpre = ldpre;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(fn, dtype == O1D_F32 ? rows::launch_f8_dgrad_f32(pl, s) : rows::launch_f8_dgrad_bf16(pl, s));
}

size_t o1d_scaled_linear_bwd_weight_workspace_bytes(int M, int I, int O, o1d_dtype_t dtype) {
  const char* fn = "o1d_scaled_linear_bwd_weight";
  if (check_dims(fn, M, I, "I", dtype) != O1D_OK || check_dims(fn, M, O, "O", dtype) != O1D_OK || M == 0) return 0;
  if (M > kMostSummed) return 0;
  const int pieces = rows::plan_f8(rows::kWgrad, O, I, M, (int)elem_size(dtype)).p.mm.nsplit;
  return pieces > 1 ? space_for((size_t)pieces * ((size_t)O * I + O) * sizeof(float)) : kNoSpace;
}

o1d_status_t o1d_scaled_linear_bwd_weight(const unsigned char* dytq, const unsigned char* dyte, o1d_scaled_t type,
                                          const unsigned char* xtq, const unsigned char* xte, void* dw, int M, int I, int O,
                                          o1d_dtype_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "o1d_scaled_linear_bwd_weight";
  O1D_TRY(check_dims(fn, M, I, "I", dtype));
  O1D_TRY(check_dims(fn, M, O, "O", dtype));
  O1D_TRY(check_type(fn, type));
  O1D_TRY(check_null(fn, {dw}));
  const size_t es = elem_size(dtype), need = o1d_scaled_linear_bwd_weight_workspace_bytes(M, I, O, dtype);
  O1D_TRY(check_elem_aligned(fn, dw, "dw", es));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (M == 0) return hip_status(fn, o1d::launch_zero((Dtype)dtype, dw, (size_t)O * I, s));
  if (M > kMostSummed) return fail(O1D_ERR_UNSUPPORTED, "%s: M=%d rows exceed %d", fn, M, kMostSummed);
  O1D_TRY(check_packed(fn, "dy", dytq, dyte));
  O1D_TRY(check_packed(fn, "x", xtq, xte));
  O1D_TRY(check_workspace(fn, workspace, workspace_bytes, need));
  const Span spans[] = {{"dy", dytq, q_bytes(O, M), false}, {"dy's exponents", dyte, e_bytes(O, M), false},
                        {"x", xtq, q_bytes(I, M), false}, {"x's exponents", xte, e_bytes(I, M), false},
                        {"dw", dw, (size_t)O * I * es, true}, {"the workspace", workspace, need, true}};
  O1D_TRY(apart(fn, spans));
  rows::F8Plan pl = planned(rows::kWgrad, O, I, M, dytq, dyte, type, xtq, xte, dtype);
  O1D_TRY(check_tiles(fn, pl));
  (void)hipGetLastError();
  rows::MmParams& p = pl.p.mm;
  p.out = dw;
  p.part = static_cast<float*>(workspace);
  O1D_TRY(hip_status(fn, dtype == O1D_F32 ? rows::launch_f8_wgrad_f32(pl, s) : rows::launch_f8_wgrad_bf16(pl, s)));
  if (p.nsplit == 1) return ok();
  rows::MmPlan sum{};
  sum.p = p;
  return hip_status(fn, rows::launch_mm_sum((Dtype)dtype, sum, dw, nullptr, s));
}

}  // extern "C"
