/*
 * o1d.h - C ABI of the MI355X (gfx950) library for depthwise convolution
 * with oriented 1D kernels.
 *
 * The operation is Definition 1, Eq. (1)-(2) of Kirchmeyer & Deng,
 * "Convolutional Networks with Oriented 1D Kernels" (ICCV 2023), with the
 * appendix "1D formulation" coordinate equation and the appendix "Padding"
 * rule (odd K, pad = K/2 inside the floor), stride 1 and zero padding:
 *
 *   y[n,c,p,q] = sum_{k=0}^{K-1} x[n,c, p + dh_c(k), q + dw_c(k)] * w[c,k]
 *   dh_c(k) = floor(-(k - K/2) * sin(theta_c)),
 *   dw_c(k) = floor( (k - K/2) * cos(theta_c)),
 *
 * where an x index outside [0,H) x [0,W) reads zero.  theta_c is given in
 * degrees; a product (k - K/2) * sin or cos that lies within 1e-9 of an
 * integer is taken to be that integer before the floor (so 0, 90, 30 ...
 * degrees give the exact-arithmetic offsets).  Taps that land on the same
 * pixel are summed.
 *
 * Layouts (all tensors dense, row-major, no strides):
 *   x, y, dy, dx : [N][C][H][W] in the element type `dtype`
 *   w, dw        : [C][K]       in the element type `dtype`
 *   theta_deg    : [C] float32 degrees, any finite value
 * Output size equals input size (P = H, Q = W).
 *
 * Memory and ownership: every tensor pointer is a DEVICE pointer owned by the
 * caller.  The library never allocates, frees or retains device memory on
 * these calls and keeps no per-call state, so calls are re-entrant.  All work
 * is enqueued asynchronously on `stream` (a hipStream_t; NULL selects the
 * null stream); the call returns after the enqueue.  Output buffers must not
 * alias input buffers.
 *
 * Precision: O1D_F32 computes and stores float32.  O1D_BF16 reads bfloat16,
 * accumulates in float32 and rounds the stored results to bfloat16 with
 * round-to-nearest-even.
 *
 * Errors: every argument check runs before any device work is enqueued; a
 * non-OK status means nothing was enqueued, except O1D_ERR_HIP, which reports
 * a failed kernel launch.  o1d_last_error() returns a human-readable detail
 * for the calling thread's most recent non-OK status.  Device faults, if
 * any, surface at the caller's next synchronisation.
 *
 * Empty tensors: a zero N, C, H or W is valid.  Nothing is launched, except
 * that o1d_bwd_weight and o1d_bwd with C > 0 write zeros to dw (an empty sum).
 */
#ifndef O1D_H_
#define O1D_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  O1D_F32 = 0,  /* float32 storage and arithmetic */
  O1D_BF16 = 1  /* bfloat16 storage, float32 accumulation, RNE stores */
} o1d_dtype_t;

typedef enum {
  O1D_NCHW = 0, /* x[n][c][h][w] */
  O1D_NHWC = 1  /* x[n][h][w][c], Definition 1's own layout */
} o1d_layout_t;

typedef enum {
  O1D_FLOOR = 0,   /* Eq. (2): offsets rounded down */
  O1D_BILINEAR = 1 /* bilinear interpolation at the unrounded offsets (section "Discretization and
                      Interpolation"): tap k reads the four pixels around (str p + rh_k, str q + rw_k),
                      (rh_k, rw_k) = (-(k - K/2) sin theta, (k - K/2) cos theta), weighted by
                      (1-fh)(1-fw), (1-fh)fw, fh(1-fw), fh fw with fh, fw the fractional parts
                      (a part within 1e-9 of 0 or 1 is taken as 0 with the integer moved accordingly) */
} o1d_sampling_t;

typedef enum {
  O1D_OK = 0,
  O1D_ERR_INVALID = 1,     /* NULL pointer for a non-empty tensor, negative size, even or non-positive K,
                              unknown dtype, aliasing output */
  O1D_ERR_UNSUPPORTED = 2, /* K above O1D_MAX_K, a stride above 64, a size beyond the kernels' 32-bit index
                              range (2^31 elements, 65535 images or channels), or a zero-margined band of the
                              plane too large for LDS */
  O1D_ERR_WORKSPACE = 3,   /* workspace smaller than o1d_bwd_weight_workspace_bytes() */
  O1D_ERR_HIP = 4          /* the HIP runtime rejected a kernel launch */
} o1d_status_t;

#define O1D_MAX_K 127

/* Forward pass, Definition 1 / Eq. (1): y = conv(x; w, theta). */
o1d_status_t o1d_fwd(const void* x, const void* w, const float* theta_deg, void* y,
                     int N, int C, int H, int W, int K, o1d_dtype_t dtype, void* stream);

/* Gradient of Eq. (1) with respect to x (its adjoint in x):
 *   dx[n,c,h,w] = sum_k w[c,k] * dy[n,c, h - dh_c(k), w - dw_c(k)]   (zero outside the plane).
 * dx is overwritten, not accumulated. */
o1d_status_t o1d_bwd_input(const void* dy, const void* w, const float* theta_deg, void* dx,
                           int N, int C, int H, int W, int K, o1d_dtype_t dtype, void* stream);

/* Gradient of Eq. (1) with respect to w (its adjoint in w):
 *   dw[c,k] = sum_{n,p,q} dy[n,c,p,q] * x[n,c, p + dh_c(k), q + dw_c(k)]   (zero outside the plane).
 * dw is overwritten, not accumulated.  `workspace` is caller-owned device
 * memory of at least o1d_bwd_weight_workspace_bytes(...) bytes (may be NULL
 * when that size is 0); its contents on entry are ignored and are clobbered.
 * Partial sums are combined in a fixed order, so dw (like the outputs of
 * o1d_fwd and o1d_bwd_input) is bitwise reproducible for the same inputs. */
o1d_status_t o1d_bwd_weight(const void* x, const void* dy, const float* theta_deg, void* dw,
                            int N, int C, int H, int W, int K, o1d_dtype_t dtype,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Both gradients of Eq. (1) in one call: dx as o1d_bwd_input computes it
 * (from dy and w) and dw as o1d_bwd_weight computes it (from x and dy).
 * One kernel reads x and dy once and produces both (then a small kernel adds
 * the weight gradient's partial rows); only where no one-pass kernel's LDS
 * tile fits (very large K with very wide planes) do the kernels of the two
 * separate entry points run in turn.  The results
 * equal those of the separate calls up to the order of floating-point
 * additions and are bitwise reproducible for the same inputs.  dx and dw
 * are overwritten.  `workspace` follows the rules of o1d_bwd_weight and
 * needs o1d_bwd_weight_workspace_bytes(...) bytes.  No output may overlap
 * an input, the other output or the workspace.  With N, H or W zero and
 * C > 0, dw is set to zeros. */
o1d_status_t o1d_bwd(const void* x, const void* dy, const void* w, const float* theta_deg, void* dx, void* dw,
                     int N, int C, int H, int W, int K, o1d_dtype_t dtype,
                     void* workspace, size_t workspace_bytes, void* stream);

/* Workspace size in bytes that o1d_bwd_weight (and o1d_bwd) needs for these sizes. */
size_t o1d_bwd_weight_workspace_bytes(int N, int C, int H, int W, int K, o1d_dtype_t dtype);

/* o1d_bwd without a workspace argument, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid allocation).  It computes exactly what o1d_bwd computes (the
 * same kernels and fixed-order sums, so dx and dw are bitwise equal to
 * o1d_bwd's) and keeps the weight gradient's partial rows in a fixed device scratch
 * array of 8 MiB that the library holds on every GPU it runs on until the
 * process ends.  It allocates and frees nothing.  Sizes whose partial rows
 * need more than 8 MiB (o1d_bwd_weight_workspace_bytes > 8 MiB) return
 * O1D_ERR_UNSUPPORTED before any launch.  All calls on one GPU share that
 * GPU's scratch: calls that overlap on one GPU (on different streams, or from
 * different threads without ordering) race and must be serialised by the
 * caller.  Nothing needs clearing between calls.  Other rules as o1d_bwd. */
o1d_status_t o1d_bwd_noalloc(const void* x, const void* dy, const void* w, const float* theta_deg, void* dx,
                             void* dw, int N, int C, int H, int W, int K, o1d_dtype_t dtype, void* stream);

/* ---- Stride, layout and sampling (Definition 1 with its stride `str`, Eq. 2).
 *
 * The _ex entry points compute the same three operations for any stride >= 1
 * (at most 64), either memory layout and either discretisation.  The input
 * plane is H x W; the output plane is P x Q with P = (H - 1) / stride + 1 and
 * Q = (W - 1) / stride + 1 (integer division: output (p, q) is centred on
 * input (stride p, stride q)):
 *   y[n,c,p,q]  = sum_k w[c,k] sample_k(x[n,c], stride p, stride q)
 *   dx[n,c,h,w] = the adjoint of that map in x (a scatter of dy, computed as a gather)
 *   dw[c,k]     = sum_{n,p,q} dy[n,c,p,q] sample_k(x[n,c], stride p, stride q)
 * where sample_k reads the pixel at the rounded-down offsets of Eq. (2)
 * (O1D_FLOOR) or interpolates bilinearly at the unrounded ones (O1D_BILINEAR),
 * pixels outside the plane reading zero.  Layouts: x and dx are N x C x H x W
 * (O1D_NCHW) or N x H x W x C (O1D_NHWC); y and dy are N x C x P x Q or
 * N x P x Q x C; w, dw are [C][K]; theta_deg is [C].  With stride 1, O1D_NCHW
 * and O1D_FLOOR they are exactly o1d_fwd, o1d_bwd_input and o1d_bwd_weight.
 * Ownership, asynchrony, precision, error and empty-tensor rules are those of
 * the plain entry points; H and W are always the input plane's, also for
 * o1d_bwd_input_ex.  O1D_ERR_UNSUPPORTED is returned where a band of the
 * plane with its zero margin does not fit in LDS (K and stride both very
 * large).  The weight gradient's workspace is
 * o1d_bwd_weight_ex_workspace_bytes(...) bytes. */
o1d_status_t o1d_fwd_ex(const void* x, const void* w, const float* theta_deg, void* y,
                        int N, int C, int H, int W, int K, int stride, o1d_layout_t layout,
                        o1d_sampling_t sampling, o1d_dtype_t dtype, void* stream);
o1d_status_t o1d_bwd_input_ex(const void* dy, const void* w, const float* theta_deg, void* dx,
                              int N, int C, int H, int W, int K, int stride, o1d_layout_t layout,
                              o1d_sampling_t sampling, o1d_dtype_t dtype, void* stream);
o1d_status_t o1d_bwd_weight_ex(const void* x, const void* dy, const float* theta_deg, void* dw,
                               int N, int C, int H, int W, int K, int stride, o1d_layout_t layout,
                               o1d_sampling_t sampling, o1d_dtype_t dtype,
                               void* workspace, size_t workspace_bytes, void* stream);
size_t o1d_bwd_weight_ex_workspace_bytes(int N, int C, int H, int W, int K, int stride, o1d_layout_t layout,
                                         o1d_sampling_t sampling, o1d_dtype_t dtype);

/* ---- Oriented 1D depthwise separable block (Sec. 3.2 "Computational cost
 * analysis", Table 1 "Oriented 1D DSC").
 *
 * The oriented depthwise convolution of Eq. (1) (stride 1, NCHW, offsets
 * rounded down) followed by a pointwise (1 x 1) convolution that mixes the C
 * channels into Cout:
 *   z = o1d_fwd(x, w_dw, theta_deg)                       (N x C x H x W)
 *   y[n,o,h,w] = sum_c w_pw[o,c] z[n,c,h,w]               (N x Cout x H x W)
 * w_dw is [C][K], w_pw [Cout][C] (row-major), theta_deg [C] float32; x, z, y,
 * w_dw and w_pw have `dtype` storage.  o1d_dsc_fwd writes z (kept for the
 * backward) and y; the pointwise product runs on the matrix cores (float32
 * products for O1D_F32, bfloat16 products for O1D_BF16, float32 accumulation).
 * o1d_dsc_bwd computes, for the upstream gradient dy (N x Cout x H x W):
 *   dz = w_pw^T dy (per pixel),  dw_pw[o,c] = sum_{n,h,w} dy[n,o,h,w] z[n,c,h,w],
 *   (dx, dw_dw) = o1d_bwd(x, dz, w_dw, theta_deg),
 * with dz kept in `workspace` (at least o1d_dsc_bwd_workspace_bytes(...)
 * bytes of caller-owned device memory, contents ignored and clobbered); its z
 * must be the forward's.  dw_pw's images are summed in groups whose float32
 * partial sums are added in a fixed order (bitwise reproducible).  Outputs
 * are overwritten; no output may overlap an input, another output or the
 * workspace.  Cout is 1 .. 65535; other rules as o1d_fwd and o1d_bwd. */
o1d_status_t o1d_dsc_fwd(const void* x, const void* w_dw, const float* theta_deg, const void* w_pw, void* z,
                         void* y, int N, int C, int Cout, int H, int W, int K, o1d_dtype_t dtype, void* stream);
o1d_status_t o1d_dsc_bwd(const void* x, const void* z, const void* dy, const void* w_dw, const float* theta_deg,
                         const void* w_pw, void* dx, void* dw_dw, void* dw_pw, int N, int C, int Cout, int H,
                         int W, int K, o1d_dtype_t dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t o1d_dsc_bwd_workspace_bytes(int N, int C, int Cout, int H, int W, int K, o1d_dtype_t dtype);

/* ---- Row operators: what a block of the network computes around the
 * convolution, on channels-last activations (an N x H x W x C tensor is M = N H W
 * rows of C features).
 *
 * Matrices have M rows; a row's features are contiguous and rows lie `ld`
 * elements apart (at least the number of features, below 2^21), so that a slice
 * of a wider tensor can be given.  Weights are dense and, like the biases,
 * of the activations' dtype.  Any number of features from 1 to 2^20 and any
 * element-aligned address is accepted.
 *
 * Sums, statistics and products accumulate in float32 and are rounded once when
 * stored.  Products of float32 take each operand to 24 bits or to a multiple of
 * 2^-133, whichever is coarser, and each product to 2^-24 of itself (an infinity
 * times an operand that rounds to 0 is NaN).  The weight gradient of a checkpointed
 * or activated input rounds that input, act(x), to dtype first, as the
 * forward's product was given it (the matrix cores' operand).  All sums have a
 * fixed order: results are bitwise reproducible.
 *
 * Ownership, asynchrony and error rules are those of the other entry points; no
 * output may overlap an input, another output or the workspace, measured over
 * the rows' whole reach.  A workspace is 16-byte aligned and has at least the
 * bytes that the call's ..._workspace_bytes gives for the same arguments (256
 * where the work needs none, and nothing is written to them; at least 512 where
 * it needs some; 0 for M = 0); what it holds before a call does not matter.
 * Calls that may run at the same time need workspaces of their own, unless nothing
 * is written to them.  M = 0 is valid: nothing is launched, except that weight
 * gradients are set to zeros. */
typedef enum {
  O1D_ACT_NONE = 0,
  O1D_ACT_RELU = 1,
  O1D_ACT_GELU = 2,      /* x Phi(x) */
  O1D_ACT_GELU_TANH = 3, /* x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2 */
  O1D_ACT_SILU = 4       /* x / (1 + exp(-x)) */
} o1d_act_t;

/* 8-bit checkpoints of a matrix of C features: signed char q[M][ldq] with ldq =
 * C rounded up to 16 (q 16-byte aligned; the padding is zero) and float
 * scale[M][ceil(C / 64)].  A group of 64 columns of a row shares a scale:
 *   amax = max |x|, scale = amax / 127, q = rint(x (127 / amax)), which stands for q scale,
 * an error of at most amax / 254 (and float32 rounding; it is finite also for the largest amax).  A group that holds a
 * NaN or an infinity gets the scale NaN: all of it reads NaN.  One whose amax is
 * below 2^-100 gets scale 0. */
o1d_status_t o1d_pack(const void* x, long long ldx, signed char* q, float* scale, int M, int C, o1d_dtype_t dtype,
                      void* stream);
/* y = act(what the checkpoint stands for). */
o1d_status_t o1d_unpack(const signed char* q, const float* scale, o1d_act_t act, void* y, long long ldy, int M, int C,
                        o1d_dtype_t dtype, void* stream);

/* Layer norm over a row's features: mean = sum x / C, var = sum (x - mean)^2 / C,
 * rstd = (var + eps)^-1/2, y = (x - mean) rstd w + b.  mean and rstd (float32, one
 * per row, for the backward) are written unless both are NULL. */
o1d_status_t o1d_ln_fwd(const void* x, long long ldx, const void* w, const void* b, void* y, long long ldy, float* mean,
                        float* rstd, int M, int C, float eps, o1d_dtype_t dtype, void* stream);
/* Its gradients: with xh = (x - mean) rstd and g = dy w,
 *   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy.
 * x is a tensor (x, ldx) or a checkpoint (xq, xscale): exactly one of x and xq is not NULL. */
o1d_status_t o1d_ln_bwd(const void* x, long long ldx, const signed char* xq, const float* xscale, const void* dy,
                        long long lddy, const float* mean, const float* rstd, const void* w, void* dx, long long lddx,
                        void* dw, void* db, int M, int C, o1d_dtype_t dtype, void* workspace, size_t workspace_bytes,
                        void* stream);
size_t o1d_ln_bwd_workspace_bytes(int M, int C, o1d_dtype_t dtype);

/* h = x W^T + b,  y = act(h) + residual, with x M x I, W [O][I], b [O] (or NULL),
 * the residual M x O (or NULL).  For the backward h is stored where asked: as a
 * tensor (pre, or NULL), as a checkpoint (q, scale, or NULL), or both. */
o1d_status_t o1d_linear_fwd(const void* x, long long ldx, const void* w, const void* b, o1d_act_t act, const void* res,
                            long long ldres, void* y, long long ldy, void* pre, long long ldpre, signed char* q,
                            float* scale, int M, int I, int O, o1d_dtype_t dtype, void* stream);
/* Gradient in the input, carried through the activation that made the input:
 *   dx = (dy W) act'(pre),  dy M x O, W [O][I], pre and dx M x I.
 * With O1D_ACT_NONE pre is not read; else it is a tensor (pre, ldpre) or a
 * checkpoint (preq, prescale), exactly one. */
o1d_status_t o1d_linear_bwd_input(const void* dy, long long lddy, const void* w, o1d_act_t act, const void* pre,
                                  long long ldpre, const signed char* preq, const float* prescale, void* dx,
                                  long long lddx, int M, int I, int O, o1d_dtype_t dtype, void* stream);
/* Gradients in the weights: dw = dy^T act(x) ([O][I]), db = sum_rows dy ([O], or
 * NULL).  x is a tensor or a checkpoint, exactly one; act is the activation
 * between it and the product's input (O1D_ACT_NONE: x is the input). */
o1d_status_t o1d_linear_bwd_weight(const void* x, long long ldx, const signed char* xq, const float* xscale, o1d_act_t act,
                                   const void* dy, long long lddy, void* dw, void* db, int M, int I, int O,
                                   o1d_dtype_t dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t o1d_linear_bwd_weight_workspace_bytes(int M, int I, int O, o1d_act_t act, int held, o1d_dtype_t dtype);
/* dh = dy act'(pre), pre a tensor or a checkpoint, exactly one. */
o1d_status_t o1d_act_bwd(const void* pre, long long ldpre, const signed char* preq, const float* prescale, o1d_act_t act,
                         const void* dy, long long lddy, void* dh, long long lddh, int M, int C, o1d_dtype_t dtype,
                         void* stream);

/* Group norm with an activation on channels-last samples: x is N samples of P pixels, rows of C = groups x D channels (x, y
 * and their gradients are N P rows, ld elements apart).  Over the P D values of a sample's group, mean = sum x / (P D),
 * var = sum (x - mean)^2 / (P D), rstd = (var + eps)^-1/2, xh = (x - mean) rstd, h = xh w + b, y = act(h).  mean and
 * rstd (float32, [N][groups]) are always written.  groups divides C and a group has at most 1024 channels; P >= 1.
 * A call that passes its samples twice keeps statistics of their parts in the workspace. */
o1d_status_t o1d_gn_fwd(const void* x, long long ldx, const void* w, const void* b, o1d_act_t act, void* y, long long ldy,
                        float* mean, float* rstd, int N, int P, int C, int groups, float eps, o1d_dtype_t dtype,
                        void* workspace, size_t workspace_bytes, void* stream);
size_t o1d_gn_fwd_workspace_bytes(int N, int P, int C, int groups, o1d_dtype_t dtype);
/* Its gradients: with dh = dy act'(h) and g = dh w,
 *   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum dh xh,  db = sum dh (over samples and pixels). */
o1d_status_t o1d_gn_bwd(const void* x, long long ldx, const void* dy, long long lddy, const float* mean, const float* rstd,
                        const void* w, const void* b, o1d_act_t act, void* dx, long long lddx, void* dw, void* db, int N,
                        int P, int C, int groups, o1d_dtype_t dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t o1d_gn_bwd_workspace_bytes(int N, int P, int C, int groups, o1d_dtype_t dtype);

/* ---- Products of 8-bit floating point operands with a power-of-two scale for each 128 values.
 *
 * An operand of R rows of K values is unsigned char q[R][ldq], ldq = K rounded up to 128 (zeros behind a row's end), of
 * OCP e4m3 or e5m2 values, and unsigned char e[ceil(K / 128)][lde], lde = R rounded up to 16 (127 behind the last row): value k of row r
 * stands for q[r][k] 2^(e[k / 128][r] - 127).  q and e are 16-byte aligned.
 *
 * o1d_pack_scaled makes the operand of x (M rows of C values): by rows (q, e: R = M, K = C), transposed (qt, et: R = C, K = M,
 * groups of 128 rows of x), or both.  The power of two is the least one that leaves the group's largest finite value in the type's
 * range (448, 57344), at least 2^-127, and 2^0 for a group of zeros; the quotient is rounded once, to nearest with ties to
 * even, and a value that is not finite becomes NaN.  sums (or NULL; with qt only): the sums of x's columns,
 * [C] of dtype, by way of the workspace. */
typedef enum { O1D_E4M3 = 0, O1D_E5M2 = 1 } o1d_scaled_t;
o1d_status_t o1d_pack_scaled(const void* x, long long ldx, o1d_scaled_t type, unsigned char* q, unsigned char* e,
                             unsigned char* qt, unsigned char* et, void* sums, int M, int C, o1d_dtype_t dtype,
                             void* workspace, size_t workspace_bytes, void* stream);
size_t o1d_pack_scaled_workspace_bytes(int M, int C, int sums);
/* The products of o1d_linear_*, of packed operands, accumulated in float32, with results of dtype.  The first operand has the
 * given type, the second is e4m3.
 *   fwd:        h = x W^T + b, y = act(h) + residual; pre (or NULL) = h.   x: M rows of I, W: O rows of I
 *   bwd_input:  dx = (dy W) act'(pre).                                     dy: M rows of O, W^T: I rows of O
 *   bwd_weight: dw = dy^T x ([O][I]).                                      dy^T: O rows of M, x^T: I rows of M
 * Results of float32 are of exact products, summed in float32 (values below 2^-126 keep fewer of their bits).  For results of
 * bfloat16, products are summed eight at a time with 13 bits behind the power of two of the largest, and those sums in
 * float32.  An exponent of 255 makes its values NaN. */
o1d_status_t o1d_scaled_linear_fwd(const unsigned char* xq, const unsigned char* xe, o1d_scaled_t type,
                                   const unsigned char* wq, const unsigned char* we, const void* b, o1d_act_t act,
                                   const void* res, long long ldres, void* y, long long ldy, void* pre, long long ldpre, int M,
                                   int I, int O, o1d_dtype_t dtype, void* stream);
o1d_status_t o1d_scaled_linear_bwd_input(const unsigned char* dyq, const unsigned char* dye, o1d_scaled_t type,
                                         const unsigned char* wtq, const unsigned char* wte, o1d_act_t act, const void* pre,
                                         long long ldpre, void* dx, long long lddx, int M, int I, int O, o1d_dtype_t dtype,
                                         void* stream);
o1d_status_t o1d_scaled_linear_bwd_weight(const unsigned char* dytq, const unsigned char* dyte, o1d_scaled_t type,
                                          const unsigned char* xtq, const unsigned char* xte, void* dw, int M, int I, int O,
                                          o1d_dtype_t dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t o1d_scaled_linear_bwd_weight_workspace_bytes(int M, int I, int O, o1d_dtype_t dtype);

/* ---- AdamW over many tensors at once.  With t = steps taken + 1 and g the gradient (times max_norm / norm where the norm is
 * larger):
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   p = p (1 - lr weight_decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 *
 * Tensor i has n values p (param_dtype) and g (grad_dtype), and its part of the states starts at value `at`, a multiple
 * of 128; behind its end the states' values up to the next multiple of 128 are set to zeros.  state_bits 32: m and v
 * are float32.  8: m and the root of v are e4m3 (a positive root at least the type's smallest value), with a scale
 * m_scale, v_scale for each 128 values: the largest / 448, at least 2^-126, or 0 for zeros.  master (or NULL): the parameters in float32, from which p is rounded;
 * without it p itself is read.  follow (not 0, with master): where p is not its master rounded, it was written since the
 * last step, and its value is taken for the master's.  The states are 16-byte aligned.
 * step: two device integers, the steps taken (read and counted up; below 0: read as 0) and 0.  lr_at: the learning rate in device memory, or NULL for
 * lr.  max_norm > 0 limits the norm of all gradients to it; the norm is then written to `norm`, and where it is not finite
 * nothing else changes.  max_norm 0: no limit, norm is not written and may be NULL.
 * Without max_norm a gradient that is not finite makes its parameter NaN and its states NaN or infinite, 8-bit ones with all 128
 * values of their scale.  A call without values counts no step.  Tensors that are written overlap no other one; gradients may be shared. */
typedef struct {
  void* p;
  const void* g;
  long long n, at;
} o1d_adamw_tensor_t;
typedef struct {
  void *m, *v;
  float *m_scale, *v_scale, *master;
  int* step;
  int bits;
} o1d_adamw_state_t;
typedef struct {
  double lr, beta1, beta2, eps, weight_decay, max_norm;
  const float* lr_at;
  int follow;
} o1d_adamw_options_t;
o1d_status_t o1d_adamw(const o1d_adamw_tensor_t* tensors, int count, o1d_dtype_t param_dtype, o1d_dtype_t grad_dtype,
                       const o1d_adamw_state_t* state, const o1d_adamw_options_t* options, float* norm, void* workspace,
                       size_t workspace_bytes, void* stream);
size_t o1d_adamw_workspace_bytes(double max_norm);

/* ---- Planning introspection (host only, no device work; for tests and tools).
 *
 * o1d_kernel_name: the kernel(s) a call with these arguments would launch,
 * e.g. "strip_gather/f32/S77/KB32" or "walk_wgrad/bf16/nhwc/S87"; two names
 * joined by '+' where o1d_bwd runs the input and weight gradients in turn.
 * op: 0 = o1d_fwd(_ex), 1 = o1d_bwd_input(_ex), 2 = o1d_bwd_weight(_ex),
 * 3 = o1d_bwd (stride 1, NCHW, O1D_FLOOR only).  `aligned` != 0 states that
 * the tensors are 16-byte (O1D_F32) or 8-byte (O1D_BF16) aligned.  Returns ""
 * for invalid or empty sizes.  The string lives in thread-local storage until
 * the thread's next call.
 * o1d_kernel_variant: the i-th kernel instantiation compiled into the
 * library, in the same naming, or NULL for i past the last. */
const char* o1d_kernel_name(int op, int N, int C, int H, int W, int K, int stride, o1d_layout_t layout,
                            o1d_sampling_t sampling, o1d_dtype_t dtype, int aligned);
const char* o1d_kernel_variant(int i);

/* The same for the row operators: e.g. "mmf/fwd/bf16/128x64" (its tile) or
 * "act+mm/wgrad/f32/64x64+mm_sum", launches joined by '+'.  op: 0 = o1d_linear_fwd (held: it
 * writes a checkpoint), 1 = o1d_linear_bwd_input, 2 = o1d_linear_bwd_weight (held: of a
 * checkpoint; act as there), 3 = o1d_ln_fwd, 4 = o1d_ln_bwd (held: of a checkpoint), both with I
 * features; act and O are read where the call has them.  `aligned` != 0 states that tensors
 * and row strides are multiples of 16 bytes. */
const char* o1d_rows_kernel_name(int op, int M, int I, int O, o1d_act_t act, int held, o1d_dtype_t dtype, int aligned);

/* Static description of a status code. */
const char* o1d_status_str(o1d_status_t status);

/* Detail for the calling thread's most recent non-OK status ("" if none). */
const char* o1d_last_error(void);

/* Library version string. */
const char* o1d_version(void);

#ifdef __cplusplus
}
#endif

#endif /* O1D_H_ */
