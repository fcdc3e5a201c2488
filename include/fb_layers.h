/*
 * fb_layers.h -- C ABI of the operators of a network's last layers (libfb_amd.so).
 *
 * The objective of fb.h starts at the network's output (emis) and ends at its derivative (grad).  These calls are what lies
 * on the network's side of it, forward and backward:
 *
 *   fb_layer_norm, fb_layer_norm_grad             normalisation of hidden frames
 *   fb_residual_norm, fb_residual_norm_grad       from one block into the next: norm, gate, scale, residual, norm
 *   fb_affine, fb_affine_grad                     y = act(x W^T + b) + residual
 *   fb_gated_affine, fb_gated_affine_grad         y = act(x G^T + a) (x U^T + b), elementwise
 *   fb_token_logprobs, fb_token_logprobs_grad     log probabilities of given tokens, entropy, best alternatives
 *   fb_affine_logprobs, fb_affine_logprobs_grad   log probabilities and entropy straight from hidden frames, logits never kept
 *
 * Conventions are those of fb.h: device pointers owned by the caller, kernels enqueued on `stream`, nothing allocated, freed
 * or synchronised, FB_OK or a negative code returned and never an exception, fb_last_error() says what was wrong.  A call may
 * be recorded into a HIP graph.  Results do not depend on timing: no sum is formed with atomics.
 *
 * Rows are frames.  A matrix is given by its first element and the distance between rows in elements (`ld`); the elements of
 * a row are contiguous.  Rows may start at any element: no alignment beyond the element's own is asked for (workspaces: 256
 * bytes).  Row counts may be 0 (sums over no rows are 0) and are below 2^31, as are row distances; widths are at least 1 and
 * below 2^28.  A matrix may have more than 2^32 elements.
 *
 * Types: FB_TYPE_F32, FB_TYPE_BF16, FB_TYPE_F16.  Sums, statistics and the products' accumulators are single precision
 * whatever the type, and a result is rounded once, when it is stored, unless a call says otherwise.
 */
#ifndef FB_LAYERS_H
#define FB_LAYERS_H

#include "fb.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FB_TYPE_F32 = 0, FB_TYPE_BF16 = 1, FB_TYPE_F16 = 2 };
enum {
    FB_ACT_NONE = 0,
    FB_ACT_RELU = 1,  /* max(z, 0), slope 0 at 0              */
    FB_ACT_GELU = 2,  /* z Phi(z), Phi the normal distribution */
    FB_ACT_SILU = 3,  /* z / (1 + e^-z)                        */
    FB_ACT_SIGMOID = 4 /* 1 / (1 + e^-z), of gated layers alone */
};

/*
 * Layer norm of R rows of H elements:
 *   mean = sum x / H,  rstd = 1 / sqrt(sum (x - mean)^2 / H + eps),  y = (x - mean) rstd weight + bias
 *   x, y          [R][H] of `type`
 *   weight, bias  [H] of `wtype` (FB_TYPE_F32 or `type`), nullable (1 and 0)
 *   mean, rstd    out, float [R], nullable (what fb_layer_norm_grad takes)
 * y may be x.  FB_EINVAL: x or y NULL, R < 0, H < 1, a row distance below H, an unknown type, eps negative or not finite.
 */
int fb_layer_norm(const void *x, int64_t ldx, const void *weight, const void *bias, int wtype, int64_t R, int64_t H, int type,
                  float eps, void *y, int64_t ldy, float *mean, float *rstd, fb_stream stream);

/* Bytes of workspace fb_layer_norm_grad needs (0 on bad arguments). */
size_t fb_layer_norm_grad_workspace_bytes(int64_t R, int64_t H);

/*
 * Its gradient.  With xh = (x - mean) rstd and g = dy weight:
 *   dx = rstd (g - sum g / H - xh sum (g xh) / H),  dweight = sum over rows of dy xh,  dbias = sum over rows of dy
 *   dx              out, [R][H] of `type`, nullable; may be dy or x
 *   dweight, dbias  out, float [H], nullable
 *   ws              fb_layer_norm_grad_workspace_bytes(), needed if dweight or dbias is wanted
 * Errors as fb_layer_norm; dy, x, mean and rstd must not be NULL, the workspace not too small.
 */
int fb_layer_norm_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx, const float *mean, const float *rstd,
                       const void *weight, int wtype, int64_t R, int64_t H, int type, void *dx, int64_t lddx, float *dweight,
                       float *dbias, void *ws, size_t ws_bytes, fb_stream stream);

enum { FB_NORM_NONE = 0, FB_NORM_LAYER = 1, FB_NORM_RMS = 2 };

/*
 * From one block into the next, R rows of H elements, H at most 8192:
 *   u = norm_inner(h),  s = residual + scale gate u,  y = norm_outer(s)
 * where a norm is (FB_NORM_LAYER)  (x - mean) rstd weight + bias,  mean = sum x / H,  rstd = 1 / sqrt(sum (x - mean)^2 / H + eps),
 * (FB_NORM_RMS) the same with mean = 0, or (FB_NORM_NONE) x itself.
 *   h, residual, s, y   [R][H] of `type`; residual nullable (0), y needed unless outer is FB_NORM_NONE
 *   gate                [R][H] of `type`, or with ldg = 0 [H] of `wtype` for all rows (for one row too); nullable (1)
 *   inner_weight, inner_bias, weight, bias   [H] of `wtype` (FB_TYPE_F32 or `type`), nullable (1 and 0), only with their norm
 *   stats               out, float [4][R]: inner mean and rstd, outer mean and rstd (0 and 1 where there is no norm, mean 0 of
 *                       FB_NORM_RMS), nullable (what fb_residual_norm_grad takes)
 * y and the outer statistics are of s before its rounding.  s and y may each be h, residual or gate of rows, at the same distances.
 * FB_EINVAL: h, s or a needed y NULL, R < 0, H < 1, a row distance below H, an unknown type or norm, a weight or bias without its
 * norm, eps negative or not finite, scale not finite.  FB_EUNSUPPORTED: H above 8192.
 */
int fb_residual_norm(const void *h, int64_t ldh, const void *residual, int64_t ldr, const void *gate, int64_t ldg, float scale, int inner,
                     const void *inner_weight, const void *inner_bias, int outer, const void *weight, const void *bias, int wtype, int64_t R,
                     int64_t H, int type, float eps, void *s, int64_t lds, void *y, int64_t ldy, float *stats, fb_stream stream);

/* Bytes of workspace fb_residual_norm_grad needs (0 on bad arguments). */
size_t fb_residual_norm_grad_workspace_bytes(int64_t R, int64_t H);

/*
 * Its gradient, from those of s and y:
 *   dresidual = ds + (dy through the outer norm at s),  du = scale gate dresidual,  dh = du through the inner norm at h,
 *   dgate = scale dresidual u,  and for each norm dweight = sum over rows of dy xh,  dbias = sum over rows of dy
 *   ds           [R][H] of `type`, nullable (0) if there is an outer norm;  dy, s  [R][H] of `type`, needed if there is one
 *   h            [R][H], needed if there is an inner norm or dgate is wanted;  stats, if there is any norm, as the forward call left them
 *   dh, dresidual  out, [R][H] of `type`, nullable
 *   dgate        out, like gate: [R][H] of `type`, or with ldg = 0 float [H], the sum over rows; nullable
 *   dinner_weight, dinner_bias, dweight, dbias   out, float [H], nullable, only with their norm
 *   ws           fb_residual_norm_grad_workspace_bytes(), needed if a sum over rows is wanted
 * Outputs of rows may each be one of the inputs of rows, at the same distances.  Errors as fb_residual_norm; what is needed must not be NULL, the
 * workspace not too small.
 */
int fb_residual_norm_grad(const void *ds, int64_t ldds, const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *s, int64_t lds,
                          const float *stats, const void *gate, int64_t ldg, float scale, int inner, const void *inner_weight, const void *inner_bias,
                          int outer, const void *weight, int wtype, int64_t R, int64_t H, int type, void *dh, int64_t lddh, void *dresidual,
                          int64_t lddr, void *dgate, int64_t lddg, float *dinner_weight, float *dinner_bias, float *dweight, float *dbias, void *ws,
                          size_t ws_bytes, fb_stream stream);

/* Bytes of workspace fb_affine needs for these arguments (0: none, or bad arguments).  Of x and weight only the address counts:
 * matrices whose rows are not whole 16-byte pieces at multiples of 16 bytes are copied to such rows first (unless M <= 64).  Where
 * K is shared between workgroups the sums of each share go there too, 4 M N bytes a share: K above 4096 in FB_TYPE_F32 is always
 * shared (4096 x 4096 x 4160: 134 MB, 69120 x 3000 x 5120: 1.7 GB), otherwise products of few tiles are. */
size_t fb_affine_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type);

/*
 * Affine layer:  z = x W^T + bias,  y = act(z) + residual
 *   x         [M][K] of `type`;  weight [N][K] of `type`
 *   bias      float [N], nullable
 *   residual  [M][N] of `out_type`, nullable
 *   y         out, [M][N] of `out_type`, `type` or FB_TYPE_F32; may be residual
 *   preact    out, [M][N] of `type`, nullable: z, rounded (what fb_affine_grad takes)
 * FB_EINVAL: x, weight or y NULL, sizes or row distances out of range, an unknown type or activation, the workspace
 * missing or too small.  FB_EUNSUPPORTED: for M > 64, rows of x or weight longer than 4 MB or rows of y, residual or preact 2^27
 * elements apart or more; for M <= 64, N of 2^26 and more.
 */
int fb_affine(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, const void *residual, int64_t ldr,
              int64_t M, int64_t N, int64_t K, int type, int act, void *y, int64_t ldy, int out_type, void *preact, int64_t ldp,
              void *ws, size_t ws_bytes, fb_stream stream);

/* Bytes of workspace fb_affine_grad needs for these arguments (0: bad arguments); addresses count, and products are shared, as in
 * fb_affine_workspace_bytes (dx along N, dweight along M). */
size_t fb_affine_grad_workspace_bytes(const void *dy, int64_t lddy, int dy_type, const void *x, int64_t ldx, const void *weight, int64_t ldw,
                                      int64_t M, int64_t N, int64_t K, int type, int act);

/*
 * Its gradient:  dz = dy act'(preact),  dx = dz W,  dweight = dz^T x,  dbias = sum over rows of dz
 * (the gradient of the residual is dy itself).
 *   dy       [M][N] of `dy_type`, `type` or FB_TYPE_F32;  preact [M][N] of `type`, needed unless act is FB_ACT_NONE
 *   dx       out, [M][K] of `type`, nullable;  dweight out, [N][K] of `type`, contiguous, nullable;  dbias out, float [N], nullable
 * Where `type` has 16 bits the matrix units take dz in it: it is rounded to `type` before the two products if act or dy_type
 * makes it anything else (an error of the size of the outputs' own rounding); dbias is summed before that.  To FB_TYPE_F16 it is
 * rounded times a power of two that brings the largest finite |dy| into [2^14, 2^15), and the products are taken times its inverse, so
 * dy may be of any size; a dz below 2^-29 of the largest |dy| is off by up to 2^-39 of that.
 * Errors as fb_affine (the limits for M > 64 hold for every M, dy among them); dy, x and weight must not be NULL.
 */
int fb_affine_grad(const void *dy, int64_t lddy, int dy_type, const void *x, int64_t ldx, const void *weight, int64_t ldw,
                   const void *preact, int64_t ldp, int64_t M, int64_t N, int64_t K, int type, int act, void *dx, int64_t lddx,
                   void *dweight, float *dbias, void *ws, size_t ws_bytes, fb_stream stream);

/* Bytes of workspace fb_gated_affine needs for these arguments (0: none, or bad arguments); as fb_affine_workspace_bytes, the weight
 * having 2 N rows. */
size_t fb_gated_affine_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type);

/*
 * Gated layer:  g = x G^T + bias[0 .. N),  u = x U^T + bias[N .. 2N),  y = act(g) u, element by element
 *   x        [M][K] of `type`;  weight [2 N][K] of `type`: G's rows, then U's;  bias float [2 N], nullable
 *   act      any activation, FB_ACT_SIGMOID among them
 *   y        out, [M][N] of `type`;  preact  out, [M][2 N] of `type`, nullable: g, then u, rounded (what fb_gated_affine_grad takes)
 * y is of g and u before their rounding.  N is below 2^27.  Errors as fb_affine (FB_EUNSUPPORTED for M <= 64: N of 2^25 and more).
 */
int fb_gated_affine(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, int64_t M, int64_t N, int64_t K, int type, int act,
                    void *y, int64_t ldy, void *preact, int64_t ldp, void *ws, size_t ws_bytes, fb_stream stream);

/* Bytes of workspace fb_gated_affine_grad needs for these arguments (0: bad arguments). */
size_t fb_gated_affine_grad_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type);

/*
 * Its gradient:  dz = [dy u act'(g), dy act(g)],  dx = dz W,  dweight = dz^T x,  dbias = sum over rows of dz
 *   dy      [M][N] of `type`;  preact [M][2 N] of `type`
 *   dx      out, [M][K] of `type`, nullable;  dweight out, [2 N][K] of `type`, contiguous, nullable;  dbias out, float [2 N], nullable
 * Where `type` has 16 bits dz is rounded to it before the two products (for M <= 64, and M <= 128 if M N K <= 2^23, kept as two
 * such numbers, and products of those added), to FB_TYPE_F16 times a power of two that brings the largest
 * finite bound of |dz| into [2^14, 2^15) (as in fb_affine_grad): |dy u| and |dy| times what |act'| and |act| do not exceed for a g of
 * its sign and size; dbias is summed before that.  Such a rounding is off by up to half a step of each entry of dz (2^-8 of its size in
 * FB_TYPE_BF16, 2^-11 in FB_TYPE_F16): where many entries count the products are off by 1.4 to 1.5 times their own rounding in the 2-norm, where one
 * rules a row or a column by up to its half step beside their own rounding.
 * Errors as fb_affine_grad; dy, x, weight and preact must not be NULL.
 */
int fb_gated_affine_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *weight, int64_t ldw, const void *preact, int64_t ldp,
                         int64_t M, int64_t N, int64_t K, int type, int act, void *dx, int64_t lddx, void *dweight, float *dbias, void *ws,
                         size_t ws_bytes, fb_stream stream);

/* The most alternatives fb_token_logprobs returns a row. */
enum { FB_TOP_MAX = 64 };

/* Bytes of workspace fb_token_logprobs needs (0: none, or bad arguments). */
size_t fb_token_logprobs_workspace_bytes(int64_t R, int64_t V, int type, int top);

/*
 * For R rows of V logits and a token for each row:
 *   logz      = log sum_j e^logits[j]
 *   logprobs  = logits[token] - logz
 *   entropy   = - sum_j p_j log p_j,  p_j = e^(logits[j] - logz)
 *   top_ids, top_logprobs  the `top` largest logits' numbers, descending, equal ones in ascending order of their numbers, and
 *                          logits[.] - logz
 *   tokens    int32 [R]; a negative one marks a row that does not count (a padded frame): its logits may hold anything and all
 *             its outputs are 0 (top_ids -1)
 *   logprobs, entropy, logz   out, float [R], nullable;  top_ids int32 [R][top], top_logprobs float [R][top], needed if top > 0
 * -inf is a legal logit (an alternative that is ruled out).  A row of nothing else has logz = logprobs = top_logprobs = -inf
 * and entropy 0.  A row with NaN or +inf has NaN for logz, logprobs and entropy and unspecified alternatives; so has a row
 * whose token is V or more for logprobs alone.
 * FB_EINVAL: logits or tokens NULL, R < 0, V < 1, a row distance below V, top < 0 or above FB_TOP_MAX or V, an unknown type,
 * the workspace missing or too small.  FB_EUNSUPPORTED: rows so long and so many that their pieces of up to 16384 elements are 2^24
 * or more.
 */
int fb_token_logprobs(const void *logits, int64_t ld, const int32_t *tokens, int64_t R, int64_t V, int type, int top,
                      float *logprobs, float *entropy, float *logz, int32_t *top_ids, float *top_logprobs, void *ws,
                      size_t ws_bytes, fb_stream stream);

/*
 * Gradient of sum over rows of g_logprobs logprobs + g_entropy entropy with respect to the logits:
 *   dlogits[j] = g_logprobs ([j = token] - p_j) - g_entropy p_j (log p_j + entropy)
 *   logz, entropy          as fb_token_logprobs returned them (entropy may be NULL if g_entropy is)
 *   g_logprobs, g_entropy  float [R], either nullable
 *   dlogits                out, [R][V] of `type`; may be logits.  0 on rows that do not count and on rows whose logz is -inf
 * Errors as fb_token_logprobs.
 */
int fb_token_logprobs_grad(const void *logits, int64_t ld, const int32_t *tokens, const float *logz, const float *entropy,
                           const float *g_logprobs, const float *g_entropy, int64_t R, int64_t V, int type, void *dlogits,
                           int64_t ldd, fb_stream stream);

/* Bytes of workspace fb_affine_logprobs needs for these arguments (0: bad arguments).  Matrices whose rows are not whole 16-byte pieces
 * at multiples of 16 bytes are copied to such rows first (unless M <= 64). */
size_t fb_affine_logprobs_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t V, int64_t K, int type);

/*
 * fb_token_logprobs of the logits  x W^T + bias,  which are formed in single precision, a tile at a time, and neither rounded nor kept (over
 * a long K in shares, except where many rows of 16 bits meet many alternatives):
 *   x         [M][K] of `type`;  weight [V][K] of `type`;  bias float [V], nullable; -inf in it rules an alternative out
 *   tokens    int32 [M]; a negative one marks a row that does not count: its x may hold anything and its outputs are 0
 *   logprobs, entropy, logz   out, float [M], nullable; as in fb_token_logprobs, rows of nothing but -inf (logits below -1e38 among
 *             them), of NaN or +inf and tokens of V or more too
 * FB_EINVAL: x, weight or tokens NULL, sizes or row distances out of range, an unknown type, the workspace missing or too small.
 * FB_EUNSUPPORTED: rows of x or weight longer than 4 MB.
 */
int fb_affine_logprobs(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, const int32_t *tokens, int64_t M, int64_t V,
                       int64_t K, int type, float *logprobs, float *entropy, float *logz, void *ws, size_t ws_bytes, fb_stream stream);

/* Bytes of workspace fb_affine_logprobs_grad needs for these arguments (0: bad arguments).  The logits' gradient is formed for a piece of
 * the vocabulary at a time, of up to 512 MB of `type` (at least 256 alternatives). */
size_t fb_affine_logprobs_grad_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t V, int64_t K, int type);

/*
 * Its gradient:  dz as in fb_token_logprobs_grad, from the logits formed once more,  dx = dz W,  dweight = dz^T x,  dbias = sum over
 * rows of dz
 *   logz, entropy          as fb_affine_logprobs returned them (entropy may be NULL if g_entropy is)
 *   g_logprobs, g_entropy  float [M], either nullable
 *   dx      out, [M][K] of `type`, nullable;  dweight out, [V][K] of `type`, contiguous, nullable;  dbias out, float [V], nullable
 * Rows that do not count and rows whose logz is -inf have dx = 0 and no part in the sums.  Where `type` has 16 bits dz is rounded to it
 * before the two products (for M <= 64, and M <= 128 if M V K <= 2^24, kept as two such numbers), to FB_TYPE_F16 times a power of two for
 * the largest |g_logprobs| + |g_entropy| (0.37 + entropy), which no |dz| exceeds (as in fb_affine_grad); dbias is summed before that.
 * A dz of one number is rounded times the factor that makes the largest |g_logprobs| a power of two, and the products are taken times its inverse:
 * where all rows that count have one g_logprobs, it is not rounded then.  Each entry is off by up to half a step (2^-8 of its size in
 * FB_TYPE_BF16, 2^-11 in FB_TYPE_F16): in the 2-norm dx and dweight are off by 1.0 (one g_logprobs, small p) to 1.4 times their own
 * rounding where many rows count, and one that hangs on a single entry by up to that half step more.
 * Errors as fb_affine_logprobs; FB_EUNSUPPORTED too: rows of dx 2^27 elements apart or more.
 */
int fb_affine_logprobs_grad(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, const int32_t *tokens, const float *logz,
                            const float *entropy, const float *g_logprobs, const float *g_entropy, int64_t M, int64_t V, int64_t K, int type,
                            void *dx, int64_t lddx, void *dweight, float *dbias, void *ws, size_t ws_bytes, fb_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* FB_LAYERS_H */
