/*
 * lc_head.h - C ABI of the supervised head: what learns to answer from the features that the layers of lc.h learn.
 *
 * The data set of Sec. 2 comes with its users' tags, a vocabulary of tens of thousands of words.  A head turns the
 * learned features into scores for them: a gated hidden layer (glu), a softmax over the vocabulary with its cross
 * entropy and gradients (xent), and the clipping of all gradients by their common norm (grad_clip).  Beside these: what the
 * softmax answers, log probabilities of given words, entropies and likeliest words, with gradients (logp); steps along the
 * orthogonalised momentum of a matrix (muon); and products and the gated layer with weights of 8 bits (q8).
 *
 * Conventions: those of lc.h (status codes, caller-owned device memory, scratch passed in as ws / ws_bytes, work only
 * enqueued on hip_stream, arguments checked on the host before anything is launched), with these of its own:
 *  - Matrices are row-major and contiguous.  Weights are [outputs][inputs], one output's weights contiguous.
 *  - `dtype` is the type of every matrix of a call, results and gradients included: each is an operand of the next
 *    call.  Sums are formed in fp32 and rounded once.  Losses, costs, norms, log probabilities, entropies and momenta are fp32.
 *  - With bf16 operands three numbers inside a call are rounded as well.  g and u are kept for glu_bwd in 16 bits (see
 *    glu_fwd), the softmax's exponentials in ten significant bits; and dg, du and the softmax's d meet the bf16 operands of
 *    the last products as bf16, for up to 32 rows as sixteen bits, because the roundings of few numbers do not average out.
 *  - Widths D, F and V are 1 to 2^20, N is 0 to 2^24 (LC_EINVAL otherwise).
 *  - A batch may have no rows (N = 0): weight gradients and costs are then zero; matrices without rows may be NULL.
 *  - Results do not depend on the workspace's contents and are the same bit for bit from call to call.
 *  - fp32 products are formed from three bf16 parts of each operand, which hold all of its bits down to 2^-133 (what an
 *    operand has below that is not counted), and again with the fp32 matrix instruction where an operand is infinite or
 *    NaN or a sum overflows on the way.
 */
#ifndef LC_HEAD_H_
#define LC_HEAD_H_

#include "lc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations of the gated layer: 1/(1+e^-g), g/(1+e^-g), g Phi(g) with the normal distribution function Phi. */
enum lc_act { LC_ACT_SIGMOID = 0, LC_ACT_SILU = 1, LC_ACT_GELU = 2 };

/* Host only.  Scratch for glu_fwd (backward = 0), or for glu_fwd and glu_bwd (backward = 1); 0 for invalid arguments.
 * Both calls of one step may be given the same scratch.  What is enough for N rows is enough for fewer. */
size_t glu_workspace_bytes(int32_t N, int32_t D, int32_t F, int dtype, int backward);

/* Gated layer: g = x wg^T, u = x wu^T, h = act(g) * u.
 * x [N][D], wg and wu [F][D], h [N][F].  gu NULL or [N][2][F] values of dtype's size: receives g and u for glu_bwd, as they
 * are for fp32, in a 16-bit code of the library's own for bf16 (ten significant bits for magnitudes from 2^-16 to 2^16,
 * seven for others). */
int glu_fwd(const void *x, const void *wg, const void *wu, void *h, void *gu, int32_t N, int32_t D, int32_t F, int act,
            int dtype, void *ws, size_t ws_bytes, void *hip_stream);

/* Gradients of glu_fwd for dh = dcost/dh, with gu from glu_fwd:
 *   dg = dh * u * act'(g), du = dh * act(g);  dx = dg wg + du wu, dwg = dg^T x, dwu = du^T x, all overwritten.
 * dx may be NULL (frozen features). */
int glu_bwd(const void *x, const void *wg, const void *wu, const void *gu, const void *dh, void *dx, void *dwg,
            void *dwu, int32_t N, int32_t D, int32_t F, int act, int dtype, void *ws, size_t ws_bytes,
            void *hip_stream);

/* Host only.  Scratch for xent_fwd (grads = 0) or xent_fwd_bwd (grads = 1); 0 for invalid arguments.  What is enough for N
 * rows is enough for fewer, with gradients also for the loss alone.  It holds no
 * [N][V] array without bound: with gradients what is kept of at most 2 GiB worth of rows at a time (fp32: of their scores,
 * with another 3 GiB of planes), none without. */
size_t xent_workspace_bytes(int32_t N, int32_t D, int32_t V, int dtype, int grads);

/* Softmax cross entropy over a vocabulary of V words, projection included:
 *   l[n][v] = sum_d x[n][d] w[v][d];  loss[n] = log sum_v exp(l[n][v]) - l[n][target[n]] for target[n] >= 0, else 0;
 *   cost = sum_n s[n] loss[n], s[n] = scale[n], or 1 / (number of targets >= 0) if scale is NULL.
 * x [N][D], w [V][D], target [N] int64 (8-byte aligned: any part of a longer list), scale NULL or [N] fp32; loss [N] and
 * cost [1] fp32.
 * A row with a negative target is masked: its x and scale are not looked at.  With no row left the cost is 0.
 * A target >= V makes the loss of its row, the cost and the gradients it enters NaN. */
int xent_fwd(const void *x, const void *w, const int64_t *target, const float *scale, float *loss, float *cost,
             int32_t N, int32_t D, int32_t V, int dtype, void *ws, size_t ws_bytes, void *hip_stream);

/* xent_fwd and the gradients of cost: with d[n][v] = s[n] (exp(l[n][v] - logsumexp) - [v = target[n]]),
 *   dx = d w (zero in masked rows), dw = d^T x, both overwritten.  dx may be NULL. */
int xent_fwd_bwd(const void *x, const void *w, const int64_t *target, const float *scale, float *loss, float *cost,
                 void *dx, void *dw, int32_t N, int32_t D, int32_t V, int dtype, void *ws, size_t ws_bytes,
                 void *hip_stream);

/* One tensor of a list: n values of type dtype at src, and where the clipped values go (src itself, or elsewhere; no
 * other overlap).  Pointers need the alignment of one value only.  The list is host memory, read during the call. */
typedef struct {
    const void *src;
    void *dst;
    int64_t n;
    int32_t dtype;
} lc_tensor_t;

/* Host only.  Scratch for grad_norm and grad_clip of a list of `count` tensors that hold at most `values` values together; 0
 * for invalid arguments. */
size_t grad_clip_workspace_bytes(int64_t values, int32_t count);

/* norm[0] = sqrt(sum of the squares of all values of all tensors), summed in 64 bits.  dst is not looked at. */
int grad_norm(const lc_tensor_t *list, int32_t count, float *norm, void *ws, size_t ws_bytes, void *hip_stream);

/* grad_norm, then every tensor times min(1, max_norm / norm) into its dst.  Where the norm is not finite in 64 bits (a
 * value is infinite or NaN) the factor is 1: norm[0] says so and nothing is spread.  A finite norm beyond fp32's range clips all
 * the same, with norm[0] infinite.  max_norm > 0. */
int grad_clip(const lc_tensor_t *list, int32_t count, float max_norm, float *norm, void *ws, size_t ws_bytes,
              void *hip_stream);

/* Weights of 8 bits.  A row of values x is held as whole numbers q, -127 to 127, and a scale s: s = max |x| / 127, but at least 2^-126; q = x / s,
 * to nearest, ties to even; q s stands for x.  A row of q takes q8_row_bytes(D) bytes: D rounded up to whole blocks of 128, zeros behind the last
 * value.  A row with an infinite or NaN value has scale NaN, and so have all results that it enters.
 * Widths D of these operators are 1 to 2^17. */

/* Host only.  Bytes of a row of D values; 0 for invalid D. */
int q8_row_bytes(int32_t D);

/* x [N][D] of type dtype to q [N][q8_row_bytes(D)] and scale [N] fp32: weights, once. */
int q8_rows(const void *x, int8_t *q, float *scale, int32_t N, int32_t D, int dtype, void *hip_stream);

/* Host only.  Scratch for q8_matmul and q8_glu_fwd; 0 for invalid arguments.  What is enough for N rows is enough for fewer. */
size_t q8_workspace_bytes(int32_t N, int32_t D, int32_t F, int dtype);

/* y[n][f] = s[n] scale[f] sum_d p[n][d] q[f][d], with p, s the 8-bit form of x, formed by the call.  x [N][D] and y [N][F] of type
 * dtype, q [F][q8_row_bytes(D)], scale [F] as from q8_rows.  The sum is exact; it, and its product with each scale, is rounded to fp32. */
int q8_matmul(const void *x, const int8_t *q, const float *scale, void *y, int32_t N, int32_t D, int32_t F, int dtype,
              void *ws, size_t ws_bytes, void *hip_stream);

/* glu_fwd with 8-bit weights: h = act(g) * u, with g and u as q8_matmul gives them in fp32, from qg, sg and qu, su. */
int q8_glu_fwd(const void *x, const int8_t *qg, const float *sg, const int8_t *qu, const float *su, void *h, int32_t N,
               int32_t D, int32_t F, int act, int dtype, void *ws, size_t ws_bytes, void *hip_stream);

/* Host only.  Scratch for logp_fwd (grads = 0), or for logp_fwd and logp_bwd (grads = 1); 0 for invalid arguments.  What is enough for N rows is
 * enough for fewer, and what is for K words for fewer.  T: words given with each row, 0 to 64; K: likeliest words asked for, 0 to 64 and no more than V.  It is bounded for any
 * number of rows but for what a few numbers and, laid out, x take. */
size_t logp_workspace_bytes(int32_t N, int32_t D, int32_t V, int32_t T, int32_t K, int dtype, int grads);

/* What a softmax over V words says, projection included: with l[n][v] = sum_d x[n][d] w[v][d] and p = softmax(l),
 *   logp[n][t] = log p[n][tags[n][t]], 0 where the tag is negative;  entropy[n] = -sum_v p log p;
 *   top[n][0 .. K-1]: the words of the K largest scores, largest first, equal ones by their number; top_logp: their log p.
 * x [N][D], w [V][D]; tags [N][T] int64 (8-byte aligned; NULL if T = 0), logp [N][T], entropy NULL or [N], top [N][K] int64 and top_logp [N][K]
 * (NULL if K = 0), all fp32 but for top.  state NULL or [N][3] fp32: receives what logp_bwd needs of the softmax.
 * Where words are given (T > 0), a row without one (all tags negative) is masked: its x is not looked at, its numbers are 0 and its top is -1.
 * A tag >= V has logp NaN.  A row with a NaN score, a score of +inf or none above -inf has no distribution: its numbers are NaN, its top is -1.
 * Scores of given and likeliest words are formed in 64 bits, and so is their order.  Where more than 256 words, and more than 32 K, come
 * as near to the K-th score as the product's sums tell scores apart (some 2^-16 of it), which of these follow is decided by those sums; and so it is
 * where the terms of scores cancel so far that their fp32 sums are off by more than that. */
int logp_fwd(const void *x, const void *w, const int64_t *tags, float *logp, float *entropy, int64_t *top, float *top_logp,
             float *state, int32_t N, int32_t D, int32_t V, int32_t T, int32_t K, int dtype, void *ws, size_t ws_bytes,
             void *hip_stream);

/* Gradients of sum dlogp logp + sum dentropy entropy, for given dlogp [N][T] (not looked at where the tag is negative) and dentropy (NULL or [N]), fp32,
 * with x, w, tags as in logp_fwd and logp and state from it:
 *   d[n][v] = sum of dlogp[n][t] over t with tags[n][t] = v - p[n][v] (sum_t dlogp[n][t] + dentropy[n] (log p[n][v] + entropy[n])),
 *   dx = d w (zero in masked rows), dw = d^T x, both overwritten.  dx may be NULL.
 * A row with a tag >= V, or without a distribution, makes the gradients it enters NaN. */
int logp_bwd(const void *x, const void *w, const int64_t *tags, const float *logp, const float *state, const float *dlogp,
             const float *dentropy, void *dx, void *dw, int32_t N, int32_t D, int32_t V, int32_t T, int dtype, void *ws,
             size_t ws_bytes, void *hip_stream);

/* Host only.  Scratch for muon_step; 0 for invalid arguments.  What is enough for a stack is enough for a shorter one.  It is bounded for
 * any number of matrices (4 GiB, or what one matrix takes). */
size_t muon_workspace_bytes(int32_t count, int32_t rows, int32_t cols, int dtype);

/* A step of gradient descent on each matrix of a stack [count][rows][cols] with an orthogonalised update:
 *   m' = momentum m + g;  u = g + momentum m' (nesterov) or m';  X = u / |u|, its 2-norm over all values of the matrix;
 *   `steps` times: A = X X^T, X = 3.4445 X + (-4.7750 A + 2.0315 A A) X;  w_out = (1 - decay) w - rate X,  m_out = m'.
 * w, g and w_out are of type dtype, m and m_out fp32.  w_out may be w and m_out may be m; no other overlap.  The untied filters of a
 * layer, [LH][LW][K][F], are a stack of LH LW matrices.  A matrix u of zeros has the update 0; one with an infinite or NaN value makes all of its
 * matrix of w_out NaN.
 * Between products X is held in fp16 for bf16 weights (scaled, so that all of its 11 bits count), and in 22 bits for fp32 weights.
 * count is 0 to 2^24, sides 1 to 2^20, the smaller one at most 2^15, all values at most 2^40; steps 1 to 32. */
int muon_step(const void *w, const void *g, const float *m, void *w_out, float *m_out, int32_t count, int32_t rows,
              int32_t cols, float rate, float decay, float momentum, int nesterov, int32_t steps, int dtype, void *ws,
              size_t ws_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* LC_HEAD_H_ */
