/*
 * hmoe_train.h -- C ABI of the operators that train mixtures whose router learns, in layers: the router
 * of a batch with its balance losses and gradients, the join of a layer's output with the residual
 * stream and the norms around it, and updates of weight matrices that are made orthogonal.
 *
 * The conventions are hmoe.h's and hmoe_lm.h's: device pointers (where not said otherwise), the caller's
 * workspace, 16-byte aligned, one stream, no allocation, no state and no host synchronisation, argument errors
 * before any launch (hmoe_last_error), HMOE_F32 or HMOE_BF16 data with sums in fp32 or wider, calls that can
 * be captured into HIP graphs.  Results are the same from call to call: no sum depends on the order in which
 * workgroups finish.
 */
#ifndef HMOE_TRAIN_H_
#define HMOE_TRAIN_H_

#include "hmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ router of a batch */

#define HMOE_ROUTER_EXPERTS 8     /* most experts of a sample */
#define HMOE_ROUTER_WIDTH (1 << 20) /* largest d */
#define HMOE_ROUTER_ROWS (1 << 28)  /* largest n */

/* A learned router: R [K][d] in dtype dt, bias float[K] or NULL, 1 <= top_k <= min(HMOE_ROUTER_EXPERTS, K).
 * d is a multiple of 8, 1 <= K <= 4096.  The scores and choices are hmoe_moe_few's, for any number of
 * samples; renorm as there: */
typedef struct {
  int32_t K, d, top_k;
  hmoe_dtype_t dt;
  int32_t renorm; /* weights: 0: the chosen experts' probabilities among all K; otherwise: a softmax over the
                   * chosen scores */
  const void* R;
  const float* bias;
} hmoe_router_t;

/* For row i of X [n x d]:
 *   s_e = R_e . x + bias[e], p = softmax(s) over the K experts;
 *   expert[i][0 .. top_k) = the top_k largest scores in decreasing order, equal ones in increasing e (NaN
 *   ranks last), weight[i][j] = p of the choice, or with renorm its share among the choices;
 * and of the batch
 *   counts[e] = choices of expert e,  share[e] = mean_i p_ie,
 *   loss[0] = K sum_e counts[e] / (n top_k) share[e]  (1 where counts and shares are even),
 *   loss[1] = mean_i (ln sum_e exp s_ie)^2.
 * An expert with a score of -inf (bias[e] = -inf: it is off) has probability and weight 0, and a choice of
 * it, where a row has fewer others than top_k, is not counted.  A row of nothing else adds nothing to shares and
 * losses.  A row with NaN or +inf makes its weights, the shares and the losses NaN; choices that are not NaN count.
 *   expert int32[n][top_k], weight float[n][top_k], scores float[n][K], counts int32[K], share float[K],
 *   loss float[2]: out; all of them are needed.  n may be 0: counts, share and loss are zeros.
 * Errors: HMOE_EINVAL (K, top_k, n or d out of range, NULL pointer), HMOE_ESHAPE (d not a multiple of 8,
 * misaligned X, R or scores), HMOE_EDTYPE, HMOE_EWORKSPACE. */
size_t hmoe_router_workspace(const hmoe_router_t* p, int64_t n); /* of both directions */
int hmoe_router_forward(const hmoe_router_t* p, int64_t n, const void* X, int32_t* expert, float* weight,
                        float* scores, int32_t* counts, float* share, float* loss, void* ws, size_t ws_bytes,
                        void* stream);

/* Gradients of  sum_ij g_weight[i][j] weight[i][j] + balance loss[0] + z loss[1]  (counts are constants):
 *   ds_i = w-part + p (q - p.q) + 2 z lse_i p / n,  q_e = balance K counts[e] / (n^2 top_k), plus g_weight[i][j] at
 *   the choices (renorm: w-part_j = weight_j (g_weight_j - sum_j weight_j g_weight_j) at the choices instead);
 *   dX = ds R (dtype dt), dR = ds^T X, dbias = sum_i ds_i (float).
 *   scores, expert and counts are the forward's; an expert id outside [0, K) is no choice.  g_weight
 *   float[n][top_k] or NULL (zeros).  dX, dR and dbias may each be NULL.  Experts that are off get zeros, and rows
 *   of nothing else too.  ds is held to fp32's accuracy.
 *   balance and z are finite.  dX may not be X with dR. */
int hmoe_router_backward(const hmoe_router_t* p, int64_t n, const void* X, const float* scores, const int32_t* expert,
                         const int32_t* counts, const float* g_weight, float balance, float z, void* dX, float* dR,
                         float* dbias, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ join with the residual stream */

#define HMOE_JOIN_ROWS 8          /* largest k */
#define HMOE_JOIN_WIDTH (1 << 15) /* largest d */

/* Where a layer ends and the next one begins.  With N(t) = t / sqrt(mean(t^2) + eps):
 *   x'_i = scale x_i + sum_{j < k} gate[i][j] gamma_y N(y_ij)     (norm_y = 0: y_ij itself instead of N(y_ij))
 *   h_i  = gamma_h N(x'_i)
 * k rows of y belong to a sample: one for a dense layer, those of its experts (0 <= k <= HMOE_JOIN_ROWS).  d is a
 * multiple of 8 up to HMOE_JOIN_WIDTH; gamma_y, gamma_h [d] in dtype dt or NULL (ones); eps >= 2^-126, the
 * smallest normal number. */
typedef struct {
  int32_t d, k;
  hmoe_dtype_t dt;
  int32_t norm_y;
  float scale, eps;
  const void *gamma_y, *gamma_h;
} hmoe_join_t;

/* x [n x d], y [n][k][d] (NULL if k = 0), gate float[n][k] or NULL (ones); x_out (x') and h [n x d] out, either
 * may be NULL; x_out may be x, but not y with k > 1.  h is the norm of x' before its rounding.  One pass, sums in fp32, no workspace.
 * Errors (of both): HMOE_EINVAL, HMOE_ESHAPE (d not a multiple of 8, misaligned rows), HMOE_EDTYPE. */
int hmoe_join_forward(const hmoe_join_t* p, int64_t n, const void* x, const void* y, const float* gate, void* x_out,
                      void* h, void* stream);

/* Gradients, with dx_out and dh those of x' and h (dtype dt, either may be NULL: zeros), x_out the rounded x' of the
 * forward (needed with dh), D = dx_out + the gradient through h's norm at x_out:
 *   dx = scale D;  dy_ij = gate gamma_y D through the norm at y_ij;  dgate[i][j] = D . gamma_y N(y_ij);
 *   dgamma_y = sum_ij gate D N(y_ij), dgamma_h = sum_i dh N(x'_i).
 * dx, dy (dtype dt), dgate, dgamma_y, dgamma_h (float) may each be NULL.  dx may be dx_out or dh, and dy may be
 * y; other results over inputs are not allowed (HMOE_EINVAL where dx is y, or dy another input with k > 1).
 * dgate, dgamma_y and dy need y (k > 0). */
size_t hmoe_join_workspace(const hmoe_join_t* p, int64_t n); /* of the backward */
int hmoe_join_backward(const hmoe_join_t* p, int64_t n, const void* x_out, const void* y, const float* gate,
                       const void* dx_out, const void* dh, void* dx, void* dy, float* dgate, float* dgamma_y,
                       float* dgamma_h, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ orthogonalised updates */

#define HMOE_ORTHO_WIDTH (1 << 21) /* largest of rows and cols */
#define HMOE_ORTHO_RANK (1 << 15)  /* largest min(rows, cols) */
#define HMOE_ORTHO_STEPS 32

/* Newton-Schulz iterations: for each of K matrices U [rows][cols], X = U / |U| (the Frobenius norm; zeros stay
 * zeros), then `steps` times
 *   X <- a X + (b A + c A^2) X,  A = X X^T  (X^T X on the other side where rows > cols: the same),
 * (a, b, c) = coef, which takes the singular values s of X to a s + b s^3 + c s^5: with (3.4445, -4.775, 2.0315) five
 * steps bring those in [0.01, 1] to [0.7, 1.2], so that X comes near to the orthogonal factor of U.
 * Iterates are kept as two fp16 numbers a value, 22 bits, and products summed in fp32, of bf16 data, too, whose result
 * is that of the same numbers in fp32, rounded.  Two steps may be taken at once, with P = a + b A + c A^2, the next A =
 * P A P and the product of two such P.  K, rows and cols choose the tiles and how sums are divided among them, and so a
 * result's last bits.  Entries of X have to stay below 8 in magnitude, those of A, b A + c A^2 and P below 16 and those of
 * products of two of them below 256; larger ones become infinities and NaN.  A matrix with infinities or NaN gives NaN and
 * leaves the others as they are.
 * cols is a multiple of 8; 1 <= K <= 4096, 1 <= steps <= HMOE_ORTHO_STEPS, coef: three finite floats on the host.
 * hmoe_orthogonalise: G [K][rows][cols] in dtype dt, O the same out; O may be G.
 * Errors (of both): HMOE_EINVAL, HMOE_ESHAPE (cols not a multiple of 8, misaligned pointer), HMOE_EDTYPE,
 * HMOE_EWORKSPACE. */
size_t hmoe_orthogonalise_workspace(int32_t K, int32_t rows, int32_t cols, hmoe_dtype_t dt);
int hmoe_orthogonalise(const void* G, hmoe_dtype_t dt, int32_t K, int32_t rows, int32_t cols, int32_t steps,
                       const float* coef, void* O, void* ws, size_t ws_bytes, void* stream);

/* One step of K weight matrices with such updates, beside hmoe_sgd_step for vectors:
 *   v = momentum v + g;  U = g + momentum v (nesterov) or v;  w = (1 - lr weight_decay) w - lr scale NS(U).
 * w, v float[K][rows][cols] in/out, g float in; v is not used, and may be NULL, when momentum == 0 (U = g).
 * w_lo out in dtype dt (the updated weights rounded to nearest even) or NULL.  v, g and w_lo are not each other, and v and
 * w_lo not w (HMOE_EINVAL).  lr, weight_decay, momentum >= 0, scale finite. */
size_t hmoe_muon_workspace(int32_t K, int32_t rows, int32_t cols);
int hmoe_muon_step(float* w, const float* g, float* v, void* w_lo, hmoe_dtype_t dt, int32_t K, int32_t rows,
                   int32_t cols, float lr, float weight_decay, float momentum, int32_t nesterov, float scale,
                   int32_t steps, const float* coef, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* HMOE_TRAIN_H_ */
