// train_api.hip -- the extern "C" entry points of include/hmoe_train.h: argument validation, workspace
// checks and dispatch to the launchers.  Host code only.
#include <float.h>
#include <math.h>

#include "checks.hpp"
#include "train_launch.hpp"

using namespace hmoe;

extern "C" {

static int check_train_ws(size_t need, size_t have, const void* ws) {
  HMOE_TRY(check_ws(need, have, ws));
  return need > 0 ? check_ptr("workspace", ws) : HMOE_OK;
}

static int check_finite(const char* name, float v) {
  return isfinite(v) ? HMOE_OK : fail(HMOE_EINVAL, "%s = %g is not finite", name, (double)v);
}
static int check_not_negative(const char* name, float v) {
  return isfinite(v) && v >= 0.f ? HMOE_OK : fail(HMOE_EINVAL, "%s = %g is negative or not finite", name, (double)v);
}

// ------------------------------------------------------------------ router of a batch

static int check_router(const hmoe_router_t* p, int64_t n) {
  if (!p) return fail(HMOE_EINVAL, "params are NULL");
  HMOE_TRY(check_dtype(p->dt));
  HMOE_TRY(check_k(p->K));
  HMOE_TRY(check_width("d", p->d));
  if (p->d > HMOE_ROUTER_WIDTH) return fail(HMOE_EINVAL, "d = %d exceeds %d", p->d, HMOE_ROUTER_WIDTH);
  if (p->top_k < 1 || p->top_k > HMOE_ROUTER_EXPERTS || p->top_k > p->K)
    return fail(HMOE_EINVAL, "top_k = %d outside [1, min(%d, K)]", p->top_k, HMOE_ROUTER_EXPERTS);
  if (n < 0 || n > HMOE_ROUTER_ROWS) return fail(HMOE_EINVAL, "n = %lld outside [0, %d]", (long long)n, HMOE_ROUTER_ROWS);
  return HMOE_OK;
}

size_t hmoe_router_workspace(const hmoe_router_t* p, int64_t n) {
  if (check_router(p, n) != HMOE_OK || n == 0) {
    clear_error();
    return 0;
  }
  return router_ws(p, n);
}

int hmoe_router_forward(const hmoe_router_t* p, int64_t n, const void* X, int32_t* expert, float* weight,
                        float* scores, int32_t* counts, float* share, float* loss, void* ws, size_t ws_bytes,
                        void* stream) {
  clear_error();
  HMOE_TRY(check_router(p, n));
  HMOE_TRY(check_ptr("counts", counts, false));
  HMOE_TRY(check_ptr("share", share, false));
  HMOE_TRY(check_ptr("loss", loss, false));
  if (n > 0) {
    HMOE_TRY(check_ptr("R", p->R));
    HMOE_TRY(check_ptr("X", X));
    HMOE_TRY(check_ptr("expert", expert, false));
    HMOE_TRY(check_ptr("weight", weight, false));
    HMOE_TRY(check_ptr("scores", scores));
    HMOE_TRY(check_train_ws(router_ws(p, n), ws_bytes, ws));
  }
  Workspace w(ws, ws_bytes);
  return launch_router_forward(p, n, X, expert, weight, scores, counts, share, loss, w, (hipStream_t)stream);
}

int hmoe_router_backward(const hmoe_router_t* p, int64_t n, const void* X, const float* scores, const int32_t* expert,
                         const int32_t* counts, const float* g_weight, float balance, float z, void* dX, float* dR,
                         float* dbias, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_router(p, n));
  HMOE_TRY(check_finite("balance", balance));
  HMOE_TRY(check_finite("z", z));
  if (dR) HMOE_TRY(check_ptr("dR", dR));
  if (dbias) HMOE_TRY(check_ptr("dbias", dbias, false));
  if (n > 0) {
    HMOE_TRY(check_ptr("scores", scores));
    HMOE_TRY(check_ptr("counts", counts, false));
    if (g_weight) HMOE_TRY(check_ptr("expert", expert, false));
    if (dX) {
      HMOE_TRY(check_ptr("dX", dX));
      HMOE_TRY(check_ptr("R", p->R));
    }
    if (dR) HMOE_TRY(check_ptr("X", X));
    HMOE_TRY(check_train_ws(router_ws(p, n), ws_bytes, ws));
    if (!dX && !dR && !dbias) return HMOE_OK;
    if (dX && dR && dX == X) return fail(HMOE_EINVAL, "dX is X, which dR still reads");
    Workspace w(ws, ws_bytes);
    return launch_router_backward(p, n, X, scores, expert, counts, g_weight, balance, z, dX, dR, dbias, w,
                                  (hipStream_t)stream);
  }
  // no rows: the router's gradients are zeros
  if (dR) HMOE_TRY(launch_zero_f32(dR, (int64_t)p->K * p->d, (hipStream_t)stream));
  if (dbias) HMOE_TRY(launch_zero_f32(dbias, p->K, (hipStream_t)stream));
  return HMOE_OK;
}

// ------------------------------------------------------------------ join with the residual stream

static int check_join(const hmoe_join_t* p, int64_t n) {
  if (!p) return fail(HMOE_EINVAL, "params are NULL");
  HMOE_TRY(check_dtype(p->dt));
  HMOE_TRY(check_width("d", p->d));
  if (p->d > HMOE_JOIN_WIDTH) return fail(HMOE_EINVAL, "d = %d exceeds %d", p->d, HMOE_JOIN_WIDTH);
  if (p->k < 0 || p->k > HMOE_JOIN_ROWS) return fail(HMOE_EINVAL, "k = %d outside [0, %d]", p->k, HMOE_JOIN_ROWS);
  HMOE_TRY(check_finite("scale", p->scale));
  // below them 1 / eps, the square of a row of zeros' factor, is past fp32
  if (!(p->eps >= FLT_MIN) || !isfinite(p->eps))
    return fail(HMOE_EINVAL, "eps = %g is not positive and normal", (double)p->eps);
  if (p->gamma_y) HMOE_TRY(check_ptr("gamma_y", p->gamma_y));
  if (p->gamma_h) HMOE_TRY(check_ptr("gamma_h", p->gamma_h));
  return check_n(n);
}

int hmoe_join_forward(const hmoe_join_t* p, int64_t n, const void* x, const void* y, const float* gate, void* x_out,
                      void* h, void* stream) {
  clear_error();
  HMOE_TRY(check_join(p, n));
  if (n == 0) return HMOE_OK;
  HMOE_TRY(check_ptr("x", x));
  if (p->k > 0) HMOE_TRY(check_ptr("y", y));
  if (x_out) HMOE_TRY(check_ptr("x_out", x_out));
  if (h) HMOE_TRY(check_ptr("h", h));
  if (!x_out && !h) return fail(HMOE_EINVAL, "x_out and h are both NULL");
  if (h && (h == x_out || h == x || (p->k > 0 && h == y))) return fail(HMOE_EINVAL, "h overlaps another row");
  if (p->k > 1 && x_out == y) return fail(HMOE_EINVAL, "x_out is y, rows of which are still read");
  return launch_join_forward(p, n, x, y, gate, x_out, h, (hipStream_t)stream);
}

size_t hmoe_join_workspace(const hmoe_join_t* p, int64_t n) {
  if (check_join(p, n) != HMOE_OK || n == 0) {
    clear_error();
    return 0;
  }
  return join_ws(p, n);
}

int hmoe_join_backward(const hmoe_join_t* p, int64_t n, const void* x_out, const void* y, const float* gate,
                       const void* dx_out, const void* dh, void* dx, void* dy, float* dgate, float* dgamma_y,
                       float* dgamma_h, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_join(p, n));
  if ((dy || dgate || dgamma_y) && p->k == 0) return fail(HMOE_EINVAL, "gradients of y with k = 0");
  if (n > 0) {
    if (dh) HMOE_TRY(check_ptr("x_out", x_out));
    if (dx_out) HMOE_TRY(check_ptr("dx_out", dx_out));
    if (dh) HMOE_TRY(check_ptr("dh", dh));
    if (dy || dgate || dgamma_y) HMOE_TRY(check_ptr("y", y));
    if (dx) HMOE_TRY(check_ptr("dx", dx));
    if (dy) HMOE_TRY(check_ptr("dy", dy));
    if (dx && dx == dy) return fail(HMOE_EINVAL, "dx and dy are the same");
    HMOE_TRY(check_train_ws(join_ws(p, n), ws_bytes, ws));
    if (dx && dx == y && (dy || dgate || dgamma_y)) return fail(HMOE_EINVAL, "dx is y, which is still read");
    if (dy && p->k > 1 && ((dh && dy == x_out) || dy == dx_out || dy == dh))
      return fail(HMOE_EINVAL, "dy is x_out, dx_out or dh, rows of which are still read");
    Workspace w(ws, ws_bytes);
    return launch_join_backward(p, n, x_out, y, gate, dx_out, dh, dx, dy, dgate, dgamma_y, dgamma_h, w,
                                (hipStream_t)stream);
  }
  if (dgamma_y) HMOE_TRY(launch_zero_f32(dgamma_y, p->d, (hipStream_t)stream));
  if (dgamma_h) HMOE_TRY(launch_zero_f32(dgamma_h, p->d, (hipStream_t)stream));
  return HMOE_OK;
}

// ------------------------------------------------------------------ orthogonalised updates

static int check_ortho(int32_t K, int32_t rows, int32_t cols) {
  HMOE_TRY(check_k(K));
  HMOE_TRY(check_width("cols", cols));
  if (rows < 1) return fail(HMOE_EINVAL, "rows = %d is not positive", rows);
  if (rows > HMOE_ORTHO_WIDTH || cols > HMOE_ORTHO_WIDTH)
    return fail(HMOE_EINVAL, "rows = %d or cols = %d exceeds %d", rows, cols, HMOE_ORTHO_WIDTH);
  if (rows > HMOE_ORTHO_RANK && cols > HMOE_ORTHO_RANK)
    return fail(HMOE_EINVAL, "the smaller of rows = %d and cols = %d exceeds %d", rows, cols, HMOE_ORTHO_RANK);
  return HMOE_OK;
}

static int check_steps(int32_t steps, const float* coef) {
  if (steps < 1 || steps > HMOE_ORTHO_STEPS) return fail(HMOE_EINVAL, "steps = %d outside [1, %d]", steps, HMOE_ORTHO_STEPS);
  if (!coef) return fail(HMOE_EINVAL, "coef is NULL");
  for (int i = 0; i < 3; ++i) HMOE_TRY(check_finite("coef", coef[i]));
  return HMOE_OK;
}

size_t hmoe_orthogonalise_workspace(int32_t K, int32_t rows, int32_t cols, hmoe_dtype_t dt) {
  if (check_ortho(K, rows, cols) != HMOE_OK || check_dtype(dt) != HMOE_OK) {
    clear_error();
    return 0;
  }
  return ortho_ws(K, rows, cols);
}

int hmoe_orthogonalise(const void* G, hmoe_dtype_t dt, int32_t K, int32_t rows, int32_t cols, int32_t steps,
                       const float* coef, void* O, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_dtype(dt));
  HMOE_TRY(check_ortho(K, rows, cols));
  HMOE_TRY(check_steps(steps, coef));
  HMOE_TRY(check_ptr("G", G));
  HMOE_TRY(check_ptr("O", O));
  HMOE_TRY(check_train_ws(ortho_ws(K, rows, cols), ws_bytes, ws));
  OrthoStep s = {};
  s.G = G;
  s.O = O;
  s.dt = dt;
  Workspace w(ws, ws_bytes);
  return launch_ortho(s, K, rows, cols, steps, coef, w, (hipStream_t)stream);
}

size_t hmoe_muon_workspace(int32_t K, int32_t rows, int32_t cols) {
  return hmoe_orthogonalise_workspace(K, rows, cols, HMOE_F32);
}

int hmoe_muon_step(float* w, const float* g, float* v, void* w_lo, hmoe_dtype_t dt, int32_t K, int32_t rows,
                   int32_t cols, float lr, float weight_decay, float momentum, int32_t nesterov, float scale,
                   int32_t steps, const float* coef, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_dtype(dt));
  HMOE_TRY(check_ortho(K, rows, cols));
  HMOE_TRY(check_steps(steps, coef));
  HMOE_TRY(check_not_negative("lr", lr));
  HMOE_TRY(check_not_negative("weight_decay", weight_decay));
  HMOE_TRY(check_not_negative("momentum", momentum));
  HMOE_TRY(check_finite("scale", scale));
  HMOE_TRY(check_ptr("w", w));
  HMOE_TRY(check_ptr("g", g));
  if (momentum > 0.f) HMOE_TRY(check_ptr("v", v));
  if (v) HMOE_TRY(check_ptr("v", v));
  if (w_lo) HMOE_TRY(check_ptr("w_lo", w_lo));
  if (w_lo == w) return fail(HMOE_EINVAL, "w_lo is w");
  HMOE_TRY(check_train_ws(ortho_ws(K, rows, cols), ws_bytes, ws));
  // g is read once more after v is written, and w_lo's matrices are written where others' g and v may be read
  if (momentum > 0.f && (v == g || v == w)) return fail(HMOE_EINVAL, "v is g or w");
  if (w_lo && (w_lo == g || (momentum > 0.f && w_lo == v))) return fail(HMOE_EINVAL, "w_lo is g or v");
  OrthoStep s = {};
  s.w = w;
  s.g = g;
  s.v = momentum > 0.f ? v : nullptr;  // as hmoe_sgd_step, which leaves it alone without momentum
  s.w_lo = w_lo;
  s.dt = dt;
  s.momentum = momentum;
  s.keep = (float)(1.0 - (double)lr * weight_decay);
  s.rate = (float)((double)lr * scale);
  s.nesterov = nesterov != 0;
  Workspace space(ws, ws_bytes);
  return launch_ortho(s, K, rows, cols, steps, coef, space, (hipStream_t)stream);
}

}  // extern "C"
