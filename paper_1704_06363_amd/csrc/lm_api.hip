// lm_api.hip -- the extern "C" entry points of include/hmoe_lm.h: argument validation, workspace
// checks and dispatch to the launchers.  Host code only.
#include "checks.hpp"
#include "lm_launch.hpp"

using namespace hmoe;

extern "C" {

// The kernels take vectors and count workgroups in the workspace.
static int check_lm_ws(size_t need, size_t have, const void* ws) {
  HMOE_TRY(check_ws(need, have, ws));
  return need > 0 ? check_ptr("workspace", ws) : HMOE_OK;
}

// ------------------------------------------------------------------ token log-probabilities

static int check_logits(const void* logits, int64_t ld, const float* anchor, hmoe_dtype_t dt, int64_t n, int32_t vocab,
                        float scale) {
  HMOE_TRY(check_dtype(dt));
  HMOE_TRY(check_n(n));
  if (vocab < 1) return fail(HMOE_EINVAL, "vocab = %d is not positive", vocab);
  if (ld < vocab) return fail(HMOE_EINVAL, "ld = %lld is less than vocab = %d", (long long)ld, vocab);
  // the kernels take scale log2 e, which has to be finite too
  if (!(scale > 0.f) || scale > 0x1p127f) return fail(HMOE_EINVAL, "scale = %g outside (0, 2^127]", (double)scale);
  if (n == 0) return HMOE_OK;
  HMOE_TRY(check_ptr("logits", logits, anchor != nullptr));
  if (reinterpret_cast<uintptr_t>(logits) % dtype_size(dt)) return fail(HMOE_ESHAPE, "logits are not aligned to their type");
  if (anchor) {
    HMOE_TRY(check_ptr("anchor", anchor));
    HMOE_TRY(check_width("vocab (with anchors)", vocab));
    if (ld != vocab) return fail(HMOE_ESHAPE, "anchored logits with rows %lld apart, vocab = %d", (long long)ld, vocab);
  }
  return HMOE_OK;
}

size_t hmoe_token_logprob_workspace(int64_t n, int32_t vocab, int32_t m, hmoe_dtype_t dt) {
  if (n <= 0 || n >= (int64_t(1) << 31) || vocab < 1 || m < 0 || m > 16 || (dt != HMOE_F32 && dt != HMOE_BF16)) return 0;
  return token_logprob_ws(n, vocab, m, dt);
}

int hmoe_token_logprob(const void* logits, int64_t ld, const float* anchor, hmoe_dtype_t dt, int64_t n, int32_t vocab,
                       float scale, const int32_t* token, int32_t m, float* logp, float* entropy, float* lse,
                       float* stat, int32_t* top_idx, float* top_logp, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_logits(logits, ld, anchor, dt, n, vocab, scale));
  if (m < 0 || m > 16 || m > vocab) return fail(HMOE_EINVAL, "m = %d outside [0, min(16, vocab)]", m);
  if (n == 0) return HMOE_OK;
  if (m > 0) HMOE_TRY(check_ptr("top_idx", top_idx, false));
  HMOE_TRY(check_lm_ws(token_logprob_ws(n, vocab, m, dt), ws_bytes, ws));
  Workspace w(ws, ws_bytes);
  return launch_token_logprob(logits, ld, anchor, dt, n, vocab, scale, token, m, logp, entropy, lse, stat, top_idx,
                              top_logp, w, (hipStream_t)stream);
}

int hmoe_token_logprob_backward(const void* logits, int64_t ld, const float* anchor, hmoe_dtype_t dt, int64_t n,
                                int32_t vocab, float scale, const int32_t* token, const float* stat,
                                const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits,
                                int64_t ld_out, void* stream) {
  clear_error();
  HMOE_TRY(check_logits(logits, ld, anchor, dt, n, vocab, scale));
  if (ld_out < vocab) return fail(HMOE_EINVAL, "ld_out = %lld is less than vocab = %d", (long long)ld_out, vocab);
  if (n == 0) return HMOE_OK;
  HMOE_TRY(check_ptr("stat", stat, false));
  HMOE_TRY(check_ptr("dlogits", dlogits, false));
  if (reinterpret_cast<uintptr_t>(dlogits) % dtype_size(dt)) return fail(HMOE_ESHAPE, "dlogits are not aligned to their type");
  if (g_logp) HMOE_TRY(check_ptr("token", token, false));
  if (g_entropy) HMOE_TRY(check_ptr("entropy", entropy, false));
  if (dlogits == logits && (anchor || ld_out != ld))
    return fail(HMOE_EINVAL, "dlogits in place of logits needs plain logits and the same stride");
  return launch_token_logprob_backward(logits, ld, anchor, dt, n, vocab, scale, token, stat, entropy, g_logp,
                                       g_entropy, dlogits, ld_out, (hipStream_t)stream);
}

// ------------------------------------------------------------------ mixture layer of a few samples

static int check_few_rows(int64_t n) {
  if (n < 0 || n > HMOE_FEW_ROWS) return fail(HMOE_EINVAL, "n = %lld outside [0, %d]", (long long)n, HMOE_FEW_ROWS);
  return HMOE_OK;
}

static int check_few(const hmoe_few_params_t* p, int64_t n) {
  if (!p) return fail(HMOE_EINVAL, "params are NULL");
  HMOE_TRY(check_dtype(p->dt));
  HMOE_TRY(check_k(p->K));
  HMOE_TRY(check_width("d_in", p->d_in));
  HMOE_TRY(check_width("d_hid", p->d_hid));
  HMOE_TRY(check_width("d_out", p->d_out));
  for (int32_t w : {p->d_in, p->d_hid, p->d_out})
    if (w > HMOE_FEW_WIDTH) return fail(HMOE_EINVAL, "width %d exceeds %d", w, HMOE_FEW_WIDTH);
  if (p->top_k < 1 || p->top_k > HMOE_FEW_EXPERTS || p->top_k > p->K)
    return fail(HMOE_EINVAL, "top_k = %d outside [1, min(%d, K)]", p->top_k, HMOE_FEW_EXPERTS);
  if (p->act != HMOE_ACT_RELU && p->act != HMOE_ACT_SILU_GATED) return fail(HMOE_EINVAL, "unknown act %d", p->act);
  return check_few_rows(n);
}

size_t hmoe_moe_few_workspace(const hmoe_few_params_t* p, int64_t n) {
  if (check_few(p, n) != HMOE_OK || n == 0) {
    clear_error();
    return 0;
  }
  return moe_few_ws(p, n);
}

int hmoe_moe_few(const hmoe_few_params_t* p, int64_t n, const void* X, int32_t* expert, float* weight, void* Y,
                 void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_few(p, n));
  if (n == 0) return HMOE_OK;
  HMOE_TRY(check_ptr("R", p->R));
  HMOE_TRY(check_ptr("W1", p->W1));
  HMOE_TRY(check_ptr("W2", p->W2));
  HMOE_TRY(check_ptr("X", X));
  HMOE_TRY(check_ptr("expert", expert, false));
  HMOE_TRY(check_ptr("weight", weight, false));
  HMOE_TRY(check_ptr("Y", Y));
  HMOE_TRY(check_lm_ws(moe_few_ws(p, n), ws_bytes, ws));
  Workspace w(ws, ws_bytes);
  return launch_moe_few(p, n, X, expert, weight, Y, w, (hipStream_t)stream);
}

// ------------------------------------------------------------------ low-rank adapters

static int check_lora(const hmoe_lora_t* p) {
  if (!p) return fail(HMOE_EINVAL, "params are NULL");
  HMOE_TRY(check_dtype(p->dt));
  if (p->E < 1 || p->E > 4096) return fail(HMOE_EINVAL, "E = %d outside [1, 4096]", p->E);
  HMOE_TRY(check_width("d_in", p->d_in));
  HMOE_TRY(check_width("d_out", p->d_out));
  HMOE_TRY(check_width("rank", p->rank));
  if (p->rank > HMOE_LORA_RANK) return fail(HMOE_EINVAL, "rank = %d exceeds %d", p->rank, HMOE_LORA_RANK);
  if (p->d_in > HMOE_LORA_WIDTH || p->d_out > HMOE_LORA_WIDTH)
    return fail(HMOE_EINVAL, "d_in = %d or d_out = %d exceeds %d", p->d_in, p->d_out, HMOE_LORA_WIDTH);
  return HMOE_OK;
}

static int check_lora_rows(int64_t n) {
  if (n < 0 || n > HMOE_LORA_ROWS) return fail(HMOE_EINVAL, "n = %lld outside [0, %d]", (long long)n, HMOE_LORA_ROWS);
  return HMOE_OK;
}

static int check_lora_params(const hmoe_lora_t* p) {
  HMOE_TRY(check_ptr("W", p->W));
  HMOE_TRY(check_ptr("A", p->A));
  return check_ptr("B", p->B);
}

size_t hmoe_lora_few_workspace(const hmoe_lora_t* p, int64_t n) {
  if (check_lora(p) != HMOE_OK || check_few_rows(n) != HMOE_OK || n == 0) {
    clear_error();
    return 0;
  }
  return lora_few_ws(p, n);
}

int hmoe_lora_few(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* adapter, void* Y, void* ws,
                  size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_lora(p));
  HMOE_TRY(check_few_rows(n));
  if (n == 0) return HMOE_OK;
  HMOE_TRY(check_lora_params(p));
  HMOE_TRY(check_ptr("X", X));
  HMOE_TRY(check_ptr("adapter", adapter, false));
  HMOE_TRY(check_ptr("Y", Y));
  HMOE_TRY(check_lm_ws(lora_few_ws(p, n), ws_bytes, ws));
  Workspace w(ws, ws_bytes);
  return launch_lora_few(p, n, X, adapter, Y, w, (hipStream_t)stream);
}

int32_t hmoe_lora_saved_width(int32_t rank, hmoe_dtype_t dt) {
  if (rank < 1 || rank > HMOE_LORA_RANK || (dt != HMOE_F32 && dt != HMOE_BF16)) return 0;
  return lora_saved_width(rank, dt);
}

size_t hmoe_lora_workspace(const hmoe_lora_t* p, int64_t n) {
  if (check_lora(p) != HMOE_OK || check_lora_rows(n) != HMOE_OK || n == 0) {
    clear_error();
    return 0;
  }
  return lora_ws(p, n);
}

int hmoe_lora_forward(const hmoe_lora_t* p, int64_t n, const void* X_sorted, const int32_t* offsets,
                      const int32_t* perm, void* U, void* Y, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_lora(p));
  HMOE_TRY(check_lora_rows(n));
  if (n == 0) return HMOE_OK;
  HMOE_TRY(check_lora_params(p));
  HMOE_TRY(check_ptr("X_sorted", X_sorted));
  HMOE_TRY(check_ptr("offsets", offsets, false));
  HMOE_TRY(check_ptr("U", U));
  HMOE_TRY(check_ptr("Y", Y));
  HMOE_TRY(check_lm_ws(lora_ws(p, n), ws_bytes, ws));
  Workspace w(ws, ws_bytes);
  return launch_lora_forward(p, n, X_sorted, offsets, perm, U, Y, w, (hipStream_t)stream);
}

int hmoe_lora_backward(const hmoe_lora_t* p, int64_t n, const void* X_sorted, const int32_t* offsets,
                       const int32_t* perm, const void* U, const void* dY, void* dX, float* dA, float* dB, void* ws,
                       size_t ws_bytes, void* stream) {
  clear_error();
  HMOE_TRY(check_lora(p));
  HMOE_TRY(check_lora_rows(n));
  if (dA) HMOE_TRY(check_ptr("dA", dA));
  if (dB) HMOE_TRY(check_ptr("dB", dB));
  if (n > 0) {
    HMOE_TRY(check_lora_params(p));
    HMOE_TRY(check_ptr("X_sorted", X_sorted));
    HMOE_TRY(check_ptr("offsets", offsets, false));
    HMOE_TRY(check_ptr("U", U));
    HMOE_TRY(check_ptr("dY", dY));
    if (dX) HMOE_TRY(check_ptr("dX", dX));
    HMOE_TRY(check_lm_ws(lora_ws(p, n), ws_bytes, ws));
    Workspace w(ws, ws_bytes);
    return launch_lora_backward(p, n, X_sorted, offsets, perm, U, dY, dX, dA, dB, w, (hipStream_t)stream);
  }
  // no rows: the adapters' gradients are zeros
  if (dA) HMOE_TRY(launch_zero_f32(dA, (int64_t)p->E * p->rank * p->d_in, (hipStream_t)stream));
  if (dB) HMOE_TRY(launch_zero_f32(dB, (int64_t)p->E * p->rank * p->d_out, (hipStream_t)stream));
  return HMOE_OK;
}

}  // extern "C"
