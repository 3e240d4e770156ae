// train_launch.hpp -- launchers behind include/hmoe_train.h.  As in launch.hpp they only enqueue work on
// `st`; sizes have been validated by the caller.
#pragma once
#include "hmoe_train.h"
#include "launch.hpp"

namespace hmoe {

// router.hip
size_t router_ws(const hmoe_router_t* p, int64_t n);
int launch_router_forward(const hmoe_router_t* p, int64_t n, const void* X, int32_t* expert, float* weight,
                          float* scores, int32_t* counts, float* share, float* loss, Workspace& ws, hipStream_t st);
int launch_router_backward(const hmoe_router_t* p, int64_t n, const void* X, const float* scores,
                           const int32_t* expert, const int32_t* counts, const float* g_weight, float balance, float z,
                           void* dX, float* dR, float* dbias, Workspace& ws, hipStream_t st);

// join.hip
size_t join_ws(const hmoe_join_t* p, int64_t n);
int launch_join_forward(const hmoe_join_t* p, int64_t n, const void* x, const void* y, const float* gate, void* x_out,
                        void* h, hipStream_t st);
int launch_join_backward(const hmoe_join_t* p, int64_t n, const void* x_out, const void* y, const float* gate,
                         const void* dx_out, const void* dh, void* dx, void* dy, float* dgate, float* dgamma_y,
                         float* dgamma_h, Workspace& ws, hipStream_t st);

// ortho.hip
struct OrthoStep {  // what becomes of the iterations' result
  const void* G;    // hmoe_orthogonalise: in and out, in dt
  void* O;
  float* w;         // hmoe_muon_step: G is NULL
  const float* g;
  float* v;
  void* w_lo;
  hmoe_dtype_t dt;
  float momentum, keep, rate;  // w = keep w - rate NS(U)
  int32_t nesterov;
};
size_t ortho_ws(int32_t K, int32_t rows, int32_t cols);
int launch_ortho(const OrthoStep& s, int32_t K, int32_t rows, int32_t cols, int32_t steps, const float* coef,
                 Workspace& ws, hipStream_t st);

}  // namespace hmoe
