// lm_launch.hpp -- launchers behind include/hmoe_lm.h.  As in launch.hpp they only enqueue work on
// `st`; sizes have been validated by the caller.
#pragma once
#include "hmoe_lm.h"
#include "launch.hpp"

namespace hmoe {

// logprob.hip
size_t token_logprob_ws(int64_t n, int V, int m, hmoe_dtype_t dt);
int launch_token_logprob(const void* L, int64_t ld, const float* anc, hmoe_dtype_t dt, int64_t n, int V, float scale,
                         const int32_t* token, int m, float* logp, float* entropy, float* lse, float* stat,
                         int32_t* top_idx, float* top_logp, Workspace& ws, hipStream_t st);
int launch_token_logprob_backward(const void* L, int64_t ld, const float* anc, hmoe_dtype_t dt, int64_t n, int V,
                                  float scale, const int32_t* token, const float* stat, const float* entropy,
                                  const float* g_logp, const float* g_entropy, void* dL, int64_t ldo, hipStream_t st);

// moe_few.hip
size_t moe_few_ws(const hmoe_few_params_t* p, int64_t n);
int launch_moe_few(const hmoe_few_params_t* p, int64_t n, const void* X, int32_t* expert, float* weight, void* Y,
                   Workspace& ws, hipStream_t st);

// lora.hip
int lora_saved_width(int rank, hmoe_dtype_t dt);
size_t lora_few_ws(const hmoe_lora_t* p, int64_t n);
size_t lora_ws(const hmoe_lora_t* p, int64_t n);
int launch_lora_few(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* adapter, void* Y, Workspace& ws,
                    hipStream_t st);
int launch_lora_forward(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* offsets, const int32_t* perm,
                        void* U, void* Y, Workspace& ws, hipStream_t st);
int launch_lora_backward(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* offsets, const int32_t* perm,
                         const void* U, const void* dY, void* dX, float* dA, float* dB, Workspace& ws, hipStream_t st);

}  // namespace hmoe
