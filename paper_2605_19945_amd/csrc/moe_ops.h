// Launchers of the operators around the experts' weights (moe_ops_api.hip checks the arguments).
#pragma once
#include "moe_grouped_pick.h"
#include "moe_internal.h"

// Matrix products grouped by expert, as planned; ws: the workspace that the plan needs (none: may be null).
hipError_t launch_grouped_gemm(const void* x, int64_t ldx, const void* w, bool transpose_w, const int32_t* offsets, int rows_cap, int E,
                               int K, int N, void* y, int64_t ldy, const GroupedPlan& plan, void* ws, hipStream_t st);
hipError_t launch_grouped_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* offsets, int rows_cap, int E,
                                int K, int N, void* dw, bool f32, bool add, const GroupedPlan& plan, void* ws, hipStream_t st);
hipError_t launch_grouped_mx(const void* xq, const void* xs, const void* wq, const void* wsc, const int32_t* offsets, int rows_cap, int E,
                             int K, int N, void* y, int64_t ldy, const GroupedPlan& plan, void* ws, hipStream_t st);
hipError_t launch_swiglu(const void* gu, int64_t ldgu, const int32_t* n_rows, int rows, int f, void* h, int64_t ldh, hipStream_t st);
hipError_t launch_swiglu_backward(const void* dh, int64_t lddh, const void* gu, int64_t ldgu, const int32_t* n_rows, int rows, int f,
                                  void* dgu, int64_t lddgu, void* h, int64_t ldh, hipStream_t st);
hipError_t launch_mx_quantize(const void* x, bool f32, int64_t ldx, const int32_t* n_rows, int rows, int K, void* q, void* s, hipStream_t st);
hipError_t launch_mx_quantize_weights(const void* w, int E, int K, int N, void* q, void* s, hipStream_t st);
hipError_t launch_mx_dequantize(const void* q, const void* s, int64_t rows, int K, void* x, int64_t ldx, hipStream_t st);

// Bytes of scales of one row: one byte per block of 32, up to the next multiple of 16.
static inline int mx_scale_cols(int K) { return (K / 32 + 15) / 16 * 16; }

// ---- lists of gradients ----
constexpr int GRAD_LIST = 128;         // tensors one launch takes as kernel arguments
constexpr int GRAD_BLOCKS = 1024;      // workgroups of such a launch, at most; each leaves one partial sum
size_t grad_norm_workspace(int64_t n_tensors);
hipError_t launch_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* f32, int n, double* partials, float* norm, hipStream_t st);
hipError_t launch_clip_grads(const void* const* grads, void* const* outs, const int64_t* counts, const int32_t* f32, int n, float max_norm,
                             double* partials, float* norm, hipStream_t st);
