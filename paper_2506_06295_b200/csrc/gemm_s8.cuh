// Host-side interface of the 8-bit integer products (gemm_s8.cu).
#pragma once
#include "internal.h"

namespace dllm {

cudaError_t launch_quantize_rows_s8(const Launch& L, const void* x, size_t ldx, int dtype, int8_t* q, size_t ldq, float* scale,
                                    int rows, int cols);
GemmPlan plan_gemm_s8(int M, int N, int K);
size_t gemm_s8_scratch_bytes(int M, int N, const GemmPlan& plan);
// With L.pdl the weights are requested while the launch before this one still runs: nothing that launch may overlap may
// write them.
cudaError_t launch_gemm_s8(const Launch& L, const int8_t* A, size_t lda, const float* sa, const int8_t* W, size_t ldw,
                           const float* sw, void* out, int out_dtype, int M, int N, int K, const GemmPlan& plan, void* scratch,
                           const char** err);
cudaError_t set_wait_limit_gemm_s8(unsigned long long ns);
cudaError_t set_debug_skip_gemm_s8(int enable);   // dllm_debug_skip_one_load

}  // namespace dllm
