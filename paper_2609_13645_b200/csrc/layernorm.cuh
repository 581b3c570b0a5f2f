// Host-side interface of the LayerNorm kernels.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace fs {

constexpr int kLayerNormMaxWidth = 16384;

// y = (x - mean) rstd gain + bias by rows of h elements; dtype 0: bf16, 1: fp32 (x, y, gain, bias); mean, rstd fp32 [rows].
cudaError_t layernorm_fwd(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean,
                          float* rstd, int rows, int h, float eps, int dtype, cudaStream_t st);

// dx = R(rstd (g - mean_h(g) - xhat mean_h(g xhat)) + resid), g = dy gain; dgain = sum dy xhat, dbias = sum dy (fp32, fixed
// summation order; dbias may be null).  scratch: layernorm_scratch_bytes() bytes, 16-byte aligned.  Two launches, or one of a cluster for few rows.
size_t layernorm_scratch_bytes(int rows, int h);
cudaError_t layernorm_bwd(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd,
                          const void* gain, const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias,
                          float* scratch, int rows, int h, int dtype, cudaStream_t st);

}  // namespace fs
