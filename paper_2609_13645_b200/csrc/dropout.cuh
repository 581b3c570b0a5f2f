// Host-side interface of the dropout kernels.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace fs {

// y[r, c] = R(resid[r, c] + scale / (1 - p) * keep(r h + c) * x[r, c]) (resid may be null: 0).
cudaError_t dropout_add(const void* x, int64_t ldx, const void* resid, int64_t ldr, void* y, int64_t ldy, int rows, int h, float p,
                        float scale, uint64_t seed, int32_t site, const long long* step, int dtype, cudaStream_t st);

}  // namespace fs
