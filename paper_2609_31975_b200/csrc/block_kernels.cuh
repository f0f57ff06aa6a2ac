// Host-side launchers of the norms around a block (see block_kernels.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "sparse_ffn.h"

namespace sffn {

// Lines of partial column sums, at most: one of every CTA that adds up columns.
constexpr int block_lines(int D) { return D <= 1024 ? 1280 : 320; }

cudaError_t launch_block_forward(const sffn_block_norm& b, int sm_count, cudaStream_t s);
// partial: [2][block_lines(D)][D] floats where a gradient of a gain or of a channel gate is wanted.
cudaError_t launch_block_backward(const sffn_block_norm& b, const sffn_block_grads& g, float* partial, int sm_count, cudaStream_t s);

}  // namespace sffn
