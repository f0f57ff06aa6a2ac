// Host-side launchers of the optimiser kernels (see optim_kernels.cu).
#pragma once

#include <cuda_runtime.h>

#include "sparse_ffn.h"

namespace sffn {

cudaError_t launch_grad_norm(const sffn_tensor* t, int n, float* norm, void* workspace, int sm_count, cudaStream_t s);
cudaError_t launch_adamw(const sffn_adamw_tensor* t, int n, const sffn_adamw_config& c, int sm_count, cudaStream_t s);
cudaError_t launch_adamw_values(const sffn_adamw_tensor* t, int n, float* const* m_out, float* const* v_out, int sm_count, cudaStream_t s);

}  // namespace sffn
