// ops_internal.h -- launchers of the operators of quasar_ops.h, called with
// checked arguments by ops_api.hip.
#pragma once

#include <hip/hip_runtime.h>

#include "quasar_ops.h"

namespace quasar {

constexpr int kCUs = 256;  // compute units of the card

// norm_kernel.hip
hipError_t launch_norm(const quasar_norm& a, hipStream_t stream);
int norm_backward_parts(int64_t rows, int64_t cols);  // workgroups, each with its share of dweight
size_t norm_backward_workspace(int64_t rows, int64_t cols);
hipError_t launch_norm_backward(const quasar_norm_backward& a, hipStream_t stream);

// distill_kernel.hip; what: 0 loss, 1 gradient, 2 both
size_t distill_workspace(int64_t rows, int64_t classes);
hipError_t launch_distill(const quasar_distill& a, int what, hipStream_t stream);

// linear_kernel.hip
size_t linear_workspace(const quasar_desc& d, int64_t tokens);
hipError_t launch_linear(const quasar_desc& d, const quasar_linear& a, hipStream_t stream);

}  // namespace quasar
