// ops_internal.h -- launchers of the operators of quasar_ops.h, called with
// checked arguments by ops_api.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "quasar_ops.h"

namespace quasar {

constexpr int kCUs = 256;  // compute units of the card
constexpr int64_t kLastLevel = (int64_t)256 << 20;  // bytes of its last-level cache

// Workgroups of a launch: HIP takes fewer than 2^32 threads in a grid.  A call
// with more rows than that many take is launched in pieces of its rows.
constexpr int64_t most_groups(int threads) { return 0xffffffffll / threads; }

inline int64_t size_of(int32_t dtype) { return dtype == QUASAR_F32 ? 4 : dtype == QUASAR_E4M3 ? 1 : 2; }
// p (may be NULL) `rows` rows on
template <typename T>
T* rows_on(T* p, int64_t rows, int64_t stride, int64_t size) {
  using byte = std::conditional_t<std::is_const_v<T>, const char, char>;
  return p ? reinterpret_cast<T*>(reinterpret_cast<byte*>(p) + rows * stride * size) : nullptr;
}

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
// whether the kernels' workgroups fit a grid; and linear_workspace()
bool linear_fits(const quasar_desc& d, int64_t tokens, int x_dtype, size_t& workspace);
hipError_t launch_linear(const quasar_desc& d, const quasar_linear& a, hipStream_t stream);

// layer_norm_kernel.hip
hipError_t launch_layer_norm(const quasar_layer_norm& a, hipStream_t stream);
size_t layer_norm_backward_workspace(int64_t rows, int64_t cols);
hipError_t launch_layer_norm_backward(const quasar_layer_norm_backward& a, hipStream_t stream);

// embed_kernel.hip
hipError_t launch_embed(const quasar_embedding& a, hipStream_t stream);
// whether the kernels' workgroups fit a grid; and the scratch memory that they need
bool embed_backward_fits(int64_t rows, int64_t cols, int64_t tokens, size_t& workspace);
hipError_t launch_embed_backward(const quasar_embedding_backward& a, hipStream_t stream);

// checkpoint_kernel.hip
hipError_t launch_checkpoint(const quasar_checkpoint& a, hipStream_t stream);
hipError_t launch_checkpoint_backward(const quasar_checkpoint_grad& a, hipStream_t stream);

// weight_grad_kernel.hip
bool weight_grad_fits(const quasar_weight_grad& a, size_t& workspace);
hipError_t launch_weight_grad(const quasar_weight_grad& a, hipStream_t stream);

}  // namespace quasar
