// Launchers of the gfx950 kernels behind include/lionmuon_grad.h. Arguments
// have been validated; each returns the hipError_t of its launches, all of them
// on `stream`.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "grad_plan.h"

namespace lm {

enum class Elem : int32_t { kF32 = 0, kBF16 = 1, kF16 = 2 };

// Row-major matrix view; ld in elements. data == nullptr: not given.
struct MatView {
  void* data = nullptr;
  int64_t ld = 0;
};

// 8-bit checkpoint view. codes == nullptr: not given.
struct CkptView {
  uint8_t* codes = nullptr;
  uint8_t* scales = nullptr;
  int64_t ld_codes = 0, ld_scales = 0;
};

constexpr int kCkptBlock = 128;

hipError_t launch_checkpoint(Elem t, MatView x, CkptView out, int64_t rows, int64_t cols,
                             hipStream_t stream);
hipError_t launch_restore(Elem t, CkptView c, MatView out, int64_t rows, int64_t cols,
                          hipStream_t stream);

// cols: of h. kind: 0 gelu, 1 swiglu.
hipError_t launch_activation(Elem t, int kind, MatView a, MatView h, CkptView kept, int64_t rows,
                             int64_t cols, hipStream_t stream);
hipError_t launch_activation_grad(Elem t, int kind, MatView dh, MatView a, CkptView kept,
                                  MatView da, MatView h, int64_t rows, int64_t cols,
                                  hipStream_t stream);

struct NormArgs {
  MatView x, residual, y, sum;      // forward
  MatView dy, s, residual_grad, dx; // backward
  CkptView kept;                    // forward: of y; backward: of s
  const float* weight = nullptr;
  float* rstd = nullptr;
  float* dweight = nullptr;
  float* partial = nullptr;         // backward: workgroups x cols
  int64_t rows = 0;
  int32_t cols = 0;
  float eps = 0.0f;
  int32_t accumulate = 0;
};
hipError_t launch_rmsnorm(Elem t, const NormArgs& a, hipStream_t stream);
hipError_t launch_rmsnorm_grad(Elem t, const NormArgs& a, hipStream_t stream);
// Workgroups of the backward pass: each sums dweight over its rows.
int64_t rmsnorm_grad_groups(int64_t rows, int64_t cols);

struct GroupArgs {
  const void* a = nullptr;          // rows x (contraction or n): X or dY
  const void* b = nullptr;          // W, or X of the weight gradient
  void* c = nullptr;
  CkptView kept;                    // X of the weight gradient in 8 bits (b is then null)
  const int32_t* offsets = nullptr;
  int64_t lda = 0, ldb = 0, ldc = 0;
  int64_t b_stride = 0, c_stride = 0;   // per expert
  int64_t rows = 0;
  int32_t experts = 0, n = 0, k = 0;
  int32_t accumulate = 0;
  float* partial = nullptr;         // weight gradient: weight_grad_partials() x n x k
  int32_t cus = 256;
};
hipError_t launch_grouped_product(Elem t, const GroupArgs& g, hipStream_t stream);
hipError_t launch_grouped_input_grad(Elem t, const GroupArgs& g, hipStream_t stream);
hipError_t launch_grouped_weight_grad(Elem t, const GroupArgs& g, hipStream_t stream);
// Whether some tile covers a product of these sizes within kMaxWorkgroups.
bool row_product_fits(int64_t rows, int64_t experts, int64_t width);
bool weight_grad_fits(int64_t experts, int64_t n, int64_t k);
// Partial sums (n x k fp32 each) that the weight gradient of these sizes needs
// room for: long experts are cut into parts where whole ones would leave CUs idle.
int64_t weight_grad_partials(int64_t rows, int64_t experts, int64_t n, int64_t k, int cus);

}  // namespace lm
