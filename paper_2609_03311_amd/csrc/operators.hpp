// operators.hpp -- launches of the operators around the attention (rows.hip,
// qproduct.hip, rotary.hip).  The arguments have been checked.
#pragma once
#include <hip/hip_runtime.h>

#include "dopr.h"

namespace dopr {

hipError_t launch_quantize_rows(const dopr_quantize_args_t &a, hipStream_t s);
hipError_t launch_norm_residual(const dopr_norm_residual_args_t &a,
                                hipStream_t s);
// bytes that a product of these sizes has a use for
size_t product_workspace(int64_t rows, int64_t cols, int64_t depth);
hipError_t launch_product(const dopr_quant_matmul_args_t &a, hipStream_t s);
hipError_t launch_rotary(const dopr_rotary_args_t &a, hipStream_t s);

}  // namespace dopr
