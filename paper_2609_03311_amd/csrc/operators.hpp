// operators.hpp -- launches of the operators around the attention (rows.hip,
// qproduct.hip, rotary.hip).  The arguments have been checked.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "dopr.h"

namespace dopr {

// A launch has at most 2^32 - 1 threads in x.  Calls of more go in slices of
// this many rows (or what else takes `threads` of them each).
constexpr int64_t a_launch(int64_t threads) {
  return ((int64_t)1 << 31) / threads;
}

// f(first, count) for each slice of `all`.
template <typename F>
hipError_t in_slices(int64_t all, int64_t most, F f) {
  for (int64_t i = 0; i < all; i += most) {
    const hipError_t e = f(i, std::min(most, all - i));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// p, `bytes` further on; NULL stays NULL.
template <typename P>
P *ahead(P *p, int64_t bytes) {
  return p ? reinterpret_cast<P *>(reinterpret_cast<uintptr_t>(p) + bytes) : p;
}

hipError_t launch_quantize_rows(const dopr_quantize_args_t &a, hipStream_t s);
hipError_t launch_norm_residual(const dopr_norm_residual_args_t &a,
                                hipStream_t s);
// bytes that this product has a use for
size_t product_workspace(const dopr_quant_matmul_args_t &a);
hipError_t launch_product(const dopr_quant_matmul_args_t &a, hipStream_t s);
hipError_t launch_rotary(const dopr_rotary_args_t &a, hipStream_t s);

}  // namespace dopr
