// join.hpp -- for the kernels that need no plan: uniform loads, and sums of a
// softmax row that several blocks formed, put together.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace dopr {

// Loads at wave-uniform places of what no kernel of this launch writes, through
// the constant address space: scalar ones.
template <class T>
__device__ __forceinline__ T uniform_load(const T *p, int64_t i) {
  return ((const __attribute__((address_space(4))) T *)p)[i];
}

constexpr int kJoinParts = 8;  // threads that share the splits of two dims

// One row by 4 D threads: x[s * step ..], s < splits, holds O[D], the
// reference m and the normaliser l of each split (a split without keys has no
// weight, and the reference 0 or -inf).  Writes the bf16 row and the LSE (NULL:
// none).
template <int D>
__device__ __forceinline__ void join_row(const float *x, int64_t step,
                                         int splits, uint16_t *out,
                                         float *lse) {
  __shared__ float so[kJoinParts][D], sl[kJoinParts], sm[kJoinParts];
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  const int part = threadIdx.x / (D / 2), d = 2 * (threadIdx.x % (D / 2));
  float M = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int s = part; s < splits; s += kJoinParts) {
    const float2 ml = *reinterpret_cast<const float2 *>(x + s * step + D);
    const float2 o = *reinterpret_cast<const float2 *>(x + s * step + d);
    const float m = fmaxf(M, ml.x), ref = m == -INFINITY ? 0.f : m;
    const float a = __builtin_amdgcn_exp2f(M - ref),
                b = __builtin_amdgcn_exp2f(ml.x - ref);
    l = fmaf(b, ml.y, a * l);
    o0 = fmaf(b, o.x, a * o0);
    o1 = fmaf(b, o.y, a * o1);
    M = m;
  }
  so[part][d] = o0;
  so[part][d + 1] = o1;
  if (d == 0) {
    sm[part] = M;
    sl[part] = l;
  }
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  M = -INFINITY;
#pragma unroll
  for (int i = 0; i < kJoinParts; ++i) M = fmaxf(M, sm[i]);
  const float ref = M == -INFINITY ? 0.f : M;
  l = o0 = o1 = 0.f;
#pragma unroll
  for (int i = 0; i < kJoinParts; ++i) {
    const float f = __builtin_amdgcn_exp2f(sm[i] - ref);
    l = fmaf(f, sl[i], l);
    o0 = fmaf(f, so[i][d], o0);
    o1 = fmaf(f, so[i][d + 1], o1);
  }
  const float inv = 1.0f / l;
  const pair w = {(__bf16)(o0 * inv), (__bf16)(o1 * inv)};
  *reinterpret_cast<uint32_t *>(out + d) = __builtin_bit_cast(uint32_t, w);
  if (lse && d == 0) *lse = (ref + __log2f(l)) * 0.69314718055994530942f;
}

}  // namespace dopr
