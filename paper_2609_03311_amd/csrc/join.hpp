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

// PARTS threads share the splits of two dims: eight where there are many (their
// loads side by side), else one, and several rows a block (4,096 rows of four
// splits: the call took 38 us with eight, and 31).
constexpr int kJoinParts = 8;
constexpr int join_parts(int splits) { return splits > 8 ? kJoinParts : 1; }
constexpr int join_threads(int D, int parts) { return parts > 1 ? 4 * D : 256; }
constexpr int join_rows(int D, int parts) { return parts > 1 ? 1 : 512 / D; }

// One row by the block's (join_rows(): D/2 of its) threads: x[s * step ..], s <
// splits, holds O[D], the reference m and the normaliser l of each split (a
// split without keys has no weight, and the reference 0 or -inf).  Writes the
// bf16 row and the LSE (NULL: none).
template <int D, int PARTS>
__device__ __forceinline__ void join_row(const float *x, int64_t step,
                                         int splits, uint16_t *out,
                                         float *lse) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  const int part = PARTS > 1 ? threadIdx.x / (D / 2) : 0;
  const int d = 2 * (threadIdx.x % (D / 2));
  float M = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  // (eight splits' loads at a time)
  for (int s0 = part; s0 < splits; s0 += 8 * PARTS) {
    float2 ml[8], o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = s0 + i * PARTS;
      const float *at = x + (s < splits ? s : s0) * step;
      ml[i] = *reinterpret_cast<const float2 *>(at + D);
      o[i] = *reinterpret_cast<const float2 *>(at + d);
    }
    float m = M;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (s0 + i * PARTS >= splits) ml[i].x = -INFINITY;
      m = fmaxf(m, ml[i].x);
    }
    const float ref = m == -INFINITY ? 0.f : m;
    const float a = __builtin_amdgcn_exp2f(M - ref);
    l *= a;
    o0 *= a;
    o1 *= a;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float b = __builtin_amdgcn_exp2f(ml[i].x - ref);
      l = fmaf(b, ml[i].y, l);
      o0 = fmaf(b, o[i].x, o0);
      o1 = fmaf(b, o[i].y, o1);
    }
    M = m;
  }
  float ref = M == -INFINITY ? 0.f : M;
  if constexpr (PARTS > 1) {
    __shared__ float so[PARTS][D], sl[PARTS], sm[PARTS];
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
    for (int i = 0; i < PARTS; ++i) M = fmaxf(M, sm[i]);
    ref = M == -INFINITY ? 0.f : M;
    l = o0 = o1 = 0.f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
      const float f = __builtin_amdgcn_exp2f(sm[i] - ref);
      l = fmaf(f, sl[i], l);
      o0 = fmaf(f, so[i][d], o0);
      o1 = fmaf(f, so[i][d + 1], o1);
    }
  }
  const float inv = 1.0f / l;
  const pair w = {(__bf16)(o0 * inv), (__bf16)(o1 * inv)};
  *reinterpret_cast<uint32_t *>(out + d) = __builtin_bit_cast(uint32_t, w);
  if (lse && d == 0) *lse = (ref + __log2f(l)) * 0.69314718055994530942f;
}

}  // namespace dopr
