// rowio.hpp -- element types of the row operators (rows.hip, rotary.hip,
// qproduct.hip): loads and stores of 8 elements at any element alignment, in
// fp32.
#pragma once
#include <cstdint>

#include "operators.hpp"

namespace dopr {

struct bf16_t {
  uint16_t bits;
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2v __attribute__((ext_vector_type(2)));
// 16 and 8 bytes that may start at any byte: one global load or store each
// (global memory is accessed in unaligned mode), at full speed where the
// address happens to be aligned
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<bf16_t>(bf16_t v) {
  return __uint_as_float((uint32_t)v.bits << 16);
}
template <>
__device__ __forceinline__ float to_f32<_Float16>(_Float16 v) {
  return (float)v;
}
template <>
__device__ __forceinline__ float to_f32<float>(float v) {
  return v;
}

// rounded to nearest even; NaN stays NaN
template <typename T>
__device__ __forceinline__ T from_f32(float f);
template <>
__device__ __forceinline__ bf16_t from_f32<bf16_t>(float f) {
  return bf16_t{__builtin_bit_cast(uint16_t, (__bf16)f)};
}
template <>
__device__ __forceinline__ _Float16 from_f32<_Float16>(float f) {
  return (_Float16)f;
}
template <>
__device__ __forceinline__ float from_f32<float>(float f) {
  return f;
}

template <typename T>
__device__ __forceinline__ void unpack2(uint32_t u, float &a, float &b);
template <>
__device__ __forceinline__ void unpack2<bf16_t>(uint32_t u, float &a,
                                                float &b) {
  a = __uint_as_float(u << 16);
  b = __uint_as_float(u & 0xffff0000u);
}
template <>
__device__ __forceinline__ void unpack2<_Float16>(uint32_t u, float &a,
                                                  float &b) {
  const f16x2v h = __builtin_bit_cast(f16x2v, u);
  a = (float)h.x;
  b = (float)h.y;
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<bf16_t>(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2v));
}
template <>
__device__ __forceinline__ uint32_t pack2<_Float16>(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2v));
}

// E elements as they lie in memory: one load of up to 16 bytes, two for 8 of
// fp32
template <typename T, int E>
struct Raw {
  static_assert(E == 8 && sizeof(T) == 2, "other forms below");
  u32x4 u;
  __device__ __forceinline__ void load(const T *p) {
    u = *reinterpret_cast<const u32x4_any *>(p);
  }
  __device__ __forceinline__ void get(float *f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(u[i], f[2 * i], f[2 * i + 1]);
  }
};
template <typename T>
struct Raw<T, 4> {
  u32x2 u;
  __device__ __forceinline__ void load(const T *p) {
    u = *reinterpret_cast<const u32x2_any *>(p);
  }
  __device__ __forceinline__ void get(float *f) const {
    unpack2<T>(u.x, f[0], f[1]);
    unpack2<T>(u.y, f[2], f[3]);
  }
};
template <>
struct Raw<float, 4> {
  u32x4 u;
  __device__ __forceinline__ void load(const float *p) {
    u = *reinterpret_cast<const u32x4_any *>(p);
  }
  __device__ __forceinline__ void get(float *f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(u[i]);
  }
};
template <>
struct Raw<float, 8> {
  Raw<float, 4> a, b;
  __device__ __forceinline__ void load(const float *p) {
    a.load(p);
    b.load(p + 4);
  }
  __device__ __forceinline__ void get(float *f) const {
    a.get(f);
    b.get(f + 4);
  }
};
template <typename T>
using Raw8 = Raw<T, 8>;

// The E elements of a row of `width` that start at c0, as one load that stays
// inside the row: chunks outside it read the row's first elements and keep
// none; a chunk that starts in front of the row (c0 < 0) reads the first E and
// keeps those below `hi`, one that ends behind it reads the last E and keeps
// those from `lo` on.  `width` is at least E.
template <int E>
struct Chunk {
  int c, lo, hi;
  __device__ __forceinline__ Chunk(int c0, int width) {
    const int n = width - c0;
    c = n > 0 ? max(min(c0, width - E), 0) : 0;
    lo = n >= E ? 0 : n > 0 ? E - n : E;
    hi = c0 >= 0 ? E : c0 > -E ? E + c0 : 0;
  }
  __device__ __forceinline__ bool whole() const { return lo == 0 && hi == E; }
  __device__ __forceinline__ void mask(float *f) const {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = e >= lo && e < hi ? f[e] : 0.f;
  }
};

// 16 and 8 bytes to any byte.  (The places keep their types: passed on as a
// template's pointer they would be taken to lie on their size.)  STREAM: past
// the caches' order of use, for stores of whole lines that nothing reads soon.
template <bool STREAM>
__device__ __forceinline__ void put(u32x4 v, void *p) {
  u32x4_any *to = static_cast<u32x4_any *>(p);
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, to);
  else
    *to = v;
}
template <bool STREAM>
__device__ __forceinline__ void put(u32x2 v, void *p) {
  u32x2_any *to = static_cast<u32x2_any *>(p);
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, to);
  else
    *to = v;
}

template <typename T, bool STREAM = false>
__device__ __forceinline__ void store4(T *p, const float *f) {
  if constexpr (sizeof(T) == 2)
    put<STREAM>(u32x2{pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3])}, p);
  else
    put<STREAM>(u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]),
                      __float_as_uint(f[2]), __float_as_uint(f[3])},
                p);
}

template <typename T, bool STREAM = false>
__device__ __forceinline__ void store8(T *p, const float *f) {
  if constexpr (sizeof(T) == 2) {
    put<STREAM>(u32x4{pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]),
                      pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7])},
                p);
  } else {
    store4<T, STREAM>(p, f);
    store4<T, STREAM>(p + 4, f + 4);
  }
}

// Elements lo..hi-1 of E to p[lo..hi-1].
template <typename T, int E, bool STREAM = false>
__device__ __forceinline__ void store_part(T *p, int lo, int hi,
                                           const float *f) {
  if (lo == 0 && hi == E) {
    if constexpr (E == 8)
      store8<T, STREAM>(p, f);
    else
      store4<T, STREAM>(p, f);
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e >= lo && e < hi) p[e] = from_f32<T>(f[e]);
}

}  // namespace dopr
