// rows.hip -- operators over the rows of an activation matrix, one pass over
// memory each: rows in 8-bit integers (k_quantize_rows) and the norms around a
// gated, scaled residual (k_norm_residual).
//
// A row is held in registers by TPR threads (a wave, or a whole block), 8
// elements of NV chunks each, so that its sums and its largest magnitude are
// known before its first output is written and nothing is read twice.  Both
// kernels are bound by HBM: a row's arithmetic is some ten vector
// instructions per 8 elements.
#include <type_traits>

#include "rowio.hpp"

namespace dopr {
namespace {

// Rows of at most this many elements belong to one wave (four rows a block).
constexpr int kWaveRow = 2048;

template <int TPR, typename S>
__device__ __forceinline__ S row_sum(S v, S *part) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if constexpr (TPR > 64) {
    __syncthreads();  // the parts of an earlier reduction have been read
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += part[w];
  }
  return v;
}

// Largest |v| as its bit pattern: unsigned order puts infinities above every
// finite value and NaN above those, where a float maximum would drop NaN.
template <int TPR>
__device__ __forceinline__ uint32_t row_max_bits(uint32_t v,
                                                 uint32_t *part) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
    v = max(v, (uint32_t)__shfl_xor((int)v, off, 64));
  if constexpr (TPR > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v = max(v, part[w]);
  }
  return v;
}

// The low byte of v + 1.5 * 2^23 is v rounded to the nearest integer, ties to
// even, in two's complement (|v| <= 127 here).
__device__ __forceinline__ uint32_t int8_bits(float v) {
  return __float_as_uint(v + 12582912.f) & 0xffu;
}
__device__ __forceinline__ uint32_t pack_int8(const float *f, float inv) {
  return int8_bits(f[0] * inv) | (int8_bits(f[1] * inv) << 8) |
         (int8_bits(f[2] * inv) << 16) | (int8_bits(f[3] * inv) << 24);
}

// Scale of a row from the bits of its largest magnitude, and what its values
// are multiplied by: scale = a'/127, inv = 127/a' with a' = max(a, 127 *
// 2^-126), so both are normal numbers for a row of zeros too.  A row with a
// value that is not finite has scale NaN and integers 0.
__device__ __forceinline__ void row_scale(uint32_t bits, float &scale,
                                          float &inv) {
  if (bits >= 0x7f800000u) {
    scale = __uint_as_float(0x7fc00000u);
    inv = 0.f;
    return;
  }
  const float a = fmaxf(__uint_as_float(bits), 127.f * 0x1p-126f);
  scale = a / 127.f;
  inv = 127.f / a;
}

__device__ __forceinline__ void store_int8(int8_t *p, int lo, const float *f,
                                           float inv) {
  if (lo >= 8) return;
  // inf * 0 and NaN * 0 are NaN: a row that is not finite stores zeros
  const u32x2 u = inv == 0.f ? u32x2{0u, 0u}
                             : u32x2{pack_int8(f, inv), pack_int8(f + 4, inv)};
  if (lo == 0) {
    *reinterpret_cast<u32x2_any *>(p) = u;
    return;
  }
#pragma unroll
  for (int e = 1; e < 8; ++e)
    if (e >= lo) p[e] = (int8_t)(u[e >> 2] >> (8 * (e & 3)));
}

struct QuantizeParams {
  const void *x, *up;
  int8_t *q;
  float *scale;
  int64_t rows, ldx, ldu, ldq;
  int32_t width;
};

template <typename T, int TPR, int NV, bool UP>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_quantize_rows(
    QuantizeParams P) {
  constexpr int kRows = TPR > 64 ? 1 : 4;
  __shared__ uint32_t part[TPR / 64];
  const int t = TPR > 64 ? threadIdx.x : threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * kRows +
                    (TPR > 64 ? 0 : threadIdx.x >> 6);
  if (r >= P.rows) return;  // one wave per row here: no barrier is missed
  const T *x = static_cast<const T *>(P.x) + r * P.ldx;
  const T *up = static_cast<const T *>(P.up) + r * P.ldu;
  Raw8<T> rx[NV], ru[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Chunk k((v * TPR + t) * 8, P.width);
    rx[v].load(x + k.c);
    if constexpr (UP) ru[v].load(up + k.c);
  }
  float f[NV][8];
  uint32_t m = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    rx[v].get(f[v]);
    if constexpr (UP) {
      float g[8];
      ru[v].get(g);
      // SiLU(x) * up.  16-bit inputs: the hardware's exponential and
      // reciprocal, a few units in fp32's last place, 2^-13 of an input's own.
      // fp32 inputs: both to the last place, as a caller who keeps 32 bits
      // expects.  Either way HBM is the bound (12,900 x 12,288: 5.5 and 5.1
      // TB/s).
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = f[v][e];
        if constexpr (sizeof(T) == 4)
          f[v][e] = a / (1.0f + expf(-a)) * g[e];
        else
          f[v][e] = a * __builtin_amdgcn_rcpf(1.0f + __expf(-a)) * g[e];
      }
    }
    // (a chunk's dropped elements are elements of the same row)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      m = max(m, __float_as_uint(f[v][e]) & 0x7fffffffu);
  }
  m = row_max_bits<TPR>(m, part);
  float scale, inv;
  row_scale(m, scale, inv);
  int8_t *q = P.q + r * P.ldq;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Chunk k((v * TPR + t) * 8, P.width);
    store_int8(q + k.c, k.lo, f[v], inv);
  }
  if (t == 0) P.scale[r] = scale;
}

// n = RMSNorm(x) * post_w (or x); h = residual_scale * residual + gate * n;
// z = RMSNorm(h) * pre_w (or h), as T or in 8 bits.  h stays in fp32 between
// its rounded copy in memory and the second norm.
struct NormParams {
  const void *x, *post_w, *gate, *res, *pre_w;
  void *h, *z;
  int8_t *q;
  float *q_scale;
  int64_t rows, ldx, ldg, ldr, ldh, ldz, ldq;
  int32_t width;
  float residual_scale, eps;
};

template <typename T, typename R, int TPR, int NV>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_norm_residual(
    NormParams P) {
  constexpr int kRows = TPR > 64 ? 1 : 4;
  // fp32 activations: sums in 64 bits, so that a row's factor is the nearest
  // fp32 to the exact one and its 8-bit form does not turn on the order
  using Sum = std::conditional_t<sizeof(T) == 4, double, float>;
  __shared__ Sum part[TPR / 64];
  const int t = TPR > 64 ? threadIdx.x : threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * kRows +
                    (TPR > 64 ? 0 : threadIdx.x >> 6);
  if (r >= P.rows) return;
  const int W = P.width;
  // everything the row reads is on its way before the first sum is waited for
  const T *x = static_cast<const T *>(P.x) + r * P.ldx;
  Raw8<T> rx[NV], rg[NV];
  Raw8<R> rr[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v)
    rx[v].load(x + Chunk((v * TPR + t) * 8, W).c);
  if (P.res) {
    const R *p = static_cast<const R *>(P.res) + r * P.ldr;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      rr[v].load(p + Chunk((v * TPR + t) * 8, W).c);
  }
  if (P.gate) {
    const T *p = static_cast<const T *>(P.gate) + r * P.ldg;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      rg[v].load(p + Chunk((v * TPR + t) * 8, W).c);
  }
  float f[NV][8];
  float g[8];
#pragma unroll
  for (int v = 0; v < NV; ++v) rx[v].get(f[v]);
  // f = RMSNorm(f) * gain
  auto norm = [&](const void *gain) {
    const T *w = static_cast<const T *>(gain);
    Raw8<T> rw[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v)
      rw[v].load(w + Chunk((v * TPR + t) * 8, W).c);
    auto squares = [&]() {
      Sum ss = 0;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          ss = fma((Sum)f[v][e], (Sum)f[v][e], ss);
      return (float)(row_sum<TPR>(ss, part) / (Sum)W);
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) Chunk((v * TPR + t) * 8, W).mask(f[v]);
    float mean = squares(), eps = P.eps;
    if (mean == __builtin_inff()) {
      // squares past fp32's range (values over 2^55 or so; the whole row
      // takes this turn together): the same with the row 2^80 times smaller
      eps *= 0x1p-80f * 0x1p-80f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) f[v][e] *= 0x1p-80f;
      mean = squares();
    }
    const float inv = 1.0f / sqrtf(mean + eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      rw[v].get(g);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[v][e] = f[v][e] * inv * g[e];
    }
  };
  if (P.post_w) norm(P.post_w);
  if (P.gate) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      rg[v].get(g);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[v][e] *= g[e];
    }
  }
  if (P.res) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      rr[v].get(g);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[v][e] += P.residual_scale * g[e];
    }
  }
  if (P.h) {
    R *p = static_cast<R *>(P.h) + r * P.ldh;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Chunk k((v * TPR + t) * 8, W);
      store8<R, true>(p + k.c, k.lo, f[v]);
    }
  }
  if (!P.z && !P.q) return;
  if (P.pre_w) norm(P.pre_w);
  if (P.z) {
    T *p = static_cast<T *>(P.z) + r * P.ldz;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Chunk k((v * TPR + t) * 8, W);
      store8<T, true>(p + k.c, k.lo, f[v]);
    }
  }
  if (P.q) {
    uint32_t m = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Chunk((v * TPR + t) * 8, W).mask(f[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        m = max(m, __float_as_uint(f[v][e]) & 0x7fffffffu);
    }
    m = row_max_bits<TPR>(m, reinterpret_cast<uint32_t *>(part));
    float scale, inv;
    row_scale(m, scale, inv);
    int8_t *q = P.q + r * P.ldq;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Chunk k((v * TPR + t) * 8, W);
      store_int8(q + k.c, k.lo, f[v], inv);
    }
    if (t == 0) P.q_scale[r] = scale;
  }
}

// The instance that holds a row of `width`: f(threads per row, chunks).
template <typename F>
hipError_t by_width(int64_t width, F f) {
  using std::integral_constant;
#define DOPR_ROW(tpr, nv)                                                  \
  if (width <= (int64_t)(tpr) * 8 * (nv))                                  \
    return f(integral_constant<int, tpr>{}, integral_constant<int, nv>{});
  DOPR_ROW(64, 1)
  DOPR_ROW(64, 2)
  DOPR_ROW(64, 4)
  DOPR_ROW(256, 2)
  DOPR_ROW(256, 4)
  DOPR_ROW(512, 4)
  DOPR_ROW(1024, 4)
  DOPR_ROW(1024, 8)
#undef DOPR_ROW
  return hipErrorInvalidValue;
}

template <int TPR>
void row_grid(int64_t rows, dim3 &grid, dim3 &block) {
  grid = dim3((unsigned)(TPR > 64 ? rows : (rows + 3) / 4));
  block = dim3(TPR > 256 ? TPR : 256);
}

template <typename T>
hipError_t quantize(const QuantizeParams &P, hipStream_t s) {
  return by_width(P.width, [&](auto tpr, auto nv) {
    dim3 grid, block;
    row_grid<tpr.value>(P.rows, grid, block);
    if (P.up)
      hipLaunchKernelGGL((k_quantize_rows<T, tpr.value, nv.value, true>), grid,
                         block, 0, s, P);
    else
      hipLaunchKernelGGL((k_quantize_rows<T, tpr.value, nv.value, false>),
                         grid, block, 0, s, P);
    return hipGetLastError();
  });
}

template <typename T, typename R>
hipError_t norm(const NormParams &P, hipStream_t s) {
  return by_width(P.width, [&](auto tpr, auto nv) {
    dim3 grid, block;
    row_grid<tpr.value>(P.rows, grid, block);
    hipLaunchKernelGGL((k_norm_residual<T, R, tpr.value, nv.value>), grid,
                       block, 0, s, P);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_quantize_rows(const dopr_quantize_args_t &a, hipStream_t s) {
  const QuantizeParams P{a.x,
                         a.up,
                         a.q,
                         a.scale,
                         a.rows,
                         a.x_row_stride,
                         a.up_row_stride,
                         a.q_row_stride,
                         (int32_t)a.width};
  if (a.dtype == DOPR_BF16) return quantize<bf16_t>(P, s);
  if (a.dtype == DOPR_F16) return quantize<_Float16>(P, s);
  return quantize<float>(P, s);
}

hipError_t launch_norm_residual(const dopr_norm_residual_args_t &a,
                                hipStream_t s) {
  const NormParams P{a.x,
                     a.post_norm_w,
                     a.gate,
                     a.residual,
                     a.pre_norm_w,
                     a.h,
                     a.z,
                     a.q,
                     a.q_scale,
                     a.rows,
                     a.x_row_stride,
                     a.gate_row_stride,
                     a.residual_row_stride,
                     a.h_row_stride,
                     a.z_row_stride,
                     a.q_row_stride,
                     (int32_t)a.width,
                     a.residual_scale,
                     a.rms_eps};
  const bool wide = a.residual_dtype == DOPR_F32;
  if (a.dtype == DOPR_BF16)
    return wide ? norm<bf16_t, float>(P, s) : norm<bf16_t, bf16_t>(P, s);
  if (a.dtype == DOPR_F16)
    return wide ? norm<_Float16, float>(P, s) : norm<_Float16, _Float16>(P, s);
  return norm<float, float>(P, s);
}

}  // namespace dopr
