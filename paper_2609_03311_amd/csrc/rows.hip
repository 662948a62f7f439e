// rows.hip -- operators over the rows of an activation matrix, one pass over
// memory each: rows in 8-bit integers (k_quantize_rows) and the norms around a
// gated, scaled residual (k_norm_residual).
//
// A row is held by TPR threads (a wave, or a whole block), 8 NV elements each, so
// that its sums and its largest magnitude are known before its first output is
// written and no input is read twice.  Up to a width of 16,384 it is held in
// registers, and both kernels are bound by HBM: a row's arithmetic is some ten
// vector instructions per 8 elements (residual sum and norm of 12,900 x 4096 in
// bf16: 71 us, 6.0 TB/s; of 4000 x 16,384 92 us, 5.7 TB/s).  Wider rows of norms
// do not fit the 128 registers a lane of 1,024 threads: 30 to 106 a lane go
// through scratch where the residual is fp32, from 32,769 on 177 to 491 in every
// type (2000 x 32,768 in bf16 97 us, 5.4 TB/s, around an fp32 residual 159 us,
// 5.0, in fp32 254 us, 4.1; 1000 x 65,536 195, 368 and 510 us, 2.7 to 2.1 TB/s).
#include <type_traits>

#include "rowio.hpp"

namespace dopr {
namespace {

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

template <int E>
__device__ __forceinline__ void store_int8(int8_t *p, const Chunk<E> &k,
                                           const float *f, float inv) {
  // inf * 0 and NaN * 0 are NaN: a row that is not finite stores zeros
  uint32_t u[E / 4];
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
    u[i] = inv == 0.f ? 0u : pack_int8(f + 4 * i, inv);
  if (k.whole()) {
    if constexpr (E == 8)
      *reinterpret_cast<u32x2_any *>(p) = u32x2{u[0], u[1]};
    else
      *reinterpret_cast<u32_any *>(p) = u[0];
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e >= k.lo && e < k.hi) p[e] = (int8_t)(u[e >> 2] >> (8 * (e & 3)));
}

// Elements of a lane's chunk: 16 bytes of the widest type, so that a wave's
// loads and stores are whole lines (with 32 bytes a lane, half of each
// line is the next instruction's: norms of 12,900 x 4096 around an fp32 residual
// 108 us, with 16 97).
constexpr int chunk_of(int bytes) { return 16 / bytes; }

struct QuantizeParams {
  const void *x, *up;
  int8_t *q;
  float *scale;
  int64_t rows, ldx, ldu, ldq;
  int32_t width;
};

template <typename T, int TPR, int NV, bool UP>
__global__ __launch_bounds__(TPR > 64 ? TPR : 256) void k_quantize_rows(
    QuantizeParams P) {
  constexpr int kRows = TPR > 64 ? 1 : 4;
  constexpr int E = chunk_of(sizeof(T)), NC = NV * 8 / E;
  __shared__ uint32_t part[TPR / 64];
  const int t = TPR > 64 ? threadIdx.x : threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * kRows +
                    (TPR > 64 ? 0 : threadIdx.x >> 6);
  if (r >= P.rows) return;  // one wave per row here: no barrier is missed
  const T *x = static_cast<const T *>(P.x) + r * P.ldx;
  const T *up = static_cast<const T *>(P.up) + r * P.ldu;
  Raw<T, E> rx[NC], ru[NC];
#pragma unroll
  for (int v = 0; v < NC; ++v) {
    const Chunk<E> k((v * TPR + t) * E, P.width);
    rx[v].load(x + k.c);
    if constexpr (UP) ru[v].load(up + k.c);
  }
  float f[NC][E];
  uint32_t m = 0;
#pragma unroll
  for (int v = 0; v < NC; ++v) {
    rx[v].get(f[v]);
    if constexpr (UP) {
      float g[E];
      ru[v].get(g);
      // SiLU(x) * up.  16-bit inputs: the hardware's exponential and
      // reciprocal, off by 3 + |x| units of fp32's last place at most (the
      // exponential's argument is rounded), 2^-18 at |x| = 20, where an 8-bit
      // step is 2^-7; x under -89 counts as 0.
      // fp32 inputs: both to the last place, as a caller who keeps 32 bits
      // expects.  Either way HBM is the bound (12,900 x 12,288 in bf16:
      // 140 us, 5.7 TB/s).
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float a = f[v][e];
        if constexpr (sizeof(T) == 4)
          f[v][e] = a / (1.0f + expf(-a)) * g[e];
        else
          f[v][e] = a * __builtin_amdgcn_rcpf(1.0f + __expf(-a)) * g[e];
      }
    }
    // (a chunk's dropped elements are elements of the same row)
#pragma unroll
    for (int e = 0; e < E; ++e)
      m = max(m, __float_as_uint(f[v][e]) & 0x7fffffffu);
  }
  m = row_max_bits<TPR>(m, part);
  float scale, inv;
  row_scale(m, scale, inv);
  int8_t *q = P.q + r * P.ldq;
#pragma unroll
  for (int v = 0; v < NC; ++v) {
    const Chunk<E> k((v * TPR + t) * E, P.width);
    store_int8(q + k.c, k, f[v], inv);
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
  // Chunks start on the output's lines, not at the row's start, so that no
  // line is written in two parts by two waves: rows of 9001 64 -> 55 us.
  bool lines;
};

// Elements between p and the 64-element line of its buffer that it lies in.
template <typename T>
__device__ __forceinline__ int line_offset(const T *p) {
  return (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T)) & 63;
}

template <typename T, typename R, int TPR, int NV>
__global__ __launch_bounds__(TPR > 64 ? TPR : 256) void k_norm_residual(
    NormParams P) {
  constexpr int kRows = TPR > 64 ? 1 : 4;
  constexpr int E = chunk_of(sizeof(T) > sizeof(R) ? sizeof(T) : sizeof(R));
  constexpr int NC = NV * 8 / E;
  // fp32 activations: sums in 64 bits, so that a row's factor does not turn on
  // their order; it is then within 2 units of fp32's last place of the exact
  // one (the mean, the epsilon, the root and the reciprocal round)
  using Sum = std::conditional_t<sizeof(T) == 4, double, float>;
  __shared__ Sum part[TPR / 64];
  const int t = TPR > 64 ? threadIdx.x : threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * kRows +
                    (TPR > 64 ? 0 : threadIdx.x >> 6);
  if (r >= P.rows) return;
  const int W = P.width;
  const int shift =
      P.lines ? P.h ? line_offset(static_cast<const R *>(P.h) + r * P.ldh)
                    : line_offset(static_cast<const T *>(P.z) + r * P.ldz)
              : 0;
  // everything the row reads is on its way before the first sum is waited for
  const T *x = static_cast<const T *>(P.x) + r * P.ldx;
  Raw<T, E> rx[NC], rg[NC];
  Raw<R, E> rr[NC];
#pragma unroll
  for (int v = 0; v < NC; ++v)
    rx[v].load(x + Chunk<E>((v * TPR + t) * E - shift, W).c);
  if (P.res) {
    const R *p = static_cast<const R *>(P.res) + r * P.ldr;
#pragma unroll
    for (int v = 0; v < NC; ++v)
      rr[v].load(p + Chunk<E>((v * TPR + t) * E - shift, W).c);
  }
  if (P.gate) {
    const T *p = static_cast<const T *>(P.gate) + r * P.ldg;
#pragma unroll
    for (int v = 0; v < NC; ++v)
      rg[v].load(p + Chunk<E>((v * TPR + t) * E - shift, W).c);
  }
  float f[NC][E];
  float g[E];
#pragma unroll
  for (int v = 0; v < NC; ++v) rx[v].get(f[v]);
  // f = RMSNorm(f) * gain
  auto norm = [&](const void *gain) {
    const T *w = static_cast<const T *>(gain);
    Raw<T, E> rw[NC];
#pragma unroll
    for (int v = 0; v < NC; ++v)
      rw[v].load(w + Chunk<E>((v * TPR + t) * E - shift, W).c);
    auto squares = [&]() {
      Sum ss = 0;
#pragma unroll
      for (int v = 0; v < NC; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e)
          ss = fma((Sum)f[v][e], (Sum)f[v][e], ss);
      return (float)(row_sum<TPR>(ss, part) / (Sum)W);
    };
#pragma unroll
    for (int v = 0; v < NC; ++v) Chunk<E>((v * TPR + t) * E - shift, W).mask(f[v]);
    float mean = squares(), eps = P.eps;
    const bool large = mean == __builtin_inff();
    if (large || mean + eps < 0x1p-100f) {
      // squares out of fp32's range (values over 2^55 or so, or, with next to
      // no epsilon, all under 2^-42; the whole row takes this turn together):
      // the same with the row 2^80 times smaller, or 2^100 times larger
      const float by = large ? 0x1p-80f : 0x1p100f;
      eps = eps * by * by;
#pragma unroll
      for (int v = 0; v < NC; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) f[v][e] *= by;
      mean = squares();
    }
    const float inv = 1.0f / sqrtf(mean + eps);
#pragma unroll
    for (int v = 0; v < NC; ++v) {
      rw[v].get(g);
#pragma unroll
      for (int e = 0; e < E; ++e) f[v][e] = f[v][e] * inv * g[e];
    }
  };
  if (P.post_w) norm(P.post_w);
  if (P.gate) {
#pragma unroll
    for (int v = 0; v < NC; ++v) {
      rg[v].get(g);
#pragma unroll
      for (int e = 0; e < E; ++e) f[v][e] *= g[e];
    }
  }
  if (P.res) {
#pragma unroll
    for (int v = 0; v < NC; ++v) {
      rr[v].get(g);
#pragma unroll
      for (int e = 0; e < E; ++e) f[v][e] += P.residual_scale * g[e];
    }
  }
  if (P.h) {
    R *p = static_cast<R *>(P.h) + r * P.ldh;
#pragma unroll
    for (int v = 0; v < NC; ++v) {
      const Chunk<E> k((v * TPR + t) * E - shift, W);
      store_part<R, E, true>(p + k.c, k.lo, k.hi, f[v]);
    }
  }
  if (!P.z && !P.q) return;
  if (P.pre_w) norm(P.pre_w);
  if (P.z) {
    T *p = static_cast<T *>(P.z) + r * P.ldz;
#pragma unroll
    for (int v = 0; v < NC; ++v) {
      const Chunk<E> k((v * TPR + t) * E - shift, W);
      store_part<T, E, true>(p + k.c, k.lo, k.hi, f[v]);
    }
  }
  if (P.q) {
    uint32_t m = 0;
#pragma unroll
    for (int v = 0; v < NC; ++v) {
      Chunk<E>((v * TPR + t) * E - shift, W).mask(f[v]);
#pragma unroll
      for (int e = 0; e < E; ++e)
        m = max(m, __float_as_uint(f[v][e]) & 0x7fffffffu);
    }
    m = row_max_bits<TPR>(m, reinterpret_cast<uint32_t *>(part));
    float scale, inv;
    row_scale(m, scale, inv);
    int8_t *q = P.q + r * P.ldq;
#pragma unroll
    for (int v = 0; v < NC; ++v) {
      const Chunk<E> k((v * TPR + t) * E - shift, W);
      store_int8(q + k.c, k, f[v], inv);
    }
    if (t == 0) P.q_scale[r] = scale;
  }
}

constexpr int64_t kMostWidth = 65536;

// The instance that holds a row of `width`: f(threads per row, chunks of 8).
// Rows of a wave need no barrier, but hold few loads in flight once their
// registers keep waves out; idle lanes cost their loads.  20,011 x 2561, fp16
// around an fp32 residual: 135, 127, 137 us at (64, 6), (128, 3), (256, 2);
// 12,900 x 4096, bf16: 64, 61, 60 at (64, 8), (128, 4), (256, 2); 5000 x 9001:
// 54 at (256, 5), 55 at (512, 3).
template <typename F>
hipError_t by_width(int64_t width, F f) {
  using std::integral_constant;
#define DOPR_ROW(tpr, nv)                                                  \
  if (width <= (int64_t)(tpr) * 8 * (nv))                                  \
    return f(integral_constant<int, tpr>{}, integral_constant<int, nv>{});
  DOPR_ROW(64, 1)
  DOPR_ROW(64, 2)
  DOPR_ROW(64, 3)
  DOPR_ROW(64, 4)
  DOPR_ROW(128, 3)
  DOPR_ROW(256, 2)
  DOPR_ROW(256, 3)
  DOPR_ROW(256, 4)
  DOPR_ROW(256, 5)
  DOPR_ROW(512, 3)
  DOPR_ROW(512, 4)
  DOPR_ROW(1024, 4)
  DOPR_ROW(1024, 8)
#undef DOPR_ROW
  return hipErrorInvalidValue;
}

template <int TPR>
void row_grid(int64_t rows, dim3 &grid, dim3 &block) {
  grid = dim3((unsigned)(TPR > 64 ? rows : (rows + 3) / 4));
  block = dim3(TPR > 64 ? TPR : 256);
}

template <typename T>
hipError_t quantize(const QuantizeParams &P, hipStream_t s) {
  return by_width(P.width, [&](auto tpr, auto nv) {
    return in_slices(P.rows, a_launch(tpr.value), [&](int64_t r, int64_t n) {
      QuantizeParams S = P;
      S.rows = n;
      S.x = ahead(P.x, r * P.ldx * (int)sizeof(T));
      S.up = ahead(P.up, r * P.ldu * (int)sizeof(T));
      S.q = ahead(P.q, r * P.ldq);
      S.scale = P.scale + r;
      dim3 grid, block;
      row_grid<tpr.value>(n, grid, block);
      if (P.up)
        hipLaunchKernelGGL((k_quantize_rows<T, tpr.value, nv.value, true>),
                           grid, block, 0, s, S);
      else
        hipLaunchKernelGGL((k_quantize_rows<T, tpr.value, nv.value, false>),
                           grid, block, 0, s, S);
      return hipGetLastError();
    });
  });
}

template <typename T, typename R>
hipError_t norm(const NormParams &P, hipStream_t s) {
  return by_width(P.width + (P.lines ? 63 : 0), [&](auto tpr, auto nv) {
    return in_slices(P.rows, a_launch(tpr.value), [&](int64_t r, int64_t n) {
      NormParams S = P;
      S.rows = n;
      S.x = ahead(P.x, r * P.ldx * (int)sizeof(T));
      S.gate = ahead(P.gate, r * P.ldg * (int)sizeof(T));
      S.res = ahead(P.res, r * P.ldr * (int)sizeof(R));
      S.h = ahead(P.h, r * P.ldh * (int)sizeof(R));
      S.z = ahead(P.z, r * P.ldz * (int)sizeof(T));
      S.q = ahead(P.q, r * P.ldq);
      S.q_scale = ahead(P.q_scale, r * (int)sizeof(float));
      dim3 grid, block;
      row_grid<tpr.value>(n, grid, block);
      hipLaunchKernelGGL((k_norm_residual<T, R, tpr.value, nv.value>), grid,
                         block, 0, s, S);
      return hipGetLastError();
    });
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
  const bool wide = a.residual_dtype == DOPR_F32;
  const uintptr_t size = (a.h ? wide : a.dtype == DOPR_F32) ? 4 : 2;
  const uintptr_t out = reinterpret_cast<uintptr_t>(a.h ? a.h : a.z);
  const uintptr_t pitch = size * (a.h ? a.h_row_stride : a.z_row_stride);
  const bool lines =
      out && (out | pitch) % 128 != 0 && a.width + 63 <= kMostWidth;
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
                     a.rms_eps,
                     lines};
  if (a.dtype == DOPR_BF16)
    return wide ? norm<bf16_t, float>(P, s) : norm<bf16_t, bf16_t>(P, s);
  if (a.dtype == DOPR_F16)
    return wide ? norm<_Float16, float>(P, s) : norm<_Float16, _Float16>(P, s);
  return norm<float, float>(P, s);
}

}  // namespace dopr
