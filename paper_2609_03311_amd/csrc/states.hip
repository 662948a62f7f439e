// states.hip -- prefix states into a store (k_put_states), keys normed and
// given their rotary positions on the way, and out of a 4-bit one
// (k_gather_fp4).
//
// A block takes chunks of 32 slots of one document, a wave the keys or the
// values of one kv head of a chunk at a time.  The chunk's rotations are formed
// once for all heads.  Rows come in as 128-byte runs: lane = 8 rg + c holds dims
// 64 j + 8 c .. + 7 (j < D/64) of slots 4 rg .. 4 rg + 3, so that a row's sum of
// squares is a butterfly over 8 lanes and a key block's maximum one over 4;
// those of the value blocks, two dims a word, are halved between the lanes at
// each step.  What is stored is laid out in the wave's part of LDS and leaves
// in whole lines.
//
// Keys are normed and turned in 64 bits and rounded at the end, to fp32 and from
// there to bf16, as a framework's conversion from 64 bits does it: a 4-bit store
// quantises that value, and a key off by a sum's order would now and then land on
// another code, half a step of the block away.  (Where fp32 rounds to the middle
// of two bf16 values, one normal value in 130,000, the key may be the farther one
// of the two.)
#include <type_traits>

#include "fp4.hpp"
#include "internal.hpp"
#include "operators.hpp"
#include "rowio.hpp"

namespace dopr {
namespace {

constexpr int kPutWaves = 4;  // of a block, at most

struct PutParams {
  StoreView sv;
  int32_t *status;
  const int32_t *doc_ids;
  const int64_t *src_cu;
  const void *k, *v, *kw;
  int64_t k_row, k_head, v_row, v_head;  // strides in elements
  int64_t rows;
  const int32_t *positions;
  const float *inv_freq;
  int32_t layer, R, inter;
  float factor, eps;
};

__device__ __forceinline__ bool put_ok(const PutParams &P, int32_t d,
                                       int64_t s0, int64_t s1) {
  return d >= 0 && (int64_t)d < P.sv.n_docs && P.sv.doc_len[d] >= 0 &&
         s1 - s0 == P.sv.doc_len[d] && s0 >= 0 && s1 <= P.rows;
}

// The wave's earlier LDS accesses, and the compiler's, end here.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A zero the compiler cannot see through: what is formed from it is formed
// here, and not held in registers across the loops around.
__device__ __forceinline__ int opaque_zero() {
  int z;
  asm volatile("s_mov_b32 %0, 0" : "=s"(z));
  return z;
}

// Values of other lanes of a lane's eight: lane ^ 1, lane ^ 2, 7 - lane (the
// other four's, once those agree), lane ^ 4; of lane ^ 8.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return __builtin_amdgcn_mov_dpp(x, CTRL, 0xF, 0xF, false);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kReverse4 = 0x1B,
              kXor8 = 0x128;
__device__ __forceinline__ uint32_t xor4(uint32_t x) {
  return dpp<kReverse4>(dpp<kMirror8>(x));
}
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)dpp<CTRL>(u >> 32) << 32 |
                                        dpp<CTRL>((uint32_t)u));
}
__device__ __forceinline__ double sum8(double x) {
  x += dpp_f64<kXor1>(x);
  x += dpp_f64<kXor2>(x);
  return x + dpp_f64<kMirror8>(x);
}
__device__ __forceinline__ float sum8(float x) {
  x += __uint_as_float(dpp<kXor1>(__float_as_uint(x)));
  x += __uint_as_float(dpp<kXor2>(__float_as_uint(x)));
  return x + __uint_as_float(dpp<kMirror8>(__float_as_uint(x)));
}

// The lane whose perm32 is r: the place of slot (or dim) r of a chunk.
__device__ __forceinline__ int lane_of(int r) {
  return ((r >> 2) & 3) * 8 + (r >> 4) * 4 + (r & 3);
}

// Two bf16 values in a word: magnitudes, the larger of each half.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t mag2(uint32_t x) { return x & 0x7fff7fffu; }
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(
      uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                          __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) {
  return a > b ? a : b;
}

// Codes of two bf16 values into byte SEL of w.
template <int SEL>
__device__ __forceinline__ uint32_t fp4_codes2(uint32_t w, uint32_t pair,
                                               float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(
      w, __builtin_bit_cast(fp4_bf16x2, pair), scale, SEL);
}

// (out of line: the rotations' loop holds two of its callers)
__device__ __attribute__((noinline)) double2 cos_sin_far(double x) {
  double sn, cs;
  sincos(x, &sn, &cs);
  return double2{cs, sn};
}

// sin and cos of x in 64 bits: x less its quarter turns (pi / 2 in two parts,
// to 2^-106 of itself) and the Taylor series, whose first terms left out are
// under 2^-60 at pi / 4.  From |x| = 2^45 on (frequencies no model has) the
// library's.
__device__ __forceinline__ double2 cos_sin(double x) {
  if (!(fabs(x) < 0x1p45)) return cos_sin_far(x);
  const double n = rint(x * 0.63661977236758134308);
  double r = fma(n, -1.57079632679489655800e+00, x);
  r = fma(n, -6.12323399573676603587e-17, r);
  const double q = r * r;
  double s = 1.0 / 355687428096000.0;  // 17!
  s = fma(s, q, -1.0 / 1307674368000.0);
  s = fma(s, q, 1.0 / 6227020800.0);
  s = fma(s, q, -1.0 / 39916800.0);
  s = fma(s, q, 1.0 / 362880.0);
  s = fma(s, q, -1.0 / 5040.0);
  s = fma(s, q, 1.0 / 120.0);
  s = fma(s, q, -1.0 / 6.0);
  s = fma(s * q, r, r);
  double c = -1.0 / 6402373705728000.0;  // 18!
  c = fma(c, q, 1.0 / 20922789888000.0);
  c = fma(c, q, -1.0 / 87178291200.0);
  c = fma(c, q, 1.0 / 479001600.0);
  c = fma(c, q, -1.0 / 3628800.0);
  c = fma(c, q, 1.0 / 40320.0);
  c = fma(c, q, -1.0 / 720.0);
  c = fma(c, q, 1.0 / 24.0);
  c = fma(c, q, -0.5);
  c = fma(c, q, 1.0);
  const int64_t k = (int64_t)n;
  const double a = k & 1 ? s : c, b = k & 1 ? c : s;
  return double2{(k + 1) & 2 ? -a : a, k & 2 ? -b : b};
}

// The chunk's rotations in LDS: pair i of slot r, in the order in which eight
// lanes (pairs 8 c + e, c = 0 .. 7) read them side by side; rows 32 bytes off
// a multiple of the banks.
template <int D>
struct Turns {
  static constexpr int PITCH = D / 2 + 2;
  double2 at[kChunkSlots * PITCH];
  static __device__ __forceinline__ int place(int r, int pair, int groups) {
    return r * PITCH + (pair & 7) * groups + (pair >> 3);
  }
};

// Bytes of LDS a wave lays its chunk out in: the chunk itself, or V^T rows of
// 32 slots (40 elements apart: 16-byte pieces on different banks).
template <int D, bool FP4>
constexpr int stage_bytes() {
  return FP4 ? fp4_chunk_bytes(D) : D * 40 * 2;
}

// Eight elements in four words of two bf16.
__device__ __forceinline__ void round8(const Raw8<bf16_t> &x, uint32_t *w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = x.u[i];
}
template <typename T>
__device__ __forceinline__ void round8(const Raw8<T> &x, uint32_t *w) {
  float f[8];
  x.get(f);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack2<bf16_t>(f[2 * i], f[2 * i + 1]);
}

// A value times its gain, exact: in fp32 for two fp16 values; the product of two
// bf16 values fits fp32's bits, but not its range.  (1,024 documents of 256 slots
// in bf16 381 -> 389 us for it.)
template <typename T>
__device__ __forceinline__ double times(float x, float w) {
  return std::is_same_v<T, _Float16> ? (double)(x * w) : (double)x * w;
}

// What a wave knows of its chunk.
template <typename T>
struct Share {
  const T *base;       // the head's first element of the document's first row
  int64_t row;         // elements between rows
  int slot0, L;        // the chunk's first slot; the document's
  int c, rg, lane;
  __device__ __forceinline__ const T *from(int it) const {
    const int slot = slot0 + 4 * rg + it;  // (past the end: the last one again)
    return base + (int64_t)(slot < L ? slot : L - 1) * row;
  }
  __device__ __forceinline__ bool whole() const {
    return slot0 + kChunkSlots <= L;
  }
  __device__ __forceinline__ bool has(int it) const {
    return slot0 + 4 * rg + it < L;
  }
};

// The elements of lane ^ 4.
__device__ __forceinline__ Raw8<bf16_t> xor4(const Raw8<bf16_t> &x) {
  Raw8<bf16_t> y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y.u[i] = xor4(x.u[i]);
  return y;
}
__device__ __forceinline__ Raw8<_Float16> xor4(const Raw8<_Float16> &x) {
  Raw8<_Float16> y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y.u[i] = xor4(x.u[i]);
  return y;
}
__device__ __forceinline__ Raw8<float> xor4(const Raw8<float> &x) {
  Raw8<float> y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y.a.u[i] = xor4(x.a.u[i]);
    y.b.u[i] = xor4(x.b.u[i]);
  }
  return y;
}

// One of four (selected word by word: an array would be indexed in memory).
__device__ __forceinline__ u32x4 pick(int i, u32x4 a, u32x4 b, u32x4 c,
                                      u32x4 d) {
  u32x4 y;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t lo = i & 1 ? b[w] : a[w], hi = i & 1 ? d[w] : c[w];
    y[w] = i & 2 ? hi : lo;
  }
  return y;
}
template <typename T>
__device__ __forceinline__ Raw8<T> pick(int i, const Raw8<T> &a,
                                        const Raw8<T> &b, const Raw8<T> &c,
                                        const Raw8<T> &d) {
  Raw8<T> y;
  if constexpr (sizeof(T) == 2) {
    y.u = pick(i, a.u, b.u, c.u, d.u);
  } else {
    y.a.u = pick(i, a.a.u, b.a.u, c.a.u, d.a.u);
    y.b.u = pick(i, a.b.u, b.b.u, c.b.u, d.b.u);
  }
  return y;
}

// What becomes of the keys on their way.
enum KeyMode {
  kAsTheyAre,   // (dopr_store_put)
  kWholeHalf,   // the whole head turned, dim i with i + D/2
  kAnyRotation
};

// The keys of a chunk: K codes and exponents into `stage`, or bf16 rows to K.
// Returns the largest squared norm of what is held.
template <typename T, int D, bool FP4, KeyMode MODE>
__device__ __forceinline__ float put_keys(const PutParams &P, const Share<T> &h,
                                          const Turns<D> &turns, char *stage,
                                          uint16_t *K) {
  constexpr int NJ = D / 64;
  const int c = h.c, half = P.R / 2, groups = (half + 7) / 8;
  Raw8<T> own[4][NJ];
#pragma unroll
  for (int it = 0; it < 4; ++it)
#pragma unroll
    for (int j = 0; j < NJ; ++j) own[it][j].load(h.from(it) + 64 * j + 8 * c);
  const T *kw = static_cast<const T *>(P.kw);
  // 1 / rms of the lane's four rows: the eight lanes of a row each know its
  // sum of squares; lane c takes row c % 4's root
  double inv4 = 1.0;
  float gain[NJ][8], partner[8];  // (of lane ^ 4's run, at head size 64)
#pragma unroll
  for (int e = 0; e < 8; ++e) partner[e] = 1.f;
  if (MODE != kAsTheyAre && kw) {
    double ss[4];
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      ss[it] = 0.0;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float f[8];
        own[it][j].get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double x = f[e];
          ss[it] = fma(x, x, ss[it]);
        }
      }
      ss[it] = sum8(ss[it]);
    }
    const double lo = c & 1 ? ss[1] : ss[0], hi = c & 1 ? ss[3] : ss[2];
    inv4 = 1.0 / sqrt((c & 2 ? hi : lo) / D + (double)P.eps);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      Raw8<T> w;
      w.load(kw + 64 * j + 8 * c);
      w.get(gain[j]);
      if (MODE == kWholeHalf && D == 64) xor4(w).get(partner);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) gain[j][e] = 1.f;
  }
  const double inv0 = dpp_f64<0x00>(inv4), inv1 = dpp_f64<0x55>(inv4),
               inv2 = dpp_f64<0xAA>(inv4), inv3 = dpp_f64<0xFF>(inv4);
  float norm2 = 0.f;
  // (a loop: unrolled, the rows' 64-bit values do not fit the registers)
#pragma unroll 1
  for (int it = 0; it < 4; ++it) {
    const int r = 4 * h.rg + it;
    Raw8<T> cur[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      cur[j] = pick(it, own[0][j], own[1][j], own[2][j], own[3][j]);
    uint32_t pk[NJ][4];
    if constexpr (MODE == kAsTheyAre) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) round8(cur[j], pk[j]);
    } else {
      const double inv = it & 2 ? (it & 1 ? inv3 : inv2)
                                : (it & 1 ? inv1 : inv0);
      double x[NJ][8];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float f[8];
        cur[j].get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // (bf16 gains widened here: 64-bit ones held across the rows spill)
          if constexpr (std::is_same_v<T, bf16_t>)
            asm volatile("" : "+v"(gain[j][e]));
          x[j][e] = times<T>(f[e], gain[j][e]);
        }
      }
      // (turned, then by 1 / rms)
      if constexpr (MODE == kWholeHalf && D == 128) {
        // (the partner of dim i is i + 64, this lane's other run)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double2 t = turns.at[Turns<D>::place(r, 8 * c + e, 8)];
          const double a = x[0][e], b = x[NJ - 1][e];
          x[0][e] = fma(a, t.x, -(b * t.y));
          x[NJ - 1][e] = fma(b, t.x, a * t.y);
        }
      } else if constexpr (MODE == kWholeHalf) {
        // (i +- 32: the run of lane ^ 4)
        const Raw8<T> other = xor4(cur[0]);
        float of[8];
        other.get(of);
        const bool first = c < 4;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double2 t = turns.at[Turns<D>::place(r, 8 * (c & 3) + e, 4)];
          const double y = times<T>(of[e], partner[e]);
          x[0][e] = fma(x[0][e], t.x, first ? -(y * t.y) : y * t.y);
        }
      } else if (P.inter) {
        const int c0 = c + opaque_zero();
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const int d = 64 * j + 8 * c0 + e;
            if (d >= P.R) continue;
            const double2 t = turns.at[Turns<D>::place(r, d / 2, groups)];
            const double a = x[j][e], b = x[j][e + 1];
            x[j][e] = fma(a, t.x, -(b * t.y));
            x[j][e + 1] = fma(b, t.x, a * t.y);
          }
      } else {
        // the partners come from memory again
        const int c0 = c + opaque_zero();
        const T *row = h.from(it);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int d0 = 64 * j + 8 * c0;
          if (d0 >= P.R) continue;
          if (half % 8 == 0) {
            const bool first = d0 < half;
            const int p0 = first ? d0 + half : d0 - half;
            Raw8<T> other, w;
            other.load(row + p0);
            float of[8], wf[8];
            other.get(of);
            if (kw) {
              w.load(kw + p0);
              w.get(wf);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const double y = kw ? times<T>(of[e], wf[e]) : (double)of[e];
              const double2 t = turns.at[Turns<D>::place(
                  r, (first ? d0 : p0) + e, groups)];
              x[j][e] = first ? fma(x[j][e], t.x, -(y * t.y))
                              : fma(x[j][e], t.x, y * t.y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int d = d0 + e;
              if (d >= P.R) continue;
              const bool first = d < half;
              const int p = first ? d + half : d - half;
              const double y =
                  times<T>(to_f32<T>(row[p]), kw ? to_f32<T>(kw[p]) : 1.f);
              const double2 t =
                  turns.at[Turns<D>::place(r, first ? d : p, groups)];
              x[j][e] = first ? fma(x[j][e], t.x, -(y * t.y))
                              : fma(x[j][e], t.x, y * t.y);
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          pk[j][e / 2] = pack2<bf16_t>((float)(x[j][e] * inv),
                                       (float)(x[j][e + 1] * inv));
    }
    if (!h.whole())
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) pk[j][i] = h.has(it) ? pk[j][i] : 0u;
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if constexpr (FP4) {
        uint32_t m = max2(max2(mag2(pk[j][0]), mag2(pk[j][1])),
                          max2(mag2(pk[j][2]), mag2(pk[j][3])));
        m = umax(m & 0xffff, m >> 16);
        m = umax(m, dpp<kXor2>(m));
        m = umax(m, xor4(m));
        const uint32_t b = fp4_exponent(m << 16);
        const float scale = fp4_scale(b);
        uint32_t w = fp4_codes2<0>(0, pk[j][0], scale);
        w = fp4_codes2<1>(w, pk[j][1], scale);
        w = fp4_codes2<2>(w, pk[j][2], scale);
        w = fp4_codes2<3>(w, pk[j][3], scale);
        const int at = (c & 1) * 32 + lane_of(r);
        *reinterpret_cast<uint32_t *>(stage + 1024 * j + 16 * at +
                                      4 * (c >> 1)) = w;
        if (c < 2)
          *reinterpret_cast<uint8_t *>(stage + 32 * D + at * NJ + j) =
              (uint8_t)b;
        // (the norm's bound is of what is held)
        const uint4 held =
            __builtin_bit_cast(uint4, fp4_fragment(w, scale));
        const uint32_t hw[4] = {held.x, held.y, held.z, held.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const fp4_bf16x2 v = __builtin_bit_cast(fp4_bf16x2, hw[i]);
          ss = __builtin_amdgcn_fdot2_f32_bf16(v, v, ss, false);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float a, b;
          unpack2<bf16_t>(pk[j][i], a, b);
          ss = fmaf(a, a, fmaf(b, b, ss));
        }
        if (h.has(it))
          *reinterpret_cast<u32x4 *>(K + (int64_t)(h.slot0 + r) * D + 64 * j +
                                     8 * c) =
              u32x4{pk[j][0], pk[j][1], pk[j][2], pk[j][3]};
      }
    }
    norm2 = fmaxf(norm2, sum8(ss));
  }
  norm2 = fmaxf(norm2, __shfl_xor(norm2, 8, 64));
  norm2 = fmaxf(norm2, __shfl_xor(norm2, 16, 64));
  return fmaxf(norm2, __shfl_xor(norm2, 32, 64));
}

// The values of a chunk: V codes and exponents, or V^T rows, into `stage`.
template <typename T, int D, bool FP4>
__device__ __forceinline__ void put_values(const Share<T> &h, char *stage) {
  constexpr int NJ = D / 64, NW = 4 * NJ;  // words of two dims a row
  const int c = h.c, rg = h.rg;
  uint32_t v[4][NW];
  {
    Raw8<T> raw[4][NJ];
#pragma unroll
    for (int it = 0; it < 4; ++it)
#pragma unroll
      for (int j = 0; j < NJ; ++j) raw[it][j].load(h.from(it) + 64 * j + 8 * c);
#pragma unroll
    for (int it = 0; it < 4; ++it)
#pragma unroll
      for (int j = 0; j < NJ; ++j) round8(raw[it][j], &v[it][4 * j]);
  }
  if (!h.whole())
#pragma unroll
    for (int it = 0; it < 4; ++it)
#pragma unroll
      for (int i = 0; i < NW; ++i) v[it][i] = h.has(it) ? v[it][i] : 0u;
  // the low (high) halves of two rows' words: two slots of one dim
  auto low = [](uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, 0x05040100u);
  };
  auto high = [](uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, 0x07060302u);
  };
  if constexpr (!FP4) {
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const int d = 64 * (i / 4) + 8 * c + 2 * (i % 4);
      uint2 *to = reinterpret_cast<uint2 *>(stage + (d * 40 + 4 * rg) * 2);
      to[0] = make_uint2(low(v[0][i], v[1][i]), low(v[2][i], v[3][i]));
      to[10] = make_uint2(high(v[0][i], v[1][i]), high(v[2][i], v[3][i]));
    }
  } else {
    // magnitudes: over the lane's rows, then over the rgs, the words halved
    // between lanes 32 and 16 apart (a swap of two words leaves a lane its
    // own and its partner's of one of them)
    uint32_t m[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i)
      m[i] = max2(max2(mag2(v[0][i]), mag2(v[1][i])),
                  max2(mag2(v[2][i]), mag2(v[3][i])));
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) {
      const auto t = __builtin_amdgcn_permlane32_swap(m[i], m[i + NW / 2],
                                                      false, false);
      m[i] = max2(t[0], t[1]);
    }
#pragma unroll
    for (int i = 0; i < NW / 4; ++i) {
      const auto t = __builtin_amdgcn_permlane16_swap(m[i], m[i + NW / 4],
                                                      false, false);
      m[i] = max2(t[0], t[1]);
    }
    // exponents of the NW/2 dims that this lane is left with, a byte each
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < NW / 4; ++i) {
      m[i] = max2(m[i], dpp<kXor8>(m[i]));
      mine |= fp4_exponent(m[i] << 16) << (16 * i);
      mine |= fp4_exponent(m[i] & 0xffff0000u) << (16 * i + 8);
    }
    // everybody's: x[q] holds those of words q NW/4 .. of the four quarters
    uint32_t x[4];
    {
      const auto t = __builtin_amdgcn_permlane16_swap(mine, mine, false, false);
      const auto a = __builtin_amdgcn_permlane32_swap(t[0], t[0], false, false);
      const auto b = __builtin_amdgcn_permlane32_swap(t[1], t[1], false, false);
      x[0] = a[0];
      x[1] = b[0];
      x[2] = a[1];
      x[3] = b[1];
    }
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      // the word's two dims: four slots of each, 16 bits
      const uint32_t two = x[i / (NW / 4)] >> (16 * (i % (NW / 4)));
      const float s0 = fp4_scale(two & 255), s1 = fp4_scale(two >> 8 & 255);
      uint32_t a = fp4_codes2<0>(0, low(v[0][i], v[1][i]), s0);
      a = fp4_codes2<1>(a, low(v[2][i], v[3][i]), s0);
      uint32_t b = fp4_codes2<0>(0, high(v[0][i], v[1][i]), s1);
      b = fp4_codes2<1>(b, high(v[2][i], v[3][i]), s1);
      // with the rg next to this one (lane ^ 8), eight slots: the even one
      // makes the first dim's word, the odd one the second's
      const uint32_t both = low(a, b), other = dpp<kXor8>(both);
      const uint32_t w = rg & 1 ? high(other, both) : low(both, other);
      const int e = 2 * (i % 4) + (rg & 1);
      const int db = 2 * (i / 4) + (c >> 2);
      const int at = lane_of(8 * (c & 3) + e);
      const int fr = 2 * db + ((rg >> 1) & 1);
      *reinterpret_cast<uint32_t *>(stage + 16 * D + 1024 * (fr >> 2) +
                                    16 * ((rg >> 2) * 32 + at) +
                                    4 * (fr & 3)) = w;
      if (rg < 2)
        *reinterpret_cast<uint8_t *>(stage + 33 * D + at * (D / 32) + db) =
            (uint8_t)(rg & 1 ? two >> 8 : two);
    }
  }
}

// (fp32 rows, or the general rotations, of heads of 128 take more registers
// than three waves a SIMD have)
template <typename T, int D, bool FP4, KeyMode MODE>
__global__ __launch_bounds__(64 * kPutWaves,
                             D == 128 && (sizeof(T) == 4 ||
                                          MODE == kAnyRotation) ? 2 : 3)
void k_put_states(PutParams P) {
  __shared__ __attribute__((aligned(16))) Turns<D> turns;
  __shared__ __attribute__((aligned(16))) char
      stage_all[kPutWaves][stage_bytes<D, FP4>()];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int64_t i = blockIdx.x;
  const int32_t doc = P.doc_ids[i];
  const int64_t s0 = P.src_cu[i], s1 = P.src_cu[i + 1];
  if (!put_ok(P, doc, s0, s1)) {  // (the whole block)
    if (threadIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)
      raise_status(P.status, DOPR_ERR_DOC_RANGE);
    return;
  }
  const int hkv = P.sv.n_kv_heads;
  const int32_t L = P.sv.doc_len[doc], Lp = pad8(L);
  const int64_t blk = P.sv.doc_off[doc];
  float *kmax =
      P.sv.kmax + ((int64_t)doc * P.sv.n_layers + P.layer) * hkv;
  char *stage = stage_all[wave];
  const int n_chunks = (L + kChunkSlots - 1) / kChunkSlots;
  const int half = P.R / 2, groups = (half + 7) / 8;
  if (L == 0 && gridDim.y == 1 && blockIdx.z == 0)
    for (int g = threadIdx.x; g < hkv; g += blockDim.x) kmax[g] = 0.f;

  for (int ch = blockIdx.y; ch < n_chunks; ch += gridDim.y) {
    const int slot0 = ch * kChunkSlots;
    if constexpr (MODE != kAsTheyAre) {
      __syncthreads();  // (the chunk before is done with the table)
      const int n = min(kChunkSlots, L - slot0) * half;
#pragma unroll 2
      for (int e = threadIdx.x; e < n; e += blockDim.x) {
        const int r = (unsigned)e / half, pair = e - r * half;
        const int slot = slot0 + r;
        const int32_t pos = P.positions ? P.positions[s0 + slot] : slot;
        double2 t = cos_sin((double)pos * (double)P.inv_freq[pair]);
        t.x *= P.factor;
        t.y *= P.factor;
        turns.at[Turns<D>::place(r, pair, groups)] = t;
      }
      __syncthreads();
    }
    // (head, keys or values) by turns, so that every wave gets some of both;
    // the turns shared between gridDim.z blocks
    for (int k = blockIdx.z; k * waves < 2 * hkv; k += gridDim.z) {
      const int task = k * waves + (wave + k) % waves;
      if (task >= 2 * hkv) continue;
      const int g = task >> 1;
      Share<T> h;
      h.slot0 = slot0;
      h.L = L;
      h.lane = lane + opaque_zero();
      h.c = h.lane & 7;
      h.rg = h.lane >> 3;
      char *chunk = reinterpret_cast<char *>(
                        P.sv.payload +
                        fp4_offset(blk, L, hkv, P.layer, g, D)) +
                    (int64_t)ch * fp4_chunk_bytes(D);
      if (!(task & 1)) {
        h.base = static_cast<const T *>(P.k) + s0 * P.k_row + g * P.k_head;
        h.row = P.k_row;
        uint16_t *K = FP4 ? nullptr
                          : P.sv.payload +
                                k_offset(blk, L, hkv, P.layer, g, D);
        const float norm2 = put_keys<T, D, FP4, MODE>(P, h, turns, stage, K);
        if (lane == 0) {
          // relative slack covers the fp32 rounding of the sum and the sqrt
          const float bound = sqrtf(norm2) * 1.0001f;
          // (no other stripe of the document: this wave takes the head's keys
          // of every chunk; else cleared by a launch in front, and
          // not negative: ordered as bits)
          if (gridDim.y == 1)
            kmax[g] = ch == 0 ? bound : fmaxf(kmax[g], bound);
          else
            atomicMax(reinterpret_cast<int *>(kmax + g),
                      __float_as_int(bound));
        }
        if constexpr (FP4) {
          wave_fence();
#pragma unroll
          for (int o = 0; o < 16 * D; o += 1024)
            *reinterpret_cast<fp4_u32x4 *>(chunk + o + 16 * lane) =
                *reinterpret_cast<const fp4_u32x4 *>(stage + o + 16 * lane);
          if (16 * lane < D)
            *reinterpret_cast<fp4_u32x4 *>(chunk + 32 * D + 16 * lane) =
                *reinterpret_cast<const fp4_u32x4 *>(stage + 32 * D +
                                                     16 * lane);
          wave_fence();
        }
      } else {
        h.base = static_cast<const T *>(P.v) + s0 * P.v_row + g * P.v_head;
        h.row = P.v_row;
        put_values<T, D, FP4>(h, stage);
        wave_fence();
        if constexpr (FP4) {
#pragma unroll
          for (int o = 16 * D; o < 32 * D; o += 1024)
            *reinterpret_cast<fp4_u32x4 *>(chunk + o + 16 * lane) =
                *reinterpret_cast<const fp4_u32x4 *>(stage + o + 16 * lane);
          if (16 * lane < D)
            *reinterpret_cast<fp4_u32x4 *>(chunk + 33 * D + 16 * lane) =
                *reinterpret_cast<const fp4_u32x4 *>(stage + 33 * D +
                                                     16 * lane);
        } else {
          uint16_t *VT =
              P.sv.payload + vt_offset(blk, L, hkv, P.layer, g, D);
          for (int d = lane >> 2; d < D; d += 16) {
            const int q = lane & 3, slot = slot0 + 8 * q;
            if (slot < Lp)  // (Lp a multiple of 8: whole pieces)
              *reinterpret_cast<fp4_u32x4 *>(VT + (int64_t)d * Lp + slot) =
                  *reinterpret_cast<const fp4_u32x4 *>(stage +
                                                       (d * 40 + 8 * q) * 2);
          }
        }
        wave_fence();
      }
    }
  }
}

// The key-norm bounds of documents whose chunks go to several blocks.
__global__ __launch_bounds__(256) void k_put_clear(PutParams P, int64_t n) {
  const int hkv = P.sv.n_kv_heads;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n * hkv;
       e += (int64_t)gridDim.x * 256) {
    const int64_t i = e / hkv;
    const int32_t doc = P.doc_ids[i];
    if (put_ok(P, doc, P.src_cu[i], P.src_cu[i + 1]))
      P.sv.kmax[((int64_t)doc * P.sv.n_layers + P.layer) * hkv + e % hkv] =
          0.f;
  }
}

// Held values as bf16, in canonical [slots][Hkv][D] rows.  A wave takes one
// chunk of one head, lays its rows out in LDS and writes them in whole lines.
template <int D>
__global__ __launch_bounds__(256) void k_gather_fp4(
    StoreView sv, int32_t *status, int32_t layer, const int32_t *doc_ids,
    const int64_t *out_cu, uint16_t *kout, uint16_t *vout) {
  // (rows 4 banks apart)
  constexpr int PITCH = D + 8;
  __shared__ __attribute__((aligned(16))) uint16_t
      rows_all[4][kChunkSlots][PITCH];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i = blockIdx.x;
  const int hkv = sv.n_kv_heads;
  const int32_t doc = doc_ids[i];
  const int64_t o0 = out_cu[i], o1 = out_cu[i + 1];
  if (doc < 0 || (int64_t)doc >= sv.n_docs || sv.doc_len[doc] < 0 ||
      o1 - o0 != sv.doc_len[doc]) {
    if (threadIdx.x == 0 && blockIdx.y == 0)
      raise_status(status, DOPR_ERR_DOC_RANGE);
    return;
  }
  const int32_t L = sv.doc_len[doc];
  const int64_t blk = sv.doc_off[doc];
  const int64_t n = (int64_t)((L + kChunkSlots - 1) / kChunkSlots) * hkv;
  uint16_t(*rows)[PITCH] = rows_all[wave];
  const int lq = lane & 31, hf = lane >> 5;
  const int mine = ((lq >> 2) & 1) * 16 + (lq >> 3) * 4 + (lq & 3);  // perm32
  for (int64_t u = blockIdx.y * 4 + wave; u < n; u += 4 * gridDim.y) {
    const int ch = (int)(u / hkv), g = (int)(u - (int64_t)ch * hkv);
    const char *chunk =
        reinterpret_cast<const char *>(
            sv.payload + fp4_offset(blk, L, hkv, layer, g, D)) +
        (int64_t)ch * fp4_chunk_bytes(D);
    Fp4Raw<D> kr, vr;
    fp4_load_k<D>(chunk, lane, kr);
    fp4_load_v<D>(chunk, lane, vr);
    const int n_rows = L - ch * kChunkSlots;
    auto leave = [&](uint16_t *out) {
      wave_fence();
#pragma unroll
      for (int o = 0; o < kChunkSlots * D / 8; o += 64) {
        const int r = (o + lane) / (D / 8), p = (o + lane) % (D / 8);
        if (r < n_rows)
          *reinterpret_cast<fp4_u32x4 *>(
              out + ((o0 + ch * kChunkSlots + r) * hkv + g) * D + 8 * p) =
              *reinterpret_cast<const fp4_u32x4 *>(&rows[r][8 * p]);
      }
      wave_fence();
    };
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      *reinterpret_cast<fp4_bf16x8 *>(&rows[mine][16 * s + 8 * hf]) =
          fp4_k<D>(kr, s);
    leave(kout);
#pragma unroll
    for (int f = 0; f < D / 16; ++f) {
      const fp4_bf16x8 h = fp4_v<D>(vr, f);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        rows[16 * hf + 8 * (f & 1) + e][32 * (f >> 1) + mine] =
            __builtin_bit_cast(uint16_t, (__bf16)h[e]);
    }
    leave(vout);
  }
}

// Blocks that share a document's chunks: enough to fill the card, as far as
// its longest document has chunks.
unsigned stripes(int64_t n, int64_t chunks) {
  const int64_t want = (4096 + n - 1) / n;
  const int64_t y = want < chunks ? want : chunks;
  return (unsigned)(y < 1 ? 1 : y > 65535 ? 65535 : y);
}

// Blocks that share a chunk's heads, each forming its rotations again: until
// 512 are there (one document of 32 slots, 8 heads: 16 -> 9.6 us).
unsigned head_groups(int64_t blocks, int hkv) {
  const int64_t turns = (2 * (int64_t)hkv + kPutWaves - 1) / kPutWaves;
  const int64_t want = 512 / blocks;
  const int64_t z = want < turns ? want : turns;
  return (unsigned)(z < 1 ? 1 : z > 65535 ? 65535 : z);
}

template <typename T, int D, bool FP4>
void launch_put1(const PutParams &P, dim3 grid, hipStream_t s) {
  const int tasks = 2 * P.sv.n_kv_heads;
  const int waves = tasks < kPutWaves ? tasks : kPutWaves;
  auto kernel = P.R == D && !P.inter ? k_put_states<T, D, FP4, kWholeHalf>
                                     : k_put_states<T, D, FP4, kAnyRotation>;
  if constexpr (FP4 && std::is_same_v<T, bf16_t>)
    if (P.R == 0) kernel = k_put_states<T, D, true, kAsTheyAre>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, s, P);
}

template <typename T>
void launch_put(int D, bool fp4, const PutParams &P, dim3 grid,
                hipStream_t s) {
  if (D == 128)
    fp4 ? launch_put1<T, 128, true>(P, grid, s)
        : launch_put1<T, 128, false>(P, grid, s);
  else
    fp4 ? launch_put1<T, 64, true>(P, grid, s)
        : launch_put1<T, 64, false>(P, grid, s);
}

}  // namespace

hipError_t launch_put_states(const dopr_store &st,
                             const dopr_put_rotary_args_t &a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  PutParams P{};
  P.sv = st.view();
  P.status = st.d_status;
  P.doc_ids = a.doc_ids;
  P.src_cu = a.src_cu_slots;
  P.k = a.k;
  P.v = a.v;
  P.kw = a.k_norm_w;
  P.k_row = a.k_row_stride;
  P.k_head = a.k_head_stride;
  P.v_row = a.v_row_stride;
  P.v_head = a.v_head_stride;
  P.rows = a.rows;
  P.positions = a.positions;
  P.inv_freq = a.inv_freq;
  P.layer = a.layer;
  P.R = a.rotary_dim;
  P.inter = a.interleaved;
  P.factor = a.attention_factor;
  P.eps = a.rms_eps;
  return in_slices(a.n, a_launch(64 * kPutWaves), [&](int64_t at, int64_t n) {
    PutParams S = P;
    S.doc_ids = P.doc_ids + at;
    S.src_cu = P.src_cu + at;
    dim3 grid((unsigned)n, stripes(n, ((int64_t)st.max_len + kChunkSlots - 1) /
                                          kChunkSlots));
    grid.z = head_groups((int64_t)grid.x * grid.y, st.n_kv_heads);
    if (grid.y > 1) {
      const int64_t blocks = (n * st.n_kv_heads + 255) / 256;
      hipLaunchKernelGGL(k_put_clear,
                         dim3((unsigned)(blocks < 4096 ? blocks : 4096)),
                         dim3(256), 0, s, S, n);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (a.dtype == DOPR_BF16)
      launch_put<bf16_t>(st.head_dim, st.fp4, S, grid, s);
    else if (a.dtype == DOPR_F16)
      launch_put<_Float16>(st.head_dim, st.fp4, S, grid, s);
    else
      launch_put<float>(st.head_dim, st.fp4, S, grid, s);
    return hipGetLastError();
  });
}

hipError_t launch_gather_fp4(const dopr_store &st, int32_t layer, int32_t n,
                             const int32_t *doc_ids, const int64_t *out_cu,
                             uint16_t *k, uint16_t *v, hipStream_t s) {
  if (n == 0) return hipSuccess;
  const int64_t waves =
      ((int64_t)st.max_len + kChunkSlots - 1) / kChunkSlots * st.n_kv_heads;
  return in_slices(n, a_launch(256), [&](int64_t at, int64_t m) {
    const dim3 grid((unsigned)m, stripes(m, (waves + 3) / 4));
    const auto kernel =
        st.head_dim == 128 ? k_gather_fp4<128> : k_gather_fp4<64>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, st.view(), st.d_status,
                       layer, doc_ids + at, out_cu + at, k, v);
    return hipGetLastError();
  });
}

}  // namespace dopr
