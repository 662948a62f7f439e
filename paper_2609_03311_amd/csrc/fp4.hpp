// fp4.hpp -- prefix states held in 4 bits (DOPR_STORE_FP4).
//
// A value is a 4-bit float (sign, 2 bits of exponent, 1 of mantissa: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6) times its block's power of two, whose biased exponent is a
// byte; a block is 32 values.  Both halves are powers of two times at most two
// bits, so a held value is a bf16 value, and gfx950 makes two of them out of a
// byte of codes and a scale in one instruction (as fast as an addition), and
// codes out of fp32 pairs, to nearest, ties to the even code.
//
// Chunks of 32 slots, 34*D bytes, in the order in which a wave's lanes take
// them as MFMA operands (lane = 32 hf + lq):
//   [K codes  16*D] part j < D/64, lane, 16 bytes: fragments s = 4j .. 4j + 3
//                   of slot perm32(lq), dims 16 s + 8 hf + e, e = 0..7 from the
//                   lowest nibble up
//   [V codes  16*D] part j, lane, 16 bytes: fragments f = 4j .. 4j + 3, (db, t)
//                   = (f / 2, f % 2): dim 32 db + perm32(lq), slots 16 hf + 8 t
//                   + e
//   [K exps     D ] lane, D/64 bytes: the block of its part's fragments
//   [V exps     D ] lq, D/32 bytes (db): the block of dim 32 db + perm32(lq)
// so a K block is the 32 dims of a part that one lane holds, and a V block one
// dim of the chunk's slots.  Slots behind the document's end are zeros.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace dopr {

constexpr int kChunkSlots = 32;
constexpr int fp4_chunk_bytes(int D) { return 34 * D; }
// Exponent bytes: 2^-125 .. 2^125, so that every held value, 0.5 * 2^-125 and
// 6 * 2^125 among them, is a normal bf16 value; 255: a block with a value that
// is not finite, all NaN.
constexpr int kFp4ExpMin = 2, kFp4ExpMax = 252, kFp4Nan = 255;

typedef uint32_t fp4_u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 fp4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 fp4_bf16x8 __attribute__((ext_vector_type(8)));

// The scale of exponent byte `b` (255 has an infinity's exponent, which the
// conversions take for NaN).
__device__ __forceinline__ float fp4_scale(uint32_t b) {
  return __uint_as_float(b << 23);
}

// Exponent byte of a block whose largest magnitude has the bits m: the
// smallest e with 7 * 2^e >= it, so that no value is off by more than 2^e,
// half of the widest step (a maximum over 6 * 2^e goes to 6 * 2^e).
__device__ __forceinline__ uint32_t fp4_exponent(uint32_t m) {
  const int e = (int)(m >> 23);
  // 7 * 2^e = 1.75 * 2^(e + 2)
  const int b = e - 2 + ((m & 0x7fffff) > 0x600000);
  if (e == 255) return kFp4Nan;
  return (uint32_t)(b < kFp4ExpMin ? kFp4ExpMin
                                   : b > kFp4ExpMax ? kFp4ExpMax : b);
}

// Eight held values as a bf16 MFMA operand.
__device__ __forceinline__ fp4_bf16x8 fp4_fragment(uint32_t w, float scale) {
  const fp4_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const fp4_bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const fp4_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const fp4_bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return fp4_bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// A lane's codes and exponents of a chunk's K and V, as they lie in memory or
// LDS.
template <int D>
struct Fp4Raw {
  fp4_u32x4 c[D / 64];
  uint32_t exps;
};

template <int D>
__device__ __forceinline__ void fp4_load_k(const char *chunk, int lane,
                                           Fp4Raw<D> &r) {
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
    r.c[j] = *reinterpret_cast<const fp4_u32x4 *>(chunk + 1024 * j + 16 * lane);
  const char *x = chunk + 32 * D + lane * (D / 64);
  if constexpr (D == 128)
    r.exps = *reinterpret_cast<const uint16_t *>(x);
  else
    r.exps = *reinterpret_cast<const uint8_t *>(x);
}

template <int D>
__device__ __forceinline__ void fp4_load_v(const char *chunk, int lane,
                                           Fp4Raw<D> &r) {
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
    r.c[j] = *reinterpret_cast<const fp4_u32x4 *>(chunk + 16 * D + 1024 * j +
                                                  16 * lane);
  const char *x = chunk + 33 * D + (lane & 31) * (D / 32);
  if constexpr (D == 128)
    r.exps = *reinterpret_cast<const uint32_t *>(x);
  else
    r.exps = *reinterpret_cast<const uint16_t *>(x);
}

// K fragment s, V fragment f (constants once the caller's loops are unrolled).
template <int D>
__device__ __forceinline__ fp4_bf16x8 fp4_k(const Fp4Raw<D> &r, int s) {
  return fp4_fragment(r.c[s >> 2][s & 3], fp4_scale(r.exps >> (8 * (s >> 2)) &
                                                    255));
}
template <int D>
__device__ __forceinline__ fp4_bf16x8 fp4_v(const Fp4Raw<D> &r, int f) {
  return fp4_fragment(r.c[f >> 2][f & 3], fp4_scale(r.exps >> (8 * (f >> 1)) &
                                                    255));
}

}  // namespace dopr
