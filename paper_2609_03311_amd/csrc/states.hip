// states.hip -- prefix states into a store (k_put_states), keys normed and
// given their rotary positions on the way, and out of a 4-bit one
// (k_gather_fp4).
//
// A block takes chunks of 32 slots of one document, a wave one kv head of a
// chunk at a time.  The chunk's rotations are formed once for all heads.  Rows
// come in as 128-byte runs: lane = 8 rg + c holds dims 64 j + 8 c .. + 7 (j <
// D/64) of slots 4 rg .. 4 rg + 3, so that a row's sum of squares and a key
// block's maximum are butterflies over 8 and 4 lanes, a value block's one over
// the 8 rgs.  What is stored is laid out in the wave's part of LDS and leaves in
// whole lines.
//
// Keys are normed and turned in 64 bits and rounded once, to bf16: a 4-bit
// store quantises that value, and a key off by fp32's rounding would now and
// then land on another code, half a step of the block away (the matrix of
// values is read once from HBM; 64-bit operations run at the rate of 32-bit
// ones here).
#include <type_traits>

#include "fp4.hpp"
#include "internal.hpp"
#include "operators.hpp"
#include "rowio.hpp"

namespace dopr {
namespace {

constexpr int kPutWaves = 8;

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

__device__ __forceinline__ double shfl_xor_f64(double x, int m) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __shfl_xor((uint32_t)u, m, 64);
  const uint32_t hi = __shfl_xor((uint32_t)(u >> 32), m, 64);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// The lane whose perm32 is r: the place of slot (or dim) r of a chunk.
__device__ __forceinline__ int lane_of(int r) {
  return ((r >> 2) & 3) * 8 + (r >> 4) * 4 + (r & 3);
}

// Codes of eight values with nearly the same scale: value e in nibble e.
__device__ __forceinline__ uint32_t fp4_codes8(const float *f, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
  return w;
}

__device__ __forceinline__ uint32_t mag(float x) {
  return __float_as_uint(x) & 0x7fffffffu;
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) {
  return a > b ? a : b;
}
// x rounded to bf16, as fp32.
__device__ __forceinline__ float as_bf16(float x) {
  return __uint_as_float(
      (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x) << 16);
}

// Bytes of LDS a wave lays its chunk out in: the chunk itself, or V^T rows of
// 32 slots (40 elements apart: 16-byte pieces on different banks).
template <int D, bool FP4>
constexpr int stage_bytes() {
  return FP4 ? fp4_chunk_bytes(D) : D * 40 * 2;
}

template <typename T, int D, bool FP4>
__global__ __launch_bounds__(64 * kPutWaves) void k_put_states(PutParams P) {
  constexpr int NJ = D / 64;
  __shared__ __attribute__((aligned(16))) char
      stage_all[kPutWaves][stage_bytes<D, FP4>()];
  __shared__ double2 turn[kChunkSlots][D / 2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 7, rg = lane >> 3;
  const int64_t i = blockIdx.x;
  const int32_t doc = P.doc_ids[i];
  const int64_t s0 = P.src_cu[i], s1 = P.src_cu[i + 1];
  if (!put_ok(P, doc, s0, s1)) {  // (the whole block)
    if (threadIdx.x == 0 && blockIdx.y == 0)
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
  const int half = P.R / 2;
  if (L == 0 && gridDim.y == 1)
    for (int g = threadIdx.x; g < hkv; g += blockDim.x) kmax[g] = 0.f;

  for (int ch = blockIdx.y; ch < n_chunks; ch += gridDim.y) {
    const int slot0 = ch * kChunkSlots;
    if (P.R > 0) {
      __syncthreads();  // (the chunk before is done with the table)
      for (int e = threadIdx.x; e < kChunkSlots * half; e += blockDim.x) {
        const int r = e / half, pair = e - r * half;
        const int slot = slot0 + r;
        if (slot >= L) break;
        const int32_t pos = P.positions ? P.positions[s0 + slot] : slot;
        double sn, cs;
        sincos((double)pos * (double)P.inv_freq[pair], &sn, &cs);
        turn[r][pair] = double2{cs * P.factor, sn * P.factor};
      }
      __syncthreads();
    }
    for (int g = wave; g < hkv; g += kPutWaves) {
      // ---- keys
      const T *kbase = static_cast<const T *>(P.k) + g * P.k_head;
      const T *kw = static_cast<const T *>(P.kw);
      uint16_t *K = FP4 ? nullptr
                        : P.sv.payload +
                              k_offset(blk, L, hkv, P.layer, g, D);
      float norm2 = 0.f;
      Raw8<T> own[4][NJ];
      const T *row[4];
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int slot = slot0 + 4 * rg + it;
        row[it] = kbase + (s0 + (slot < L ? slot : L - 1)) * P.k_row;
#pragma unroll
        for (int j = 0; j < NJ; ++j) own[it][j].load(row[it] + 64 * j + 8 * c);
      }
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int r = 4 * rg + it;
        const bool valid = slot0 + r < L;
        float f[NJ][8];
        double x[NJ][8];
#pragma unroll
        for (int j = 0; j < NJ; ++j) own[it][j].get(f[j]);
        if (P.R > 0) {
          double inv = 1.0;
          if (kw) {
            double ss = 0.0;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                ss = fma((double)f[j][e], (double)f[j][e], ss);
            ss += shfl_xor_f64(ss, 1);
            ss += shfl_xor_f64(ss, 2);
            ss += shfl_xor_f64(ss, 4);
            inv = 1.0 / sqrt(ss / D + (double)P.eps);
          }
          // x[j]: this lane's normed values of dims d0 .. d0 + 7
          auto normed = [&](const float *v, int d0, double *to) {
            if (kw) {
              Raw8<T> w;
              w.load(kw + d0);
              float wf[8];
              w.get(wf);
#pragma unroll
              for (int e = 0; e < 8; ++e) to[e] = (double)v[e] * inv * wf[e];
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) to[e] = v[e];
            }
          };
#pragma unroll
          for (int j = 0; j < NJ; ++j) normed(f[j], 64 * j + 8 * c, x[j]);
          if (P.inter) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
              for (int e = 0; e < 8; e += 2) {
                const int d = 64 * j + 8 * c + e;
                if (d >= P.R) continue;
                const double2 t = turn[r][d / 2];
                const double a = x[j][e], b = x[j][e + 1];
                x[j][e] = fma(a, t.x, -(b * t.y));
                x[j][e + 1] = fma(b, t.x, a * t.y);
              }
          } else if (D == 128 && P.R == 128) {
            // (the partner of dim i is i + 64, this lane's other run)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const double2 t = turn[r][8 * c + e];
              const double a = x[0][e], b = x[NJ - 1][e];
              x[0][e] = fma(a, t.x, -(b * t.y));
              x[NJ - 1][e] = fma(b, t.x, a * t.y);
            }
          } else {
            // the partners come from memory again
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
              const int d0 = 64 * j + 8 * c;
              if (d0 >= P.R) continue;
              if (half % 8 == 0) {
                const bool first = d0 < half;
                const int p0 = first ? d0 + half : d0 - half;
                Raw8<T> other;
                other.load(row[it] + p0);
                float of[8];
                other.get(of);
                double y[8];
                normed(of, p0, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const double2 t = turn[r][first ? d0 + e : p0 + e];
                  x[j][e] = first ? fma(x[j][e], t.x, -(y[e] * t.y))
                                  : fma(x[j][e], t.x, y[e] * t.y);
                }
              } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const int d = d0 + e;
                  if (d >= P.R) continue;
                  const bool first = d < half;
                  const int p = first ? d + half : d - half;
                  double y = to_f32<T>(row[it][p]);
                  if (kw) y = y * inv * to_f32<T>(kw[p]);
                  const double2 t = turn[r][first ? d : p];
                  x[j][e] = first ? fma(x[j][e], t.x, -(y * t.y))
                                  : fma(x[j][e], t.x, y * t.y);
                }
              }
            }
          }
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[j][e] = (float)x[j][e];
        }
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            f[j][e] = valid ? as_bf16(f[j][e]) : 0.f;
          if constexpr (FP4) {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = umax(m, mag(f[j][e]));
            m = umax(m, __shfl_xor(m, 2, 64));
            m = umax(m, __shfl_xor(m, 4, 64));
            const uint32_t b = fp4_exponent(m);
            const float scale = fp4_scale(b);
            const uint32_t w = fp4_codes8(f[j], scale);
            const int at = (c & 1) * 32 + lane_of(r);
            *reinterpret_cast<uint32_t *>(stage + 1024 * j + 16 * at +
                                          4 * (c >> 1)) = w;
            if (c < 2)
              *reinterpret_cast<uint8_t *>(stage + 32 * D + at * NJ + j) =
                  (uint8_t)b;
            // (the norm's bound is of what is held)
            const fp4_bf16x8 held = fp4_fragment(w, scale);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float h = (float)held[e];
              ss = fmaf(h, h, ss);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(f[j][e], f[j][e], ss);
            if (valid)
              store8(reinterpret_cast<bf16_t *>(K) +
                         (int64_t)(slot0 + r) * D + 64 * j + 8 * c,
                     f[j]);
          }
        }
        ss += __shfl_xor(ss, 1, 64);
        ss += __shfl_xor(ss, 2, 64);
        ss += __shfl_xor(ss, 4, 64);
        norm2 = fmaxf(norm2, ss);
      }
      norm2 = fmaxf(norm2, __shfl_xor(norm2, 8, 64));
      norm2 = fmaxf(norm2, __shfl_xor(norm2, 16, 64));
      norm2 = fmaxf(norm2, __shfl_xor(norm2, 32, 64));
      if (lane == 0) {
        // relative slack covers the fp32 rounding of the sum and the sqrt
        const float bound = sqrtf(norm2) * 1.0001f;
        if (gridDim.y == 1)  // (this lane alone writes the head's bound)
          kmax[g] = ch == 0 ? bound : fmaxf(kmax[g], bound);
        else  // (cleared by a launch in front; not negative: ordered as bits)
          atomicMax(reinterpret_cast<int *>(kmax + g), __float_as_int(bound));
      }

      // ---- values
      const T *vbase = static_cast<const T *>(P.v) + g * P.v_head;
      float v[4][NJ][8];
      {
        Raw8<T> raw[4][NJ];
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const int slot = slot0 + 4 * rg + it;
          const T *from = vbase + (s0 + (slot < L ? slot : L - 1)) * P.v_row;
#pragma unroll
          for (int j = 0; j < NJ; ++j) raw[it][j].load(from + 64 * j + 8 * c);
        }
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            raw[it][j].get(v[it][j]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              v[it][j][e] = slot0 + 4 * rg + it < L ? as_bf16(v[it][j][e])
                                                    : 0.f;
          }
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (FP4) {
            uint32_t m = umax(umax(mag(v[0][j][e]), mag(v[1][j][e])),
                              umax(mag(v[2][j][e]), mag(v[3][j][e])));
            m = umax(m, __shfl_xor(m, 8, 64));
            m = umax(m, __shfl_xor(m, 16, 64));
            m = umax(m, __shfl_xor(m, 32, 64));
            const uint32_t b = fp4_exponent(m);
            const float scale = fp4_scale(b);
            uint32_t w = 0;
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][j][e],
                                                         v[1][j][e], scale, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2][j][e],
                                                         v[3][j][e], scale, 1);
            // dim 32 db + m of the chunk's slots 4 rg ..: fragment (db, t) of
            // lane (hf, lane_of(m)), the word's half rg % 2
            const int db = 2 * j + (c >> 2);
            const int at = lane_of(8 * (c & 3) + e);
            const int fr = 2 * db + ((rg >> 1) & 1);
            *reinterpret_cast<uint16_t *>(
                stage + 16 * D + 1024 * (fr >> 2) +
                16 * ((rg >> 2) * 32 + at) + 4 * (fr & 3) + 2 * (rg & 1)) =
                (uint16_t)w;
            if (rg == 0)
              *reinterpret_cast<uint8_t *>(stage + 33 * D + at * (D / 32) +
                                           db) = (uint8_t)b;
          } else {
            uint2 pk;
            pk.x = pack2<bf16_t>(v[0][j][e], v[1][j][e]);
            pk.y = pack2<bf16_t>(v[2][j][e], v[3][j][e]);
            *reinterpret_cast<uint2 *>(
                stage + ((64 * j + 8 * c + e) * 40 + 4 * rg) * 2) = pk;
          }
        }
      wave_fence();
      if constexpr (FP4) {
        char *to = reinterpret_cast<char *>(
                       P.sv.payload +
                       fp4_offset(blk, L, hkv, P.layer, g, D)) +
                   (int64_t)ch * fp4_chunk_bytes(D);
#pragma unroll
        for (int o = 0; o < fp4_chunk_bytes(D); o += 1024)
          if (o + 16 * lane < fp4_chunk_bytes(D))
            *reinterpret_cast<fp4_u32x4 *>(to + o + 16 * lane) =
                *reinterpret_cast<const fp4_u32x4 *>(stage + o + 16 * lane);
      } else {
        uint16_t *VT =
            P.sv.payload + vt_offset(blk, L, hkv, P.layer, g, D);
        for (int d = lane >> 2; d < D; d += 16) {
          const int q = lane & 3, slot = slot0 + 8 * q;
          if (slot < Lp)  // (Lp a multiple of 8: whole pieces)
            *reinterpret_cast<fp4_u32x4 *>(VT + (int64_t)d * Lp + slot) =
                *reinterpret_cast<const fp4_u32x4 *>(stage + (d * 40 + 8 * q) *
                                                                 2);
        }
      }
      wave_fence();
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

template <typename T, int D>
void launch_put1(bool fp4, const PutParams &P, dim3 grid, hipStream_t s) {
  if (fp4)
    hipLaunchKernelGGL((k_put_states<T, D, true>), grid, dim3(64 * kPutWaves),
                       0, s, P);
  else
    hipLaunchKernelGGL((k_put_states<T, D, false>), grid,
                       dim3(64 * kPutWaves), 0, s, P);
}

template <typename T>
void launch_put(int D, bool fp4, const PutParams &P, dim3 grid,
                hipStream_t s) {
  if (D == 128)
    launch_put1<T, 128>(fp4, P, grid, s);
  else
    launch_put1<T, 64>(fp4, P, grid, s);
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
    const dim3 grid((unsigned)n,
                    stripes(n, ((int64_t)st.max_len + kChunkSlots - 1) /
                                   kChunkSlots));
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
