// qproduct.hip -- products of 8-bit integer matrices with a scale per row and
// per column:
//   y[m][n] = (sum_k x[m][k] w[n][k]) * x_scale[m] * w_scale[n]
//             (+ bias[n]) (+ residual[m][n])
// The sum is exact in 32-bit integers (depth <= 131071 keeps 128^2 * depth
// below 2^31), so it does not depend on the order or the split of the depth;
// the rest is fp32, rounded once.
//
// Matrix cores: v_mfma_i32_16x16x64_i8 with 16 rows of w as the first operand
// and 16 rows of x as the second: lane l holds 16 consecutive bytes (depth
// 16 * (l / 16) ..) of row l % 16 of each, and of the result column l % 16 (a
// row of x) at rows 4 * (l / 16) .. + 3 (of w).  A wave's 64 rows of w are
// dealt to its four operands so that a lane's 16 results of one x row are 16
// consecutive columns of y: operand f, row i is w row
// 16 * (i / 4) + 4 * f + i % 4.
#include <type_traits>

#include "rowio.hpp"

namespace dopr {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct ProductParams {
  const int8_t *x, *w;
  const float *x_scale, *w_scale;
  const void *bias, *res;
  void *y;
  int64_t M, N, K, ldx, ldw, ldr, ldy;
};

// w row (of 64) behind LDS row p
__device__ __forceinline__ int w_row(int p) {
  return (p & ~63) + ((p & 15) >> 2) * 16 + ((p >> 4) & 3) * 4 + (p & 3);
}

// 16 results of y row m from column n on: scales, bias, residual, store.
template <typename T>
__device__ __forceinline__ void store16(const ProductParams &P, int64_t m,
                                        int64_t n, const float *acc) {
  if (m >= P.M || n >= P.N) return;
  const float xs = P.x_scale[m];
  const T *bias = static_cast<const T *>(P.bias);
  const T *res = static_cast<const T *>(P.res) + m * P.ldr;
  T *y = static_cast<T *>(P.y) + m * P.ldy;
  float v[16];
  if (n + 16 <= P.N) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float s[8], b[8];
      Raw8<float> rs;
      Raw8<T> rb;
      rs.load(P.w_scale + n + 8 * h);
      rs.get(s);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[8 * h + e] = acc[8 * h + e] * xs * s[e];
      if (P.bias) {
        rb.load(bias + n + 8 * h);
        rb.get(b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * h + e] += b[e];
      }
      if (P.res) {
        rb.load(res + n + 8 * h);
        rb.get(b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * h + e] += b[e];
      }
    }
    store8<T>(y + n, 0, v);
    store8<T>(y + n + 8, 0, v + 8);
    return;
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (n + e >= P.N) break;
    float f = acc[e] * xs * P.w_scale[n + e];
    if (P.bias) f += to_f32<T>(bias[n + e]);
    if (P.res) f += to_f32<T>(res[n + e]);
    y[n + e] = from_f32<T>(f);
  }
}

// ---------------------------------------------------------------------------
// Any strides and alignment: 128 x 128 tiles, 4 waves of 64 x 64, depth in
// steps of 64 bytes through registers into two LDS buffers.

constexpr int kAnyTile = 128;
constexpr int kAnyStep = 64;

// 16 bytes of a row from depth k, zeros from K on
__device__ __forceinline__ u32x4 row_bytes(const int8_t *p, int64_t k,
                                           int64_t K) {
  if (k + 16 <= K) return *reinterpret_cast<const u32x4_any *>(p + k);
  u32x4 u = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (k + e < K) u[e >> 2] |= (uint32_t)(uint8_t)p[k + e] << (8 * (e & 3));
  return u;
}

// LDS address (16-byte units) of chunk c of 64-byte row r: 16 rows' equal
// chunks fall on all 64 banks
__device__ __forceinline__ int any_slot(int r, int c) {
  return r * 4 + (c ^ ((r >> 2) & 3));
}

template <typename T>
__global__ __launch_bounds__(256) void k_product_any(ProductParams P,
                                                     int64_t tiles_n) {
  __shared__ u32x4 lds[2][2][kAnyTile * 4];  // [buffer][x, w]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t bm = blockIdx.x / tiles_n, bn = blockIdx.x - bm * tiles_n;
  const int64_t m0 = bm * kAnyTile, n0 = bn * kAnyTile;
  const int8_t *xp[2], *wp[2];
  int slot[2], kc[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int id = tid + 256 * i, r = id >> 2;
    kc[i] = (id & 3) * 16;
    slot[i] = any_slot(r, id & 3);
    // rows behind the end repeat the last one; their results are not stored
    xp[i] = P.x + min(m0 + r, P.M - 1) * P.ldx;
    wp[i] = P.w + min(n0 + w_row(r), P.N - 1) * P.ldw;
  }
  u32x4 xr[2], wr[2];
  auto fetch = [&](int64_t k0) {
    if (k0 + kAnyStep <= P.K) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        xr[i] = *reinterpret_cast<const u32x4_any *>(xp[i] + k0 + kc[i]);
        wr[i] = *reinterpret_cast<const u32x4_any *>(wp[i] + k0 + kc[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        xr[i] = row_bytes(xp[i], k0 + kc[i], P.K);
        wr[i] = row_bytes(wp[i], k0 + kc[i], P.K);
      }
    }
  };
  auto put = [&](int b) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lds[b][0][slot[i]] = xr[i];
      lds[b][1][slot[i]] = wr[i];
    }
  };
  i32x4 acc[4][4] = {};  // [x operand][w operand]
  const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  const int64_t steps = (P.K + kAnyStep - 1) / kAnyStep;
  if (steps > 0) {
    fetch(0);
    put(0);
  }
  __syncthreads();
  for (int64_t s = 0; s < steps; ++s) {
    const int b = (int)(s & 1);
    if (s + 1 < steps) fetch((s + 1) * kAnyStep);
    i32x4 xf[4], wf[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      xf[f] = __builtin_bit_cast(
          i32x4, lds[b][0][any_slot(wm + 16 * f + (lane & 15), lane >> 4)]);
      wf[f] = __builtin_bit_cast(
          i32x4, lds[b][1][any_slot(wn + 16 * f + (lane & 15), lane >> 4)]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[j], xf[i],
                                                          acc[i][j], 0, 0, 0);
    if (s + 1 < steps) put(b ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[16];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] = (float)acc[i][j][e];
    store16<T>(P, m0 + wm + 16 * i + (lane & 15),
               n0 + wn + 16 * (lane >> 4), v);
  }
}

// ---------------------------------------------------------------------------
// Rows on 16-byte addresses: WGM x WGN waves of 16 FM x 64, the depth in steps
// of 64 bytes that go straight from memory to LDS, kStages steps deep.
//
// Step t's operands are read from LDS to registers during step t - 1's
// products, so at a barrier every wave is done with the LDS buffer of the
// step it starts to multiply, and the loads of step t + kStages go there: a
// load has kStages - 1 steps to arrive.

constexpr int kStep = 64;
constexpr int kStages = 4;
constexpr int kGroupM = 8;  // tile rows that share w tiles while in L2

// 64 lanes' 16 bytes each from base + off to LDS, in lane order from m0 on.
// (The compiler does not know of the LDS write: stage_wait orders it.)
__device__ __forceinline__ void dma16(uint32_t lds, const void *base,
                                      uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\t"
               "global_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(base)
               : "m0");
}

// At most `left` of this wave's loads are on their way, its LDS reads have
// returned, and every wave is here.
template <int left>
__device__ __forceinline__ void stage_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(left)
               : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3)))
                                   void *)p;
}

// Tile of block b: the blocks of one XCD (b % 8) take consecutive tiles, in
// groups of kGroupM tile rows, so the 32 that run together cover 8 x 4 tiles.
__device__ __forceinline__ void tile_of(int64_t b, int64_t tm, int64_t tn,
                                        int64_t &m, int64_t &n) {
  const int64_t all = tm * tn, per = all / 8, rem = all % 8, xcd = b % 8;
  const int64_t t = xcd * per + (xcd < rem ? xcd : rem) + b / 8;
  const int64_t g = t / (kGroupM * tn);
  const int64_t rows = min((int64_t)kGroupM, tm - g * kGroupM);
  const int64_t in = t - g * kGroupM * tn;
  m = g * kGroupM + in % rows;
  n = in / rows;
}

template <typename T, int FM, int WGM, int WGN>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void k_product(
    ProductParams P, int64_t tm, int64_t tn) {
  constexpr int kBM = 16 * FM * WGM, kBN = 64 * WGN;
  // a wave's loads of a step: 16 rows of 64 bytes each
  constexpr int kXLoads = FM / WGN, kWLoads = 4 / WGM;
  constexpr int kLoads = kXLoads + kWLoads;
  static_assert(kXLoads * WGN == FM && kWLoads * WGM == 4, "even shares");
  constexpr int kStageBytes = (kBM + kBN) * kStep;
  extern __shared__ u32x4 lds[];  // [kStages][x rows | w rows]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t bm, bn;
  tile_of(blockIdx.x, tm, tn, bm, bn);
  const int64_t m0 = bm * kBM, n0 = bn * kBN;
  // rows behind the end repeat the last one; their results are not stored
  const int last_m = (int)min(P.M - 1 - m0, (int64_t)kBM - 1);
  const int last_n = (int)min(P.N - 1 - n0, (int64_t)kBN - 1);
  const int8_t *xbase = P.x + m0 * P.ldx, *wbase = P.w + n0 * P.ldw;
  const int full = (int)(P.K / kStep);

  // LDS row r of a part holds its 16-byte chunk c at slot any_slot(r, c); the
  // lanes of a load fill 64 slots in order
  auto x_row = [&](int i) { return (wave * kXLoads + i) * 16 + (lane >> 2); };
  auto w_lds_row = [&](int i) {
    return (wave * kWLoads + i) * 16 + (lane >> 2);
  };
  const int chunk = ((lane & 3) ^ ((lane >> 4) & 3)) * 16;
  uint32_t xoff[kXLoads], woff[kWLoads];
#pragma unroll
  for (int i = 0; i < kXLoads; ++i)
    xoff[i] = (uint32_t)min(x_row(i), last_m) * (uint32_t)P.ldx + chunk;
#pragma unroll
  for (int i = 0; i < kWLoads; ++i)
    woff[i] =
        (uint32_t)min(w_row(w_lds_row(i)), last_n) * (uint32_t)P.ldw + chunk;
  const uint32_t xdst = lds_address(lds) + wave * kXLoads * 1024;
  const uint32_t wdst =
      lds_address(lds) + kBM * kStep + wave * kWLoads * 1024;
  auto issue = [&](int s) {
    const uint32_t b = (s % kStages) * kStageBytes;
#pragma unroll
    for (int i = 0; i < kXLoads; ++i)
      dma16(xdst + b + i * 1024, xbase + (int64_t)s * kStep, xoff[i]);
#pragma unroll
    for (int i = 0; i < kWLoads; ++i)
      dma16(wdst + b + i * 1024, wbase + (int64_t)s * kStep, woff[i]);
  };

  const int wm = (wave / WGN) * (16 * FM), wn = (wave % WGN) * 64;
  const int slot = any_slot(lane & 15, lane >> 4);
  const int xslot = wm * 4 + slot, wslot = (kBM + wn) * 4 + slot;
  i32x4 acc[FM][4] = {};
  auto read = [&](int s, i32x4 *x, i32x4 *w) {
    const u32x4 *p = lds + (s % kStages) * (kStageBytes / 16);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = __builtin_bit_cast(i32x4, p[wslot + j * 64]);
#pragma unroll
    for (int i = 0; i < FM; ++i)
      x[i] = __builtin_bit_cast(i32x4, p[xslot + i * 64]);
  };
  auto multiply = [&](const i32x4 *x, const i32x4 *w) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[i],
                                                          acc[i][j], 0, 0, 0);
  };

#pragma unroll 1
  for (int s = 0; s < kStages - 1 && s < full; ++s) issue(s);
  i32x4 xa[FM], wa[4], xb[FM], wb[4];
  if (P.K % kStep) {
    // the partial step comes first, through the last buffer, while the first
    // loads are on their way: zeros from the depth on
    u32x4 *p = lds + (kStages - 1) * (kStageBytes / 16) + lane;
    const int64_t k = (int64_t)full * kStep + chunk;
#pragma unroll 1
    for (int i = 0; i < kXLoads; ++i)
      p[(wave * kXLoads + i) * 64] = row_bytes(
          xbase + (int64_t)min(x_row(i), last_m) * P.ldx, k, P.K);
#pragma unroll 1
    for (int i = 0; i < kWLoads; ++i)
      p[kBM * 4 + (wave * kWLoads + i) * 64] =
          row_bytes(wbase + (int64_t)min(w_row(w_lds_row(i)), last_n) * P.ldw,
                    k, P.K);
    __syncthreads();
    read(kStages - 1, xa, wa);
    multiply(xa, wa);
    __syncthreads();
  }
  if (full > 0) {
    if (full >= kStages) issue(kStages - 1);
    stage_wait<0>();
    read(0, xa, wa);
    // products of step s, held in (x, w), while step s + 1 is read into
    // (y, v); behind the last step that is a stale buffer, never used
    int s = 0;
    auto step = [&](const i32x4 *x, const i32x4 *w, i32x4 *y, i32x4 *v) {
      stage_wait<(kStages - 2) * kLoads>();
      issue(s + kStages);
      read(s + 1, y, v);
      multiply(x, w);
      ++s;
    };
    while (s + kStages + 1 < full) {
      step(xa, wa, xb, wb);
      step(xb, wb, xa, wa);
    }
#pragma unroll 1
    for (; s < full; ++s) {
      stage_wait<0>();
      if (s + kStages < full) issue(s + kStages);
      read(s + 1, xb, wb);
      multiply(xa, wa);
#pragma unroll
      for (int i = 0; i < FM; ++i) xa[i] = xb[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) wa[j] = wb[j];
    }
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    float v[16];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] = (float)acc[i][j][e];
    store16<T>(P, m0 + wm + 16 * i + (lane & 15), n0 + wn + 16 * (lane >> 4),
               v);
  }
}

template <typename T, int FM, int WGM, int WGN>
hipError_t product_tiles(const ProductParams &P, hipStream_t s) {
  constexpr int kBM = 16 * FM * WGM, kBN = 64 * WGN;
  const int64_t tm = (P.M + kBM - 1) / kBM, tn = (P.N + kBN - 1) / kBN;
  const size_t lds = (size_t)kStages * (kBM + kBN) * kStep;
  const auto kernel = &k_product<T, FM, WGM, WGN>;
  // (the runtime's own limit is 64 KB until a kernel asks for more)
  static const hipError_t allowed = hipFuncSetAttribute(
      reinterpret_cast<const void *>(kernel),
      hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (allowed != hipSuccess) return allowed;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(tm * tn)),
                     dim3(64 * WGM * WGN), lds, s, P, tm, tn);
  return hipGetLastError();
}

// x, w and their strides on 16 bytes, and a tile's rows within 32-bit offsets
bool aligned_rows(const ProductParams &P) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(P.x) |
                      reinterpret_cast<uintptr_t>(P.w) | (uintptr_t)P.ldx |
                      (uintptr_t)P.ldw;
  return a % 16 == 0 && P.ldx < (1 << 22) && P.ldw < (1 << 22);
}

template <typename T>
hipError_t product(const ProductParams &P, hipStream_t s) {
  if (aligned_rows(P)) {
    if (P.M > 512) return product_tiles<T, 8, 2, 4>(P, s);
    return product_tiles<T, 4, 2, 2>(P, s);
  }
  const int64_t tm = (P.M + kAnyTile - 1) / kAnyTile,
                tn = (P.N + kAnyTile - 1) / kAnyTile;
  hipLaunchKernelGGL((k_product_any<T>), dim3((unsigned)(tm * tn)), dim3(256),
                     0, s, P, tn);
  return hipGetLastError();
}

}  // namespace

size_t product_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_product(const dopr_quant_matmul_args_t &a, hipStream_t s) {
  const ProductParams P{a.x,    a.w,      a.x_scale,      a.w_scale,
                        a.bias, a.residual, a.y,          a.rows,
                        a.cols, a.depth,  a.x_row_stride, a.w_row_stride,
                        a.residual_row_stride, a.y_row_stride};
  if (a.dtype == DOPR_BF16) return product<bf16_t>(P, s);
  if (a.dtype == DOPR_F16) return product<_Float16>(P, s);
  return product<float>(P, s);
}

}  // namespace dopr
