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

// 16 bytes of a row from depth k, zeros from K on.  Nothing behind the row is
// read: the row's last 16 bytes, shifted down.
__device__ __forceinline__ u32x4 row_bytes(const int8_t *p, int64_t k,
                                           int64_t K) {
  if (K < 16) {  // (k = 0 or past the end)
    u32x4 u = {0u, 0u, 0u, 0u};
#pragma unroll 1
    for (int e = (int)(K - k) - 1; e >= 0; --e) {
      u.w = u.w << 8 | u.z >> 24;
      u.z = u.z << 8 | u.y >> 24;
      u.y = u.y << 8 | u.x >> 24;
      u.x = u.x << 8 | (uint8_t)p[k + e];
    }
    return u;
  }
  const int64_t at = min(k, K - 16);
  u32x4 u = *reinterpret_cast<const u32x4_any *>(p + at);
  const uint32_t s = (uint32_t)min(k - at, (int64_t)16);
  if (s & 16) u = u32x4{0u, 0u, 0u, 0u};
  if (s & 8) u = u32x4{u.z, u.w, 0u, 0u};
  if (s & 4) u = u32x4{u.y, u.z, u.w, 0u};
  const uint32_t b = s & 3;
  return u32x4{__builtin_amdgcn_alignbyte(u.y, u.x, b),
               __builtin_amdgcn_alignbyte(u.z, u.y, b),
               __builtin_amdgcn_alignbyte(u.w, u.z, b),
               __builtin_amdgcn_alignbyte(0u, u.w, b)};
}

// ---------------------------------------------------------------------------
// Any strides and alignment: 128 x 128 tiles, 4 waves of 64 x 64, depth in
// steps of 64 bytes through registers into two LDS buffers.

constexpr int kAnyTile = 128;
constexpr int kAnyStep = 64;

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

// ---------------------------------------------------------------------------
// Few rows: a block's WK waves share one strip of 16 FN w rows and split the
// depth, in batches of U steps of 64 bytes, each wave's operands coming
// straight from memory to its registers, one batch ahead of the products.
// The waves' sums meet in LDS (integers: the split does not show).

// 4 results of y row m from column n on.
template <typename T>
__device__ __forceinline__ void store4(const ProductParams &P, int64_t m,
                                       int64_t n, const i32x4 &acc) {
  if (m >= P.M || n >= P.N) return;
  const float xs = P.x_scale[m];
  const T *bias = static_cast<const T *>(P.bias);
  const T *res = static_cast<const T *>(P.res) + m * P.ldr;
  T *y = static_cast<T *>(P.y) + m * P.ldy;
  const int left = (int)min(P.N - n, (int64_t)4);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t c = n + min(e, left - 1);
    v[e] = (float)acc[e] * xs * P.w_scale[c];
    if (P.bias) v[e] += to_f32<T>(bias[c]);
    if (P.res) v[e] += to_f32<T>(res[c]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) y[n + e] = from_f32<T>(v[e]);
}

template <typename T, int FM, int FN, int U, int WK>
__global__ __launch_bounds__(64 * WK) void k_product_few(ProductParams P) {
  __shared__ i32x4 sums[WK][FM * FN][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * (16 * FN);
  const int64_t m0 = (int64_t)blockIdx.y * (16 * FM);
  const int kc = (lane >> 4) * 16;
  // rows behind the end repeat the last one; their results are not stored
  const int8_t *xp[FM], *wp[FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
    xp[i] = P.x + min(m0 + 16 * i + (lane & 15), P.M - 1) * P.ldx + kc;
#pragma unroll
  for (int j = 0; j < FN; ++j)
    wp[j] = P.w + min(n0 + 16 * j + (lane & 15), P.N - 1) * P.ldw + kc;
  constexpr int kBatch = U * kStep;
  i32x4 acc[FM][FN] = {};
  struct Batch {
    u32x4 x[U][FM], w[U][FN];
  };
  auto fetch = [&](int64_t batch, Batch &b) {
    const int64_t k = batch * kBatch;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
        b.w[u][j] =
            *reinterpret_cast<const u32x4_any *>(wp[j] + k + u * kStep);
#pragma unroll
      for (int i = 0; i < FM; ++i)
        b.x[u][i] =
            *reinterpret_cast<const u32x4_any *>(xp[i] + k + u * kStep);
    }
  };
  auto product1 = [&](const u32x4 *x, const u32x4 *w) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
            __builtin_bit_cast(i32x4, w[j]), __builtin_bit_cast(i32x4, x[i]),
            acc[i][j], 0, 0, 0);
  };
  auto multiply = [&](const Batch &b) {
#pragma unroll
    for (int u = 0; u < U; ++u) product1(b.x[u], b.w[u]);
  };
  const int batches = (int)(P.K / kBatch);
  Batch a, b;
  if (wave < batches) fetch(wave, a);
  for (int i = wave; i < batches; i += 2 * WK) {
    if (i + WK < batches) fetch(i + WK, b);
    multiply(a);
    if (i + WK >= batches) break;
    if (i + 2 * WK < batches) fetch(i + 2 * WK, a);
    multiply(b);
  }
  // steps behind the last whole batch, one at a time, first to the waves that
  // had a batch less
  const int first = batches * U;
#pragma unroll 1
  for (int s = first + (wave + WK - batches % WK) % WK;
       (int64_t)s * kStep < P.K; s += WK) {
    u32x4 x[FM], w[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j)
      w[j] = row_bytes(wp[j] - kc, (int64_t)s * kStep + kc, P.K);
#pragma unroll
    for (int i = 0; i < FM; ++i)
      x[i] = row_bytes(xp[i] - kc, (int64_t)s * kStep + kc, P.K);
    product1(x, w);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) sums[wave][i * FN + j][lane] = acc[i][j];
  __syncthreads();
  for (int f = wave; f < FM * FN; f += WK) {
    i32x4 s = sums[0][f][lane];
#pragma unroll
    for (int w = 1; w < WK; ++w) s += sums[w][f][lane];
    store4<T>(P, m0 + 16 * (f / FN) + (lane & 15),
              n0 + 16 * (f % FN) + 4 * (lane >> 4), s);
  }
}

template <typename T, int FM, int FN, int U, int WK>
hipError_t product_few(const ProductParams &P, hipStream_t s) {
  const unsigned strips = (unsigned)((P.N + 16 * FN - 1) / (16 * FN));
  const unsigned rows = (unsigned)((P.M + 16 * FM - 1) / (16 * FM));
  hipLaunchKernelGGL((k_product_few<T, FM, FN, U, WK>), dim3(strips, rows),
                     dim3(64 * WK), 0, s, P);
  return hipGetLastError();
}

// Depth split over 4, 8 or 16 waves: until some 16 waves a CU have work, as
// long as a wave keeps a batch.
template <typename T, int FM, int FN, int U>
hipError_t product_few(const ProductParams &P, hipStream_t s) {
  const int64_t strips = (P.N + 16 * FN - 1) / (16 * FN);
  const int64_t batches = P.K / (U * kStep);
  if constexpr (FM < 4)  // (four x operands of 16 waves would spill)
    if (strips * 8 < 4096 && batches > 8)
      return product_few<T, FM, FN, U, 16>(P, s);
  if (strips * 4 < 4096 && batches > 4)
    return product_few<T, FM, FN, U, 8>(P, s);
  return product_few<T, FM, FN, U, 4>(P, s);
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
  if (P.M <= 16) return product_few<T, 1, 1, 4>(P, s);
  if (P.M <= 32) return product_few<T, 2, 1, 4>(P, s);
  if (P.M <= 64) return product_few<T, 4, 2, 2>(P, s);
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
