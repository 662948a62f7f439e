// qproduct.hip -- products of 8-bit integer matrices with a scale per row and
// per column:
//   y[m][n] = (sum_k x[m][k] w[n][k]) * x_scale[m] * w_scale[n]
//             (+ bias[n]) (+ residual[m][n])
// The sum is exact in 32-bit integers (depth <= 131071 keeps 128^2 * depth
// below 2^31), so it does not depend on the order or the split of the depth.
// The rest is fp32: the sum's conversion (exact up to 2^24), the two scales, bias
// and residual in this order, each rounded to fp32 (five roundings, 5 * 2^-24 of
// the magnitudes that are added), then the output's own rounding.
//
// Matrix cores: v_mfma_i32_16x16x64_i8 with 16 rows of w as the first operand
// and 16 rows of x as the second: lane l holds 16 consecutive bytes (depth
// 16 * (l / 16) ..) of row l % 16 of each, and of the result column l % 16 (a
// row of x) at rows 4 * (l / 16) .. + 3 (of w).  A wave's 64 rows of w are
// dealt to its four operands so that the four lanes that hold an x row store 64
// whole bytes of it at a time: with outputs of 16 bits a lane's 16 results of
// one x row are two runs of 8 consecutive columns of y, 32 apart (operand f,
// row i is w row 32 * (f / 2) + 8 * (i / 4) + 4 * (f % 2) + i % 4), with fp32
// four runs of 4, 16 apart (w row 16 f + i).
#include <atomic>
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
  // y's rows lie on 64 bytes: four lanes' stores fill a piece of memory, so they
  // go past the caches' order of use.  Off them, two waves' stores meet in a
  // piece, in L2 (10,014 x 14,985 x 3968 to bf16 609 -> 537 us).
  bool stream;
};

// The runs of columns of y that a lane's 16 results make up in an x row.
template <typename T>
struct Runs {
  static constexpr int kLength = 16 / (int)sizeof(T);  // 16 bytes
  static constexpr int kApart = 4 * kLength;           // of four lanes: 64
  static constexpr int kCount = 16 / kLength;
  // a run's first column in the first run's place, among a wave's 64
  static __device__ __forceinline__ int column(int lane) {
    return (lane >> 4) * kLength;
  }
  // result e's column behind it
  static __device__ __forceinline__ constexpr int of(int e) {
    return kApart * (e / kLength) + e % kLength;
  }
  // w row (of 64) behind LDS row p
  static __device__ __forceinline__ int w_row(int p) {
    if constexpr (kLength == 4)
      return p;
    else
      return (p & ~31) + ((p >> 2) & 3) * 8 + ((p >> 4) & 1) * 4 + (p & 3);
  }
};

// Finishes a lane's part of a tile: its runs of columns of y, the first from n
// on, in the FM rows m, m + 16, .. with own(i).  sums(i, v) gives row i's
// integer sums, column_scales(scale) and row_scale(i) the scales.
template <typename T, int FM, bool STREAM, typename Columns, typename Row,
          typename Sums, typename Own>
__device__ __forceinline__ void finish_rows(const ProductParams &P, int m,
                                            int n, Columns &&column_scales,
                                            Row &&row_scale, Sums &&sums,
                                            Own &&own) {
  const int left = (int)P.N - n;
  if (left <= 0) return;
  float scale[16];
  column_scales(scale);
  const T *bias = static_cast<const T *>(P.bias) + n;
  const T *res = static_cast<const T *>(P.res) + m * P.ldr + n;
  T *y = static_cast<T *>(P.y) + m * P.ldy + n;
  using R = Runs<T>;
  constexpr int L = R::kLength;
  const bool whole = left > R::of(15);
  Raw<T, L> add[R::kCount];
  if (P.bias && whole)
#pragma unroll
    for (int h = 0; h < R::kCount; ++h) add[h].load(bias + R::kApart * h);
  float plus[16] = {};
  if (P.bias && whole)
#pragma unroll
    for (int h = 0; h < R::kCount; ++h) add[h].get(plus + L * h);
  // a row's residual is asked for ahead of the stores of the row before it,
  // which it would otherwise wait for (loads and stores complete in order)
  auto ask = [&](int i) {
    if (P.res && whole && own(i) && m + 16 * i < (int)P.M)
#pragma unroll
      for (int h = 0; h < R::kCount; ++h)
        add[h].load(res + 16 * i * P.ldr + R::kApart * h);
  };
  ask(0);
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const bool mine = own(i) && m + 16 * i < (int)P.M;
    float v[16];
    if (mine) {
      const float xs = row_scale(i);
      sums(i, v);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = v[e] * xs * scale[e];
      if (P.bias)
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] += plus[e];
      if (P.res && whole) {
        float f[16];
#pragma unroll
        for (int h = 0; h < R::kCount; ++h) add[h].get(f + L * h);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] += f[e];
      }
    }
    if (i + 1 < FM) ask(i + 1);
    if (mine) {
      if (whole) {
#pragma unroll
        for (int h = 0; h < R::kCount; ++h) {
          T *to = y + R::kApart * h;
          store_part<T, L, STREAM>(to, 0, L, v + L * h);
        }
      } else {  // the matrix ends inside: one by one
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int c = R::of(e);
          if (c < left) {
            if (P.bias) v[e] += to_f32<T>(bias[c]);
            if (P.res) v[e] += to_f32<T>(res[16 * i * P.ldr + c]);
            y[c] = from_f32<T>(v[e]);
          }
        }
      }
    }
    y += 16 * P.ldy;
    __builtin_amdgcn_sched_barrier(0);  // (one row's values at a time)
  }
}

template <typename T, int FM, typename Columns, typename Row, typename Sums,
          typename Own>
__device__ __forceinline__ void finish(const ProductParams &P, int m, int n,
                                       Columns &&column_scales,
                                       Row &&row_scale, Sums &&sums,
                                       Own &&own) {
  // (apart: one loop with both kinds of store was slower than either)
  if (P.stream)
    finish_rows<T, FM, true>(P, m, n, column_scales, row_scale, sums, own);
  else
    finish_rows<T, FM, false>(P, m, n, column_scales, row_scale, sums, own);
}

// The scales of finish from memory.
template <typename T>
__device__ __forceinline__ void columns_from_memory(const ProductParams &P,
                                                    int n, float *scale) {
#pragma unroll
  for (int e = 0; e < 16; ++e)
    scale[e] = P.w_scale[min(n + Runs<T>::of(e), (int)P.N - 1)];
}

// 16 bytes of a row from depth k, zeros from K on.  Nothing behind the row is
// read: the row's last 16 bytes, shifted down.
__device__ __forceinline__ u32x4 row_bytes(const int8_t *p, int64_t k,
                                           int64_t K) {
  u32x4 u = {0u, 0u, 0u, 0u};
  uint32_t s;
  if (K < 16) {  // a row of less: byte by byte
    s = (uint32_t)k;
#pragma unroll 1
    for (int e = (int)K - 1; e >= 0; --e)
      u = u32x4{u.x << 8 | (uint8_t)p[e], u.y << 8 | u.x >> 24,
                u.z << 8 | u.y >> 24, u.w << 8 | u.z >> 24};
  } else {
    const int64_t at = min(k, K - 16);
    u = *reinterpret_cast<const u32x4_any *>(p + at);
    s = (uint32_t)min(k - at, (int64_t)16);
  }
  if (s > 16) s = 16;
  if (s & 16) u = u32x4{0u, 0u, 0u, 0u};
  if (s & 8) u = u32x4{u.z, u.w, 0u, 0u};
  if (s & 4) u = u32x4{u.y, u.z, u.w, 0u};
  const uint32_t b = s & 3;
  return u32x4{__builtin_amdgcn_alignbyte(u.y, u.x, b),
               __builtin_amdgcn_alignbyte(u.z, u.y, b),
               __builtin_amdgcn_alignbyte(u.w, u.z, b),
               __builtin_amdgcn_alignbyte(0u, u.w, b)};
}

// The depth goes in spans of 128 bytes, two matrix steps of 64, through LDS
// rows of 128 bytes.
constexpr int kCUs = 256;
constexpr int kStep = 64;
constexpr int kSpan = 128;

// LDS slot (16-byte units) of chunk c of row r: 16 rows' equal chunks fall on
// all 64 banks.
__device__ __forceinline__ int span_slot(int r, int c) {
  return r * 8 + (c ^ ((r >> 1) & 7));
}

// ---------------------------------------------------------------------------
// Any strides and alignment: 64 x 128 tiles of 4 waves (32 x 64 each), a span
// ahead in registers, two in LDS; three blocks a CU hide one another's loads.

constexpr int kAnyM = 64, kAnyN = 128;

template <typename T>
__global__ __launch_bounds__(256, 3) void k_product_any(ProductParams P,
                                                        int tiles_n) {
  constexpr int kLoads = (kAnyM + kAnyN) * 8 / 256;
  __shared__ u32x4 lds[2][(kAnyM + kAnyN) * 8];  // [x rows | w rows]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int bm = blockIdx.x / tiles_n, bn = blockIdx.x - bm * tiles_n;
  const int m0 = bm * kAnyM, n0 = bn * kAnyN;
  const int chunk = (tid & 7) * 16;
  const int8_t *at[kLoads];
  int slot[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = i * 32 + (tid >> 3);
    // rows behind the end repeat the last one; their results are not stored
    at[i] = r < kAnyM
                ? P.x + (int64_t)min(m0 + r, (int)P.M - 1) * P.ldx
                : P.w + (int64_t)min(n0 + Runs<T>::w_row(r - kAnyM),
                                     (int)P.N - 1) * P.ldw;
    slot[i] = span_slot(r, tid & 7);
  }
  u32x4 next[kLoads];
  auto fetch = [&](int64_t k0) {
    if (k0 + kSpan <= P.K) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        next[i] = *reinterpret_cast<const u32x4_any *>(at[i] + k0 + chunk);
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        next[i] = row_bytes(at[i], k0 + chunk, P.K);
    }
  };
  i32x4 acc[2][4] = {};  // [x operand][w operand]
  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 64;
  const int spans = (int)((P.K + kSpan - 1) / kSpan);
  if (spans > 0) fetch(0);
  for (int s = 0; s < spans; ++s) {
    u32x4 *buf = lds[s & 1];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) buf[slot[i]] = next[i];
    if (s + 1 < spans) fetch((int64_t)(s + 1) * kSpan);
    // (one barrier a span: the buffer written next was read a span ago)
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i32x4 xf[2], wf[4];
      const int c = 4 * h + (lane >> 4);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        wf[j] = __builtin_bit_cast(
            i32x4, buf[span_slot(kAnyM + wn + 16 * j + (lane & 15), c)]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        xf[i] = __builtin_bit_cast(
            i32x4, buf[span_slot(wm + 16 * i + (lane & 15), c)]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              wf[j], xf[i], acc[i][j], 0, 0, 0);
    }
  }
  const int m = m0 + wm + (lane & 15), n = n0 + wn + Runs<T>::column(lane);
  finish<T, 2>(
      P, m, n,
      [&](float *scale) { columns_from_memory<T>(P, n, scale); },
      [&](int i) { return P.x_scale[m + 16 * i]; },
      [&](int i, float *v) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = (float)acc[i][e >> 2][e & 3];
      },
      [](int) { return true; });
}

// P's rows m .. m + n - 1.
template <typename T>
ProductParams rows_of(const ProductParams &P, int64_t m, int64_t n) {
  ProductParams S = P;
  S.M = n;
  S.x = ahead(P.x, m * P.ldx);
  S.x_scale = P.x_scale + m;
  S.res = ahead(P.res, m * P.ldr * (int)sizeof(T));
  S.y = ahead(P.y, m * P.ldy * (int)sizeof(T));
  return S;
}

template <typename T>
hipError_t product_any(const ProductParams &P, hipStream_t s) {
  const int64_t tn = (P.N + kAnyN - 1) / kAnyN;
  const int64_t most = std::max<int64_t>(a_launch(256) / tn, 1) * kAnyM;
  return in_slices(P.M, most, [&](int64_t m, int64_t n) {
    const int64_t tm = (n + kAnyM - 1) / kAnyM;
    hipLaunchKernelGGL((k_product_any<T>), dim3((unsigned)(tm * tn)),
                       dim3(256), 0, s, rows_of<T>(P, m, n), (int)tn);
    return hipGetLastError();
  });
}

// ---------------------------------------------------------------------------
// Rows on 16-byte addresses: WK groups of WGM x WGN waves of 16 FM x 64.  The
// depth goes in spans of 128 bytes, a whole cache line of every row, straight
// from memory to LDS, ST spans deep (halves of a line would be fetched twice:
// a tile's lines outlast the L1 cache).  Group g takes the spans g, g + WK,
// ...; the groups' sums meet in LDS.
//
// A span is multiplied in two steps of 64 bytes, each step's operands read
// from LDS to registers during the step before.  So halfway through a span
// every wave is done with its LDS buffer: the one barrier of a span stands
// there, and the loads of ST spans later follow it.

// Measured: 12,900 x 24576 x 4096 1040 us, 2.5 POP/s, the matrix cores busy for
// 63 % of the cycles and the rest of the time behind the next span's loads (two
// spans fill the LDS); 129 x 24576 x 4096 28 us on 192 of the CUs, with neither
// HBM (3.8 TB/s) nor the matrix cores (busy for a quarter of the cycles) at its
// rate.  L2, through which every tile reads all of x beside its part of w, hands
// out 219 MB, 7.8 TB/s, half of it hits; what bounds that size is open.

constexpr int kGroupM = 8;  // tile rows that share w tiles while in L2

// 64 lanes' 16 bytes each from base + off to LDS, in lane order from m0 on.
// (The compiler does not know of the LDS write: stage_wait orders it.)
__device__ __forceinline__ void dma16(uint32_t lds, const int8_t *at,
                                      uint32_t off) {
  // (wave-uniform, but not always in scalar registers)
  const uint64_t a = (uint64_t)at;
  const uint64_t base =
      (uint64_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32 |
      (uint32_t)__builtin_amdgcn_readfirstlane((int)a);
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\t"
               "global_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(base)
               : "m0");
}

// 64 lanes' 4 bytes each, in the same way.
__device__ __forceinline__ void dma4(uint32_t lds, const float *at) {
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\t"
               "global_load_lds_dword %1, off"
               :: "s"(lds), "v"(at)
               : "m0");
}

// At most `left` of this wave's loads and stores are on their way (they
// complete in order), its LDS reads have returned, and every wave is here.
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
__device__ __forceinline__ void tile_of(int b, int tm, int tn, int &m,
                                        int &n) {
  const int all = tm * tn, per = all / 8, rem = all % 8, xcd = b % 8;
  const int t = xcd * per + min(xcd, rem) + b / 8;
  const int g = t / (kGroupM * tn);
  const int rows = min(kGroupM, tm - g * kGroupM);
  const int in = t - g * kGroupM * tn;
  m = g * kGroupM + in % rows;
  n = in / rows;
}

// Waves a SIMD's registers are shared out to: 16 FM sums, twice 4 FM + 16
// operands and some 60 more each.  That is over the share of the largest and the
// smallest tiles, and instances that LDS holds to one block a CU get no more than
// others.  What does not fit goes to scratch, none of it in the steady depth
// loop: 24 registers and less (FM 8: 1, FM 7: 16), 39 in 64 x 128 tiles of two
// groups (48 with fp32 outputs).
constexpr int waves_per_simd(int FM) { return FM > 4 ? 2 : FM > 2 ? 3 : 4; }

template <typename T, int FM, int WGM, int WGN, int WK, int ST>
__global__ __launch_bounds__(64 * WGM * WGN * WK, waves_per_simd(FM)) void
k_product(ProductParams P, int tm, int tn) {
  constexpr int kWaves = WGM * WGN;  // of a group
  constexpr int kBM = 16 * FM * WGM, kBN = 64 * WGN;
  // a span's loads: 8 rows each, dealt to the group's waves (a wave whose
  // share is short repeats the last one)
  constexpr int kBlocks = (kBM + kBN) / 8;
  constexpr int kLoads = (kBlocks + kWaves - 1) / kWaves;
  constexpr int kStageBytes = (kBM + kBN) * kSpan;
  constexpr int kScaleSlots = (kBM + kBN + 63) / 64 * 64;
  // a whole tile's stores, left on their way while the next tile starts
  constexpr int kStores = WK == 1 ? FM * (int)sizeof(T) : 0;
  static_assert((ST - 1) * kLoads + kStores < 64, "countable by vmcnt");
  static_assert(WK == 1 || kBM * kBN * 4 <= ST * kStageBytes,
                "a group's sums fit its buffers");
  // [WK][ST][x rows | w rows], then two tiles' scales [x rows | w rows]
  extern __shared__ u32x4 lds_all[];
  const int lane = threadIdx.x & 63;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wave_all / kWaves, wave = wave_all % kWaves;
  u32x4 *lds = lds_all + group * (ST * kStageBytes / 16);
  const int full = (int)(P.K / kSpan), rest = (int)(P.K % kSpan);
  const int common = full / WK;                     // every group's spans
  const int most = (full + WK - 1) / WK;
  const int mine = common + (group < full % WK ? 1 : 0);

  // The tile: its rows, and where this lane's part of a load starts.  Rows
  // behind the end repeat the last one; their results are not stored.
  int m0, n0;
  const int8_t *xbase, *wbase;
  uint32_t off[kLoads];
  int turned = 0;  // the span that the depth starts with
  // the lanes of a load fill 64 slots in order (rows 4 to 7 of 8: chunks 4
  // apart too, in odd blocks)
  const int chunk = ((lane & 7) ^ ((lane >> 4) & 3)) * 16;
  auto block_of = [&](int i) { return min(wave + i * kWaves, kBlocks - 1); };
  auto chunk_of = [&](int blk) { return chunk ^ ((blk & 1) * 64); };
  auto row_offset = [&](int blk) {
    const bool w = blk >= kBM / 8;
    const int r = (w ? blk - kBM / 8 : blk) * 8 + (lane >> 3);
    return w ? (uint32_t)min(Runs<T>::w_row(r), (int)P.N - 1 - n0) *
                   (uint32_t)P.ldw
             : (uint32_t)min(r, (int)P.M - 1 - m0) * (uint32_t)P.ldx;
  };
  auto take = [&](int64_t b) {
    int bm, bn;
    tile_of(b, tm, tn, bm, bn);
    m0 = bm * kBM;
    n0 = bn * kBN;
    // Rows a multiple of 4096 bytes apart put equal depths on the same memory
    // channels.  A single row of tiles shares nothing but x, so every tile can
    // start elsewhere (129 x 24576 x 4096 31.7 -> 28.7 us, x 32768 38.8 ->
    // 33.1); tiles that share w stay in step.
    if (tm == 1 && full > 0) turned = bn % full;
    xbase = P.x + (int64_t)m0 * P.ldx;
    wbase = P.w + (int64_t)n0 * P.ldw;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      off[i] = row_offset(block_of(i)) + chunk_of(block_of(i));
  };
  const uint32_t dst = lds_address(lds);
  auto issue1 = [&](int t, int i) {
    const int blk = block_of(i);
    int span = t * WK + group + turned;
    span -= span >= full ? full : 0;
    dma16(dst + (t % ST) * kStageBytes + blk * 1024,
          (blk >= kBM / 8 ? wbase : xbase) +
              (int64_t)span * kSpan,
          off[i]);
  };
  // the tile's scales, to the half of theirs that its turn picks
  float *scale_lds = reinterpret_cast<float *>(
      lds_all + WK * ST * (kStageBytes / 16));
  int turn = 0;
  auto issue_scales = [&]() {
    if (group == 0)
#pragma unroll
      for (int r0 = wave * 64; r0 < kBM + kBN; r0 += kWaves * 64) {
        // (64 at a time: x and w meet inside one where BM is not 64 times
        // something; lanes behind the last row repeat it)
        const int r = min(r0 + lane, kBM + kBN - 1);
        const float *at =
            r < kBM ? P.x_scale + min(m0 + r, (int)P.M - 1)
                    : P.w_scale + min(n0 + r - kBM, (int)P.N - 1);
        dma4(lds_address(scale_lds + turn * kScaleSlots + r0), at);
      }
  };
  auto issue_first = [&](int spans) {
#pragma unroll 1
    for (int t = 0; t < spans && t < mine; ++t)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) issue1(t, i);
  };

  const int wm = (wave / WGN) * (16 * FM), wn = (wave % WGN) * 64;
  // step h reads chunks 4 h + lane / 16 of the wave's rows
  const int slot = span_slot(lane & 15, lane >> 4);
  i32x4 acc[FM][4];
  auto read1 = [&](int t, int h, int r, i32x4 *x, i32x4 *w) {
    const u32x4 *p =
        lds + (t % ST) * (kStageBytes / 16) + (slot ^ (4 * h));
    if (r < 4)
      w[r] = __builtin_bit_cast(i32x4, p[(kBM + wn + r * 16) * 8]);
    else
      x[r - 4] = __builtin_bit_cast(i32x4, p[(wm + (r - 4) * 16) * 8]);
  };
  auto read = [&](int t, int h, i32x4 *x, i32x4 *w) {
#pragma unroll
    for (int r = 0; r < FM + 4; ++r) read1(t, h, r, x, w);
  };
  // One step's products from (x, w), and between them what the wave has to
  // start meanwhile: the next step's operand reads (span t, half h, to (y,
  // v)) and loads d0 .. d1 - 1 of span `to` (none if !load).  Issued in one
  // go, the loads would hold up the products behind them: the address unit
  // takes 16 cycles for each and serves every wave of the CU.
  auto step = [&](const i32x4 *x, const i32x4 *w, int t, int h, i32x4 *y,
                  i32x4 *v, int to, int d0, int d1, bool load, bool use) {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int r = i * (FM + 4) / FM; r < (i + 1) * (FM + 4) / FM; ++r)
        read1(t, h, r, y, v);
      if (load)
#pragma unroll
        for (int d = d0 + i * (d1 - d0) / FM;
             d < d0 + (i + 1) * (d1 - d0) / FM; ++d)
          issue1(to, d);
      if (use)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              w[j], x[i], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  int tile = blockIdx.x;
  take(tile);
  issue_scales();
  bool loading = false;  // the tile's first ST spans are on their way,
  bool storing = false;  // and the stores of a whole tile behind them
  while (true) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    i32x4 xa[FM], wa[4], xb[FM], wb[4];
    if (rest) {
      // the partial span comes first, through the last group's last buffer,
      // while the first loads are on their way: zeros from the depth on
      issue_first(ST - 1);
      if (group == WK - 1) {
        u32x4 *p = lds + (ST - 1) * (kStageBytes / 16) + lane;
        const int64_t k = (int64_t)full * kSpan;
        u32x4 last[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int blk = block_of(i);
          last[i] =
              row_bytes((blk >= kBM / 8 ? wbase : xbase) + row_offset(blk),
                        k + chunk_of(blk), k + rest);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) p[block_of(i) * 64] = last[i];
      }
      __syncthreads();
      if (group == WK - 1) {
#pragma unroll 1
        for (int h = 0; h * kStep < rest; ++h) {
          read(ST - 1, h, xa, wa);
          step(xa, wa, ST - 1, h, xb, wb, 0, 0, 0, false, true);
        }
      }
      __syncthreads();
      if (mine >= ST)
#pragma unroll
        for (int i = 0; i < kLoads; ++i) issue1(ST - 1, i);
    } else if (!loading) {
      issue_first(ST);
    }
    if (full > 0) {
      if (mine >= ST && storing)
        stage_wait<(ST - 1) * kLoads + kStores>();
      else if (mine >= ST)
        stage_wait<(ST - 1) * kLoads>();
      else
        stage_wait<0>();
      read(0, 0, xa, wa);
      // loads of a span: the first half in the step behind the barrier, the
      // others in the step after it; two spans deep, all at once, or they
      // would come too late
      constexpr int kHalf = ST > 2 ? kLoads / 2 : kLoads;
      int t = 0;
      for (; t + ST < common; ++t) {
        step(xa, wa, t, 1, xb, wb, t + ST - 1, kHalf, kLoads, t > 0, true);
        // (spans issued ahead of the stores need not wait for them)
        if (storing && t < ST - 1)
          stage_wait<(ST - 2) * kLoads + kStores>();
        else
          stage_wait<(ST - 2) * kLoads>();
        step(xb, wb, t + 1, 0, xa, wa, t + ST, 0, kHalf, true, true);
      }
#pragma unroll 1
      for (; t < most; ++t) {
        // (behind a group's last span: a stale buffer, never multiplied)
        const bool late = t > 0 && t + ST - 1 < mine;
        step(xa, wa, t, 1, xb, wb, t + ST - 1, kHalf, kLoads, late, t < mine);
        stage_wait<0>();
        step(xb, wb, t + 1, 0, xa, wa, t + ST, 0, kHalf, t + ST < mine,
             t < mine);
      }
    }
    if constexpr (WK > 1) {
      // group g finishes the x operands i with i % WK == g
      __syncthreads();
      i32x4 *sums =
          reinterpret_cast<i32x4 *>(lds) + wave * (FM * 4 * 64) + lane;
#pragma unroll
      for (int i = 0; i < FM; ++i)
        if (i % WK != group)
#pragma unroll
          for (int j = 0; j < 4; ++j) sums[(i * 4 + j) * 64] = acc[i][j];
      __syncthreads();
      const i32x4 *from = reinterpret_cast<const i32x4 *>(lds_all) +
                          wave * (FM * 4 * 64) + lane;
#pragma unroll
      for (int i = 0; i < FM; ++i)
        if (i % WK == group)
#pragma unroll
          for (int g = 0; g < WK; ++g)
            if (g != group)
#pragma unroll
              for (int j = 0; j < 4; ++j)
                acc[i][j] +=
                    from[g * (ST * kStageBytes / 16) + (i * 4 + j) * 64];
    }
    // every wave is behind the last barrier, so all buffers are free: the
    // next tile's first loads go out before this one is finished
    if (full == 0) stage_wait<0>();  // (the scales: else they came first)
    const int m = m0 + wm + (lane & 15), n = n0 + wn + Runs<T>::column(lane);
    const float *tile_scale = scale_lds + turn * kScaleSlots;
    tile += gridDim.x;
    const bool more = tile < tm * tn;
    storing = kStores > 0 && m0 + kBM <= (int)P.M &&
              n0 + kBN <= (int)P.N;
    if (more) {
      if (WK > 1) __syncthreads();  // (the sums have been read)
      take(tile);
      turn ^= 1;
      issue_scales();
      loading = !rest;
      if (loading) issue_first(ST);
      storing &= loading;
    }
    auto own = [&](int i) { return WK == 1 || i % WK == group; };
    finish<T, FM>(
        P, m, n,
        [&](float *scale) {
          const float *s = tile_scale + kBM + wn + Runs<T>::column(lane);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            scale[e] = s[Runs<T>::of(e)];
        },
        [&](int i) { return tile_scale[wm + 16 * i + (lane & 15)]; },
        [&](int i, float *v) {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = (float)acc[i][e >> 2][e & 3];
        },
        own);
    if (!more) break;
  }
}

// Lets a kernel have so much dynamic LDS on the current device (64 KB until it
// asks for more); `devices` holds those that have granted it, by bits.
hipError_t allow_lds(const void *kernel, size_t bytes,
                     std::atomic<uint64_t> &devices) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? 1ull << device : 0;  // (others: each call)
  if (devices.load() & bit) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                          (int)bytes);
  if (e == hipSuccess) devices.fetch_or(bit);
  return e;
}

template <typename T, int FM, int WGM, int WGN, int WK, int ST>
hipError_t product_tiles(const ProductParams &P, hipStream_t s) {
  constexpr int kBM = 16 * FM * WGM, kBN = 64 * WGN;
  constexpr int kThreads = 64 * WGM * WGN * WK;
  constexpr size_t kLds = (size_t)ST * WK * (kBM + kBN) * kSpan +
                          2 * ((kBM + kBN + 63) / 64 * 64) * sizeof(float);
  static_assert(kLds <= 160 * 1024, "LDS of a CU");
  // blocks a CU holds at once, by LDS and by registers
  constexpr int kByLds = (int)(160 * 1024 / kLds);
  constexpr int kByRegs = waves_per_simd(FM) * 256 / kThreads;
  constexpr int kBlocks = kByLds < kByRegs ? kByLds : kByRegs;
  static_assert(kBlocks > 0, "a block fits a CU");
  const int64_t tm = (P.M + kBM - 1) / kBM, tn = (P.N + kBN - 1) / kBN;
  if (tm * tn > INT32_MAX) return hipErrorInvalidValue;
  const int64_t slots = (int64_t)kCUs * kBlocks;
  const auto kernel = &k_product<T, FM, WGM, WGN, WK, ST>;
  static std::atomic<uint64_t> devices{0};
  const hipError_t e =
      allow_lds(reinterpret_cast<const void *>(kernel), kLds, devices);
  if (e != hipSuccess) return e;
  const int64_t grid = tm * tn < slots ? tm * tn : slots;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid),
                     dim3(kThreads), kLds, s, P, (int)tm, (int)tn);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Few rows: a block's four waves share one strip of 16 w rows and split the
// depth, in batches of 4 steps of 64 bytes, each wave's operands coming
// straight from memory to its registers, one batch ahead of the products.
// The waves' sums meet in LDS (integers: the split does not show).

// 4 results of y row m from column n on (m and n inside), with the scales xs
// and scale[0..3].
template <typename T>
__device__ __forceinline__ void finish4(const ProductParams &P, int64_t m,
                                       int64_t n, const i32x4 &acc, float xs,
                                       const float *scale) {
  const T *bias = static_cast<const T *>(P.bias);
  const T *res = static_cast<const T *>(P.res) + m * P.ldr;
  T *y = static_cast<T *>(P.y) + m * P.ldy;
  const int left = (int)min(P.N - n, (int64_t)4);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t c = n + min(e, left - 1);
    v[e] = (float)acc[e] * xs * scale[e];
    if (P.bias) v[e] += to_f32<T>(bias[c]);
    if (P.res) v[e] += to_f32<T>(res[c]);
  }
  if (left == 4) {
    store4<T>(y + n, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < left) y[n + e] = from_f32<T>(v[e]);
}

constexpr int kFewWaves = 4;   // 8 and 16, and batches of 2 to 8 steps,
constexpr int kFewSteps = 4;   // measured no faster at any size

template <typename T, int FM>
__global__ __launch_bounds__(256) void k_product_few(ProductParams P) {
  constexpr int WK = kFewWaves;
  __shared__ i32x4 sums[WK][FM][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t m0 = (int64_t)blockIdx.y * (16 * FM);
  const int kc = (lane >> 4) * 16;
  // rows behind the end repeat the last one; their results are not stored
  const int8_t *wp = P.w + min(n0 + (lane & 15), P.N - 1) * P.ldw;
  const int8_t *xp[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i)
    xp[i] = P.x + min(m0 + 16 * i + (lane & 15), P.M - 1) * P.ldx;
  // wave i < FM finishes x operand i: its scales, ahead of the depth
  static_assert(FM <= WK);
  const int64_t m = m0 + 16 * wave + (lane & 15), n = n0 + 4 * (lane >> 4);
  const float xs = P.x_scale[min(m, P.M - 1)];
  float scale[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) scale[e] = P.w_scale[min(n + e, P.N - 1)];
  constexpr int kBatch = kFewSteps * kStep;
  i32x4 acc[FM] = {};
  struct Batch {
    u32x4 x[kFewSteps][FM], w[kFewSteps];
  };
  auto fetch = [&](int batch, Batch &b) {
#pragma unroll
    for (int u = 0; u < kFewSteps; ++u) {
      const int64_t k = (int64_t)batch * kBatch + u * kStep + kc;
      b.w[u] = *reinterpret_cast<const u32x4_any *>(wp + k);
#pragma unroll
      for (int i = 0; i < FM; ++i)
        b.x[u][i] = *reinterpret_cast<const u32x4_any *>(xp[i] + k);
    }
  };
  auto product1 = [&](const u32x4 *x, const u32x4 &w) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
      acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
          __builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, x[i]),
          acc[i], 0, 0, 0);
  };
  auto multiply = [&](const Batch &b) {
#pragma unroll
    for (int u = 0; u < kFewSteps; ++u) product1(b.x[u], b.w[u]);
  };
  const int batches = (int)(P.K / kBatch);
  // blocks start at different depths, those of an XCD (every 8th) one batch
  // apart: rows 4096 bytes apart put equal depths on the same memory channels
  // (1 x 24576 x 4096 23.5 -> 19.1 us, 5.3 TB/s, x 6144 8.0 -> 6.9)
  const int turned =
      batches > 0 ? (int)(blockIdx.x / 8 % (unsigned)batches) : 0;
  auto next = [&](int i, Batch &to) {
    i += turned;
    fetch(i >= batches ? i - batches : i, to);
  };
  Batch a, b;
  if (wave < batches) next(wave, a);
  for (int i = wave; i < batches; i += 2 * WK) {
    if (i + WK < batches) next(i + WK, b);
    multiply(a);
    if (i + WK >= batches) break;
    if (i + 2 * WK < batches) next(i + 2 * WK, a);
    multiply(b);
  }
  // steps behind the last whole batch, one at a time, first to the waves that
  // had a batch less
#pragma unroll 1
  for (int s = batches * kFewSteps + (wave + WK - batches % WK) % WK;
       (int64_t)s * kStep < P.K; s += WK) {
    u32x4 x[FM];
    const u32x4 w = row_bytes(wp, (int64_t)s * kStep + kc, P.K);
#pragma unroll
    for (int i = 0; i < FM; ++i)
      x[i] = row_bytes(xp[i], (int64_t)s * kStep + kc, P.K);
    product1(x, w);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave < FM && m < P.M && n < P.N) {
    i32x4 s = sums[0][wave][lane];
#pragma unroll
    for (int w = 1; w < WK; ++w) s += sums[w][wave][lane];
    finish4<T>(P, m, n, s, xs, scale);
  }
}

// P's columns n .. n + count - 1.
template <typename T>
ProductParams columns_of(const ProductParams &P, int64_t n, int64_t count) {
  ProductParams S = P;
  S.N = count;
  S.w = ahead(P.w, n * P.ldw);
  S.w_scale = P.w_scale + n;
  S.bias = ahead(P.bias, n * (int)sizeof(T));
  S.res = ahead(P.res, n * (int)sizeof(T));
  S.y = ahead(P.y, n * (int)sizeof(T));
  return S;
}

template <typename T, int FM>
hipError_t product_few(const ProductParams &P, hipStream_t s) {
  constexpr int kThreads = 64 * kFewWaves;
  const unsigned rows = (unsigned)((P.M + 16 * FM - 1) / (16 * FM));
  return in_slices(P.N, 16 * a_launch(kThreads), [&](int64_t n, int64_t count) {
    hipLaunchKernelGGL((k_product_few<T, FM>),
                       dim3((unsigned)((count + 15) / 16), rows),
                       dim3(kThreads), 0, s, columns_of<T>(P, n, count));
    return hipGetLastError();
  });
}

// ---------------------------------------------------------------------------
// Rows off 16-byte addresses, laid out again in the workspace: w behind x, rows
// of whole spans, zeros behind the depth.

struct RepackParams {
  const int8_t *x, *w;
  int8_t *to;
  int64_t M, rows, K, ldx, ldw, pitch;
  int64_t first;  // row that the launch begins with
};

__global__ __launch_bounds__(256) void k_repack(RepackParams P) {
  const int64_t per = P.pitch / 16;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t in = i / per, k = (i - in * per) * 16;
  const int64_t r = P.first + in;
  if (r >= P.rows) return;
  const int8_t *row = r < P.M ? P.x + r * P.ldx : P.w + (r - P.M) * P.ldw;
  u32x4 u = {0u, 0u, 0u, 0u};
  if (k < P.K) u = row_bytes(row, k, P.K);
  *reinterpret_cast<u32x4 *>(P.to + r * P.pitch + k) = u;
}

hipError_t repack(const RepackParams &R, hipStream_t s) {
  const int64_t per = R.pitch / 16;
  return in_slices(R.rows, a_launch(per), [&](int64_t r, int64_t n) {
    RepackParams S = R;
    S.first = r;
    hipLaunchKernelGGL(k_repack, dim3((unsigned)((n * per + 255) / 256)),
                       dim3(256), 0, s, S);
    return hipGetLastError();
  });
}

int64_t repack_pitch(int64_t K) { return (K + kSpan - 1) / kSpan * kSpan; }

// ---------------------------------------------------------------------------
// Choice of the kernel.

// The tiles, the few-row blocks, and a cost by which a call picks one: fitted to
// the times of each on 18 (cols, depth) pairs x up to 22 row counts from 17 to
// 12,900 (bf16 outputs, operands mostly fresh from HBM), then moved to what picks
// the fastest most often.  So costs are near microseconds but no forecast (the
// largest product measured, 1040 us, costs 874):
//   cost = base + rounds * (round + spans * span)
//                  + spans * block_span * (blocks a CU runs, over all rounds)
// with `rounds` the times the 256 CUs are filled and `spans` the spans of 128
// a group of waves goes through; for the few-row blocks
//   base + round * fill + depth * (span + block_span * fill),
// fill = blocks / 256 and depth in units of 256 bytes a wave.  What it picks was
// on average 1.1 % slower than the fastest kernel from 65 rows on (1.3 times at
// worst) and 3.7 % below (1.5 times).  The 224 and 192 row tiles fill rounds that
// leave the 256 row ones idle (9001 x 6144 x 2560 138 -> 129 us by 224, 9001 x
// 2560 x 9728 198 -> 171 by 192).
enum Kernel {
  kTile256, kTile224, kTile192, kTile160, kTile192x128, kTile160x128,
  kTile128, kTile128Deep, kTile64x128, kTile64x128Two, kTile64Two,
  kTile48Four, kTile32Four, kTile16Four, kFew, kKernels
};
struct Shape {
  int rows, cols;    // of a tile or block
  int groups;        // groups of waves that share the depth
  int per_cu;        // blocks a CU holds (0: a few-row block)
  float base, round, span, block_span;
};
constexpr Shape kShapes[kKernels] = {
    {256, 256, 1, 1, 0.17f, 7.26f, 1.138f, 0.000f},
    {224, 256, 1, 1, 0.37f, 8.44f, 1.068f, 0.000f},
    {192, 256, 1, 1, 0.00f, 5.79f, 1.035f, 0.000f},
    {160, 256, 1, 1, 0.34f, 7.82f, 0.739f, 0.000f},
    {192, 128, 1, 1, 1.29f, 6.02f, 0.703f, 0.000f},
    {160, 128, 1, 1, 1.73f, 5.27f, 0.577f, 0.000f},
    {128, 128, 1, 2, 1.91f, 3.73f, 0.389f, 0.262f},
    {128, 128, 1, 1, 1.58f, 4.89f, 0.499f, 0.000f},
    {64, 128, 1, 3, 2.84f, 2.86f, 0.215f, 0.241f},
    {64, 128, 2, 1, 1.91f, 5.31f, 0.602f, 0.000f},
    {64, 64, 2, 2, 2.43f, 1.86f, 0.383f, 0.182f},
    {48, 64, 4, 1, 1.44f, 3.54f, 0.907f, 0.000f},
    {32, 64, 4, 1, 1.78f, 2.54f, 0.611f, 0.000f},
    {16, 64, 4, 1, 0.57f, 3.54f, 0.475f, 0.000f},
    {32, 16, 4, 0, 2.35f, 0.16f, 0.694f, 0.798f},
};
constexpr int kFewRows = 16;   // up to here: one x operand, k_product_few

float expected_us(const Shape &c, int64_t M, int64_t N, int64_t K) {
  const int64_t tiles =
      ((M + c.rows - 1) / c.rows) * ((N + c.cols - 1) / c.cols);
  float us = c.base;
  if (c.per_cu == 0) {
    const float fill = (float)tiles / kCUs;
    const float depth = (float)K / (256.f * c.groups);
    us += c.round * fill + depth * (c.span + c.block_span * fill);
  } else {
    const int64_t slots = (int64_t)c.per_cu * kCUs;
    const int64_t whole = tiles / slots, left = tiles % slots;
    const int64_t rounds = whole + (left ? 1 : 0);
    const int64_t deep = (int64_t)c.groups * kSpan;
    const float spans = (float)((K + deep - 1) / deep);
    us += rounds * (c.round + spans * c.span) +
          spans * c.block_span *
              (whole * c.per_cu + (left + kCUs - 1) / kCUs);
  }
  return us;
}

int choose(int64_t M, int64_t N, int64_t K) {
  int best = 0;
  float least = 0.f;
  for (int i = 0; i < kKernels; ++i) {
    if (kShapes[i].per_cu == 0 && M > 256) continue;  // (not measured)
    const float us = expected_us(kShapes[i], M, N, K);
    if (i == 0 || us < least) {
      least = us;
      best = i;
    }
  }
  return best;
}

// x, w and their strides on 16 bytes, and a tile's rows within 32-bit offsets
bool aligned_rows(const void *x, const void *w, int64_t ldx, int64_t ldw) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x) |
                      reinterpret_cast<uintptr_t>(w) | (uintptr_t)ldx |
                      (uintptr_t)ldw;
  return a % 16 == 0 && ldx < (1 << 22) && ldw < (1 << 22);
}
bool aligned_rows(const ProductParams &P) {
  return aligned_rows(P.x, P.w, P.ldx, P.ldw);
}

template <typename T>
hipError_t product_by_size(const ProductParams &P, hipStream_t s) {
  switch (choose(P.M, P.N, P.K)) {
    case kTile256: return product_tiles<T, 8, 2, 4, 1, 2>(P, s);
    case kTile224: return product_tiles<T, 7, 2, 4, 1, 2>(P, s);
    case kTile192: return product_tiles<T, 6, 2, 4, 1, 2>(P, s);
    case kTile160: return product_tiles<T, 5, 2, 4, 1, 3>(P, s);
    case kTile192x128: return product_tiles<T, 6, 2, 2, 1, 3>(P, s);
    case kTile160x128: return product_tiles<T, 5, 2, 2, 1, 4>(P, s);
    case kTile128: return product_tiles<T, 4, 2, 2, 1, 2>(P, s);
    case kTile128Deep: return product_tiles<T, 4, 2, 2, 1, 4>(P, s);
    case kTile64x128: return product_tiles<T, 2, 2, 2, 1, 2>(P, s);
    case kTile64x128Two: return product_tiles<T, 2, 2, 2, 2, 3>(P, s);
    case kTile64Two: return product_tiles<T, 2, 2, 1, 2, 2>(P, s);
    case kTile48Four: return product_tiles<T, 3, 1, 1, 4, 2>(P, s);
    case kTile32Four: return product_tiles<T, 1, 2, 1, 4, 3>(P, s);
    case kTile16Four: return product_tiles<T, 1, 1, 1, 4, 3>(P, s);
    case kFew: return product_few<T, 2>(P, s);
  }
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t product(ProductParams P, void *workspace, size_t bytes,
                   hipStream_t s) {
  if (P.M <= kFewRows) {
    // the loads of a whole operand cost the few-row blocks as much as w's:
    // from 9 rows, wide and deep products go through LDS tiles instead (16
    // rows through 6144 x 4096 9.4 and 7.5 us, through 24576 x 4096 26.2 and
    // 24.3, but through 4096 x 12288 12.9 and 14.2: three sizes, of which the
    // first stands for the edge)
    if (P.M > 8 && P.N >= 6144 && P.K >= 4096 && aligned_rows(P))
      return product_tiles<T, 1, 1, 1, 4, 3>(P, s);
    return product_few<T, 1>(P, s);
  }
  if (!aligned_rows(P)) {
    RepackParams R{P.x,   P.w, static_cast<int8_t *>(workspace), P.M,
                   P.M + P.N, P.K, P.ldx, P.ldw, repack_pitch(P.K), 0};
    if (!workspace || bytes < (size_t)(R.rows * R.pitch) || P.K == 0)
      return product_any<T>(P, s);
    const hipError_t e = repack(R, s);
    if (e != hipSuccess) return e;
    P.x = R.to;
    P.w = R.to + P.M * R.pitch;
    P.ldx = P.ldw = P.K = R.pitch;
  }
  return product_by_size<T>(P, s);
}

}  // namespace

// Strides that are not set: rows back to back.
size_t product_workspace(const dopr_quant_matmul_args_t &a) {
  if (a.rows <= kFewRows || a.cols == 0 || a.depth == 0 ||
      aligned_rows(a.x, a.w, a.x_row_stride ? a.x_row_stride : a.depth,
                   a.w_row_stride ? a.w_row_stride : a.depth))
    return 0;
  return (size_t)((a.rows + a.cols) * repack_pitch(a.depth));
}

static bool whole_pieces(const dopr_quant_matmul_args_t &a) {
  const int64_t size = a.dtype == DOPR_F32 ? 4 : 2;
  return (reinterpret_cast<uintptr_t>(a.y) |
          (uintptr_t)(a.y_row_stride * size)) % 64 == 0;
}

hipError_t launch_product(const dopr_quant_matmul_args_t &a, hipStream_t s) {
  const ProductParams P{a.x,    a.w,      a.x_scale,      a.w_scale,
                        a.bias, a.residual, a.y,          a.rows,
                        a.cols, a.depth,  a.x_row_stride, a.w_row_stride,
                        a.residual_row_stride, a.y_row_stride,
                        whole_pieces(a)};
  if (a.dtype == DOPR_BF16) return product<bf16_t>(P, a.workspace, a.workspace_bytes, s);
  if (a.dtype == DOPR_F16) return product<_Float16>(P, a.workspace, a.workspace_bytes, s);
  return product<float>(P, a.workspace, a.workspace_bytes, s);
}

}  // namespace dopr
