// direct.hip -- prefix attention over a 4-bit store without a plan: k_own_keys
// forms k^ and the rotations of every token, k_rows_fp4 attends.
//
// A prefix held in 4 bits is small enough not to be kept on the chip: a 32-slot
// chunk of K and V is 34 D bytes, six loads a wave, which go straight into
// operand registers.  So a wave needs no other: it takes 32 of a (pair, kv
// head)'s stacked rows (token, latest first, by q head) and streams the
// document's chunks and then the pair's own keys by itself, with no barrier and
// no work queue, and the pairs need no grouping by document.  (The pass kernel's
// blocks of four waves wait for one another at every batch of keys, issue its
// loads for a thousand cycles, and run waves without rows: 516 rows, 129 tokens
// of 4 heads, take 20 waves there and 17 here.)
//
// Measured, 32 q / 8 kv heads of 128, against the pass kernel and its plan: 64
// pairs of 129 tokens on 4,096 slots each 623 and 665 us, one pair of 4,000 on
// 256 199 and 222, 1,024 pairs of 8 on 64 86 and 138, 1,600 pairs of 129 on 256
// (a thousand documents) 2,070 and 2,000-2,085.  The plan stays ahead where many
// short pairs share few documents, whose rows it puts into common tiles: 1,024
// pairs of 4 tokens on 16 documents of 4,096 slots 541 and 330.
//
// What bounds it: the vector unit (51 % busy; of 2,127 vector instructions a
// wave of the 1,600 pairs, beside 169 products, a chunk's are about 116, 64 of
// them the codes' conversions, q^ 416) and, at its ends, q's loads and the
// output's stores, which two waves a SIMD overlap only in part.  Three (168 registers) were no faster
// at D = 128: the own keys have to be asked for late.
//
// Own keys: k_own_keys stores k^ in groups of four keys, the 16-byte pieces
// that one operand load takes side by side (128 bytes a group), each pair from
// a group of its own; own values are copied into the wave's part of LDS, behind
// the products before them, and read transposed.
//
// The chunks' order, operands and sums are those of the planned kernels, so a
// row that one wave forms comes out bit for bit as theirs.  Where there are few
// rows, up to four waves of a block share a unit's chunks, and several blocks
// where prefixes are long too; their sums meet in LDS and in k_rows_join.
//
// The softmax has no reference where |q^| |k| bounds the logits; without QK-norm
// no bound is known, and a unit whose normaliser leaves the safe range is run
// again with the exact maximum, which shared units take at once.
#include <cmath>

#include "attn_common.hpp"
#include "join.hpp"
#include "operators.hpp"

namespace dopr {
namespace {

constexpr int kMostWaves = 4;  // of a unit
constexpr int waves_a_simd(int D) { return D == 64 ? 4 : 2; }
constexpr int kKeyThreads = 256;
constexpr int kSlab = 8;  // tokens that a block of k_own_keys takes at a time

struct RowsParams {
  StoreView sv;
  const uint16_t *q, *k, *v, *qw, *kw;  // (gains NULL: no norm)
  const int32_t *doc_ids, *cu;
  const float *inv_freq;
  int32_t *status;
  uint16_t *out;
  float *lse;
  int32_t *tiles;    // pair of each 32-row tile
  uint16_t *unit_w;  // [D] ones: the gains where there is no norm
  float *bounds;     // of |k^| and |q^| / c from the gains (0: no norm)
  float2 *rope;      // [Ntok][D / 2]
  uint16_t *kh;      // [Hkv][rows_cap][D], by groups of four keys
  float *part;       // [tile, kv head, split][32][D + 2]: O, m, l
  double log_theta;
  int64_t n_pairs, total_tokens, rows_cap, n_tiles;
  int64_t first;     // first pair, or block, of this launch
  float eps, c;
  int32_t Hq, n_rep, layer, splits, max_tokens;
};

struct Pair {
  int64_t t0;
  int T;
  bool well;
};
__device__ __forceinline__ Pair pair_at(const RowsParams &P, int64_t p) {
  const int64_t t0 = uniform_load(P.cu, p), t1 = uniform_load(P.cu, p + 1);
  return {t0, (int)(t1 - t0),
          t0 >= 0 && t1 > t0 && t1 <= P.total_tokens &&
              t1 - t0 <= P.max_tokens};
}
__device__ __forceinline__ bool has_document(const RowsParams &P, int32_t d) {
  return d >= 0 && (int64_t)d < P.sv.n_docs && uniform_load(P.sv.doc_len, d) >= 0;
}
// The first of a pair's tiles, and of its groups of own keys: bounds that need
// no sum over the pairs before it.
__device__ __forceinline__ int64_t first_tile(const RowsParams &P, int64_t p,
                                              int64_t t0) {
  return t0 * P.n_rep / 32 + p;
}
__device__ __forceinline__ int64_t first_group(int64_t p, int64_t t0) {
  return t0 / 4 + p;
}
// Element offset of a key's 16-byte piece of k-step s, half hf, in its head's
// part of kh.
template <int D>
__device__ __forceinline__ int64_t key_piece(int64_t group0, int key, int s,
                                             int hf) {
  return (group0 + (key >> 2)) * (4 * D) + s * 64 + (key & 3) * 16 + hf * 8;
}

// k^ and the rotations of every token, the tiles' pairs, zero outputs of pairs
// without a document.  A pair's tokens, kSlab at a time, by gridDim.y blocks.
// (Few at a time, and up to 4,096 blocks of a call: what a block waits for is
// its tokens' sines and loads in turn.  32 tokens a block and 1,024 blocks: one
// pair of 129 21 us with the attention for 16, 512 ragged ones 321 for 310, 1,600
// of 129 2,078 for 2,056.)
template <int D>
__global__ __launch_bounds__(kKeyThreads) void k_own_keys(RowsParams P) {
  constexpr int NSUB = D / 16, ROWS = kKeyThreads / NSUB;
  // (pairs side by side, as khat_part takes them; rows off the banks)
  __shared__ __attribute__((aligned(16))) float2 rope[kSlab][D / 2 + 2];
  __shared__ float red[4];
  const int64_t p = P.first + blockIdx.x;
  const int hkv = P.sv.n_kv_heads;
  if (p == 0 && blockIdx.y == 0)
    norm_bound(P.kw, P.qw, D, red, P.bounds, P.unit_w);
  const Pair me = pair_at(P, p);
  if (threadIdx.x == 0 && blockIdx.y == 0 &&
      (!me.well || (p == 0 && P.cu[0] != 0) ||
       (p == P.n_pairs - 1 && P.cu[P.n_pairs] != P.total_tokens)))
    raise_status(P.status, DOPR_ERR_SEQLEN);
  if (!me.well) return;
  const int32_t doc = P.doc_ids[p];
  if (!has_document(P, doc)) {
    if (blockIdx.y != 0) return;
    if (threadIdx.x == 0) raise_status(P.status, DOPR_ERR_DOC_RANGE);
    zero_pair((int32_t)p, P.cu, P.Hq, D, P.out, P.lse);
    return;
  }
  const int L = P.sv.doc_len[doc];
  const int64_t tile0 = first_tile(P, p, me.t0);
  const int n_tiles = (int)(((int64_t)me.T * P.n_rep + 31) / 32);
  for (int i = blockIdx.y * kKeyThreads + threadIdx.x; i < n_tiles;
       i += gridDim.y * kKeyThreads)
    P.tiles[tile0 + i] = (int32_t)p;
  const int64_t group0 = first_group(p, me.t0);
  const int sub = threadIdx.x % NSUB;
  uint4 g0, g1;
  g0 = g1 = make_uint4(0x3F803F80, 0x3F803F80, 0x3F803F80, 0x3F803F80);
  if (P.kw) {
    g0 = *reinterpret_cast<const uint4 *>(P.kw + 8 * sub);
    g1 = *reinterpret_cast<const uint4 *>(P.kw + D / 2 + 8 * sub);
  }
  for (int64_t at = (int64_t)kSlab * blockIdx.y; at < me.T;
       at += (int64_t)kSlab * gridDim.y) {
    const int j0 = (int)at, n = min(kSlab, me.T - j0);
    __syncthreads();  // (the tokens before are done with the table)
    for (int e = threadIdx.x; e < n * (D / 2); e += kKeyThreads) {
      const int j = e / (D / 2), i = e % (D / 2);
      const double freq = P.inv_freq
                              ? (double)P.inv_freq[i]
                              : exp(-(double)i / (D / 2) * P.log_theta);
      double sn, cs;
      sincos((double)((int64_t)L + j0 + j) * freq, &sn, &cs);
      const float2 t = make_float2((float)cs, (float)sn);
      rope[j][i] = t;
      P.rope[(me.t0 + j0 + j) * (D / 2) + i] = t;
    }
    __syncthreads();
    // two rows a thread and step, their loads issued before the first is used
    for (int r0 = threadIdx.x / NSUB; r0 < n * hkv; r0 += 2 * ROWS) {
      uint4 a0[2], a1[2];
      int j[2], g[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int r = r0 + b * ROWS < n * hkv ? r0 + b * ROWS : r0;
        j[b] = r / hkv;
        g[b] = r - j[b] * hkv;
        const uint16_t *kr =
            P.k + ((me.t0 + j0 + j[b]) * hkv + g[b]) * D;
        a0[b] = *reinterpret_cast<const uint4 *>(kr + 8 * sub);
        a1[b] = *reinterpret_cast<const uint4 *>(kr + D / 2 + 8 * sub);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (b > 0 && r0 + ROWS >= n * hkv) break;
        const float4 *c =
            reinterpret_cast<const float4 *>(&rope[j[b]][8 * sub]);
        float x[16];
        khat_part<D>(a0[b], a1[b], g0, g1, c[0], c[1], c[2], c[3], true, P.eps,
                     P.kw != nullptr, x);
        uint16_t *o = P.kh + g[b] * P.rows_cap * D;
        const int key = j0 + j[b], hf = sub & 1;
        *reinterpret_cast<uint4 *>(
            o + key_piece<D>(group0, key, sub >> 1, hf)) =
            as_uint4(to_bf16x8(x));
        *reinterpret_cast<uint4 *>(
            o + key_piece<D>(group0, key, (sub + NSUB) >> 1, hf)) =
            as_uint4(to_bf16x8(x + 8));
      }
    }
  }
}

// One direct load of 1 KB into LDS, lane i's 16 bytes to lds + 16 i; written as
// assembly so that the compiler does not wait for it before the wave's next LDS
// read.  s_nop 4 covers the wait states after vector writes of the base's scalar
// registers and after the write of m0.
__device__ __forceinline__ void to_lds(uint32_t lds, const void *base,
                                       uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\t"
               "global_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *LdsTr;

// A unit, as its waves see it.
struct Rows {
  const char *slice;       // the prefix's chunks
  const uint16_t *kh, *v;  // own keys (first group's head), own values
  int64_t group0;
  int L, T, n_prefix;      // slots, tokens, chunks of the prefix
  int first, end, step;    // chunks of this wave, the prefix's and then own
  int stride;              // elements between own value rows
};

// A chunk's logits, masked past lim, as weights, and O.
template <int SMX, int D, typename VF>
__device__ __forceinline__ void weigh(floatx16 *S, int lim, int hf, VF vf,
                                      Acc<D> *acc) {
  if (!__all(lim >= KC - 1)) {
    const int li = lim - 16 * hf;
#pragma unroll
    for (int i = 0; i < 16; ++i) S[0][i] = i <= li ? S[0][i] : -INFINITY;
  }
  bf16x8 pb[1][2];
  softmax_part<0, 1, SMX, D>(S, acc, hf, 0.f, nullptr, pb);
#pragma unroll
  for (int f = 0; f < D / 16; ++f)
    acc[0].o[f >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
        vf(f), pb[0][f & 1], acc[0].o[f >> 1], 0, 0, 0);
}

// The wave's chunks.  kr, vr: the first one's codes, if it is of the prefix.
// lds: the wave's [32][D] of own values, and its address.
template <int SMX, int D>
__device__ __forceinline__ void row_chunks(const Rows &R, int lane, int j,
                                           const bf16x8 (*qf)[D / 16],
                                           Fp4Raw<D> &kr, Fp4Raw<D> &vr,
                                           const uint16_t *lds, uint32_t lds_at,
                                           Acc<D> *acc) {
  constexpr int G = D / 8, RPB = 64 / G, VB = KC / RPB;
  const int lq = lane & 31, hf = lane >> 5;
  // prefix chunks, from two sets of codes by turns (one that is copied into the
  // other has arrived before it has to)
  int i = R.first;
  const int stop = R.end < R.n_prefix ? R.end : R.n_prefix;
  auto ask = [&](int c, Fp4Raw<D> &k, Fp4Raw<D> &v) {
    if (c >= stop) return;
    const char *chunk = R.slice + (int64_t)c * fp4_chunk_bytes(D);
    fp4_load_k<D>(chunk, lane, k);
    fp4_load_v<D>(chunk, lane, v);
  };
  auto attend = [&](int c, const Fp4Raw<D> &k, const Fp4Raw<D> &v) {
    floatx16 S[1];
#pragma unroll
    for (int x = 0; x < 16; ++x) S[0][x] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      S[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp4_k<D>(k, s), qf[0][s],
                                                     S[0], 0, 0, 0);
    weigh<SMX, D>(S, R.L - 1 - c * KC,
                  hf, [&](int f) { return fp4_v<D>(v, f); }, acc);
  };
  Fp4Raw<D> k2{}, v2{};
  while (i < stop) {
    ask(i + R.step, k2, v2);
    attend(i, kr, vr);
    i += R.step;
    if (i >= stop) break;
    ask(i + R.step, kr, vr);
    attend(i, k2, v2);
    i += R.step;
  }
  if (i >= R.end) return;

  // own chunks: K pieces into registers, V rows into LDS, both asked for behind
  // the products of the chunk before.  (Rows past the pair's last token repeat
  // it: their weights are zero.)
  const int key = perm32(lq), c0 = (i - R.n_prefix) * KC;
  const int row = lane / G;
  const uint32_t col = (uint32_t)((lane % G) ^ (D == 128 ? (row & 3) << 2
                                                         : ((row >> 1) & 1)
                                                               << 2)) << 3;
  const int e4 = (lane >> 2) & 3, q4 = lane & 3;
  const int ex = D == 128 ? e4 : (e4 >> 1);
  const uint16_t *va =
      lds + (16 * hf + e4) * D + perm32(16 * ((lane >> 4) & 1) + 4 * q4);
  bf16x8 kf[D / 16];
  auto ask_k = [&](int c) {
    const uint16_t *from = R.kh + key_piece<D>(R.group0, c + key, 0, hf);
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      kf[s] = *reinterpret_cast<const bf16x8 *>(from + 64 * s);
  };
  auto ask_v = [&](int c) {
    const uint16_t *base = R.v + (int64_t)c * R.stride;
    const int last = R.T - 1 - c;
#pragma unroll
    for (int b = 0; b < VB; ++b) {
      const int r = RPB * b + row;
      to_lds(lds_at + 1024 * b, base,
             ((uint32_t)(r < last ? r : last) * R.stride + col) * 2);
    }
  };
  ask_k(c0);
  ask_v(c0);
  for (int c = c0; i < R.end; i += R.step, c += R.step * KC) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    floatx16 S[1];
#pragma unroll
    for (int x = 0; x < 16; ++x) S[0][x] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      S[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[0][s], S[0], 0,
                                                     0, 0);
    bf16x8 vf[D / 16];
#pragma unroll
    for (int f = 0; f < D / 16; ++f) {
      const uint16_t *a = va + 32 * ((f >> 1) ^ ex) + (f & 1) * 8 * D;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)a);
      const s16x4 hi =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)(a + 4 * D));
      vf[f] = __builtin_bit_cast(
          bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    if (i + R.step < R.end) {
      // (every read of the rows has returned)
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      ask_v(c + R.step * KC);
      ask_k(c + R.step * KC);
    }
    weigh<SMX, D>(S, j - c, hf, [&](int f) { return vf[f]; }, acc);
  }
}

// LDS of a wave: own values, or (shared units) its sums.
template <int D, int WU>
struct RowsSm {
  static constexpr int kBytes = WU == 1 ? KC * D * 2 : 32 * D * 4;
  char wave[WU][kBytes];
  float m[WU][32], l[WU][32];
};

// One block of WU waves a unit, (tile, kv head, split).
template <int D, int WU>
__global__ __launch_bounds__(64 * WU) __attribute__((
    amdgpu_waves_per_eu(WU == 1 ? waves_a_simd(D) : 2,
                        WU == 1 ? waves_a_simd(D)
                                : 2))) void k_rows_fp4(RowsParams P) {
  __shared__ __attribute__((aligned(16))) RowsSm<D, WU> sm;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lq = lane & 31, hf = lane >> 5;
  const int hkv = P.sv.n_kv_heads;
  // blocks of one kv head's tiles, heads and splits side by side: block b runs
  // on XCD b % 8, so that with 8 heads a head's prefix goes through one L2
  const int64_t b = P.first + blockIdx.x;
  const int g = (int)(b % hkv);
  const int64_t rest = b / hkv;
  const int split = (int)(rest % P.splits);
  const int64_t tile = rest / P.splits;
  // (tiles that no pair has hold anything)
  const int64_t p = uniform_load(P.tiles, tile);
  if (p < 0 || p >= P.n_pairs) return;
  const Pair me = pair_at(P, p);
  const int32_t doc = uniform_load(P.doc_ids, p);
  const int64_t at0 = (tile - first_tile(P, p, me.t0)) * 32;
  const int64_t all = (int64_t)me.T * P.n_rep;
  if (!me.well || !has_document(P, doc) || at0 < 0 || at0 >= all) return;
  const int r0 = (int)at0;
  const int rows = (int)(all - at0 < 32 ? all - at0 : 32);

  const int rl = r0 + (lq < rows ? lq : rows - 1);
  const int back = rl / P.n_rep;
  const int j = me.T - 1 - back;  // this lane's position
  const int head = g * P.n_rep + (rl - back * P.n_rep);
  const int64_t tokq = me.t0 + j;
  const bool valid = lq < rows;
  Acc<D> acc[1];
  acc[0].m = 0.f;
  acc[0].l = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int x = 0; x < 16; ++x) acc[0].o[db][x] = 0.f;
  bool bounded = true;
  float lt = 0.f;
  {
    Rows R;
    R.L = uniform_load(P.sv.doc_len, doc);
    R.T = me.T;
    R.slice = reinterpret_cast<const char *>(
        P.sv.payload +
        fp4_offset(uniform_load(P.sv.doc_off, doc), R.L, hkv, P.layer, g, D));
    R.n_prefix = (R.L + KC - 1) / KC;
    // (the tile's latest position is at its first row)
    const int jmax = me.T - 1 - r0 / P.n_rep;
    const int n = R.n_prefix + jmax / KC + 1;
    const int per = (n + P.splits - 1) / P.splits;
    const int begin = min(split * per, n);
    R.end = min(begin + per, n);
    R.first = begin + wave;
    R.step = WU;
    R.stride = hkv * D;
    R.kh = P.kh + g * P.rows_cap * D;
    R.group0 = first_group(p, me.t0);
    R.v = P.v + (me.t0 * hkv + g) * D;
    Fp4Raw<D> kr{}, vr{};
    auto ask_first = [&]() {
      if (R.first < R.end && R.first < R.n_prefix) {
        const char *chunk = R.slice + (int64_t)R.first * fp4_chunk_bytes(D);
        fp4_load_k<D>(chunk, lane, kr);
        fp4_load_v<D>(chunk, lane, vr);
      }
    };
    ask_first();
    bf16x8 qf[1][D / 16];
    q_fragments_any<D>(P.q + (tokq * P.Hq + head) * D,
                       P.qw ? P.qw : P.unit_w, P.rope + tokq * (D / 2), hf,
                       lane, P.n_rep, P.eps, P.c, P.qw != nullptr, qf[0]);
    // every logit (log2 units) lies in [-bound, bound]: the gains' bounds and
    // the stored keys'
    const bool known = P.kw != nullptr;
    const float kmax = uniform_load(
        P.sv.kmax, ((int64_t)doc * P.sv.n_layers + P.layer) * hkv + g);
    const float bound = P.c * uniform_load(P.bounds, 1) *
                        fmaxf(kmax, uniform_load(P.bounds, 0)) * 1.001f;
    // (one wave's sums without a bound are looked at behind the chunks)
    const bool alone = WU == 1;  // (never of several blocks)
    bounded = known ? bound <= kNoRefBound : alone;
    uint16_t *lds = reinterpret_cast<uint16_t *>(sm.wave[wave]);
    const uint32_t at = (uint32_t)(uintptr_t)(
        const __attribute__((address_space(3))) void *)lds;
    if (bounded) {
      row_chunks<0, D>(R, lane, j, qf, kr, vr, lds, at, acc);
      lt = acc[0].l + __shfl_xor(acc[0].l, 32, 64);
      if (!known && __any(valid && !(lt >= kLoOk && lt <= kHiOk))) {
        bounded = false;
        acc[0].l = 0.f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int x = 0; x < 16; ++x) acc[0].o[db][x] = 0.f;
        ask_first();
      }
    }
    if (!bounded) {
      acc[0].m = -INFINITY;
      row_chunks<2, D>(R, lane, j, qf, kr, vr, lds, at, acc);
      lt = acc[0].l + __shfl_xor(acc[0].l, 32, 64);
    }
  }

  if constexpr (WU == 1) {
    if (!valid) return;
    const int64_t orow = tokq * P.Hq + head;
    const float inv = 1.0f / lt;
    uint16_t *op = P.out + orow * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      float o[16];
#pragma unroll
      for (int x = 0; x < 16; ++x) o[x] = acc[0].o[db][x] * inv;
      uint4 *dst = reinterpret_cast<uint4 *>(op + 32 * db + 16 * hf);
      dst[0] = as_uint4(to_bf16x8(o));
      dst[1] = as_uint4(to_bf16x8(o + 8));
    }
    if (P.lse && hf == 0) P.lse[orow] = (acc[0].m + __log2f(lt)) * kLn2;
  } else {
    // the waves' sums meet.  (The wave's own values in LDS have been read.)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (valid) {
      float *o = reinterpret_cast<float *>(sm.wave[wave]) + lq * D;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int x = 0; x < 16; x += 4)
          *reinterpret_cast<float4 *>(o + 32 * db + 16 * hf + x) =
              make_float4(acc[0].o[db][x], acc[0].o[db][x + 1],
                          acc[0].o[db][x + 2], acc[0].o[db][x + 3]);
      if (hf == 0) {
        sm.m[wave][lq] = acc[0].m;
        sm.l[wave][lq] = lt;
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * (D / 4); e += 64 * WU) {
      const int rr = e / (D / 4), d = 4 * (e % (D / 4));
      float M = 0.f;
      if (!bounded) {
        M = -INFINITY;
#pragma unroll
        for (int w = 0; w < WU; ++w) M = fmaxf(M, sm.m[w][rr]);
      }
      // (nothing seen, M = -inf: all weights are zero)
      const float ref = M == -INFINITY ? 0.f : M;
      float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WU; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm.m[w][rr] - ref);
        const float4 x = *reinterpret_cast<const float4 *>(
            reinterpret_cast<const float *>(sm.wave[w]) + rr * D + d);
        l = fmaf(f, sm.l[w][rr], l);
        o[0] = fmaf(f, x.x, o[0]);
        o[1] = fmaf(f, x.y, o[1]);
        o[2] = fmaf(f, x.z, o[2]);
        o[3] = fmaf(f, x.w, o[3]);
      }
      if (P.splits > 1) {
        float *to = P.part + ((tile * hkv + g) * P.splits + split) *
                                 (int64_t)(32 * (D + 2)) +
                    rr * (D + 2);
        *reinterpret_cast<float2 *>(to + d) = make_float2(o[0], o[1]);
        *reinterpret_cast<float2 *>(to + d + 2) = make_float2(o[2], o[3]);
        if (d == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(M, l);
        continue;
      }
      const int rw = r0 + rr, bk = rw / P.n_rep;
      const int64_t orow = (me.t0 + me.T - 1 - bk) * P.Hq + g * P.n_rep +
                           (rw - bk * P.n_rep);
      const float inv = 1.0f / l;
      const bf16x2 a = {(__bf16)(o[0] * inv), (__bf16)(o[1] * inv)};
      const bf16x2 c = {(__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
      *reinterpret_cast<uint2 *>(P.out + orow * D + d) =
          make_uint2(__builtin_bit_cast(uint32_t, a),
                     __builtin_bit_cast(uint32_t, c));
      if (P.lse && d == 0) P.lse[orow] = (ref + __log2f(l)) * kLn2;
    }
  }
}

// The sums of a row's blocks, rows (tile, row of it, kv head).
template <int D, int PARTS>
__global__ __launch_bounds__(join_threads(D, PARTS)) void k_rows_join(
    RowsParams P) {
  const int hkv = P.sv.n_kv_heads;
  const int64_t at =
      PARTS > 1 ? blockIdx.x
                : (int64_t)blockIdx.x * join_rows(D, 1) + threadIdx.x / (D / 2);
  const int g = at % hkv, rr = at / hkv % 32;
  const int64_t tile = at / hkv / 32;
  if (tile >= P.n_tiles) return;
  const int64_t p = P.tiles[tile];
  if (p < 0 || p >= P.n_pairs) return;
  const Pair me = pair_at(P, p);
  const int64_t r = (tile - first_tile(P, p, me.t0)) * 32 + rr;
  if (!me.well || !has_document(P, P.doc_ids[p]) || r < rr ||
      r >= (int64_t)me.T * P.n_rep)
    return;
  const int64_t back = r / P.n_rep;
  const int64_t row = (me.t0 + me.T - 1 - back) * P.Hq + g * P.n_rep +
                      (r - back * P.n_rep);
  const int64_t step = 32 * (D + 2);
  join_row<D, PARTS>(P.part + (tile * hkv + g) * P.splits * step + rr * (D + 2), step,
              P.splits, P.out + row * D, P.lse ? P.lse + row : nullptr);
}

// How a call's (tile, kv head)s are shared out: one wave each where they take
// more than half of the 2,048 waves the SIMDs hold (D = 64: 4,096), two or four
// below, and several blocks of four, of at least four chunks a wave of the
// longest sequence, where that leaves waves free and saves more than the sums'
// way through memory and their join cost: about where there are more chunks
// than units and 32 more.  (32 q / 8 kv heads: 16 pairs of 8 tokens on 2,048
// slots 24.5 us, in four blocks 31; one on 4,096 29, in eight 20; four on 4,096
// 29 and 22.5.)
struct RowsShare {
  int waves, splits;
};
RowsShare rows_share(int D, int64_t units, int64_t max_len,
                     int64_t max_tokens) {
  const int64_t full = 1024 * waves_a_simd(D);
  if (2 * units > full) return {1, 1};
  if (4 * units > full) return {2, 1};
  const int64_t chunks = (max_len + max_tokens + KC - 1) / KC;
  if (chunks <= 32 + units) return {kMostWaves, 1};
  const int64_t want = full / (units * kMostWaves);
  const int64_t most = chunks / (4 * kMostWaves);
  return {kMostWaves, (int)std::max<int64_t>(1, std::min(want, most))};
}

struct RowsLayout {
  int64_t n_tiles, rows_cap;
  RowsShare share;
  size_t tiles, unit_w, bounds, rope, kh, part, bytes;
};
RowsLayout rows_layout(const dopr_store &st, const dopr_attn_args_t &a) {
  const int64_t hkv = st.n_kv_heads, D = st.head_dim;
  const int64_t n_rep = a.n_q_heads / hkv, P = a.n_pairs;
  RowsLayout l;
  l.n_tiles = a.total_tokens * n_rep / 32 + P;
  // (groups of four keys, and the last chunk's load)
  l.rows_cap = 4 * (a.total_tokens / 4 + P) + 32;
  l.share = rows_share((int)D, l.n_tiles * hkv, st.max_len,
                       std::min<int64_t>(a.max_tokens, a.total_tokens));
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at = align_up(at + n, kAlign);
    return here;
  };
  l.tiles = take(sizeof(int32_t) * l.n_tiles);
  l.unit_w = take(sizeof(uint16_t) * D);
  l.bounds = take(sizeof(float) * 2);
  l.rope = take(sizeof(float2) * a.total_tokens * (D / 2));
  l.kh = take(sizeof(uint16_t) * hkv * l.rows_cap * D);
  l.part = take(l.share.splits == 1 ? 0
                                    : sizeof(float) * l.n_tiles * hkv *
                                          l.share.splits * 32 * (D + 2));
  l.bytes = at;
  return l;
}

template <int D>
hipError_t launch_rows1(RowsParams P, int waves, hipStream_t s) {
  const int64_t hkv = P.sv.n_kv_heads;
  // (few pairs of many tokens: blocks share a pair's)
  const int64_t most = std::min<int64_t>(P.max_tokens, P.total_tokens);
  const int64_t y = std::min((most + kSlab - 1) / kSlab,
                             std::max<int64_t>(1, 4096 / P.n_pairs));
  hipError_t e =
      in_slices(P.n_pairs, a_launch(kKeyThreads), [&](int64_t at, int64_t n) {
        RowsParams S = P;
        S.first = at;
        hipLaunchKernelGGL(k_own_keys<D>, dim3((unsigned)n, (unsigned)y),
                           dim3(kKeyThreads), 0, s, S);
        return hipGetLastError();
      });
  if (e != hipSuccess) return e;
  const int64_t blocks = P.n_tiles * hkv * P.splits;
  e = in_slices(blocks, a_launch(64 * waves), [&](int64_t at, int64_t n) {
    RowsParams S = P;
    S.first = at;
    const auto kernel = waves == 1   ? k_rows_fp4<D, 1>
                        : waves == 2 ? k_rows_fp4<D, 2>
                                     : k_rows_fp4<D, 4>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(64 * waves), 0, s,
                       S);
    return hipGetLastError();
  });
  if (e != hipSuccess || P.splits == 1) return e;
  // (units of several blocks are few: below 2^20 rows)
  const int parts = join_parts(P.splits), per = join_rows(D, parts);
  const auto join = parts > 1 ? k_rows_join<D, kJoinParts> : k_rows_join<D, 1>;
  hipLaunchKernelGGL(join,
                     dim3((unsigned)((P.n_tiles * 32 * hkv + per - 1) / per)),
                     dim3(join_threads(D, parts)), 0, s, P);
  return hipGetLastError();
}

}  // namespace

size_t rows_bytes(const dopr_store &st, const dopr_attn_args_t &a) {
  return rows_layout(st, a).bytes;
}

hipError_t launch_rows(const AttnCall &c, void *workspace, hipStream_t s) {
  const dopr_attn_args_t *a = c.a;
  const dopr_store &st = *c.st;
  const RowsLayout l = rows_layout(st, *a);
  char *ws = static_cast<char *>(workspace);
  RowsParams P{};
  P.sv = st.view();
  P.q = static_cast<const uint16_t *>(a->q);
  P.k = static_cast<const uint16_t *>(a->k);
  P.v = static_cast<const uint16_t *>(a->v);
  P.qw = static_cast<const uint16_t *>(a->q_norm_w);
  P.kw = static_cast<const uint16_t *>(a->k_norm_w);
  P.doc_ids = a->doc_ids;
  P.cu = a->cu_seqlens;
  P.inv_freq = a->rope_inv_freq;
  P.status = st.d_status;
  P.out = static_cast<uint16_t *>(a->out);
  P.lse = a->lse;
  P.tiles = reinterpret_cast<int32_t *>(ws + l.tiles);
  P.unit_w = reinterpret_cast<uint16_t *>(ws + l.unit_w);
  P.bounds = reinterpret_cast<float *>(ws + l.bounds);
  P.rope = reinterpret_cast<float2 *>(ws + l.rope);
  P.kh = reinterpret_cast<uint16_t *>(ws + l.kh);
  P.part = reinterpret_cast<float *>(ws + l.part);
  P.log_theta = std::log((double)a->rope_theta);
  P.n_pairs = a->n_pairs;
  P.total_tokens = a->total_tokens;
  P.rows_cap = l.rows_cap;
  P.n_tiles = l.n_tiles;
  P.eps = a->rms_eps;
  P.c = a->softmax_scale * 1.4426950408889634f;
  P.Hq = a->n_q_heads;
  P.n_rep = c.n_rep;
  P.layer = c.layer;
  P.splits = l.share.splits;
  P.max_tokens = a->max_tokens;
  hipError_t e = hipSuccess;
  if (a->timing_begin)
    e = hipEventRecord(static_cast<hipEvent_t>(a->timing_begin), s);
  if (e == hipSuccess)
    e = st.head_dim == 128 ? launch_rows1<128>(P, l.share.waves, s)
                           : launch_rows1<64>(P, l.share.waves, s);
  if (e == hipSuccess && a->timing_end)
    e = hipEventRecord(static_cast<hipEvent_t>(a->timing_end), s);
  return e;
}

}  // namespace dopr
