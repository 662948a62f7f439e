// token.hip -- prefix attention of pairs of one token over a 4-bit store
// (k_token_fp4), the form that serving a token at a time takes.
//
// A pair has n_rep rows a kv head, one own key (its own), and a prefix to
// read: bound by HBM, 17/16 bytes a slot and dim of K and V.  No plan: the waves
// of a (pair, kv head) find its document and each form q^ and k^ and the own
// key's logit for themselves; they take the document's 32-slot chunks two at a
// time, codes straight from memory into operand registers, the next two asked
// for before the present ones' products, and keep their own sums, which meet
// in LDS.  One wave takes a (pair, kv head) where there are enough of them to
// fill the card, up to four where there are not, and where pairs are few and
// prefixes long several blocks, which leave their sums to k_token_join.
//
// Rows are few, so the products are of 16 columns (v_mfma_f32_16x16x32_bf16):
// half the matrix cycles, logits and sums of the 32-column ones.  With lane = 16
// kg + m, a 16-byte piece of a chunk's codes is one lane's operand of a tile's
// four (D = 128) k-steps: piece (part kg / 2, half kg % 2) of the key of row m
// for S^T = K Q^T, dims 64 (kg / 2) + 16 ks + 8 (kg % 2) + e in step ks; row m
// of tile mt is slot 16 (m / 8) + 4 mt + m % 4 of chunk (m / 4) % 2, so that a
// lane's 16 logits are the slots 16 (kg / 2) .. + 15 of chunk kg % 2, two
// operands of O^T = V^T P^T, against the pieces (chunk kg % 2, half kg / 2) of
// the values.
//
// The softmax has no running maximum where |q^| |k| bounds the logits (exact
// norms of this pair's rows; kmax of the document's keys), and an exact one
// elsewhere, in the same launch.  q^ enters the products as two bf16 parts (16
// bits of mantissa): the matrix cores have room, and the keys are exact.
#include <cmath>
#include <type_traits>

#include "attn_common.hpp"
#include "join.hpp"
#include "operators.hpp"

namespace dopr {
namespace {

constexpr int kTokenWaves = 4;  // of a unit, at most

struct TokenParams {
  StoreView sv;
  const uint16_t *q, *k, *v, *qw, *kw;  // (no gains: no norm)
  const int32_t *doc_ids, *cu;
  const float *inv_freq;
  int32_t *status;
  uint16_t *out;
  float *lse;
  float *part;  // [pair, kv head, split][n_rep][D + 2]: O, m, l
  double log_theta;
  int64_t p0, n_pairs, total_tokens;  // first pair of this launch; all pairs
  float eps, c;
  int32_t Hq, n_rep, layer, splits;
  uint32_t units;                     // (pair, kv head, split) of this launch
};

// Whether pair p has one token, and which.
__device__ __forceinline__ bool one_token(const TokenParams &P, int64_t p,
                                          int64_t &t0) {
  t0 = uniform_load(P.cu, p);
  return t0 >= 0 && uniform_load(P.cu, p + 1) == t0 + 1 && t0 < P.total_tokens;
}
__device__ __forceinline__ bool has_document(const TokenParams &P, int32_t d) {
  return d >= 0 && (int64_t)d < P.sv.n_docs &&
         uniform_load(P.sv.doc_len, d) >= 0;
}

__device__ __forceinline__ void store_out(uint16_t *to, const float *o,
                                          float inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bf16x2 h = {(__bf16)(o[2 * i] * inv), (__bf16)(o[2 * i + 1] * inv)};
    w[i] = __builtin_bit_cast(uint32_t, h);
  }
  *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
}

constexpr int kTokenRows = 16;  // of a tile

// What a wave keeps of a unit's rows.
template <int D>
struct TokenRows {
  float q[kTokenRows][D];  // c q^, then the wave's sums O
  float k[D];              // k^ of the own key
  float2 rope[D / 2];
  float norm2[kTokenRows + 1];  // of the rows of q, and of k
  float own[kTokenRows];        // logits of the own key
  float m[kTokenRows], l[kTokenRows];
};

// The wave's LDS accesses so far, and the compiler's, end here.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A lane's codes and exponents of two chunks.
template <int D>
struct Codes {
  std::conditional_t<D == 128, fp4_u32x4, u32x2> k[4];  // by tile
  fp4_u32x4 v[D / 32];  // [part][lq / 16]
  uint8_t kx[4];
  std::conditional_t<D == 128, uint32_t, uint16_t> vx[2];
};

// Chunks c and c + 1 of `end` (the last one again past it).  (The lane's places
// are formed here: held across the loops they take the registers of a wave.)
template <int D>
__device__ __forceinline__ void load_keys(const char *slice, int c, int end,
                                          int lane, Codes<D> &r) {
  const int ln = lane + opaque_zero(), m = ln & 15, kg = ln >> 4;
  const char *chunk =
      slice + (int64_t)min(c + ((m >> 2) & 1), end - 1) * fp4_chunk_bytes(D);
  const int lk = (kg & 1) * 32 + 4 * (m >> 3) + (m & 3);  // (of tile 0)
  const char *at = chunk + (D == 128 ? 1024 : 8) * (kg >> 1) + 16 * lk;
  const char *ax =
      chunk + 32 * D + lk * (D / 64) + (D == 128 ? kg >> 1 : 0);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    r.k[t] = *reinterpret_cast<const decltype(r.k[0] + 0) *>(at + 128 * t);
    r.kx[t] = *reinterpret_cast<const uint8_t *>(ax + 8 * (D / 64) * t);
  }
}
template <int D>
__device__ __forceinline__ void load_values(const char *slice, int c, int end,
                                            int lane, Codes<D> &r) {
  const int ln = lane + opaque_zero(), m = ln & 15, kg = ln >> 4;
  const char *chunk =
      slice + (int64_t)min(c + (kg & 1), end - 1) * fp4_chunk_bytes(D);
  const char *at = chunk + 16 * D + 16 * ((kg >> 1) * 32 + m);
  const char *ax = chunk + 33 * D + m * (D / 32);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
      r.v[2 * j + h] =
          *reinterpret_cast<const fp4_u32x4 *>(at + 1024 * j + 256 * h);
    r.vx[h] = *reinterpret_cast<const decltype(r.vx[0] + 0) *>(ax + h * (D / 2));
  }
}

// Sums of a tile's 16 columns: O^T by tiles of 16 dims, tile (j, dbl, h) dims
// 32 (2 j + dbl) + 16 (kg % 2) + 8 h + 4 (kg / 2) + i, and as Acc.
template <int D>
struct Sums {
  floatx4 o[D / 16];
  float m, l;
};

// x of the lanes with the same m: all four's largest.
__device__ __forceinline__ float max4(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}

// Chunks c, c + 1; c + 2 step, ..: O and the normaliser of this wave's share of
// the chunks below `end`.  r: the first two's codes, on their way or there; the
// next two's are asked for as soon as the registers are free, the keys' behind
// the logits, the values' behind the sums.
template <int SMX, int D>
__device__ __forceinline__ void token_chunks(const char *slice, int c, int end,
                                             int step, int L, int lane,
                                             const bf16x8 *qh, const bf16x8 *ql,
                                             Codes<D> &r, Sums<D> &acc) {
  constexpr int KS = D / 32;
  const int kg = lane >> 4;
  step *= 2;
  for (; c < end; c += step) {
    const bool more = c + step < end;
    floatx4 S[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      S[t] = floatx4{0.f, 0.f, 0.f, 0.f};
      const float scale = fp4_scale(r.kx[t]);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 kf = fp4_fragment(r.k[t][ks], scale);
        S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qh[ks], S[t], 0, 0,
                                                       0);
        S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, ql[ks], S[t], 0, 0,
                                                       0);
      }
    }
    if (more) load_keys<D>(slice, c + step, end, lane, r);
    if ((c + 2) * KC > L || c + 2 > end) {
      // (a second chunk past the share's end is the last one again)
      const int lim = c + (kg & 1) < end
                          ? L - (c + (kg & 1)) * KC - 16 * (kg >> 1) : 0;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          S[t][i] = 4 * t + i < lim ? S[t][i] : -INFINITY;
    }
    float muse = 0.f;
    if constexpr (SMX == 2) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S[t][i]);
      mx = max4(mx);
      const bool need = mx > acc.m + kTau;
      const float mnew = need ? mx : acc.m;
      const float alpha = need ? __builtin_amdgcn_exp2f(acc.m - mnew) : 1.0f;
      acc.l *= alpha;
      acc.m = mnew;
      if (__any(need)) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc.o[d][i] *= alpha;
      }
      muse = acc.m == -INFINITY ? 0.f : acc.m;
    }
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
    bf16x8 pb[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float p[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float s = S[2 * t + (x >> 2)][x & 3];
        p[x] = __builtin_amdgcn_exp2f(SMX == 2 ? s - muse : s);
      }
      pb[t] = to_bf16x8(p);
      // (the normaliser sums the weights that the products use)
      const bf16x8 &w = pb[t];
      acc.l = __builtin_amdgcn_fdot2_f32_bf16(
          __builtin_shufflevector(w, w, 0, 1), one, acc.l, false);
      acc.l = __builtin_amdgcn_fdot2_f32_bf16(
          __builtin_shufflevector(w, w, 2, 3), one, acc.l, false);
      acc.l = __builtin_amdgcn_fdot2_f32_bf16(
          __builtin_shufflevector(w, w, 4, 5), one, acc.l, false);
      acc.l = __builtin_amdgcn_fdot2_f32_bf16(
          __builtin_shufflevector(w, w, 6, 7), one, acc.l, false);
    }
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int dbl = 0; dbl < 2; ++dbl)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float scale = fp4_scale(r.vx[h] >> (8 * (2 * j + dbl)) & 255);
          floatx4 &o = acc.o[4 * j + 2 * dbl + h];
#pragma unroll
          for (int t = 0; t < 2; ++t)
            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                fp4_fragment(r.v[2 * j + h][2 * dbl + t], scale), pb[t], o, 0,
                0, 0);
        }
    if (more) load_values<D>(slice, c + step, end, lane, r);
  }
}

// One block of WU waves a unit, (pair, kv head, split).  (With four units of
// one wave in a block, whose waves and LDS come free together, 4,096 pairs on 64
// to 512 slots take 307 us for 290.)
template <int D, int WU>
__global__ __launch_bounds__(64 * WU) __attribute__((
    amdgpu_waves_per_eu(2, 2))) void k_token_fp4(TokenParams P) {
  constexpr int G = D / 8;    // lanes a row, eight dims each
  constexpr int RP = 64 / G;  // rows at a time
  constexpr int RT = kTokenRows;
  __shared__ __attribute__((aligned(16))) TokenRows<D> sm_all[WU];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kg = lane >> 4;
  const int hkv = P.sv.n_kv_heads;
  TokenRows<D> &sm = sm_all[wave];
  const unsigned u = blockIdx.x;
  const int g = u % hkv;
  const unsigned rest = u / hkv;
  const int split = rest % P.splits;
  const int64_t p = P.p0 + rest / P.splits;
  int64_t tok;
  const int32_t doc = uniform_load(P.doc_ids, p);
  const bool well = one_token(P, p, tok);
  const bool first_of_pair = lane == 0 && wave == 0 && g == 0 && split == 0;
  if (first_of_pair &&
      (!well || (p == 0 && P.cu[0] != 0) ||
       (p == P.n_pairs - 1 && P.cu[P.n_pairs] != P.total_tokens)))
    raise_status(P.status, DOPR_ERR_SEQLEN);
  if (!well) return;  // (the whole block)
  const int64_t row0 = tok * P.Hq + g * P.n_rep;
  if (!has_document(P, doc)) {
    if (first_of_pair) raise_status(P.status, DOPR_ERR_DOC_RANGE);
    if (split == 0 && wave == 0) {
      for (int e = lane; e < P.n_rep * G; e += 64)
        reinterpret_cast<uint4 *>(P.out + row0 * D)[e] =
            make_uint4(0, 0, 0, 0);
      if (P.lse)
        for (int e = lane; e < P.n_rep; e += 64) P.lse[row0 + e] = -INFINITY;
    }
    return;
  }
  // (asked for before what hangs on the pair)
  float freq = 0.f;
  if (P.inv_freq && lane < D / 2) freq = P.inv_freq[lane];
  uint4 gain_q, gain_k;
  if (P.qw) {
    gain_q = *reinterpret_cast<const uint4 *>(P.qw + 8 * (lane % G));
    gain_k = *reinterpret_cast<const uint4 *>(P.kw + 8 * (lane % G));
  }
  const int L = uniform_load(P.sv.doc_len, doc);
  const char *slice = reinterpret_cast<const char *>(
      P.sv.payload + fp4_offset(uniform_load(P.sv.doc_off, doc), L, hkv,
                                P.layer, g, D));
  const float kmax = uniform_load(
      P.sv.kmax, ((int64_t)doc * P.sv.n_layers + P.layer) * hkv + g);
  const int n_chunks = (L + KC - 1) / KC;
  const int per = (n_chunks + P.splits - 1) / P.splits;
  const int begin = min(split * per, n_chunks);
  const int end = min(begin + per, n_chunks), first = begin + 2 * wave;

  for (int r0 = 0; r0 < P.n_rep; r0 += RT) {
    const int rows = min(RT, P.n_rep - r0);
    bool bounded = true;
    Codes<D> codes{};
    if (first < end) {
      load_keys<D>(slice, first, end, lane, codes);
      load_values<D>(slice, first, end, lane, codes);
    }
    // c q^ of the rows and k^, G lanes a row; row `rows` is the own key
    const int gc = lane % G;
    auto row_of = [&](int rr) {
      return rr < rows ? P.q + (row0 + r0 + rr) * D
                       : P.k + (tok * hkv + g) * D;
    };
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (lane / G <= rows)
      raw = *reinterpret_cast<const uint4 *>(row_of(lane / G) + 8 * gc);
    if (r0 == 0 && lane < D / 2) {
      // whole turns are dropped in 64 bits
      const double by = P.inv_freq
                            ? (double)freq
                            : exp(-(double)lane / (D / 2) * P.log_theta);
      const double turns = (double)L * by * 0.15915494309189533577;
      float sn, cs;
      sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
      sm.rope[lane] = make_float2(cs, sn);
    }
    wave_fence();
    for (int rr = lane / G; rr <= rows; rr += RP) {
      float x[8], y[8];
      unpack8(raw, x);
      if (rr + RP <= rows)
        raw = *reinterpret_cast<const uint4 *>(row_of(rr + RP) + 8 * gc);
      if (P.qw) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int off = 1; off < G; off <<= 1) ss += __shfl_xor(ss, off, 64);
        const float inv = 1.0f / sqrtf(ss * (1.0f / D) + P.eps);
        float gain[8];
        unpack8(rr < rows ? gain_q : gain_k, gain);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * gain[e];
      }
      // (the partner of dim i is i +- D/2)
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = __shfl_xor(x[e], G / 2, 64);
      const float sign = gc < G / 2 ? -1.f : 1.f, by = rr < rows ? P.c : 1.f;
      float n2 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 t = sm.rope[(8 * gc + e) % (D / 2)];
        x[e] = by * fmaf(x[e], t.x, sign * y[e] * t.y);
        n2 = fmaf(x[e], x[e], n2);
      }
#pragma unroll
      for (int off = 1; off < G; off <<= 1) n2 += __shfl_xor(n2, off, 64);
      if (gc == 0) sm.norm2[rr < rows ? rr : RT] = n2;
      float4 *to = reinterpret_cast<float4 *>(
          (rr < rows ? sm.q[rr] : sm.k) + 8 * gc);
      to[0] = make_float4(x[0], x[1], x[2], x[3]);
      to[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
    wave_fence();
    if (split == 0 && wave == 0)
      for (int rr = lane / G; rr < rows; rr += RP) {
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          dot = fmaf(sm.q[rr][8 * gc + e], sm.k[8 * gc + e], dot);
#pragma unroll
        for (int off = 1; off < G; off <<= 1) dot += __shfl_xor(dot, off, 64);
        if (gc == 0) sm.own[rr] = dot;
      }
    // every logit (log2 units) lies in [-bound, bound] (rows with NaN aside,
    // which come out NaN either way)
    float top = 0.f;
    for (int rr = 0; rr < rows; ++rr) top = fmaxf(top, sm.norm2[rr]);
    const float bound =
        sqrtf(top) * fmaxf(kmax, sqrtf(sm.norm2[RT])) * 1.001f;
    bounded = bound <= kNoRefBound;

    bf16x8 qh[D / 32], ql[D / 32];
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const int dim = D == 128 ? 64 * (kg >> 1) + 16 * ks + 8 * (kg & 1)
                               : 32 * (kg >> 1) + 16 * ks + 8 * (kg & 1);
      float x[8];
      const float4 *from = reinterpret_cast<const float4 *>(
          &sm.q[col < rows ? col : 0][dim]);
      const float4 a = from[0], b = from[1];
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
      x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
      qh[ks] = to_bf16x8(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] -= (float)qh[ks][e];
      ql[ks] = to_bf16x8(x);
    }
    Sums<D> acc;
    acc.m = bounded ? 0.f : -INFINITY;
    acc.l = 0.f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) acc.o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (bounded)
      token_chunks<0, D>(slice, first, end, WU, L, lane, qh, ql, codes, acc);
    else
      token_chunks<2, D>(slice, first, end, WU, L, lane, qh, ql, codes, acc);

    // the wave's sums, where q^ was
    float lt = acc.l + __shfl_xor(acc.l, 16, 64);
    lt += __shfl_xor(lt, 32, 64);
    wave_fence();
    if (col < rows) {
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        *reinterpret_cast<floatx4 *>(
            &sm.q[col][32 * (d >> 1) + 16 * (kg & 1) + 8 * (d & 1) +
                       4 * (kg >> 1)]) = acc.o[d];
      if (kg == 0) {
        sm.m[col] = acc.m;
        sm.l[col] = lt;
      }
    }
    if constexpr (WU == 1)
      wave_fence();
    else
      __syncthreads();
    for (int e = threadIdx.x; e < rows * (D / 4); e += 64 * WU) {
      const int rr = e / (D / 4), d = 4 * (e % (D / 4));
      const float own = split == 0 ? sm_all[0].own[rr] : -INFINITY;
      float M = 0.f;
      if (!bounded) {
        M = own;
#pragma unroll
        for (int w = 0; w < WU; ++w) M = fmaxf(M, sm_all[w].m[rr]);
      }
      // (nothing seen, M = -inf: all weights are zero)
      const float ref = M == -INFINITY ? 0.f : M;
      float l = __builtin_amdgcn_exp2f(own - ref);
      float o[4] = {0.f, 0.f, 0.f, 0.f};
      if (split == 0) {
        const uint2 x = *reinterpret_cast<const uint2 *>(
            P.v + (tok * hkv + g) * D + d);
        o[0] = l * __uint_as_float(x.x << 16);
        o[1] = l * __uint_as_float(x.x & 0xffff0000u);
        o[2] = l * __uint_as_float(x.y << 16);
        o[3] = l * __uint_as_float(x.y & 0xffff0000u);
      }
#pragma unroll
      for (int w = 0; w < WU; ++w) {
        const TokenRows<D> &from = sm_all[w];
        const float f = __builtin_amdgcn_exp2f(from.m[rr] - ref);
        const float4 x = *reinterpret_cast<const float4 *>(&from.q[rr][d]);
        l = fmaf(f, from.l[rr], l);
        o[0] = fmaf(f, x.x, o[0]);
        o[1] = fmaf(f, x.y, o[1]);
        o[2] = fmaf(f, x.z, o[2]);
        o[3] = fmaf(f, x.w, o[3]);
      }
      if (P.splits == 1) {
        store_out(P.out + (row0 + r0 + rr) * D + d, o, 1.0f / l);
        if (P.lse && d == 0)
          P.lse[row0 + r0 + rr] = (ref + __log2f(l)) * kLn2;
      } else {
        float *to = P.part +
                    (((p - P.p0) * hkv + g) * P.splits + split) * P.n_rep *
                        (int64_t)(D + 2) +
                    (int64_t)(r0 + rr) * (D + 2);
        // (rows of D + 2: two 8-byte halves)
        *reinterpret_cast<float2 *>(to + d) = make_float2(o[0], o[1]);
        *reinterpret_cast<float2 *>(to + d + 2) = make_float2(o[2], o[3]);
        if (d == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(M, l);
      }
    }
    // (the next tile writes where this one was read)
    if constexpr (WU == 1)
      wave_fence();
    else
      __syncthreads();
  }
}

// The sums of a row's blocks, rows (pair, q head).
template <int D, int PARTS>
__global__ __launch_bounds__(join_threads(D, PARTS)) void k_token_join(
    TokenParams P) {
  const unsigned at =
      PARTS > 1 ? blockIdx.x
                : blockIdx.x * join_rows(D, 1) + threadIdx.x / (D / 2);
  const int64_t p = P.p0 + at / P.Hq;
  if (p >= P.n_pairs) return;
  const int h = at % P.Hq, g = h / P.n_rep, rr = h - g * P.n_rep;
  int64_t tok;
  if (!one_token(P, p, tok) || !has_document(P, P.doc_ids[p])) return;
  const int64_t step = (int64_t)P.n_rep * (D + 2), row = tok * P.Hq + h;
  join_row<D, PARTS>(
      P.part + ((p - P.p0) * P.sv.n_kv_heads + g) * P.splits * step +
          (int64_t)rr * (D + 2),
      step, P.splits, P.out + row * D, P.lse ? P.lse + row : nullptr);
}

// How a call's (pair, kv head)s are shared out: one wave each from kTokenFull
// of them on (two waves a SIMD), two or four below, and past 32 chunks several
// blocks of four where that leaves waves free, of at least two chunks a wave of
// the longest document and within 32 MB of sums (half of the no-alloc call's
// scratch).  (One pair of 32 q / 8 kv heads: 512 slots 8.9 us, in two blocks
// 11.4; 1,024 10.7 and 11.4; 2,048 14.4, in eight 11.1; 16,384 13.3 in 32.)
constexpr int64_t kTokenFull = 2048;
struct TokenShare {
  int waves, splits;
};
TokenShare token_share(const dopr_store &st, int64_t pairs, int32_t n_rep) {
  const int64_t units = pairs * st.n_kv_heads;
  const int64_t chunks = ((int64_t)st.max_len + KC - 1) / KC;
  if (2 * units > kTokenFull) return {1, 1};
  if (4 * units > kTokenFull) return {2, 1};
  if (chunks <= 32) return {kTokenWaves, 1};
  const int64_t want = kTokenFull / (units * kTokenWaves);
  const int64_t most = chunks / (2 * kTokenWaves);
  const int64_t fit = ((int64_t)32 << 20) /
                      (4 * units * n_rep * (int64_t)(st.head_dim + 2));
  return {kTokenWaves,
          (int)std::max<int64_t>(1, std::min({want, most, fit}))};
}

template <int D>
void launch_token2(int waves, const TokenParams &P, hipStream_t s) {
  const auto kernel = waves == 1   ? k_token_fp4<D, 1>
                      : waves == 2 ? k_token_fp4<D, 2>
                                   : k_token_fp4<D, 4>;
  hipLaunchKernelGGL(kernel, dim3(P.units), dim3(64 * waves), 0, s, P);
}

template <int D>
hipError_t launch_token1(const TokenParams &P, int waves, int64_t pairs,
                         hipStream_t s) {
  const int64_t hkv = P.sv.n_kv_heads;
  return in_slices(
      pairs, a_launch(std::max<int64_t>(64 * waves * hkv * P.splits,
                                        P.splits > 1 ? 4 * D * P.Hq : 1)),
      [&](int64_t at, int64_t n) {
        TokenParams S = P;
        S.p0 = P.p0 + at;
        S.units = (uint32_t)(n * hkv * P.splits);
        launch_token2<D>(waves, S, s);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || P.splits == 1) return e;
        const int parts = join_parts(P.splits), rows = join_rows(D, parts);
        const auto join =
            parts > 1 ? k_token_join<D, kJoinParts> : k_token_join<D, 1>;
        hipLaunchKernelGGL(join, dim3((unsigned)((n * P.Hq + rows - 1) / rows)),
                           dim3(join_threads(D, parts)), 0, s, S);
        return hipGetLastError();
      });
}

}  // namespace

size_t token_bytes(const dopr_store &st, int64_t pairs, int32_t n_rep) {
  const int64_t splits = token_share(st, pairs, n_rep).splits;
  return splits == 1 ? 0
                     : sizeof(float) * (size_t)(pairs * st.n_kv_heads) *
                           splits * n_rep * (st.head_dim + 2);
}

hipError_t launch_token(const AttnCall &c, void *workspace, hipStream_t s) {
  const dopr_attn_args_t *a = c.a;
  const dopr_store &st = *c.st;
  TokenParams P{};
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
  P.part = static_cast<float *>(workspace);
  P.log_theta = std::log((double)a->rope_theta);
  P.n_pairs = a->n_pairs;
  P.total_tokens = a->total_tokens;
  P.eps = a->rms_eps;
  P.c = a->softmax_scale * 1.4426950408889634f;
  P.Hq = a->n_q_heads;
  P.n_rep = c.n_rep;
  P.layer = c.layer;
  const TokenShare share = token_share(st, a->n_pairs, c.n_rep);
  P.splits = share.splits;
  hipError_t e = hipSuccess;
  if (a->timing_begin)
    e = hipEventRecord(static_cast<hipEvent_t>(a->timing_begin), s);
  if (e == hipSuccess)
    e = st.head_dim == 128 ? launch_token1<128>(P, share.waves, a->n_pairs, s)
                           : launch_token1<64>(P, share.waves, a->n_pairs, s);
  if (e == hipSuccess && a->timing_end)
    e = hipEventRecord(static_cast<hipEvent_t>(a->timing_end), s);
  return e;
}

}  // namespace dopr
