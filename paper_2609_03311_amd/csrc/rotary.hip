// rotary.hip -- rotary positions of query and key heads (k_rotary), with the
// heads' RMSNorm in front.
//
// Pair i of a head (elements (i, i + R/2), or (2i, 2i+1) where the layout is
// interleaved) turns by position * inv_freq[i]; elements from R on pass
// through.  A wave takes one token: its lanes form the token's R/2 rotations
// once, then every head uses them.  A lane holds 8 pairs (16 elements) of a
// head, so a rotation never leaves the lane, in-place calls are safe, and a
// head's sum of squares is a butterfly over the 1 to 64 lanes of that head.
// Bound by HBM: each head is read and written once (32,768 tokens, 40 heads of
// 128 in bf16: 115 us, 5.8 TB/s, with the norm 118, interleaved 120; half of
// each head interleaved, out of a fused q, k, v buffer, 120).
//
// The angle's whole turns are dropped in 64 bits (four operations per pair
// and token): in 32 bits the product of a position and a frequency is off by
// up to 2^-25 of itself, at position 2^17 0.004 rad, more than a bf16
// rounding.  Normed fp32 heads are turned in 64 bits too (244 us for the above,
// 5.5 TB/s).
#include <type_traits>

#include "rowio.hpp"

namespace dopr {
namespace {

constexpr int kRotaryWaves = 4;
constexpr int kRotaryBatch = 4;  // head groups whose loads are in flight

struct RotaryHeads {
  const void *x;
  void *out;
  const void *norm_w;
  int64_t row, head, out_row, out_head;  // strides in elements
};

struct RotaryParams {
  RotaryHeads q, k;
  const int32_t *positions;
  const float *inv_freq;
  int64_t items;             // tokens * splits
  int32_t n_q, n_heads;      // query heads, all heads
  int32_t D, R;
  int32_t group_log2;        // lanes per head
  int32_t pair_units, units; // 16-element units of a head: rotated (where
                             // they lie apart), all
  int32_t splits;            // waves that share a token's heads
  float factor, sign, eps;
  bool whole;    // every lane's elements are its own
  bool stream;   // stores past the caches' order of use
};

// A unit's two runs of 8 elements, of which [lo, n) are its own (lo = 8: none).
// The units' first runs lie side by side, and so do their second ones: a wave
// loads and stores whole lines.
struct Unit {
  int pa, pb, lo_a, lo_b, n_a, n_b;
  bool rotated;        // some of its elements turn
  int pair_a, pair_b;  // first pairs: of the first four of the unit's 8 and of
                       // the others
};

// SMALL: runs are cut at their part's end (element loads); else the last run
// of a part moves back to end with it and keeps its own tail.  Rotate-half
// layouts deal out the rotated part (pairs of runs R / 2 apart) and the rest of
// a head apart; interleaved ones, whose pairs lie inside a run, the whole head.
template <bool INTER, bool SMALL>
__device__ __forceinline__ Unit unit_of(int u, int pair_units, int D, int R) {
  Unit k;
  k.n_a = k.n_b = 8;
  k.lo_a = k.lo_b = 0;
  k.rotated = u < pair_units;
  if (k.rotated && !INTER) {
    const int half = R / 2;
    int i0 = 8 * u;
    if (SMALL) {
      k.n_a = k.n_b = min(8, half - i0);
    } else if (i0 + 8 > half) {
      k.lo_a = k.lo_b = i0 + 8 - half;
      i0 = half - 8;
    }
    k.pa = i0;
    k.pb = i0 + half;
    k.pair_a = i0;
    k.pair_b = i0 + 4;
    return k;
  }
  // runs of 8 elements of [from, D): unit j takes the runs j and j + units
  const int from = INTER ? 0 : R;
  const int j = INTER ? u : u - pair_units;
  const int runs = (D - from + 7) / 8, units = (runs + 1) / 2;
  auto run = [&](int r, int &p, int &lo, int &n) {
    p = from + 8 * r;
    if (r >= runs) {  // an odd number of runs: no second one here
      p = from;
      lo = 8;
      n = SMALL ? 0 : 8;
    } else if (SMALL) {
      n = min(8, D - p);
    } else if (p + 8 > D) {
      lo = p + 8 - D;
      p = D - 8;
    }
    // (a run past the end starts in front of D; D < 8 only in SMALL, which
    // cuts it)
  };
  run(j, k.pa, k.lo_a, k.n_a);
  run(j + units, k.pb, k.lo_b, k.n_b);
  if (!SMALL && k.lo_b == 8) k.pb = k.pa;  // (any run of this head)
  k.pair_a = k.pa / 2;
  k.pair_b = k.pb / 2;
  k.rotated = INTER && k.pa < R;
  return k;
}

// A run of 8 elements; SMALL reads and writes elements [lo, n) one by one.
template <typename T, bool SMALL>
struct Run {
  Raw8<T> raw;
  float f[SMALL ? 8 : 1];
  __device__ __forceinline__ void load(const T *p, int n) {
    if constexpr (SMALL) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e < n ? to_f32<T>(p[e]) : 0.f;
    } else {
      raw.load(p);
    }
  }
  __device__ __forceinline__ void get(float *g) const {
    if constexpr (SMALL) {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = f[e];
    } else {
      raw.get(g);
    }
  }
  static __device__ __forceinline__ void store(T *p, int lo, int n,
                                               const float *g, bool stream) {
    if constexpr (SMALL) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = from_f32<T>(g[e]);
    } else {
      if (stream)
        store_part<T, 8, true>(p, lo, 8, g);
      else
        store_part<T, 8>(p, lo, 8, g);
    }
  }
};

// What a run's values are held in behind its load: wide, or f itself.
template <typename V>
__device__ __forceinline__ auto &values(V (&wide)[8], float (&f)[8]) {
  if constexpr (std::is_same_v<V, float>)
    return f;
  else
    return wide;
}

template <typename T, bool INTER, bool SMALL, bool NORM>
__global__ __launch_bounds__(64 * kRotaryWaves, 3) void k_rotary(RotaryParams P) {
  // fp32 heads are normed and turned in 64 bits, so that what is rounded in
  // between does not show next to the output's own rounding (subnormals too)
  using Value = std::conditional_t<NORM && sizeof(T) == 4, double, float>;
  __shared__ float2 table[kRotaryWaves][256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t item = (int64_t)blockIdx.x * kRotaryWaves + wave;
  if (item >= P.items) return;  // no block barrier below
  const int64_t tok = item / P.splits;
  const int split = (int)(item - tok * P.splits);
  const int per_wave = 64 >> P.group_log2;
  const int sub = lane >> P.group_log2;          // head of a group
  const int u_raw = lane & ((1 << P.group_log2) - 1);
  const int u = min(u_raw, P.units - 1);
  const Unit k = unit_of<INTER, SMALL>(u, P.pair_units, P.D, P.R);
  const int step = per_wave * P.splits;

  // the token's rotations, times the factor
  const double pos = (double)P.positions[tok];
  for (int i = lane; i < P.R / 2; i += 64) {
    const double turns =
        pos * (double)P.inv_freq[i] * 0.15915494309189533577;
    const float r = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.f * r, &s, &c);
    table[wave][i] = make_float2(c * P.factor, s * P.factor * P.sign);
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  float c[8], s[8];
  uint32_t turns = 0;  // pairs that turn
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // (pairs behind a part's end belong to no element, or to none that turns)
    const int i = e < 4 ? k.pair_a + e : k.pair_b + e - 4;
    const bool in = k.rotated && i < P.R / 2;
    const float2 t = table[wave][in ? i : 0];
    c[e] = t.x;
    s[e] = t.y;
    turns |= in ? 1u << e : 0u;
  }

  // the token's heads, as if they all were q's or k's
  const T *q_in = static_cast<const T *>(P.q.x) + tok * P.q.row;
  const T *k_in = static_cast<const T *>(P.k.x) + tok * P.k.row -
                  P.n_q * P.k.head;
  T *q_out = static_cast<T *>(P.q.out) + tok * P.q.out_row;
  T *k_out = static_cast<T *>(P.k.out) + tok * P.k.out_row -
             P.n_q * P.k.out_head;

  for (int h0 = split * per_wave; h0 < P.n_heads; h0 += step * kRotaryBatch) {
    Run<T, SMALL> ra[kRotaryBatch], rb[kRotaryBatch];
#pragma unroll
    for (int b = 0; b < kRotaryBatch; ++b) {
      const int h = min(h0 + b * step + sub, P.n_heads - 1);
      const bool is_k = h >= P.n_q;
      const T *x = (is_k ? k_in : q_in) + h * (is_k ? P.k.head : P.q.head);
      ra[b].load(x + k.pa, k.n_a);
      rb[b].load(x + k.pb, k.n_b);
    }
#pragma unroll
    for (int b = 0; b < kRotaryBatch; ++b) {
      const int hr = h0 + b * step + sub;
      if (h0 + b * step >= P.n_heads) break;
      const int h = min(hr, P.n_heads - 1);
      const bool is_k = h >= P.n_q;
      float fa[8], fb[8];
      ra[b].get(fa);
      rb[b].get(fb);
      Value wide_a[8], wide_b[8];
      auto &va = values(wide_a, fa);
      auto &vb = values(wide_b, fb);
      if constexpr (NORM) {
        auto mean_square = [&]() {
          float ss = 0.f;
          if (P.whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              ss = fmaf(fa[e], fa[e], fmaf(fb[e], fb[e], ss));
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float a = e >= k.lo_a && u == u_raw ? fa[e] : 0.f;
              const float b2 = e >= k.lo_b && u == u_raw ? fb[e] : 0.f;
              ss = fmaf(a, a, fmaf(b2, b2, ss));
            }
          }
          for (int off = (1 << P.group_log2) >> 1; off > 0; off >>= 1)
            ss += __shfl_xor(ss, off, 64);
          return ss / (float)P.D;
        };
        float mean = mean_square(), eps = P.eps;
        const bool large = mean == __builtin_inff();
        const bool small = mean + eps < 0x1p-100f;
        const T *w = static_cast<const T *>(is_k ? P.k.norm_w : P.q.norm_w);
        if (__any(w && (large || small))) {
          // squares out of fp32's range (values over 2^59 or so, or, with next
          // to no epsilon, all under 2^-45): the same with those heads 2^80
          // times smaller, or 2^100 times larger
          const float by =
              !w ? 1.f : large ? 0x1p-80f : small ? 0x1p100f : 1.f;
          eps = eps * by * by;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            fa[e] *= by;
            fb[e] *= by;
          }
          mean = mean_square();
        }
        // 16-bit outputs: the hardware's 1 / sqrt, off by a unit of fp32's last
        // place, 2^-15 of theirs (no subnormals come here, which it takes for 0)
        const float inv = sizeof(T) == 2 ? __builtin_amdgcn_rsqf(mean + eps)
                                         : 1.0f / sqrtf(mean + eps);
        if constexpr (sizeof(Value) == 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            va[e] = fa[e];
            vb[e] = fb[e];
          }
        }
        if (w) {
          Run<T, SMALL> wa, wb;
          wa.load(w + k.pa, k.n_a);
          wb.load(w + k.pb, k.n_b);
          float ga[8], gb[8];
          wa.get(ga);
          wb.get(gb);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            va[e] = (Value)fa[e] * inv * ga[e];
            vb[e] = (Value)fb[e] * inv * gb[e];
          }
        }
      }
      if (k.rotated) {
        Value a[8], b2[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          a[e] = INTER ? (e < 4 ? va[2 * e] : vb[2 * e - 8]) : va[e];
          b2[e] = INTER ? (e < 4 ? va[2 * e + 1] : vb[2 * e - 7]) : vb[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // (selected, not turned by zero: 0 times an infinity is NaN)
          const bool in = !INTER || (turns >> e & 1);
          const Value x0 = in ? a[e] * c[e] - b2[e] * s[e] : a[e];
          const Value x1 = in ? b2[e] * c[e] + a[e] * s[e] : b2[e];
          if (INTER) {
            (e < 4 ? va[2 * e] : vb[2 * e - 8]) = x0;
            (e < 4 ? va[2 * e + 1] : vb[2 * e - 7]) = x1;
          } else {
            va[e] = x0;
            vb[e] = x1;
          }
        }
      }
      if constexpr (sizeof(Value) == 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          fa[e] = (float)va[e];
          fb[e] = (float)vb[e];
        }
      }
      if (hr < P.n_heads && u == u_raw) {
        T *o = (is_k ? k_out : q_out) +
               h * (is_k ? P.k.out_head : P.q.out_head);
        Run<T, SMALL>::store(o + k.pa, k.lo_a, k.n_a, fa, P.stream);
        Run<T, SMALL>::store(o + k.pb, k.lo_b, k.n_b, fb, P.stream);
      }
    }
  }
}

template <typename T, bool INTER, bool SMALL>
void launch1(const RotaryParams &P, hipStream_t s) {
  const dim3 grid((unsigned)((P.items + kRotaryWaves - 1) / kRotaryWaves));
  const dim3 block(64 * kRotaryWaves);
  if (P.q.norm_w || P.k.norm_w)
    hipLaunchKernelGGL((k_rotary<T, INTER, SMALL, true>), grid, block, 0, s, P);
  else
    hipLaunchKernelGGL((k_rotary<T, INTER, SMALL, false>), grid, block, 0, s,
                       P);
}

template <typename T>
hipError_t launch(const RotaryParams &P, int64_t tokens, bool inter, bool small,
                  hipStream_t s) {
  auto from = [](const RotaryHeads &h, int64_t token) {
    RotaryHeads f = h;
    f.x = ahead(h.x, token * h.row * (int)sizeof(T));
    f.out = ahead(h.out, token * h.out_row * (int)sizeof(T));
    return f;
  };
  // (many tokens: one wave each)
  return in_slices(tokens, a_launch(64 * P.splits), [&](int64_t t, int64_t n) {
    RotaryParams S = P;
    S.q = from(P.q, t);
    S.k = from(P.k, t);
    S.positions = P.positions + t;
    S.items = n * P.splits;
    if (inter)
      small ? launch1<T, true, true>(S, s) : launch1<T, true, false>(S, s);
    else
      small ? launch1<T, false, true>(S, s) : launch1<T, false, false>(S, s);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_rotary(const dopr_rotary_args_t &a, hipStream_t s) {
  RotaryParams P{};
  P.q = {a.q, a.q_out, a.q_norm_w, a.q_row_stride, a.q_head_stride,
         a.q_out_row_stride, a.q_out_head_stride};
  P.k = {a.k, a.k_out, a.k_norm_w, a.k_row_stride, a.k_head_stride,
         a.k_out_row_stride, a.k_out_head_stride};
  P.positions = a.positions;
  P.inv_freq = a.inv_freq;
  P.n_q = a.n_q_heads;
  P.n_heads = a.n_q_heads + a.n_kv_heads;
  P.D = a.head_dim;
  P.R = a.rotary_dim;
  P.pair_units = (a.rotary_dim / 2 + 7) / 8;
  P.units = a.interleaved
                ? (a.head_dim + 15) / 16
                : P.pair_units + (a.head_dim - a.rotary_dim + 15) / 16;
  while ((1 << P.group_log2) < P.units) ++P.group_log2;
  P.factor = a.attention_factor;
  P.sign = a.inverse ? -1.f : 1.f;
  P.eps = a.rms_eps;
  P.whole = (a.interleaved || a.rotary_dim % 16 == 0) &&
            (a.interleaved || (a.head_dim - a.rotary_dim) % 16 == 0) &&
            a.head_dim % 16 == 0 && P.units == 1 << P.group_log2;
  // Streamed where every store of a wave fills lines (32,768 tokens, 40 heads
  // of 128: 118 us, else 125); in rotate-half layouts of part of a head, two
  // stores fill one (half of each head turned: 138 us streamed, else 130).
  P.stream = a.interleaved || a.rotary_dim == a.head_dim;
  // (runs of 8 elements that end with their part have to fit in it, or, those
  // behind the rotated part, in the head; a run that moves back to end with an
  // odd head would split its pairs)
  const bool small = a.interleaved ? a.head_dim < 8 || a.head_dim % 2
                                   : a.rotary_dim < 16;
  // few tokens: a token's head groups go to several waves (each forms the
  // rotations again) until about eight waves a SIMD are there
  const int groups = (P.n_heads + (64 >> P.group_log2) - 1) /
                     (64 >> P.group_log2);
  P.splits = 1;
  while (P.splits < groups && a.rows * P.splits < 8192) P.splits *= 2;
  if (P.splits > groups) P.splits = groups;
  if (a.dtype == DOPR_BF16)
    return launch<bf16_t>(P, a.rows, a.interleaved, small, s);
  if (a.dtype == DOPR_F16)
    return launch<_Float16>(P, a.rows, a.interleaved, small, s);
  return launch<float>(P, a.rows, a.interleaved, small, s);
}

}  // namespace dopr
