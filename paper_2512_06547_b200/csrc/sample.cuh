// What the sampling kernels share: weights of tokens in more than 32 bits, and the edges of a row of logits.
//
//   w(l) = exp((l - m) / t),  m the largest logit,  t the temperature
//
// A random number (or a share of the mass) is compared with running sums of weights, and the token has to be the one that
// exact sums give, whatever order they are added in.  Sums of fp32 exponentials (2^-23 each) would move a border between two
// tokens of a flat row of 150,000 by a tenth of a token; fp64 exponentials take the time of several passes over the logits.  So:
// with d = l - m and e its rounding error (both fp32; two-sum of Knuth) and y = (d + e) log2(e) / t, the sum of d log2(e) / t and
// 1.5 2^16 rounds y to k + j / 128, two fused products leave f = y - k - j / 128 with |f| <= 2^-8 exact to 2^-32, and
//   w = 2^k T[j] (1 + p),  T[j] = 2^(j / 128) in 64 bits,  p = 2^f - 1 from the first three terms of its series.
// The error is that of f and p: half a step of fp32 numbers of at most 0.004, below 2^-31 of w (and for bf16 logits that of d, see
// exact_diff below).  d = 0 gives 1 exactly.  Sums
// take T in 64 bits and T p, 400 times smaller, in 32, so that no value is converted between the two types, and the fp32 part
// runs on pairs: 14 (bf16) to 17 instructions per logit, of which one is a 64-bit one (39 without the pairs, with checks for what
// a warp's logits do not hold, and with conflicts on a table that is not there once per lane of a half-warp).
#pragma once

#include <cfloat>
#include <climits>
#include <initializer_list>

#include "a3po_common.cuh"

namespace a3po {
namespace {

constexpr int kPowSteps = 128;
struct PowTable {
  double t[kPowSteps];
};
constexpr double root_of(double x) {   // Newton's iteration from above
  double r = x;
  for (int i = 0; i < 60; ++i) r = 0.5 * (r + x / r);
  return r;
}
constexpr PowTable make_pow_table() {   // T[j]: product of the roots 2^(1/2), 2^(1/4), ... that the bits of j name
  PowTable p{};
  for (int j = 0; j < kPowSteps; ++j) {
    double v = 1.0, r = 2.0;
    for (int bit = kPowSteps / 2; bit > 0; bit /= 2) {
      r = root_of(r);
      if (j & bit) v *= r;
    }
    p.t[j] = v;
  }
  return p;
}
__device__ const PowTable kPow2 = make_pow_table();

// In shared memory the table is there once for each lane of a half-warp (the lanes whose 64-bit accesses go out together).
// An entry is T[j] 2^-64, so that the upper 32 bits of its fp32 form are two shifted words (below), with what the bits of the
// rounded sum add to its upper word taken off beforehand.
template <int COPIES> struct SharedTable;   // COPIES: 16, or 1 where few weights are taken
constexpr uint32_t kRoundBits = 0x47c00000u;   // 98304.f = 1.5 2^16, whose last bit is 2^-7
constexpr float kRound = 98304.f;
template <int COPIES> struct SharedTable {
  uint2 e[kPowSteps * COPIES];
};
template <int COPIES>
__device__ __forceinline__ void fill_table(SharedTable<COPIES>& t, int thread, int threads) {
  for (int i = thread; i < kPowSteps * COPIES; i += threads) {
    const int j = i / COPIES;
    const double v = kPow2.t[j] * 0x1p-64;
    t.e[i] = make_uint2(static_cast<uint32_t>(__double2loint(v)),
                        static_cast<uint32_t>(__double2hiint(v)) - ((kRoundBits + static_cast<uint32_t>(j)) << 13));
  }
}

struct F2 {
  unsigned long long u;
};
__device__ __forceinline__ F2 f2(float x, float y) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.u) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 both(F2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.u));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}

// A sum of weights: high 2^64 - low 2^-64.
struct WeightSum {
  double high = 0.0;
  F2 low = {0ull};
  __device__ __forceinline__ double value() const {
    const float2 l = both(low);
    return fma(-(static_cast<double>(l.x) + static_cast<double>(l.y)), 0x1p-64, high * 0x1p64);
  }
};

constexpr float kA = 0.693147180559945f, kB = 0.240226506959101f, kC = 0.0555041086648216f;   // ln 2^n / n!

template <int COPIES>
struct Weights {
  float max, c_hi, c_lo;   // c = log2(e) / t
  float floor;             // differences below count as this one (w = 2^-100): what is that small adds nothing to a sum that holds a 1
  float zero;              // differences below have weight 0, as exp in 64 bits has
  bool at_inf;             // the largest logit is infinite: it alone has weight
  const uint2* table;      // this lane's copy

  __device__ __forceinline__ void set_max(float row_max) {
    max = row_max;
    at_inf = row_max == INFINITY;
  }
  __device__ __forceinline__ void set_temperature(float temperature, const SharedTable<COPIES>& t) {
    table = t.e + threadIdx.x % COPIES;
    const double c = fmin(1.4426950408889634 / static_cast<double>(temperature), 1e37);
    c_hi = static_cast<float>(c);
    c_lo = static_cast<float>(c - static_cast<double>(c_hi));
    floor = static_cast<float>(-100.0 / c);
    zero = fmaxf(static_cast<float>(-745.13321910194122 * static_cast<double>(temperature)), -FLT_MAX);
  }
  // 2^(k - 64) T[j] for the bits of a rounded sum, and -2^(k + 64) T[j] cut to 32 bits: the exponent field of the former, 959 + k, has
  // lost its upper two bits there, and its third is the sign.
  __device__ __forceinline__ void entry(float s, double& t64, float& t32) const {
    const uint32_t bits = __float_as_uint(s);
    const uint2 e = table[(bits & (kPowSteps - 1)) * COPIES];
    const uint32_t hi = e.y + (bits << 13);
    t64 = __hiloint2double(static_cast<int>(hi), static_cast<int>(e.x));
    t32 = __uint_as_float(__funnelshift_l(e.x, hi, 3));
  }
  // Two logits whose differences lie between floor and 0.
  template <bool EXACT_DIFF>
  __device__ __forceinline__ void add(F2 l, WeightSum& sum) const {
    // a - b as fma(b, -1, a), rounded once as the difference is: a pair has no sign to turn
    const F2 minus = f2(-1.f, -1.f), round = f2(kRound, kRound);
    const F2 d = add2(l, f2(-max, -max)), c = f2(c_hi, c_hi);
    const F2 s = fma2(d, c, round);
    F2 f = fma2(d, f2(c_lo, c_lo), fma2(d, c, fma2(s, minus, round)));
    if (!EXACT_DIFF) {
      const F2 back = fma2(l, minus, d);
      const F2 e = fma2(add2(f2(max, max), back), minus, fma2(fma2(back, minus, d), minus, l));
      f = fma2(e, c, f);
    }
    const F2 q = fma2(f, fma2(f, f2(kC, kC), f2(kB, kB)), f2(kA, kA));
    const float2 s2 = both(s);
    double ta, tb;
    float a, b;
    entry(s2.x, ta, a);
    entry(s2.y, tb, b);
    sum.high += ta;
    sum.high += tb;
    sum.low = fma2(mul2(f, f2(a, b)), q, sum.low);
  }
  static __device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
  }
  // Any logit.
  template <bool EXACT_DIFF>
  __device__ __forceinline__ double operator()(float l) const {
    float d = __fsub_rn(l, max), e = 0.f;
    if (!EXACT_DIFF) {
      const float back = __fsub_rn(d, l);
      e = __fsub_rn(__fsub_rn(l, __fsub_rn(d, back)), __fadd_rn(max, back));
    }
    if (at_inf) d = l == max ? 0.f : -INFINITY;
    if (!(d >= zero)) return 0.0;   // NaN too
    if (d < floor) {
      d = floor;
      e = 0.f;
    }
    const float s = fmaf(d, c_hi, kRound);
    float f = fmaf(d, c_lo, fmaf(d, c_hi, __fsub_rn(kRound, s)));
    if (!EXACT_DIFF && !at_inf) f = fmaf(e, c_hi, f);
    const float p = f * fmaf(f, fmaf(f, kC, kB), kA);
    double t64;
    float t32;
    entry(s, t64, t32);
    t64 *= 0x1p64;
    return fma(t64, static_cast<double>(p), t64);
  }
};

// The difference of two bf16 numbers is an fp32 number unless one is about 2^15 times smaller than the other, a logit that is close
// to 0 beside the largest; the rounding, 2^-24 of the difference and so 2^-24 |l - m| / t of the weight, is left in (with it the
// fp32 form's three instructions a logit more, 14 to 17).
template <typename T> constexpr bool exact_diff() { return sizeof(T) == 2; }

// Logits are read 16 bytes at a time from the 16-byte boundary at or below the row's (or slice's) first element on: `head`
// elements before it, and what is past its end, count as -inf and are not read.
template <typename T> constexpr int per_vec() { return 16 / static_cast<int>(sizeof(T)); }
template <typename T>
__device__ __forceinline__ int head_of(const T* row) {
  return static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
}
template <typename T> struct Vec {
  uint32_t w[4];
  __device__ __forceinline__ float at(int e) const {
    if (sizeof(T) == 4) return __uint_as_float(w[e]);
    return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  __device__ __forceinline__ F2 pair(int e) const { return f2(at(e), at(e + 1)); }   // e even
};
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float min3_nan(float a, float b, float c) {
  float d;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// The largest (NaN passed over) and the smallest (NaN if there is one) of N vectors' logits.
template <typename T, int N>
__device__ __forceinline__ void extremes(const Vec<T> (&v)[N], float& most, float& least) {
  if constexpr (sizeof(T) == 4) {
    most = v[0].at(0);
    least = v[0].at(0);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        most = max3(most, v[i].at(e), v[i].at(e + 1));
        least = min3_nan(least, v[i].at(e), v[i].at(e + 1));
      }
  } else {
    uint32_t hi = v[0].w[0], lo = v[0].w[0];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        asm("max.bf16x2 %0, %0, %1;" : "+r"(hi) : "r"(v[i].w[e]));
        asm("min.NaN.bf16x2 %0, %0, %1;" : "+r"(lo) : "r"(v[i].w[e]));
      }
    const float a = __uint_as_float(hi << 16), b = __uint_as_float(hi & 0xffff0000u);
    const float c = __uint_as_float(lo << 16), d = __uint_as_float(lo & 0xffff0000u);
    most = fmaxf(a, b);
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(least) : "f"(c), "f"(d));
  }
}
__device__ __forceinline__ float warp_max_any(float v) {   // NaN only if all are
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// Elements first .. first + per_vec - 1 of a row of n (first may be negative).
template <typename T>
__device__ __forceinline__ Vec<T> load_vec(const T* row, int first, int n) {
  Vec<T> v;
  if (first >= 0 && first + per_vec<T>() <= n) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(row + first));
    v.w[0] = u.x; v.w[1] = u.y; v.w[2] = u.z; v.w[3] = u.w;
    return v;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      v.w[i] = first + i >= 0 && first + i < n ? __float_as_uint(to_float(row[first + i])) : 0xff800000u;
    } else {
      uint32_t half[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = first + i * 2 + e;
        half[e] = at >= 0 && at < n ? __float_as_uint(to_float(row[at])) >> 16 : 0xff80u;
      }
      v.w[i] = half[0] | half[1] << 16;
    }
  }
  return v;
}

struct SampleArgs {
  const void* logits;
  long long ld;
  const uint8_t* row_mask;
  int n, v;
  const float* temperature;
  const int* top_k;
  const float *top_p, *min_p;
  const float* u;
  int* token;
  float *logp, *kept_logp;
  int* n_kept;

  __device__ __forceinline__ void put(int row, int tok, double lp, double klp, int kept) const {
    token[row] = tok;
    if (logp) logp[row] = static_cast<float>(lp);
    if (kept_logp) kept_logp[row] = static_cast<float>(klp);
    if (n_kept) n_kept[row] = kept;
  }
  // Temperature of a row; 1 where it is greedy.  An infinite one would make 0 times infinity of an infinite logit and of min-p = 1.
  __device__ __forceinline__ float temp(int row, bool& greedy) const {
    const float t = temperature ? temperature[row] : 1.f;
    greedy = !(t > 0.f);
    return greedy ? 1.f : fminf(t, 1e30f);
  }
};

}  // namespace

// Rows without a filter (sample_stream.cu): workspace, and the two launches.
size_t sample_stream_bytes(long long n, int v);
int sample_stream(const void* args, a3po_dtype dt, void* ws, cudaStream_t stream);
// Rows with filters (sample_filter.cu): a row stays in the shared memory of a cluster of blocks.  sample_in_one: short and few ones
// without filters go there too.
bool sample_in_one(long long n, int v);
long long sample_filter_max_v(a3po_dtype dt);
int sample_filter(const void* args, a3po_dtype dt, cudaStream_t stream);

}  // namespace a3po
