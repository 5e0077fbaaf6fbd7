// What the sampling kernels share: weights of tokens in more than 32 bits, and the edges of a row of logits.
//
//   w(l) = exp((l - m) / t),  m the largest logit,  t the temperature
//
// A random number (or a share of the mass) is compared with running sums of weights, and the token has to be the one that
// exact sums give, whatever order they are added in.  Sums of fp32 exponentials (2^-23 each) would move a border between two
// tokens of a flat row of 150,000 by a tenth of a token; fp64 exponentials take the time of several passes over the logits.  So:
// with d = l - m and e its rounding error (both fp32; two-sum of Knuth), y = (d + e) log2(e) / t as an unevaluated pair of
// fp32 numbers, y = k + j / 128 + f with |f| <= 2^-8, and
//   w = 2^k T[j] (1 + p),  T[j] = 2^(j / 128) in 64 bits,  p = 2^f - 1 from the first three terms of its series.
// The error is that of p: half a step of an fp32 number of at most 0.0027, below 2^-32 of w.  d = 0 gives 1 exactly.  Sums take
// T in 64 bits and T p, 400 times smaller, in 32, so that no value is converted between the two types: per element 20
// (bf16) to 26 instructions, of which one is a 64-bit one.
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

struct Weights {
  float max, c_hi, c_lo;   // c = log2(e) / t
  float floor;             // differences below count as this one (w = 2^-100): what is that small adds nothing to a sum that holds a 1
  float zero;              // differences below have weight 0, as exp in 64 bits has
  bool at_inf;             // the largest logit is infinite: it alone has weight

  __device__ __forceinline__ void set(float row_max, float temperature) {
    max = row_max;
    at_inf = row_max == INFINITY;
    const double c = fmin(1.4426950408889634 / static_cast<double>(temperature), 1e37);
    c_hi = static_cast<float>(c);
    c_lo = static_cast<float>(c - static_cast<double>(c_hi));
    floor = static_cast<float>(-100.0 / c);
    zero = fmaxf(static_cast<float>(-745.13321910194122 * static_cast<double>(temperature)), -FLT_MAX);
  }
  // hi, lo: 2^k T[j], f32 the same rounded down to 32 bits; p as above.  False: the weight is 0.
  template <bool EXACT_DIFF>
  __device__ __forceinline__ bool parts(float l, const double* table, double& t64, float& t32, float& p) const {
    float d = __fsub_rn(l, max), e = 0.f;
    if (!EXACT_DIFF) {
      const float back = __fsub_rn(d, l);
      e = __fsub_rn(__fsub_rn(l, __fsub_rn(d, back)), __fadd_rn(max, back));
    }
    if (at_inf) d = l == max ? 0.f : -INFINITY;
    const bool some = d >= zero;   // false for NaN
    d = fmaxf(d, floor);
    const float y = __fmul_rn(d, c_hi);
    float y_lo = fmaf(d, c_lo, fmaf(d, c_hi, -y));
    if (!EXACT_DIFF && !at_inf) y_lo = fmaf(e, c_hi, y_lo);
    constexpr float kRound = 98304.f;   // 1.5 2^16: the sum's last bit is 2^-7
    const float s = __fadd_rn(y, kRound);
    const float f = __fadd_rn(__fsub_rn(y, __fsub_rn(s, kRound)), y_lo);
    const int i = __float_as_int(s) - 0x47c00000;   // 128 k + j
    constexpr float kA = 0.693147180559945f, kB = 0.240226506959101f, kC = 0.0555041086648216f;   // ln 2^n / n!
    p = f * fmaf(f, fmaf(f, kC, kB), kA);
    const double t = table[i & (kPowSteps - 1)];
    const int hi = __double2hiint(t) + ((i >> 7) << 20), lo = __double2loint(t);
    t64 = __hiloint2double(hi, lo);
    t32 = __int_as_float(static_cast<int>(__funnelshift_l(lo, hi - 0x38000000, 3)));
    return some;
  }
  template <bool EXACT_DIFF>
  __device__ __forceinline__ double operator()(float l, const double* table) const {
    double t64;
    float t32, p;
    const bool some = parts<EXACT_DIFF>(l, table, t64, t32, p);
    return some ? fma(t64, static_cast<double>(p), t64) : 0.0;
  }
};

// The difference of two bf16 numbers is an fp32 number unless one is 2^16 times smaller than the other; the rounding (2^-25
// of the difference) of those few is left in.
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
};
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
  // Temperature of a row; 1 where it is greedy.
  __device__ __forceinline__ float temp(int row, bool& greedy) const {
    const float t = temperature ? temperature[row] : 1.f;
    greedy = !(t > 0.f);
    return greedy ? 1.f : t;
  }
};

}  // namespace

// Rows without a filter (sample_stream.cu): workspace, and the two launches.
size_t sample_stream_bytes(long long n, int v);
int sample_stream(const void* args, a3po_dtype dt, void* ws, cudaStream_t stream);
// Rows with filters (sample_filter.cu): a row stays in the shared memory of a cluster of blocks.
long long sample_filter_max_v(a3po_dtype dt);
int sample_filter(const void* args, a3po_dtype dt, cudaStream_t stream);

}  // namespace a3po
