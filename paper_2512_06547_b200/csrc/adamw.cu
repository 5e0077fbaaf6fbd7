// AdamW over many tensors at once, with the global gradient norm and its clip in the same call.
//
//   s  = min(1, max_norm / (norm + 1e-6)),  norm = sqrt(sum of the squares of all gradients),  g = s grad
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   w' = w - lr (decay w + (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps))
//
// Two launches: sums of squares (64 bits, one number per block), and the update, whose blocks make the numbers of the step (norm, s,
// bias corrections) from them and from the learning rate and the count of steps on the device, so that a captured graph follows these.  The tensors come as a table in the kernel's
// arguments: no table in device memory to keep, and a captured graph has its own.
//
// States are fp32, or 8 bits in blocks of 256 elements with an fp32 scale each: value = q(code) scale,
// q(c) = c for c < 8, else (8 + c mod 8) 2^(c div 8 - 1).  First moment: a sign and codes to 127, q to 245,760 (half a step is
// at most 1/16 of a value); second moment: codes to 255, q to 1.6e10, so that the smallest square root that is not 0 is
// 1/127,000 of the largest.  A second moment above 0 is stored as 1 at least: 0 would leave eps alone under a first moment
// that is not 0.  A block is a warp's work: its largest value is a warp reduction.
// Rounding: to the nearest code in the first 32 steps, at random after them.  A gradient's share in an average is
// (1 - b) / (1 - b^t), at least 1 / t and 1 - b in the long run, and half a step between codes is 1/32 to 1/16 of a value: with b2 =
// 0.999 a nearest code hardly follows gradients that fall (v is 22 times too large 2,500 steps after they fell to a tenth).  At random,
// up with the probability that makes the code right on average, E v is the 32-bit v at every step.  The random numbers are
// Philox's for (step, tensor, element) and hang on nothing else: 16 bits and half of the last for each rounding, one call for
// a lane's eight elements, whose words serve the first moment of one element and the second of another.
// What is rounded to a code is computed in 64 bits, as a code is a step of several percent and two evaluations in 32 bits
// would disagree about one in 10^5 of them; the update itself is fp32.
//
// Bound: HBM (32 bits: 30 bytes an element with fp32 gradients and masters beside bf16 weights, 18 with 8 bits, and 4 more for
// the norm); with states of 8 bits the issue slots are about as far.  255 million weights: norm 169 us (6.0 TB/s), update 1,260
// (6.1 TB/s), with 8 bits 950 (4.8 TB/s) to the nearest code and 980 at random.  A few small tensors are two launches, 8 us.

#include <cfloat>
#include <climits>

#include "a3po_common.cuh"
#include "row_ops.cuh"

namespace a3po {
namespace {

constexpr int kBlock = 256;                 // elements that share a scale
constexpr int kThreads = 256, kWarps = kThreads / kWarp;
constexpr int kChunk = kWarps * kBlock;     // elements that a block takes at a time
constexpr int kNormBlocks = 2048;           // sums of squares at most
constexpr int kSmallTable = 32, kLargeTable = 400;
constexpr long long kNearestSteps = 32;     // see above

struct Entry {
  void* weight;
  float* master;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  long long n;
  float decay;
  int wide;   // every pointer allows accesses of four elements
};
template <int CAP>
struct Table {
  Entry e[CAP];
  int first[CAP + 1];   // chunks before entry i
  int count;
};

struct Numbers {   // of the step
  double g1, g2;   // (1 - b1) s and (1 - b2) s^2
  float scale, lr, inv_bc1, inv_bc2;
  int skip;
  long long t;     // this step's number
};
// What they are made of.  Every block of an update makes them for itself, from the same sums in the same order; the count of steps
// comes from a copy that the norm's first launch makes, so that the last update's first block may write the new one at any time.
struct StepArgs {
  const double* sums;
  int count;             // of sums
  float max_norm;
  double b1, b2;
  float eps;
  const float* lr;
  const long long* old_step;
  long long* step;       // null: an update that another follows
  float* grad_norm;
  int first_tensor;      // of the table, in the call
};

// Entry that holds a chunk.
template <int CAP>
__device__ __forceinline__ int entry_of(const Table<CAP>& t, int chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// A lane's eight elements of a block of 256: four neighbours at 4 lane and at 128 + 4 lane where pointers allow it, else
// element lane + 32 i.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int lane, int left, bool wide, float (&x)[8]) {
  if (wide) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const T* q = p + h * 128 + lane * 4;
      if (sizeof(T) == 4) {
        const float4 f = __ldcs(reinterpret_cast<const float4*>(q));
        x[h * 4] = f.x; x[h * 4 + 1] = f.y; x[h * 4 + 2] = f.z; x[h * 4 + 3] = f.w;
      } else {
        const uint2 u = __ldcs(reinterpret_cast<const uint2*>(q));
        x[h * 4] = __uint_as_float(u.x << 16); x[h * 4 + 1] = __uint_as_float(u.x & 0xffff0000u);
        x[h * 4 + 2] = __uint_as_float(u.y << 16); x[h * 4 + 3] = __uint_as_float(u.y & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = lane + 32 * i < left ? to_float(p[lane + 32 * i]) : 0.f;
  }
}
__device__ __forceinline__ void store8(float* p, int lane, int left, bool wide, const float (&x)[8]) {
  if (wide) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      __stcs(reinterpret_cast<float4*>(p + h * 128 + lane * 4), make_float4(x[h * 4], x[h * 4 + 1], x[h * 4 + 2], x[h * 4 + 3]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < left) p[lane + 32 * i] = x[i];
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, int lane, int left, bool wide, const float (&x)[8]) {
  if (wide) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(x[h * 4], x[h * 4 + 1]), b = __floats2bfloat162_rn(x[h * 4 + 2], x[h * 4 + 3]);
      uint2 u;
      u.x = *reinterpret_cast<const uint32_t*>(&a);
      u.y = *reinterpret_cast<const uint32_t*>(&b);
      __stcs(reinterpret_cast<uint2*>(p + h * 128 + lane * 4), u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < left) p[lane + 32 * i] = __float2bfloat16_rn(x[i]);
  }
}
// Codes as they lie in two words: element k of the lane is byte k % 4 of word k / 4.
__device__ __forceinline__ void load8(const uint8_t* p, int lane, int left, bool wide, uint32_t (&c)[2]) {
  if (wide) {
#pragma unroll
    for (int h = 0; h < 2; ++h) c[h] = __ldcs(reinterpret_cast<const uint32_t*>(p + h * 128 + lane * 4));
  } else {
    c[0] = c[1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < left) c[i / 4] |= static_cast<uint32_t>(p[lane + 32 * i]) << (i % 4 * 8);
  }
}
__device__ __forceinline__ void store8(uint8_t* p, int lane, int left, bool wide, const uint32_t (&c)[2]) {
  if (wide) {
#pragma unroll
    for (int h = 0; h < 2; ++h) __stcs(reinterpret_cast<uint32_t*>(p + h * 128 + lane * 4), c[h]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < left) p[lane + 32 * i] = static_cast<uint8_t>(c[i / 4] >> (i % 4 * 8));
  }
}

// ------------------------------------------------------------------------------------ norm
template <typename G, int CAP>
__global__ void __launch_bounds__(kThreads)
grad_norm_kernel(const __grid_constant__ Table<CAP> t, double* sums, const long long* step, long long* old_step) {
  __shared__ double part[kWarps];
  if (!step) wait_for_previous();   // else the call's first launch
  allow_next();
  if (step && blockIdx.x == 0 && threadIdx.x == 0) *old_step = *step;
  const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
  const int chunks = t.first[t.count];
  int chunk = static_cast<int>(static_cast<long long>(chunks) * blockIdx.x / gridDim.x);
  const int end = static_cast<int>(static_cast<long long>(chunks) * (blockIdx.x + 1) / gridDim.x);
  double sum = 0.0;
  int i = chunk < end ? entry_of(t, chunk) : 0;
  for (; chunk < end; ++chunk) {
    while (chunk >= t.first[i + 1]) ++i;
    const Entry& e = t.e[i];
    const long long at = static_cast<long long>(chunk - t.first[i]) * kChunk + warp * kBlock;
    if (at >= e.n) continue;
    const int left = static_cast<int>(e.n - at < kBlock ? e.n - at : kBlock);
    float g[8];
    load8(static_cast<const G*>(e.grad) + at, lane, left, e.wide && left == kBlock, g);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = fma(static_cast<double>(g[k]), static_cast<double>(g[k]), sum);
  }
  sum = warp_sum(sum);
  if (lane == 0) part[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) s += part[k];
    sums[blockIdx.x] = s;
  }
}

// ------------------------------------------------------------------------------------ numbers of the step
// By all threads, with barriers.  out: shared.  Not inlined: its powers are none of the update's registers' business.
__device__ __noinline__ void step_numbers(const StepArgs a, Numbers& out) {
  __shared__ double part[kWarps];
  double s = 0.0;
  for (int i = threadIdx.x; i < a.count; i += kThreads) s += a.sums[i];
  s = warp_sum(s);
  if (threadIdx.x % kWarp == 0) part[threadIdx.x / kWarp] = s;
  __syncthreads();
  const long long t = *a.old_step + 1;
  if (threadIdx.x < 2) {   // a warp's lanes: the two powers at once
    const double b = threadIdx.x ? a.b2 : a.b1;
    const float inv = static_cast<float>(1.0 / (1.0 - pow(b, static_cast<double>(t))));
    if (threadIdx.x) out.inv_bc2 = inv; else out.inv_bc1 = inv;
  }
  if (threadIdx.x == 0) {
    s = 0.0;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) s += part[k];
    const double norm = sqrt(s);
    float scale = 1.f;
    if (a.max_norm > 0.f) scale = static_cast<float>(fmin(static_cast<double>(a.max_norm) / (norm + 1e-6), 1.0));
    out.g1 = (1.0 - a.b1) * scale;
    out.g2 = (1.0 - a.b2) * scale * scale;
    out.scale = scale;
    out.lr = *a.lr;
    out.t = t;
    out.skip = !isfinite(norm);
    if (a.step && blockIdx.x == 0) {
      if (a.grad_norm) *a.grad_norm = static_cast<float>(norm);
      if (!out.skip) *a.step = t;
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------------------------ update
// sqrt(x) to two steps; x below 2^-126 counts as 0, which is seen beside a tiny eps only.
__device__ __forceinline__ float fast_root(float x) {
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__host__ __device__ constexpr double code_value(int c) {
  return c < 8 ? static_cast<double>(c) : static_cast<double>(static_cast<long long>(8 + c % 8) << (c / 8 - 1));
}
// The code nearest to x >= 0 (in units of the scale), halves to the even code.  From 8 on it is the leading four bits of x: three
// below the exponent, rounded by an addition that carries into it.  Below 8 the codes are the whole numbers, which are those
// of x + 8 less 8.
constexpr int kEight = 0x40200000;   // upper word of 8.0
// half a step less one, and what takes the bits of 8.0 to code 8
constexpr unsigned long long kRoundCode = (1ull << 48) - 1 - (static_cast<unsigned long long>((kEight >> 17) - 8) << 49);
__device__ __forceinline__ int code_of(double x, int top) {
  const bool small = __double2hiint(x) < kEight;
  if (small) x += 8.0;
  const int hi = __double2hiint(x);
  const int odd = hi >> 17 & 1, more = __double2loint(x) != 0 ? 1 : 0;
  const int c = (hi + 0xffff + (odd | more)) >> 17;
  return min(c - ((kEight >> 17) - (small ? 0 : 8)), top);
}
// x (in units of the scale) and a share of the step to the next code (odd multiples of 2^-17 of it), cut off.
__device__ __forceinline__ int code_at_random(double x, uint32_t share, int top) {
  const bool small = __double2hiint(x) < kEight;
  if (small) x += 8.0;
  return min(((__double2hiint(x) + static_cast<int>(share)) >> 17) - ((kEight >> 17) - (small ? 0 : 8)), top);
}
// What a lane's elements are rounded by: a word for each of the first four, which their counterparts in the block's other half share:
// the first moments take its upper half for the former and its lower for the latter, the second moments the other one.
// A word belongs to an element's place in the block, whoever holds it: a lane with every 32nd element asks the lanes that have its
// elements among their neighbours.
struct Random {
  uint32_t w[4];
  __device__ __forceinline__ void draw(long long t, int tensor, long long block, int lane, bool wide) {
    const uint32_t far = static_cast<uint32_t>(block >> 32) << 24;   // 0 but for tensors of 2^40 elements
    const PhiloxState ph{0u, 0u, static_cast<uint32_t>(t), static_cast<uint32_t>(t >> 32) ^ far};
    const uint4 u = ph.draw(static_cast<uint32_t>(tensor) * kWarp + static_cast<uint32_t>(lane), static_cast<uint32_t>(block));
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    if (!wide) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int from = lane / 4 + 8 * i;
        const uint32_t x = __shfl_sync(0xffffffffu, u.x, from), y = __shfl_sync(0xffffffffu, u.y, from);
        const uint32_t z = __shfl_sync(0xffffffffu, u.z, from), v = __shfl_sync(0xffffffffu, u.w, from);
        w[i] = lane % 4 == 0 ? x : lane % 4 == 1 ? y : lane % 4 == 2 ? z : v;
      }
    }
  }
  // 16 random bits and half of the last: of the 17 bits of a number's upper word below a code's
  template <bool FIRST>
  __device__ __forceinline__ uint32_t share(int k) const {
    return ((k < 4) == FIRST ? w[k % 4] >> 15 : w[k % 4] << 1 & 0x1ffffu) | 1u;
  }
};
__device__ __forceinline__ uint32_t min3u(uint32_t a, uint32_t b, uint32_t c) { return __vimin3_u32(a, b, c); }
__device__ __forceinline__ uint32_t max3u(uint32_t a, uint32_t b, uint32_t c) { return __vimax3_u32(a, b, c); }
// Largest over the warp of eight non-negative numbers a lane, ordered as their bits are: the upper words first, then the lower
// words of those that share the largest.
__device__ __forceinline__ double warp_max64(const double (&v)[8]) {
  uint32_t hi = 0;
#pragma unroll
  for (int k = 0; k < 8; k += 2)
    hi = max3u(hi, static_cast<uint32_t>(__double2hiint(v[k])) & 0x7fffffffu, static_cast<uint32_t>(__double2hiint(v[k + 1])) & 0x7fffffffu);
  hi = __reduce_max_sync(0xffffffffu, hi);
  uint32_t lo = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if ((static_cast<uint32_t>(__double2hiint(v[k])) & 0x7fffffffu) == hi) lo = max(lo, static_cast<uint32_t>(__double2loint(v[k])));
  lo = __reduce_max_sync(0xffffffffu, lo);
  return __hiloint2double(static_cast<int>(hi), static_cast<int>(lo));
}

// 1 / x for normal x: the fp32 quotient and two steps of Newton's iteration.
__device__ __forceinline__ double reciprocal(float x) {
  const double d = static_cast<double>(x);
  double r = static_cast<double>(__frcp_rn(x));
  r = fma(r, fma(-d, r, 1.0), r);
  return fma(r, fma(-d, r, 1.0), r);
}

// New first (second) moments of a block of 256, in 64 bits, stored as codes and a scale; out: their fp32 values.
template <bool FIRST, bool RANDOM>
__device__ __forceinline__ void new_states(uint8_t* codes, float* scale, uint32_t (&c)[2], float old, const double* q, double b,
                                           double more, int lane, int left, bool wide, const Random& random, const float (&g)[8],
                                           float (&out)[8]) {
  constexpr int kTop = FIRST ? 127 : 255;
  const double was = b * static_cast<double>(old);
  double x[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const double gk = static_cast<double>(g[k]);
    x[k] = fma(q[c[k / 4] >> (k % 4 * 8) & 255], was, more * (FIRST ? gk : gk * gk));
    out[k] = static_cast<float>(x[k]);
  }
  const float now = static_cast<float>(warp_max64(x) * (1.0 / code_value(kTop)));
  const double inv = now >= FLT_MIN ? reciprocal(now) : now > 0.f ? 1.0 / static_cast<double>(now) : 0.0;
  uint32_t least = 0xffffffffu;
#pragma unroll
  for (int k = 0; k < 8; k += 2)
    least = min3u(least, static_cast<uint32_t>(__double2hiint(fabs(x[k]) * inv)), static_cast<uint32_t>(__double2hiint(fabs(x[k + 1]) * inv)));
  uint32_t byte[8];
  const bool usual = __all_sync(0xffffffffu, least >= static_cast<uint32_t>(kEight)) && now >= FLT_MIN;   // nearly every block
  if (RANDOM && usual) {
    // the leading four bits; the largest is 2^-24 past the last code at most, too little for any share to make it another
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t hi = static_cast<uint32_t>(__double2hiint(fabs(x[k]) * inv));
      byte[k] = (hi + random.share<FIRST>(k) - (static_cast<uint32_t>((kEight >> 17) - 8) << 17)) >> 17;
      if (FIRST) byte[k] |= static_cast<uint32_t>(__double2hiint(x[k])) >> 24 & 0x80u;
    }
  } else if (usual) {
    // the leading four bits, rounded, and nothing else
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const unsigned long long u = static_cast<unsigned long long>(__double_as_longlong(fabs(x[k]) * inv));
      const uint32_t r = static_cast<uint32_t>((u + (u >> 49 & 1) + kRoundCode) >> 49);
      byte[k] = FIRST ? (r & 0x7fu) | (static_cast<uint32_t>(__double2hiint(x[k])) >> 24 & 0x80u) : r;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const double a = fabs(x[k]) * inv;
      byte[k] = static_cast<uint32_t>(RANDOM ? code_at_random(a, random.share<FIRST>(k), kTop) : code_of(a, kTop));
      if (FIRST) byte[k] |= x[k] < 0.0 ? 128u : 0u;
      else if (byte[k] == 0 && x[k] > 0.0 && now > 0.f) byte[k] = 1;
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    c[h] = __byte_perm(__byte_perm(byte[h * 4], byte[h * 4 + 1], 0x0040), __byte_perm(byte[h * 4 + 2], byte[h * 4 + 3], 0x0040), 0x5410);
  store8(codes, lane, left, wide, c);
  if (lane == 0) *scale = now;
}

// w' from the new moments (m is overwritten).
__device__ __forceinline__ void apply(float (&w)[8], float (&m)[8], const float (&v)[8], const Numbers& s, float decay, float eps) {
  if (eps < 1e-12f) {
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = m[k] * s.inv_bc1 / (__fsqrt_rn(v[k] * s.inv_bc2) + eps);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = m[k] * s.inv_bc1 * fast_rcp(fast_root(v[k] * s.inv_bc2) + eps);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = fmaf(-s.lr, fmaf(decay, w[k], m[k]), w[k]);
}

// A lane's own elements of the block that comes next, on their way into shared memory while a block is worked on: two blocks of
// the widest types a warp, filled and read by the same lane (no barrier).
template <typename G>
struct Ring {
  static constexpr int kW = 0, kG = 1024, kM = kG + kBlock * static_cast<int>(sizeof(G)), kV = kM + kBlock, kStage = kV + kBlock;
  static constexpr int kBytes = kWarps * 2 * kStage;
  uint32_t at;   // this warp's first stage
  int lane;
  template <int BYTES>
  __device__ __forceinline__ void copy(uint32_t to, const void* p) const {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(p), "n"(BYTES) : "memory");
  }
  // four elements of `SIZE` bytes at 4 lane, and at 128 + 4 lane
  template <int SIZE>
  __device__ __forceinline__ void copy8(uint32_t to, const void* p) const {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      copy<4 * SIZE>(to + (h * 32 + lane) * 4 * SIZE, static_cast<const char*>(p) + (h * 32 + lane) * 4 * SIZE);
  }
  __device__ __forceinline__ uint32_t stage(int s) const { return at + s * kStage; }
  template <typename T>
  __device__ __forceinline__ void read8(uint32_t from, float (&x)[8]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t a = from + (h * 32 + lane) * 4 * static_cast<uint32_t>(sizeof(T));
      if constexpr (sizeof(T) == 4) {
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(x[h * 4]), "=f"(x[h * 4 + 1]), "=f"(x[h * 4 + 2]), "=f"(x[h * 4 + 3]) : "r"(a) : "memory");
      } else {
        uint32_t u, v;
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(u), "=r"(v) : "r"(a) : "memory");
        x[h * 4] = __uint_as_float(u << 16); x[h * 4 + 1] = __uint_as_float(u & 0xffff0000u);
        x[h * 4 + 2] = __uint_as_float(v << 16); x[h * 4 + 3] = __uint_as_float(v & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void read8(uint32_t from, uint32_t (&c)[2]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(c[h]) : "r"(from + (h * 32 + lane) * 4) : "memory");
  }
};

// Where a warp's block of 256 lies.
struct Place {
  int entry;
  long long at;
  int left;     // elements, at most 256; 0: none
  bool wide;
};
template <int CAP>
__device__ __forceinline__ Place place_of(const Table<CAP>& t, int chunk, int end, int entry, int warp) {
  Place p{entry, 0, 0, false};
  if (chunk >= end) return p;
  while (chunk >= t.first[p.entry + 1]) ++p.entry;
  const Entry& e = t.e[p.entry];
  p.at = static_cast<long long>(chunk - t.first[p.entry]) * kChunk + warp * kBlock;
  if (p.at < e.n) p.left = static_cast<int>(e.n - p.at < kBlock ? e.n - p.at : kBlock);
  p.wide = e.wide && p.left == kBlock;
  return p;
}

// RANDOM: codes are rounded at random.  A function of its own for each of the two, so that neither holds the other's registers.
template <bool RANDOM, typename W, typename G, int CAP>
__device__ __forceinline__ void update_8bit(const Table<CAP>& t, const StepArgs& step, const Numbers& made, const double* q, uint8_t* smem) {
  const Numbers s = made;
  const long long t_now = made.t;
  const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
  using R = Ring<G>;
  R ring;
  ring.at = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + warp * 2 * R::kStage;
  ring.lane = lane;
  const int chunks = t.first[t.count];
  int chunk = static_cast<int>(static_cast<long long>(chunks) * blockIdx.x / gridDim.x);
  const int end = static_cast<int>(static_cast<long long>(chunks) * (blockIdx.x + 1) / gridDim.x);
  float next_ms = 0.f, next_vs = 0.f;   // the scales come with the block
  auto start = [&](const Place& p, int stage) {
    if (p.left > 0) {
      const Entry& e = t.e[p.entry];
      next_ms = e.m_scale[p.at / kBlock];
      next_vs = e.v_scale[p.at / kBlock];
      if (p.wide) {
        const uint32_t to = ring.stage(stage);
        ring.template copy8<sizeof(G)>(to + R::kG, static_cast<const G*>(e.grad) + p.at);
        ring.template copy8<1>(to + R::kM, static_cast<const uint8_t*>(e.m) + p.at);
        ring.template copy8<1>(to + R::kV, static_cast<const uint8_t*>(e.v) + p.at);
        if (sizeof(W) == 2 && e.master) ring.template copy8<4>(to + R::kW, e.master + p.at);
        else ring.template copy8<sizeof(W)>(to + R::kW, static_cast<const W*>(e.weight) + p.at);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  Place next = place_of(t, chunk, end, chunk < end ? entry_of(t, chunk) : 0, warp);
  start(next, 0);
  for (int stage = 0; chunk < end; ++chunk, stage ^= 1) {
    const Place p = next;
    const float old_ms = next_ms, old_vs = next_vs;
    next = place_of(t, chunk + 1, end, p.entry, warp);
    start(next, stage ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    if (p.left == 0) continue;   // the same for the warp
    const Entry& e = t.e[p.entry];
    const uint32_t from = ring.stage(stage);
    uint8_t *pm = static_cast<uint8_t*>(e.m) + p.at, *pv = static_cast<uint8_t*>(e.v) + p.at;
    float *ms = e.m_scale + p.at / kBlock, *vs = e.v_scale + p.at / kBlock;
    const bool master = sizeof(W) == 2 && e.master;
    float w[8], g[8], m[8], v[8];
    uint32_t cm[2], cv[2];
    Random random;
    if (RANDOM) random.draw(t_now, step.first_tensor + p.entry, p.at / kBlock, lane, p.wide);
    if (p.wide) {
      ring.template read8<G>(from + R::kG, g);
      ring.read8(from + R::kM, cm);
    } else {
      load8(static_cast<const G*>(e.grad) + p.at, lane, p.left, false, g);
      load8(pm, lane, p.left, false, cm);
    }
    new_states<true, RANDOM>(pm, ms, cm, old_ms, q, step.b1, s.g1, lane, p.left, p.wide, random, g, m);
    if (p.wide) ring.read8(from + R::kV, cv);
    else load8(pv, lane, p.left, false, cv);
    new_states<false, RANDOM>(pv, vs, cv, old_vs, q + 256, step.b2, s.g2, lane, p.left, p.wide, random, g, v);
    if (p.wide) {
      if (master) ring.template read8<float>(from + R::kW, w);
      else ring.template read8<W>(from + R::kW, w);
    } else {
      if (master) load8(static_cast<const float*>(e.master) + p.at, lane, p.left, false, w);
      else load8(static_cast<const W*>(e.weight) + p.at, lane, p.left, false, w);
    }
    apply(w, m, v, s, e.decay, step.eps);
    if (master) store8(e.master + p.at, lane, p.left, p.wide, w);
    store8(static_cast<W*>(e.weight) + p.at, lane, p.left, p.wide, w);
  }
}

// States of 8 bits.  18 bytes an element with fp32 gradients and masters beside bf16 weights: 980 us for 255 million, 1,060 with the
// registers of four blocks per SM; 950 and 1,016 to the nearest code (the latter when the next block is loaded into registers only
// once the one before it is done).
template <typename W, typename G, int CAP>
__global__ void __launch_bounds__(kThreads, 3)
adamw_8bit_kernel(const __grid_constant__ Table<CAP> t, const StepArgs step) {
  __shared__ double q[512];   // values of the codes, first moment (with the sign) and second
  extern __shared__ __align__(128) uint8_t smem[];   // rows of 128 bytes: 950 us, 1,020 where a copy's row lies across two of them
  const int c = threadIdx.x;
  q[c] = c < 128 ? code_value(c) : -code_value(c - 128);
  q[256 + c] = code_value(c);
  __syncthreads();
  wait_for_previous();
  allow_next();
  __shared__ Numbers made;
  step_numbers(step, made);
  if (made.skip) return;   // gradients that are not finite: nothing changes
  if (made.t <= kNearestSteps) update_8bit<false, W, G>(t, step, made, q, smem);
  else update_8bit<true, W, G>(t, step, made, q, smem);
}

template <typename W, typename G, int CAP>
__global__ void __launch_bounds__(kThreads, 4)
adamw_kernel(const __grid_constant__ Table<CAP> t, const StepArgs step) {
  wait_for_previous();
  allow_next();
  __shared__ Numbers s;
  step_numbers(step, s);
  if (s.skip) return;   // gradients that are not finite: nothing changes
  const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
  const int chunks = t.first[t.count];
  int chunk = static_cast<int>(static_cast<long long>(chunks) * blockIdx.x / gridDim.x);
  const int end = static_cast<int>(static_cast<long long>(chunks) * (blockIdx.x + 1) / gridDim.x);
  int entry = chunk < end ? entry_of(t, chunk) : 0;
  const float f1 = static_cast<float>(step.b1), f2 = static_cast<float>(step.b2);
  const float h1 = static_cast<float>(1.0 - step.b1), h2 = static_cast<float>(1.0 - step.b2);
  for (; chunk < end; ++chunk) {
    const Place p = place_of(t, chunk, end, entry, warp);
    entry = p.entry;
    if (p.left == 0) continue;   // the same for the warp
    const Entry& e = t.e[p.entry];
    const bool master = sizeof(W) == 2 && e.master;
    float w[8], g[8], m[8], v[8];
    if (master) load8(static_cast<const float*>(e.master) + p.at, lane, p.left, p.wide, w);
    else load8(static_cast<const W*>(e.weight) + p.at, lane, p.left, p.wide, w);
    load8(static_cast<const G*>(e.grad) + p.at, lane, p.left, p.wide, g);
    float *pm = static_cast<float*>(e.m) + p.at, *pv = static_cast<float*>(e.v) + p.at;
    load8(pm, lane, p.left, p.wide, m);
    load8(pv, lane, p.left, p.wide, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float x = g[k] * s.scale;
      m[k] = fmaf(f1, m[k], h1 * x);
      v[k] = fmaf(f2, v[k], h2 * x * x);
    }
    store8(pm, lane, p.left, p.wide, m);
    store8(pv, lane, p.left, p.wide, v);
    apply(w, m, v, s, e.decay, step.eps);
    if (master) store8(e.master + p.at, lane, p.left, p.wide, w);
    store8(static_cast<W*>(e.weight) + p.at, lane, p.left, p.wide, w);
  }
}

// ------------------------------------------------------------------------------------ host side
bool aligned4(const void* p, size_t elt) { return aligned_to(p, 4 * elt); }

template <int CAP>
void fill(Table<CAP>* t, const a3po_adamw_tensor* tensors, int count, size_t ws, size_t gs, int bits) {
  t->count = count;
  int chunks = 0;
  for (int i = 0; i < count; ++i) {
    const a3po_adamw_tensor& x = tensors[i];
    Entry& e = t->e[i];
    e = Entry{x.weight, x.master, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.n, x.weight_decay, 0};
    const size_t ss = bits == 8 ? 1 : 4;
    e.wide = aligned4(x.weight, ws) && aligned4(x.master, 4) && aligned4(x.grad, gs) && aligned4(x.m, ss) && aligned4(x.v, ss);
    t->first[i] = chunks;
    chunks += static_cast<int>((x.n + kChunk - 1) / kChunk);
  }
  t->first[count] = chunks;
}

template <typename W, typename G, int BITS, int CAP>
int launch_update(const Table<CAP>& t, const StepArgs& step, cudaStream_t s) {
  const int chunks = t.first[t.count], most = sm_count() * 8;
  if (chunks == 0 && !step.step) return A3PO_OK;
  const int grid = chunks < 1 ? 1 : chunks < most ? chunks : most;
  if constexpr (BITS == 8) {
    constexpr int kBytes = Ring<G>::kBytes;
    static_assert(kBytes <= 48 * 1024, "no opt-in needed");
    A3PO_LAUNCH(kKAdamStep, s, (launch_early(adamw_8bit_kernel<W, G, CAP>, grid, kThreads, kBytes, s, 1, true, t, step)));
  } else {
    A3PO_LAUNCH(kKAdamStep, s, (launch_early(adamw_kernel<W, G, CAP>, grid, kThreads, 0, s, 1, true, t, step)));
  }
  return after_launch();
}

template <int CAP>
int update(const a3po_adamw_tensor* tensors, int count, a3po_dtype wdt, a3po_dtype gdt, int bits, const StepArgs& step,
           cudaStream_t s) {
  using B = __nv_bfloat16;
  Table<CAP> t;
  fill(&t, tensors, count, wdt == A3PO_F32 ? 4 : 2, gdt == A3PO_F32 ? 4 : 2, bits);
#define A3PO_UPDATE(W, G)                                                                                      \
  (bits == 8 ? launch_update<W, G, 8>(t, step, s) : launch_update<W, G, 32>(t, step, s))
  if (wdt == A3PO_F32) return gdt == A3PO_F32 ? A3PO_UPDATE(float, float) : A3PO_UPDATE(float, B);
  return gdt == A3PO_F32 ? A3PO_UPDATE(B, float) : A3PO_UPDATE(B, B);
#undef A3PO_UPDATE
}

// Sums of squares of one table; returns their number through `blocks`.  step: the call's first launch, which copies it.
template <int CAP>
int norm_sums(const a3po_adamw_tensor* tensors, int count, a3po_dtype gdt, double* sums, int room, const long long* step,
              long long* old_step, int* blocks, cudaStream_t s) {
  Table<CAP> t;
  fill(&t, tensors, count, 1, gdt == A3PO_F32 ? 4 : 2, 8);
  for (int i = 0; i < count; ++i) t.e[i].wide = aligned4(tensors[i].grad, gdt == A3PO_F32 ? 4 : 2);
  const int chunks = t.first[t.count];
  int grid = sm_count() * 6 < chunks ? sm_count() * 6 : chunks;
  if (grid > room) grid = room;
  if (step && grid < 1) grid = 1;
  *blocks = grid;
  if (grid == 0) return A3PO_OK;
  if (gdt == A3PO_F32)
    A3PO_LAUNCH(kKAdamNorm, s, (launch_early(grad_norm_kernel<float, CAP>, grid, kThreads, 0, s, 1, !step, t, sums, step, old_step)));
  else
    A3PO_LAUNCH(kKAdamNorm, s, (launch_early(grad_norm_kernel<__nv_bfloat16, CAP>, grid, kThreads, 0, s, 1, !step, t, sums, step,
                                             old_step)));
  return after_launch();
}

int norm_room(int count) {   // sums: kNormBlocks for each table of kLargeTable tensors, and for none
  return (count > 0 ? (count + kLargeTable - 1) / kLargeTable : 1) * kNormBlocks;
}

// Four codes per thread and step where the pointers allow it.  Bound: HBM, 5 bytes an element (255 million: 235 us, 5.4 TB/s).
__global__ void __launch_bounds__(256)
state_values_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales, long long n, int is_signed, int wide,
                    float* __restrict__ out) {
  __shared__ float q[256];
  const int c = threadIdx.x;
  q[c] = static_cast<float>(!is_signed ? code_value(c) : c < 128 ? code_value(c) : -code_value(c - 128));
  __syncthreads();
  const long long me = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x, all = static_cast<long long>(gridDim.x) * 256;
  const long long quads = wide ? n / 4 : 0;
  for (long long i = me; i < quads; i += all) {
    const uint32_t u = __ldcs(reinterpret_cast<const uint32_t*>(codes) + i);
    const float s = __ldg(scales + i / (kBlock / 4));
    __stcs(reinterpret_cast<float4*>(out) + i,
           make_float4(q[u & 255] * s, q[u >> 8 & 255] * s, q[u >> 16 & 255] * s, q[u >> 24] * s));
  }
  for (long long i = quads * 4 + me; i < n; i += all) out[i] = q[codes[i]] * scales[i / kBlock];
}

}  // namespace
}  // namespace a3po

using namespace a3po;

extern "C" {

size_t a3po_adamw_workspace_bytes(int count) {
  if (count < 0) return 0;
  return 256 /* the count of steps */ + round_up(static_cast<size_t>(norm_room(count)) * sizeof(double), 256) + 256;
}

int a3po_adamw_step(const a3po_adamw_tensor* tensors, int count, a3po_dtype weight_dt, a3po_dtype grad_dt, int state_bits,
                    double beta1, double beta2, float eps, float max_grad_norm, const float* lr, int64_t* step,
                    float* grad_norm, void* ws, size_t ws_bytes, void* stream_) {
  if (count < 0 || (count > 0 && !tensors) || !lr || !step) return A3PO_ERR_INVALID_ARG;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps > 0.f) || !(max_grad_norm >= 0.f))
    return A3PO_ERR_INVALID_ARG;
  if ((weight_dt != A3PO_F32 && weight_dt != A3PO_BF16) || (grad_dt != A3PO_F32 && grad_dt != A3PO_BF16)) return A3PO_ERR_UNSUPPORTED;
  if (state_bits != 8 && state_bits != 32) return A3PO_ERR_UNSUPPORTED;
  if (!aligned_to(lr, 4) || !aligned_to(step, 8) || !aligned_to(grad_norm, 4)) return A3PO_ERR_UNSUPPORTED;
  const size_t wsz = weight_dt == A3PO_F32 ? 4 : 2, gsz = grad_dt == A3PO_F32 ? 4 : 2, ssz = state_bits == 8 ? 1 : 4;
  long long chunks = 0;
  for (int i = 0; i < count; ++i) {
    const a3po_adamw_tensor& t = tensors[i];
    if (t.n < 0 || (t.n > 0 && (!t.weight || !t.grad || !t.m || !t.v))) return A3PO_ERR_INVALID_ARG;
    if (t.n > 0 && state_bits == 8 && (!t.m_scale || !t.v_scale)) return A3PO_ERR_INVALID_ARG;
    if (t.master && weight_dt == A3PO_F32) return A3PO_ERR_INVALID_ARG;   // the weights are the masters
    if (!aligned_to(t.weight, wsz) || !aligned_to(t.master, 4) || !aligned_to(t.grad, gsz) || !aligned_to(t.m, ssz) ||
        !aligned_to(t.v, ssz) || !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4))
      return A3PO_ERR_UNSUPPORTED;
    if (t.n > (1ll << 41)) return A3PO_ERR_UNSUPPORTED;
    chunks += (t.n + kChunk - 1) / kChunk;
  }
  if (chunks > INT_MAX) return A3PO_ERR_UNSUPPORTED;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_adamw_workspace_bytes(count)) return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  cudaStream_t stream = as_stream(stream_);
  Arena ar(ws, ws_bytes);
  long long* old_step = ar.take<long long>(1);
  double* sums = ar.take<double>(static_cast<size_t>(norm_room(count)));
  if (!ar.ok()) return A3PO_ERR_WORKSPACE;
  // without a norm the first launch sees no tensors: it copies the count of steps, and the norm is 0
  const int normed = max_grad_norm > 0.f || grad_norm ? count : 0;
  int total = 0, at = 0;
  do {
    const int part = normed - at < kLargeTable ? normed - at : kLargeTable;
    const long long* first = at == 0 ? reinterpret_cast<const long long*>(step) : nullptr;
    int blocks = 0;
    if (part <= kSmallTable)
      A3PO_RETURN_IF(norm_sums<kSmallTable>(tensors + at, part, grad_dt, sums + total, kNormBlocks, first, old_step, &blocks, stream));
    else
      A3PO_RETURN_IF(norm_sums<kLargeTable>(tensors + at, part, grad_dt, sums + total, kNormBlocks, first, old_step, &blocks, stream));
    total += blocks;
    at += part;
  } while (at < normed);
  StepArgs args{sums, total, max_grad_norm, beta1, beta2, eps, lr, old_step, nullptr, grad_norm, 0};
  at = 0;
  do {
    const int part = count - at < kLargeTable ? count - at : kLargeTable;
    if (at + part == count) args.step = reinterpret_cast<long long*>(step);
    args.first_tensor = at;
    if (part <= kSmallTable) A3PO_RETURN_IF(update<kSmallTable>(tensors + at, part, weight_dt, grad_dt, state_bits, args, stream));
    else A3PO_RETURN_IF(update<kLargeTable>(tensors + at, part, weight_dt, grad_dt, state_bits, args, stream));
    at += part;
  } while (at < count);
  return A3PO_OK;
}

int a3po_adamw_state_values(const uint8_t* codes, const float* scales, int64_t n, int is_signed, float* values, void* stream_) {
  if (n < 0 || (n > 0 && (!codes || !scales || !values))) return A3PO_ERR_INVALID_ARG;
  if (!aligned_to(scales, 4) || !aligned_to(values, 4)) return A3PO_ERR_UNSUPPORTED;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (n == 0) return A3PO_OK;
  cudaStream_t stream = as_stream(stream_);
  const int wide = aligned_to(codes, 4) && aligned_to(values, 16);
  const long long per = wide ? 1024 : 256, want = (n + per - 1) / per, most = sm_count() * 64ll;
  A3PO_LAUNCH(kKAdamStep, stream, (state_values_kernel<<<static_cast<unsigned>(want < most ? want : most), 256, 0, stream>>>(
                                      codes, scales, n, is_signed, wide, values)));
  return after_launch();
}

}  // extern "C"
