// Row-wise training operators on the residual stream in front of the LM head: norm (RMS or layer), dropout whose
// mask is never stored, and the join of both (dropout, add to the residual stream, norm) in one pass; forward and
// backward.
//
//   norm      xhat = (x - mean) rstd,  mean = sum x / H (0 for RMS),  rstd = 1 / sqrt(sum (x - mean)^2 / H + eps)
//             y = xhat gamma + beta
//   backward  gx = gy gamma,  dx = rstd (gx - [mean(gx)] - xhat mean(gx xhat))      ([.]: layer norm only)
//             dgamma = sum_rows gy xhat,  dbeta = sum_rows gy
//   dropout   d(x)[t, c] = keep(t, c) x[t, c] 65536 / (65536 - T),  T = round(65536 p),  keep = (u16(t, c) >= T)
//   join      r = residual + d(x) (stored),  y = norm(r)
//
// All of them stream [N, H] matrices and compute next to nothing, so HBM bytes are the bound: every element is read
// once (a row stays in registers between its statistics and its result) and written once.  A thread owns 8
// consecutive columns (16 bytes of bf16), which is also what one Philox call decides.  Sums, statistics and partial
// weight gradients are fp32; the only rounding to fewer bits is the final store in the matrices' own type.
//
// Random numbers: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC'11),
// key = seed, counter = (column / 8, row, offset low, offset high); its four words are eight 16-bit numbers, low half
// first.  16 bits decide one element: the drop probability is a multiple of 2^-16 and the scale is exact for it, at
// half the integer work of 32-bit numbers (with those the multiplies, not HBM, would bound dropout).

#include "a3po_common.cuh"

namespace a3po {
namespace {

constexpr int kVec = 8;   // columns of a thread's chunk

// ------------------------------------------------------------------------------------ pieces
struct Dropout {
  const unsigned long long* rng;  // device: {seed, offset}; null = nothing is dropped
  uint32_t threshold;             // element dropped iff u16 < threshold
  float scale;                    // 65536 / (65536 - threshold), 0 when everything is dropped
};

struct PhiloxState {
  uint32_t k0, k1, o0, o1;
  __device__ __forceinline__ void load(const unsigned long long* rng) {
    const unsigned long long seed = rng[0], offset = rng[1];
    k0 = static_cast<uint32_t>(seed);
    k1 = static_cast<uint32_t>(seed >> 32);
    o0 = static_cast<uint32_t>(offset);
    o1 = static_cast<uint32_t>(offset >> 32);
  }
  __device__ __forceinline__ uint4 draw(uint32_t group, uint32_t row) const {
    uint32_t c0 = group, c1 = row, c2 = o0, c3 = o1, a = k0, b = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint32_t h0 = __umulhi(0xD2511F53u, c0), l0 = 0xD2511F53u * c0;
      const uint32_t h1 = __umulhi(0xCD9E8D57u, c2), l1 = 0xCD9E8D57u * c2;
      c0 = h1 ^ c1 ^ a;
      c1 = l1;
      c2 = h0 ^ c3 ^ b;
      c3 = l0;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
  }
};

// x -> d(x) for the 8 columns of one chunk
__device__ __forceinline__ void drop_chunk(float (&x)[kVec], const Dropout& d, const PhiloxState& ph, uint32_t group,
                                           uint32_t row) {
  const uint4 w = ph.draw(group, row);
  const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = (words[j] & 0xffffu) >= d.threshold ? x[2 * j] * d.scale : 0.f;
    x[2 * j + 1] = (words[j] >> 16) >= d.threshold ? x[2 * j + 1] * d.scale : 0.f;
  }
}

// Eight columns of a row.  `vec`: rows are 16-byte aligned and h % 8 == 0, so a chunk is whole and moves in 16-byte
// pieces; otherwise element by element, columns at and beyond h read as 0 and are not written.
template <typename T>
__device__ __forceinline__ void load_chunk(const T* row, int col, int h, bool vec, float (&x)[kVec]) {
  if (vec) {
    if (col < h) {
      if constexpr (sizeof(T) == 2) {
        const uint4 u = __ldcs(reinterpret_cast<const uint4*>(row + col));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[2 * j] = __uint_as_float(w[j] << 16);
          x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
      } else {
        const float4 a = __ldcs(reinterpret_cast<const float4*>(row + col));
        const float4 b = __ldcs(reinterpret_cast<const float4*>(row + col) + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) x[j] = 0.f;
    return;
  }
#pragma unroll
  for (int j = 0; j < kVec; ++j) x[j] = (col + j < h) ? to_float(row[col + j]) : 0.f;
}

template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int col, int h, bool vec, const float (&x)[kVec]) {
  if (vec) {
    if (col >= h) return;
    if constexpr (sizeof(T) == 2) {
      uint4 u;
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
        w[j] = *reinterpret_cast<uint32_t*>(&p);
      }
      u.x = w[0]; u.y = w[1]; u.z = w[2]; u.w = w[3];
      __stcs(reinterpret_cast<uint4*>(row + col), u);
    } else {
      __stcs(reinterpret_cast<float4*>(row + col), make_float4(x[0], x[1], x[2], x[3]));
      __stcs(reinterpret_cast<float4*>(row + col) + 1, make_float4(x[4], x[5], x[6], x[7]));
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < kVec; ++j)
    if (col + j < h) row[col + j] = from_float<T>(x[j]);
}

// Parameters (gamma, beta) are shared by every row: the default load keeps them in L1.
template <typename T>
__device__ __forceinline__ void load_param(const T* __restrict__ p, int col, int h, bool vec, float (&x)[kVec]) {
  if (vec && sizeof(T) == 2) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (col < h) u = __ldg(reinterpret_cast<const uint4*>(p + col));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < kVec; ++j) x[j] = (col + j < h) ? to_float(p[col + j]) : 0.f;
}

// Rounds to the storage type and back.
template <typename T>
__device__ __forceinline__ float as_stored(float x) { return to_float(from_float<T>(x)); }

// Sum over the TPR threads of a row (a warp, or the whole block).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* sh) {
  v = warp_sum(v);
  if constexpr (TPR > kWarp) {
    const int warp = threadIdx.x / kWarp;
    __syncthreads();   // the previous use of `sh` has been read
    if (threadIdx.x % kWarp == 0) sh[warp] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / kWarp; ++w) t += sh[w];
    v = t;
  }
  return v;
}
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* sh) {
  a = warp_sum(a);
  b = warp_sum(b);
  if constexpr (TPR > kWarp) {
    const int warp = threadIdx.x / kWarp;
    __syncthreads();
    if (threadIdx.x % kWarp == 0) sh[warp] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / kWarp; ++w) {
      a += sh[w].x;
      b += sh[w].y;
    }
  }
  return make_float2(a, b);
}

// Rows a block works on at once: blocks of 256 threads hold several rows when a row is a warp's, one otherwise.
template <int TPR> constexpr int threads_of() { return TPR == kWarp ? 256 : TPR; }
template <int TPR> constexpr int rows_per_block() { return TPR == kWarp ? 256 / kWarp : 1; }

template <typename T>
struct NormFwdArgs {
  const T* x;           // normalised input; with JOIN the branch that goes through dropout
  const T* residual;    // JOIN: residual stream
  const T* gamma;
  const T* beta;        // null: none
  const uint8_t* row_mask;
  long long n;
  int h;
  float eps;
  float inv_h;
  T* r;                 // JOIN: stored sum
  T* y;
  float* mean;          // null: not wanted
  float* rstd;          // null: not wanted
  Dropout drop;
  int vec;
};

// One row per TPR threads, the row in registers between its statistics and its result.
template <typename T, int TPR, int CPT, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(threads_of<TPR>())
norm_fwd_kernel(const NormFwdArgs<T> a) {
  __shared__ float sh[kWarp];
  const int tid = threadIdx.x % TPR;
  const long long t = static_cast<long long>(blockIdx.x) * rows_per_block<TPR>() + threadIdx.x / TPR;
  if (t >= a.n) return;                 // whole warps (TPR = 32), or never (one row per block)
  const bool vec = a.vec != 0;
  T* y = a.y + t * a.h;
  float v[CPT][kVec];
  if (a.row_mask && a.row_mask[t] == 0) {   // same for all threads of the row
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[0][j] = 0.f;
    for (int col = tid * kVec; col < a.h; col += TPR * kVec) {
      store_chunk(y, col, a.h, vec, v[0]);
      if (JOIN) store_chunk(a.r + t * a.h, col, a.h, vec, v[0]);
    }
    if (tid == 0) {
      if (a.mean) a.mean[t] = 0.f;
      if (a.rstd) a.rstd[t] = 0.f;
    }
    return;
  }
  const T* x = a.x + t * a.h;
#pragma unroll
  for (int i = 0; i < CPT; ++i) load_chunk(x, (tid + i * TPR) * kVec, a.h, vec, v[i]);
  if constexpr (JOIN) {
    float res[CPT][kVec];
#pragma unroll
    for (int i = 0; i < CPT; ++i) load_chunk(a.residual + t * a.h, (tid + i * TPR) * kVec, a.h, vec, res[i]);
    const bool drop = a.drop.rng != nullptr;
    PhiloxState ph;
    if (drop) ph.load(a.drop.rng);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      if (drop) drop_chunk(v[i], a.drop, ph, static_cast<uint32_t>(tid + i * TPR), static_cast<uint32_t>(t));
      // the norm is that of the stored sum, which is what the backward will read
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[i][j] = as_stored<T>(v[i][j] + res[i][j]);
      store_chunk(a.r + t * a.h, (tid + i * TPR) * kVec, a.h, vec, v[i]);
    }
  }
  float mean = 0.f;
  if constexpr (LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < CPT; ++i)
#pragma unroll
      for (int j = 0; j < kVec; ++j) s += v[i][j];
    mean = row_sum<TPR>(s, sh) * a.inv_h;
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    const int col = (tid + i * TPR) * kVec;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      if (LAYER) v[i][j] = (col + j < a.h) ? v[i][j] - mean : 0.f;
      q = fmaf(v[i][j], v[i][j], q);
    }
  }
  const float rstd = 1.0f / sqrtf(row_sum<TPR>(q, sh) * a.inv_h + a.eps);
  if (tid == 0) {
    if (a.mean) a.mean[t] = mean;
    if (a.rstd) a.rstd[t] = rstd;
  }
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    const int col = (tid + i * TPR) * kVec;
    float g[kVec];
    load_param(a.gamma, col, a.h, vec, g);
    if (a.beta) {
      float b[kVec];
      load_param(a.beta, col, a.h, vec, b);
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[i][j] = fmaf(v[i][j] * rstd, g[j], b[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[i][j] = v[i][j] * rstd * g[j];
    }
    store_chunk(y, col, a.h, vec, v[i]);
  }
}

template <typename T>
struct NormBwdArgs {
  const T* x;             // what was normalised
  const T* gamma;
  const float* mean;      // layer norm only
  const float* rstd;
  const uint8_t* row_mask;
  const T* grad_y;
  const T* grad_r;        // JOIN: gradient that reaches the sum past the norm, or null
  long long n;
  int h;
  float inv_h;
  T* grad_x;              // gradient of x; with JOIN of the branch (through dropout), or null: not wanted
  T* grad_residual;       // JOIN: gradient of the residual stream
  float* part;            // [parts][1 or 2][h] partial sums of dgamma (and dbeta)
  Dropout drop;
  int vec;
};

// Persistent: a block (or warp, TPR = 32) takes every parts-th row and keeps its share of dgamma / dbeta in
// registers, one column's sum per thread and column; the shares are added up by reduce_parts_kernel in index order,
// so results do not depend on the order in which blocks run.
template <typename T, int TPR, int CPT, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(threads_of<TPR>())
norm_bwd_kernel(const NormBwdArgs<T> a) {
  __shared__ float2 sh[kWarp];
  const int tid = threadIdx.x % TPR;
  const long long part = static_cast<long long>(blockIdx.x) * rows_per_block<TPR>() + threadIdx.x / TPR;
  const long long parts = static_cast<long long>(gridDim.x) * rows_per_block<TPR>();
  const bool vec = a.vec != 0;
  float dg[CPT][kVec], db[CPT][kVec];
#pragma unroll
  for (int i = 0; i < CPT; ++i)
#pragma unroll
    for (int j = 0; j < kVec; ++j) dg[i][j] = db[i][j] = 0.f;
  const bool drop = JOIN && a.drop.rng != nullptr;
  PhiloxState ph;
  if (drop) ph.load(a.drop.rng);

  for (long long t = part; t < a.n; t += parts) {
    T* gx_row = a.grad_x + t * a.h;
    if (a.row_mask && a.row_mask[t] == 0) {
      float z[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) z[j] = 0.f;
      for (int col = tid * kVec; col < a.h; col += TPR * kVec) {
        if (!JOIN || a.grad_x) store_chunk(gx_row, col, a.h, vec, z);
        if (JOIN) store_chunk(a.grad_residual + t * a.h, col, a.h, vec, z);
      }
      continue;
    }
    float x[CPT][kVec], gy[CPT][kVec];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      load_chunk(a.x + t * a.h, (tid + i * TPR) * kVec, a.h, vec, x[i]);
      load_chunk(a.grad_y + t * a.h, (tid + i * TPR) * kVec, a.h, vec, gy[i]);
    }
    const float rstd = a.rstd[t];
    const float mean = LAYER ? a.mean[t] : 0.f;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int col = (tid + i * TPR) * kVec;
      float g[kVec];
      load_param(a.gamma, col, a.h, vec, g);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        x[i][j] = LAYER ? (x[i][j] - mean) * rstd : x[i][j] * rstd;   // xhat (columns past h meet gy = g = 0)
        dg[i][j] = fmaf(gy[i][j], x[i][j], dg[i][j]);
        if (LAYER) db[i][j] += gy[i][j];
        gy[i][j] *= g[j];
        if (LAYER) s0 += gy[i][j];
        s1 = fmaf(gy[i][j], x[i][j], s1);
      }
    }
    const float2 s = row_sum2<TPR>(s0, s1, sh);
    const float m0 = LAYER ? s.x * a.inv_h : 0.f, m1 = s.y * a.inv_h;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int col = (tid + i * TPR) * kVec;
#pragma unroll
      for (int j = 0; j < kVec; ++j) gy[i][j] = (gy[i][j] - m0 - x[i][j] * m1) * rstd;
      if constexpr (JOIN) {
        if (a.grad_r) {
          float gr[kVec];
          load_chunk(a.grad_r + t * a.h, col, a.h, vec, gr);
#pragma unroll
          for (int j = 0; j < kVec; ++j) gy[i][j] += gr[j];
        }
        store_chunk(a.grad_residual + t * a.h, col, a.h, vec, gy[i]);
        if (!a.grad_x) continue;
        if (drop) drop_chunk(gy[i], a.drop, ph, static_cast<uint32_t>(tid + i * TPR), static_cast<uint32_t>(t));
      }
      store_chunk(gx_row, col, a.h, vec, gy[i]);
    }
  }
  float* out = a.part + part * (LAYER ? 2 : 1) * a.h;
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    const int col = (tid + i * TPR) * kVec;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      if (col + j < a.h) {
        out[col + j] = dg[i][j];
        if (LAYER) out[a.h + col + j] = db[i][j];
      }
    }
  }
}

// grad[c] (+)= sum over parts, in a fixed order: 8 threads per column take every 8th part, then the eight sums.
constexpr int kReduceCols = 32, kReduceLanes = 8;
__global__ void __launch_bounds__(kReduceCols* kReduceLanes)
reduce_parts_kernel(const float* __restrict__ part, int parts, long long row_pitch, int h, int accumulate,
                    float* __restrict__ grad_gamma, float* __restrict__ grad_beta) {
  const float* src = part + (blockIdx.y ? h : 0);
  float* dst = blockIdx.y ? grad_beta : grad_gamma;
  if (!dst) return;
  const int c = blockIdx.x * kReduceCols + threadIdx.x;
  float s = 0.f;
  if (c < h)
    for (int p = threadIdx.y; p < parts; p += kReduceLanes) s += src[p * row_pitch + c];
  __shared__ float sh[kReduceLanes][kReduceCols];
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y == 0 && c < h) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kReduceLanes; ++i) t += sh[i][threadIdx.x];
    dst[c] = accumulate ? dst[c] + t : t;
  }
}

// Rows longer than the register form holds: the row is read again for each use (from L2), one row per block, and the
// weight gradients are summed by a second kernel whose threads own columns.
constexpr int kLongThreads = 1024;
template <typename T, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(kLongThreads)
norm_fwd_long_kernel(const NormFwdArgs<T> a) {
  __shared__ float sh[kWarp];
  const long long t = blockIdx.x;
  const bool vec = a.vec != 0;
  const bool masked = a.row_mask && a.row_mask[t] == 0;
  T* y = a.y + t * a.h;
  T* r = JOIN ? a.r + t * a.h : nullptr;
  const T* x = JOIN ? r : a.x + t * a.h;
  const bool drop = JOIN && a.drop.rng != nullptr;
  PhiloxState ph;
  if (drop) ph.load(a.drop.rng);
  float s = 0.f;
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float v[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = 0.f;
    if (masked) {
      store_chunk(y, col, a.h, vec, v);
      if (JOIN) store_chunk(r, col, a.h, vec, v);
      continue;
    }
    load_chunk(a.x + t * a.h, col, a.h, vec, v);
    if constexpr (JOIN) {
      float res[kVec];
      load_chunk(a.residual + t * a.h, col, a.h, vec, res);
      if (drop) drop_chunk(v, a.drop, ph, static_cast<uint32_t>(col / kVec), static_cast<uint32_t>(t));
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[j] = as_stored<T>(v[j] + res[j]);
      store_chunk(r, col, a.h, vec, v);
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) s += v[j];
  }
  if (masked) {
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[t] = 0.f;
      if (a.rstd) a.rstd[t] = 0.f;
    }
    return;
  }
  // each thread reads back only chunks that it wrote itself
  const float mean = LAYER ? row_sum<kLongThreads>(s, sh) * a.inv_h : 0.f;
  float q = 0.f;
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float v[kVec];
    load_chunk(x, col, a.h, vec, v);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const float d = (col + j < a.h) ? v[j] - mean : 0.f;
      q = fmaf(d, d, q);
    }
  }
  const float rstd = 1.0f / sqrtf(row_sum<kLongThreads>(q, sh) * a.inv_h + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[t] = mean;
    if (a.rstd) a.rstd[t] = rstd;
  }
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float v[kVec], g[kVec], b[kVec];
    load_chunk(x, col, a.h, vec, v);
    load_param(a.gamma, col, a.h, vec, g);
#pragma unroll
    for (int j = 0; j < kVec; ++j) b[j] = 0.f;
    if (a.beta) load_param(a.beta, col, a.h, vec, b);
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = fmaf((v[j] - mean) * rstd, g[j], b[j]);
    store_chunk(y, col, a.h, vec, v);
  }
}

template <typename T, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(kLongThreads)
norm_bwd_long_kernel(const NormBwdArgs<T> a) {
  __shared__ float2 sh[kWarp];
  const long long t = blockIdx.x;
  const bool vec = a.vec != 0;
  float z[kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) z[j] = 0.f;
  if (a.row_mask && a.row_mask[t] == 0) {
    for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
      if (!JOIN || a.grad_x) store_chunk(a.grad_x + t * a.h, col, a.h, vec, z);
      if (JOIN) store_chunk(a.grad_residual + t * a.h, col, a.h, vec, z);
    }
    return;
  }
  const float rstd = a.rstd[t];
  const float mean = LAYER ? a.mean[t] : 0.f;
  float s0 = 0.f, s1 = 0.f;
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float x[kVec], gy[kVec], g[kVec];
    load_chunk(a.x + t * a.h, col, a.h, vec, x);
    load_chunk(a.grad_y + t * a.h, col, a.h, vec, gy);
    load_param(a.gamma, col, a.h, vec, g);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const float gx = gy[j] * g[j];
      s0 += gx;
      s1 = fmaf(gx, (x[j] - mean) * rstd, s1);
    }
  }
  const float2 s = row_sum2<kLongThreads>(s0, s1, sh);
  const float m0 = LAYER ? s.x * a.inv_h : 0.f, m1 = s.y * a.inv_h;
  const bool drop = JOIN && a.drop.rng != nullptr;
  PhiloxState ph;
  if (drop) ph.load(a.drop.rng);
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float x[kVec], gy[kVec], g[kVec];
    load_chunk(a.x + t * a.h, col, a.h, vec, x);
    load_chunk(a.grad_y + t * a.h, col, a.h, vec, gy);
    load_param(a.gamma, col, a.h, vec, g);
#pragma unroll
    for (int j = 0; j < kVec; ++j) gy[j] = (gy[j] * g[j] - m0 - (x[j] - mean) * rstd * m1) * rstd;
    if constexpr (JOIN) {
      if (a.grad_r) {
        load_chunk(a.grad_r + t * a.h, col, a.h, vec, g);
#pragma unroll
        for (int j = 0; j < kVec; ++j) gy[j] += g[j];
      }
      store_chunk(a.grad_residual + t * a.h, col, a.h, vec, gy);
      if (!a.grad_x) continue;
      if (drop) drop_chunk(gy, a.drop, ph, static_cast<uint32_t>(col / kVec), static_cast<uint32_t>(t));
    }
    store_chunk(a.grad_x + t * a.h, col, a.h, vec, gy);
  }
}

// Partial weight gradients of the long form: block (x: 256 columns, y: part), rows part, part + parts, ...
template <typename T, bool LAYER>
__global__ void __launch_bounds__(256)
norm_weight_long_kernel(const NormBwdArgs<T> a, int parts) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.h) return;
  float dg = 0.f, db = 0.f;
  for (long long t = blockIdx.y; t < a.n; t += parts) {
    if (a.row_mask && a.row_mask[t] == 0) continue;
    const float gy = to_float(a.grad_y[t * a.h + c]);
    const float x = to_float(a.x[t * a.h + c]);
    dg = fmaf(gy, (LAYER ? x - a.mean[t] : x) * a.rstd[t], dg);
    db += gy;
  }
  float* out = a.part + static_cast<long long>(blockIdx.y) * (LAYER ? 2 : 1) * a.h;
  out[c] = dg;
  if (LAYER) out[a.h + c] = db;
}

// y = d(x) (+ residual), and the gradient of d(x).  Grid-stride over the N x ceil(H/8) chunks; a thread steps from
// chunk to chunk by a fixed (rows, chunks) stride, so there is one 64-bit division per thread and none in the loop.
// Two chunks are in flight per thread.
constexpr int kDropThreads = 256;
constexpr int kDropUnroll = 2;
template <typename T>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const T* __restrict__ x, const T* __restrict__ residual, const uint8_t* __restrict__ row_mask,
               long long n, int h, Dropout drop, T* __restrict__ y, int vec_) {
  const bool vec = vec_ != 0;
  const int groups = (h + kVec - 1) / kVec;
  const long long stride = static_cast<long long>(gridDim.x) * kDropThreads;
  const long long first = static_cast<long long>(blockIdx.x) * kDropThreads + threadIdx.x;
  const long long step_rows = stride / groups;
  const int step_groups = static_cast<int>(stride - step_rows * groups);
  long long row = first / groups;
  int group = static_cast<int>(first - row * groups);
  PhiloxState ph;
  const bool dropping = drop.rng != nullptr;
  if (dropping) ph.load(drop.rng);
  while (row < n) {
    float v[kDropUnroll][kVec], res[kDropUnroll][kVec];
    long long r[kDropUnroll];
    int g[kDropUnroll];
    bool on[kDropUnroll];
#pragma unroll
    for (int i = 0; i < kDropUnroll; ++i) {
      r[i] = row;
      g[i] = group;
      row += step_rows;
      group += step_groups;
      if (group >= groups) {
        group -= groups;
        ++row;
      }
      on[i] = r[i] < n && (!row_mask || row_mask[r[i]] != 0);
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[i][j] = res[i][j] = 0.f;
      if (on[i]) {
        load_chunk(x + r[i] * h, g[i] * kVec, h, vec, v[i]);
        if (residual) load_chunk(residual + r[i] * h, g[i] * kVec, h, vec, res[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kDropUnroll; ++i) {
      if (r[i] >= n) continue;
      if (dropping) drop_chunk(v[i], drop, ph, static_cast<uint32_t>(g[i]), static_cast<uint32_t>(r[i]));
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[i][j] += res[i][j];
      store_chunk(y + r[i] * h, g[i] * kVec, h, vec, v[i]);
    }
  }
}

// ------------------------------------------------------------------------------------ host side
// Rows of the partial weight gradients at most (bounds the workspace): the more columns, the fewer blocks fill an SM.
int max_parts(int h) { return h <= 512 ? 2048 : h <= 2048 ? 1280 : 640; }

bool rows_vectorise(int h, std::initializer_list<const void*> ptrs) {
  if (h % kVec != 0) return false;
  for (const void* p : ptrs)
    if (p && !aligned_to(p, 16)) return false;
  return true;
}

// Drop probability as a multiple of 2^-16 and its exact scale.
Dropout make_dropout(float p, const void* rng) {
  Dropout d;
  const double t = static_cast<double>(p) * 65536.0;
  d.threshold = static_cast<uint32_t>(__builtin_rint(t));
  d.scale = d.threshold < 65536u ? static_cast<float>(65536.0 / (65536.0 - d.threshold)) : 0.f;
  d.rng = d.threshold == 0u ? nullptr : static_cast<const unsigned long long*>(rng);
  return d;
}

int check_rows(long long n, int h, a3po_dtype dt) {
  if (n < 0 || h <= 0) return A3PO_ERR_INVALID_ARG;
  if (dt != A3PO_F32 && dt != A3PO_BF16) return A3PO_ERR_UNSUPPORTED;
  if (n > 0x7fffffffll) return A3PO_ERR_UNSUPPORTED;   // one grid dimension of rows, one 32-bit counter word
  return A3PO_OK;
}

// Pointers must at least be aligned to their own elements.
bool elements_aligned(a3po_dtype dt, std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!aligned_to(p, dt == A3PO_F32 ? 4 : 2)) return false;
  return true;
}

int check_dropout(float p, const void* rng) {
  if (!(p >= 0.f && p <= 1.f)) return A3PO_ERR_INVALID_ARG;
  if (p > 0.f && !rng) return A3PO_ERR_INVALID_ARG;
  if (!aligned_to(rng, 8)) return A3PO_ERR_UNSUPPORTED;
  return A3PO_OK;
}

template <typename T, int TPR, int CPT, bool LAYER, bool JOIN>
int launch_norm_fwd(const NormFwdArgs<T>& a, cudaStream_t stream) {
  const long long blocks = (a.n + rows_per_block<TPR>() - 1) / rows_per_block<TPR>();
  A3PO_LAUNCH(kKNorm, stream, (norm_fwd_kernel<T, TPR, CPT, LAYER, JOIN>
                                   <<<static_cast<unsigned>(blocks), threads_of<TPR>(), 0, stream>>>(a)));
  return after_launch();
}

// Threads per row by row length: as few as keep at most 4 chunks (32 columns) per thread.
template <typename T, bool LAYER, bool JOIN>
int norm_fwd_impl(const NormFwdArgs<T>& a, cudaStream_t stream) {
  const int groups = (a.h + kVec - 1) / kVec;
  if (groups <= 32) return launch_norm_fwd<T, 32, 1, LAYER, JOIN>(a, stream);
  if (groups <= 128) return launch_norm_fwd<T, 32, 4, LAYER, JOIN>(a, stream);
  if (groups <= 256) return launch_norm_fwd<T, 128, 2, LAYER, JOIN>(a, stream);
  if (groups <= 512) return launch_norm_fwd<T, 256, 2, LAYER, JOIN>(a, stream);
  if (groups <= 1024) return launch_norm_fwd<T, 512, 2, LAYER, JOIN>(a, stream);
  if (groups <= 2048) return launch_norm_fwd<T, 1024, 2, LAYER, JOIN>(a, stream);
  A3PO_LAUNCH(kKNorm, stream, (norm_fwd_long_kernel<T, LAYER, JOIN>
                                   <<<static_cast<unsigned>(a.n), kLongThreads, 0, stream>>>(a)));
  return after_launch();
}

template <typename T, int TPR, int CPT, bool LAYER, bool JOIN>
int launch_norm_bwd(const NormBwdArgs<T>& a, int* parts, cudaStream_t stream) {
  int sms = sm_count();
  constexpr int kRows = rows_per_block<TPR>();
  constexpr int kThreads = threads_of<TPR>();
  long long blocks = (a.n + kRows - 1) / kRows;
  long long most = static_cast<long long>(sms) * (1024 / kThreads > 0 ? 1024 / kThreads : 1);
  if (most * kRows > max_parts(a.h)) most = max_parts(a.h) / kRows;
  if (blocks > most) blocks = most;
  *parts = static_cast<int>(blocks) * kRows;
  A3PO_LAUNCH(kKNormBwd, stream, (norm_bwd_kernel<T, TPR, CPT, LAYER, JOIN>
                                      <<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(a)));
  return after_launch();
}

template <typename T, bool LAYER, bool JOIN>
int norm_bwd_impl(const NormBwdArgs<T>& a, float* grad_gamma, float* grad_beta, int accumulate, cudaStream_t stream) {
  const int groups = (a.h + kVec - 1) / kVec;
  int parts = 0;
  if (groups <= 32) A3PO_RETURN_IF((launch_norm_bwd<T, 32, 1, LAYER, JOIN>(a, &parts, stream)));
  else if (groups <= 64) A3PO_RETURN_IF((launch_norm_bwd<T, 32, 2, LAYER, JOIN>(a, &parts, stream)));
  else if (groups <= 256) A3PO_RETURN_IF((launch_norm_bwd<T, 128, 2, LAYER, JOIN>(a, &parts, stream)));
  else if (groups <= 512) A3PO_RETURN_IF((launch_norm_bwd<T, 256, 2, LAYER, JOIN>(a, &parts, stream)));
  else if (groups <= 1024) A3PO_RETURN_IF((launch_norm_bwd<T, 512, 2, LAYER, JOIN>(a, &parts, stream)));
  else if (groups <= 2048) A3PO_RETURN_IF((launch_norm_bwd<T, 1024, 2, LAYER, JOIN>(a, &parts, stream)));
  else {
    A3PO_LAUNCH(kKNormBwd, stream, (norm_bwd_long_kernel<T, LAYER, JOIN>
                                        <<<static_cast<unsigned>(a.n), kLongThreads, 0, stream>>>(a)));
    A3PO_RETURN_IF(after_launch());
    parts = a.n < 64 ? static_cast<int>(a.n) : 64;
    const dim3 grid(static_cast<unsigned>((a.h + 255) / 256), static_cast<unsigned>(parts));
    A3PO_LAUNCH(kKNormBwd, stream, (norm_weight_long_kernel<T, LAYER><<<grid, 256, 0, stream>>>(a, parts)));
    A3PO_RETURN_IF(after_launch());
  }
  const dim3 grid(static_cast<unsigned>((a.h + kReduceCols - 1) / kReduceCols), LAYER ? 2u : 1u);
  A3PO_LAUNCH(kKNormBwd, stream, (reduce_parts_kernel<<<grid, dim3(kReduceCols, kReduceLanes), 0, stream>>>(
                                     a.part, parts, static_cast<long long>(LAYER ? 2 : 1) * a.h, a.h, accumulate,
                                     grad_gamma, grad_beta)));
  return after_launch();
}

template <typename T, bool JOIN>
int norm_fwd_typed(const void* x, const void* residual, const void* gamma, const void* beta, const uint8_t* row_mask,
                   long long n, int h, a3po_norm_kind kind, float eps, const Dropout& drop, void* r, void* y,
                   float* mean, float* rstd, cudaStream_t stream) {
  NormFwdArgs<T> a{static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<const T*>(gamma),
                   static_cast<const T*>(beta), row_mask, n, h, eps, 1.0f / static_cast<float>(h),
                   static_cast<T*>(r), static_cast<T*>(y), mean, rstd, drop,
                   rows_vectorise(h, {x, residual, gamma, beta, r, y}) ? 1 : 0};
  return kind == A3PO_NORM_LAYER ? norm_fwd_impl<T, true, JOIN>(a, stream) : norm_fwd_impl<T, false, JOIN>(a, stream);
}

template <typename T, bool JOIN>
int norm_bwd_typed(const void* x, const void* gamma, const float* mean, const float* rstd, const uint8_t* row_mask,
                   const void* grad_y, const void* grad_r, long long n, int h, a3po_norm_kind kind,
                   const Dropout& drop, void* grad_residual, void* grad_x, float* grad_gamma, float* grad_beta,
                   int accumulate, float* part, cudaStream_t stream) {
  NormBwdArgs<T> a{static_cast<const T*>(x), static_cast<const T*>(gamma), mean, rstd, row_mask,
                   static_cast<const T*>(grad_y), static_cast<const T*>(grad_r), n, h, 1.0f / static_cast<float>(h),
                   static_cast<T*>(grad_x), static_cast<T*>(grad_residual), part, drop,
                   rows_vectorise(h, {x, gamma, grad_y, grad_r, grad_x, grad_residual}) ? 1 : 0};
  return kind == A3PO_NORM_LAYER ? norm_bwd_impl<T, true, JOIN>(a, grad_gamma, grad_beta, accumulate, stream)
                                 : norm_bwd_impl<T, false, JOIN>(a, grad_gamma, grad_beta, accumulate, stream);
}

int norm_bwd_entry(bool join, const void* x, const void* gamma, const float* mean, const float* rstd,
                   const uint8_t* row_mask, const void* grad_y, const void* grad_r, long long n, int h, a3po_dtype dt,
                   a3po_norm_kind kind, float p, const void* rng, void* grad_residual, void* grad_x,
                   float* grad_gamma, float* grad_beta, int accumulate, void* ws, size_t ws_bytes,
                   cudaStream_t stream) {
  A3PO_RETURN_IF(check_rows(n, h, dt));
  if (kind != A3PO_NORM_RMS && kind != A3PO_NORM_LAYER) return A3PO_ERR_UNSUPPORTED;
  if (!gamma || !grad_gamma || (n > 0 && (!x || !rstd || !grad_y || (!join && !grad_x)))) return A3PO_ERR_INVALID_ARG;
  if (n > 0 && kind == A3PO_NORM_LAYER && !mean) return A3PO_ERR_INVALID_ARG;
  if (kind == A3PO_NORM_RMS && grad_beta) return A3PO_ERR_INVALID_ARG;   // an RMS norm has no beta gradient to give
  if (join) {
    if (n > 0 && !grad_residual) return A3PO_ERR_INVALID_ARG;
    A3PO_RETURN_IF(check_dropout(p, rng));
  }
  if (!elements_aligned(dt, {x, gamma, grad_y, grad_r, grad_residual, grad_x}) ||
      !elements_aligned(A3PO_F32, {mean, rstd, grad_gamma, grad_beta}))
    return A3PO_ERR_UNSUPPORTED;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_norm_bwd_workspace_bytes(n, h)) return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (n == 0) {
    if (accumulate) return A3PO_OK;
    if (cudaMemsetAsync(grad_gamma, 0, sizeof(float) * static_cast<size_t>(h), stream) != cudaSuccess ||
        (grad_beta && cudaMemsetAsync(grad_beta, 0, sizeof(float) * static_cast<size_t>(h), stream) != cudaSuccess)) {
      cudaGetLastError();
      return A3PO_ERR_CUDA;
    }
    return A3PO_OK;
  }
  const Dropout drop = make_dropout(join ? p : 0.f, rng);
  float* part = static_cast<float*>(ws);
#define A3PO_NORM_BWD(T, J)                                                                                       \
  norm_bwd_typed<T, J>(x, gamma, mean, rstd, row_mask, grad_y, grad_r, n, h, kind, drop, grad_residual, grad_x, \
                       grad_gamma, grad_beta, accumulate, part, stream)
  if (dt == A3PO_F32) return join ? A3PO_NORM_BWD(float, true) : A3PO_NORM_BWD(float, false);
  return join ? A3PO_NORM_BWD(__nv_bfloat16, true) : A3PO_NORM_BWD(__nv_bfloat16, false);
#undef A3PO_NORM_BWD
}

int norm_fwd_entry(bool join, const void* x, const void* residual, const void* gamma, const void* beta,
                   const uint8_t* row_mask, long long n, int h, a3po_dtype dt, a3po_norm_kind kind, float eps, float p,
                   const void* rng, void* r, void* y, float* mean, float* rstd, cudaStream_t stream) {
  A3PO_RETURN_IF(check_rows(n, h, dt));
  if (kind != A3PO_NORM_RMS && kind != A3PO_NORM_LAYER) return A3PO_ERR_UNSUPPORTED;
  if (!(eps >= 0.f)) return A3PO_ERR_INVALID_ARG;
  if (!gamma || (n > 0 && (!x || !y))) return A3PO_ERR_INVALID_ARG;
  if (kind == A3PO_NORM_RMS && mean) return A3PO_ERR_INVALID_ARG;   // an RMS norm has no mean to report
  if (join) {
    if (n > 0 && (!residual || !r)) return A3PO_ERR_INVALID_ARG;
    A3PO_RETURN_IF(check_dropout(p, rng));
  }
  if (!elements_aligned(dt, {x, residual, gamma, beta, r, y}) || !elements_aligned(A3PO_F32, {mean, rstd}))
    return A3PO_ERR_UNSUPPORTED;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (n == 0) return A3PO_OK;
  const Dropout drop = make_dropout(join ? p : 0.f, rng);
#define A3PO_NORM_FWD(T, J) \
  norm_fwd_typed<T, J>(x, residual, gamma, beta, row_mask, n, h, kind, eps, drop, r, y, mean, rstd, stream)
  if (dt == A3PO_F32) return join ? A3PO_NORM_FWD(float, true) : A3PO_NORM_FWD(float, false);
  return join ? A3PO_NORM_FWD(__nv_bfloat16, true) : A3PO_NORM_FWD(__nv_bfloat16, false);
#undef A3PO_NORM_FWD
}

int dropout_entry(const void* x, const void* residual, const uint8_t* row_mask, long long n, int h, a3po_dtype dt,
                  float p, const void* rng, void* y, cudaStream_t stream) {
  A3PO_RETURN_IF(check_rows(n, h, dt));
  if (n > 0 && (!x || !y)) return A3PO_ERR_INVALID_ARG;
  A3PO_RETURN_IF(check_dropout(p, rng));
  if (!elements_aligned(dt, {x, residual, y})) return A3PO_ERR_UNSUPPORTED;
  const int sms = sm_count();
  if (sms <= 0) return A3PO_ERR_NO_DEVICE;
  if (n == 0) return A3PO_OK;
  const Dropout drop = make_dropout(p, rng);
  const int vec = rows_vectorise(h, {x, residual, y}) ? 1 : 0;
  const long long chunks = n * ((h + kVec - 1) / kVec);
  long long blocks = (chunks + kDropThreads * kDropUnroll - 1) / (kDropThreads * kDropUnroll);
  const long long most = static_cast<long long>(sms) * 8;
  if (blocks > most) blocks = most;
  if (dt == A3PO_F32)
    A3PO_LAUNCH(kKDropout, stream, (dropout_kernel<float><<<static_cast<unsigned>(blocks), kDropThreads, 0, stream>>>(
                                       static_cast<const float*>(x), static_cast<const float*>(residual), row_mask, n,
                                       h, drop, static_cast<float*>(y), vec)));
  else
    A3PO_LAUNCH(kKDropout, stream,
                (dropout_kernel<__nv_bfloat16><<<static_cast<unsigned>(blocks), kDropThreads, 0, stream>>>(
                    static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(residual), row_mask, n, h,
                    drop, static_cast<__nv_bfloat16*>(y), vec)));
  return after_launch();
}

}  // namespace
}  // namespace a3po

using namespace a3po;

extern "C" {

int a3po_norm_fwd(const void* x, const void* gamma, const void* beta, const uint8_t* row_mask, int64_t N, int H,
                  a3po_dtype dt, a3po_norm_kind kind, float eps, void* y, float* mean, float* rstd, void* stream) {
  return norm_fwd_entry(false, x, nullptr, gamma, beta, row_mask, N, H, dt, kind, eps, 0.f, nullptr, nullptr, y, mean,
                        rstd, as_stream(stream));
}

size_t a3po_norm_bwd_workspace_bytes(int64_t N, int H) {
  if (N < 0 || H <= 0) return 0;
  const size_t parts = static_cast<size_t>(N + 7 < max_parts(H) ? N + 7 : max_parts(H));   // a block of 8 rows at most past N
  return round_up(parts * 2 * static_cast<size_t>(H) * sizeof(float), 256) + 256;
}

int a3po_norm_bwd(const void* x, const void* gamma, const float* mean, const float* rstd, const uint8_t* row_mask,
                  const void* grad_y, int64_t N, int H, a3po_dtype dt, a3po_norm_kind kind, void* grad_x,
                  float* grad_gamma, float* grad_beta, int accumulate_grad_w, void* ws, size_t ws_bytes,
                  void* stream) {
  return norm_bwd_entry(false, x, gamma, mean, rstd, row_mask, grad_y, nullptr, N, H, dt, kind, 0.f, nullptr, nullptr,
                        grad_x, grad_gamma, grad_beta, accumulate_grad_w, ws, ws_bytes, as_stream(stream));
}

int a3po_dropout_fwd(const void* x, const void* residual, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt,
                     float p, const uint64_t* rng, void* y, void* stream) {
  return dropout_entry(x, residual, row_mask, N, H, dt, p, rng, y, as_stream(stream));
}

int a3po_dropout_bwd(const void* grad_y, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt, float p,
                     const uint64_t* rng, void* grad_x, void* stream) {
  return dropout_entry(grad_y, nullptr, row_mask, N, H, dt, p, rng, grad_x, as_stream(stream));
}

int a3po_dropout_norm_fwd(const void* x, const void* residual, float p, const uint64_t* rng, const void* gamma,
                          const void* beta, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt,
                          a3po_norm_kind kind, float eps, void* r, void* y, float* mean, float* rstd, void* stream) {
  return norm_fwd_entry(true, x, residual, gamma, beta, row_mask, N, H, dt, kind, eps, p, rng, r, y, mean, rstd,
                        as_stream(stream));
}

int a3po_dropout_norm_bwd(const void* r, float p, const uint64_t* rng, const void* gamma, const float* mean,
                          const float* rstd, const uint8_t* row_mask, const void* grad_y, const void* grad_r,
                          int64_t N, int H, a3po_dtype dt, a3po_norm_kind kind, void* grad_residual, void* grad_x,
                          float* grad_gamma, float* grad_beta, int accumulate_grad_w, void* ws, size_t ws_bytes,
                          void* stream) {
  return norm_bwd_entry(true, r, gamma, mean, rstd, row_mask, grad_y, grad_r, N, H, dt, kind, p, rng, grad_residual,
                        grad_x, grad_gamma, grad_beta, accumulate_grad_w, ws, ws_bytes, as_stream(stream));
}

}  // extern "C"
