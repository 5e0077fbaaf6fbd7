// Device pieces and interfaces of the row operators (norm, dropout, join): see row_ops.cu for the mathematics.
#pragma once

#include "a3po_common.cuh"

namespace a3po {

constexpr int kVec = 8;   // consecutive columns that one Philox call decides; 16 bytes of bf16

struct Dropout {
  const unsigned long long* rng;  // device: {seed, offset}; null = nothing is dropped
  uint32_t below;                 // (T << 16) - 1 for the threshold T >= 1: element kept iff (u16 << 16) > below
  float scale;                    // 65536 / (65536 - T), 0 when everything is dropped (T = 65536)
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
      const uint64_t p0 = static_cast<uint64_t>(c0) * 0xD2511F53u, p1 = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
      const uint32_t h0 = static_cast<uint32_t>(p0 >> 32), l0 = static_cast<uint32_t>(p0);
      const uint32_t h1 = static_cast<uint32_t>(p1 >> 32), l1 = static_cast<uint32_t>(p1);
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


constexpr int kLongThreads = 1024;
constexpr int kWideThreads = 512;      // most threads of a WIDE block
constexpr int kNarrowThreads = 256;
constexpr int kMaxRingBytes = 200 * 1024;
// Rows in flight per block: as many as fit kMaxRingBytes for the longest row of the form (2 chunks per thread: 512 threads
// of them), up to 4 of bf16 and 2 of fp32.
template <typename T> constexpr int ring_rows(int inputs, int cpt) {
  int rows = sizeof(T) == 2 ? 4 : 2;
  while (rows > 1 && static_cast<size_t>(rows) * inputs * cpt * kWideThreads * kVec * sizeof(T) > kMaxRingBytes) --rows;
  return rows;
}

#ifdef __CUDACC__
// The 8 keep decisions of one Philox call.  Kept halves compare as (half << 16) > below: the low half is shifted up, the
// high half needs no shift, because the bits under it cannot carry it over a multiple of 2^16.
__device__ __forceinline__ void keep_bits(const uint4& w, uint32_t below, bool (&keep)[kVec]) {
  const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    keep[2 * j] = (words[j] << 16) > below;
    keep[2 * j + 1] = words[j] > below;
  }
}
// d(x) + add.  Dropped elements are selected away, not multiplied by 0 (x may be infinite).  The product is rounded before the
// sum: with a scale that fp32 cannot hold (4/3, say) a fused multiply-add would carry the scale's own error into sums that
// are ties in bf16 for the exact scale, and round those the other way.
__device__ __forceinline__ float drop_add(bool keep, float x, float scale, float add) {
  return __fadd_rn(__fmul_rn(keep ? x : 0.f, scale), add);
}

__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&p);
}

// Two fp32 values in one 64-bit register: sm_100 multiplies and adds them in one instruction, each half rounded as the
// scalar instruction rounds it.  These kernels run out of instruction slots before they run out of HBM: with scalar
// arithmetic the norm's backward took 281 instructions per warp and chunk.
struct F2 {
  unsigned long long u;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.u) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ F2 f2(float both) { return f2(both, both); }
__device__ __forceinline__ float2 parts(F2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.u));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
constexpr int kPairs = kVec / 2;   // a chunk's 8 columns as pairs
// d(x) of a pair.  Scalar products: a paired one is contracted with a paired sum that follows it (see drop_add).
__device__ __forceinline__ F2 drop2(bool keep_lo, bool keep_hi, F2 x, float scale) {
  const float2 v = parts(x);
  return f2(__fmul_rn(keep_lo ? v.x : 0.f, scale), __fmul_rn(keep_hi ? v.y : 0.f, scale));
}

// One 8-column chunk as it lies in memory: 16 bytes of bf16, 32 of fp32.
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void clear() { a = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float (&x)[kVec]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = low_half(w[j]);
      x[2 * j + 1] = high_half(w[j]);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[kVec]) {
    a = make_uint4(pack_pair(x[0], x[1]), pack_pair(x[2], x[3]), pack_pair(x[4], x[5]), pack_pair(x[6], x[7]));
  }
  __device__ __forceinline__ void get(F2 (&x)[kPairs]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = f2(low_half(w[j]), high_half(w[j]));
  }
  __device__ __forceinline__ void set(const F2 (&x)[kPairs]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 v = parts(x[j]);
      w[j] = pack_pair(v.x, v.y);
    }
    a = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { __stcs(reinterpret_cast<uint4*>(p), a); }
};
template <> struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void get(float (&x)[kVec]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&x)[kVec]) {
    a = make_float4(x[0], x[1], x[2], x[3]);
    b = make_float4(x[4], x[5], x[6], x[7]);
  }
  __device__ __forceinline__ void get(F2 (&x)[kPairs]) const {
    x[0] = f2(a.x, a.y); x[1] = f2(a.z, a.w); x[2] = f2(b.x, b.y); x[3] = f2(b.z, b.w);
  }
  __device__ __forceinline__ void set(const F2 (&x)[kPairs]) {
    const float2 p = parts(x[0]), q = parts(x[1]), r = parts(x[2]), s = parts(x[3]);
    a = make_float4(p.x, p.y, q.x, q.y);
    b = make_float4(r.x, r.y, s.x, s.y);
  }
  __device__ __forceinline__ void store(float* p) const {
    __stcs(reinterpret_cast<float4*>(p), a);
    __stcs(reinterpret_cast<float4*>(p) + 1, b);
  }
};

__device__ __forceinline__ void cp_async_16(void* smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(smem))),
               "l"(gmem)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rounds to the storage type and back.
template <typename T>
__device__ __forceinline__ float as_stored(float x) { return to_float(from_float<T>(x)); }

// How the norm kernels lay rows over threads.
//   WIDE    a row per block of up to 512 threads; CPT chunks of 8 columns per thread
//   narrow  (rows of at most 512 columns) 256-thread blocks of 256 / lanes rows, lanes = a power of two
// VEC (16-byte rows): a thread's chunk i is the 8 consecutive columns from (i * tpr + tid) * 8 on; chunks come through a
// ring of kRing rows in shared memory that the thread fills with cp.async for itself and reads back alone (no barrier),
// which keeps kRing rows in flight per block without registers.
// Otherwise (rows that start at any element): within the same 256 (or 8 x lanes) columns the threads of a segment
// take every L-th column, so that a warp's element loads are contiguous.  One Philox call per thread still decides 8
// columns; its bits are handed to the lanes that own them by shuffles.
template <bool WIDE>
struct RowThreads {
  int tid, tpr, slot, rows;   // thread in row, threads per row, row in block, rows per block
  int seg, L;                 // lane within its segment, lanes per segment
  __device__ __forceinline__ explicit RowThreads(int lanes) {
    if (WIDE) {
      tid = threadIdx.x; tpr = blockDim.x; slot = 0; rows = 1;
      seg = threadIdx.x % kWarp; L = kWarp;
    } else {
      tid = threadIdx.x % lanes; tpr = lanes; slot = threadIdx.x / lanes; rows = blockDim.x / lanes;
      seg = tid; L = lanes;
    }
  }
  template <bool VEC>
  __device__ __forceinline__ int col(int i, int j) const {
    return VEC ? (i * tpr + tid) * kVec + j : (i * tpr + tid - seg) * kVec + j * L + seg;
  }
  // keep decisions of this thread's columns from the 8 of its own Philox call (all threads of the warp together)
  template <bool VEC>
  __device__ __forceinline__ void own_bits(bool (&keep)[kVec]) const {
    if (VEC) return;
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < kVec; ++j) m |= keep[j] ? 1u << j : 0u;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = j * L + seg;   // column within the segment: decided by its thread c / 8, bit c % 8
      keep[j] = (__shfl_sync(0xffffffffu, m, c / kVec, L) >> (c % kVec)) & 1u;
    }
  }
};

// Sums of V values over the threads of a row.  WIDE: the warps' sums meet in shared memory; two buffers alternate, so one
// barrier per call is enough (whoever still reads a buffer is past the barrier of the call in between before anyone
// writes it again).  Entries of warps that do not exist stay 0.
template <bool WIDE>
struct RowSum {
  static constexpr int kSlots = kWideThreads / kWarp;
  float* sh;      // [2][2][kSlots]
  int turn = 0;
  __device__ __forceinline__ explicit RowSum(float* buffer) : sh(buffer) {
    if constexpr (WIDE) {
      for (int i = threadIdx.x; i < 4 * kSlots; i += blockDim.x) sh[i] = 0.f;
      __syncthreads();
    }
  }
  template <int V>
  __device__ __forceinline__ void operator()(float (&v)[V], const RowThreads<WIDE>& rt) {
    if constexpr (WIDE) {
#pragma unroll
      for (int o = kWarp / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
      if (rt.tpr == kWarp) return;
      float* buf = sh + turn * 2 * kSlots;
      turn ^= 1;
      if (rt.seg == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) buf[i * kSlots + threadIdx.x / kWarp] = v[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float4* p = reinterpret_cast<const float4*>(buf + i * kSlots);
        float4 q = p[0];
        v[i] = (q.x + q.y) + (q.z + q.w);
        for (int w = 4; w * kWarp < rt.tpr; w += 4) {
          q = p[w / 4];
          v[i] += (q.x + q.y) + (q.z + q.w);
        }
      }
    } else {
      for (int o = rt.L / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
  }
};

// The rows of a persistent block: turn k of block b is group (k >> shift) * gridDim + b of 2^shift neighbouring units
// (a unit is the block's rows_at_once rows).  Neighbours share the sectors that hold their mask bytes and statistics, so
// all but the first of a group find them in L1; groups are dealt out in turn, so runs of padding spread over the blocks.
struct Turns {
  int shift;
  // 32-bit: units <= rows < 2^31, and what lies past the end is compared before it is used
  __device__ __forceinline__ uint32_t unit(uint32_t k) const {
    return (((k >> shift) * gridDim.x + blockIdx.x) << shift) + (k & ((1u << shift) - 1u));
  }
};
// Group size: as large as leaves every block 8 groups, at most 8 units.
inline int turn_shift(long long units, long long blocks) {
  int shift = 0;
  while (shift < 3 && (units >> (shift + 1)) >= 8 * blocks) ++shift;
  return shift;
}

// What a thread knows about its chunks: whether they exist, and (element-wise rows) the columns.
template <typename T, int CPT, bool WIDE, bool VEC>
struct Columns {
  int at[CPT];       // first column of the chunk (VEC), or of the segment's block plus this lane
  bool have[CPT];    // VEC: the whole chunk lies within the row
  int h, L;
  __device__ __forceinline__ Columns(const RowThreads<WIDE>& rt, int h_) : h(h_), L(rt.L) {
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      at[i] = rt.template col<VEC>(i, 0);
      have[i] = at[i] < h;
    }
  }
  __device__ __forceinline__ int col(int i, int j) const { return at[i] + (VEC ? j : j * L); }
  // a row's (or a parameter's) chunk i; zeros where there is no column
  __device__ __forceinline__ Raw<T> read(const T* row, int i, bool on = true) const {
    Raw<T> r;
    if constexpr (VEC) {
      if (on && have[i]) r.load(row + at[i]); else r.clear();
    } else {
      float x[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[j] = on && col(i, j) < h ? to_float(row[col(i, j)]) : 0.f;
      r.set(x);
    }
    return r;
  }
  __device__ __forceinline__ void write(T* row, int i, const Raw<T>& r) const {
    if constexpr (VEC) {
      if (have[i]) r.store(row + at[i]);
    } else {
      float x[kVec];
      r.get(x);
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (col(i, j) < h) row[col(i, j)] = from_float<T>(x[j]);
    }
  }
  __device__ __forceinline__ void write(T* row, int i, const F2 (&x)[kPairs]) const {
    Raw<T> r;
    r.set(x);
    write(row, i, r);
  }
};

// A thread's own ring of row chunks in shared memory.
template <typename T, int CPT, int INPUTS, int ROWS>
struct Ring {
  uint8_t* mine;       // this thread's 16 (or 32) bytes of the first chunk
  uint32_t pitch;      // bytes from chunk to chunk
  uint32_t stage = 0;  // row slot that is read next
  __device__ __forceinline__ explicit Ring(uint8_t* smem)
      : mine(smem + threadIdx.x * sizeof(Raw<T>)), pitch(blockDim.x * static_cast<uint32_t>(sizeof(Raw<T>))) {}
  __device__ __forceinline__ uint8_t* slot(uint32_t st, int in, int i) const {
    return mine + (st * (INPUTS * CPT) + in * CPT + i) * pitch;
  }
  __device__ __forceinline__ void fetch(uint32_t st, int in, int i, const T* src) const {
#pragma unroll
    for (int b = 0; b < static_cast<int>(sizeof(Raw<T>)) / 16; ++b)
      cp_async_16(slot(st, in, i) + 16 * b, reinterpret_cast<const uint4*>(src) + b);
  }
  __device__ __forceinline__ Raw<T> take(int in, int i, bool on) const {
    Raw<T> r;
    if (on) r = *reinterpret_cast<const Raw<T>*>(slot(stage, in, i)); else r.clear();
    return r;
  }
  // chunks past the end of the row, and inputs that are not given, are never fetched: they stay zero
  __device__ __forceinline__ void clear() const {
    Raw<T> z;
    z.clear();
#pragma unroll
    for (int st = 0; st < ROWS; ++st)
#pragma unroll
      for (int c = 0; c < INPUTS * CPT; ++c) *reinterpret_cast<Raw<T>*>(slot(st, 0, c)) = z;
  }
  __device__ __forceinline__ void advance() { stage = stage + 1 == ROWS ? 0 : stage + 1; }
};

// ---- rows longer than the register form holds: chunks of 8 consecutive columns, element by element unless `vec` ----
template <typename T>
__device__ __forceinline__ void load_chunk(const T* row, int col, int h, bool vec, float (&x)[kVec]) {
  if (vec) {
    Raw<T> r;
    if (col < h) r.load(row + col); else r.clear();
    r.get(x);
    return;
  }
#pragma unroll
  for (int j = 0; j < kVec; ++j) x[j] = (col + j < h) ? to_float(row[col + j]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int col, int h, bool vec, const float (&x)[kVec]) {
  if (vec) {
    if (col >= h) return;
    Raw<T> r;
    r.set(x);
    r.store(row + col);
    return;
  }
#pragma unroll
  for (int j = 0; j < kVec; ++j)
    if (col + j < h) row[col + j] = from_float<T>(x[j]);
}
// Sum over a block of 1024 threads.
__device__ __forceinline__ float2 block_sum2(float a, float b, float2* sh) {
  a = warp_sum(a);
  b = warp_sum(b);
  __syncthreads();
  if (threadIdx.x % kWarp == 0) sh[threadIdx.x / kWarp] = make_float2(a, b);
  __syncthreads();
  a = b = 0.f;
#pragma unroll
  for (int w = 0; w < kWarp; ++w) {
    a += sh[w].x;
    b += sh[w].y;
  }
  return make_float2(a, b);
}
#endif  // __CUDACC__

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


// Rows of the partial weight gradients at most (bounds the workspace).
inline int max_parts(int h) { return h <= 2048 ? 1280 : 640; }

// norm_fwd.cu / norm_bwd.cu
int launch_norm_fwd(const NormFwdArgs<float>& a, bool layer, bool join, cudaStream_t stream);
int launch_norm_fwd(const NormFwdArgs<__nv_bfloat16>& a, bool layer, bool join, cudaStream_t stream);
int launch_norm_bwd(const NormBwdArgs<float>& a, bool layer, bool join, float* grad_gamma, float* grad_beta,
                    int accumulate, cudaStream_t stream);
int launch_norm_bwd(const NormBwdArgs<__nv_bfloat16>& a, bool layer, bool join, float* grad_gamma, float* grad_beta,
                    int accumulate, cudaStream_t stream);

#ifdef __CUDACC__
// Blocks of a persistent kernel that fit one SM, at most `most`; raises the kernel's shared-memory limit on first use.
// 0 on a CUDA error.  The answer for the latest launch shape on each device is remembered (threads in the high half).
template <typename K>
int blocks_per_sm(K kernel, int threads, size_t smem, int most, std::atomic<uint64_t> (&cached)[64]) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return 0;
  }
  uint64_t c = cached[dev].load(std::memory_order_relaxed);
  if (static_cast<int>(c >> 32) != threads) {
    int n = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxRingBytes) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess || n < 1) {
      cudaGetLastError();
      return 0;
    }
    c = static_cast<uint64_t>(threads) << 32 | static_cast<uint64_t>(n);
    cached[dev].store(c, std::memory_order_relaxed);
  }
  const int n = static_cast<int>(c & 0xffffffffu);
  return n < most ? n : most;
}
#endif

}  // namespace a3po
