// Products on the FP32 pipes, shared by the feed-forward block and the linear operator: fp32 operands (tcgen05 has no fp32 x fp32
// kind) and bf16 ones that the tensor-core kernels reject (see ffn_simt.cu for the tiles).
#pragma once

#include "ffn_internal.cuh"

namespace a3po {
namespace {

constexpr int kBK = 32, kSimtThreads = 256;

// Operand: element (m, k) at base[m * ms + k * ks], one of ms, ks being 1; zero outside [m_dim) x [k_dim) and where the
// token row that the element belongs to is masked out (mask null: none; the token is m where k is contiguous, else k).
template <typename T>
struct Mat {
  const T* base;
  long long ms, ks;
  long long m_dim, k_dim;
  const uint8_t* mask;
  bool k_contig;   // which of the two strides is the 1 (both are where a row has one element)
};

// One TILE x kBK slice of an operand: from memory into registers, read along its contiguous index, and from there into
// shared memory, k-major.  The next slice is on its way while the present one is multiplied.  A thread's element
// addresses differ by fixed strides, so a load costs an add and a compare besides itself.
template <typename T, int TILE>
struct Slice {
  static constexpr int kPer = TILE * kBK / kSimtThreads;
  float r[kPer];
  const T* p;          // element 0 of this thread in the slice that is loaded next
  const uint8_t* mask; // masks by token k, at that element's k
  long long i_step;    // elements from one of the thread's elements to the next
  long long k_left;    // k_dim minus element 0's k
  uint32_t rows_on;    // k contiguous: bit i, row of element i exists and is not masked out; else: all or none
  bool k_contig;

  // k contiguous: a warp takes 8 neighbours of each of 4 rows, 32 different banks of the slice's k-major rows of TILE + 4
  static __device__ __forceinline__ int k_of(int t) { return t % 8 + t / 32 % 4 * 8; }
  static __device__ __forceinline__ int row_of(int t) { return t / 8 % 4 + t / 128 * 4; }

  __device__ __forceinline__ void start(const Mat<T>& a, long long m0, long long k0) {
    const int t = threadIdx.x % kSimtThreads;
    k_contig = a.k_contig;
    rows_on = 0;
    mask = nullptr;
    if (k_contig) {
      const long long m = m0 + row_of(t), k = k0 + k_of(t);
      p = a.base + m * a.ms + k;
      i_step = (kSimtThreads / kBK) * a.ms;
      k_left = a.k_dim - k;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const long long row = m + i * (kSimtThreads / kBK);
        if (row < a.m_dim && (!a.mask || a.mask[row] != 0)) rows_on |= 1u << i;
      }
    } else {
      const long long m = m0 + t % TILE, k = k0 + t / TILE;
      p = a.base + m + k * a.ks;
      i_step = (kSimtThreads / TILE) * a.ks;
      k_left = a.k_dim - k;
      if (m < a.m_dim) rows_on = ~0u;
      if (a.mask) mask = a.mask + k;
    }
  }
  // the slice at p, then on to the one `ahead` k further
  __device__ __forceinline__ void load(const Mat<T>& a, int ahead) {
    if (k_contig) {
      const bool in = k_left > 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) r[i] = in && (rows_on >> i & 1u) ? to_float(p[i * i_step]) : 0.f;
      p += ahead;
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        constexpr int kStep = kSimtThreads / TILE;
        const bool in = rows_on && i * kStep < k_left;
        const bool on = in && (!mask || mask[i * kStep] != 0);
        r[i] = on ? to_float(p[i * i_step]) : 0.f;
      }
      p += ahead * a.ks;
      if (mask) mask += ahead;
    }
    k_left -= ahead;
  }
  __device__ __forceinline__ void store(float (*sh)[TILE + 4]) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int t = threadIdx.x % kSimtThreads, e = t + i * kSimtThreads;
      if (k_contig) sh[k_of(t)][row_of(t) + i * (kSimtThreads / kBK)] = r[i]; else sh[e / TILE][e % TILE] = r[i];
    }
  }
};

// R x R outputs per thread, 16 x 16 threads.
template <int R>
__device__ __forceinline__ void multiply(const float (*as)[16 * R + 4], const float (*bs)[16 * R + 4], float (&acc)[R][R]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x % kSimtThreads / 16;
#pragma unroll
  for (int k = 0; k < kBK; ++k) {
    float av[R], bv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) av[i] = as[k][ty * R + i];
#pragma unroll
    for (int j = 0; j < R; ++j) bv[j] = bs[k][tx * R + j];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < R; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
  }
}

// A block is G groups of 256 threads that take the slices of K in turn, so that a long K over few output tiles is not one
// block's serial loop; their sums are added in group order.
template <int R, int G>
struct Tiles {
  float a[G][kBK][16 * R + 4], b[G][kBK][16 * R + 4];
};

// acc += A's 16 R rows from m0 on times B's 16 R rows from n0 on, over all of K; the total is with group 0
template <int R, int G, typename TA, typename TB>
__device__ __forceinline__ void tile_product(const Mat<TA>& a, const Mat<TB>& b, long long m0, long long n0, Tiles<R, G>& sh,
                                             float (&acc)[R][R]) {
  const int group = threadIdx.x / kSimtThreads, t = threadIdx.x % kSimtThreads;
  Slice<TA, 16 * R> sa;
  Slice<TB, 16 * R> sb;
  sa.start(a, m0, group * kBK);
  sb.start(b, n0, group * kBK);
  sa.load(a, G * kBK);
  sb.load(b, G * kBK);
  for (long long k0 = 0; k0 < a.k_dim; k0 += G * kBK) {   // the same trips for all groups; slices past K are zeros
    __syncthreads();   // the previous slices have been read
    sa.store(sh.a[group]);
    sb.store(sh.b[group]);
    __syncthreads();
    if (k0 + G * kBK < a.k_dim) {
      sa.load(a, G * kBK);
      sb.load(b, G * kBK);
    }
    multiply<R>(sh.a[group], sh.b[group], acc);
  }
  if constexpr (G > 1) {
    float* sums = reinterpret_cast<float*>(&sh);
    static_assert(sizeof(sh) >= (G - 1) * kSimtThreads * R * R * sizeof(float), "sums reuse the slices");
    __syncthreads();
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < R * R; ++i) sums[((group - 1) * R * R + i) * kSimtThreads + t] = acc[i / R][i % R];
    }
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int g = 0; g < G - 1; ++g)
#pragma unroll
        for (int i = 0; i < R * R; ++i) acc[i / R][i % R] += sums[(g * R * R + i) * kSimtThreads + t];
    }
  }
}

__device__ __forceinline__ void activation_any(int gelu, float g, float& a, float& slope) {
  // the accurate exponential: this is the precision path
  float t = g, dt = 1.f;
  if (gelu) {
    constexpr float kTwoC = 1.5957691216057308f;
    const float c = fminf(fmaxf(g, -16.f), 16.f);
    t = kTwoC * c * fmaf(0.044715f, c * c, 1.f);
    dt = kTwoC * fmaf(3.f * 0.044715f, c * c, 1.f);
    if (g != g) t = g;
  }
  const float s = 1.f / (1.f + expf(-t));
  a = g * s;
  slope = fmaf(a * (1.f - s), dt, s);
}

// C[m, c] (+)= sum_k A(m, k) B(c, k).  beside: launched early behind a kernel of the same call that has waited for what this one
// reads; it waits for that one at its end alone (see Begin in gemm_tc.cuh).
template <typename TA, typename TB, typename TC, int R, int G>
__global__ void __launch_bounds__(kSimtThreads* G)
simt_gemm_kernel(Mat<TA> a, Mat<TB> b, TC* c, long long ldc, int accumulate, int beside) {
  constexpr int kTile = 16 * R;
  if (!beside) wait_for_previous();
  allow_next();
  extern __shared__ __align__(16) uint8_t smem[];
  Tiles<R, G>& sh = *reinterpret_cast<Tiles<R, G>*>(smem);
  const long long m0 = static_cast<long long>(blockIdx.x) * kTile, n0 = static_cast<long long>(blockIdx.y) * kTile;
  float acc[R][R] = {};
  tile_product<R, G>(a, b, m0, n0, sh, acc);
  if (beside) wait_for_previous();
  if (threadIdx.x >= kSimtThreads) return;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const long long r = m0 + threadIdx.x / 16 * R + i;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const long long col = n0 + threadIdx.x % 16 * R + j;
      if (r >= a.m_dim || col >= b.m_dim) continue;
      TC* d = c + r * ldc + col;
      *d = from_float<TC>(accumulate ? to_float(*d) + acc[i][j] : acc[i][j]);
    }
  }
}

dim3 tiles(long long m, long long c, int tile) {
  return dim3(static_cast<unsigned>((m + tile - 1) / tile), static_cast<unsigned>((c + tile - 1) / tile));
}
// Tile and K groups by the number of 64 x 64 tiles: 32 x 32 tiles and four groups where even those are one block per SM at
// most (the time is one block's serial loop); 64 x 64 and four groups up to one block per SM, two up to two, else one.
// 2,048 x 256 outputs of K = 1,536: 139 us with the first, 71 with the third.
enum class Shape { kSmall, kSplit4, kSplit2, kPlain };
Shape shape_of(long long m, long long c) {
  const dim3 t = tiles(m, c, 64);
  const long long blocks = static_cast<long long>(t.x) * t.y, sms = sm_count();
  return blocks * 4 <= sms ? Shape::kSmall : blocks <= sms ? Shape::kSplit4 : blocks <= 2 * sms ? Shape::kSplit2
                                                                                               : Shape::kPlain;
}
// Launches a kernel whose shared memory is a Tiles<R, G> (64 x 64 tiles of four groups take 68 KB).  early: not
// the first launch of a call, so that it may begin while its predecessor (one of the call's own) still runs.
template <int ID, int R, int G, typename K, typename... Args>
int launch_tiles(K kernel, dim3 grid, bool early, cudaStream_t s, Args... args) {
  constexpr int kBytes = sizeof(Tiles<R, G>);
  if (kBytes > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes) != cudaSuccess) {
    cudaGetLastError();
    return A3PO_ERR_CUDA;
  }
  A3PO_LAUNCH(ID, s, (launch_early(kernel, grid, dim3(kSimtThreads * G), kBytes, s, 1, early, args...)));
  return after_launch();
}

template <int ID, typename TA, typename TB, typename TC>
int gemm(const Mat<TA>& a, const Mat<TB>& b, TC* c, long long ldc, int accumulate, cudaStream_t s, bool beside = false) {
#define A3PO_GEMM(R, G)                                                                                              \
  launch_tiles<ID, R, G>(simt_gemm_kernel<TA, TB, TC, R, G>, tiles(a.m_dim, b.m_dim, 16 * R), true, s, a, b, c, ldc, \
                         accumulate, beside ? 1 : 0)
  switch (shape_of(a.m_dim, b.m_dim)) {
    case Shape::kSmall: return A3PO_GEMM(2, 4);
    case Shape::kSplit4: return A3PO_GEMM(4, 4);
    case Shape::kSplit2: return A3PO_GEMM(4, 2);
    default: return A3PO_GEMM(4, 1);
  }
#undef A3PO_GEMM
}

}  // namespace
}  // namespace a3po
