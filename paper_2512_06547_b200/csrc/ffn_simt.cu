// Gated feed-forward block on the FP32 pipes: fp32 inputs (tcgen05 has no fp32 x fp32 kind) and bf16 shapes that the
// tensor-core kernels reject (H or F not a multiple of 8).  64 x 64 x 32 tiles, 4 x 4 accumulators per thread (32 x 32
// and 2 x 2 for small outputs), the same data flow as the tensor-core path with fp32 intermediates.  The precision path: not tuned beyond that.

#include "ffn_internal.cuh"

namespace a3po {
namespace {

constexpr int kBK = 32, kSimtThreads = 256;

// Element (m, k) of an operand: base[m * ms + k * ks], zero outside [m_dim) x [k_dim) and where the token row that
// the element belongs to is masked out (mask_on_m: the token is m, else k; mask null: none).
template <typename T>
struct Mat {
  const T* base;
  long long ms, ks;
  long long m_dim, k_dim;
  const uint8_t* mask;
  bool mask_on_m;
  __device__ __forceinline__ float at(long long m, long long k) const {
    if (m >= m_dim || k >= k_dim) return 0.f;
    const float v = to_float(base[m * ms + k * ks]);
    if (mask && mask[mask_on_m ? m : k] == 0) return 0.f;   // selected, whatever v is; both loads are in flight at once
    return v;
  }
};

// One TILE x kBK slice of an operand: from memory into registers, read along its contiguous index, and from there into
// shared memory, k-major.  The next slice is on its way while the present one is multiplied.
template <typename T, int TILE>
struct Slice {
  static constexpr int kPer = TILE * kBK / kSimtThreads;
  float r[kPer];
  __device__ __forceinline__ void load(const Mat<T>& a, long long m0, long long k0) {
    const bool k_contig = a.ks == 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = threadIdx.x + i * kSimtThreads;
      r[i] = k_contig ? a.at(m0 + e / kBK, k0 + e % kBK) : a.at(m0 + e % TILE, k0 + e / TILE);
    }
  }
  __device__ __forceinline__ void store(const Mat<T>& a, float (*sh)[TILE + 4]) const {
    const bool k_contig = a.ks == 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = threadIdx.x + i * kSimtThreads;
      if (k_contig) sh[e % kBK][e / kBK] = r[i]; else sh[e / TILE][e % TILE] = r[i];
    }
  }
};

// R x R outputs per thread, 16 x 16 threads.
template <int R>
__device__ __forceinline__ void multiply(const float (*as)[16 * R + 4], const float (*bs)[16 * R + 4], float (&acc)[R][R]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
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

// acc += A's TILE rows from m0 on times B's TILE rows from n0 on, over all of K
template <int R, typename TA, typename TB>
__device__ __forceinline__ void tile_product(const Mat<TA>& a, const Mat<TB>& b, long long m0, long long n0,
                                             float (*as)[16 * R + 4], float (*bs)[16 * R + 4], float (&acc)[R][R]) {
  Slice<TA, 16 * R> sa;
  Slice<TB, 16 * R> sb;
  sa.load(a, m0, 0);
  sb.load(b, n0, 0);
  for (long long k0 = 0; k0 < a.k_dim; k0 += kBK) {
    __syncthreads();   // the previous slices have been read
    sa.store(a, as);
    sb.store(b, bs);
    __syncthreads();
    if (k0 + kBK < a.k_dim) {
      sa.load(a, m0, k0 + kBK);
      sb.load(b, n0, k0 + kBK);
    }
    multiply<R>(as, bs, acc);
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

template <typename T, int R>
__global__ void __launch_bounds__(kSimtThreads)
simt_gate_up_kernel(Mat<T> x, Mat<T> wg, Mat<T> wu, long long n, int f, int gelu, float* __restrict__ hid,
                    T* __restrict__ kept) {
  constexpr int kTile = 16 * R;
  __shared__ float xs[kBK][kTile + 4], gs[kBK][kTile + 4], us[kBK][kTile + 4];
  const long long m0 = static_cast<long long>(blockIdx.x) * kTile;
  const int n0 = blockIdx.y * kTile;
  float ag[R][R] = {}, au[R][R] = {};
  Slice<T, kTile> sx, sg, su;
  sx.load(x, m0, 0);
  sg.load(wg, n0, 0);
  su.load(wu, n0, 0);
  for (long long k0 = 0; k0 < x.k_dim; k0 += kBK) {
    __syncthreads();
    sx.store(x, xs);
    sg.store(wg, gs);
    su.store(wu, us);
    __syncthreads();
    if (k0 + kBK < x.k_dim) {
      sx.load(x, m0, k0 + kBK);
      sg.load(wg, n0, k0 + kBK);
      su.load(wu, n0, k0 + kBK);
    }
    multiply<R>(xs, gs, ag);
    multiply<R>(xs, us, au);
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const long long r = m0 + threadIdx.x / 16 * R + i;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = n0 + threadIdx.x % 16 * R + j;
      if (r >= n || c >= f) continue;
      float a, slope;
      activation_any(gelu, ag[i][j], a, slope);
      hid[r * f + c] = a * au[i][j];
      if (kept) {
        kept[r * f + c] = from_float<T>(ag[i][j]);
        kept[(n + r) * f + c] = from_float<T>(au[i][j]);
      }
    }
  }
}

// C[m, c] (+)= sum_k A(m, k) B(c, k)
template <typename TA, typename TB, typename TC, int R>
__global__ void __launch_bounds__(kSimtThreads)
simt_gemm_kernel(Mat<TA> a, Mat<TB> b, TC* __restrict__ c, long long ldc, int accumulate) {
  constexpr int kTile = 16 * R;
  __shared__ float as[kBK][kTile + 4], bs[kBK][kTile + 4];
  const long long m0 = static_cast<long long>(blockIdx.x) * kTile, n0 = static_cast<long long>(blockIdx.y) * kTile;
  float acc[R][R] = {};
  tile_product<R>(a, b, m0, n0, as, bs, acc);
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

// dh = dy Wd with the gradient of the gate in the epilogue: z[r][0..2][c] = dg, du, h
template <typename T, int R>
__global__ void __launch_bounds__(kSimtThreads)
simt_grad_gate_up_kernel(Mat<T> dy, Mat<T> wd, const T* __restrict__ kept, long long n, int f, int gelu,
                         float* __restrict__ z) {
  constexpr int kTile = 16 * R;
  __shared__ float as[kBK][kTile + 4], bs[kBK][kTile + 4];
  const long long m0 = static_cast<long long>(blockIdx.x) * kTile;
  const int n0 = blockIdx.y * kTile;
  float acc[R][R] = {};
  tile_product<R>(dy, wd, m0, n0, as, bs, acc);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const long long r = m0 + threadIdx.x / 16 * R + i;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = n0 + threadIdx.x % 16 * R + j;
      if (r >= n || c >= f) continue;
      const float g = to_float(kept[r * f + c]), u = to_float(kept[(n + r) * f + c]);
      float a, slope;
      activation_any(gelu, g, a, slope);
      float* out = z + r * 3 * f + c;
      out[0] = acc[i][j] * u * slope;
      out[f] = acc[i][j] * a;
      out[2ll * f] = a * u;
    }
  }
}

dim3 tiles(long long m, long long c, int tile) {
  return dim3(static_cast<unsigned>((m + tile - 1) / tile), static_cast<unsigned>((c + tile - 1) / tile));
}
// 32 x 32 tiles where 64 x 64 ones would leave most SMs without a block: the time is then that of one block's K loop,
// which a quarter of the outputs per thread makes three times shorter.
bool small_tiles(long long m, long long c) {
  const dim3 t = tiles(m, c, 64);
  return static_cast<long long>(t.x) * t.y < sm_count();
}

template <typename TA, typename TB, typename TC>
int gemm(const Mat<TA>& a, const Mat<TB>& b, TC* c, long long ldc, int accumulate, cudaStream_t s) {
  if (small_tiles(a.m_dim, b.m_dim))
    A3PO_LAUNCH(kKFfnSimt, s, (simt_gemm_kernel<TA, TB, TC, 2><<<tiles(a.m_dim, b.m_dim, 32), kSimtThreads, 0, s>>>(
                                  a, b, c, ldc, accumulate)));
  else
    A3PO_LAUNCH(kKFfnSimt, s, (simt_gemm_kernel<TA, TB, TC, 4><<<tiles(a.m_dim, b.m_dim, 64), kSimtThreads, 0, s>>>(
                                  a, b, c, ldc, accumulate)));
  return after_launch();
}

template <typename T>
int fwd_impl(const T* x, const T* wgu, const T* wd, const uint8_t* mask, long long n, int h, int f, int gelu, float* hid,
             T* y, T* kept, cudaStream_t s) {
  const Mat<T> xm{x, h, 1, n, h, mask, true}, wg{wgu, h, 1, f, h, nullptr, false},
      wu{wgu + static_cast<long long>(f) * h, h, 1, f, h, nullptr, false};
  if (small_tiles(n, f))
    A3PO_LAUNCH(kKFfnSimt, s, (simt_gate_up_kernel<T, 2><<<tiles(n, f, 32), kSimtThreads, 0, s>>>(xm, wg, wu, n, f, gelu,
                                                                                                  hid, kept)));
  else
    A3PO_LAUNCH(kKFfnSimt, s, (simt_gate_up_kernel<T, 4><<<tiles(n, f, 64), kSimtThreads, 0, s>>>(xm, wg, wu, n, f, gelu,
                                                                                                  hid, kept)));
  A3PO_RETURN_IF(after_launch());
  return gemm(Mat<float>{hid, f, 1, n, f, nullptr, false}, Mat<T>{wd, f, 1, h, f, nullptr, false}, y, h, 0, s);
}

template <typename T, typename TG>
int bwd_impl(const T* x, const T* wgu, const T* wd, const uint8_t* mask, const T* kept, const T* gy, long long n, int h,
             int f, int gelu, float* z, T* gx, TG* gwgu, TG* gwd, int accumulate, cudaStream_t s) {
  const long long zf = 3ll * f;
  const Mat<T> dy{gy, h, 1, n, h, mask, true}, wdt{wd, 1, f, f, h, nullptr, false};
  if (small_tiles(n, f))
    A3PO_LAUNCH(kKFfnSimt, s, (simt_grad_gate_up_kernel<T, 2><<<tiles(n, f, 32), kSimtThreads, 0, s>>>(dy, wdt, kept, n, f,
                                                                                                       gelu, z)));
  else
    A3PO_LAUNCH(kKFfnSimt, s, (simt_grad_gate_up_kernel<T, 4><<<tiles(n, f, 64), kSimtThreads, 0, s>>>(dy, wdt, kept, n, f,
                                                                                                       gelu, z)));
  A3PO_RETURN_IF(after_launch());
  A3PO_RETURN_IF(gemm(Mat<float>{z, zf, 1, n, 2ll * f, nullptr, false}, Mat<T>{wgu, 1, h, h, 2ll * f, nullptr, false}, gx,
                      h, 0, s));
  A3PO_RETURN_IF(gemm(Mat<float>{z, 1, zf, 2ll * f, n, nullptr, false}, Mat<T>{x, 1, h, h, n, mask, false}, gwgu, h,
                      accumulate, s));
  return gemm(Mat<T>{gy, 1, h, h, n, mask, false}, Mat<float>{z + 2ll * f, 1, zf, f, n, nullptr, false}, gwd, f,
              accumulate, s);
}

}  // namespace

int ffn_fwd_simt(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, long long n, int h,
                 int f, a3po_dtype dt, a3po_activation act, float* hid, void* y, void* kept, cudaStream_t stream) {
  const int gelu = act == A3PO_ACT_GELU_TANH;
  if (dt == A3PO_F32)
    return fwd_impl(static_cast<const float*>(x), static_cast<const float*>(w_gate_up), static_cast<const float*>(w_down),
                    row_mask, n, h, f, gelu, hid, static_cast<float*>(y), static_cast<float*>(kept), stream);
  using B = __nv_bfloat16;
  return fwd_impl(static_cast<const B*>(x), static_cast<const B*>(w_gate_up), static_cast<const B*>(w_down), row_mask, n,
                  h, f, gelu, hid, static_cast<B*>(y), static_cast<B*>(kept), stream);
}

int ffn_bwd_simt(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, const void* kept,
                 const void* grad_y, long long n, int h, int f, a3po_dtype dt, a3po_activation act, float* z,
                 void* grad_x, void* grad_w_gate_up, void* grad_w_down, a3po_dtype grad_dt, int accumulate,
                 cudaStream_t stream) {
  const int gelu = act == A3PO_ACT_GELU_TANH;
  using B = __nv_bfloat16;
#define A3PO_FFN_BWD(T, TG)                                                                                            \
  bwd_impl(static_cast<const T*>(x), static_cast<const T*>(w_gate_up), static_cast<const T*>(w_down), row_mask,        \
           static_cast<const T*>(kept), static_cast<const T*>(grad_y), n, h, f, gelu, z, static_cast<T*>(grad_x),      \
           static_cast<TG*>(grad_w_gate_up), static_cast<TG*>(grad_w_down), accumulate, stream)
  if (dt == A3PO_F32) return A3PO_FFN_BWD(float, float);
  return grad_dt == A3PO_F32 ? A3PO_FFN_BWD(B, float) : A3PO_FFN_BWD(B, B);
#undef A3PO_FFN_BWD
}

}  // namespace a3po
