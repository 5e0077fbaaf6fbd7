// Gated feed-forward block on the FP32 pipes: fp32 inputs (tcgen05 has no fp32 x fp32 kind) and bf16 shapes that the
// tensor-core kernels reject (H or F not a multiple of 8).  64 x 64 x 32 tiles, 4 x 4 accumulators per thread (32 x 32 and
// 2 x 2 for small outputs), K split over thread groups of a block; the same data flow as the tensor-core path with fp32
// intermediates.  The precision path, bound by launches and latency at the sizes it is for: forward and backward of 512 rows,
// H 64, F 192, fp32: 60 us (six launches).  Not tuned for large shapes.

#include "simt_gemm.cuh"

namespace a3po {
namespace {

template <typename T, int R>
__global__ void __launch_bounds__(kSimtThreads)
simt_gate_up_kernel(Mat<T> x, Mat<T> wg, Mat<T> wu, long long n, int f, int gelu, float* __restrict__ hid,
                    float* __restrict__ kept) {
  constexpr int kTile = 16 * R;
  allow_next();
  __shared__ float xs[kBK][kTile + 4], gs[kBK][kTile + 4], us[kBK][kTile + 4];
  const long long m0 = static_cast<long long>(blockIdx.x) * kTile;
  const int n0 = blockIdx.y * kTile;
  float ag[R][R] = {}, au[R][R] = {};
  Slice<T, kTile> sx, sg, su;
  sx.start(x, m0, 0);
  sg.start(wg, n0, 0);
  su.start(wu, n0, 0);
  sx.load(x, kBK);
  sg.load(wg, kBK);
  su.load(wu, kBK);
  for (long long k0 = 0; k0 < x.k_dim; k0 += kBK) {
    __syncthreads();
    sx.store(xs);
    sg.store(gs);
    su.store(us);
    __syncthreads();
    if (k0 + kBK < x.k_dim) {
      sx.load(x, kBK);
      sg.load(wg, kBK);
      su.load(wu, kBK);
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
        kept[r * f + c] = ag[i][j];
        kept[(n + r) * f + c] = au[i][j];
      }
    }
  }
}

// dh = dy Wd with the gradient of the gate in the epilogue: z[r][0..2][c] = dg, du, h
template <typename T, int R, int G>
__global__ void __launch_bounds__(kSimtThreads* G)
simt_grad_gate_up_kernel(Mat<T> dy, Mat<T> wd, const float* kept, long long n, int f, int gelu, float* z) {
  constexpr int kTile = 16 * R;
  wait_for_previous();
  allow_next();
  extern __shared__ __align__(16) uint8_t smem[];
  Tiles<R, G>& sh = *reinterpret_cast<Tiles<R, G>*>(smem);
  const long long m0 = static_cast<long long>(blockIdx.x) * kTile;
  const int n0 = blockIdx.y * kTile;
  float acc[R][R] = {};
  tile_product<R, G>(dy, wd, m0, n0, sh, acc);
  if (threadIdx.x >= kSimtThreads) return;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const long long r = m0 + threadIdx.x / 16 * R + i;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = n0 + threadIdx.x % 16 * R + j;
      if (r >= n || c >= f) continue;
      const float g = kept[r * f + c], u = kept[(n + r) * f + c];
      float a, slope;
      activation_any(gelu, g, a, slope);
      float* out = z + r * 3 * f + c;
      out[0] = acc[i][j] * u * slope;
      out[f] = acc[i][j] * a;
      out[2ll * f] = a * u;
    }
  }
}

template <typename T>
int fwd_impl(const T* x, const T* wgu, const T* wd, const uint8_t* mask, long long n, int h, int f, int gelu, float* hid,
             T* y, float* kept, cudaStream_t s) {
  const Mat<T> xm{x, h, 1, n, h, mask, true}, wg{wgu, h, 1, f, h, nullptr, true},
      wu{wgu + static_cast<long long>(f) * h, h, 1, f, h, nullptr, true};
  if (shape_of(n, f) != Shape::kPlain)
    A3PO_LAUNCH(kKFfnSimt, s, (simt_gate_up_kernel<T, 2><<<tiles(n, f, 32), kSimtThreads, 0, s>>>(xm, wg, wu, n, f, gelu,
                                                                                                  hid, kept)));
  else
    A3PO_LAUNCH(kKFfnSimt, s, (simt_gate_up_kernel<T, 4><<<tiles(n, f, 64), kSimtThreads, 0, s>>>(xm, wg, wu, n, f, gelu,
                                                                                                  hid, kept)));
  A3PO_RETURN_IF(after_launch());
  return gemm<kKFfnSimt>(Mat<float>{hid, f, 1, n, f, nullptr, true}, Mat<T>{wd, f, 1, h, f, nullptr, true}, y, h, 0, s);
}

template <typename T, typename TG>
int bwd_impl(const T* x, const T* wgu, const T* wd, const uint8_t* mask, const float* kept, const T* gy, long long n, int h,
             int f, int gelu, float* z, T* gx, TG* gwgu, TG* gwd, int accumulate, cudaStream_t s) {
  const long long zf = 3ll * f;
  const Mat<T> dy{gy, h, 1, n, h, mask, true}, wdt{wd, 1, f, f, h, nullptr, false};
#define A3PO_GRAD_GATE(R, G) \
  launch_tiles<kKFfnSimt, R, G>(simt_grad_gate_up_kernel<T, R, G>, tiles(n, f, 16 * R), false, s, dy, wdt, kept, n, f, gelu, z)
  switch (shape_of(n, f)) {
    case Shape::kSmall: A3PO_RETURN_IF(A3PO_GRAD_GATE(2, 4)); break;
    case Shape::kSplit4: A3PO_RETURN_IF(A3PO_GRAD_GATE(4, 4)); break;
    case Shape::kSplit2: A3PO_RETURN_IF(A3PO_GRAD_GATE(4, 2)); break;
    default: A3PO_RETURN_IF(A3PO_GRAD_GATE(4, 1));
  }
#undef A3PO_GRAD_GATE
  A3PO_RETURN_IF(gemm<kKFfnSimt>(Mat<float>{z, zf, 1, n, 2ll * f, nullptr, true}, Mat<T>{wgu, 1, h, h, 2ll * f, nullptr, false}, gx,
                      h, 0, s));
  A3PO_RETURN_IF(gemm<kKFfnSimt>(Mat<float>{z, 1, zf, 2ll * f, n, nullptr, false}, Mat<T>{x, 1, h, h, n, mask, false}, gwgu, h,
                      accumulate, s));
  return gemm<kKFfnSimt>(Mat<T>{gy, 1, h, h, n, mask, false}, Mat<float>{z + 2ll * f, 1, zf, f, n, nullptr, false}, gwd, f,
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
                  h, f, gelu, hid, static_cast<B*>(y), static_cast<float*>(kept), stream);
}

int ffn_bwd_simt(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, const void* kept,
                 const void* grad_y, long long n, int h, int f, a3po_dtype dt, a3po_activation act, float* z,
                 void* grad_x, void* grad_w_gate_up, void* grad_w_down, a3po_dtype grad_dt, int accumulate,
                 cudaStream_t stream) {
  const int gelu = act == A3PO_ACT_GELU_TANH;
  using B = __nv_bfloat16;
#define A3PO_FFN_BWD(T, TG)                                                                                            \
  bwd_impl(static_cast<const T*>(x), static_cast<const T*>(w_gate_up), static_cast<const T*>(w_down), row_mask,        \
           static_cast<const float*>(kept), static_cast<const T*>(grad_y), n, h, f, gelu, z, static_cast<T*>(grad_x),      \
           static_cast<TG*>(grad_w_gate_up), static_cast<TG*>(grad_w_down), accumulate, stream)
  if (dt == A3PO_F32) return A3PO_FFN_BWD(float, float);
  return grad_dt == A3PO_F32 ? A3PO_FFN_BWD(B, float) : A3PO_FFN_BWD(B, B);
#undef A3PO_FFN_BWD
}

}  // namespace a3po
