// The linear operator on the FP32 pipes: fp32 inputs, and bf16 with K or M not a multiple of 8.  The tiles of simt_gemm.cuh;
// the precision path, bound by launches and latency at the sizes it is for: 509 rows of 65 to 193 there and back 29 us replayed
// from a graph; 2,048 rows of 512 to 768 253 us (19 TFLOP/s, a quarter of the FP32 pipes).

#include "linear_internal.cuh"
#include "simt_gemm.cuh"

namespace a3po {
namespace {

__device__ __forceinline__ void any_activation(int act, float z, float& a, float& slope) {
  if (act == kActNone) {
    a = z;
    slope = 1.f;
  } else {
    activation_any(act == kActGelu, z, a, slope);
  }
}

template <typename T, typename TY, int R, int G>
__global__ void __launch_bounds__(kSimtThreads* G)
simt_linear_kernel(Mat<T> x, Mat<T> w, const T* bias, const T* residual, int act, TY* y, float* kept) {
  constexpr int kTile = 16 * R;
  extern __shared__ __align__(16) uint8_t smem[];
  Tiles<R, G>& sh = *reinterpret_cast<Tiles<R, G>*>(smem);
  const long long m0 = static_cast<long long>(blockIdx.x) * kTile, n0 = static_cast<long long>(blockIdx.y) * kTile;
  float acc[R][R] = {};
  tile_product<R, G>(x, w, m0, n0, sh, acc);
  if (threadIdx.x >= kSimtThreads) return;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const long long r = m0 + threadIdx.x / 16 * R + i;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const long long c = n0 + threadIdx.x % 16 * R + j;
      if (r >= x.m_dim || c >= w.m_dim) continue;
      const long long at = r * w.m_dim + c;
      float z = acc[i][j], a, slope;
      if (bias) z += to_float(bias[c]);
      if (kept) kept[at] = z;
      any_activation(act, z, a, slope);
      if (x.mask && x.mask[r] == 0) a = 0.f;
      else if (residual) a += to_float(residual[at]);
      y[at] = from_float<TY>(a);
    }
  }
}

// dz[r][c] in fp32 and, of kSimtSumRows rows at a time, its column sums.
template <typename T>
__global__ void __launch_bounds__(256)
simt_grad_z_kernel(const T* gy, const float* kept, const uint8_t* mask, long long n, int m, int act, float* dz, float* sums, int add) {
  __shared__ float part[8][33];
  allow_next();
  const int x = threadIdx.x % 32, ty = threadIdx.x / 32;
  const long long c = static_cast<long long>(blockIdx.y) * 32 + x, r0 = static_cast<long long>(blockIdx.x) * kSimtSumRows;
  float t = 0.f;
  if (c < m) {
    for (int i = ty; i < kSimtSumRows; i += 8) {
      const long long r = r0 + i;
      if (r >= n) break;
      float v = 0.f;
      if (!mask || mask[r] != 0) {
        float a, slope = 1.f;
        if (act != kActNone) any_activation(act, kept[r * m + c], a, slope);
        v = to_float(gy[r * m + c]) * slope;
      }
      dz[r * m + c] = v;
      t += v;
    }
  }
  part[ty][x] = t;
  __syncthreads();
  if (sums && ty == 0 && c < m) {
    t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += part[i][x];
    float* to = sums + static_cast<long long>(blockIdx.x) * m + c;
    *to = add ? *to + t : t;
  }
}

template <typename T, typename TY>
int fwd_typed(const LinearFwd& c) {
  const Mat<T> x{static_cast<const T*>(c.x), c.k, 1, c.n, c.k, c.row_mask, true};
  const Mat<T> w{static_cast<const T*>(c.w), c.k, 1, c.m, c.k, nullptr, true};
#define A3PO_SIMT_LINEAR(R, G)                                                                                             \
  launch_tiles<kKLinearSimt, R, G>(simt_linear_kernel<T, TY, R, G>, tiles(c.n, c.m, 16 * R), false, c.stream, x, w,         \
                                   static_cast<const T*>(c.bias), static_cast<const T*>(c.residual), static_cast<int>(c.act), \
                                   static_cast<TY*>(c.y), static_cast<float*>(c.kept))
  switch (shape_of(c.n, c.m)) {
    case Shape::kSmall: return A3PO_SIMT_LINEAR(2, 4);
    case Shape::kSplit4: return A3PO_SIMT_LINEAR(4, 4);
    case Shape::kSplit2: return A3PO_SIMT_LINEAR(4, 2);
    default: return A3PO_SIMT_LINEAR(4, 1);
  }
#undef A3PO_SIMT_LINEAR
}

template <typename T, typename TG>
int bwd_typed(const T* x, const T* w, const uint8_t* mask, const float* kept, const T* gy, long long n, int k, int m, int act,
              float* dz, float* sums, T* gx, TG* gw, float* gb, int accumulate, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>((n + kSimtSumRows - 1) / kSimtSumRows), static_cast<unsigned>((m + 31) / 32));
  const bool few = grid.x == 1;   // a block's sums are the bias gradient
  A3PO_LAUNCH(kKLinearSimt, s, (simt_grad_z_kernel<T><<<grid, 256, 0, s>>>(gy, kept, mask, n, m, act, dz, !gb || few ? gb : sums,
                                                                         few && accumulate)));
  A3PO_RETURN_IF(after_launch());
  // the three that follow read what that kernel wrote and share nothing else: the second and third run beside the first
  if (gw)
    A3PO_RETURN_IF(gemm<kKLinearSimt>(Mat<float>{dz, 1, m, m, n, nullptr, false}, Mat<T>{x, 1, k, k, n, mask, false}, gw, k,
                                      accumulate, s));
  if (gx)
    A3PO_RETURN_IF(gemm<kKLinearSimt>(Mat<float>{dz, m, 1, n, m, nullptr, true}, Mat<T>{w, 1, k, k, m, nullptr, false}, gx, k, 0, s,
                                      gw != nullptr));
  return gb && !few ? linear_grad_bias(sums, grid.x, nullptr, m, gb, accumulate, gw || gx, s) : A3PO_OK;
}

}  // namespace

int linear_fwd_simt(const LinearFwd& c, a3po_dtype dt) {
  using B = __nv_bfloat16;
  if (dt == A3PO_F32) return fwd_typed<float, float>(c);
  return c.y_f32 ? fwd_typed<B, float>(c) : fwd_typed<B, B>(c);
}

int linear_bwd_simt(const void* x, const void* w, const uint8_t* row_mask, const void* kept, const void* grad_y, long long n,
                    int k, int m, a3po_dtype dt, Act act, float* dz, float* sums, void* grad_x, void* grad_w,
                    a3po_dtype grad_dt, float* grad_bias, int accumulate, cudaStream_t stream) {
  using B = __nv_bfloat16;
#define A3PO_LINEAR_BWD(T, TG)                                                                                                  \
  bwd_typed(static_cast<const T*>(x), static_cast<const T*>(w), row_mask, static_cast<const float*>(kept),                        \
            static_cast<const T*>(grad_y), n, k, m, static_cast<int>(act), dz, sums, static_cast<T*>(grad_x), static_cast<TG*>(grad_w), \
            grad_bias, accumulate, stream)
  if (dt == A3PO_F32) return A3PO_LINEAR_BWD(float, float);
  return grad_dt == A3PO_F32 ? A3PO_LINEAR_BWD(B, float) : A3PO_LINEAR_BWD(B, B);
#undef A3PO_LINEAR_BWD
}

}  // namespace a3po
