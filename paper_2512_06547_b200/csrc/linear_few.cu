// The linear operator for a few rows (logits and projections of single tokens and small batches): the weight stream of
// few_rows.cuh with bias, activation and residual behind the sums.  Bound: HBM, 2 bytes per weight: 151,936 logits of one token of
// 4,096, 197 us (6.3 TB/s); 13 tokens of 4,608 to 1,536 are launches and latency, 8 us.

#include "few_rows.cuh"
#include "linear_internal.cuh"

namespace a3po {
namespace {

struct FewOut {
  const __nv_bfloat16 *bias, *residual;
  const uint8_t* row_mask;
  void* y;
  uint8_t* kept;
  int n, m, y_f32, act;
};

__device__ __forceinline__ void finish(const FewOut& o, int row, int col, float z) {
  const long long at = static_cast<long long>(row) * o.m + col;
  if (o.bias) z += to_float(o.bias[col]);
  if (o.kept)
    reinterpret_cast<float*>(o.kept + z_tile(row, col, o.m))[(col % kZCols / 4 * kZRows + row % kZRows) * 4 + col % 4] = z;
  float a, slope;
  if (o.act == kActNone) a = z;
  else if (o.act == kActSilu) linear_activation<kActSilu>(z, a, slope);
  else linear_activation<kActGelu>(z, a, slope);
  if (o.row_mask && o.row_mask[row] == 0) a = 0.f;
  else if (o.residual) a += to_float(o.residual[at]);
  if (o.y_f32) static_cast<float*>(o.y)[at] = a;
  else static_cast<__nv_bfloat16*>(o.y)[at] = __float2bfloat16_rn(a);
}

template <int MT, bool HALF, int S>
__global__ void __launch_bounds__(kFewThreads)
few_linear_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ w, int k, FewOut out) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp;
  const int rank = S > 1 ? static_cast<int>(blockIdx.x % S) : 0;
  const int j0 = static_cast<int>(blockIdx.x / S) * 8 * S;
  Stream<MT, HALF, S> st;
#pragma unroll
  for (int o = 0; o < S; ++o) {
    int unit = j0 + o * 8 + lane / 4;
    if (unit >= out.m) unit = out.m - 1;   // past the last column: not stored
    st.w[o] = w + static_cast<long long>(unit) * k;
  }
  const int first = (rank * kFewWarps + warp) * 32;
  st.start_weights(smem, k, first + (lane & 3) * 8, S * kFewWarps * 32);
  st.start_x(x, out.n, out.row_mask, lane);
  float acc[MT][S][4] = {};
  st.sweep(first, lane, acc);
  float* sh = reinterpret_cast<float*>(smem);
  add_warps<MT, S>(acc, warp, lane, sh);
  if (S > 1) ptx::cluster_sync_all();
  const int c0 = j0 + rank * 8;
  for (int i = threadIdx.x; i < 16 * MT * 8; i += kFewThreads) {
    const int row = i / 8, col = i % 8;
    if (row < out.n && c0 + col < out.m) finish(out, row, c0 + col, cluster_total<S>(sh, (rank * 16 * MT + row) * 8 + col));
  }
  if (S > 1) ptx::cluster_sync_all();   // the peer may still read this block's sums
}

template <int MT, bool HALF>
int few_linear(const LinearFwd& c, const FewOut& out) {
  constexpr int kSmem = ring_bytes(MT);
  const __nv_bfloat16 *x = static_cast<const __nv_bfloat16*>(c.x), *w = static_cast<const __nv_bfloat16*>(c.w);
  if (c.n > 4 && c.k >= 2048) return launch_few<kKLinearFew>(few_linear_kernel<MT, HALF, 2>, c.m, 2, kSmem, false, c.stream, x, w, c.k, out);
  return launch_few<kKLinearFew>(few_linear_kernel<MT, HALF, 1>, c.m, 1, kSmem, false, c.stream, x, w, c.k, out);
}

}  // namespace

int linear_few_rows_fwd(const LinearFwd& c) {
  const FewOut out{static_cast<const __nv_bfloat16*>(c.bias), static_cast<const __nv_bfloat16*>(c.residual), c.row_mask, c.y,
                   static_cast<uint8_t*>(c.kept), static_cast<int>(c.n), c.m, c.y_f32 ? 1 : 0, c.act};
  if (c.n <= 8) return few_linear<1, true>(c, out);
  if (c.n <= 16) return few_linear<1, false>(c, out);
  return few_linear<2, false>(c, out);
}

}  // namespace a3po
