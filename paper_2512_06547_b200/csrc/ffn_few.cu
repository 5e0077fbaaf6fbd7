// Gated feed-forward block for a few rows (single tokens and small batches while serving): the weights are read once
// and used for at most kFewRows rows (few_rows() says when), so the bound is HBM, 2 bytes per weight, and everything
// serves the weight stream.
//
// The weights come through per-lane rings in shared memory (cp.async, 48 KB in flight per block, four blocks per SM; loaded
// straight to registers, 40 warps per SM kept too few bytes in flight: 3.1 TB/s) and go into mma.sync.m16n8k16 with
// the token rows as M (16 per tile) and 8 weight rows as N; at one flop per weight byte and row the legacy tensor path is
// far from being the limit, and it needs no staging, no barriers in the loop and no padding to 128 rows (on
// 128 x 256 tcgen05 tiles one token keeps only F / 128 of the SMs busy).  4096 x 12288: one row 58 us (5.2 TB/s of 302 MB), 13
// rows of 1536 x 4608 19 us.  The contraction index is permuted: a lane takes
// 8 consecutive k of its row, words 0 and 1 as the fragment of one instruction, 2 and 3 as that of the next; both
// operands are taken alike, so the sum is the same sum.  A block owns 8 output columns (gate/up: the 8 rows of
// Wg and the same 8 of Wu), its warps take the 32-wide k-blocks in turn and add their accumulators up through shared
// memory in warp order, so results are bit-identical from run to run.

#include "few_rows.cuh"

namespace a3po {
namespace {

// S = 2: a cluster of two blocks owns 16 output columns and each block sweeps half of k.  The rows of x are then read half
// as often as by two blocks with 8 columns each; for more than a few rows that traffic out of L2, not HBM, is the limit.
template <int MT, bool HALF, int S, bool GELU>
__global__ void __launch_bounds__(kFewThreads)
few_gate_up_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ w_gate_up,
                   const uint8_t* __restrict__ row_mask, int n, int h, int f, __nv_bfloat16* __restrict__ hid,
                   uint8_t* __restrict__ kept) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int OUT = 2 * S;   // gate blocks, then up blocks
  const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp;
  const int rank = S > 1 ? static_cast<int>(blockIdx.x % S) : 0;
  const int f0 = static_cast<int>(blockIdx.x / S) * 8 * S;
  allow_next();
  Stream<MT, HALF, OUT> st;
#pragma unroll
  for (int o = 0; o < OUT; ++o) {
    int unit = f0 + (o % S) * 8 + lane / 4;
    if (unit >= f) unit = f - 1;   // f is a multiple of 8, not of 16: the last block's columns past f are not stored
    st.w[o] = w_gate_up + (static_cast<long long>(o / S) * f + unit) * h;
  }
  const int first = (rank * kFewWarps + warp) * 32;
  st.start_weights(smem, h, first + (lane & 3) * 8, S * kFewWarps * 32);
  st.start_x(x, n, row_mask, lane);
  float acc[MT][OUT][4] = {};
  st.sweep(first, lane, acc);
  float* sh = reinterpret_cast<float*>(smem);
  add_warps<MT, OUT>(acc, warp, lane, sh);
  if (S > 1) ptx::cluster_sync_all();
  const int c0 = f0 + rank * 8;   // this block finishes its 8 of the cluster's columns
  for (int i = threadIdx.x; i < 16 * MT * 8; i += kFewThreads) {
    const int row = i / 8, col = i % 8;
    if (row >= n || c0 >= f) continue;
    const float g = cluster_total<S>(sh, (rank * 16 * MT + row) * 8 + col);
    const float u = cluster_total<S>(sh, ((S + rank) * 16 * MT + row) * 8 + col);
    float a, slope;
    gate_activation<GELU>(g, a, slope);
    // bf16: the operand of the second product's matrix instruction, as on tiles (half a step, 2^-8 of an element at most)
    hid[static_cast<long long>(row) * f + c0 + col] = __float2bfloat16_rn(a * u);
    if (kept) {
      const int c = c0 + col, j = c % kKeptCols;
      uint8_t* tile = kept + kept_tile(row, c, f);
      uint8_t* upper = tile + (j / 8 * kKeptRows + row) * 16 + j % 8 * 2;
      uint8_t* third = tile + 2 * kKeptUpper + (j / 16 * kKeptRows + row) * 16 + j % 16;
      *reinterpret_cast<uint16_t*>(upper) = static_cast<uint16_t>(__float_as_uint(g) >> 16);
      *reinterpret_cast<uint16_t*>(upper + kKeptUpper) = static_cast<uint16_t>(__float_as_uint(u) >> 16);
      *third = static_cast<uint8_t>(__float_as_uint(g) >> 8);
      third[kKeptThird] = static_cast<uint8_t>(__float_as_uint(u) >> 8);
    }
  }
  if (S > 1) ptx::cluster_sync_all();   // the peer may still read this block's sums
}

// Launched while the first kernel still runs (programmatic dependent launch): the weights start at once, x = h is
// waited for.
template <int MT, bool HALF, int S>
__global__ void __launch_bounds__(kFewThreads)
few_down_kernel(const __nv_bfloat16* hid, const __nv_bfloat16* __restrict__ w_down, int n, int h, int f,
                __nv_bfloat16* __restrict__ y) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp;
  const int rank = S > 1 ? static_cast<int>(blockIdx.x % S) : 0;
  const int j0 = static_cast<int>(blockIdx.x / S) * 8 * S;
  Stream<MT, HALF, S> st;
#pragma unroll
  for (int o = 0; o < S; ++o) {
    int unit = j0 + o * 8 + lane / 4;
    if (unit >= h) unit = h - 1;
    st.w[o] = w_down + static_cast<long long>(unit) * f;
  }
  const int first = (rank * kFewWarps + warp) * 32;
  st.start_weights(smem, f, first + (lane & 3) * 8, S * kFewWarps * 32);
  wait_for_previous();
  allow_next();
  st.start_x(hid, n, nullptr, lane);
  float acc[MT][S][4] = {};
  st.sweep(first, lane, acc);
  float* sh = reinterpret_cast<float*>(smem);
  add_warps<MT, S>(acc, warp, lane, sh);
  if (S > 1) ptx::cluster_sync_all();
  const int c0 = j0 + rank * 8;
  for (int i = threadIdx.x; i < 16 * MT * 8; i += kFewThreads) {
    const int row = i / 8, col = i % 8;
    if (row < n && c0 < h)
      y[static_cast<long long>(row) * h + c0 + col] = __float2bfloat16_rn(cluster_total<S>(sh, (rank * 16 * MT + row) * 8 + col));
  }
  if (S > 1) ptx::cluster_sync_all();
}

__global__ void __launch_bounds__(256)
select_rows_kernel(const uint4* __restrict__ src, const uint8_t* __restrict__ row_mask, long long n, int vec_per_row,
                   uint4* __restrict__ dst) {
  const long long total = n * vec_per_row;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < total;
       i += static_cast<long long>(gridDim.x) * 256)
    dst[i] = row_mask[i / vec_per_row] ? src[i] : make_uint4(0, 0, 0, 0);
}

template <int MT, bool HALF>
int few_impl(const __nv_bfloat16* x, const __nv_bfloat16* wgu, const __nv_bfloat16* wd, const uint8_t* mask, int n, int h,
             int f, a3po_activation act, __nv_bfloat16* hid, __nv_bfloat16* y, uint8_t* kept, cudaStream_t s) {
  constexpr int kSmem = ring_bytes(MT);
  const bool gelu = act == A3PO_ACT_GELU_TANH;
  const __nv_bfloat16* hid_in = hid;
  if (pair_blocks(n, h))
    A3PO_RETURN_IF(launch_few<kKFfnFew>(gelu ? few_gate_up_kernel<MT, HALF, 2, true> : few_gate_up_kernel<MT, HALF, 2, false>, f, 2,
                              kSmem, false, s, x, wgu, mask, n, h, f, hid, kept));
  else
    A3PO_RETURN_IF(launch_few<kKFfnFew>(gelu ? few_gate_up_kernel<MT, HALF, 1, true> : few_gate_up_kernel<MT, HALF, 1, false>, f, 1,
                              kSmem, false, s, x, wgu, mask, n, h, f, hid, kept));
  if (pair_blocks(n, f)) return launch_few<kKFfnFew>(few_down_kernel<MT, HALF, 2>, h, 2, kSmem, true, s, hid_in, wd, n, h, f, y);
  return launch_few<kKFfnFew>(few_down_kernel<MT, HALF, 1>, h, 1, kSmem, true, s, hid_in, wd, n, h, f, y);
}

}  // namespace

int ffn_few_rows_fwd(const void* x_, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, long long n,
                     int h, int f, a3po_activation act, void* hid_, void* y_, void* kept_, cudaStream_t stream) {
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(x_);
  const __nv_bfloat16* wgu = static_cast<const __nv_bfloat16*>(w_gate_up);
  const __nv_bfloat16* wd = static_cast<const __nv_bfloat16*>(w_down);
  __nv_bfloat16* hid = static_cast<__nv_bfloat16*>(hid_);
  __nv_bfloat16* y = static_cast<__nv_bfloat16*>(y_);
  uint8_t* kept = static_cast<uint8_t*>(kept_);
  const int rows = static_cast<int>(n);
  if (n <= 8) return few_impl<1, true>(x, wgu, wd, row_mask, rows, h, f, act, hid, y, kept, stream);
  if (n <= 16) return few_impl<1, false>(x, wgu, wd, row_mask, rows, h, f, act, hid, y, kept, stream);
  return few_impl<2, false>(x, wgu, wd, row_mask, rows, h, f, act, hid, y, kept, stream);
}

int ffn_select_rows(const void* src, const uint8_t* row_mask, long long n, int h, void* dst, cudaStream_t stream) {
  const long long want = (n * (h / 8) + 255) / 256;
  const int blocks = static_cast<int>(want < sm_count() * 8ll ? want : sm_count() * 8ll);
  if (blocks < 1) return A3PO_OK;
  A3PO_LAUNCH(kKFfnFew, stream, (select_rows_kernel<<<blocks, 256, 0, stream>>>(
                                    static_cast<const uint4*>(src), row_mask, n, h / 8, static_cast<uint4*>(dst))));
  return after_launch();
}

}  // namespace a3po
