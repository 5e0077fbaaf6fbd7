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

#include "ffn_internal.cuh"
#include "sm100_ptx.cuh"

namespace a3po {
namespace {

constexpr int kFewWarps = 8;
constexpr int kFewThreads = kFewWarps * kWarp;
// Operands in flight per block: four blocks fit an SM (three with two row tiles, which need 64 KB for two k-blocks).
constexpr int ring_bytes(int mt) { return mt == 1 ? 48 * 1024 : 64 * 1024; }

__device__ __forceinline__ void copy_16(uint32_t smem, const __nv_bfloat16* p) {   // asynchronous, past L1
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(p) : "memory");
}
__device__ __forceinline__ uint4 read_shared(uint32_t smem) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem) : "memory");
  return v;
}

// d[16 x 8] += a[16 x 16] b[16 x 8]
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A lane's share of the operands of its warp's k-blocks: 16 bytes per weight block and per token row, kDepth k-blocks ahead
// of their use, in a ring in shared memory that the lane fills and reads alone (no barrier).  A lane takes rows
// lane / 4 (and + 8) of each 16-row tile of x and row lane / 4 of each weight block, 8 consecutive k each.
// MT: tiles of 16 rows; HALF: only the first 8 rows of the (single) tile exist; OUT: weight blocks.
template <int MT, bool HALF, int OUT>
struct Stream {
  static constexpr int kRows = HALF ? 1 : 2 * MT;
  static constexpr int kDepth = ring_bytes(MT) / (kFewThreads * 16 * (OUT + kRows));
  static_assert(kDepth >= 2, "at least one k-block ahead");
  uint32_t ring;
  const __nv_bfloat16* w[OUT];
  const __nv_bfloat16* xr[kRows];
  bool row_on[kRows];
  int k, step;          // row length; distance between two k-blocks of a warp
  int w_next, x_next;   // this lane's k of the next copies

  __device__ __forceinline__ uint32_t at(int slot, int o) const { return ring + (slot * (OUT + kRows) + o) * kFewThreads * 16; }
  __device__ __forceinline__ void copy_w(int slot) {
    if (w_next < k) {
#pragma unroll
      for (int o = 0; o < OUT; ++o) copy_16(at(slot, o), w[o] + w_next);
    }
    w_next += step;
  }
  __device__ __forceinline__ void copy_x(int slot) {
    if (x_next < k) {
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (row_on[i]) copy_16(at(slot, OUT + i), xr[i] + x_next);
    }
    x_next += step;
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // The weights may start before x is there.
  __device__ __forceinline__ void start_weights(uint8_t* smem, int k_, int first, int step_) {
    ring = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + threadIdx.x * 16;
    k = k_;
    step = step_;
    w_next = x_next = first;
#pragma unroll
    for (int s = 0; s < kDepth; ++s) copy_w(s);
  }
  __device__ __forceinline__ void start_x(const __nv_bfloat16* x, int n, const uint8_t* row_mask, int lane) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = lane / 4 + 8 * i;
      row_on[i] = r < n && (!row_mask || row_mask[r] != 0);
      xr[i] = x + static_cast<long long>(row_on[i] ? r : 0) * k;
    }
#pragma unroll
    for (int s = 0; s < kDepth; ++s) copy_x(s);   // the first group holds the weights of all slots too
  }
  // acc[m][o] += x[16 m .. +16, :] . w_o[8 rows, :] over this warp's k-blocks, `first` (of lane 0), first + step, ...
  __device__ __forceinline__ void sweep(int first, int lane, float (&acc)[MT][OUT][4]) {
    int slot = 0;
    for (int kb = first; kb < k; kb += step) {   // the same for all lanes: the instruction is warp-wide
      const bool in = kb + (lane & 3) * 8 < k;   // a lane past the end of k takes part with zeros
      asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
      uint4 wv[OUT], xv[kRows];
#pragma unroll
      for (int o = 0; o < OUT; ++o) wv[o] = in ? read_shared(at(slot, o)) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < kRows; ++i) xv[i] = in && row_on[i] ? read_shared(at(slot, OUT + i)) : make_uint4(0, 0, 0, 0);
      copy_w(slot);
      copy_x(slot);
      slot = slot + 1 == kDepth ? 0 : slot + 1;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const uint4 a = xv[HALF ? 0 : 2 * m];
        const uint4 b = HALF ? make_uint4(0, 0, 0, 0) : xv[HALF ? 0 : 2 * m + 1];
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
          mma_16816(acc[m][o], a.x, b.x, a.y, b.y, wv[o].x, wv[o].y);
          mma_16816(acc[m][o], a.z, b.z, a.w, b.w, wv[o].z, wv[o].w);
        }
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
};

// The block's sums over its warps, in warp order, in shared memory: sh[o][row][col], OUT x 16 MT x 8 floats.
template <int MT, int OUT>
__device__ __forceinline__ void add_warps(float (&acc)[MT][OUT][4], int warp, int lane, float* sh) {
  constexpr int kTile = OUT * 16 * MT * 8;
  static_assert(kFewWarps * kTile * sizeof(float) <= ring_bytes(MT), "the sums reuse the rings' memory");
  __syncthreads();   // every lane is done with its ring
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int o = 0; o < OUT; ++o)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 16 * m + lane / 4 + 8 * (e / 2), col = (lane & 3) * 2 + (e & 1);
        sh[warp * kTile + (o * 16 * MT + row) * 8 + col] = acc[m][o][e];
      }
  __syncthreads();
  for (int i = threadIdx.x; i < kTile; i += kFewThreads) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) t += sh[w * kTile + i];
    sh[i] = t;   // read and written by this thread alone (w = 0's entry)
  }
  __syncthreads();
}

// One element of the sums over the S blocks of a cluster, in rank order.
template <int S>
__device__ __forceinline__ float cluster_total(const float* sh, int i) {
  if constexpr (S == 1) return sh[i];
  float t = 0.f;
  const uint32_t here = static_cast<uint32_t>(__cvta_generic_to_shared(sh + i));
#pragma unroll
  for (int r = 0; r < S; ++r) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(ptx::map_to_cta(here, r)) : "memory");
    t += v;
  }
  return t;
}

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

// Launch with a cluster of `cluster` blocks; `early`: may start before the kernel ahead of it in the stream is done.
template <typename... Params, typename... Args>
int launch_few(void (*kernel)(Params...), int columns, int cluster, int smem, bool early, cudaStream_t s, Args... args) {
  if (smem > 48 * 1024 &&
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
    cudaGetLastError();
    return A3PO_ERR_CUDA;
  }
  const int units = (columns + 8 * cluster - 1) / (8 * cluster);
  A3PO_LAUNCH(kKFfnFew, s, (launch_early(kernel, static_cast<unsigned>(units * cluster), kFewThreads,
                                         static_cast<size_t>(smem), s, cluster, early, args...)));
  return after_launch();
}

// Two blocks per 16 columns once the traffic of x out of L2 counts and a block's share of k stays long enough to cover the
// cluster's two barriers.  gate/up, 8 rows: H = 4096 31 -> 26 us for the down projection (F = 12288) and 13 rows 42 -> 28 us,
// but H = 1536 gate/up 12.7 -> 16.5 us (three k-blocks per warp left).
bool pair_blocks(long long n, int k) { return n > 4 && k >= 2048; }

template <int MT, bool HALF>
int few_impl(const __nv_bfloat16* x, const __nv_bfloat16* wgu, const __nv_bfloat16* wd, const uint8_t* mask, int n, int h,
             int f, a3po_activation act, __nv_bfloat16* hid, __nv_bfloat16* y, uint8_t* kept, cudaStream_t s) {
  constexpr int kSmem = ring_bytes(MT);
  const bool gelu = act == A3PO_ACT_GELU_TANH;
  const __nv_bfloat16* hid_in = hid;
  if (pair_blocks(n, h))
    A3PO_RETURN_IF(launch_few(gelu ? few_gate_up_kernel<MT, HALF, 2, true> : few_gate_up_kernel<MT, HALF, 2, false>, f, 2,
                              kSmem, false, s, x, wgu, mask, n, h, f, hid, kept));
  else
    A3PO_RETURN_IF(launch_few(gelu ? few_gate_up_kernel<MT, HALF, 1, true> : few_gate_up_kernel<MT, HALF, 1, false>, f, 1,
                              kSmem, false, s, x, wgu, mask, n, h, f, hid, kept));
  if (pair_blocks(n, f)) return launch_few(few_down_kernel<MT, HALF, 2>, h, 2, kSmem, true, s, hid_in, wd, n, h, f, y);
  return launch_few(few_down_kernel<MT, HALF, 1>, h, 1, kSmem, true, s, hid_in, wd, n, h, f, y);
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
