// Gated feed-forward block for a few rows (single tokens and small batches while serving): the weights are read once
// and used for at most kFewRows rows, so the bound is HBM, 2 bytes per weight, and everything serves the weight stream.
//
// The weights come through per-lane rings in shared memory (cp.async, 48 KB in flight per block, four blocks per SM; loaded
// straight to registers, 40 warps per SM kept too few bytes in flight: 3.1 TB/s) and go into mma.sync.m16n8k16 with
// the token rows as M (16 per tile) and 8 weight rows as N; at 16 flops per weight byte per row the legacy tensor path is
// far from being the limit, and it needs no staging, no barriers in the loop and no padding to 128 rows (on
// 128 x 256 tcgen05 tiles one token keeps only F / 128 of the SMs busy).  The contraction index is permuted: a lane takes
// 8 consecutive k of its row, words 0 and 1 as the fragment of one instruction, 2 and 3 as that of the next; both
// operands are taken alike, so the sum is the same sum.  A block owns 8 output columns (gate/up: the 8 rows of
// Wg and the same 8 of Wu), its warps take the 32-wide k-blocks in turn and add their accumulators up through shared
// memory in warp order, so results are bit-identical from run to run.

#include "ffn_internal.cuh"

namespace a3po {
namespace {

constexpr int kFewWarps = 8;
constexpr int kFewThreads = kFewWarps * kWarp;
constexpr int kRingBytes = 48 * 1024;   // weights in flight per block; four blocks fit an SM

__device__ __forceinline__ void copy_weight(uint32_t smem, const __nv_bfloat16* p) {   // asynchronous, past L1
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

// A lane's share of the weight stream: 16 bytes per weight block and 32-wide k-block, kDepth k-blocks ahead of their use, in
// a ring that it fills and reads alone (no barrier).  Started before x is touched, so that in the second kernel the
// weights are on their way while the first one still computes x.
template <int OUT>
struct WeightStream {
  static constexpr int kDepth = kRingBytes / (kFewThreads * 16 * OUT);
  uint32_t ring;
  const __nv_bfloat16* w[OUT];
  int k, next;   // row length; this lane's k of the next copy
  __device__ __forceinline__ void copy(int slot) {
    if (next < k) {
#pragma unroll
      for (int o = 0; o < OUT; ++o) copy_weight(ring + (slot * OUT + o) * kFewThreads * 16, w[o] + next);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    next += kFewWarps * 32;
  }
  __device__ __forceinline__ void start(uint8_t* smem, int k_, int first) {
    ring = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + threadIdx.x * 16;
    k = k_;
    next = first;
#pragma unroll
    for (int s = 0; s < kDepth; ++s) copy(s);
  }
};

// Accumulates acc[m][o] += x[16 m .. +16, :] . w_o[8 rows, :] over this warp's share of k.  A lane reads rows lane / 4
// (and + 8) of each tile of x, row lane / 4 of each weight block, 8 consecutive k each.
// MT: tiles of 16 rows; HALF: only the first 8 rows of the (single) tile exist; OUT: weight blocks.
template <int MT, bool HALF, int OUT>
__device__ __forceinline__ void sweep(const __nv_bfloat16* __restrict__ x, const bool (&row_on)[2 * MT], int n, int k,
                                      WeightStream<OUT>& ws, int warp, int lane, float (&acc)[MT][OUT][4]) {
  constexpr int kRows = HALF ? 1 : 2 * MT;
  const int sub = (lane & 3) * 8;
  const __nv_bfloat16* xr[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = lane / 4 + 8 * i;
    xr[i] = x + static_cast<long long>(r < n ? r : n - 1) * k;
  }
  const int step = kFewWarps * 32;
  uint4 ahead[kRows];   // x of the next k-block
  auto load_x = [&](int kk) {
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      ahead[i] = kk < k && row_on[i] ? *reinterpret_cast<const uint4*>(xr[i] + kk) : make_uint4(0, 0, 0, 0);
  };
  load_x(warp * 32 + sub);
  int slot = 0;
  for (int kb = warp * 32; kb < k; kb += step) {   // the same for all lanes: the instruction is warp-wide
    const int kk = kb + sub;
    uint4 xv[kRows], wv[OUT];
#pragma unroll
    for (int i = 0; i < kRows; ++i) xv[i] = ahead[i];
    load_x(kk + step);
    asm volatile("cp.async.wait_group %0;" ::"n"(WeightStream<OUT>::kDepth - 1) : "memory");
#pragma unroll
    for (int o = 0; o < OUT; ++o)   // a lane past the end of k takes part with zeros
      wv[o] = kk < k ? read_shared(ws.ring + (slot * OUT + o) * kFewThreads * 16) : make_uint4(0, 0, 0, 0);
    ws.copy(slot);
    slot = slot + 1 == WeightStream<OUT>::kDepth ? 0 : slot + 1;
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

// The block's sums: thread (row, column) of the 16 MT x 8 tile gets the total of its element over the warps, in order.
template <int MT, int OUT>
__device__ __forceinline__ void add_warps(float (&acc)[MT][OUT][4], int warp, int lane, float* sh) {
  static_assert(kFewWarps * OUT * 16 * MT * 8 * sizeof(float) <= kRingBytes, "the sums reuse the rings' memory");
  __syncthreads();   // every lane is done with its ring
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int o = 0; o < OUT; ++o)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 16 * m + lane / 4 + 8 * (e / 2), col = (lane & 3) * 2 + (e & 1);
        sh[((warp * OUT + o) * 16 * MT + row) * 8 + col] = acc[m][o][e];
      }
  __syncthreads();
}
template <int MT, int OUT>
__device__ __forceinline__ float warp_total(const float* sh, int o, int row, int col) {
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < kFewWarps; ++w) t += sh[((w * OUT + o) * 16 * MT + row) * 8 + col];
  return t;
}

template <int MT, bool HALF, bool GELU>
__global__ void __launch_bounds__(kFewThreads)
few_gate_up_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ w_gate_up,
                   const uint8_t* __restrict__ row_mask, int n, int h, int f, __nv_bfloat16* __restrict__ hid,
                   __nv_bfloat16* __restrict__ kept) {
  extern __shared__ __align__(16) uint8_t smem[];
  float* sh = reinterpret_cast<float*>(smem);   // after the sweep
  const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp;
  const int f0 = blockIdx.x * 8;
  bool on[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    const int r = lane / 4 + 8 * i;
    on[i] = r < n && (!row_mask || row_mask[r] != 0);
  }
  WeightStream<2> ws;
  ws.w[0] = w_gate_up + static_cast<long long>(f0 + lane / 4) * h;
  ws.w[1] = w_gate_up + (static_cast<long long>(f) + f0 + lane / 4) * h;
  ws.start(smem, h, warp * 32 + (lane & 3) * 8);
  float acc[MT][2][4] = {};
  sweep<MT, HALF, 2>(x, on, n, h, ws, warp, lane, acc);
  add_warps<MT, 2>(acc, warp, lane, sh);
  for (int i = threadIdx.x; i < 16 * MT * 8; i += kFewThreads) {
    const int row = i / 8, col = i % 8;
    if (row >= n) continue;
    const float g = warp_total<MT, 2>(sh, 0, row, col), u = warp_total<MT, 2>(sh, 1, row, col);
    float a, slope;
    gate_activation<GELU>(g, a, slope);
    hid[static_cast<long long>(row) * f + f0 + col] = __float2bfloat16_rn(a * u);
    if (kept) {
      __nv_bfloat16* k = kept + kept_offset(row, f0 + col, f);
      k[0] = __float2bfloat16_rn(g);
      k[kKeptElems] = __float2bfloat16_rn(u);
    }
  }
}

template <int MT, bool HALF>
__global__ void __launch_bounds__(kFewThreads)
few_down_kernel(const __nv_bfloat16* hid, const __nv_bfloat16* __restrict__ w_down, int n, int h, int f,
                __nv_bfloat16* __restrict__ y) {
  extern __shared__ __align__(16) uint8_t smem[];
  float* sh = reinterpret_cast<float*>(smem);   // after the sweep
  const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp;
  const int j0 = blockIdx.x * 8;
  bool on[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) on[i] = lane / 4 + 8 * i < n;
  WeightStream<1> ws;
  ws.w[0] = w_down + static_cast<long long>(j0 + lane / 4) * f;
  ws.start(smem, f, warp * 32 + (lane & 3) * 8);
  float acc[MT][1][4] = {};
  sweep<MT, HALF, 1>(hid, on, n, f, ws, warp, lane, acc);
  add_warps<MT, 1>(acc, warp, lane, sh);
  for (int i = threadIdx.x; i < 16 * MT * 8; i += kFewThreads) {
    const int row = i / 8, col = i % 8;
    if (row < n) y[static_cast<long long>(row) * h + j0 + col] = __float2bfloat16_rn(warp_total<MT, 1>(sh, 0, row, col));
  }
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
             int f, a3po_activation act, __nv_bfloat16* hid, __nv_bfloat16* y, __nv_bfloat16* kept, cudaStream_t s) {
  const unsigned fb = static_cast<unsigned>(f / 8), hb = static_cast<unsigned>(h / 8);
  if (act == A3PO_ACT_GELU_TANH)
    A3PO_LAUNCH(kKFfnFew, s, (few_gate_up_kernel<MT, HALF, true><<<fb, kFewThreads, kRingBytes, s>>>(x, wgu, mask, n, h, f, hid,
                                                                                            kept)));
  else
    A3PO_LAUNCH(kKFfnFew, s, (few_gate_up_kernel<MT, HALF, false><<<fb, kFewThreads, kRingBytes, s>>>(x, wgu, mask, n, h, f, hid,
                                                                                             kept)));
  A3PO_RETURN_IF(after_launch());
  A3PO_LAUNCH(kKFfnFew, s, (few_down_kernel<MT, HALF><<<hb, kFewThreads, kRingBytes, s>>>(hid, wd, n, h, f, y)));
  return after_launch();
}

}  // namespace

int ffn_few_rows_fwd(const void* x_, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, long long n,
                     int h, int f, a3po_activation act, void* hid_, void* y_, void* kept_, cudaStream_t stream) {
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(x_);
  const __nv_bfloat16* wgu = static_cast<const __nv_bfloat16*>(w_gate_up);
  const __nv_bfloat16* wd = static_cast<const __nv_bfloat16*>(w_down);
  __nv_bfloat16* hid = static_cast<__nv_bfloat16*>(hid_);
  __nv_bfloat16* y = static_cast<__nv_bfloat16*>(y_);
  __nv_bfloat16* kept = static_cast<__nv_bfloat16*>(kept_);
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
