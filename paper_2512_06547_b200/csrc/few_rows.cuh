// Weight streams of products with a few rows, shared by the feed-forward block and the linear operator: the weights are read once
// through per-lane rings in shared memory and multiplied with mma.sync, the rows as M (see ffn_few.cu for the reasons).
#pragma once

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

// Launch with a cluster of `cluster` blocks; `early`: may start before the kernel ahead of it in the stream is done.
template <int ID, typename... Params, typename... Args>
int launch_few(void (*kernel)(Params...), int columns, int cluster, int smem, bool early, cudaStream_t s, Args... args) {
  if (smem > 48 * 1024 &&
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
    cudaGetLastError();
    return A3PO_ERR_CUDA;
  }
  const int units = (columns + 8 * cluster - 1) / (8 * cluster);
  A3PO_LAUNCH(ID, s, (launch_early(kernel, static_cast<unsigned>(units * cluster), kFewThreads,
                                         static_cast<size_t>(smem), s, cluster, early, args...)));
  return after_launch();
}

// Two blocks per 16 columns once the traffic of x out of L2 counts and a block's share of k stays long enough to cover the
// cluster's two barriers.  gate/up, 8 rows: H = 4096 31 -> 26 us for the down projection (F = 12288) and 13 rows 42 -> 28 us,
// but H = 1536 gate/up 12.7 -> 16.5 us (three k-blocks per warp left).
bool pair_blocks(long long n, int k) { return n > 4 && k >= 2048; }

}  // namespace
}  // namespace a3po
