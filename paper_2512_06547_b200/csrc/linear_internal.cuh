// Interfaces between the linear operator's entry points (linear.cu) and its three kernel families.
//
//   z = x W^T + b,   y = act(z) + r                                             x [N, K], W [M, K], b [M], r and y [N, M]
//   dz = dy act'(z),   dx = dz W,   dW = dz^T x,   db = sum of dz's rows,   dr = dy
#pragma once

#include "ffn_internal.cuh"
#include "lmhead_internal.cuh"

namespace a3po {

// Kept values of the forward (bf16 shapes of the tensor-core path, with an activation): z in fp32, in tiles of 128 rows and 32
// columns whose 16-byte pieces lie as the epilogues write and the backward reads them, one row per thread: piece q (4
// columns) of row r at (q * 128 + r) * 16 bytes, so that 32 rows are one contiguous 512-byte access.  fp32, because the bias
// gradient is a long sum of dy act'(z) in fp32 and should not have a 16-bit slope in it.
constexpr int kZRows = 128, kZCols = 32, kZTile = kZRows * kZCols * 4;
__host__ __device__ inline long long z_col_tiles(int m) { return (static_cast<long long>(m) + kZCols - 1) / kZCols; }
__host__ __device__ inline long long z_tile(long long row, int col, int m) {   // bytes
  return ((row / kZRows) * z_col_tiles(m) + col / kZCols) * kZTile;
}

enum Act { kActNone = 0, kActSilu = 1, kActGelu = 2 };

#ifdef __CUDACC__
template <int ACT>
__device__ __forceinline__ void linear_activation(float z, float& a, float& slope) {
  if (ACT == kActNone) {
    a = z;
    slope = 1.f;
  } else {
    gate_activation<ACT == kActGelu>(z, a, slope);
  }
}
#endif

// One forward call.  Tensor cores with a row mask: x and kept are in the compact row space of n rows, of which `count` exist;
// row_index[i] is row i's place among the `rows` rows of y and the residual.
struct LinearFwd {
  const void *x, *w, *bias, *residual;
  long long n;
  int k, m;
  Act act;
  void* y;
  bool y_f32;
  void* kept;
  float* parts;               // scratch of a K split, or null
  const uint8_t* row_mask;
  const int *row_index, *count;
  long long rows;
  uint32_t* status;
  cudaStream_t stream;
};

// ---- tcgen05 kernels (linear_tc.cu): bf16, k % 8 == 0, m % 8 == 0, 16-byte aligned operands
// cb.idx, cb.count: the rows with a nonzero mask, in order.
int linear_row_index(const uint8_t* row_mask, long long n, const CompactBuffers& cb, cudaStream_t stream);
int linear_fwd_tc(const LinearFwd& c);
// K parts of a product with few output tiles, and the fp32 scratch for them whatever y's type.
int linear_k_parts(long long n, int k, int m, bool y_f32);
size_t linear_parts_bytes(long long n, int k, int m);
// Parts of the rows for the weight gradient, and the fp32 scratch for them whatever its type.
int linear_weight_parts(long long n, int k, int m, bool grad_f32);
size_t linear_weight_parts_bytes(long long n, int k, int m);
// dz (bf16 [rows to the next multiple of 128][m], or null) and, of blocks of 128 rows, its column sums (fp32, or null) from dy and
// what was kept (add: added to what is there).  Row i is row row_index[i] of dy (null: i); rows from *count (null: n) on, and rows with row_mask 0, are zeros.
int linear_grad_z(const void* grad_y, const void* kept, long long n, int m, Act act, const int* row_index, const int* count,
                  const uint8_t* row_mask, void* dz, float* sums, int add, bool early, cudaStream_t stream);
// grad_bias (+)= the sums of `blocks` blocks (rows / 128 of *count where it is given).  beside: see Begin in gemm_tc.cuh.
int linear_grad_bias(const float* sums, long long blocks, const int* count, int m, float* grad_bias, int accumulate, bool beside,
                     cudaStream_t stream);
// grad_w[m, k] = dz^T x, grad_x = dz W (either null: not wanted), the latter's rows at row_index[i] of `rows` where that is given.
// first: the call's first launch.
int linear_grads_tc(const void* dz, const void* x, const void* w, long long n, int k, int m, void* grad_x, void* grad_w,
                    a3po_dtype grad_dt, int accumulate, float* parts, float* w_parts, const int* row_index, const int* count,
                    const uint8_t* row_mask, long long rows, bool first, uint32_t* status, cudaStream_t stream);

// ---- few rows (linear_few.cu)
int linear_few_rows_fwd(const LinearFwd& c);
inline bool linear_few(long long n, int k, int m) {
  return n <= 16 || (n <= kFewRows && static_cast<long long>(k) * m <= 20000000ll);
}

// ---- FP32 pipes (linear_simt.cu); kept: fp32 [n, m], dz: fp32 [n, m]
constexpr int kSimtSumRows = 64;   // rows of a partial column sum
int linear_fwd_simt(const LinearFwd& c, a3po_dtype dt);
int linear_bwd_simt(const void* x, const void* w, const uint8_t* row_mask, const void* kept, const void* grad_y, long long n,
                    int k, int m, a3po_dtype dt, Act act, float* dz, float* sums, void* grad_x, void* grad_w,
                    a3po_dtype grad_dt, float* grad_bias, int accumulate, cudaStream_t stream);

}  // namespace a3po
