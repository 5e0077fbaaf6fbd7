// Interfaces between the feed-forward block's entry points (ffn.cu) and its three kernel families.
//
//   g = x Wg^T,  u = x Wu^T,  a = act(g),  h = a u,  y = h Wd^T                 Wg | Wu stacked: [2 F, H];  Wd: [H, F]
//   dh = dy Wd,  dg = dh u act'(g),  du = dh a,  dx = dg Wg + du Wu
//   dWd = dy^T h,  dWg = dg^T x,  dWu = du^T x
#pragma once

#include "a3po_common.cuh"

namespace a3po {

// Kept values of the forward (bf16 shapes of the tensor-core path): g and u in 24 bits each (the upper 24 of the fp32 value),
// as the backward's epilogue reads them, one accumulator row per thread.  bf16 would be a third less, but its rounding
// of g and u is then the largest error of grad_x and grad_w_gate_up (2-norm 0.0030 against 0.0024, of which the
// rounding of dg, du and of the results themselves is the rest); 24 bits unpack with one byte permutation per value.
// Tile (128 rows, 32 columns), 24 KB: upper halves of g, of u, third bytes of g, of u.  Inside, 16-byte piece j of row r
// sits at (j * 128 + r) * 16 bytes (8 columns a piece, 16 for the third bytes), so that the 32 rows of a warp are one
// contiguous 512-byte access.
// h itself follows the tiles, row-major [n, f] bf16: the forward writes it for its second product anyway, and the backward
// then need not write it again.
constexpr int kKeptRows = 128;
constexpr int kKeptCols = 32;
constexpr int kKeptUpper = kKeptRows * kKeptCols * 2;   // bytes of the upper halves of g (or u) in a tile
constexpr int kKeptThird = kKeptRows * kKeptCols;       // bytes of the third bytes
constexpr int kKeptTile = 2 * (kKeptUpper + kKeptThird);
__host__ __device__ inline long long kept_col_tiles(int f) { return (static_cast<long long>(f) + kKeptCols - 1) / kKeptCols; }
// Byte offset of the tile that holds column `col` of row `row`.
__host__ __device__ inline long long kept_tile(long long row, int col, int f) {
  return ((row / kKeptRows) * kept_col_tiles(f) + col / kKeptCols) * kKeptTile;
}
// Bytes of g and u, after which h starts.
inline size_t kept_gate_bytes(long long n, int f) {
  return static_cast<size_t>((n + kKeptRows - 1) / kKeptRows) * static_cast<size_t>(kept_col_tiles(f)) * kKeptTile;
}

#ifdef __CUDACC__
// a = g s(t), with s the logistic function: t = g (SiLU), or t = 2 sqrt(2 / pi) (g + 0.044715 g^3), which is
// g (1 + tanh(t / 2)) / 2, the tanh form of GELU.  slope = s + g s (1 - s) t'.
// The GELU polynomial is evaluated at g limited to [-16, 16], where s has long been 0 or 1 in fp32, so that its cube
// and derivative stay finite for any g.
template <bool GELU>
__device__ __forceinline__ void gate_activation(float g, float& a, float& slope) {
  float t = g, dt = 1.f;
  if (GELU) {
    constexpr float kTwoC = 1.5957691216057308f;   // 2 sqrt(2 / pi)
    const float c = fminf(fmaxf(g, -16.f), 16.f);
    const float c2 = c * c;
    t = kTwoC * c * fmaf(0.044715f, c2, 1.f);
    dt = kTwoC * fmaf(3.f * 0.044715f, c2, 1.f);
    if (g != g) t = g;   // fmin / fmax would hide a NaN
  }
  const float s = fast_rcp(1.f + fast_exp2(-kLog2e * t));
  a = g * s;
  slope = fmaf(a * (1.f - s), dt, s);
}
#endif

// ---- tcgen05 kernels (ffn_tc.cu): bf16, h % 8 == 0, f % 8 == 0, 16-byte aligned operands ----
// `dyn_rows` (device, may be null): rows really present of the n that the buffers hold.
// hid[n, f] = act(x Wg^T) * (x Wu^T); kept: see above, or null.
int ffn_gate_up_tc(const void* x, const void* w_gate_up, long long n, int h, int f, a3po_activation act, void* hid,
                   void* kept, const int* dyn_rows, uint32_t* status, cudaStream_t stream);
// K parts that C[n, cols] = A[n, k] B wants so that few output tiles still fill the GPU, and the fp32 scratch for them.
int ffn_k_parts(long long n, int cols, int k);
size_t ffn_parts_bytes(long long n, int cols, int k);
// y[n, h] = hid Wd^T;  dx[n, h] = [dg | du] [Wg; Wu].  `parts`: scratch of ffn_parts_bytes, or null where that is 0.
int ffn_down_tc(const void* hid, const void* w_down, long long n, int h, int f, void* y, float* parts,
                const int* dyn_rows, uint32_t* status, cudaStream_t stream);
// z[n][2][f] = dg | du from dy and the kept values.
int ffn_grad_gate_up_tc(const void* grad_y, const void* w_down, const void* kept, long long n, int h, int f,
                        a3po_activation act, void* z, const int* dyn_rows, uint32_t* status, cudaStream_t stream);
// grad_w[2 f, h] = [dg | du]^T x and grad_w_down[h, f] = dy^T h.
int ffn_grad_w_tc(const void* z, const void* hid, const void* x, const void* grad_y, long long n, int h, int f, void* grad_w_gate_up,
                  void* grad_w_down, a3po_dtype grad_dt, int accumulate, const int* dyn_rows, uint32_t* status,
                  cudaStream_t stream);
// grad_x[n, h] = [dg | du] w_gate_up.  Launched right behind ffn_grad_w_tc, beside which it may run.
int ffn_grad_x_tc(const void* z, const void* w_gate_up, long long n, int h, int f, void* grad_x, float* parts,
                  const int* dyn_rows, uint32_t* status, cudaStream_t stream);

// ---- few rows (ffn_few.cu): bf16, same shapes; masked rows are read as zeros ----
// Up to 16 rows always; up to 32 (two row tiles, twice the traffic of x out of L2) while the weights are small enough that
// the tile kernels' fixed costs weigh more.  32 rows, forward, here / on tiles: 1024 x 2048 11 / 23 us, 1536 x 4608 24 / 32,
// 2560 x 7680 (118 MB of weights) 47 / 47, 4096 x 12288 94 / 73; 16 rows of that 69 / 73.
constexpr int kFewRows = 32;
inline bool few_rows(long long n, int h, int f) {
  return n <= 16 || (n <= kFewRows && static_cast<long long>(h) * f <= 20000000ll);
}
int ffn_few_rows_fwd(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, long long n,
                     int h, int f, a3po_activation act, void* hid, void* y, void* kept, cudaStream_t stream);
// dst[t, :] = row_mask[t] ? src[t, :] : 0
int ffn_select_rows(const void* src, const uint8_t* row_mask, long long n, int h, void* dst, cudaStream_t stream);

// ---- FP32-pipe kernels (ffn_simt.cu): fp32, and bf16 shapes the others do not take ----
// kept (may be null): fp32 [2][n][f];  hid: fp32 [n, f];  z: fp32 [n][3][f] (dg | du | h).
int ffn_fwd_simt(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, long long n, int h,
                 int f, a3po_dtype dt, a3po_activation act, float* hid, void* y, void* kept, cudaStream_t stream);
int ffn_bwd_simt(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, const void* kept,
                 const void* grad_y, long long n, int h, int f, a3po_dtype dt, a3po_activation act, float* z,
                 void* grad_x, void* grad_w_gate_up, void* grad_w_down, a3po_dtype grad_dt, int accumulate,
                 cudaStream_t stream);

}  // namespace a3po
