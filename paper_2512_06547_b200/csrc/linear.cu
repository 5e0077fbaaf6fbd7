// Entry points of the linear operator: argument checks, workspace layout, choice of the kernel family.

#include <climits>

#include "linear_internal.cuh"

namespace a3po {
namespace {

size_t elt(a3po_dtype dt) { return dt == A3PO_F32 ? 4 : 2; }

// The family is a function of dtype and shape alone, so that forward and backward agree on the kept layout.
bool tensor_cores(a3po_dtype dt, int k, int m) { return dt == A3PO_BF16 && k % 8 == 0 && m % 8 == 0; }

bool act_of(a3po_activation act, Act* out) {
  if (act == A3PO_ACT_NONE) *out = kActNone;
  else if (act == A3PO_ACT_SILU) *out = kActSilu;
  else if (act == A3PO_ACT_GELU_TANH) *out = kActGelu;
  else return false;
  return true;
}

int check(long long n, int k, int m, a3po_dtype dt, a3po_activation act_, Act* act) {
  if (n < 0 || k <= 0 || m <= 0) return A3PO_ERR_INVALID_ARG;
  if (dt != A3PO_F32 && dt != A3PO_BF16) return A3PO_ERR_UNSUPPORTED;
  if (!act_of(act_, act)) return A3PO_ERR_UNSUPPORTED;
  // the FP32-pipe kernels have a grid row for every 32 columns, dz's for every 128
  if (n > INT_MAX - 256 || k > 65535 * 32 || m > 65535 * 32) return A3PO_ERR_UNSUPPORTED;
  return A3PO_OK;
}

struct Layout {
  CompactBuffers cb{};
  char* x_c = nullptr;     // rows of x that take part (or x with masked rows zeroed)
  char* dz = nullptr;
  float* sums = nullptr;   // column sums of dz by blocks of rows
  float* parts = nullptr;
  float* w_parts = nullptr;   // apart from them: the two products run beside one another
};

bool lay_out(Arena& ar, long long n, int k, int m, a3po_dtype dt, Act act, bool masked, bool bwd, Layout* l) {
  const size_t rows = static_cast<size_t>(n);
  if (!tensor_cores(dt, k, m)) {
    if (bwd) {
      l->dz = ar.take<char>(rows * m * sizeof(float));
      l->sums = ar.take<float>((rows + kSimtSumRows - 1) / kSimtSumRows * m);
    }
    return ar.ok();
  }
  const bool compact = masked && !linear_few(n, k, m);
  const size_t cap = compact ? static_cast<size_t>(compact_capacity(n)) : rows;
  if (compact) {
    constexpr size_t kScan = 4096;   // block counts of the row index (compact_rows.cu)
    l->cb.cap = static_cast<long long>(cap);
    l->cb.count = ar.take<int>(1);
    l->cb.block_counts = ar.take<int>(kScan);
    l->cb.block_offsets = ar.take<int>(kScan);
    l->cb.pos = ar.take<int>(rows);
    l->cb.idx = ar.take<int>(cap);
  }
  if (compact || (masked && bwd)) l->x_c = ar.take<char>(cap * k * 2);
  if (bwd) {
    if (masked || act != kActNone) l->dz = ar.take<char>(cap * m * 2);
    l->sums = ar.take<float>((cap + kZRows - 1) / kZRows * m);
  }
  const size_t parts = !bwd && linear_few(n, k, m) ? 0 : bwd ? ffn_parts_bytes(static_cast<long long>(cap), k, m)
                                                             : linear_parts_bytes(static_cast<long long>(cap), k, m);
  if (parts) l->parts = ar.take<float>(parts / sizeof(float));
  const size_t w_parts = bwd ? linear_weight_parts_bytes(static_cast<long long>(cap), k, m) : 0;
  if (w_parts) l->w_parts = ar.take<float>(w_parts / sizeof(float));
  return ar.ok();
}

int zero(void* p, size_t bytes, cudaStream_t s) {
  if (cudaMemsetAsync(p, 0, bytes, s) != cudaSuccess) {
    cudaGetLastError();
    return A3PO_ERR_CUDA;
  }
  return A3PO_OK;
}

}  // namespace
}  // namespace a3po

using namespace a3po;

extern "C" {

size_t a3po_linear_kept_bytes(int64_t N, int M, a3po_dtype dt, a3po_activation act_) {
  Act act;
  if (check(N, 1, M, dt, act_, &act) != A3PO_OK || act == kActNone) return 0;
  if (dt == A3PO_F32) return round_up(static_cast<size_t>(N) * M * 4, 256) + 256;
  return static_cast<size_t>((N + kZRows - 1) / kZRows) * static_cast<size_t>(z_col_tiles(M)) * kZTile + 256;
}

size_t a3po_linear_workspace_bytes(int64_t N, int K, int M, a3po_dtype dt, a3po_activation act_, int has_row_mask, int is_bwd) {
  Act act;
  if (check(N, K, M, dt, act_, &act) != A3PO_OK) return 0;
  Arena ar(reinterpret_cast<void*>(256), static_cast<size_t>(-1) / 2);   // sizes only: nothing is dereferenced
  Layout l;
  lay_out(ar, N, K, M, dt, act, has_row_mask != 0, is_bwd != 0, &l);
  return round_up(ar.used, 256) + 256;
}

int a3po_linear_fwd(const void* x, const void* w, const void* bias, const void* residual, const uint8_t* row_mask, int64_t N,
                    int K, int M, a3po_dtype dt, a3po_activation act_, void* y, a3po_dtype y_dt, void* kept,
                    size_t kept_bytes, void* ws, size_t ws_bytes, uint32_t* status, void* stream_) {
  Act act;
  A3PO_RETURN_IF(check(N, K, M, dt, act_, &act));
  if (y_dt != dt && y_dt != A3PO_F32) return A3PO_ERR_UNSUPPORTED;
  if (!w || (N > 0 && (!x || !y))) return A3PO_ERR_INVALID_ARG;
  const bool tc = tensor_cores(dt, K, M);
  const size_t align = tc ? 16 : elt(dt), align_y = tc ? 16 : elt(y_dt);
  if (!aligned_to(x, align) || !aligned_to(w, align) || !aligned_to(bias, align) || !aligned_to(residual, align) ||
      !aligned_to(y, align_y))
    return A3PO_ERR_UNSUPPORTED;
  if (act == kActNone) kept = nullptr;   // the backward needs nothing
  if (kept && (!aligned_to(kept, 256) || kept_bytes < a3po_linear_kept_bytes(N, M, dt, act_))) return A3PO_ERR_WORKSPACE;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_linear_workspace_bytes(N, K, M, dt, act_, row_mask != nullptr, 0))
    return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (N == 0) return A3PO_OK;
  Arena ar(ws, ws_bytes);
  Layout l;
  if (!lay_out(ar, N, K, M, dt, act, row_mask != nullptr, false, &l)) return A3PO_ERR_WORKSPACE;
  LinearFwd c{x, w, bias, residual, N, K, M, act, y, y_dt == A3PO_F32, kept, l.parts, row_mask, nullptr, nullptr, N, status,
              as_stream(stream_)};
  if (!tc) return linear_fwd_simt(c, dt);
  if (linear_few(N, K, M)) return linear_few_rows_fwd(c);
  if (!row_mask) return linear_fwd_tc(c);
  A3PO_RETURN_IF(linear_row_index(row_mask, N, l.cb, c.stream));
  A3PO_RETURN_IF(gather_rows_range(x, K, l.cb.idx, l.cb.count, 0, l.cb.cap, l.x_c, c.stream, true));
  c.x = l.x_c;
  c.n = l.cb.cap;
  c.row_index = l.cb.idx;
  c.count = l.cb.count;
  return linear_fwd_tc(c);
}

int a3po_linear_bwd(const void* x, const void* w, const uint8_t* row_mask, const void* kept, size_t kept_bytes,
                    const void* grad_y, int64_t N, int K, int M, a3po_dtype dt, a3po_activation act_, void* grad_x,
                    void* grad_w, a3po_dtype grad_w_dt, float* grad_bias, int accumulate, void* ws, size_t ws_bytes,
                    uint32_t* status, void* stream_) {
  Act act;
  A3PO_RETURN_IF(check(N, K, M, dt, act_, &act));
  if (!grad_x && !grad_w && !grad_bias) return A3PO_ERR_INVALID_ARG;
  if (N > 0 && (!grad_y || (grad_w && !x) || (grad_x && !w) || (act != kActNone && !kept))) return A3PO_ERR_INVALID_ARG;
  if (grad_w_dt != A3PO_F32 && grad_w_dt != dt) return A3PO_ERR_UNSUPPORTED;
  if (accumulate && grad_w && grad_w_dt != A3PO_F32) return A3PO_ERR_UNSUPPORTED;   // every addition would round to bf16
  const bool tc = tensor_cores(dt, K, M);
  const size_t align = tc ? 16 : elt(dt), align_w = tc ? 16 : elt(grad_w_dt);
  if (!aligned_to(x, align) || !aligned_to(w, align) || !aligned_to(grad_y, align) || !aligned_to(grad_x, align) ||
      !aligned_to(grad_w, align_w) || !aligned_to(grad_bias, 4))
    return A3PO_ERR_UNSUPPORTED;
  if (act != kActNone && kept && (!aligned_to(kept, 256) || kept_bytes < a3po_linear_kept_bytes(N, M, dt, act_)))
    return A3PO_ERR_WORKSPACE;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_linear_workspace_bytes(N, K, M, dt, act_, row_mask != nullptr, 1))
    return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  cudaStream_t stream = as_stream(stream_);
  if (N == 0) {
    if (accumulate) return A3PO_OK;
    if (grad_w) A3PO_RETURN_IF(zero(grad_w, static_cast<size_t>(M) * K * elt(grad_w_dt), stream));
    return grad_bias ? zero(grad_bias, static_cast<size_t>(M) * 4, stream) : A3PO_OK;
  }
  Arena ar(ws, ws_bytes);
  Layout l;
  if (!lay_out(ar, N, K, M, dt, act, row_mask != nullptr, true, &l)) return A3PO_ERR_WORKSPACE;
  if (!tc)
    return linear_bwd_simt(x, w, row_mask, kept, grad_y, N, K, M, dt, act, reinterpret_cast<float*>(l.dz), l.sums, grad_x, grad_w,
                           grad_w_dt, grad_bias, accumulate, stream);
  const bool compact = row_mask && !linear_few(N, K, M);
  long long rows = N;
  const int *count = nullptr, *index = nullptr;
  bool first = true;
  const void* xs = x;
  if (compact) {   // the same index as the forward's: what was kept is in the compact row space
    A3PO_RETURN_IF(linear_row_index(row_mask, N, l.cb, stream));
    if (grad_w) A3PO_RETURN_IF(gather_rows_range(x, K, l.cb.idx, l.cb.count, 0, l.cb.cap, l.x_c, stream, true));
    rows = l.cb.cap;
    count = l.cb.count;
    index = l.cb.idx;
    first = false;
  } else if (row_mask && grad_w) {
    A3PO_RETURN_IF(ffn_select_rows(x, row_mask, N, K, l.x_c, stream));
    first = false;
  }
  if (row_mask) xs = l.x_c;
  const void* dz = grad_y;
  const bool few = rows <= kZRows;   // a block's sums are the bias gradient
  if (l.dz || grad_bias) {
    if (l.dz) dz = l.dz;
    A3PO_RETURN_IF(linear_grad_z(grad_y, kept, rows, M, act, index, count, compact ? nullptr : row_mask, l.dz,
                                 !grad_bias || few ? grad_bias : l.sums, few && accumulate, compact, stream));
    first = false;
  }
  if (grad_x || grad_w)
    A3PO_RETURN_IF(linear_grads_tc(dz, xs, w, rows, K, M, grad_x, grad_w, grad_w_dt, accumulate, l.parts, l.w_parts, index, count,
                                   row_mask, N, first, status, stream));
  // the column sums are there before either product begins: they are added up beside the last of them
  return grad_bias && !few ? linear_grad_bias(l.sums, (rows + kZRows - 1) / kZRows, count, M, grad_bias, accumulate, grad_x || grad_w, stream)
                   : A3PO_OK;
}

}  // extern "C"
