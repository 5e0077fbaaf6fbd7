// Entry points of the gated feed-forward block: argument checks, workspace layout, choice of the kernel family.

#include <climits>

#include "ffn_internal.cuh"
#include "lmhead_internal.cuh"

namespace a3po {
namespace {

size_t elt(a3po_dtype dt) { return dt == A3PO_F32 ? 4 : 2; }

// The family is a function of dtype and shape alone, so that forward and backward agree on the kept layout.
bool tensor_cores(a3po_dtype dt, int h, int f) { return dt == A3PO_BF16 && h % 8 == 0 && f % 8 == 0; }
// The tensor-core and few-row kernels move 16 bytes at a time, the FP32-pipe kernels elements (of type `dt`).
size_t row_alignment(a3po_dtype dt, int h, int f) { return tensor_cores(dt, h, f) ? 16 : elt(dt); }

int check(const void* x, const void* w_gate_up, const void* w_down, long long n, int h, int f, a3po_dtype dt,
          a3po_activation act) {
  if (n < 0 || h <= 0 || f <= 0) return A3PO_ERR_INVALID_ARG;
  if (dt != A3PO_F32 && dt != A3PO_BF16) return A3PO_ERR_UNSUPPORTED;
  if (act != A3PO_ACT_SILU && act != A3PO_ACT_GELU_TANH) return A3PO_ERR_UNSUPPORTED;
  if (n > INT_MAX - 256 || f > INT_MAX / 4 || h > INT_MAX / 4) return A3PO_ERR_UNSUPPORTED;
  // the FP32-pipe kernels have a grid row for every 32 (or 64) columns
  if (!tensor_cores(dt, h, f) && (f > 65535 * 32 || h > 65535 * 32)) return A3PO_ERR_UNSUPPORTED;
  if (!w_gate_up || !w_down || (n > 0 && !x)) return A3PO_ERR_INVALID_ARG;
  const size_t align = row_alignment(dt, h, f);
  if (!aligned_to(x, align) || !aligned_to(w_gate_up, align) || !aligned_to(w_down, align)) return A3PO_ERR_UNSUPPORTED;
  return A3PO_OK;
}

// Device buffers of one call.
struct Layout {
  CompactBuffers cb{};
  char* x_c = nullptr;      // rows of x that take part (or x with masked rows zeroed)
  char* gy_c = nullptr;     // same of grad_y
  char* out_c = nullptr;    // y or grad_x in the compact row space
  char* hid = nullptr;      // forward: h
  char* z = nullptr;        // backward: dg | du | h
  float* parts = nullptr;
};

bool lay_out(Arena& ar, long long n, int h, int f, a3po_dtype dt, bool masked, bool bwd, Layout* l) {
  const size_t rows = static_cast<size_t>(n);
  if (!tensor_cores(dt, h, f)) {
    if (bwd) l->z = ar.take<char>(rows * 3 * f * sizeof(float));
    else l->hid = ar.take<char>(rows * f * sizeof(float));
    return ar.ok();
  }
  const bool few = few_rows(n, h, f);
  const size_t cap = masked && !few ? static_cast<size_t>(compact_capacity(n)) : rows;
  if (masked && !few) {
    constexpr size_t kScan = 4096;   // block counts of the row index (compact_rows.cu)
    l->cb.cap = static_cast<long long>(cap);
    l->cb.count = ar.take<int>(1);
    l->cb.block_counts = ar.take<int>(kScan);
    l->cb.block_offsets = ar.take<int>(kScan);
    l->cb.pos = ar.take<int>(rows);
    l->cb.idx = ar.take<int>(cap);
    l->x_c = ar.take<char>(cap * h * 2);
    l->out_c = ar.take<char>(cap * h * 2);
    if (bwd) l->gy_c = ar.take<char>(cap * h * 2);
  } else if (masked && bwd) {
    l->x_c = ar.take<char>(rows * h * 2);
    l->gy_c = ar.take<char>(rows * h * 2);
  }
  if (bwd) l->z = ar.take<char>(cap * 2 * f * 2);
  else l->hid = ar.take<char>(cap * f * 2);   // used when nothing is kept
  const size_t parts = few && !bwd ? 0 : ffn_parts_bytes(static_cast<long long>(cap), h, bwd ? 2 * f : f);
  if (parts) l->parts = ar.take<float>(parts / sizeof(float));
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

size_t a3po_gated_ffn_kept_bytes(int64_t N, int F, a3po_dtype dt) {
  if (N < 0 || F <= 0) return 0;
  if (dt == A3PO_F32) return round_up(static_cast<size_t>(N) * F * 8, 256) + 256;
  return kept_gate_bytes(N, F) + static_cast<size_t>(compact_capacity(N)) * F * 2 + 256;
}

size_t a3po_gated_ffn_workspace_bytes(int64_t N, int H, int F, a3po_dtype dt, int has_row_mask, int is_bwd) {
  if (N < 0 || H <= 0 || F <= 0 || H > INT_MAX / 4 || F > INT_MAX / 4 || N > INT_MAX - 256) return 0;
  Arena ar(reinterpret_cast<void*>(256), static_cast<size_t>(-1) / 2);   // sizes only: nothing is dereferenced
  Layout l;
  lay_out(ar, N, H, F, dt, has_row_mask != 0, is_bwd != 0, &l);
  return round_up(ar.used, 256) + 256;
}

int a3po_gated_ffn_fwd(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, int64_t N,
                       int H, int F, a3po_dtype dt, a3po_activation act, void* y, void* kept, size_t kept_bytes, void* ws,
                       size_t ws_bytes, uint32_t* status, void* stream_) {
  A3PO_RETURN_IF(check(x, w_gate_up, w_down, N, H, F, dt, act));
  if (N > 0 && !y) return A3PO_ERR_INVALID_ARG;
  if (!aligned_to(y, row_alignment(dt, H, F))) return A3PO_ERR_UNSUPPORTED;
  if (kept && (!aligned_to(kept, 256) || kept_bytes < a3po_gated_ffn_kept_bytes(N, F, dt))) return A3PO_ERR_WORKSPACE;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_gated_ffn_workspace_bytes(N, H, F, dt, row_mask != nullptr, 0))
    return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (N == 0) return A3PO_OK;
  cudaStream_t stream = as_stream(stream_);
  Arena ar(ws, ws_bytes);
  Layout l;
  if (!lay_out(ar, N, H, F, dt, row_mask != nullptr, false, &l)) return A3PO_ERR_WORKSPACE;
  if (!tensor_cores(dt, H, F))
    return ffn_fwd_simt(x, w_gate_up, w_down, row_mask, N, H, F, dt, act, reinterpret_cast<float*>(l.hid), y, kept,
                        stream);
  if (kept) l.hid = static_cast<char*>(kept) + kept_gate_bytes(N, F);
  if (few_rows(N, H, F)) return ffn_few_rows_fwd(x, w_gate_up, w_down, row_mask, N, H, F, act, l.hid, y, kept, stream);
  if (!row_mask) {
    A3PO_RETURN_IF(ffn_gate_up_tc(x, w_gate_up, N, H, F, act, l.hid, kept, nullptr, status, stream));
    return ffn_down_tc(l.hid, w_down, N, H, F, y, l.parts, nullptr, status, stream);
  }
  A3PO_RETURN_IF(compact_index(nullptr, row_mask, nullptr, nullptr, N, l.cb, stream));
  A3PO_RETURN_IF(gather_rows_range(x, H, l.cb.idx, l.cb.count, 0, l.cb.cap, l.x_c, stream, true));
  A3PO_RETURN_IF(ffn_gate_up_tc(l.x_c, w_gate_up, l.cb.cap, H, F, act, l.hid, kept, l.cb.count, status, stream));
  A3PO_RETURN_IF(ffn_down_tc(l.hid, w_down, l.cb.cap, H, F, l.out_c, l.parts, l.cb.count, status, stream));
  return scatter_rows(l.out_c, H, l.cb.pos, N, y, stream, true);
}

int a3po_gated_ffn_bwd(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask,
                       const void* kept, size_t kept_bytes, const void* grad_y, int64_t N, int H, int F, a3po_dtype dt,
                       a3po_activation act, void* grad_x, void* grad_w_gate_up, void* grad_w_down, a3po_dtype grad_w_dt,
                       int accumulate_grad_w, void* ws, size_t ws_bytes, uint32_t* status, void* stream_) {
  A3PO_RETURN_IF(check(x, w_gate_up, w_down, N, H, F, dt, act));
  if (!grad_w_gate_up || !grad_w_down || (N > 0 && (!grad_y || !grad_x || !kept))) return A3PO_ERR_INVALID_ARG;
  if (grad_w_dt != A3PO_F32 && grad_w_dt != dt) return A3PO_ERR_UNSUPPORTED;
  if (accumulate_grad_w && grad_w_dt != A3PO_F32) return A3PO_ERR_UNSUPPORTED;   // every addition would round to bf16
  const size_t align = row_alignment(dt, H, F), align_w = tensor_cores(dt, H, F) ? 16 : elt(grad_w_dt);
  if (!aligned_to(grad_y, align) || !aligned_to(grad_x, align) || !aligned_to(grad_w_gate_up, align_w) ||
      !aligned_to(grad_w_down, align_w))
    return A3PO_ERR_UNSUPPORTED;
  if (kept && (!aligned_to(kept, 256) || kept_bytes < a3po_gated_ffn_kept_bytes(N, F, dt))) return A3PO_ERR_WORKSPACE;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_gated_ffn_workspace_bytes(N, H, F, dt, row_mask != nullptr, 1))
    return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  cudaStream_t stream = as_stream(stream_);
  if (N == 0) {
    if (accumulate_grad_w) return A3PO_OK;
    const size_t weights = static_cast<size_t>(F) * H * elt(grad_w_dt);
    A3PO_RETURN_IF(zero(grad_w_gate_up, 2 * weights, stream));
    return zero(grad_w_down, weights, stream);
  }
  Arena ar(ws, ws_bytes);
  Layout l;
  if (!lay_out(ar, N, H, F, dt, row_mask != nullptr, true, &l)) return A3PO_ERR_WORKSPACE;
  if (!tensor_cores(dt, H, F))
    return ffn_bwd_simt(x, w_gate_up, w_down, row_mask, kept, grad_y, N, H, F, dt, act, reinterpret_cast<float*>(l.z),
                        grad_x, grad_w_gate_up, grad_w_down, grad_w_dt, accumulate_grad_w, stream);
  const void *xs = x, *gys = grad_y;
  void* gx = grad_x;
  long long rows = N;
  const int* count = nullptr;
  const bool compact = row_mask && !few_rows(N, H, F);
  if (compact) {
    // the same index as the forward's: the kept values are in the compact row space
    A3PO_RETURN_IF(compact_index(nullptr, row_mask, nullptr, nullptr, N, l.cb, stream));
    A3PO_RETURN_IF(gather_rows_range(x, H, l.cb.idx, l.cb.count, 0, l.cb.cap, l.x_c, stream, true));
    A3PO_RETURN_IF(gather_rows_range(grad_y, H, l.cb.idx, l.cb.count, 0, l.cb.cap, l.gy_c, stream, true, true));
    rows = l.cb.cap;
    count = l.cb.count;
    gx = l.out_c;
  } else if (row_mask) {
    A3PO_RETURN_IF(ffn_select_rows(x, row_mask, N, H, l.x_c, stream));
    A3PO_RETURN_IF(ffn_select_rows(grad_y, row_mask, N, H, l.gy_c, stream));
  }
  if (row_mask) {
    xs = l.x_c;
    gys = l.gy_c;
  }
  A3PO_RETURN_IF(ffn_grad_gate_up_tc(gys, w_down, kept, rows, H, F, act, l.z, count, status, stream));
  // Three products that read z, x, grad_y and h and write apart: each begins on the SMs that the last wave of the one
  // before leaves idle.  Backward of 16,384 rows (62 % valid), 1536 x 4608: 821 -> 769 us with the compaction's early launches.
  A3PO_RETURN_IF(ffn_grad_w_tc(l.z, static_cast<const char*>(kept) + kept_gate_bytes(N, F), xs, gys, rows, H, F, grad_w_gate_up,
                               grad_w_down, grad_w_dt, accumulate_grad_w, count, status, stream));
  A3PO_RETURN_IF(ffn_grad_x_tc(l.z, w_gate_up, rows, H, F, gx, l.parts, count, status, stream));
  return compact ? scatter_rows(l.out_c, H, l.cb.pos, N, grad_x, stream, true) : A3PO_OK;
}

}  // extern "C"
