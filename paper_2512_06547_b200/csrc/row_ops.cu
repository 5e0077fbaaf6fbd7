// Row-wise training operators on the residual stream in front of the LM head: norm (RMS or layer), dropout whose
// mask is never stored, and the join of both (dropout, add to the residual stream, norm) in one pass; forward and
// backward.
//
//   norm      xhat = (x - mean) rstd,  mean = sum x / H (0 for RMS),  rstd = 1 / sqrt(sum (x - mean)^2 / H + eps)
//             y = xhat gamma + beta
//   backward  gx = gy gamma,  dx = rstd (gx - [mean(gx)] - xhat mean(gx xhat))      ([.]: layer norm only)
//             dgamma = sum_rows gy xhat,  dbeta = sum_rows gy
//   dropout   d(x)[t, c] = keep(t, c) x[t, c] 65536 / (65536 - T),  T = round(65536 p),  keep = (u16(t, c) >= T)
//   join      r = residual + d(x) (stored),  y = norm(r)
//
// All of them stream [N, H] matrices and compute next to nothing, so HBM bytes are the bound: every element is read
// once (a row stays in registers between its statistics and its result) and written once.  A thread owns 8
// consecutive columns (16 bytes of bf16), which is also what one Philox call decides.  Sums, statistics and partial
// weight gradients are fp32; the only rounding to fewer bits is the final store in the matrices' own type.
//
// Random numbers: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC'11),
// key = seed, counter = (column / 8, row, offset low, offset high); its four words are eight 16-bit numbers, low half
// first.  16 bits decide one element: the drop probability is a multiple of 2^-16 and the scale is exact for it, at
// half the integer work of 32-bit numbers (with those the multiplies, not HBM, would bound dropout).

#include "row_ops.cuh"

namespace a3po {
namespace {

// ------------------------------------------------------------------------------------ dropout (+ residual)
// 16-byte rows: the matrix is one run of chunks; a block takes kDropThreads * U consecutive ones, every thread U of them
// kDropThreads apart, all loads before the arithmetic, and is done: the next block's loads fill the pause that a grid-stride
// loop has between its iterations.  131,072 x 4,096 bf16 with a residual: 491-532 us (6.1-6.5 TB/s; 823 us with a
// grid-stride loop of two chunks per thread).
constexpr int kDropThreads = 256;
template <typename T> constexpr int drop_unroll() { return sizeof(T) == 2 ? 4 : 2; }

template <typename T, bool RES>
__global__ void __launch_bounds__(kDropThreads)
dropout_vec_kernel(const T* __restrict__ x, const T* __restrict__ residual, const uint8_t* __restrict__ row_mask,
                   long long chunks, int groups, double inv_groups, uint32_t magic, int shift, const Dropout drop,
                   T* __restrict__ y) {
  constexpr int U = drop_unroll<T>();
  const long long first = static_cast<long long>(blockIdx.x) * (kDropThreads * U);
  // first = row0 * groups + group0: the quotient in double is within 1 of it (first < 2^53), then put right
  long long row0 = static_cast<long long>(static_cast<double>(first) * inv_groups);
  long long rem = first - row0 * groups;
  if (rem < 0) { rem += groups; --row0; }
  if (rem >= groups) { rem -= groups; ++row0; }
  const uint32_t at = static_cast<uint32_t>(rem) + threadIdx.x;
  Raw<T> v[U], r[U];
  uint32_t group[U];
  long long row[U];
  bool in[U], on[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const long long c = first + i * kDropThreads + threadIdx.x;
    const uint32_t from = at + static_cast<uint32_t>(i * kDropThreads);   // groups past the start of row0
    const uint32_t over = (__umulhi(magic, from) + from) >> shift;        // from / groups for from < 2^31
    group[i] = from - over * static_cast<uint32_t>(groups);
    row[i] = row0 + over;
    in[i] = c < chunks;
    on[i] = in[i] && (!row_mask || row_mask[row[i]] != 0);
    if (on[i]) {
      v[i].load(x + c * kVec);
      if (RES) r[i].load(residual + c * kVec); else r[i].clear();
    } else {
      v[i].clear();
      r[i].clear();
    }
  }
  PhiloxState ph;
  const bool dropping = drop.rng != nullptr;
  if (dropping) ph.load(drop.rng);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    F2 a[kPairs], b[kPairs];
    v[i].get(a);
    r[i].get(b);
    if (dropping) {
      bool keep[kVec];
      keep_bits(ph.draw(group[i], static_cast<uint32_t>(row[i])), drop.below, keep);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        a[j] = drop2(keep[2 * j], keep[2 * j + 1], a[j], drop.scale);
        if (RES) a[j] = add2(a[j], b[j]);
      }
    } else if (RES) {
#pragma unroll
      for (int j = 0; j < kPairs; ++j) a[j] = add2(a[j], b[j]);
    }
    if (in[i]) {
      v[i].set(a);
      v[i].store(y + (first + i * kDropThreads + threadIdx.x) * kVec);
    }
  }
}

// Rows that start at any element: `lanes` threads (a power of two up to a warp) take 8 x lanes consecutive columns of a
// row, every lanes-th column each, so that element loads are contiguous; see RowThreads.
template <typename T>
__global__ void __launch_bounds__(kDropThreads)
dropout_any_kernel(const T* __restrict__ x, const T* __restrict__ residual, const uint8_t* __restrict__ row_mask,
                   long long n, int h, int lanes, int segments, const Dropout drop, T* __restrict__ y) {
  const RowThreads<false> rt(lanes);
  PhiloxState ph;
  const bool dropping = drop.rng != nullptr;
  if (dropping) ph.load(drop.rng);
  const long long items = n * segments, stride = static_cast<long long>(gridDim.x) * rt.rows;
  for (long long base = static_cast<long long>(blockIdx.x) * rt.rows; base < items; base += stride) {
    const long long item = base + rt.slot;
    const long long row = items < 0x7fffffffll ? static_cast<uint32_t>(item) / static_cast<uint32_t>(segments) : item / segments;
    const int seg0 = static_cast<int>(item - row * segments) * lanes;   // first group of the segment
    const bool in = item < items;
    const bool on = in && (!row_mask || row_mask[row] != 0);
    float v[kVec], r[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = seg0 * kVec + j * lanes + rt.tid;
      v[j] = on && c < h ? to_float(x[row * h + c]) : 0.f;
      r[j] = residual && on && c < h ? to_float(residual[row * h + c]) : 0.f;
    }
    if (dropping) {
      bool keep[kVec];
      keep_bits(ph.draw(static_cast<uint32_t>(seg0 + rt.tid), static_cast<uint32_t>(row)), drop.below, keep);
      rt.template own_bits<false>(keep);
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[j] = drop_add(keep[j], v[j], drop.scale, r[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[j] += r[j];
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int c = seg0 * kVec + j * lanes + rt.tid;
      if (in && c < h) y[row * h + c] = from_float<T>(v[j]);
    }
  }
}

template <typename T>
int launch_dropout(const T* x, const T* residual, const uint8_t* row_mask, long long n, int h, const Dropout& drop, T* y,
                   bool vec, cudaStream_t stream) {
  const int groups = (h + kVec - 1) / kVec;
  if (vec) {
    const long long chunks = n * groups;
    constexpr long long kPerBlock = kDropThreads * drop_unroll<T>();
    const long long blocks = (chunks + kPerBlock - 1) / kPerBlock;
    if (blocks > 0x7fffffffll) return A3PO_ERR_UNSUPPORTED;   // 2^41 chunks and more: not in any GPU's memory
    const double inv = 1.0 / groups;
    // division by a constant as multiplication (Granlund and Montgomery 1994): with 2^shift >= groups,
    // m = floor(2^32 (2^shift - groups) / groups) + 1, n / groups = (floor(m n / 2^32) + n) >> shift
    int shift = 0;
    while ((1u << shift) < static_cast<uint32_t>(groups)) ++shift;
    const uint32_t magic = static_cast<uint32_t>(((((1ull << shift) - groups) << 32) / groups) + 1);
    if (residual)
      A3PO_LAUNCH(kKDropout, stream, (dropout_vec_kernel<T, true><<<static_cast<unsigned>(blocks), kDropThreads, 0, stream>>>(
                                         x, residual, row_mask, chunks, groups, inv, magic, shift, drop, y)));
    else
      A3PO_LAUNCH(kKDropout, stream, (dropout_vec_kernel<T, false><<<static_cast<unsigned>(blocks), kDropThreads, 0, stream>>>(
                                         x, residual, row_mask, chunks, groups, inv, magic, shift, drop, y)));
    return after_launch();
  }
  int lanes = 1;
  while (lanes < kWarp && lanes < groups) lanes *= 2;
  const int segments = (groups + lanes - 1) / lanes;
  const long long want = (n * segments + kDropThreads / lanes - 1) / (kDropThreads / lanes);
  const long long most = static_cast<long long>(sm_count()) * 16;
  A3PO_LAUNCH(kKDropout, stream, (dropout_any_kernel<T><<<static_cast<unsigned>(want < most ? want : most), kDropThreads, 0,
                                                          stream>>>(x, residual, row_mask, n, h, lanes, segments, drop, y)));
  return after_launch();
}

// ------------------------------------------------------------------------------------ host side
bool rows_vectorise(int h, std::initializer_list<const void*> ptrs) {
  if (h % kVec != 0) return false;
  for (const void* p : ptrs)
    if (p && !aligned_to(p, 16)) return false;
  return true;
}

// Drop probability as a multiple of 2^-16 and its exact scale.
Dropout make_dropout(float p, const void* rng) {
  Dropout d;
  const uint32_t t = static_cast<uint32_t>(__builtin_rint(static_cast<double>(p) * 65536.0));
  d.below = t == 0u ? 0u : (t << 16) - 1u;   // T = 65536: 2^32 - 1, which nothing exceeds
  d.scale = t < 65536u ? static_cast<float>(65536.0 / (65536.0 - t)) : 0.f;
  d.rng = t == 0u ? nullptr : static_cast<const unsigned long long*>(rng);
  return d;
}

int check_rows(long long n, int h, a3po_dtype dt) {
  if (n < 0 || h <= 0) return A3PO_ERR_INVALID_ARG;
  if (dt != A3PO_F32 && dt != A3PO_BF16) return A3PO_ERR_UNSUPPORTED;
  if (n > 0x7fffffffll) return A3PO_ERR_UNSUPPORTED;   // one grid dimension of rows, one 32-bit counter word
  if (h > 1 << 30) return A3PO_ERR_UNSUPPORTED;        // columns are int, and the loops over them step past the end
  return A3PO_OK;
}

// Pointers must at least be aligned to their own elements.
bool elements_aligned(a3po_dtype dt, std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!aligned_to(p, dt == A3PO_F32 ? 4 : 2)) return false;
  return true;
}

int check_dropout(float p, const void* rng) {
  if (!(p >= 0.f && p <= 1.f)) return A3PO_ERR_INVALID_ARG;
  if (p > 0.f && !rng) return A3PO_ERR_INVALID_ARG;
  if (!aligned_to(rng, 8)) return A3PO_ERR_UNSUPPORTED;
  return A3PO_OK;
}

template <typename T, bool JOIN>
int norm_fwd_typed(const void* x, const void* residual, const void* gamma, const void* beta, const uint8_t* row_mask,
                   long long n, int h, a3po_norm_kind kind, float eps, const Dropout& drop, void* r, void* y,
                   float* mean, float* rstd, cudaStream_t stream) {
  NormFwdArgs<T> a{static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<const T*>(gamma),
                   static_cast<const T*>(beta), row_mask, n, h, eps, 1.0f / static_cast<float>(h),
                   static_cast<T*>(r), static_cast<T*>(y), mean, rstd, drop,
                   rows_vectorise(h, {x, residual, gamma, beta, r, y}) ? 1 : 0};
  return launch_norm_fwd(a, kind == A3PO_NORM_LAYER, JOIN, stream);
}

template <typename T, bool JOIN>
int norm_bwd_typed(const void* x, const void* gamma, const float* mean, const float* rstd, const uint8_t* row_mask,
                   const void* grad_y, const void* grad_r, long long n, int h, a3po_norm_kind kind,
                   const Dropout& drop, void* grad_residual, void* grad_x, float* grad_gamma, float* grad_beta,
                   int accumulate, float* part, cudaStream_t stream) {
  NormBwdArgs<T> a{static_cast<const T*>(x), static_cast<const T*>(gamma), mean, rstd, row_mask,
                   static_cast<const T*>(grad_y), static_cast<const T*>(grad_r), n, h, 1.0f / static_cast<float>(h),
                   static_cast<T*>(grad_x), static_cast<T*>(grad_residual), part, drop,
                   rows_vectorise(h, {x, gamma, grad_y, grad_r, grad_x, grad_residual}) ? 1 : 0};
  return launch_norm_bwd(a, kind == A3PO_NORM_LAYER, JOIN, grad_gamma, grad_beta, accumulate, stream);
}

int norm_bwd_entry(bool join, const void* x, const void* gamma, const float* mean, const float* rstd,
                   const uint8_t* row_mask, const void* grad_y, const void* grad_r, long long n, int h, a3po_dtype dt,
                   a3po_norm_kind kind, float p, const void* rng, void* grad_residual, void* grad_x,
                   float* grad_gamma, float* grad_beta, int accumulate, void* ws, size_t ws_bytes,
                   cudaStream_t stream) {
  A3PO_RETURN_IF(check_rows(n, h, dt));
  if (kind != A3PO_NORM_RMS && kind != A3PO_NORM_LAYER) return A3PO_ERR_UNSUPPORTED;
  if (!gamma || !grad_gamma || (n > 0 && (!x || !rstd || !grad_y || (!join && !grad_x)))) return A3PO_ERR_INVALID_ARG;
  if (n > 0 && kind == A3PO_NORM_LAYER && !mean) return A3PO_ERR_INVALID_ARG;
  if (kind == A3PO_NORM_RMS && mean) return A3PO_ERR_INVALID_ARG;   // an RMS norm has none, as in the forward
  if (join) {
    if (n > 0 && !grad_residual) return A3PO_ERR_INVALID_ARG;
    A3PO_RETURN_IF(check_dropout(p, rng));
  }
  if (!elements_aligned(dt, {x, gamma, grad_y, grad_r, grad_residual, grad_x}) ||
      !elements_aligned(A3PO_F32, {mean, rstd, grad_gamma, grad_beta}))
    return A3PO_ERR_UNSUPPORTED;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_norm_bwd_workspace_bytes(n, h)) return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (n == 0) {
    if (accumulate) return A3PO_OK;
    if (cudaMemsetAsync(grad_gamma, 0, sizeof(float) * static_cast<size_t>(h), stream) != cudaSuccess ||
        (grad_beta && cudaMemsetAsync(grad_beta, 0, sizeof(float) * static_cast<size_t>(h), stream) != cudaSuccess)) {
      cudaGetLastError();
      return A3PO_ERR_CUDA;
    }
    return A3PO_OK;
  }
  const Dropout drop = make_dropout(join ? p : 0.f, rng);
  float* part = static_cast<float*>(ws);
#define A3PO_NORM_BWD(T, J)                                                                                       \
  norm_bwd_typed<T, J>(x, gamma, mean, rstd, row_mask, grad_y, grad_r, n, h, kind, drop, grad_residual, grad_x, \
                       grad_gamma, grad_beta, accumulate, part, stream)
  if (dt == A3PO_F32) return join ? A3PO_NORM_BWD(float, true) : A3PO_NORM_BWD(float, false);
  return join ? A3PO_NORM_BWD(__nv_bfloat16, true) : A3PO_NORM_BWD(__nv_bfloat16, false);
#undef A3PO_NORM_BWD
}

int norm_fwd_entry(bool join, const void* x, const void* residual, const void* gamma, const void* beta,
                   const uint8_t* row_mask, long long n, int h, a3po_dtype dt, a3po_norm_kind kind, float eps, float p,
                   const void* rng, void* r, void* y, float* mean, float* rstd, cudaStream_t stream) {
  A3PO_RETURN_IF(check_rows(n, h, dt));
  if (kind != A3PO_NORM_RMS && kind != A3PO_NORM_LAYER) return A3PO_ERR_UNSUPPORTED;
  if (!(eps >= 0.f)) return A3PO_ERR_INVALID_ARG;
  if (!gamma || (n > 0 && (!x || !y))) return A3PO_ERR_INVALID_ARG;
  if (kind == A3PO_NORM_RMS && mean) return A3PO_ERR_INVALID_ARG;   // an RMS norm has no mean to report
  if (join) {
    if (n > 0 && (!residual || !r)) return A3PO_ERR_INVALID_ARG;
    A3PO_RETURN_IF(check_dropout(p, rng));
  }
  if (!elements_aligned(dt, {x, residual, gamma, beta, r, y}) || !elements_aligned(A3PO_F32, {mean, rstd}))
    return A3PO_ERR_UNSUPPORTED;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (n == 0) return A3PO_OK;
  const Dropout drop = make_dropout(join ? p : 0.f, rng);
#define A3PO_NORM_FWD(T, J) \
  norm_fwd_typed<T, J>(x, residual, gamma, beta, row_mask, n, h, kind, eps, drop, r, y, mean, rstd, stream)
  if (dt == A3PO_F32) return join ? A3PO_NORM_FWD(float, true) : A3PO_NORM_FWD(float, false);
  return join ? A3PO_NORM_FWD(__nv_bfloat16, true) : A3PO_NORM_FWD(__nv_bfloat16, false);
#undef A3PO_NORM_FWD
}

int dropout_entry(const void* x, const void* residual, const uint8_t* row_mask, long long n, int h, a3po_dtype dt,
                  float p, const void* rng, void* y, cudaStream_t stream) {
  A3PO_RETURN_IF(check_rows(n, h, dt));
  if (n > 0 && (!x || !y)) return A3PO_ERR_INVALID_ARG;
  A3PO_RETURN_IF(check_dropout(p, rng));
  if (!elements_aligned(dt, {x, residual, y})) return A3PO_ERR_UNSUPPORTED;
  const int sms = sm_count();
  if (sms <= 0) return A3PO_ERR_NO_DEVICE;
  if (n == 0) return A3PO_OK;
  const Dropout drop = make_dropout(p, rng);
  const bool vec = rows_vectorise(h, {x, residual, y});
  if (dt == A3PO_F32)
    return launch_dropout(static_cast<const float*>(x), static_cast<const float*>(residual), row_mask, n, h, drop,
                          static_cast<float*>(y), vec, stream);
  return launch_dropout(static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(residual), row_mask, n, h,
                        drop, static_cast<__nv_bfloat16*>(y), vec, stream);
}

}  // namespace
}  // namespace a3po

using namespace a3po;

extern "C" {

int a3po_norm_fwd(const void* x, const void* gamma, const void* beta, const uint8_t* row_mask, int64_t N, int H,
                  a3po_dtype dt, a3po_norm_kind kind, float eps, void* y, float* mean, float* rstd, void* stream) {
  return norm_fwd_entry(false, x, nullptr, gamma, beta, row_mask, N, H, dt, kind, eps, 0.f, nullptr, nullptr, y, mean,
                        rstd, as_stream(stream));
}

size_t a3po_norm_bwd_workspace_bytes(int64_t N, int H) {
  if (N < 0 || H <= 0) return 0;
  const size_t parts = static_cast<size_t>(N < max_parts(H) ? N : max_parts(H));
  return round_up(parts * 2 * static_cast<size_t>(H) * sizeof(float), 256) + 256;
}

int a3po_norm_bwd(const void* x, const void* gamma, const float* mean, const float* rstd, const uint8_t* row_mask,
                  const void* grad_y, int64_t N, int H, a3po_dtype dt, a3po_norm_kind kind, void* grad_x,
                  float* grad_gamma, float* grad_beta, int accumulate_grad_w, void* ws, size_t ws_bytes,
                  void* stream) {
  return norm_bwd_entry(false, x, gamma, mean, rstd, row_mask, grad_y, nullptr, N, H, dt, kind, 0.f, nullptr, nullptr,
                        grad_x, grad_gamma, grad_beta, accumulate_grad_w, ws, ws_bytes, as_stream(stream));
}

int a3po_dropout_fwd(const void* x, const void* residual, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt,
                     float p, const uint64_t* rng, void* y, void* stream) {
  return dropout_entry(x, residual, row_mask, N, H, dt, p, rng, y, as_stream(stream));
}

int a3po_dropout_bwd(const void* grad_y, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt, float p,
                     const uint64_t* rng, void* grad_x, void* stream) {
  return dropout_entry(grad_y, nullptr, row_mask, N, H, dt, p, rng, grad_x, as_stream(stream));
}

int a3po_dropout_norm_fwd(const void* x, const void* residual, float p, const uint64_t* rng, const void* gamma,
                          const void* beta, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt,
                          a3po_norm_kind kind, float eps, void* r, void* y, float* mean, float* rstd, void* stream) {
  return norm_fwd_entry(true, x, residual, gamma, beta, row_mask, N, H, dt, kind, eps, p, rng, r, y, mean, rstd,
                        as_stream(stream));
}

int a3po_dropout_norm_bwd(const void* r, float p, const uint64_t* rng, const void* gamma, const float* mean,
                          const float* rstd, const uint8_t* row_mask, const void* grad_y, const void* grad_r,
                          int64_t N, int H, a3po_dtype dt, a3po_norm_kind kind, void* grad_residual, void* grad_x,
                          float* grad_gamma, float* grad_beta, int accumulate_grad_w, void* ws, size_t ws_bytes,
                          void* stream) {
  return norm_bwd_entry(true, r, gamma, mean, rstd, row_mask, grad_y, grad_r, N, H, dt, kind, p, rng, grad_residual,
                        grad_x, grad_gamma, grad_beta, accumulate_grad_w, ws, ws_bytes, as_stream(stream));
}

}  // extern "C"
