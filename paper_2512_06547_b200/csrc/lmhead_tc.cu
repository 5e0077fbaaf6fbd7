// LM-head log-prob forward/backward on the sm_100a tensor cores (bf16 in, fp32 accumulate).
//
// One persistent, warp-specialised kernel template does every contraction of the path,
//     C[M, N] = A[M, K] * B[N, K]^T,
// and differs only in its epilogue:
//   forward      A = hidden, B = W           online (max, sum-exp) per row + target gather
//   forward+keep same, and every probability is kept as a bf16 ratio to the target token's for a backward
//                without recomputation
//   dz           A = hidden, B = W           dz = g (1[v = y] - exp(z - lse)) -> bf16 chunk of rows
//   grad_hidden  A = dz,     B = W^T         bf16 store, optional per-row scale (W read in place, N-major)
//   grad_w       A = dz^T,   B = hidden^T    fp32 store/accumulate (both read in place, M-/N-major)
// (with kept probability ratios in place of dz the per-row factor of dz moves into the grad_hidden epilogue
// and into the hidden operand of grad_w)
//
// Per CTA (one per SM): warp 0 = TMA producer (one elected lane), warp 1 = tcgen05.mma issuer
// (one elected lane; it also owns the TMEM allocation), warps 2-5 = epilogue (one TMEM lane
// quarter each, one accumulator row per thread).  Operand tiles (128 x 64 and 256 x 64 bf16,
// 128-byte swizzle) move through a 4-stage shared-memory ring guarded by full/empty mbarriers;
// the 128 x 256 fp32 accumulator is double-buffered in TMEM (2 x 256 columns) so the epilogue
// of tile i overlaps the MMAs of tile i+1.  Output tiles (kept ratios, dz, gradients) leave through
// two swizzled shared-memory slabs and TMA tile stores.  The full logits matrix never exists: the
// plain forward keeps nothing, the keeping forward writes only the rows that take part, into scratch.
//
// Every mbarrier wait is bounded; on expiry the CTA raises A3PO_STATUS_WAIT_TIMEOUT in the
// caller's status word, releases its TMEM and exits.

#include "gemm_tc.cuh"
#include "lmhead_internal.cuh"

namespace a3po {
namespace {

// Waits on an mbarrier that never completes; the wait gives up after limit_ns and raises the
// status bit, exactly as a stuck pipeline stage would.
__global__ void wait_timeout_kernel(uint32_t* status, unsigned long long limit_ns) {
  __shared__ uint64_t bar;
  __shared__ uint32_t abort_flag;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool completed = mbar_wait(&bar, 0, &abort_flag, limit_ns);
    if (!completed && status) atomicOr(status, A3PO_STATUS_WAIT_TIMEOUT);
  }
}

// ------------------------------------------------------------------------------------ epilogues
// Each epilogue thread owns one accumulator row (`row` = global row of the A operand).
// begin(): per-item state; chunk(): 32 consecutive fp32 columns starting at global column `col0`;
// end(): per-item output.

template <bool ENT>
struct FwdEpilogue : PlainEpilogue {
  static constexpr int kKernelId = kKTcFwd;
  struct Params {
    const int32_t* targets;
    long long n;
    int v;
    float scale_log2;  // inv_temperature * log2(e)
    float inv_t;
    SoftmaxPartial* part;
    float* part_ent;
    float* zy;
  };
  static int make_c_map(const Params&, CUtensorMap* map) {
    memset(map, 0, sizeof(*map));  // the forward stores nothing through the copy engine
    return A3PO_OK;
  }
  float m, s, e;
  int y;
  long long row;
  __device__ __forceinline__ void begin(const Params& p, long long row_) {
    row = row_;
    m = -INFINITY; s = 0.f; e = 0.f;
    y = -1;
    if (row < p.n) y = min(max(p.targets[row], 0), p.v - 1);
  }
  __device__ __forceinline__ void chunk(const Params& p, int /*tile_row0*/, int col0, uint32_t (&r)[kEpiChunk],
                                        SlabStore&) {
    if (col0 + kEpiChunk > p.v) {  // ragged vocabulary tail: columns past V do not exist
#pragma unroll
      for (int j = 0; j < kEpiChunk; ++j)
        if (col0 + j >= p.v) r[j] = 0xff800000u;  // -inf
    }
    float zmax = -INFINITY;
#pragma unroll
    for (int j = 0; j < kEpiChunk; ++j) zmax = fmaxf(zmax, bits_to_float(r[j]));
    const float xm = zmax * p.scale_log2;
    if (xm > m) {
      const float f = fast_exp2(m - xm);
      s *= f;
      if (ENT) e *= f;
      m = xm;
    }
    float acc = 0.f, ee = 0.f;
#pragma unroll
    for (int j = 0; j < kEpiChunk; ++j) {
      const float z = bits_to_float(r[j]);
      const float pj = fast_exp2(fmaf(z, p.scale_log2, -m));
      acc += pj;
      if (ENT) ee = fmaf(pj, pj > 0.f ? z : 0.f, ee);
    }
    s += acc;
    if (ENT) e = fmaf(ee, p.inv_t, e);
    if (y >= col0 && y < col0 + kEpiChunk) {
      float zyv = 0.f;
#pragma unroll
      for (int j = 0; j < kEpiChunk; ++j)
        if (col0 + j == y) zyv = bits_to_float(r[j]);
      p.zy[row] = zyv * p.inv_t;
    }
  }
  __device__ __forceinline__ void end(const Params& p, long long row, int split) {
    if (row < p.n) {
      p.part[static_cast<long long>(split) * p.n + row] = SoftmaxPartial{m * kLn2, s};
      if (ENT) p.part_ent[static_cast<long long>(split) * p.n + row] = e;
    }
  }
};

struct DzEpilogue : PlainEpilogue {
  static constexpr int kKernelId = kKTcDz;
  struct Params {
    const int32_t* targets;   // indexed by global token row
    const float* lse;
    const float* grad_logp;
    long long row_begin;      // first token row of this chunk; A-operand row 0 == row_begin
    long long row_end;
    int v;
    int vpad;                 // row pitch of dz
    float scale_log2;
    float inv_t;
    __nv_bfloat16* dz;        // [chunk rows, vpad]
  };
  static int make_c_map(const Params& p, CUtensorMap* map) {
    return make_out_map(map, p.dz, /*bytes per element*/ 2, p.v, p.row_end - p.row_begin, p.vpad);
  }
  float g, l2;
  int y;
  uint8_t* cur;
  __device__ __forceinline__ void begin(const Params& p, long long row) {
    const long long t = p.row_begin + row;
    g = 0.f; l2 = INFINITY; y = -1;
    if (t < p.row_end) {
      g = p.grad_logp[t] * p.inv_t;
      if (g != 0.f) l2 = p.lse[t] * kLog2e;   // g == 0: exp2(-inf) = 0, the row contributes nothing
      y = min(max(p.targets[t], 0), p.v - 1);
    }
  }
  __device__ __forceinline__ void chunk(const Params& p, int tile_row0, int col0, uint32_t (&r)[kEpiChunk],
                                        SlabStore& st) {
    float d[kEpiChunk];
    const float ng = -g;
#pragma unroll
    for (int j = 0; j < kEpiChunk; ++j)
      d[j] = ng * fast_exp2(fmaf(bits_to_float(r[j]), p.scale_log2, -l2));
    if (y >= col0 && y < col0 + kEpiChunk) {
#pragma unroll
      for (int j = 0; j < kEpiChunk; ++j)
        if (col0 + j == y) d[j] += g;
    }
    // a slab holds 64 bf16 columns: two consecutive 32-column chunks
    const int half = (col0 >> 5) & 1;
    if (half == 0) cur = st.acquire();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint4 u;
      u.x = pack_bf16x2(d[q * 8 + 0], d[q * 8 + 1]);
      u.y = pack_bf16x2(d[q * 8 + 2], d[q * 8 + 3]);
      u.z = pack_bf16x2(d[q * 8 + 4], d[q * 8 + 5]);
      u.w = pack_bf16x2(d[q * 8 + 6], d[q * 8 + 7]);
      *st.piece(cur, half * 4 + q) = u;
    }
    if (half == 1) st.submit(cur, col0 - 32, tile_row0, col0 - 32 < p.v, false);
  }
  __device__ __forceinline__ void end(const Params&, long long, int) {}
};

// Forward that also keeps the row's softmax for the backward, so that the backward need not recompute
// the logits.  The reference of row t is its own target logit zy (computed beforehand, one dot product
// per row), and what is kept is the probability ratio
//     q[t, v] = exp(z[t, v] - zy[t]) = p[t, v] / p[t, y_t]                  (bf16, 0 at v = y_t)
// A ratio is a floating-point number with bf16's uniform relative precision whatever its size, so
// peaked and flat rows are kept equally well, and every split of a row shares the one reference, so
// no running maximum, rescaling or extra sweep is needed.  The target column is left out of the sum:
//     s[t] = sum_{v != y_t} q[t, v],  lse = zy + log1p(s),  logp = -log1p(s),  1 - p_y = s / (1 + s),
// which stays accurate when p_y approaches 1.  The exponent is clamped at 126 (a ratio above 2^126
// means p_y < 1e-37; the merge flags such a row).
template <bool ENT>
struct KeepEpilogue : PlainEpilogue {
  static constexpr int kKernelId = kKTcFwdKeep;
  struct Params {
    const int32_t* targets;   // [n] rows of this launch
    const float* zy;          // [n] target logit / T, natural-log units
    long long n;
    int v;
    int vpad;                 // row pitch of q
    float scale_log2;
    float inv_t;
    float* part_s;            // [splits][n] sum of the ratios over the split's columns, target left out
    float* part_e;            // [splits][n] sum of ratio * raw logit (entropy), or null
    __nv_bfloat16* q;         // [n, vpad]
  };
  static int make_c_map(const Params& p, CUtensorMap* map) { return make_out_map(map, p.q, 2, p.v, p.n, p.vpad); }
  float s, e, ref2;
  int y;
  uint8_t* cur;
  __device__ __forceinline__ void begin(const Params& p, long long row) {
    s = 0.f; e = 0.f; ref2 = 0.f;
    y = -1;
    if (row < p.n) {
      y = min(max(p.targets[row], 0), p.v - 1);
      ref2 = p.zy[row] * kLog2e;
    }
  }
  __device__ __forceinline__ void chunk(const Params& p, int tile_row0, int col0, uint32_t (&r)[kEpiChunk],
                                        SlabStore& st) {
    if (col0 + kEpiChunk > p.v) {
#pragma unroll
      for (int j = 0; j < kEpiChunk; ++j)
        if (col0 + j >= p.v) r[j] = 0xff800000u;  // -inf: columns past V do not exist
    }
    float q[kEpiChunk];
#pragma unroll
    for (int j = 0; j < kEpiChunk; ++j)
      q[j] = fast_exp2(fminf(fmaf(bits_to_float(r[j]), p.scale_log2, -ref2), 126.f));
    if (y >= col0 && y < col0 + kEpiChunk) {
#pragma unroll
      for (int j = 0; j < kEpiChunk; ++j)
        if (col0 + j == y) q[j] = 0.f;   // the target's own entry is written by the backward (-s)
    }
    float acc = 0.f, ee = 0.f;
#pragma unroll
    for (int j = 0; j < kEpiChunk; ++j) {
      acc += q[j];
      if (ENT) ee = fmaf(q[j], q[j] > 0.f ? bits_to_float(r[j]) : 0.f, ee);
    }
    s += acc;
    if (ENT) e += ee;
    const int half = (col0 >> 5) & 1;
    if (half == 0) cur = st.acquire();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint4 w;
      w.x = pack_bf16x2(q[k * 8 + 0], q[k * 8 + 1]);
      w.y = pack_bf16x2(q[k * 8 + 2], q[k * 8 + 3]);
      w.z = pack_bf16x2(q[k * 8 + 4], q[k * 8 + 5]);
      w.w = pack_bf16x2(q[k * 8 + 6], q[k * 8 + 7]);
      *st.piece(cur, half * 4 + k) = w;
    }
    if (half == 1) st.submit(cur, col0 - 32, tile_row0, col0 - 32 < p.v, false);
  }
  __device__ __forceinline__ void end(const Params& p, long long row, int split) {
    if (row < p.n) {
      p.part_s[static_cast<long long>(split) * p.n + row] = s;
      if (ENT) p.part_e[static_cast<long long>(split) * p.n + row] = e;
    }
  }
};

// Scratch of the backward: one bf16 dz chunk [chunk_rows, vpad].
size_t bwd_dz_bytes(long long chunk_rows, int v) {
  const size_t vpad = round_up(static_cast<size_t>(v), 8);
  return round_up(static_cast<size_t>(chunk_rows) * vpad * 2, 256);
}
// ... followed by one int (the tile choice of the chunk's grad_hidden launch)
size_t bwd_ws_layout(long long chunk_rows, int v) { return bwd_dz_bytes(chunk_rows, v) + 256; }

}  // namespace

// Pacing counters (see Pace) live in the library's device image, 8 KB per GPU: all zero when the library is
// loaded, and every paced launch leaves its block zero again.  In host code the array's name is only a handle for
// cudaGetSymbolAddress.
static __device__ __align__(256) unsigned int g_pace_counters[kPaceBlocks * kPaceBlockWords];
unsigned int* next_pace_block() {
  static std::mutex mu;
  static unsigned int* cached[64];
  static unsigned int turn[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return nullptr;
  }
  std::lock_guard<std::mutex> lock(mu);
  if (!cached[dev]) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_pace_counters) != cudaSuccess || !p) {
      cudaGetLastError();
      return nullptr;   // the launch then runs unpaced
    }
    cached[dev] = static_cast<unsigned int*>(p);
  }
  return cached[dev] + static_cast<size_t>(turn[dev]++ % kPaceBlocks) * kPaceBlockWords;
}

#ifdef A3PO_TUNING
}  // namespace a3po
// Tuning builds only (not part of the ABI in include/): where the GEMM kernels record their per-CTA trace.
// `records` is a device buffer of `capacity` 64-byte records, or null to stop tracing; resets the write position.
extern "C" int a3po_tuning_set_trace(void* records, unsigned int capacity) {
  a3po::TraceRecord* p = static_cast<a3po::TraceRecord*>(records);
  unsigned int zero = 0;
  if (cudaMemcpyToSymbol(a3po::g_trace, &p, sizeof(p)) != cudaSuccess ||
      cudaMemcpyToSymbol(a3po::g_trace_capacity, &capacity, sizeof(capacity)) != cudaSuccess ||
      cudaMemcpyToSymbol(a3po::g_trace_next, &zero, sizeof(zero)) != cudaSuccess) {
    cudaGetLastError();
    return A3PO_ERR_CUDA;
  }
  return A3PO_OK;
}
extern "C" unsigned int a3po_tuning_trace_count() {
  unsigned int n = 0;
  if (cudaMemcpyFromSymbol(&n, a3po::g_trace_next, sizeof(n)) != cudaSuccess) cudaGetLastError();
  return n;
}
namespace a3po {
#endif

// Exercises the bounded wait the pipelines rely on: a barrier nothing ever arrives at.
int selftest_wait_timeout(uint32_t* status, unsigned timeout_ms, cudaStream_t stream) {
  A3PO_LAUNCH(kKSelfTest, stream, (wait_timeout_kernel<<<1, 32, 0, stream>>>(
                                      status, static_cast<unsigned long long>(timeout_ms) * 1000000ull)));
  return after_launch();
}

bool lmhead_tc_supported(const void* hidden, const void* w, long long n, int h, int v) {
  return n > 0 && h >= 8 && (h % 8) == 0 && v >= 1 && aligned_to(hidden, 16) && aligned_to(w, 16) &&
         n < (1ll << 31) - 256;
}

// Whether the forward contractions run on CTA pairs (gemm_pair_kernel).  Off: measured on B200 under its power
// cap (seconds-long loops on one GPU) the pair kernel sustains 1083 TFLOP/s against 1241 for the single-CTA
// kernel on the same forward, although its tensor pipe is busier when the clock is free (99 % against 90 % under
// the profiler).  A tuning build switches it on with A3PO_FWD_PAIR=1 for comparisons and for its parity test.
bool fwd_uses_pairs() {
  if (tuning_override("A3PO_FWD_PAIR", 2) != 1) return false;
  return pair_capacity<KeepEpilogue<false>, false, false>() > 0;
}

// Picks the number of vocabulary splits so that (row tiles x splits) items spread evenly over
// the workers (SMs, or CTA pairs with 256-row tiles; static round-robin) while every item still sweeps several
// column tiles.  With G row tiles per group and SMs / G splits in flight, a split count that is a multiple of
// SMs / G makes every full group a whole number of waves, so that the CTAs never hold the row tiles of two
// groups at once (8B-shaped batch, 65,536 rows: 23 GB read from HBM per launch against 47 GB with 13 splits).
int lmhead_tc_fwd_splits(long long n, int h, int v) {
  const bool pairs = fwd_uses_pairs();
  const int tile_rows = pairs ? 2 * BM : BM;
  const long long m_tiles = (n + tile_rows - 1) / tile_rows;
  const int n_tiles = (v + BN - 1) / BN;
  if (m_tiles <= 0) return 1;
  int workers = pairs ? pair_capacity<KeepEpilogue<false>, false, false>() : sm_count();
  if (workers <= 0) workers = pairs ? 74 : 148;
  const int forced = tuning_override("A3PO_FWD_SPLITS", 0);
  if (forced > 0) return forced < n_tiles ? (forced < 64 ? forced : 64) : n_tiles;
  const int s_max = n_tiles < 64 ? n_tiles : 64;
  int s_min = s_max < 8 ? s_max : 8;  // several splits in flight keep the row-tile working set inside L2
  int step = 1;
  if (!pairs) {
    const int group = tuning_override("A3PO_GROUP_M", fwd_group_m(h));
    if (group > kGroupM && m_tiles >= group && workers % group == 0 && workers / group <= s_max) step = workers / group;
  }
  int best = 0;
  double best_cost = 1e300;
  for (int s = (s_min + step - 1) / step * step; s <= s_max; s += step) {
    const long long items = m_tiles * s;
    const long long waves = (items + workers - 1) / workers;
    const long long tiles_per_item = (n_tiles + s - 1) / s;
    const double cost = static_cast<double>(waves) * (static_cast<double>(tiles_per_item) + 0.5);
    if (cost < best_cost - 1e-9) { best_cost = cost; best = s; }
  }
  return best > 0 ? best : s_min;
}

int lmhead_fwd_tc(const void* hidden, const void* w, const int32_t* targets, long long n, int h, int v, float inv_t,
                  int splits, SoftmaxPartial* part, float* part_ent, float* zy, const int* dyn_rows, uint32_t* status,
                  cudaStream_t stream) {
  const Operand a{hidden, n, h, h};
  const Operand b{w, v, h, h};
  DynRows dyn;
  dyn.rows = dyn_rows;
  dyn.cap = n;
  const bool pairs = fwd_uses_pairs();
  if (part_ent) {
    FwdEpilogue<true>::Params p{targets, n, v, inv_t * kLog2e, inv_t, part, part_ent, zy};
    if (pairs) return launch_pair_gemm<FwdEpilogue<true>, false, false>(a, b, splits, p, dyn, status, stream);
    return launch_gemm<FwdEpilogue<true>, false, false>(a, b, splits, p, dyn, status, stream);
  }
  FwdEpilogue<false>::Params p{targets, n, v, inv_t * kLog2e, inv_t, part, nullptr, zy};
  if (pairs) return launch_pair_gemm<FwdEpilogue<false>, false, false>(a, b, splits, p, dyn, status, stream);
  return launch_gemm<FwdEpilogue<false>, false, false>(a, b, splits, p, dyn, status, stream);
}

size_t lmhead_tc_kept_bytes(long long rows, int v) {
  const size_t vpad = round_up(static_cast<size_t>(v), 8);
  return round_up(static_cast<size_t>(rows > 0 ? rows : 0) * vpad * 2, 256);
}

int lmhead_fwd_keep_tc(const void* hidden, const void* w, const int32_t* targets, const float* zy, long long n, int h,
                       int v, float inv_t, int splits, float* part_s, float* part_e, void* q, const int* dyn_rows,
                       long long dyn_offset, uint32_t* status, cudaStream_t stream) {
  const Operand a{hidden, n, h, h};
  const Operand b{w, v, h, h};
  DynRows dyn;
  dyn.rows = dyn_rows;
  dyn.offset = dyn_offset;
  dyn.cap = n;
  const int vpad = static_cast<int>(round_up(static_cast<size_t>(v), 8));
  const bool pairs = fwd_uses_pairs();
  if (part_e) {
    KeepEpilogue<true>::Params p{targets, zy, n, v, vpad, inv_t * kLog2e, inv_t, part_s, part_e,
                                 static_cast<__nv_bfloat16*>(q)};
    if (pairs) return launch_pair_gemm<KeepEpilogue<true>, false, false>(a, b, splits, p, dyn, status, stream);
    return launch_gemm<KeepEpilogue<true>, false, false>(a, b, splits, p, dyn, status, stream);
  }
  KeepEpilogue<false>::Params p{targets, zy, n, v, vpad, inv_t * kLog2e, inv_t, part_s, nullptr,
                                static_cast<__nv_bfloat16*>(q)};
  if (pairs) return launch_pair_gemm<KeepEpilogue<false>, false, false>(a, b, splits, p, dyn, status, stream);
  return launch_gemm<KeepEpilogue<false>, false, false>(a, b, splits, p, dyn, status, stream);
}

size_t lmhead_tc_bwd_ws_bytes(long long chunk_rows, long long /*n*/, int /*h*/, int v) {
  return bwd_ws_layout(chunk_rows, v);
}

int lmhead_bwd_tc(const void* hidden_, const void* w_, const int32_t* targets, const float* lse,
                  const float* grad_logp, long long n, int h, int v, float inv_t, void* grad_hidden_, float* grad_w,
                  int accumulate, void* ws, size_t ws_bytes, long long chunk_rows, const int* dyn_rows,
                  uint32_t* status, cudaStream_t stream) {
  const __nv_bfloat16* hidden = static_cast<const __nv_bfloat16*>(hidden_);
  const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(w_);
  __nv_bfloat16* grad_hidden = static_cast<__nv_bfloat16*>(grad_hidden_);
  if (bwd_ws_layout(chunk_rows, v) > ws_bytes) return A3PO_ERR_WORKSPACE;
  __nv_bfloat16* dz = static_cast<__nv_bfloat16*>(ws);  // [chunk_rows, vpad]
  int* select = reinterpret_cast<int*>(static_cast<char*>(ws) + bwd_dz_bytes(chunk_rows, v));
  const int vpad = static_cast<int>(round_up(static_cast<size_t>(v), 8));

  for (long long r0 = 0; r0 < n; r0 += chunk_rows) {
    const long long r1 = (r0 + chunk_rows < n) ? r0 + chunk_rows : n;
    const long long nc = r1 - r0;
    const __nv_bfloat16* hid_c = hidden + r0 * h;
    // dz[t, v] for this chunk of rows, from recomputed logits:  A = hidden (K-major), B = W (K-major)
    DzEpilogue::Params dp{targets, lse, grad_logp, r0, r1, v, vpad, inv_t * kLog2e, inv_t, dz};
    DynRows dyn_m;  // dz and grad_hidden: the rows are the M extent
    dyn_m.rows = dyn_rows;
    dyn_m.offset = r0;
    dyn_m.cap = nc;
    DynRows dyn_k = dyn_m;  // grad_w: the rows are the K extent
    dyn_k.is_k = 1;
    dyn_k.zero_when_empty = (r0 == 0 && !accumulate) ? 1 : 0;
    A3PO_RETURN_IF((launch_gemm<DzEpilogue, false, false>(Operand{hid_c, nc, h, h}, Operand{w, v, h, h}, 0, dp,
                                                          dyn_m, status, stream)));
    // grad_hidden[t, j] = sum_v dz[t, v] W[v, j]:  A = dz (K = v contiguous), B = W read N-major
    StoreBf16Epilogue::Params hp{grad_hidden + r0 * h, h, nc, h, nullptr};
    A3PO_RETURN_IF((launch_grad_gemm<StoreBf16Epilogue, false, true>(Operand{dz, nc, v, vpad}, Operand{w, h, v, h}, hp,
                                                                     dyn_m, true, select, status, stream)));
    // grad_w[v, j] (+)= sum_t dz[t, v] hidden[t, j]:  A = dz read M-major, B = hidden read N-major (K = t)
    StoreF32Epilogue::Params wp{grad_w, h, v, h, (accumulate || r0 > 0) ? 1 : 0};
    A3PO_RETURN_IF((launch_grad_gemm<StoreF32Epilogue, true, true>(Operand{dz, v, nc, vpad}, Operand{hid_c, h, nc, h},
                                                                   wp, dyn_k, false, nullptr, status, stream)));
  }
  return A3PO_OK;
}

// The two contractions of the backward on kept probability ratios q [n, v^8] (rows of one launch of the
// keeping forward, `dyn_offset` rows into the compact row space whose size is *dyn_rows):
//   grad_hidden[r, :] = row_scale[r] * sum_v q[r, v] W[v, :]
//   grad_w[v, :]    (+)= sum_r q[r, v] hs[r, :]                 hs = row_scale * hidden, made by the caller
// which equal dz W and dz^T hidden for dz[r, v] = row_scale[r] q[r, v].
int lmhead_grad_hidden_from_kept_tc(const void* q_, const void* w_, const float* row_scale, long long n, int h, int v,
                                    void* grad_hidden_, const int* dyn_rows, long long dyn_offset, int* select,
                                    uint32_t* status, cudaStream_t stream) {
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(q_);
  const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(w_);
  const int vpad = static_cast<int>(round_up(static_cast<size_t>(v), 8));
  DynRows dyn_m;
  dyn_m.rows = dyn_rows;
  dyn_m.offset = dyn_offset;
  dyn_m.cap = n;
  StoreBf16Epilogue::Params hp{static_cast<__nv_bfloat16*>(grad_hidden_), h, n, h, row_scale};
  return launch_grad_gemm<StoreBf16Epilogue, false, true>(Operand{q, n, v, vpad}, Operand{w, h, v, h}, hp, dyn_m, true,
                                                          select, status, stream);
}

int lmhead_grad_w_from_kept_tc(const void* q_, const void* hs_, long long n, int h, int v, float* grad_w,
                               int accumulate, int zero_when_empty, const int* dyn_rows, long long dyn_offset,
                               uint32_t* status, cudaStream_t stream) {
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(q_);
  const __nv_bfloat16* hs = static_cast<const __nv_bfloat16*>(hs_);
  const int vpad = static_cast<int>(round_up(static_cast<size_t>(v), 8));
  DynRows dyn_k;
  dyn_k.rows = dyn_rows;
  dyn_k.offset = dyn_offset;
  dyn_k.cap = n;
  dyn_k.is_k = 1;
  dyn_k.zero_when_empty = zero_when_empty;
  StoreF32Epilogue::Params wp{grad_w, h, v, h, accumulate ? 1 : 0};
  return launch_grad_gemm<StoreF32Epilogue, true, true>(Operand{q, v, n, vpad}, Operand{hs, h, n, h}, wp, dyn_k, false,
                                                        nullptr, status, stream);
}

}  // namespace a3po
