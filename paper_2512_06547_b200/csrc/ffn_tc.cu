// Gated feed-forward block on the sm_100a tensor cores: the contractions of gemm_tc.cuh with the block's own epilogues.
//
//   gate/up   A = x, B tile = 128 rows of Wg and the same 128 of Wu: the two accumulators of a hidden unit lie in the
//             same TMEM lane 128 columns apart, so the epilogue thread that owns the row has both and writes
//             h = act(g) u; g and u themselves never leave the SM unless a backward will need them
//   dgate/up  A = dy, B = Wd read N-major: dh stays in TMEM; the epilogue reads the kept g and u of its elements and
//             writes dg, du and (again) h, the operands of the three gradient contractions
//   down, dx, dW   plain contractions
//
// Rounding: h, dg, du and the kept g and u are bf16, because they are operands of bf16 matrix instructions (and half
// the bytes); each costs half a step (2^-9 relative) of an element that enters a long sum.  Everything between (the
// activation, the products, dh) is fp32.

#include "ffn_internal.cuh"
#include "gemm_tc.cuh"

namespace a3po {
namespace {

__device__ __forceinline__ uint4 pack8(const float (&v)[kEpiChunk], int q) {
  uint4 u;
  u.x = pack_bf16x2(v[q * 8 + 0], v[q * 8 + 1]);
  u.y = pack_bf16x2(v[q * 8 + 2], v[q * 8 + 3]);
  u.z = pack_bf16x2(v[q * 8 + 4], v[q * 8 + 5]);
  u.w = pack_bf16x2(v[q * 8 + 6], v[q * 8 + 7]);
  return u;
}

template <bool GELU, bool KEEP>
struct GateUpEpilogue {
  static constexpr int kKernelId = kKFfnGate;
  static constexpr bool kGated = true;
  struct Params {
    __nv_bfloat16* hid;    // [n, f]
    __nv_bfloat16* kept;   // see ffn_internal.cuh
    long long n;
    int b_rows;            // f: rows of each of the two stacked matrices
  };
  static int make_c_map(const Params& p, CUtensorMap* map) { return make_out_map(map, p.hid, 2, p.b_rows, p.n, p.b_rows); }
  uint8_t* cur;
  __device__ __forceinline__ void begin(const Params&, long long) {}
  __device__ __forceinline__ void chunk_pair(const Params& p, int tile_row0, int col0, uint32_t (&rg)[kEpiChunk],
                                             uint32_t (&ru)[kEpiChunk], SlabStore& st) {
    if (KEEP && col0 < p.b_rows) {
      uint4* k = reinterpret_cast<uint4*>(p.kept + kept_offset(tile_row0 + st.row_in_tile, col0, p.b_rows));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint4 a, b;
        a.x = pack_bf16x2(bits_to_float(rg[q * 8 + 0]), bits_to_float(rg[q * 8 + 1]));
        a.y = pack_bf16x2(bits_to_float(rg[q * 8 + 2]), bits_to_float(rg[q * 8 + 3]));
        a.z = pack_bf16x2(bits_to_float(rg[q * 8 + 4]), bits_to_float(rg[q * 8 + 5]));
        a.w = pack_bf16x2(bits_to_float(rg[q * 8 + 6]), bits_to_float(rg[q * 8 + 7]));
        b.x = pack_bf16x2(bits_to_float(ru[q * 8 + 0]), bits_to_float(ru[q * 8 + 1]));
        b.y = pack_bf16x2(bits_to_float(ru[q * 8 + 2]), bits_to_float(ru[q * 8 + 3]));
        b.z = pack_bf16x2(bits_to_float(ru[q * 8 + 4]), bits_to_float(ru[q * 8 + 5]));
        b.w = pack_bf16x2(bits_to_float(ru[q * 8 + 6]), bits_to_float(ru[q * 8 + 7]));
        __stcs(k + q * kKeptRows, a);
        __stcs(k + q * kKeptRows + kKeptElems / 8, b);
      }
    }
    float hv[kEpiChunk];
#pragma unroll
    for (int j = 0; j < kEpiChunk; ++j) {
      float a, slope;
      gate_activation<GELU>(bits_to_float(rg[j]), a, slope);
      hv[j] = a * bits_to_float(ru[j]);
    }
    const int half = (col0 >> 5) & 1;   // a slab holds 64 columns
    if (half == 0) cur = st.acquire();
#pragma unroll
    for (int q = 0; q < 4; ++q) *st.piece(cur, half * 4 + q) = pack8(hv, q);
    if (half == 1) st.submit(cur, col0 - 32, tile_row0, col0 - 32 < p.b_rows, false);
  }
  __device__ __forceinline__ void end(const Params&, long long, int) {}
};

// dg | du | h of 32 columns at a time: three 128-row x 64-byte slabs in the staging area and one three-dimensional
// output tensor [rows][3][f], so that each of the three is clipped at its own column f.
template <bool GELU>
struct GradGateUpEpilogue : PlainEpilogue {
  static constexpr int kKernelId = kKFfnGradGate;
  struct Params {
    const __nv_bfloat16* kept;
    __nv_bfloat16* z;   // [n][3][f]
    long long n;        // rows of z
    int f;
  };
  static int make_c_map(const Params& p, CUtensorMap* map) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return A3PO_ERR_CUDA;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(p.f), 3, static_cast<cuuint64_t>(p.n)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(p.f) * 2, static_cast<cuuint64_t>(p.f) * 6};
    const cuuint32_t box[3] = {kEpiChunk, 1, static_cast<cuuint32_t>(BM)};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.z, dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? A3PO_OK : A3PO_ERR_CUDA;
  }
  static constexpr uint32_t kPart = BM * kEpiChunk * 2;   // 8 KB
  long long row;
  __device__ __forceinline__ void begin(const Params&, long long row_) { row = row_; }
  // 16-byte piece j (0..3) of this thread's row in a slab of 64-byte rows with the 64-byte swizzle
  static __device__ __forceinline__ uint4* piece(uint8_t* s, int r, int j) {
    return reinterpret_cast<uint4*>(s + r * 64 + ((j ^ ((r >> 1) & 3)) << 4));
  }
  __device__ __forceinline__ void chunk(const Params& p, int tile_row0, int col0, uint32_t (&r)[kEpiChunk],
                                        SlabStore& st) {
    if (col0 >= p.f) return;   // the same for all threads
    const uint4* k = reinterpret_cast<const uint4*>(p.kept + kept_offset(row, col0, p.f));
    uint4 kg[4], ku[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      kg[q] = __ldcs(k + q * kKeptRows);
      ku[q] = __ldcs(k + q * kKeptRows + kKeptElems / 8);
    }
    if (st.issuer) bulk_wait_group_read<0>();   // the previous 32 columns have left the staging area
    named_barrier_sync(SlabStore::kBarrierId, 128);
    uint8_t* s = st.slab0;   // the two slabs of the staging area are contiguous
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t wg[4] = {kg[q].x, kg[q].y, kg[q].z, kg[q].w}, wu[4] = {ku[q].x, ku[q].y, ku[q].z, ku[q].w};
      uint32_t og[4], ou[4], oh[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float dg[2], du[2], hh[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float g = __uint_as_float(e ? wg[i] & 0xffff0000u : wg[i] << 16);
          const float u = __uint_as_float(e ? wu[i] & 0xffff0000u : wu[i] << 16);
          const float dh = bits_to_float(r[q * 8 + i * 2 + e]);
          float a, slope;
          gate_activation<GELU>(g, a, slope);
          dg[e] = dh * u * slope;
          du[e] = dh * a;
          hh[e] = a * u;
        }
        og[i] = pack_bf16x2(dg[0], dg[1]);
        ou[i] = pack_bf16x2(du[0], du[1]);
        oh[i] = pack_bf16x2(hh[0], hh[1]);
      }
      *piece(s, st.row_in_tile, q) = make_uint4(og[0], og[1], og[2], og[3]);
      *piece(s + kPart, st.row_in_tile, q) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
      *piece(s + 2 * kPart, st.row_in_tile, q) = make_uint4(oh[0], oh[1], oh[2], oh[3]);
    }
    fence_proxy_async_smem();
    named_barrier_sync(SlabStore::kBarrierId, 128);
    if (st.issuer) {
#pragma unroll
      for (int w = 0; w < 3; ++w) tma_store_3d(st.map, s + w * kPart, col0, w, tile_row0);
      bulk_commit_group();
    }
  }
  __device__ __forceinline__ void end(const Params&, long long, int) {}
};

// out[r, c] = sum over parts, in index order.  8 columns per thread.
__global__ void __launch_bounds__(256)
add_parts_kernel(const float* __restrict__ parts, int n_parts, long long part_stride, long long n, int cols,
                 const int* __restrict__ dyn_rows, __nv_bfloat16* __restrict__ out) {
  const long long rows = dyn_rows ? (*dyn_rows < n ? *dyn_rows : n) : n;
  const int groups = cols / 8;
  const long long total = rows * groups;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < total;
       i += static_cast<long long>(gridDim.x) * 256) {
    const float* src = parts + i * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    for (int p = 0; p < n_parts; ++p) {
      const float4 a = __ldcs(reinterpret_cast<const float4*>(src + p * part_stride));
      const float4 b = __ldcs(reinterpret_cast<const float4*>(src + p * part_stride) + 1);
      v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
      v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    uint4 u;
    u.x = pack_bf16x2(v[0], v[1]);
    u.y = pack_bf16x2(v[2], v[3]);
    u.z = pack_bf16x2(v[4], v[5]);
    u.w = pack_bf16x2(v[6], v[7]);
    reinterpret_cast<uint4*>(out)[i] = u;
  }
}

DynRows rows_as_m(const int* dyn_rows, long long n) {
  DynRows d;
  d.rows = dyn_rows;
  d.cap = n;
  return d;
}

// Rows and columns of the output are the token rows and h: a contraction over a long K with, for few tokens, far fewer
// output tiles than SMs.
template <int ID, bool B_MN>
int rows_gemm(const Operand& a, const Operand& b, __nv_bfloat16* out, float* parts, const int* dyn_rows, int* select,
              uint32_t* status, cudaStream_t stream) {
  const long long n = a.mn_extent;
  const int cols = static_cast<int>(b.mn_extent);
  const int k_parts = parts ? ffn_k_parts(n, cols, static_cast<int>(a.k_extent)) : 1;
  if (k_parts > 1) {
    const long long rows_pad = (n + BM - 1) / BM * BM;
    typename StoreF32EpilogueT<ID>::Params ep{parts, cols, rows_pad * k_parts, cols, 0};
    A3PO_RETURN_IF((launch_gemm<StoreF32EpilogueT<ID>, false, B_MN, 1>(a, b, 0, ep, rows_as_m(dyn_rows, n), status,
                                                                      stream, k_parts)));
    const long long want = (n * (cols / 8) + 255) / 256;
    const int blocks = static_cast<int>(want < sm_count() * 8ll ? want : sm_count() * 8ll);
    A3PO_LAUNCH(ID, stream, (add_parts_kernel<<<blocks, 256, 0, stream>>>(parts, k_parts, rows_pad * cols, n, cols,
                                                                          dyn_rows, out)));
    return after_launch();
  }
  typename StoreBf16EpilogueT<ID>::Params ep{out, cols, n, cols, nullptr};
  return launch_grad_gemm<StoreBf16EpilogueT<ID>, false, B_MN>(a, b, ep, rows_as_m(dyn_rows, n), true, select, status,
                                                               stream);
}

// Weight gradient C[m, c] = A^T B over the token rows (both operands read with the token index as K).
template <class Epi>
int weight_gemm(const Operand& a, const Operand& b, const typename Epi::Params& ep, int accumulate,
                const int* dyn_rows, uint32_t* status, cudaStream_t stream) {
  DynRows d = rows_as_m(dyn_rows, a.k_extent);
  d.is_k = 1;
  d.zero_when_empty = accumulate ? 0 : 1;
  const int n_tiles = static_cast<int>((b.mn_extent + BN - 1) / BN);
  if (choose_mt(a.mn_extent, n_tiles, sm_count()) == 1)
    return launch_gemm<Epi, true, true, 1>(a, b, 0, ep, d, status, stream);
  return launch_gemm<Epi, true, true, 2>(a, b, 0, ep, d, status, stream);
}

}  // namespace

int ffn_gate_up_tc(const void* x, const void* w_gate_up, long long n, int h, int f, a3po_activation act, void* hid,
                   void* kept, const int* dyn_rows, uint32_t* status, cudaStream_t stream) {
  const Operand a{x, n, h, h}, b{w_gate_up, 2ll * f, h, h};
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(hid);
  __nv_bfloat16* k = static_cast<__nv_bfloat16*>(kept);
  const DynRows d = rows_as_m(dyn_rows, n);
#define A3PO_GATE_UP(G, K)                                                                              \
  launch_gemm<GateUpEpilogue<G, K>, false, false>(a, b, 0, typename GateUpEpilogue<G, K>::Params{o, k, n, f}, d, status, \
                                                  stream)
  if (act == A3PO_ACT_GELU_TANH) return kept ? A3PO_GATE_UP(true, true) : A3PO_GATE_UP(true, false);
  return kept ? A3PO_GATE_UP(false, true) : A3PO_GATE_UP(false, false);
#undef A3PO_GATE_UP
}

int ffn_k_parts(long long n, int cols, int k) {
  const long long tiles = ((n + BM - 1) / BM) * ((cols + BN - 1) / BN);
  const int sms = sm_count() > 0 ? sm_count() : 148;
  if (tiles <= 0 || tiles * 2 > sms) return 1;
  const int k_blocks = (k + BK - 1) / BK;
  long long parts = sms / tiles;
  if (parts > k_blocks / 8) parts = k_blocks / 8;
  return parts > 1 ? static_cast<int>(parts) : 1;
}

size_t ffn_parts_bytes(long long n, int cols, int k) {
  const int parts = ffn_k_parts(n, cols, k);
  return parts > 1 ? static_cast<size_t>((n + BM - 1) / BM * BM) * cols * parts * sizeof(float) : 0;
}

int ffn_down_tc(const void* hid, const void* w_down, long long n, int h, int f, void* y, float* parts,
                const int* dyn_rows, int* select, uint32_t* status, cudaStream_t stream) {
  return rows_gemm<kKFfnDown, false>(Operand{hid, n, f, f}, Operand{w_down, h, f, f}, static_cast<__nv_bfloat16*>(y),
                                     parts, dyn_rows, select, status, stream);
}

int ffn_grad_gate_up_tc(const void* grad_y, const void* w_down, const void* kept, long long n, int h, int f,
                        a3po_activation act, void* z, const int* dyn_rows, uint32_t* status, cudaStream_t stream) {
  const Operand a{grad_y, n, h, h}, b{w_down, f, h, f};
  const DynRows d = rows_as_m(dyn_rows, n);
  const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(kept);
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(z);
  if (act == A3PO_ACT_GELU_TANH)
    return launch_gemm<GradGateUpEpilogue<true>, false, true>(a, b, 0, GradGateUpEpilogue<true>::Params{k, o, n, f}, d,
                                                              status, stream);
  return launch_gemm<GradGateUpEpilogue<false>, false, true>(a, b, 0, GradGateUpEpilogue<false>::Params{k, o, n, f}, d,
                                                             status, stream);
}

int ffn_grad_x_tc(const void* z, const void* w_gate_up, long long n, int h, int f, void* grad_x, float* parts,
                  const int* dyn_rows, int* select, uint32_t* status, cudaStream_t stream) {
  return rows_gemm<kKFfnGradX, true>(Operand{z, n, 2ll * f, 3ll * f}, Operand{w_gate_up, h, 2ll * f, h},
                                     static_cast<__nv_bfloat16*>(grad_x), parts, dyn_rows, select, status, stream);
}

int ffn_grad_w_tc(const void* z_, const void* x, const void* grad_y, long long n, int h, int f, void* grad_w_gate_up,
                  void* grad_w_down, a3po_dtype grad_dt, int accumulate, const int* dyn_rows, uint32_t* status,
                  cudaStream_t stream) {
  const __nv_bfloat16* z = static_cast<const __nv_bfloat16*>(z_);
  const Operand dgu{z, 2ll * f, n, 3ll * f}, xo{x, h, n, h};           // [dg | du]^T x
  const Operand dy{grad_y, h, n, h}, hid{z + 2ll * f, f, n, 3ll * f};  // dy^T h
  if (grad_dt == A3PO_F32) {
    using Epi = StoreF32EpilogueT<kKFfnGradW>;
    A3PO_RETURN_IF((weight_gemm<Epi>(dgu, xo, Epi::Params{static_cast<float*>(grad_w_gate_up), h, 2ll * f, h, accumulate},
                                     accumulate, dyn_rows, status, stream)));
    return weight_gemm<Epi>(dy, hid, Epi::Params{static_cast<float*>(grad_w_down), f, h, f, accumulate}, accumulate,
                            dyn_rows, status, stream);
  }
  using Epi = StoreBf16EpilogueT<kKFfnGradW>;
  A3PO_RETURN_IF((weight_gemm<Epi>(dgu, xo, Epi::Params{static_cast<__nv_bfloat16*>(grad_w_gate_up), h, 2ll * f, h, nullptr},
                                   0, dyn_rows, status, stream)));
  return weight_gemm<Epi>(dy, hid, Epi::Params{static_cast<__nv_bfloat16*>(grad_w_down), f, h, f, nullptr}, 0, dyn_rows,
                          status, stream);
}

}  // namespace a3po
