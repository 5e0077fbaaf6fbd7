// Gated feed-forward block on the sm_100a tensor cores: the contractions of gemm_tc.cuh with the block's own epilogues.
//
//   gate/up   A = x, B tile = 128 rows of Wg and the same 128 of Wu: the two accumulators of a hidden unit lie in the
//             same TMEM lane 128 columns apart, so the epilogue thread that owns the row has both and writes
//             h = act(g) u; g and u themselves never leave the SM unless a backward will need them
//   dgate/up  A = dy, B = Wd read N-major: dh stays in TMEM; the epilogue reads the kept g and u of its elements and
//             writes dg and du, operands of two gradient contractions (h, the third's, is the forward's own)
//   down, dx, dW   plain contractions
//
// Rounding: h, dg and du are bf16, because they are operands of bf16 matrix instructions; each costs half a step (2^-8
// relative at most) of an element that enters a long sum.  The kept g and u are cut to 24 bits (ffn_internal.cuh).  Everything
// between (the activation, the products, dh) is fp32.
//
// Bound: the tensor pipe, 90-97 % active at the clock that the board's power cap leaves (profiler, 9,472 rows, H 4096,
// F 12288).  Forward and backward: 16,384 rows of 4096 x 12288 11.4-12.2 ms (1,220-1,300 TFLOP/s; the six bare products in
// cuBLAS take 10.3-10.7), 10,240 rows of 1536 x 4608 1.10 ms (1,190 TFLOP/s; cuBLAS 1.01).

#include "contract.cuh"

namespace a3po {
namespace {

// The upper 24 bits of 32 fp32 values: 16-byte pieces of their upper halves and of their third bytes, kKeptRows apart.
__device__ __forceinline__ void keep24(const uint32_t (&v)[kEpiChunk], uint8_t* upper, uint8_t* third) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __byte_perm(v[q * 8 + i * 2], v[q * 8 + i * 2 + 1], 0x7632);
    __stcs(reinterpret_cast<uint4*>(upper) + q * kKeptRows, make_uint4(w[0], w[1], w[2], w[3]));
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t* e = v + q * 16 + i * 4;
      w[i] = __byte_perm(__byte_perm(e[0], e[1], 0x0051), __byte_perm(e[2], e[3], 0x0051), 0x5410);
    }
    __stcs(reinterpret_cast<uint4*>(third) + q * kKeptRows, make_uint4(w[0], w[1], w[2], w[3]));
  }
}
// Value e (0 or 1) of a word of upper halves, with its third byte b (0..3) of word t; the lowest byte repeats the third,
// which is below what is kept.
__device__ __forceinline__ float kept24(uint32_t upper, int e, uint32_t third, int b) {
  return __uint_as_float(__byte_perm(upper, third, (e ? 0x3200u : 0x1000u) | static_cast<uint32_t>(0x44 + b * 0x11)));
}

template <bool GELU, bool KEEP>
struct GateUpEpilogue {
  static constexpr int kKernelId = kKFfnGate;
  static constexpr bool kGated = true;
  static constexpr bool kPrefetch = false;
  static constexpr int kGroups = 2;
  static constexpr bool kChained = true;
  static constexpr bool kSplitK = false;
  static constexpr int kPromote = 0;
  struct Params {
    __nv_bfloat16* hid;    // [n, f]
    uint8_t* kept;         // see ffn_internal.cuh
    long long n;
    int b_rows;            // f: rows of each of the two stacked matrices
  };
  static int make_c_map(const Params& p, CUtensorMap* map) { return make_out_map(map, p.hid, 2, p.b_rows, p.n, p.b_rows); }
  uint8_t* cur;
  __device__ __forceinline__ void begin(const Params&, long long) {}
  __device__ __forceinline__ void chunk_pair(const Params& p, int tile_row0, int col0, uint32_t (&rg)[kEpiChunk],
                                             uint32_t (&ru)[kEpiChunk], SlabStore& st) {
    if (KEEP && col0 < p.b_rows && tile_row0 < p.n) {   // a pair's second tile may lie past the buffers
      uint8_t* tile = p.kept + kept_tile(tile_row0, col0, p.b_rows) + st.row_in_tile * 16;
      keep24(rg, tile, tile + 2 * kKeptUpper);
      keep24(ru, tile + kKeptUpper, tile + 2 * kKeptUpper + kKeptThird);
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
    if (half == 1) st.submit(cur, col0 - 32, tile_row0, col0 - 32 < p.b_rows && tile_row0 < p.n, false);
  }
  __device__ __forceinline__ void end(const Params&, long long, int) {}
};

// dg | du of 32 columns at a time: two 128-row x 64-byte halves of a slab and one three-dimensional output tensor
// [rows][2][f], so that each of the two is clipped at its own column f.
template <bool GELU>
struct GradGateUpEpilogue : PlainEpilogue {
  static constexpr bool kChained = true;
  static constexpr bool kPrefetch = true;
  static constexpr int kGroups = 2;
  static constexpr int kKernelId = kKFfnGradGate;
  struct Params {
    const uint8_t* kept;
    __nv_bfloat16* z;   // [n][2][f]
    long long n;        // rows of z
    int f;
  };
  static int make_c_map(const Params& p, CUtensorMap* map) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return A3PO_ERR_CUDA;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(p.f), 2, static_cast<cuuint64_t>(p.n)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(p.f) * 2, static_cast<cuuint64_t>(p.f) * 4};
    const cuuint32_t box[3] = {kEpiChunk, 1, static_cast<cuuint32_t>(BM)};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.z, dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? A3PO_OK : A3PO_ERR_CUDA;
  }
  static constexpr uint32_t kPart = BM * kEpiChunk * 2;   // 8 KB
  long long row;
  int end_col;                  // of the columns that this thread works through in the tile
  uint4 next_g[6], next_u[6];   // g and u of the columns that come next: upper halves, third bytes
  __device__ __forceinline__ void read_kept(const Params& p, int col0) {
    const uint8_t* tile = p.kept + kept_tile(row, col0, p.f) + (row % kKeptRows) * 16;
    const uint4* g = reinterpret_cast<const uint4*>(tile);
    const uint4* t = reinterpret_cast<const uint4*>(tile + 2 * kKeptUpper);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      next_g[q] = __ldcs(g + q * kKeptRows);
      next_u[q] = __ldcs(g + kKeptUpper / 16 + q * kKeptRows);
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      next_g[4 + q] = __ldcs(t + q * kKeptRows);
      next_u[4 + q] = __ldcs(t + kKeptThird / 16 + q * kKeptRows);
    }
  }
  __device__ __forceinline__ void begin(const Params&, long long row_) { row = row_; }
  // before the tile's product is waited for
  __device__ __forceinline__ void prefetch(const Params& p, int tile_row0, int col0, int cols) {
    end_col = min(col0 + cols, p.f);
    if (col0 < p.f && tile_row0 < p.n) read_kept(p, col0);
  }
  // 16-byte piece j (0..3) of this thread's row in a slab of 64-byte rows with the 64-byte swizzle
  static __device__ __forceinline__ uint4* piece(uint8_t* s, int r, int j) {
    return reinterpret_cast<uint4*>(s + r * 64 + ((j ^ ((r >> 1) & 3)) << 4));
  }
  __device__ __forceinline__ void chunk(const Params& p, int tile_row0, int col0, uint32_t (&r)[kEpiChunk],
                                        SlabStore& st) {
    if (col0 >= p.f || tile_row0 >= p.n) return;   // the same for all threads
    uint4 kg[6], ku[6];
#pragma unroll
    for (int q = 0; q < 6; ++q) {
      kg[q] = next_g[q];
      ku[q] = next_u[q];
    }
    if (col0 + kEpiChunk < end_col) read_kept(p, col0 + kEpiChunk);   // the next 32 columns, while these are worked on
    uint4 og[4], ou[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t wg[4] = {kg[q].x, kg[q].y, kg[q].z, kg[q].w}, wu[4] = {ku[q].x, ku[q].y, ku[q].z, ku[q].w};
      const uint4 tg = kg[4 + q / 2], tu = ku[4 + q / 2];   // third bytes of columns 16 (q / 2) .. + 15
      const uint32_t bg[2] = {q % 2 ? tg.z : tg.x, q % 2 ? tg.w : tg.y}, bu[2] = {q % 2 ? tu.z : tu.x, q % 2 ? tu.w : tu.y};
      uint32_t vg[4], vu[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float dg[2], du[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float g = kept24(wg[i], e, bg[i / 2], (i % 2) * 2 + e);
          const float u = kept24(wu[i], e, bu[i / 2], (i % 2) * 2 + e);
          const float dh = bits_to_float(r[q * 8 + i * 2 + e]);
          float a, slope;
          gate_activation<GELU>(g, a, slope);
          dg[e] = dh * u * slope;
          du[e] = dh * a;
        }
        vg[i] = pack_bf16x2(dg[0], dg[1]);
        vu[i] = pack_bf16x2(du[0], du[1]);
      }
      og[q] = make_uint4(vg[0], vg[1], vg[2], vg[3]);
      ou[q] = make_uint4(vu[0], vu[1], vu[2], vu[3]);
    }
    uint8_t* s = st.acquire();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      *piece(s, st.row_in_tile, q) = og[q];
      *piece(s + kPart, st.row_in_tile, q) = ou[q];
    }
    fence_proxy_async_smem();
    named_barrier_sync(st.barrier_id, 128);
    if (st.issuer) {
      tma_store_3d(st.map, s, col0, 0, tile_row0);
      tma_store_3d(st.map, s + kPart, col0, 1, tile_row0);
      bulk_commit_group();
    }
    ++st.issued;
  }
  __device__ __forceinline__ void end(const Params&, long long, int) {}
};

}  // namespace

int ffn_gate_up_tc(const void* x, const void* w_gate_up, long long n, int h, int f, a3po_activation act, void* hid,
                   void* kept, const int* dyn_rows, uint32_t* status, cudaStream_t stream) {
  const Operand a{x, n, h, h}, b{w_gate_up, 2ll * f, h, h};
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(hid);
  uint8_t* k = static_cast<uint8_t*>(kept);
  const DynRows d = rows_as_m(dyn_rows, n);
#define A3PO_GATE_UP(G, K)                                                                                        \
  contract<GateUpEpilogue<G, K>, false, false>(a, b, typename GateUpEpilogue<G, K>::Params{o, k, n, f}, d, status, \
                                               stream, first_launch(dyn_rows))
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
                const int* dyn_rows, uint32_t* status, cudaStream_t stream) {
  return rows_gemm<kKFfnDown, false>(Operand{hid, n, f, f}, Operand{w_down, h, f, f}, static_cast<__nv_bfloat16*>(y),
                                     parts, dyn_rows, status, stream, Begin::kEarly);
}

int ffn_grad_gate_up_tc(const void* grad_y, const void* w_down, const void* kept, long long n, int h, int f,
                        a3po_activation act, void* z, const int* dyn_rows, uint32_t* status, cudaStream_t stream) {
  const Operand a{grad_y, n, h, h}, b{w_down, f, h, f};
  const DynRows d = rows_as_m(dyn_rows, n);
  const uint8_t* k = static_cast<const uint8_t*>(kept);
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(z);
  if (act == A3PO_ACT_GELU_TANH)
    return contract<GradGateUpEpilogue<true>, false, true>(a, b, GradGateUpEpilogue<true>::Params{k, o, n, f}, d, status,
                                                           stream, first_launch(dyn_rows));
  return contract<GradGateUpEpilogue<false>, false, true>(a, b, GradGateUpEpilogue<false>::Params{k, o, n, f}, d, status,
                                                          stream, first_launch(dyn_rows));
}

int ffn_grad_x_tc(const void* z, const void* w_gate_up, long long n, int h, int f, void* grad_x, float* parts,
                  const int* dyn_rows, uint32_t* status, cudaStream_t stream) {
  return rows_gemm<kKFfnGradX, true>(Operand{z, n, 2ll * f, 2ll * f}, Operand{w_gate_up, h, 2ll * f, h},
                                     static_cast<__nv_bfloat16*>(grad_x), parts, dyn_rows, status, stream, Begin::kBeside);
}

int ffn_grad_w_tc(const void* z, const void* hid_, const void* x, const void* grad_y, long long n, int h, int f,
                  void* grad_w_gate_up, void* grad_w_down, a3po_dtype grad_dt, int accumulate, const int* dyn_rows,
                  uint32_t* status, cudaStream_t stream) {
  const Operand dgu{z, 2ll * f, n, 2ll * f}, xo{x, h, n, h};   // [dg | du]^T x
  const Operand dy{grad_y, h, n, h}, hid{hid_, f, n, f};       // dy^T h
  if (grad_dt == A3PO_F32) {
    using Epi = StoreF32EpilogueT<kKFfnGradW>;
    A3PO_RETURN_IF((weight_gemm<Epi>(dgu, xo, Epi::Params{static_cast<float*>(grad_w_gate_up), h, 2ll * f, h, accumulate},
                                     accumulate, dyn_rows, status, stream, Begin::kEarly)));
    return weight_gemm<Epi>(dy, hid, Epi::Params{static_cast<float*>(grad_w_down), f, h, f, accumulate}, accumulate,
                            dyn_rows, status, stream, Begin::kBeside);
  }
  using Epi = StoreBf16EpilogueT<kKFfnGradW>;
  A3PO_RETURN_IF((weight_gemm<Epi>(dgu, xo, Epi::Params{static_cast<__nv_bfloat16*>(grad_w_gate_up), h, 2ll * f, h, nullptr},
                                   0, dyn_rows, status, stream, Begin::kEarly)));
  return weight_gemm<Epi>(dy, hid, Epi::Params{static_cast<__nv_bfloat16*>(grad_w_down), f, h, f, nullptr}, 0, dyn_rows,
                          status, stream, Begin::kBeside);
}

}  // namespace a3po
