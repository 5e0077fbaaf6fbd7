// Launches of the tcgen05 contractions (gemm_tc.cuh) that the feed-forward block and the linear operator have in common: pairs of
// CTAs or single ones, K splits of products with few output tiles, weight gradients.
#pragma once

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

// Partial products of a K split, fp32: part s of output row r at [s][r].  The tensor is three-dimensional so that the copy
// engine clips each part at the rows that exist (of a 128-row tile a few are real when few tokens come).
template <int KERNEL_ID>
struct StorePartsEpilogue : PlainEpilogue {
  static constexpr int kKernelId = KERNEL_ID;
  static constexpr bool kChained = true;
  static constexpr bool kSplitK = true;
  struct Params {
    float* c;
    long long n;          // rows of a part
    int rows_pad;         // from part to part; tile rows count on through the parts (ItemMap::k_split_rows)
    int parts;
    int n_cols;           // multiple of 8
  };
  static int make_c_map(const Params& p, CUtensorMap* map) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return A3PO_ERR_CUDA;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(p.n_cols), static_cast<cuuint64_t>(p.n),
                                static_cast<cuuint64_t>(p.parts)};
    const cuuint64_t row = static_cast<cuuint64_t>(p.n_cols) * sizeof(float);
    const cuuint64_t strides[2] = {row, row * static_cast<cuuint64_t>(p.rows_pad)};
    const cuuint32_t box[3] = {kEpiChunk, static_cast<cuuint32_t>(BM), 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, p.c, dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? A3PO_OK : A3PO_ERR_CUDA;
  }
  __device__ __forceinline__ void begin(const Params&, long long) {}
  __device__ __forceinline__ void chunk(const Params& p, int tile_row0, int col0, uint32_t (&r)[kEpiChunk], SlabStore& st) {
    uint8_t* s = st.acquire();
#pragma unroll
    for (int q = 0; q < 8; ++q) *st.piece(s, q) = make_uint4(r[q * 4 + 0], r[q * 4 + 1], r[q * 4 + 2], r[q * 4 + 3]);
    fence_proxy_async_smem();
    named_barrier_sync(st.barrier_id, 128);
    if (st.issuer) {
      const int part = tile_row0 / p.rows_pad, row0 = tile_row0 - part * p.rows_pad;
      if (col0 < p.n_cols && row0 < p.n) tma_store_3d(st.map, s, col0, row0, part);
      bulk_commit_group();
    }
    ++st.issued;
  }
  __device__ __forceinline__ void end(const Params&, long long, int) {}
};

// out[r, c] = sum over parts, in index order.  4 columns per thread, 8 parts on their way at a time.
constexpr int kAddCols = 4, kAddBatch = 8;
__global__ void __launch_bounds__(256)
add_parts_kernel(const float* parts, int n_parts, long long part_stride, long long n, int cols,
                 const int* dyn_rows, __nv_bfloat16* out) {
  wait_for_previous();
  allow_next();
  const long long rows = dyn_rows ? (*dyn_rows < n ? *dyn_rows : n) : n;
  const long long total = rows * (cols / kAddCols);
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < total;
       i += static_cast<long long>(gridDim.x) * 256) {
    const float* src = parts + i * kAddCols;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < n_parts; p0 += kAddBatch) {
      float4 a[kAddBatch];
#pragma unroll
      for (int k = 0; k < kAddBatch; ++k)
        a[k] = p0 + k < n_parts ? __ldcs(reinterpret_cast<const float4*>(src + (p0 + k) * part_stride))
                                : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kAddBatch; ++k) {
        v.x += a[k].x; v.y += a[k].y; v.z += a[k].z; v.w += a[k].w;
      }
    }
    reinterpret_cast<uint2*>(out)[i] = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
  }
}

// The first contraction of a call is its first launch unless the rows were compacted before.
Begin first_launch(const int* dyn_rows) { return dyn_rows ? Begin::kEarly : Begin::kAfter; }

DynRows rows_as_m(const int* dyn_rows, long long n) {
  DynRows d;
  d.rows = dyn_rows;
  d.cap = n;
  return d;
}

// Launches of fewer waves of tiles than this run unpaced: there is no time to drift apart, and a CTA that begins a tile later
// than the others (see Begin::kBeside) would be waited for (backward of 16,384 rows of 1536 x 4608, 1 to 6 waves a launch:
// 1,177 us paced, 1,144 unpaced; of 4096 x 12288, 10 to 21 waves, no difference between the two).
constexpr int kPacedWaves = 8;

// One contraction: pairs of CTAs on 256 x 256 tiles, or single CTAs when the output has at most 128 rows.
template <class Epi, bool A_MN, bool B_MN>
int contract(const Operand& a, const Operand& b, const typename Epi::Params& ep, const DynRows& dyn, uint32_t* status,
             cudaStream_t stream, Begin begin) {
  const bool pairs = a.mn_extent > BM || Epi::kPromote > 0;   // sums are taken out of the accumulators by the pair kernel alone
  const int rows = pairs ? 2 * BM : BM;
  const long long tiles = ((a.mn_extent + rows - 1) / rows) * ((b.mn_extent + BN - 1) / BN);
  const bool paced = (pairs ? 2 : 1) * tiles >= kPacedWaves * sm_count();
  if constexpr (Epi::kPromote == 0) {
    if (!pairs) return launch_gemm<Epi, A_MN, B_MN, 1>(a, b, 0, ep, dyn, status, stream, 1, begin, paced);
  }
  const int group = !A_MN && !B_MN ? fwd_group_m(a.k_extent, 2 * BM) : kGroupM;
  return launch_pair_gemm<Epi, A_MN, B_MN>(a, b, 0, ep, dyn, status, stream, group, paced, begin);
}

// Rows and columns of the output are the token rows and h: a contraction over a long K with, for few tokens, far fewer
// output tiles than SMs.
template <int ID, bool B_MN>
int rows_gemm(const Operand& a, const Operand& b, __nv_bfloat16* out, float* parts, const int* dyn_rows,
              uint32_t* status, cudaStream_t stream, Begin begin) {
  const long long n = a.mn_extent;
  const int cols = static_cast<int>(b.mn_extent);
  const int k_parts = parts ? ffn_k_parts(n, cols, static_cast<int>(a.k_extent)) : 1;
  if (k_parts > 1) {
    const long long rows_pad = (n + BM - 1) / BM * BM;
    typename StorePartsEpilogue<ID>::Params ep{parts, n, static_cast<int>(rows_pad), k_parts, cols};
    A3PO_RETURN_IF((launch_gemm<StorePartsEpilogue<ID>, false, B_MN, 1>(a, b, 0, ep, rows_as_m(dyn_rows, n), status,
                                                                       stream, k_parts, begin)));
    const long long want = (n * (cols / kAddCols) + 255) / 256;
    const int blocks = static_cast<int>(want < sm_count() * 8ll ? want : sm_count() * 8ll);
    A3PO_LAUNCH(ID, stream, (launch_early(add_parts_kernel, blocks, 256, 0, stream, 1, true,
                                          static_cast<const float*>(parts), k_parts, rows_pad * cols, n, cols, dyn_rows,
                                          out)));
    return after_launch();
  }
  typename StoreBf16EpilogueT<ID>::Params ep{out, cols, n, cols, nullptr};
  return contract<StoreBf16EpilogueT<ID>, false, B_MN>(a, b, ep, rows_as_m(dyn_rows, n), status, stream, begin);
}

// Weight gradient C[m, c] = A^T B over the token rows (both operands read with the token index as K).
template <class Epi>
int weight_gemm(const Operand& a, const Operand& b, const typename Epi::Params& ep, int accumulate,
                const int* dyn_rows, uint32_t* status, cudaStream_t stream, Begin begin) {
  DynRows d = rows_as_m(dyn_rows, a.k_extent);
  d.is_k = 1;
  d.zero_when_empty = accumulate ? 0 : 1;
  return contract<Epi, true, true>(a, b, ep, d, status, stream, begin);
}

}  // namespace
}  // namespace a3po
