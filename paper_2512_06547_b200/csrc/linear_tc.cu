// The linear operator on the sm_100a tensor cores: the contractions of gemm_tc.cuh with bias, activation, residual and the kept z
// in the epilogue, so that nothing but y (and z, for a backward) leaves the SM.
//
// Rounding: y is rounded once; dz is bf16, because it is an operand of bf16 matrix instructions (half a step, 2^-8 of an
// element at most, that enters a long sum), but its column sums, the bias gradient, are taken of the fp32 values.
//
// Bound: the tensor pipe (the products are those of the feed-forward block, see ffn_tc.cu).  10,240 of 16,384 rows, 1,536 to 4,608,
// with bias and SiLU: forward product 117 us (1,240 TFLOP/s; it also writes z, 189 MB), dz 87, weight gradient 111, input
// gradient 104; gathering x 15 there and 19 back, zeros 16.  16,384 rows of 4,096 to 4,096 with a residual and fp32 weight
// gradients: 365, 430 and 338 us, 1,125 in all (1,466 TFLOP/s).

#include "contract.cuh"
#include "linear_internal.cuh"

namespace a3po {
namespace {

// 8 consecutive bf16 as fp32.
__device__ __forceinline__ void unpack8(const uint4& u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// 32 bytes at a 32-byte boundary.
__device__ __forceinline__ void store_32(void* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w),
               "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
               : "memory");
}

// Outputs that stay in fp32 are sums of 512 products at a time (see PlainEpilogue::kPromote).
constexpr int kSumBlocks = 8;
// Sums over fewer rows are not split.  There and back, bf16: 16,384 rows of 128 x 128 58 us split, 102 as one tile's sum, of 512 x 512
// 84 and 134; 4,096 rows of 128 x 128 27 and 34, of 2,048 x 512 59 and 59; 1,024 rows of 128 x 128 27 and 24.
constexpr long long kSplitRows = 4096;

struct WeightGradEpilogue : StoreF32EpilogueT<kKLinearGradW> {
  static constexpr int kGroups = 2;
  static constexpr int kPromote = kSumBlocks;
};

// SCATTER: the rows are those of a compact row space and go straight to their places row_index[i] (32 bytes a store: whole
// sectors), so that no pass has to move them there; otherwise through the copy engine.
template <int ACT, bool KEEP, typename OUT, bool SCATTER = false, int KERNEL_ID = kKLinear>
struct LinearEpilogue : PlainEpilogue {
  static constexpr int kKernelId = KERNEL_ID;
  static constexpr bool kChained = true;
  static constexpr bool kPrefetch = true;
  static constexpr int kGroups = 2;
  static constexpr int kPromote = sizeof(OUT) == 4 ? kSumBlocks : 0;
  struct Params {
    OUT* y;
    const __nv_bfloat16 *bias, *residual;
    uint8_t* kept;
    const int *row_index, *count;   // SCATTER
    long long n;
    int m;
    int whole_sectors;              // SCATTER: rows start at 32-byte boundaries and end there
  };
  static int make_c_map(const Params& p, CUtensorMap* map) {
    return make_out_map(map, p.y, sizeof(OUT), p.m, p.n, p.m);
  }
  const __nv_bfloat16* res;   // this thread's row of the residual, or null
  OUT* out;                   // SCATTER: its row of y, or null
  int end_col;
  uint4 next[4];              // its next 32 columns
  uint8_t* cur;
  __device__ __forceinline__ void begin(const Params& p, long long row) {
    res = nullptr;
    out = nullptr;
    if (!SCATTER && !p.residual) return;
    if (row >= (SCATTER ? min(static_cast<long long>(*p.count), p.n) : p.n)) return;
    const long long at = (SCATTER ? p.row_index[row] : row) * static_cast<long long>(p.m);
    if (SCATTER) out = p.y + at;
    if (p.residual) res = p.residual + at;
  }
  __device__ __forceinline__ void read_residual(int col0) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      next[q] = res && col0 + q * 8 < end_col ? __ldcs(reinterpret_cast<const uint4*>(res + col0) + q) : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void prefetch(const Params& p, int, int col0, int cols) {
    end_col = min(col0 + cols, p.m);
    if (p.residual) read_residual(col0);
  }
  __device__ __forceinline__ void chunk(const Params& p, int tile_row0, int col0, uint32_t (&r)[kEpiChunk], SlabStore& st) {
    float v[kEpiChunk];
    const bool in = col0 < p.m && tile_row0 < p.n;   // the same for all threads
    if (p.bias && col0 < p.m) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float b[8] = {};
        if (col0 + q * 8 < p.m) unpack8(__ldg(reinterpret_cast<const uint4*>(p.bias + col0) + q), b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[q * 8 + i] = bits_to_float(r[q * 8 + i]) + b[i];
      }
    } else {
#pragma unroll
      for (int j = 0; j < kEpiChunk; ++j) v[j] = bits_to_float(r[j]);
    }
    if (KEEP && in) {   // a pair's second tile may lie past the buffer
      uint8_t* tile = p.kept + z_tile(tile_row0, col0, p.m) + st.row_in_tile * 16;
#pragma unroll
      for (int q = 0; q < 8; ++q)
        __stcs(reinterpret_cast<float4*>(tile) + q * kZRows, make_float4(v[q * 4], v[q * 4 + 1], v[q * 4 + 2], v[q * 4 + 3]));
    }
    if (ACT != kActNone) {
#pragma unroll
      for (int j = 0; j < kEpiChunk; ++j) {
        float a, slope;
        linear_activation<ACT>(v[j], a, slope);
        v[j] = a;
      }
    }
    if (p.residual) {
      uint4 now[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) now[q] = next[q];
      if (col0 + kEpiChunk < end_col) read_residual(col0 + kEpiChunk);   // while these are worked on
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float b[8];
        unpack8(now[q], b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[q * 8 + i] += b[i];
      }
    }
    if constexpr (SCATTER) {
      if (!out) return;   // no barriers on this path
      constexpr int kPer = 32 / sizeof(OUT), kStores = kEpiChunk / kPer;
#pragma unroll
      for (int q = 0; q < kStores; ++q) {
        const int c = col0 + q * kPer;
        if (c >= p.m) break;
        uint4 a, b;
        if constexpr (sizeof(OUT) == 4) {
          const float* f = v + q * 8;
          a = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
          b = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
        } else {
          a = pack8(v, 2 * q);
          b = pack8(v, 2 * q + 1);
        }
        if (p.whole_sectors) {
          store_32(out + c, a, b);
        } else {   // rows start at multiples of 16 bytes, and the second half may lie past the row
          *reinterpret_cast<uint4*>(out + c) = a;
          if (c + kPer / 2 < p.m) *reinterpret_cast<uint4*>(out + c + kPer / 2) = b;
        }
      }
    } else if constexpr (sizeof(OUT) == 4) {
      uint8_t* s = st.acquire();
#pragma unroll
      for (int q = 0; q < 8; ++q)
        *st.piece(s, q) = make_uint4(__float_as_uint(v[q * 4]), __float_as_uint(v[q * 4 + 1]), __float_as_uint(v[q * 4 + 2]),
                                     __float_as_uint(v[q * 4 + 3]));
      st.submit(s, col0, tile_row0, in, false);
    } else {
      const int half = (col0 >> 5) & 1;   // a slab holds 64 columns
      if (half == 0) cur = st.acquire();
#pragma unroll
      for (int q = 0; q < 4; ++q) *st.piece(cur, half * 4 + q) = pack8(v, q);
      if (half == 1) st.submit(cur, col0 - 32, tile_row0, col0 - 32 < p.m && tile_row0 < p.n, false);
    }
  }
  __device__ __forceinline__ void end(const Params&, long long, int) {}
};

// The same after the parts of a K split: 4 columns per thread, the parts in index order, 8 on their way at a time.
template <class Epi, int ACT, bool KEEP, typename OUT>
__global__ void __launch_bounds__(256)
linear_add_parts_kernel(const float* parts, int n_parts, long long part_stride, typename Epi::Params p) {
  wait_for_previous();
  allow_next();
  const long long rows = p.count ? (*p.count < p.n ? *p.count : p.n) : p.n;
  const int vecs = p.m / kAddCols;
  const long long total = rows * vecs;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < total;
       i += static_cast<long long>(gridDim.x) * 256) {
    const float* src = parts + i * kAddCols;
    float v[4] = {};
    for (int p0 = 0; p0 < n_parts; p0 += kAddBatch) {
      float4 a[kAddBatch];
#pragma unroll
      for (int k = 0; k < kAddBatch; ++k)
        a[k] = p0 + k < n_parts ? __ldcs(reinterpret_cast<const float4*>(src + (p0 + k) * part_stride))
                                : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kAddBatch; ++k) {
        v[0] += a[k].x; v[1] += a[k].y; v[2] += a[k].z; v[3] += a[k].w;
      }
    }
    const long long row = i / vecs;
    const int col = static_cast<int>(i - row * vecs) * kAddCols;
    if (p.bias) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += to_float(p.bias[col + j]);
    }
    if (KEEP) {
      uint8_t* tile = p.kept + z_tile(row, col, p.m);
      reinterpret_cast<float4*>(tile)[col % kZCols / 4 * kZRows + row % kZRows] = make_float4(v[0], v[1], v[2], v[3]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float a, slope;
      linear_activation<ACT>(v[j], a, slope);
      v[j] = a;
    }
    const long long at = (p.row_index ? p.row_index[row] : row) * static_cast<long long>(p.m) + col;
    if (p.residual) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += to_float(p.residual[at + j]);
    }
    if constexpr (sizeof(OUT) == 4) *reinterpret_cast<float4*>(p.y + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(p.y + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

// A weight gradient from the parts of a split over its rows: 4 columns per thread, the parts in index order, 8 on their way at a
// time.  Parts that got no k-block (the rows that take part are fewer than the buffer's) were not written.
template <typename OUT>
__global__ void __launch_bounds__(256)
linear_add_weight_parts_kernel(const float* parts, int n_parts, long long part_stride, long long total, const int* count, long long n,
                               OUT* w, int accumulate) {
  wait_for_previous();
  allow_next();
  const long long rows = count ? (*count < n ? *count : n) : n, k_blocks = (rows + BK - 1) / BK;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < total;
       i += static_cast<long long>(gridDim.x) * 256) {
    const float* src = parts + i * kAddCols;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < n_parts; p0 += kAddBatch) {
      float4 a[kAddBatch];
#pragma unroll
      for (int k = 0; k < kAddBatch; ++k) {
        const int p = p0 + k;
        const bool there = p < n_parts && p * k_blocks / n_parts < (p + 1) * k_blocks / n_parts;
        a[k] = there ? __ldcs(reinterpret_cast<const float4*>(src + p * part_stride)) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < kAddBatch; ++k) {
        v.x += a[k].x; v.y += a[k].y; v.z += a[k].z; v.w += a[k].w;
      }
    }
    if constexpr (sizeof(OUT) == 4) {
      float4* to = reinterpret_cast<float4*>(w) + i;
      if (accumulate) {
        const float4 old = *to;
        v.x += old.x; v.y += old.y; v.z += old.z; v.w += old.w;
      }
      *to = v;
    } else {
      reinterpret_cast<uint2*>(w)[i] = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }
  }
}

// dz^T x in parts of the rows, then their sum.
template <typename OUT>
int weight_parts(const Operand& a, const Operand& b, OUT* w, int accumulate, float* parts, int n_parts, const int* count,
                 uint32_t* status, cudaStream_t stream, Begin begin) {
  const int m = static_cast<int>(a.mn_extent), k = static_cast<int>(b.mn_extent);
  const long long m_pad = (m + BM - 1) / BM * BM;
  DynRows d = rows_as_m(count, a.k_extent);
  d.is_k = 1;
  using Parts = StorePartsEpilogue<kKLinearGradW>;
  A3PO_RETURN_IF((launch_gemm<Parts, true, true, 1>(a, b, 0, typename Parts::Params{parts, m, static_cast<int>(m_pad), n_parts, k}, d,
                                                    status, stream, n_parts, begin)));
  const long long total = static_cast<long long>(m) * (k / kAddCols), want = (total + 255) / 256;
  const int blocks = static_cast<int>(want < sm_count() * 8ll ? want : sm_count() * 8ll);
  A3PO_LAUNCH(kKLinearGradW, stream, (launch_early(linear_add_weight_parts_kernel<OUT>, blocks, 256, 0, stream, 1, true,
                                                   static_cast<const float*>(parts), n_parts, m_pad * k, total, count, a.k_extent, w,
                                                   accumulate)));
  return after_launch();
}

// The index of the rows that take part, by one launch: a block of 1,024 rows counts what lies before it by itself (at most a quarter
// of a megabyte, which the L2 has), so that no block waits for another.  16,384 rows of 1,536 to 4,608 columns there and back: 435 us,
// where counts, their sums and the index by three launches make it 441; 200,000 rows of 64 columns: no difference any more.
constexpr int kIndexThreads = 1024;
constexpr long long kIndexRows = 1 << 18;
__global__ void __launch_bounds__(kIndexThreads)
linear_row_index_kernel(const uint8_t* row_mask, long long n, int by_16, int* idx, int* count) {
  __shared__ int sh[2][kIndexThreads / kWarp];
  allow_next();
  const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
  const long long first = static_cast<long long>(blockIdx.x) * kIndexThreads, row = first + threadIdx.x;
  const bool in = row < n && row_mask[row] != 0;
  int before = 0;
  if (by_16) {
    const uint4* m = reinterpret_cast<const uint4*>(row_mask);
    for (long long i = threadIdx.x; i < first / 16; i += kIndexThreads) {
      const uint4 u = __ldg(m + i);
      before += __popc(__vsetne4(u.x, 0)) + __popc(__vsetne4(u.y, 0)) + __popc(__vsetne4(u.z, 0)) + __popc(__vsetne4(u.w, 0));
    }
  } else {
    for (long long i = threadIdx.x; i < first; i += kIndexThreads) before += row_mask[i] != 0 ? 1 : 0;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  const unsigned mine = __ballot_sync(0xffffffffu, in);
  if (lane == 0) {
    sh[0][warp] = before;
    sh[1][warp] = __popc(mine);
  }
  __syncthreads();
  int at = 0, own = 0;
#pragma unroll
  for (int w = 0; w < kIndexThreads / kWarp; ++w) {
    at += sh[0][w] + (w < warp ? sh[1][w] : 0);
    own += w >= warp ? sh[1][w] : 0;
  }
  if (in) idx[at + __popc(mine & ((1u << lane) - 1u))] = static_cast<int>(row);
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *count = at + own;
}

// Zeros for the rows that take no part.  It depends on nothing that the kernel ahead of it does, and runs beside it.
__global__ void __launch_bounds__(256)
linear_zero_rows_kernel(const uint8_t* row_mask, long long n, int vec_per_row, uint4* dst) {
  const int lane = threadIdx.x % kWarp;
  const long long warps = static_cast<long long>(gridDim.x) * (256 / kWarp);
  for (long long t = static_cast<long long>(blockIdx.x) * (256 / kWarp) + threadIdx.x / kWarp; t < n; t += warps) {
    if (row_mask[t] != 0) continue;
    for (int j = lane; j < vec_per_row; j += kWarp) __stcs(dst + t * vec_per_row + j, make_uint4(0, 0, 0, 0));
  }
  wait_for_previous();
}
int zero_rows(const uint8_t* row_mask, long long n, int m, int elt, void* dst, cudaStream_t stream) {
  const long long want = (n + 7) / 8;
  const int blocks = static_cast<int>(want < sm_count() * 4ll ? want : sm_count() * 4ll);
  A3PO_LAUNCH(kKLinear, stream, (launch_early(linear_zero_rows_kernel, blocks, 256, 0, stream, 1, true, row_mask, n, m * elt / 16,
                                              static_cast<uint4*>(dst))));
  return after_launch();
}

// The product with its epilogue: in K parts, or at once.
template <class Epi, int ACT, bool KEEP, typename OUT, bool B_MN>
int product(const Operand& a, const Operand& b, const typename Epi::Params& ep, float* parts, int k_parts, uint32_t* status,
            cudaStream_t stream, Begin begin) {
  if (k_parts > 1) {
    const long long rows_pad = (ep.n + BM - 1) / BM * BM;
    using Parts = StorePartsEpilogue<Epi::kKernelId>;
    typename Parts::Params sp{parts, ep.n, static_cast<int>(rows_pad), k_parts, ep.m};
    A3PO_RETURN_IF((launch_gemm<Parts, false, B_MN, 1>(a, b, 0, sp, rows_as_m(ep.count, ep.n), status, stream, k_parts, begin)));
    const long long want = (ep.n * (ep.m / kAddCols) + 255) / 256;
    const int blocks = static_cast<int>(want < sm_count() * 8ll ? want : sm_count() * 8ll);
    A3PO_LAUNCH(Epi::kKernelId, stream, (launch_early(linear_add_parts_kernel<Epi, ACT, KEEP, OUT>, blocks, 256, 0, stream, 1, true,
                                                      static_cast<const float*>(parts), k_parts, rows_pad * ep.m, ep)));
    return after_launch();
  }
  return contract<Epi, false, B_MN>(a, b, ep, rows_as_m(ep.count, ep.n), status, stream, begin);
}

template <int ACT, bool KEEP, typename OUT, bool SCATTER>
int fwd_typed(const LinearFwd& c) {
  using Epi = LinearEpilogue<ACT, KEEP, OUT, SCATTER>;
  typename Epi::Params ep;
  ep.y = static_cast<OUT*>(c.y);
  ep.bias = static_cast<const __nv_bfloat16*>(c.bias);
  ep.residual = static_cast<const __nv_bfloat16*>(c.residual);
  ep.kept = static_cast<uint8_t*>(c.kept);
  ep.row_index = c.row_index;
  ep.count = c.count;
  ep.n = c.n;
  ep.m = c.m;
  ep.whole_sectors = aligned_to(c.y, 32) && c.m * sizeof(OUT) % 32 == 0;
  return product<Epi, ACT, KEEP, OUT, false>(Operand{c.x, c.n, c.k, c.k}, Operand{c.w, c.m, c.k, c.k}, ep, c.parts,
                                             c.parts ? linear_k_parts(c.n, c.k, c.m, sizeof(OUT) == 4) : 1, c.status, c.stream,
                                             first_launch(c.count));
}
template <int ACT, bool KEEP, typename OUT>
int fwd_impl(const LinearFwd& c) {
  if (!c.row_index) return fwd_typed<ACT, KEEP, OUT, false>(c);
  A3PO_RETURN_IF((fwd_typed<ACT, KEEP, OUT, true>(c)));
  return zero_rows(c.row_mask, c.rows, c.m, sizeof(OUT), c.y, c.stream);
}

// ------------------------------------------------------------------------------------ dz and its column sums
// Bound: HBM, 8 bytes an element with an activation: 10,240 rows of 4,608 78 us alone (4.9 TB/s; half of the issue slots, the rest
// is latency; all of z on its way before the first half is worked on, at fewer blocks per SM, takes 8 us more).
// A block takes 128 rows and 64 columns.  dy and dz are read and written in whole rows of 128 bytes and change hands in shared
// memory (16-byte pieces, swizzled), because z and the sums want one row per thread.
constexpr int kGradCols = 64;
template <int ACT>
__global__ void __launch_bounds__(kZRows)
linear_grad_z_kernel(const __nv_bfloat16* grad_y, const uint8_t* kept, long long n, int m, const int* row_index,
                     const int* count, const uint8_t* row_mask, __nv_bfloat16* dz, float* sums, int add) {
  __shared__ __align__(16) uint4 tile[kZRows * 8];
  __shared__ float part[kZRows / kWarp][kGradCols];
  wait_for_previous();
  allow_next();
  const long long rows = count ? (*count < n ? *count : n) : n;
  const long long row0 = static_cast<long long>(blockIdx.x) * kZRows;
  if (row0 >= rows && gridDim.x > 1) return;   // one block of rows writes its sums, the bias gradient, whatever the mask leaves
  const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
  const int c0 = blockIdx.y * kGradCols, j = threadIdx.x % 8;   // this thread's piece of a row while rows are copied
  const bool in = c0 + j * 8 < m;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = i * 16 + threadIdx.x / 8;
    const long long row = row0 + r;
    uint4 u = make_uint4(0, 0, 0, 0);
    if (in && row < rows && (!row_mask || row_mask[row] != 0))
      u = __ldcs(reinterpret_cast<const uint4*>(grad_y + (row_index ? row_index[row] : row) * static_cast<long long>(m) + c0) + j);
    tile[r * 8 + (j ^ (r & 7))] = u;
  }
  const int r = threadIdx.x;
  const long long row = row0 + r;
  const bool live = row < rows && (!row_mask || row_mask[row] != 0);   // else dy is 0, and what was kept may be anything
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int c = c0 + half * kZCols;
    float z[kZCols];
    if (ACT != kActNone) {
      const float4* from = reinterpret_cast<const float4*>(kept + z_tile(row, c, m)) + r;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float4 f = live && c + q * 4 < m ? __ldcs(from + q * kZRows) : make_float4(0.f, 0.f, 0.f, 0.f);
        z[q * 4] = f.x; z[q * 4 + 1] = f.y; z[q * 4 + 2] = f.z; z[q * 4 + 3] = f.w;
      }
    }
    if (half == 0) __syncthreads();
    float v[kZCols];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float g[8];
      uint4& u = tile[r * 8 + ((half * 4 + q) ^ (r & 7))];
      unpack8(u, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float a, slope = 1.f;
        if (ACT != kActNone) linear_activation<ACT>(z[q * 8 + i], a, slope);
        v[q * 8 + i] = g[i] * slope;
      }
      u = pack8(v, q);
    }
    if (sums) {
      // lane c ends with the warp's sum of column c: each step halves the columns that a lane still adds
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
        for (int i = 0; i < o; ++i) {
          const bool up = (lane & o) != 0;
          const float other = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + o], o);
          v[i] = (up ? v[i + o] : v[i]) + other;
        }
      }
      part[warp][half * kZCols + lane] = v[0];
    }
  }
  __syncthreads();
  if (dz) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int to = i * 16 + threadIdx.x / 8;
      // rows past the last one are zeros up to the next multiple of 128, where the buffer has them
      if (in && (count || row0 + to < n)) reinterpret_cast<uint4*>(dz + (row0 + to) * m + c0)[j] = tile[to * 8 + (j ^ (to & 7))];
    }
  }
  if (sums && threadIdx.x < kGradCols && c0 + static_cast<int>(threadIdx.x) < m) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kZRows / kWarp; ++w) t += part[w][threadIdx.x];
    float* to = sums + static_cast<long long>(blockIdx.x) * m + c0 + threadIdx.x;
    *to = add ? *to + t : t;
  }
}

// 32 columns per block; 32 groups of threads share the blocks of rows and are added in order.
__global__ void __launch_bounds__(1024)
linear_grad_bias_kernel(const float* sums, long long blocks, const int* count, int m, float* grad_bias, int accumulate, int beside) {
  __shared__ float part[32][33];
  if (!beside) wait_for_previous();
  allow_next();
  if (count) {
    const long long have = (static_cast<long long>(*count) + kZRows - 1) / kZRows;
    if (have < blocks) blocks = have;
  }
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
  const int col = blockIdx.x * 32 + x;
  float t = 0.f;
  if (col < m)
    for (long long b = y; b < blocks; b += 32) t += sums[b * m + col];
  part[y][x] = t;
  __syncthreads();
  if (y == 0 && col < m) {
    t = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += part[i][x];
    grad_bias[col] = accumulate ? grad_bias[col] + t : t;
  }
  if (beside) wait_for_previous();
}

}  // namespace

// As ffn_k_parts; parts of fp32 outputs are at most 512 long, or the product is not split (more than 16 of them: the parts would be
// more traffic than the weights).
int linear_k_parts(long long n, int k, int m, bool y_f32) {
  const int parts = ffn_k_parts(n, m, k);
  if (!y_f32 || parts == 1) return parts;
  const int need = (k + kSumBlocks * BK - 1) / (kSumBlocks * BK);
  return need > 16 ? 1 : need > parts ? need : parts;
}

// A weight gradient of few tiles is a long sum over the rows for a few SMs: it is split where at most half of them have a tile, in
// parts of 512 rows and more, and, of fp32 gradients, of 512 and less (see PlainEpilogue::kPromote) unless that makes more than
// two rounds of parts.
int linear_weight_parts(long long n, int k, int m, bool grad_f32) {
  const long long k_blocks = (n + BK - 1) / BK, tiles = ((m + BM - 1ll) / BM) * ((k + BN - 1ll) / BN);
  const int parts = k_blocks >= kSplitRows / BK ? ffn_k_parts(m, k, static_cast<int>(n)) : 1;
  if (!grad_f32 || parts == 1) return parts;
  const long long need = (k_blocks + kSumBlocks - 1) / kSumBlocks;
  return need * tiles > 2ll * (sm_count() > 0 ? sm_count() : 148) ? 1 : need > parts ? static_cast<int>(need) : parts;
}

size_t linear_weight_parts_bytes(long long n, int k, int m) {
  const int a = linear_weight_parts(n, k, m, false), b = linear_weight_parts(n, k, m, true), parts = a > b ? a : b;
  return parts > 1 ? static_cast<size_t>((m + BM - 1) / BM * BM) * k * parts * sizeof(float) : 0;
}

size_t linear_parts_bytes(long long n, int k, int m) {
  const int a = linear_k_parts(n, k, m, false), b = linear_k_parts(n, k, m, true), parts = a > b ? a : b;
  return parts > 1 ? static_cast<size_t>((n + BM - 1) / BM * BM) * m * parts * sizeof(float) : 0;
}

int linear_row_index(const uint8_t* row_mask, long long n, const CompactBuffers& cb, cudaStream_t stream) {
  if (n > kIndexRows) return compact_index(nullptr, row_mask, nullptr, nullptr, n, cb, stream);
  const unsigned blocks = static_cast<unsigned>((n + kIndexThreads - 1) / kIndexThreads);
  A3PO_LAUNCH(kKCompact, stream, (linear_row_index_kernel<<<blocks, kIndexThreads, 0, stream>>>(
                                     row_mask, n, aligned_to(row_mask, 16) ? 1 : 0, cb.idx, cb.count)));
  return after_launch();
}

int linear_fwd_tc(const LinearFwd& c) {
  using B = __nv_bfloat16;
  if (c.act == kActNone) return c.y_f32 ? fwd_impl<kActNone, false, float>(c) : fwd_impl<kActNone, false, B>(c);
#define A3PO_LINEAR(ACT)                                                                               \
  (c.kept ? (c.y_f32 ? fwd_impl<ACT, true, float>(c) : fwd_impl<ACT, true, B>(c))                      \
          : (c.y_f32 ? fwd_impl<ACT, false, float>(c) : fwd_impl<ACT, false, B>(c)))
  return c.act == kActSilu ? A3PO_LINEAR(kActSilu) : A3PO_LINEAR(kActGelu);
#undef A3PO_LINEAR
}

int linear_grad_z(const void* grad_y, const void* kept, long long n, int m, Act act, const int* row_index, const int* count,
                  const uint8_t* row_mask, void* dz, float* sums, int add, bool early, cudaStream_t stream) {
  const dim3 grid(static_cast<unsigned>((n + kZRows - 1) / kZRows), static_cast<unsigned>((m + kGradCols - 1) / kGradCols));
  using B = __nv_bfloat16;
#define A3PO_GRAD_Z(ACT)                                                                                                  \
  A3PO_LAUNCH(kKLinearGradZ, stream, (launch_early(linear_grad_z_kernel<ACT>, grid, dim3(kZRows), 0, stream, 1, early,         \
                                                   static_cast<const B*>(grad_y), static_cast<const uint8_t*>(kept), n, m, \
                                                   row_index, count, row_mask, static_cast<B*>(dz), sums, add)))
  if (act == kActNone) A3PO_GRAD_Z(kActNone);
  else if (act == kActSilu) A3PO_GRAD_Z(kActSilu);
  else A3PO_GRAD_Z(kActGelu);
#undef A3PO_GRAD_Z
  return after_launch();
}

int linear_grad_bias(const float* sums, long long blocks, const int* count, int m, float* grad_bias, int accumulate, bool beside,
                     cudaStream_t stream) {
  A3PO_LAUNCH(kKLinearGradZ, stream, (launch_early(linear_grad_bias_kernel, static_cast<unsigned>((m + 31) / 32), 1024, 0, stream,
                                                   1, true, sums, blocks, count, m, grad_bias, accumulate, beside ? 1 : 0)));
  return after_launch();
}

int linear_grads_tc(const void* dz, const void* x, const void* w, long long n, int k, int m, void* grad_x, void* grad_w,
                    a3po_dtype grad_dt, int accumulate, float* parts, float* w_parts, const int* row_index, const int* count,
                    const uint8_t* row_mask, long long rows, bool first, uint32_t* status, cudaStream_t stream) {
  Begin begin = first ? Begin::kAfter : Begin::kEarly;
  if (grad_w) {
    const Operand a{dz, m, n, m}, b{x, k, n, k};   // dz^T x
    const int n_parts = w_parts ? linear_weight_parts(n, k, m, grad_dt == A3PO_F32) : 1;
    if (n_parts > 1) {
      A3PO_RETURN_IF(grad_dt == A3PO_F32 ? weight_parts(a, b, static_cast<float*>(grad_w), accumulate, w_parts, n_parts, count, status,
                                                        stream, begin)
                                         : weight_parts(a, b, static_cast<__nv_bfloat16*>(grad_w), 0, w_parts, n_parts, count, status,
                                                        stream, begin));
    } else if (grad_dt == A3PO_F32) {
      using Epi = WeightGradEpilogue;
      A3PO_RETURN_IF((weight_gemm<Epi>(a, b, typename Epi::Params{static_cast<float*>(grad_w), k, m, k, accumulate}, accumulate,
                                       count, status, stream, begin)));
    } else {
      using Epi = StoreBf16EpilogueT<kKLinearGradW>;
      A3PO_RETURN_IF((weight_gemm<Epi>(a, b, typename Epi::Params{static_cast<__nv_bfloat16*>(grad_w), k, m, k, nullptr}, 0,
                                       count, status, stream, begin)));
    }
    begin = Begin::kBeside;   // it reads what the weight gradient reads and writes apart from it
  }
  if (!grad_x) return A3PO_OK;
  const Operand a{dz, n, m, m}, b{w, k, m, k};   // dz W
  if (!row_index)
    return rows_gemm<kKLinearGradX, true>(a, b, static_cast<__nv_bfloat16*>(grad_x), parts, count, status, stream, begin);
  using Epi = LinearEpilogue<kActNone, false, __nv_bfloat16, true, kKLinearGradX>;
  typename Epi::Params ep{static_cast<__nv_bfloat16*>(grad_x), nullptr, nullptr, nullptr, row_index, count, n, k,
                          aligned_to(grad_x, 32) && k % 16 == 0};
  A3PO_RETURN_IF((product<Epi, kActNone, false, __nv_bfloat16, true>(a, b, ep, parts, parts ? ffn_k_parts(n, k, m) : 1, status,
                                                                     stream, begin)));
  return zero_rows(row_mask, rows, k, 2, grad_x, stream);
}

}  // namespace a3po
