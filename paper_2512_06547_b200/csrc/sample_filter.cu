// Sampling from rows with filters (top-k, top-p, min-p).  A row is spread over the shared memory of a cluster of up to
// eight blocks, so that HBM is read once and all that follows runs on the copy:
//
//   largest logit and sum of all weights: warps of neighbouring logits by themselves, then blocks, then the cluster
//   how many logits lie at which distance from the largest, in 2,048 steps, added up in the first block.  The counts bound what
//     top-k or top-p can keep: the first step that has, with all above it, k tokens, or the share p of the mass even if every
//     token of a step has the least weight of the step (min-p's bound is known beforehand)
//     The lanes' largest logits, a thousandth of all, are counted first; they bound peaked rows and small k as well
//   few candidates (up to 2,048): the first block gets them in index order and finishes alone
//   more: the exact mass of the steps in which top-p's border may lie, the tokens of the one step that holds the border, which the
//     first block puts in order, and another pass over those between
//   rows whose borders the steps do not bound (more tokens on one step than the block holds, a border far from the largest
//     logit): the border's key (the logit's bits, ordered) by histograms of the key's leading bits, 11 at a time
//
// Masses that are compared are whole numbers of 2^-43, so that they do not depend on the order of atomics, and all other sums are
// taken in a fixed order: results are bit-identical from run to run.
// Bound: latency.  A row is a chain of passes of one to four microseconds and four to twelve cluster barriers of half a one; for many
// rows the instructions of the passes (40 to 78 a logit).  64 rows of 151,936 bf16: top-k 44 us, min-p 37, all three 51, settings that
// differ by row 74, flat rows under top-p alone (tens of thousands of candidates, every pass of the list above) 76; 1,024 rows
// 415 to 655 us; 37 rows of 32,003 in fp32, all three, 30 to 34.
// Sums by segment for all rows first (sample_stream.cu), a block per row for those whose candidates the segments bound, and
// this kernel for the rest only was measured: 1,024 rows 440 -> 340 us, 64 rows 44 -> 78; not kept.

#include "sample.cuh"
#include "sm100_ptx.cuh"

namespace a3po {
namespace {

constexpr int kMaxCluster = 8;
constexpr int kMaxSlice = 196608;        // bytes of a row in one block
constexpr int kNarrowRow = 1024;            // logits of a row that goes to a small block,
constexpr long long kNarrowBytes = 16384;   // and its bytes where there are more rows than large blocks that run at once
constexpr double kFixed = 8796093022208.0;   // 2^43: a weight as a whole number

using u32 = uint32_t;
using u64 = unsigned long long;

__device__ __forceinline__ u32 key_of(float l) {
  const u32 b = __float_as_uint(l);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(u32 k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
// Keys as wide as the logits: a bf16 key is the upper half of the fp32 one.
template <typename T> constexpr int key_drop() { return sizeof(T) == 2 ? 16 : 0; }
template <typename T> __device__ __forceinline__ u32 tkey(float l) { return key_of(l) >> key_drop<T>(); }
template <typename T> __device__ __forceinline__ float of_tkey(u32 k) {
  const float l = of_key(k << key_drop<T>());
  return sizeof(T) == 2 ? __uint_as_float(__float_as_uint(l) & 0xffff0000u) : l;
}

__device__ __forceinline__ u64 fixed_of(double w) {   // rounded to the nearest multiple of 2^-43; 0 <= w <= 1
  constexpr double kMagic = 6755399441055744.0;       // 1.5 2^52
  return static_cast<u64>(__double_as_longlong(fma(w, kFixed, kMagic)) - __double_as_longlong(kMagic));
}

__device__ __forceinline__ void store_remote(u64* here, u32 rank, u64 v) {
  const u32 at = ptx::map_to_cta(static_cast<u32>(__cvta_generic_to_shared(here)), rank);
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory");
}
__device__ __forceinline__ u32 load_remote(const u32* here, u32 rank) {
  const u32 at = ptx::map_to_cta(static_cast<u32>(__cvta_generic_to_shared(here)), rank);
  u32 v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

__device__ __forceinline__ u64 load_remote(const u64* here, u32 rank) {
  const u32 at = ptx::map_to_cta(static_cast<u32>(__cvta_generic_to_shared(here)), rank);
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint4 load_remote4(const u32* here, u32 rank) {
  const u32 at = ptx::map_to_cta(static_cast<u32>(__cvta_generic_to_shared(here)), rank);
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ u32 take_from_remote(u32* here, u32 rank, u32 v) {   // the value before
  const u32 at = ptx::map_to_cta(static_cast<u32>(__cvta_generic_to_shared(here)), rank);
  u32 old;
  asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(at), "r"(v) : "memory");
  return old;
}

// Sum of a word over the cluster, all loads on their way at once.
__device__ __forceinline__ void add_remote(const u32* here, int cluster, u64& sum) {
  u32 v[kMaxCluster];
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) v[r] = r < cluster ? load_remote(here, r) : 0;
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) sum += v[r];
}

__device__ __forceinline__ u64 warp_sum64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

namespace wide {
constexpr int kThreads = 512, kBlocks = 2, kBinBits = 11;
constexpr float kCountSteps = 32.f, kMassSteps = 128.f;
constexpr size_t kLongestSlice = kMaxSlice;
#include "sample_rows.cuh"
}  // namespace wide

namespace narrow {
constexpr int kThreads = 128, kBlocks = 7, kBinBits = 9;
constexpr float kCountSteps = 16.f, kMassSteps = 32.f;
constexpr size_t kLongestSlice = kNarrowBytes;
#include "sample_rows.cuh"
}  // namespace narrow

// Short rows go to small blocks, of which seven share an SM: a row is a chain of latencies whatever a block's size, and small blocks
// have shorter ones up to about 1,024 logits.  All three filters, 129, 1,000 and 4,096 logits in fp32: 64 rows 11, 13 and 48 us by
// small blocks, 15, 17 and 25 by large ones; 2,048 rows, which are several rounds of large blocks, 41, 34 and 101 against 109, 98
// and 137 (1,000 rows of 8,192: 96 and 85).

template <typename T>
int filter_impl(const SampleArgs& a, cudaStream_t stream) {
  const long long bytes = static_cast<long long>(a.v) * static_cast<int>(sizeof(T));
  const bool filters = a.top_k || a.top_p || a.min_p;
  if (!filters || a.v <= kNarrowRow || (bytes <= kNarrowBytes && a.n > 2ll * sm_count())) return narrow::launch<T>(a, 1, stream);
  // Blocks per row: two share an SM, each with at most 76 KB of logits (eight blocks of up to kMaxSlice where that does not do).
  // More than that, up to eight of at least 8 KB, while all rows still run at once.
  int cluster = 1;
  while (cluster < kMaxCluster && bytes > 77824ll * cluster) cluster *= 2;
  while (cluster < kMaxCluster && bytes > 16384ll * cluster && 2ll * cluster * a.n <= 2ll * sm_count()) cluster *= 2;
  return wide::launch<T>(a, cluster, stream);
}

}  // namespace

// A launch less than sample_stream.cu's two.  128 rows of 512 logits: 6.7 us and 9.7, of 2,048 7.1 and 8.7, of 4,096 8.8 and 8.6;
// 600 rows of 512 8 and 10, 2,048 rows 16 to 18 and 15 to 17.
bool sample_in_one(long long n, int v) { return v <= 2048 && n <= 4ll * sm_count(); }

long long sample_filter_max_v(a3po_dtype dt) { return static_cast<long long>(kMaxCluster) * kMaxSlice / (dt == A3PO_F32 ? 4 : 2); }

int sample_filter(const void* args, a3po_dtype dt, cudaStream_t stream) {
  const SampleArgs& a = *static_cast<const SampleArgs*>(args);
  if (a.n > INT_MAX / kMaxCluster) return A3PO_ERR_UNSUPPORTED;
  return dt == A3PO_F32 ? filter_impl<float>(a, stream) : filter_impl<__nv_bfloat16>(a, stream);
}

}  // namespace a3po
