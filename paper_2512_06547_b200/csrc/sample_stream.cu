// Sampling from rows without a filter: the logits are read once, front to back, by warps that know nothing of one another.
//
//   first kernel   a warp per segment of 1,024 logits: its largest m_s and S_s = sum exp((l - m_s) / t)
//   second kernel  a block per row: m = max m_s, W = sum S_s exp((m_s - m) / t); the segment in which the running sum passes
//                  u W is read again, and the token found in it
//
// Bound: the instructions of a weight (sample.cuh) for bf16 logits, HBM and those about alike for fp32.  2,048 rows of 151,936: bf16
// 225 us for the sums (2.8 TB/s; 17.3 instructions a logit, 65 % of the issue slots) and 18 for the pick; 1,024 rows in fp32 162 us
// (3.8 TB/s).  More blocks per SM, fewer registers or longer unrolled stretches change nothing.  One row is a chain of latencies:
// 12 us, 6 for each kernel.

#include "sample.cuh"

namespace a3po {
namespace {

constexpr int kSegment = 1024;   // elements, counted from the aligned start of a row
constexpr int kSumThreads = 256, kPickThreads = 128;
constexpr int kSumBlocks = 3;    // per SM, all at once: every warp has the same share of the segments

struct Segments {   // per row and segment, of rows that take part
  double* sum;
  float* max;
  int* count;       // logits above -inf
  int per_row;
};

// v[i] without an array that the compiler has to put into memory.
template <typename T, int N>
__device__ __forceinline__ Vec<T> select(const Vec<T> (&v)[N], int i) {
  Vec<T> r = v[0];
#pragma unroll
  for (int k = 1; k < N; ++k)
    if (k == i) r = v[k];
  return r;
}

template <typename T>
__global__ void __launch_bounds__(kSumThreads, kSumBlocks)
sample_sums_kernel(SampleArgs a, Segments out, long long items) {
  constexpr int VE = per_vec<T>(), kVecs = kSegment / VE / kWarp;
  __shared__ SharedTable<16> table;
  allow_next();
  // A warp takes neighbouring segments, so that what belongs to a row is looked up once per row.  bf16: the next segment is on its
  // way while one is worked on (fp32 segments take the registers that this needs).
  constexpr bool kAhead = sizeof(T) == 2;
  const int lane = threadIdx.x % kWarp;
  const long long warps = static_cast<long long>(gridDim.x) * (kSumThreads / kWarp);
  const long long me = static_cast<long long>(blockIdx.x) * (kSumThreads / kWarp) + threadIdx.x / kWarp;
  int item = static_cast<int>(items * me / warps);
  const int end = static_cast<int>(items * (me + 1) / warps);
  int row = item / out.per_row, seg = item - row * out.per_row;
  const T* l = nullptr;
  int head = 0;
  bool on = false;
  auto enter = [&]() {   // a row
    on = row < a.n && (!a.row_mask || a.row_mask[row] != 0);
    l = static_cast<const T*>(a.logits) + row * a.ld;
    head = head_of(l);
  };
  auto load = [&](Vec<T> (&v)[kVecs]) {
    const int first = seg * kSegment - head;
    if (first >= 0 && first + kSegment <= a.v) {   // the same for the warp
      const uint4* p = reinterpret_cast<const uint4*>(l + first) + lane;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const uint4 u = __ldcs(p + i * kWarp);
        v[i].w[0] = u.x; v[i].w[1] = u.y; v[i].w[2] = u.z; v[i].w[3] = u.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) v[i] = load_vec(l, first + (i * kWarp + lane) * VE, a.v);
    }
  };
  Weights<16> w;
  Vec<T> next[kAhead ? kVecs : 1];
  if (item < end) {
    enter();
    if constexpr (kAhead) {
      if (on) load(next);
    }
  }
  fill_table(table, threadIdx.x, kSumThreads);
  __syncthreads();
  bool fresh = true;
  while (item < end) {
    if (fresh) {
      bool greedy;
      if (on) w.set_temperature(a.temp(row, greedy), table);
    }
    const int here = item;
    const bool work = on;
    Vec<T> v[kVecs];
    if constexpr (kAhead) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) v[i] = next[i];
    } else {
      if (work) load(v);
    }
    ++item;
    fresh = ++seg == out.per_row;
    if (fresh) {
      seg = 0;
      ++row;
      enter();
    }
    if constexpr (kAhead) {
      if (item < end && on) load(next);
    }
    if (!work) continue;
    float m, least;
    extremes(v, m, least);
    m = warp_max_any(m);
    if (!(m > -INFINITY)) m = -INFINITY;
    double sum = 0.0;
    int count = 0;
    if (m > -INFINITY) {
      w.set_max(m);
      // no infinity, NaN or end of a row among the warp's logits, and none that is negligible: nearly always
      if (__all_sync(0xffffffffu, least - m >= w.floor && least > -INFINITY)) {
        WeightSum s;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
          for (int e = 0; e < VE; e += 2) w.template add<exact_diff<T>()>(v[i].pair(e), s);
        sum = s.value();
        count = kSegment;
      } else {
#pragma unroll 1
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float x = select(v, i).at(e);
            sum += w.template operator()<exact_diff<T>()>(x);
            count += x > -INFINITY ? 1 : 0;
          }
        count = __reduce_add_sync(0xffffffffu, count);
      }
      sum = warp_sum(sum);
    }
    if (lane == 0 && a.n_kept) out.count[here] = count;
    if (lane == 0) {
      out.sum[here] = sum;
      out.max[here] = m;
    }
  }
}

// Inclusive sum over the block in thread order; `before`: that of the threads below.  (Each is a tree of its own, so a
// thread that adds nothing may end a rounding away from its neighbour: only threads that add something are asked for.)
__device__ __forceinline__ double block_scan(double x, double* sh, double& before, double& total) {
  const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
  double inc = x;
#pragma unroll
  for (int o = 1; o < kWarp; o <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == kWarp - 1) sh[warp] = inc;
  __syncthreads();
  double base = 0.0;
  total = 0.0;
#pragma unroll
  for (int i = 0; i < kPickThreads / kWarp; ++i) {
    if (i == warp) base = total;
    total += sh[i];
  }
  double prev = __shfl_up_sync(0xffffffffu, inc, 1);
  before = lane ? base + prev : base;
  return lane == kWarp - 1 ? base + sh[warp] : base + inc;
}

template <typename T>
__global__ void __launch_bounds__(kPickThreads)
sample_pick_kernel(SampleArgs a, Segments in) {
  constexpr int VE = per_vec<T>();
  __shared__ SharedTable<1> table;
  __shared__ double sh_scan[kPickThreads / kWarp], sh_target;
  __shared__ float sh_max[kPickThreads / kWarp];
  __shared__ int sh_seg, sh_first, sh_last, sh_count, sh_best[kPickThreads / kWarp];
  const int row = blockIdx.x, lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
  if (a.row_mask && a.row_mask[row] == 0) {
    if (threadIdx.x == 0) a.put(row, -1, 0.0, 0.0, 0);
    wait_for_previous();   // what follows in the stream waits for this kernel alone, and may write what the one before it reads
    return;
  }
  fill_table(table, threadIdx.x, kPickThreads);
  if (threadIdx.x == 0) {
    sh_seg = sh_first = INT_MAX;
    sh_last = -1;
    sh_count = 0;
  }
  bool greedy;
  const float t = a.temp(row, greedy);
  const double inv_t = 1.0 / static_cast<double>(t);
  wait_for_previous();
  const double* sums = in.sum + static_cast<long long>(row) * in.per_row;
  const float* maxes = in.max + static_cast<long long>(row) * in.per_row;
  const int* counts = in.count + static_cast<long long>(row) * in.per_row;
  // a thread takes `per` neighbouring segments
  const int per = (in.per_row + kPickThreads - 1) / kPickThreads;
  const int s0 = min(static_cast<int>(threadIdx.x) * per, in.per_row), s1 = min(s0 + per, in.per_row);
  float m = -INFINITY;
  int count = 0;
  for (int s = s0; s < s1; ++s) {
    m = fmaxf(m, maxes[s]);
    if (a.n_kept) count += counts[s];
  }
  m = warp_max(m);
  if (lane == 0) sh_max[warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPickThreads / kWarp; ++i) m = fmaxf(m, sh_max[i]);
  if (!(m > -INFINITY)) {   // nothing to sample; the same for all threads
    if (threadIdx.x == 0) a.put(row, -1, 0.0, 0.0, 0);
    return;
  }
  if (a.n_kept) {
    count = __reduce_add_sync(0xffffffffu, count);
    if (lane == 0) atomicAdd(&sh_count, count);   // whole numbers: in any order
  }
  // what a segment's sum counts for in the row's
  auto factor = [&](float seg_max) {
    return seg_max == m ? 1.0 : exp((static_cast<double>(seg_max) - static_cast<double>(m)) * inv_t);
  };
  double mine = 0.0;
  for (int s = s0; s < s1; ++s)
    if (maxes[s] > -INFINITY) mine += sums[s] * factor(maxes[s]);
  double before, total;
  const double upto = block_scan(mine, sh_scan, before, total);
  const double target = static_cast<double>(fmaxf(a.u[row], 0.f)) * total;   // NaN and what is below 0 count as 0
  if (mine > 0.0) {
    if (target < upto) atomicMin(&sh_first, static_cast<int>(threadIdx.x));
    atomicMax(&sh_last, static_cast<int>(threadIdx.x));
  }
  __syncthreads();
  // the thread whose share the target falls into; past the end (u >= 1): the last that has any
  const bool here = static_cast<int>(threadIdx.x) == (sh_first < kPickThreads ? sh_first : sh_last);
  if (greedy) {
    for (int s = s0; s < s1; ++s)
      if (maxes[s] == m) {
        atomicMin(&sh_seg, s);
        break;
      }
  } else if (here) {
    double run = before, at = before;
    int seg = -1;
    for (int s = s0; s < s1; ++s) {
      if (!(maxes[s] > -INFINITY)) continue;
      const double x = sums[s] * factor(maxes[s]);
      if (!(x > 0.0)) continue;
      seg = s;
      at = run;
      run += x;
      if (target < run) break;
    }
    sh_seg = seg;
    sh_target = (target - at) / factor(maxes[seg]);
  }
  __syncthreads();
  // the segment again, in index order, 8 neighbours per thread
  const int seg = min(sh_seg, in.per_row - 1);
  const T* l = static_cast<const T*>(a.logits) + row * a.ld;
  constexpr int kEach = kSegment / kPickThreads;
  const int first = seg * kSegment - head_of(l) + static_cast<int>(threadIdx.x) * kEach;
  Weights<1> w;
  w.set_temperature(t, table);
  w.set_max(maxes[seg]);
  float x[kEach];
#pragma unroll
  for (int i = 0; i < kEach / VE; ++i) {
    const Vec<T> v = load_vec(l, first + i * VE, a.v);
#pragma unroll
    for (int e = 0; e < VE; ++e) x[i * VE + e] = v.at(e);
  }
  double y[kEach], sum = 0.0, all;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    y[e] = greedy ? (x[e] == m ? 1.0 : 0.0) : w.template operator()<exact_diff<T>()>(x[e]);
    sum += y[e];
  }
  double run;
  block_scan(sum, sh_scan, run, all);
  const double want = greedy ? 0.0 : sh_target;
  // the first that passes the target; rounding may leave it past the segment's sum: then the last that has a weight
  int pick = INT_MAX;
  float picked = 0.f;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    run += y[e];
    const int place = static_cast<int>(threadIdx.x) * kEach + e;
    const int me = run > want ? place : 2 * kSegment - place;
    if (y[e] > 0.0 && me < pick) {
      pick = me;
      picked = x[e];
    }
  }
  const int best = __reduce_min_sync(0xffffffffu, pick);
  if (lane == 0) sh_best[warp] = best;
  __syncthreads();
  int chosen = INT_MAX;
#pragma unroll
  for (int i = 0; i < kPickThreads / kWarp; ++i) chosen = min(chosen, sh_best[i]);
  if (pick == chosen && pick < INT_MAX) {   // one thread: places differ
    const int place = pick < kSegment ? pick : 2 * kSegment - pick;
    const double z = picked == m ? 0.0 : (static_cast<double>(picked) - static_cast<double>(m)) * inv_t;
    const double lp = z - log(total);
    a.put(row, first - static_cast<int>(threadIdx.x) * kEach + place, lp, greedy ? 0.0 : lp, greedy ? 1 : sh_count);
  }
}

template <typename T>
int stream_impl(const SampleArgs& a, const Segments& seg, cudaStream_t stream) {
  const int items = a.n * seg.per_row;
  constexpr int kWarps = kSumThreads / kWarp;
  // few segments go to as many SMs as there are
  const int want = items < sm_count() * kWarps ? (items < sm_count() ? items : sm_count()) : (items + kWarps - 1) / kWarps;
  const int most = sm_count() * kSumBlocks;
  A3PO_LAUNCH(kKSample, stream, (sample_sums_kernel<T><<<want < most ? want : most, kSumThreads, 0, stream>>>(a, seg, static_cast<long long>(items))));
  A3PO_RETURN_IF(after_launch());
  A3PO_LAUNCH(kKSample, stream, (launch_early(sample_pick_kernel<T>, a.n, kPickThreads, 0, stream, 1, true, a, seg)));
  return after_launch();
}

// A row that starts inside 16 bytes needs up to 7 places before its first element.
long long segments_per_row(int v) { return (static_cast<long long>(v) + 7 + kSegment - 1) / kSegment; }

}  // namespace

size_t sample_stream_bytes(long long n, int v) {
  const size_t items = static_cast<size_t>(n) * static_cast<size_t>(segments_per_row(v));
  return round_up(items * sizeof(double), 256) + round_up(items * sizeof(float), 256) + round_up(items * sizeof(int), 256);
}

int sample_stream(const void* args, a3po_dtype dt, void* ws, cudaStream_t stream) {
  const SampleArgs& a = *static_cast<const SampleArgs*>(args);
  const size_t items = static_cast<size_t>(a.n) * static_cast<size_t>(segments_per_row(a.v));
  if (items > static_cast<size_t>(INT_MAX) / 2) return A3PO_ERR_UNSUPPORTED;
  Arena ar(ws, sample_stream_bytes(a.n, a.v));
  Segments seg;
  seg.sum = ar.take<double>(items);
  seg.max = ar.take<float>(items);
  seg.count = ar.take<int>(items);
  seg.per_row = static_cast<int>(segments_per_row(a.v));
  return dt == A3PO_F32 ? stream_impl<float>(a, seg, stream) : stream_impl<__nv_bfloat16>(a, seg, stream);
}

}  // namespace a3po
