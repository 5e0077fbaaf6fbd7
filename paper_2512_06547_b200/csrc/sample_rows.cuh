// A row of logits in the shared memory of a cluster of blocks, and what sample_filter.cu says of it (below, "2,048" steps and
// candidates are those of the large blocks).  Included once for each size of
// block, inside a namespace that defines
//   kThreads                  a block's threads;   kBlocks   blocks that share an SM
//   kBinBits                  a histogram has 2^kBinBits = 4 kThreads bins, and one block finishes that many candidates alone
//   kCountSteps, kMassSteps   see Steps
//   kLongestSlice             bytes of a row that one block holds at most
constexpr int kWarps = kThreads / kWarp, kBins = 1 << kBinBits;
constexpr int kSlots = 20 + 6 * ((32 + kBinBits - 1) / kBinBits);   // more than a row by every way there is uses
constexpr int kList = kBins;             // candidates that one block finishes alone
static_assert(kList * sizeof(u64) == 2 * kBins * sizeof(u32), "the list takes the histograms' place");

struct Shared {
  SharedTable<16> table;
  u64 slot[kSlots][kMaxCluster];   // what the blocks of the cluster tell one another, each slot once
  u64 part[2][kWarps];
  double stretch[kWarps];          // sums of the warps' weights, relative to the largest of each
  float stretch_max[kWarps];
  double total;                    // of the row, relative to its largest logit
  int warp_count[kWarps];
  union {
    struct __align__(16) {
      u32 lo[kBins], hi[kBins];    // histograms
    };
    u64 list[kList];               // the first block's: candidates (ordered bits, index)
  };
};

constexpr size_t kSharedBytes = (sizeof(Shared) + 15) / 16 * 16;   // ahead of the slice
// Bytes behind it: the slice and the places before and behind it; the first block's sums by step, and one step's candidates, take its
// place.
constexpr size_t room_of(size_t slice) {
  const size_t alone = (kBins + kList) * sizeof(u64), room = (slice + 47) / 16 * 16;
  return room < alone ? alone : room;
}
constexpr size_t kMostShared = kSharedBytes + room_of(kLongestSlice);
static_assert(kMostShared <= 227 * 1024, "the longest slice");

template <typename T>
struct Row {
  Shared& sh;
  const uint4* data;       // this block's slice, 16-byte pieces; places outside the slice hold -inf
  int vecs;
  int base;                // index in the row of place 0
  int cluster, rank;
  int flip, slot;
  int lane, warp, v0, v1;  // this warp's pieces

  __device__ __forceinline__ Row(Shared& s) : sh(s) {}

  // ---- the cluster
  __device__ __forceinline__ u64* tell(u64 v) {   // v: the same in all threads.  Seen by the others after sync()
    u64* s = sh.slot[slot++];
    if (threadIdx.x < static_cast<unsigned>(cluster)) store_remote(s + rank, threadIdx.x, v);
    return s;
  }
  // The next slot, for a thread that tells everyone by itself (say); read at [0].
  __device__ __forceinline__ u64* next_slot() { return sh.slot[slot++]; }
  __device__ __forceinline__ void say(u64* s, u64 v) const {
    for (int r = 0; r < cluster; ++r) store_remote(s, r, v);
  }
  __device__ __forceinline__ void sync() { ptx::cluster_sync_all(); }
  // Sum over the block's threads, in warp order, in all threads.
  __device__ __forceinline__ u64 block_sum(u64 v) {
    v = warp_sum64(v);
    u64* p = sh.part[flip ^= 1];
    if (lane == 0) p[warp] = v;
    __syncthreads();
    u64 t = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) t += p[i];
    return t;
  }
  __device__ __forceinline__ double block_sum(double v) {
    v = warp_sum(v);
    u64* p = sh.part[flip ^= 1];
    if (lane == 0) p[warp] = static_cast<u64>(__double_as_longlong(v));
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) t += __longlong_as_double(static_cast<long long>(p[i]));
    return t;
  }
  __device__ __forceinline__ u64 cluster_sum(u64 v) {
    const u64* s = tell(block_sum(v));
    sync();
    u64 t = 0;
    for (int r = 0; r < cluster; ++r) t += s[r];
    return t;
  }
  __device__ __forceinline__ double cluster_sum(double v) {
    const u64* s = tell(static_cast<u64>(__double_as_longlong(block_sum(v))));
    sync();
    double t = 0.0;
    for (int r = 0; r < cluster; ++r) t += __longlong_as_double(static_cast<long long>(s[r]));
    return t;
  }
  __device__ __forceinline__ u64 block_min(u64 v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = min(v, __shfl_xor_sync(0xffffffffu, v, o));
    u64* p = sh.part[flip ^= 1];
    if (lane == 0) p[warp] = v;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWarps; ++i) v = min(v, p[i]);
    return v;
  }
  __device__ __forceinline__ u64 cluster_min(u64 v) {
    v = block_min(v);
    const u64* s = tell(v);
    sync();
    for (int r = 0; r < cluster; ++r) v = min(v, s[r]);
    return v;
  }
  // Sum over the threads below this one; total: over all.
  template <typename S>
  __device__ __forceinline__ S scan(S x, S& total) {
    S inc = x;
#pragma unroll
    for (int o = 1; o < kWarp; o <<= 1) {
      const S y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    static_assert(sizeof(S) <= sizeof(u64), "");
    S* p = reinterpret_cast<S*>(sh.part[flip ^= 1]);
    if (lane == kWarp - 1) p[warp] = inc;
    __syncthreads();
    S before = __shfl_up_sync(0xffffffffu, inc, 1);
    if (lane == 0) before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) before += p[i];
      total += p[i];
    }
    return before;
  }

  // ---- the slice.  f(l, index) for the logits of this thread
  __device__ __forceinline__ Vec<T> piece(int j) const {
    const uint4 u = data[j];
    Vec<T> v;
    v.w[0] = u.x; v.w[1] = u.y; v.w[2] = u.z; v.w[3] = u.w;
    return v;
  }
  // Sum of the weights of the logits that `in` takes: pairs, of which one that is not taken (or far below the largest) counts as
  // its 2^-100th; a sum below 2^-60 is taken again one by one.  count: how many of this thread's it takes.
  template <class W, class F>
  __device__ __forceinline__ double weigh(const W& w, F in, int& count) const {
    double s = 0.0;
    count = 0;
    if (w.floor > -1e37f && fabsf(w.max) < 1e6f * -w.floor) {   // the limit below is a number well under the largest
      const float least = w.max + w.floor;
      WeightSum even, odd;
      for (int j = v0 + lane; j < v1; j += kWarp) {
        const Vec<T> v = piece(j);
#pragma unroll
        for (int e = 0; e < per_vec<T>(); e += 2) {
          const int i = base + j * per_vec<T>() + e;
          const float x = v.at(e), y = v.at(e + 1);
          const bool in_x = in(x, i), in_y = in(y, i + 1);
          count += (in_x ? 1 : 0) + (in_y ? 1 : 0);
          w.template add<exact_diff<T>()>(f2(in_x ? fmaxf(x, least) : least, in_y ? fmaxf(y, least) : least), e % 4 ? odd : even);
        }
      }
      s = warp_sum(even.value() + odd.value());
      if (s >= 0x1p-60) return s;
      s = 0.0;
      count = 0;
    }
    each([&](float x, int i) {
      if (!in(x, i)) return;
      s += w.template operator()<exact_diff<T>()>(x);
      ++count;
    });
    return warp_sum(s);
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    for (int j = v0 + lane; j < v1; j += kWarp) {
      const Vec<T> v = piece(j);
#pragma unroll
      for (int e = 0; e < per_vec<T>(); ++e) f(v.at(e), base + j * per_vec<T>() + e);
    }
  }

  // The same for those that `in` takes, where they are few: a lane marks its own of 32 first, so that f runs as often as the lane
  // with the most of them asks, not once for each place that any lane asks for.
  template <class P, class F>
  __device__ __forceinline__ void each_of(P in, F f) const {
    constexpr int VE = per_vec<T>(), kPieces = kWarp / VE;
    const T* flat = reinterpret_cast<const T*>(data);
    for (int j0 = v0 + lane; j0 < v1; j0 += kWarp * kPieces) {
      u32 marks = 0;
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        const int j = j0 + p * kWarp;
        if (j >= v1) continue;
        const Vec<T> v = piece(j);
#pragma unroll
        for (int e = 0; e < VE; ++e) marks |= in(v.at(e)) ? 1u << (p * VE + e) : 0u;
      }
      while (marks) {
        const int bit = __ffs(marks) - 1;
        marks &= marks - 1;
        const int at = (j0 + bit / VE * kWarp) * VE + bit % VE;
        f(to_float(flat[at]), base + at);
      }
    }
  }

  // ---- the border of the `need` largest (each counting for amount(l)): the key at which the sum over larger keys and its own
  // reaches `need`, among keys lo .. hi; above: the sum over larger keys.
  template <bool MASS, class F>
  __device__ __forceinline__ u32 border(u32 lo, u32 hi, u64 need, F amount, u64& above) {
    above = 0;
    for (;;) {
      const u32 range = hi - lo;
      const int bits = 32 - __clz(range);
      const int shift = bits > kBinBits ? bits - kBinBits : 0;
      for (int i = threadIdx.x; i < kBins; i += kThreads) {
        sh.lo[i] = 0;
        if (MASS) sh.hi[i] = 0;
      }
      __syncthreads();
      each([&](float l, int) {
        const u32 k = tkey<T>(l);
        if (k < lo || k > hi) return;
        const u32 bin = (k - lo) >> shift;
        if (!MASS) {
          atomicAdd(&sh.lo[bin], 1u);
        } else {   // 64 bits from two words: the carry goes with the thread that saw it
          const u64 x = amount(l);
          const u32 xl = static_cast<u32>(x), old = atomicAdd(&sh.lo[bin], xl);
          const u32 xh = static_cast<u32>(x >> 32) + (old + xl < old ? 1u : 0u);
          if (xh) atomicAdd(&sh.hi[bin], xh);
        }
      });
      sync();
      // Rank 0 adds up the highest bins of the cluster, the last rank the lowest; a thread takes neighbouring ones, from
      // the top down.
      const int mine = kBins / cluster, per = (mine + kThreads - 1) / kThreads;
      const int top = kBins - rank * mine;   // bins top - 1, top - 2, ...
      u64 got[kBins / kThreads], sum = 0;
#pragma unroll
      for (int i = 0; i < kBins / kThreads; ++i) {
        got[i] = 0;
        const int at = static_cast<int>(threadIdx.x) * per + i;
        if (i < per && at < mine) {
          u64 words_hi = 0;
          add_remote(&sh.lo[top - 1 - at], cluster, got[i]);
          if (MASS) add_remote(&sh.hi[top - 1 - at], cluster, words_hi);
          got[i] += words_hi << 32;
          sum += got[i];
        }
      }
      u64 inc = sum;
#pragma unroll
      for (int o = 1; o < kWarp; o <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      u64* p = sh.part[flip ^= 1];
      if (lane == kWarp - 1) p[warp] = inc;
      __syncthreads();
      u64 total = 0;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        if (i < warp) inc += p[i];
        total += p[i];
      }
      const u64* totals = tell(total);
      u64* said_bin = sh.slot[slot++];
      u64* said_above = sh.slot[slot++];
      sync();
      u64 before = 0;
      int owner = cluster - 1;   // where rounding leaves `need` past the sum of all: the lowest bin that holds anything
      for (int r = 0; r < cluster; ++r) {
        if (before + totals[r] >= need) {
          owner = r;
          break;
        }
        if (r < cluster - 1) before += totals[r];
      }
      if (owner == rank) {
        u64 run = before + inc - sum;   // over the bins above this thread's
        const bool last = threadIdx.x == kThreads - 1;
        if (run < need && (run + sum >= need || last)) {
          int bin = 0;
          u64 at = run;
          bool found = false;
#pragma unroll
          for (int i = 0; i < kBins / kThreads; ++i) {
            if (i < per && !found) {
              bin = top - 1 - (static_cast<int>(threadIdx.x) * per + i);
              at = run;
              run += got[i];
              found = run >= need;
            }
          }
          if (bin < 0) bin = 0;
          for (int r = 0; r < cluster; ++r) {
            store_remote(said_bin, r, static_cast<u64>(bin));
            store_remote(said_above, r, at);
          }
        }
      }
      sync();
      const u32 bin = static_cast<u32>(said_bin[0]);
      above += said_above[0];
      need -= min(need - 1, said_above[0]);
      lo += bin << shift;
      if (shift == 0) return min(lo, hi);
      hi = min(hi, lo + ((1u << shift) - 1u));
      if (lo >= hi) return hi;
    }
  }
};

// Index of this warp's nth logit that `in` takes, in index order (there are that many).
template <typename T, class F>
__device__ __forceinline__ int find_nth(const Row<T>& row, int nth, F in) {
  constexpr int VE = per_vec<T>();
  int run = 0, at = -1;
  for (int j0 = row.v0; j0 < row.v1 && run < nth; j0 += kWarp) {
    const int j = j0 + row.lane;
    u32 marks = 0;
    if (j < row.v1) {
      const Vec<T> v = row.piece(j);
#pragma unroll
      for (int e = 0; e < VE; ++e) marks |= in(v.at(e)) ? 1u << e : 0u;
    }
    int inc = __popc(marks);
#pragma unroll
    for (int o = 1; o < kWarp; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (row.lane >= o) inc += y;
    }
    int skip = nth - run - (inc - __popc(marks));   // of this lane's, the skip-th
    if (skip >= 1 && skip <= __popc(marks)) {
      while (--skip) marks &= marks - 1;
      at = row.base + j * VE + __ffs(marks) - 1;
    }
    run += __shfl_sync(0xffffffffu, inc, kWarp - 1);
  }
  return __reduce_max_sync(0xffffffffu, at);
}

// Place (in the slice) of the first logit among the pieces v0 .. v1 at which the sum of x(logit, index) passes `want`; where rounding
// keeps it below, of the last that counts for anything.  By all threads of the block, a piece each.
template <typename T, class F>
__device__ __forceinline__ int find_by_sum(Row<T>& row, int v0, int v1, double want, F x) {
  constexpr int VE = per_vec<T>();
  constexpr u64 kPast = 1ull << 40;
  u64 pick = ~0ull;
  double run = 0.0;
  for (int j0 = v0; j0 < v1; j0 += kThreads) {
    const int j = j0 + static_cast<int>(threadIdx.x);
    double got[VE], sum = 0.0, all;
    Vec<T> v;
    if (j < v1) v = row.piece(j);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      got[e] = j < v1 ? x(v.at(e), row.base + j * VE + e) : 0.0;
      sum += got[e];
    }
    double upto = run + row.scan(sum, all);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      upto += got[e];
      const u64 place = static_cast<u64>(j * VE + e);
      if (got[e] > 0.0) pick = min(pick, upto > want ? place : kPast - place);
    }
    pick = row.block_min(pick);
    if (pick < kPast / 2) break;
    run += all;
  }
  return static_cast<int>(pick < kPast / 2 ? pick : kPast - pick);
}

// The share that top-p asks for; 2^-48 less, so that one that is reached exactly is reached.
__device__ __forceinline__ u64 share_of(double all, float top_p) {
  const double share = static_cast<double>(fmaxf(top_p, 0.f)) * all * (1.0 - 0x1p-48);
  return share > 1.0 ? static_cast<u64>(ceil(share)) : 1;
}

// A token as a number: larger logits first, then lower indexes.
__device__ __forceinline__ u64 entry_of(float l, int index) { return static_cast<u64>(~key_of(l)) << 32 | static_cast<u32>(index); }
__device__ __forceinline__ float logit_of(u64 entry) { return of_key(~static_cast<u32>(entry >> 32)); }

// What one row asks for.
struct Ask {
  int top_k;
  float top_p, min_p;
  bool by_count, by_mass, by_min;
  double min_bound;   // the smallest logit that min-p keeps
};

// Steps of distance to the largest logit: 1 / kCountSteps of the temperature each, 1 / kMassSteps for top-p alone (whose bound is the
// sharper the finer they are; 99 % of the mass is out of its reach).
// Rounded to the nearest step by the last bit of a sum with 2^23, whose bits are then kZeroStep + the step; what is beyond 2^24
// steps, infinite or NaN has larger ones.
constexpr u32 kZeroStep = 0x4b000000u;
struct Steps {
  float max, scale;
  __device__ __forceinline__ u32 at(float l) const { return __float_as_uint(fmaf(__fsub_rn(max, l), scale, 8388608.f)) - kZeroStep; }
};

// Among m entries and what they count for: the last one, in rank order, that is kept, when the entries before them count `before`
// and all up to it have to count `need`; ~0: all of them do not.
template <class R>
__device__ __forceinline__ u64 border_among(R& row, const u64* entries, const u64* amounts, int m, u64 before, u64 need) {
  u64 border = ~0ull;
  for (int i = threadIdx.x; i < m; i += kThreads) {
    const u64 me = entries[i];
    u64 upto = before;
#pragma unroll 4
    for (int j = 0; j < m; ++j) upto += entries[j] <= me ? amounts[j] : 0;
    if (upto >= need) border = min(border, me);
  }
  return row.block_min(border);
}

// The first block with n candidates in index order in `list`; the rest of the cluster is done.
// scratch: two arrays of kList words besides.
template <typename T, class W>
__device__ __forceinline__ void finish_alone(Row<T>& row, const SampleArgs& a, int row_id, const W& w, const Steps& steps, float t,
                                             double total, const Ask& ask, const u64* list, int n, u64* bins, u64* among) {
  Shared& sh = row.sh;
  auto weight = [&](u64 entry) { return w.template operator()<exact_diff<T>()>(logit_of(entry)); };
  constexpr int kEach = kList / kThreads;
  double x[kEach], sum = 0.0, all;
  u32 kept = 0, all_kept;
  int s0;
  constexpr int kFew = kThreads < 192 ? kThreads : 192;
  if (n <= kFew) {
    // one candidate per thread, compared with all: its rank and the mass before it
    s0 = threadIdx.x;
    const bool in = s0 < n;
    const u64 me = in ? list[s0] : ~0ull;
    const double weigh = in ? weight(me) : 0.0;
    const u64 fixed = in ? fixed_of(weigh) : 0;
    ulonglong2* pair = reinterpret_cast<ulonglong2*>(among);
    if (in) pair[s0] = make_ulonglong2(me, fixed);
    __syncthreads();
    u32 rank = 0;
    u64 before = 0;
    if (row.warp * kWarp < n) {
      for (int j = 0; j < n; ++j) {
        const ulonglong2 other = pair[j];
        if (other.x < me) {
          ++rank;
          before += other.y;
        }
      }
    }
    bool on = in && (!ask.by_count || rank < static_cast<u32>(ask.top_k));
    if (ask.by_mass) {
      const double of = ask.by_count ? static_cast<double>(row.block_sum(on ? fixed : 0)) : total * kFixed;
      on = on && before < share_of(of, ask.top_p);
    }
    if (ask.by_min) on = on && (rank == 0 || (ask.min_p <= 1.f && static_cast<double>(logit_of(me)) >= ask.min_bound));
    kept = on ? 1 : 0;
    x[0] = on ? weigh : 0.0;
    sum = x[0];
#pragma unroll
    for (int i = 1; i < kEach; ++i) x[i] = 0.0;
  } else {
    s0 = static_cast<int>(threadIdx.x) * kEach;
    u64 last = ~0ull;   // the last entry, in rank order, that is kept
    if (ask.by_count || ask.by_mass) {
      // top-k's border, then, of the mass above it, top-p's: sums by step, the step that they pass `need` in, its entries
      constexpr int kMost = kBins / kThreads;
      u64 need = static_cast<u64>(ask.top_k);
      bool weigh = !ask.by_count;
      if (weigh) need = share_of(total * kFixed, ask.top_p);
      for (;;) {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
        if (threadIdx.x == 0) sh.warp_count[0] = 0;
        __syncthreads();
        u64 f[kEach], mass = 0;
        int bin[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          f[i] = 0;
          bin[i] = -1;
          if (s0 + i < n && list[s0 + i] <= last) {
            f[i] = weigh ? fixed_of(weight(list[s0 + i])) : 1;
            bin[i] = static_cast<int>(steps.at(logit_of(list[s0 + i])));
            atomicAdd(&bins[bin[i]], f[i]);   // whole numbers: in any order
          }
        }
        __syncthreads();
        u64 own[kMost], part = 0;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          own[i] = bins[static_cast<int>(threadIdx.x) * kMost + i];
          part += own[i];
        }
        u64 run = row.scan(part, mass);
        if (weigh && ask.by_count) need = share_of(static_cast<double>(mass), ask.top_p);
        u64 found = ~0ull, before = 0;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          if (run < need && run + own[i] >= need) {
            found = static_cast<u64>(static_cast<int>(threadIdx.x) * kMost + i);
            before = run;
          }
          run += own[i];
        }
        if (found != ~0ull) sh.slot[kSlots - 1][0] = before;   // one thread
        found = row.block_min(found);
        if (found != ~0ull) {   // else fewer than k tokens, or rounding: all of them
          // the step's entries and what they count for into one place (the sums by step have been read)
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            if (bin[i] == static_cast<int>(found)) {
              const int to = atomicAdd(&sh.warp_count[0], 1);   // in any order: what follows compares all with all
              among[to] = list[s0 + i];
              bins[to] = f[i];
            }
          }
          __syncthreads();
          last = min(last, border_among(row, among, bins, sh.warp_count[0], sh.slot[kSlots - 1][0], need));
        }
        if (weigh || !ask.by_mass) break;
        weigh = true;
      }
    }
    if (ask.by_min) {
      u64 top = ~0ull, low = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (s0 + i >= n) continue;
        const u64 entry = list[s0 + i];
        top = min(top, entry);
        if (static_cast<double>(logit_of(entry)) >= ask.min_bound) low = max(low, entry);
      }
      top = row.block_min(top);              // the first rank is kept whatever min-p is
      low = ~row.block_min(~low);
      last = min(last, ask.min_p > 1.f ? top : max(top, low));
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const bool in = s0 + i < n && list[s0 + i] <= last;
      x[i] = in ? weight(list[s0 + i]) : 0.0;
      sum += x[i];
      kept += in ? 1 : 0;
    }
  }
  // the weights of what is kept, in index order
  double run = row.scan(sum, all);
  row.scan(kept, all_kept);
  const double target = static_cast<double>(fmaxf(a.u[row_id], 0.f)) * all;   // NaN and what is below 0 count as 0
  // the first that passes the target; past the end the last that has a weight
  u64 pick = ~0ull;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    run += x[i];
    if (x[i] > 0.0) pick = min(pick, static_cast<u64>(run > target ? s0 + i : 2 * kList - (s0 + i)));
  }
  pick = row.block_min(pick);
  if (threadIdx.x == 0) {
    const u64 entry = list[pick < kList ? pick : 2 * kList - pick];
    const float l = logit_of(entry);
    const double z = l == w.max ? 0.0 : (static_cast<double>(l) - static_cast<double>(w.max)) / static_cast<double>(t);
    a.put(row_id, static_cast<int>(entry & 0xffffffffu), z - log(total), z - log(all), static_cast<int>(all_kept));
  }
}

enum class Way { kDone, kBorder, kKeys };   // sampled; the border is known; it is not

// How far the candidates reach, from counts by step (sh.lo of all blocks): the first step that has, with all above it, enough of
// them, and the first in which top-k's or top-p's border may lie; each with the count up to it (before it), ~0 where there is none.
struct Reach {
  u64 end, low;
};
template <typename T>
__device__ __forceinline__ Reach reach_of(Row<T>& row, const Ask& ask, double total, float per_t) {
  Shared& sh = row.sh;
  const bool mass_alone = ask.by_mass && !ask.by_count;
  u64* said = row.next_slot();
  u64* said_low = row.next_slot();
  row.sync();
  if (row.rank == 0) {
    constexpr int kMost = kBins / kThreads;
    static_assert(kMost == 4, "a thread's steps are one 16-byte load");
    const int first = static_cast<int>(threadIdx.x) * kMost;
    u32 got[kMost] = {}, count = 0, all_count;
    float least[kMost];   // weights at the far end of each step
    double mass = 0.0, all_mass;
    {
      uint4 v[kMaxCluster];
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) v[r] = r < row.cluster ? load_remote4(&sh.lo[first], r) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        got[0] += v[r].x; got[1] += v[r].y; got[2] += v[r].z; got[3] += v[r].w;
      }
    }
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      count += got[i];
      if (mass_alone) {
        least[i] = expf((static_cast<float>(first + i) + 0.5f) * (-1.f / per_t));
        mass += static_cast<double>(got[i]) * static_cast<double>(least[i]);
      }
    }
    u32 cum = row.scan(count, all_count);
    double cum_mass = mass_alone ? row.scan(mass, all_mass) : 0.0;
    const double share = static_cast<double>(fmaxf(ask.top_p, 0.f)) * total;
    const double enough = share * (1.0 + 1e-5);   // expf and the distances are not exact
    // with the weights at the near ends, which are this much larger, the mass is not enough either
    const double too_little = share * static_cast<double>(expf(-1.f / per_t)) * (1.0 - 1e-5);
    int min_bin = INT_MAX;   // the first step that lies below what min-p keeps
    if (ask.by_min && !ask.by_mass) {
      const float at = ask.min_p >= 1.f ? 0.f : -logf(ask.min_p) * per_t;
      if (at < static_cast<float>(kBins - 3)) min_bin = static_cast<int>(at) + 2;
    }
    u64 best = ~0ull, low = ~0ull;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int b = first + i;
      const u32 before = cum;
      cum += got[i];
      if (mass_alone) cum_mass += static_cast<double>(got[i]) * static_cast<double>(least[i]);
      const bool by_count = ask.by_count && cum >= static_cast<u32>(ask.top_k);
      if (best == ~0ull && (by_count || (mass_alone && cum_mass >= enough) || b >= min_bin)) best = static_cast<u64>(b) << 32 | cum;
      if (low == ~0ull && (mass_alone ? cum_mass >= too_little : by_count)) low = static_cast<u64>(b) << 32 | before;
    }
    best = row.block_min(best);
    low = row.block_min(low);
    if (threadIdx.x == 0) {
      row.say(said, best);
      row.say(said_low, low);
    }
  }
  row.sync();
  return Reach{said[0], said_low[0]};
}

// The tokens of the steps below `end`, in index order, to the first block, which then finishes alone: true; false: they are too
// many (of one block).
template <typename T, class W>
__device__ __forceinline__ bool gather_and_finish(Row<T>& row, const SampleArgs& a, int row_id, const W& w, const Steps& steps, float t,
                                                  double total, const Ask& ask, u32 end, u64* scratch) {
  constexpr int VE = per_vec<T>();
  Shared& sh = row.sh;
  const int region = kList / row.cluster;   // of the list, for each block
  int c = 0;
  for (int j = row.v0 + row.lane; j < row.v1; j += kWarp) {
    const Vec<T> v = row.piece(j);
#pragma unroll
    for (int e = 0; e < VE; ++e) c += steps.at(v.at(e)) < end ? 1 : 0;
  }
  c = __reduce_add_sync(0xffffffffu, c);
  if (row.lane == 0) sh.warp_count[row.warp] = c;
  __syncthreads();
  int block = 0, at = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    if (i == row.warp) at = block;
    block += sh.warp_count[i];
  }
  const u64* blocks = row.tell(static_cast<u64>(block));
  if (c > 0 && block <= region) {
    for (int j0 = row.v0; j0 < row.v1; j0 += kWarp) {
      const int j = j0 + row.lane;
      u32 in = 0;
      Vec<T> v;
      if (j < row.v1) {
        v = row.piece(j);
#pragma unroll
        for (int e = 0; e < VE; ++e) in |= steps.at(v.at(e)) < end ? 1u << e : 0u;
      }
      if (!__any_sync(0xffffffffu, in != 0)) continue;
      int inc = __popc(in);
#pragma unroll
      for (int o = 1; o < kWarp; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (row.lane >= o) inc += y;
      }
      int to = at + inc - __popc(in);
      at += __shfl_sync(0xffffffffu, inc, kWarp - 1);
      if (in) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          if (in >> e & 1u) {
            store_remote(&sh.list[row.rank * region + to], 0, entry_of(v.at(e), row.base + j * VE + e));
            ++to;
          }
        }
      }
    }
  }
  row.sync();
  bool fits = true;
  int n = 0;
  for (int r = 0; r < row.cluster; ++r) {
    fits &= blocks[r] <= static_cast<u64>(region);
    n += static_cast<int>(blocks[r]);
  }
  if (!fits) return false;
  if (row.rank != 0) return true;
  // one behind another; the step's sums and candidates then take the list's place and what follows it
  for (int i = threadIdx.x; i < n; i += kThreads) {
    int from = i, r = 0;
    while (from >= static_cast<int>(blocks[r])) from -= static_cast<int>(blocks[r++]);
    scratch[i] = sh.list[r * region + from];
  }
  __syncthreads();
  finish_alone(row, a, row_id, w, steps, t, total, ask, scratch, n, sh.list, scratch + kList);
  return true;
}

// A row by steps.  kBorder: `border` is the last entry, in rank order, that top-k and top-p keep; where `sure` is set, the tokens of the
// steps below its upper word, of which it counts as many as its lower word says, are kept, and their weights added up by warps in
// sh.stretch.  The same for the whole cluster.
template <typename T, class W>
__device__ __forceinline__ Way sample_by_steps(Row<T>& row, const SampleArgs& a, int row_id, const W& w, float t, float lane_top,
                                               const Ask& ask, u64* scratch, u64& border, u64& sure_out) {
  Shared& sh = row.sh;
  const bool mass_alone = ask.by_mass && !ask.by_count;
  const float per_t = mass_alone ? kMassSteps : kCountSteps;
  const Steps steps{w.max, per_t / t};
  const bool usable = !w.at_inf && steps.scale < 1e30f;
  // ---- the lanes' largest logits alone: k of them, or the share of the mass, bound the candidates too, and are counted in no time.
  // Peaked rows and small k end here.
  const u32 x = steps.at(lane_top);
  if (usable && x < kBins) atomicAdd(&sh.lo[x], 1u);
  __syncthreads();   // and the row's total is there
  if (!usable) return Way::kKeys;
  const double total = sh.total;
  if (!mass_alone || total < 4.0) {   // a share of a flat row's mass is out of their reach, and asking takes 6 us (90 -> 84 in all)
    const Reach near = reach_of(row, ask, total, per_t);
    if (near.end != ~0ull &&
        gather_and_finish(row, a, row_id, w, steps, t, total, ask, static_cast<u32>(near.end >> 32) + 1u, scratch))
      return Way::kDone;
  }
  // ---- all logits
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads) sh.lo[i] = 0;
  __syncthreads();
  row.each([&](float l, int) {
    const u32 b = steps.at(l);
    if (b < kBins) atomicAdd(&sh.lo[b], 1u);
  });
  const Reach all = reach_of(row, ask, total, per_t);
  const u64 best = all.end, low = all.low;
  if (best == ~0ull) return Way::kKeys;
  const int end = static_cast<int>(best >> 32) + 1;
  const u32 limit = static_cast<u32>(end);
  if ((best & 0xffffffffu) <= kList && gather_and_finish(row, a, row_id, w, steps, t, total, ask, limit, scratch)) return Way::kDone;
  if ((ask.by_count && ask.by_mass) || low == ~0ull) return Way::kKeys;

  // ---- the step that holds the border, and what lies before it
  const int step0 = static_cast<int>(low >> 32);
  u64 need = static_cast<u64>(ask.top_k), before = low & 0xffffffffu;
  int step = step0;
  u64* slot_step = row.next_slot();
  u64* slot_before = row.next_slot();
  if (mass_alone) {
    const int range = end - step0;
    need = share_of(total * kFixed, ask.top_p);
    u64* own = reinterpret_cast<u64*>(sh.lo);   // 8 bytes a step: up to kBins steps, the histograms have been read
    __syncthreads();
    for (int i = threadIdx.x; i < range; i += kThreads) own[i] = 0;
    __syncthreads();
    const u32 sure = static_cast<u32>(step0);
    row.each_of([&](float l) { return steps.at(l) - sure < static_cast<u32>(range); },
                [&](float l, int) { atomicAdd(&own[steps.at(l) - sure], fixed_of(w.template operator()<exact_diff<T>()>(l))); });
    int unused;
    double sum = row.weigh(w, [&](float l, int) { return steps.at(l) < sure; }, unused);
    if (row.lane == 0) sh.stretch[row.warp] = sum;
    sure_out = low;
    sum = row.block_sum(row.lane == 0 ? sum : 0.0);
    u64* sums = row.tell(static_cast<u64>(__double_as_longlong(sum)));
    row.sync();
    if (row.rank == 0) {
      // by step over the cluster
      double below = 0.0;
      for (int r = 0; r < row.cluster; ++r) below += __longlong_as_double(static_cast<long long>(sums[r]));
      u64 run = static_cast<u64>(__double2ll_rn(below * kFixed));
      u64 found = ~0ull;
      for (int i0 = 0; i0 < range && found == ~0ull; i0 += kThreads) {
        u64 m = 0, all;
        if (i0 + static_cast<int>(threadIdx.x) < range) {
          u64 v[kMaxCluster];   // all on their way at once
#pragma unroll
          for (int r = 0; r < kMaxCluster; ++r) v[r] = r < row.cluster ? load_remote(&own[i0 + threadIdx.x], r) : 0;
#pragma unroll
          for (int r = 0; r < kMaxCluster; ++r) m += v[r];
        }
        const u64 pre = run + row.scan(m, all);
        const bool here = pre < need && pre + m >= need;
        if (here) sh.slot[kSlots - 1][0] = pre;
        found = row.block_min(here ? static_cast<u64>(step0 + i0 + static_cast<int>(threadIdx.x)) : ~0ull);
        run += all;
      }
      if (threadIdx.x == 0) {
        row.say(slot_step, found);
        row.say(slot_before, sh.slot[kSlots - 1][0]);
      }
    }
    row.sync();
    if (slot_step[0] == ~0ull) return Way::kKeys;
    step = static_cast<int>(slot_step[0]);
    before = slot_before[0];
  }
  // ---- the step's tokens, in any order, to the first block
  u64* said_border = row.next_slot();
  u32* taken = reinterpret_cast<u32*>(&sh.warp_count[0]);
  if (threadIdx.x == 0) *taken = 0;
  row.sync();   // nobody reads what the list takes the place of
  row.each_of([&](float l) { return steps.at(l) == static_cast<u32>(step); },   // a hundred or so of the row
              [&](float l, int i) {
                const u32 at = take_from_remote(taken, 0, 1);
                if (at < kList) store_remote(&sh.list[at], 0, entry_of(l, i));
              });
  row.sync();
  if (row.rank == 0) {
    const int m = static_cast<int>(*taken);
    u64 found = ~0ull;
    if (m <= kList / 2) {   // the slice is still needed: the amounts take the list's other half
      u64* amounts = sh.list + kList / 2;
      for (int i = threadIdx.x; i < m; i += kThreads)
        amounts[i] = mass_alone ? fixed_of(w.template operator()<exact_diff<T>()>(logit_of(sh.list[i]))) : 1;
      __syncthreads();
      found = border_among(row, sh.list, amounts, m, before, need);
    }
    if (threadIdx.x == 0) row.say(said_border, found);
  }
  row.sync();
  border = said_border[0];
  return border == ~0ull ? Way::kKeys : Way::kBorder;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kBlocks)
sample_filter_kernel(SampleArgs a, int cluster, int slice) {
  constexpr int VE = per_vec<T>();
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  uint4* data = reinterpret_cast<uint4*>(smem + kSharedBytes);
  const int row_id = blockIdx.x / cluster;
  if (a.row_mask && a.row_mask[row_id] == 0) {   // the same for the whole cluster
    if (blockIdx.x % cluster == 0 && threadIdx.x == 0) a.put(row_id, -1, 0.0, 0.0, 0);
    return;
  }
  cluster_arrive();   // waited for before anything is written to another block's shared memory
  Row<T> row(sh);
  row.cluster = cluster;
  row.rank = static_cast<int>(blockIdx.x % cluster);
  row.flip = row.slot = 0;
  row.lane = threadIdx.x % kWarp;
  row.warp = threadIdx.x / kWarp;

  // ---- the slice into shared memory, NaN as -inf and -0 as 0
  const int from = row.rank * slice, len = max(0, min(slice, a.v - from));
  const T* l = static_cast<const T*>(a.logits) + row_id * a.ld + from;
  const int head = head_of(l);
  row.data = data;
  row.vecs = len > 0 ? (head + len + VE - 1) / VE : 0;
  row.base = from - head;
  const int stretch = (row.vecs + kWarps - 1) / kWarps;
  row.v0 = min(row.warp * stretch, row.vecs);
  row.v1 = min(row.v0 + stretch, row.vecs);
  constexpr int kAtOnce = 4;
  float lane_top = -INFINITY;          // the largest of this lane's logits
  u32 lane_pair = 0xff80ff80u;
  bool table = false;
  for (int j0 = row.v0 + row.lane; ; j0 += kWarp * kAtOnce) {
    Vec<T> v[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int j = j0 + i * kWarp;
      if (j < row.v1) v[i] = load_vec(l, j * VE - head, len);
    }
    if (!table) {   // while the first of them are on their way
      table = true;
      fill_table(sh.table, threadIdx.x, kThreads);
      for (int i = threadIdx.x; i < kBins; i += kThreads) sh.lo[i] = 0;
    }
    if (j0 >= row.v1) break;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int j = j0 + i * kWarp;
      if (j >= row.v1) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
          const float x = __fadd_rn(fmaxf(__uint_as_float(v[i].w[e]), -INFINITY), 0.f);
          v[i].w[e] = __float_as_uint(x);
          lane_top = fmaxf(lane_top, x);
        } else {
          asm("max.bf16x2 %0, %0, %1;" : "+r"(v[i].w[e]) : "r"(0xff80ff80u));   // passes over NaN
          asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(v[i].w[e]) : "r"(0u));
          asm("max.bf16x2 %0, %0, %1;" : "+r"(lane_pair) : "r"(v[i].w[e]));
        }
      }
      data[j] = make_uint4(v[i].w[0], v[i].w[1], v[i].w[2], v[i].w[3]);   // a warp reads its own stretch alone
    }
  }
  __syncthreads();   // the table

  // ---- the sums of the warps' weights, relative to their largest, and from them the row's
  bool greedy;
  const float t = a.temp(row_id, greedy);
  Weights<16> w;
  w.set_temperature(t, sh.table);
  constexpr bool kExact = exact_diff<T>();
  auto weight = [&](float x) { return w.template operator()<kExact>(x); };
  if (sizeof(T) == 2) lane_top = fmaxf(__uint_as_float(lane_pair << 16), __uint_as_float(lane_pair & 0xffff0000u));
  const float own_max = of_key(__reduce_max_sync(0xffffffffu, key_of(lane_top)));
  w.set_max(own_max);
  {
    double s = 0.0;
    if (own_max > -INFINITY) {
      if (w.floor > -1e37f && fabsf(own_max) < 1e6f * -w.floor) {   // the limit below is a number well under the largest
        // What is -inf or far below the largest counts as its 2^-100th here, which no sum that holds a 1 shows.
        const float least = own_max + w.floor;
        WeightSum even, odd;
        for (int j0 = row.v0 + row.lane; j0 < row.v1; j0 += 2 * kWarp) {
          const int j1 = j0 + kWarp;
          const Vec<T> x = row.piece(j0), y = row.piece(min(j1, row.v1 - 1));
#pragma unroll
          for (int e = 0; e < VE; e += 2) w.template add<kExact>(f2(fmaxf(x.at(e), least), fmaxf(x.at(e + 1), least)), even);
          if (j1 < row.v1) {
#pragma unroll
            for (int e = 0; e < VE; e += 2) w.template add<kExact>(f2(fmaxf(y.at(e), least), fmaxf(y.at(e + 1), least)), odd);
          }
        }
        s = even.value() + odd.value();
      } else {
        row.each([&](float x, int) { s += weight(x); });
      }
    }
    s = warp_sum(s);
    if (row.lane == 0) {
      sh.stretch[row.warp] = s;
      sh.stretch_max[row.warp] = own_max;
    }
  }
  // what a sum relative to x counts for relative to y
  auto factor = [&](float x, float y) {
    return x == y ? 1.0 : x > -INFINITY ? exp((static_cast<double>(x) - static_cast<double>(y)) / static_cast<double>(t)) : 0.0;
  };
  cluster_wait();
  __syncthreads();
  u64* maxes = row.next_slot();
  u64* block_sums = row.next_slot();
  if (row.warp == 0) {
    const float x = row.lane < kWarps ? sh.stretch_max[row.lane] : -INFINITY;
    const float most = of_key(__reduce_max_sync(0xffffffffu, key_of(x)));
    const double s = warp_sum(row.lane < kWarps ? sh.stretch[row.lane] * factor(x, most) : 0.0);
    if (row.lane < cluster) {
      store_remote(maxes + row.rank, row.lane, key_of(most));
      store_remote(block_sums + row.rank, row.lane, static_cast<u64>(__double_as_longlong(s)));
    }
  }
  row.sync();
  u32 top_key = 0;
  for (int r = 0; r < cluster; ++r) top_key = max(top_key, static_cast<u32>(maxes[r]));
  const float m = of_key(top_key);
  if (!(m > -INFINITY)) {   // the same for the whole cluster
    if (row.rank == 0 && threadIdx.x == 0) a.put(row_id, -1, 0.0, 0.0, 0);
    return;
  }
  if (row.warp == kWarps - 1) {   // read after the next barrier of the block
    const double s = row.lane < cluster ? __longlong_as_double(static_cast<long long>(block_sums[row.lane])) *
                                              factor(of_key(static_cast<u32>(maxes[row.lane])), m)
                                        : 0.0;
    const double all = warp_sum(s);
    if (row.lane == 0) sh.total = all;
  }
  w.set_max(m);

  // ---- greedy: the first of the largest
  if (greedy) {
    u64 first = ~0ull;
    row.each([&](float x, int i) {
      if (x == m) first = min(first, static_cast<u64>(i));
    });
    first = row.cluster_min(first);
    if (row.rank == 0 && threadIdx.x == 0) a.put(row_id, static_cast<int>(first), -log(sh.total), 0.0, 1);
    return;
  }

  Ask ask;
  ask.top_k = a.top_k ? a.top_k[row_id] : 0;
  ask.top_p = a.top_p ? a.top_p[row_id] : 1.f;
  ask.min_p = a.min_p ? a.min_p[row_id] : 0.f;
  ask.by_count = ask.top_k > 0 && ask.top_k < a.v;
  ask.by_mass = ask.top_p < 1.f;
  ask.by_min = ask.min_p > 0.f;
  ask.min_bound = ask.by_min ? static_cast<double>(m) + log(static_cast<double>(ask.min_p)) * static_cast<double>(t) : 0.0;

  // ---- what is kept: keys above `edge`, and of those equal to it the indexes up to `limit`
  const u32 none = tkey<T>(-INFINITY), best = tkey<T>(m);
  u32 edge = none;
  int limit = -1;
  bool many = false;   // more than a few thousand are kept, as far as is known
  u64 sure = 0;        // of them: see sample_by_steps
  if (ask.by_count || ask.by_mass || ask.by_min) {
    u64 border = 0;
    const Way way = sample_by_steps(row, a, row_id, w, t, lane_top, ask, reinterpret_cast<u64*>(data), border, sure);
    if (way == Way::kDone) return;
    const double total = sh.total;
    if (way == Way::kBorder) {
      edge = tkey<T>(logit_of(border));
      limit = static_cast<int>(border & 0xffffffffu);
      many = true;
    } else {
      int ties = 0;
      u64 above;
      double of = total * kFixed;   // the mass that top-p has a share of
      if (ask.by_count) {
        const u32 k = row.template border<false>(none, best, static_cast<u64>(ask.top_k), [](float) { return 0ull; }, above);
        if (k > none) {
          edge = k;
          ties = ask.top_k - static_cast<int>(above);
        }
        if (ask.by_mass) {
          const u32 e = edge;
          u64 all = 0;
          row.each([&](float x, int) {
            if (tkey<T>(x) > e) all += fixed_of(weight(x));
          });
          all = row.cluster_sum(all);
          if (edge > none) all += static_cast<u64>(ties) * fixed_of(weight(of_tkey<T>(edge)));
          of = static_cast<double>(all);
        }
      }
      if (ask.by_mass) {
        const u64 need = share_of(of, ask.top_p);
        u32 lo = edge;
        if (edge == none) {   // lighter than (1 - p) / V of all: even together they are not the part that is left out
          const double cut = (1.0 - static_cast<double>(fmaxf(ask.top_p, 0.f))) * total / a.v * 0.999;
          const double bound = static_cast<double>(m) + log(cut) * static_cast<double>(t);
          const float f = bound < static_cast<double>(m) ? __double2float_rd(bound) : m;
          lo = min(max(tkey<T>(f), none), best);
        }
        const u32 k = row.template border<true>(lo, best, need, [&](float x) { return fixed_of(weight(x)); }, above);
        const u64 each = fixed_of(weight(of_tkey<T>(k)));
        u64 c = each > 0 && need > above ? (need - above + each - 1) / each : 1;
        if (c < 1) c = 1;
        if (c > static_cast<u64>(a.v)) c = a.v;
        if (k > edge || edge == none) {
          edge = k;
          ties = static_cast<int>(c);
        } else if (static_cast<int>(c) < ties) {
          ties = static_cast<int>(c);
        }
      }
      // the index of the last tie that is kept
      if (edge > none) {
        int c = 0;
        row.each([&](float x, int) { c += tkey<T>(x) == edge ? 1 : 0; });
        c = __reduce_add_sync(0xffffffffu, c);
        __syncthreads();
        if (row.lane == 0) sh.warp_count[row.warp] = c;
        __syncthreads();
        int block = 0, mine = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
          if (i == row.warp) mine = block;
          block += sh.warp_count[i];
        }
        const u64* s = row.tell(static_cast<u64>(block));
        u64* said = row.next_slot();
        row.sync();
        int before = 0, sum = 0;
        for (int r = 0; r < cluster; ++r) {
          if (r == row.rank) before = sum;
          sum += static_cast<int>(s[r]);
        }
        limit = INT_MAX;
        if (sum > ties) {
          const int from_here = ties - before - mine;   // the from_here-th of this warp's ties is the last
          if (from_here >= 1 && from_here <= c) {
            const int at = find_nth(row, from_here, [&](float x) { return tkey<T>(x) == edge; });
            if (row.lane == 0) row.say(said, static_cast<u64>(at));
          }
          row.sync();
          limit = static_cast<int>(said[0]);
        }
      }
    }
    if (ask.min_p > 1.f) {   // the first rank alone: the first of the largest
      u64 first = ~0ull;
      row.each([&](float x, int i) {
        if (x == m) first = min(first, static_cast<u64>(i));
      });
      edge = best;
      limit = static_cast<int>(row.cluster_min(first));
      sure = 0;
    } else if (ask.by_min) {
      float f = __double2float_ru(ask.min_bound);   // the smallest logit that stays
      if (f > m) f = m;
      u32 k = tkey<T>(f + 0.f);
      if (of_tkey<T>(k) < f) ++k;
      if (k > edge) {
        edge = k;
        limit = INT_MAX;
        sure = 0;
      }
    }
  } else {
    __syncthreads();   // the total
  }
  const double total = sh.total;
  const float edge_at = of_tkey<T>(edge);
  auto kept = [&](float x, int i) { return x > edge_at || (x == edge_at && i <= limit); };

  // ---- the kept weights by stretches
  double s = 0.0;
  int count = 0;
  if (sure != 0) {   // (whichever way the border was found: their sums have taken the place of the row's) what lies between them and it
    const Steps steps{m, kMassSteps / t};
    const u32 from = static_cast<u32>(sure >> 32);
    row.each_of([&](float x) { return x >= edge_at && steps.at(x) >= from; },
                [&](float x, int i) {
                  if (kept(x, i)) {
                    s += weight(x);
                    ++count;
                  }
                });
    s = warp_sum(s) + sh.stretch[row.warp];
    if (row.rank == 0 && threadIdx.x == 0) count += static_cast<int>(sure & 0xffffffffu);
  } else if (edge == none) {   // all of them: their sums are there
    row.each([&](float x, int) { count += x > -INFINITY ? 1 : 0; });
    s = sh.stretch[row.warp] * factor(sh.stretch_max[row.warp], m);
    if (s < 0x1p-60) {   // perhaps nothing but what counts as 2^-100 there and as 0 here
      s = 0.0;
      row.each([&](float x, int) { s += weight(x); });
      s = warp_sum(s);
    }
  } else if (many) {
    s = row.weigh(w, kept, count);
  } else {
    row.each([&](float x, int i) {
      if (kept(x, i)) {
        s += weight(x);
        ++count;
      }
    });
    s = warp_sum(s);
  }
  count = __reduce_add_sync(0xffffffffu, count);
  __syncthreads();   // warp_count has been read
  u64* sums = sh.part[row.flip ^= 1];
  if (row.lane == 0) {
    sums[row.warp] = static_cast<u64>(__double_as_longlong(s));
    sh.warp_count[row.warp] = count;
  }
  __syncthreads();
  double block = 0.0;
  int block_count = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    block += __longlong_as_double(static_cast<long long>(sums[i]));
    block_count += sh.warp_count[i];
  }
  const u64* all_sums = row.tell(static_cast<u64>(__double_as_longlong(block)));
  const u64* all_counts = row.tell(static_cast<u64>(block_count));
  row.sync();
  double kept_total = 0.0;
  int kept_count = 0;
  for (int r = 0; r < cluster; ++r) {
    kept_total += __longlong_as_double(static_cast<long long>(all_sums[r]));
    kept_count += static_cast<int>(all_counts[r]);
  }
  const double target = static_cast<double>(fmaxf(a.u[row_id], 0.f)) * kept_total;   // NaN and what is below 0 count as 0
  // the block, and in it the stretch, that the target falls into; past the end the last that has any
  double run = 0.0, at = 0.0;
  int owner = 0;
  for (int r = 0; r < cluster; ++r) {
    const double x = __longlong_as_double(static_cast<long long>(all_sums[r]));
    if (!(x > 0.0)) continue;
    owner = r;
    at = run;
    run += x;
    if (target < run) break;
  }
  if (owner != row.rank) return;
  const double rest = target - at;
  double upto = 0.0, first = 0.0;
  int who = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    const double x = __longlong_as_double(static_cast<long long>(sums[i]));
    if (x > 0.0 && (upto <= rest || i == 0)) {
      who = i;
      first = upto;
    }
    upto += x;
  }
  const int place = find_by_sum(row, min(who * stretch, row.vecs), min((who + 1) * stretch, row.vecs), rest - first,
                                [&](float x, int i) { return kept(x, i) ? weight(x) : 0.0; });
  if (threadIdx.x == 0) {
    const float picked = to_float(reinterpret_cast<const T*>(data)[place]);
    const double z = picked == m ? 0.0 : (static_cast<double>(picked) - static_cast<double>(m)) / static_cast<double>(t);
    a.put(row_id, row.base + place, z - log(total), z - log(kept_total), kept_count);
  }
}

template <typename T>
int launch(const SampleArgs& a, int cluster, cudaStream_t stream) {
  const int slice = ((a.v + cluster - 1) / cluster + 7) / 8 * 8;
  const size_t smem = kSharedBytes + room_of(static_cast<size_t>(slice) * sizeof(T));   // kMostShared at most
  // The limit belongs to the kernel, not to the call: every call sets the same one, so that none lowers it between another
  // thread's setting it and its launch.
  if (cudaFuncSetAttribute(sample_filter_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMostShared)) !=
      cudaSuccess) {
    cudaGetLastError();
    return A3PO_ERR_CUDA;
  }
  A3PO_LAUNCH(kKSampleFilter, stream, (launch_early(sample_filter_kernel<T>, static_cast<unsigned>(a.n) * cluster, kThreads,
                                                    smem, stream, cluster, false, a, cluster, slice)));
  return after_launch();
}
