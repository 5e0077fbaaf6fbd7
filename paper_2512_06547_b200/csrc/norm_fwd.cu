// Norm and dropout + add + norm, forward (mathematics in row_ops.cu).
//
// Bound by HBM: 2 (join: 4) elements moved per element, a few dozen instructions for 8 of them.  Blocks are persistent and
// stream their rows through a ring in shared memory (row_ops.cuh), because with one row per block and plain loads the
// memory system sat idle between the phases of a row: join on 32,768 x 4,096 bf16 ran at 0.51 of DRAM throughput with
// 48 registers, 62 % occupancy and half of all stalls on loads.  Now, 32,768 x 4,096 bf16, RMS: norm 88 us (6.1 TB/s), join
// 174 us (6.2 TB/s).  Batches of a few rows per block are bound by latency and by the block that the mask leaves most rows:
// 16,384 x 1,536, 38 % masked, layer norm: join 41-45 us for 164 MB.

#include "row_ops.cuh"

namespace a3po {
namespace {

// MAXT: most threads of a block (a register limit: three blocks of 256 threads on an SM, or two
// where three would spill; one of 512).
template <typename T, int CPT, bool WIDE, int MAXT, bool VEC, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(MAXT, MAXT == 256 ? (JOIN || sizeof(T) == 4 ? 2 : 3) : 1)
norm_fwd_kernel(const NormFwdArgs<T> a, int lanes, Turns turns) {
  constexpr int kIn = JOIN ? 2 : 1;
  constexpr int kRing = ring_rows<T>(kIn, CPT);
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float sums[4 * RowSum<WIDE>::kSlots];
  const RowThreads<WIDE> rt(lanes);
  const Columns<T, CPT, WIDE, VEC> cols(rt, a.h);
  RowSum<WIDE> row_sum(sums);
  Ring<T, CPT, kIn, kRing> ring(smem);
  if constexpr (VEC) ring.clear();
  Raw<T> gamma[CPT], beta[CPT];
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    gamma[i] = cols.read(a.gamma, i);
    beta[i] = cols.read(a.beta, i, a.beta != nullptr);
  }
  const bool drop = JOIN && a.drop.rng != nullptr;
  PhiloxState ph;
  if (drop) ph.load(a.drop.rng);
  const uint32_t n = static_cast<uint32_t>(a.n);

  auto row_at = [&](uint32_t k) { return turns.unit(k) * static_cast<uint32_t>(rt.rows) + static_cast<uint32_t>(rt.slot); };
  auto row_on = [&](uint32_t t) { return t < n && (!a.row_mask || a.row_mask[t] != 0); };
  auto fetch = [&](uint32_t t, uint32_t st, bool on) {   // this thread's chunks of row t into the ring
    if (on) {
#pragma unroll
      for (int in = 0; in < kIn; ++in) {
        const T* src = (in ? a.residual : a.x) + static_cast<long long>(t) * a.h;
#pragma unroll
        for (int i = 0; i < CPT; ++i)
          if (cols.have[i]) ring.fetch(st, in, i, src + cols.at[i]);
      }
    }
    cp_async_commit();
  };
  // masks are read ahead of their use: of the row fetched next, and of the row after this one
  bool on_next = false;
  if constexpr (VEC) {
#pragma unroll
    for (int k = 0; k < kRing; ++k) fetch(row_at(k), k, row_on(row_at(k)));
    on_next = row_on(row_at(kRing));
  }
  bool on = row_on(row_at(0));
  for (uint32_t k = 0; turns.unit(k) * static_cast<uint32_t>(rt.rows) < n; ++k) {   // the same trips for the whole block
    const uint32_t t = row_at(k);
    const bool on_ahead = row_on(row_at(k + 1));
    const long long off = static_cast<long long>(t) * a.h;
    if (WIDE && !on) {   // the whole block: zeros
      Raw<T> z;
      z.clear();
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        cols.write(a.y + off, i, z);
        if (JOIN) cols.write(a.r + off, i, z);
      }
      if (rt.tid == 0) {
        if (a.mean) a.mean[t] = 0.f;
        if (a.rstd) a.rstd[t] = 0.f;
      }
      if constexpr (VEC) {
        fetch(row_at(k + kRing), ring.stage, on_next);
        on_next = row_on(row_at(k + kRing + 1));
        ring.advance();
      }
      on = on_ahead;
      continue;
    }
    F2 v[CPT][kPairs], res[JOIN ? CPT : 1][kPairs];
    if constexpr (VEC) {
      cp_async_wait<kRing - 1>();
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        ring.take(0, i, WIDE || on).get(v[i]);
        if constexpr (JOIN) ring.take(1, i, WIDE || on).get(res[i]);
      }
      fetch(row_at(k + kRing), ring.stage, on_next);
      on_next = row_on(row_at(k + kRing + 1));
      ring.advance();
    } else {
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        cols.read(a.x + off, i, on).get(v[i]);
        if constexpr (JOIN) cols.read(a.residual + off, i, on).get(res[i]);
      }
    }
    if constexpr (JOIN) {
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        if (drop) {
          bool keep[kVec];
          keep_bits(ph.draw(static_cast<uint32_t>(i * rt.tpr + rt.tid), t), a.drop.below, keep);
          rt.template own_bits<VEC>(keep);
#pragma unroll
          for (int j = 0; j < kPairs; ++j)
            v[i][j] = add2(drop2(keep[2 * j], keep[2 * j + 1], v[i][j], a.drop.scale), res[i][j]);
        } else {
#pragma unroll
          for (int j = 0; j < kPairs; ++j) v[i][j] = add2(v[i][j], res[i][j]);
        }
        // the norm is that of the stored sum, which is what the backward will read
        Raw<T> stored;
        stored.set(v[i]);
        if (t < n) cols.write(a.r + off, i, stored);
        stored.get(v[i]);
      }
    }
    float mean = 0.f;
    if constexpr (LAYER) {
      F2 s = f2(0.f);
#pragma unroll
      for (int i = 0; i < CPT; ++i)
#pragma unroll
        for (int j = 0; j < kPairs; ++j) s = add2(s, v[i][j]);
      float total[1] = {parts(s).x + parts(s).y};
      row_sum(total, rt);
      mean = total[0] * a.inv_h;
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        if constexpr (VEC) {
          if (cols.have[i]) {
#pragma unroll
            for (int j = 0; j < kPairs; ++j) v[i][j] = add2(v[i][j], f2(-mean));
          }
        } else {
#pragma unroll
          for (int j = 0; j < kPairs; ++j)
            v[i][j] = add2(v[i][j], f2(cols.col(i, 2 * j) < a.h ? -mean : 0.f, cols.col(i, 2 * j + 1) < a.h ? -mean : 0.f));
        }
      }
    }
    F2 q = f2(0.f);
#pragma unroll
    for (int i = 0; i < CPT; ++i)
#pragma unroll
      for (int j = 0; j < kPairs; ++j) q = fma2(v[i][j], v[i][j], q);
    float total[1] = {parts(q).x + parts(q).y};
    row_sum(total, rt);
    const float rstd = 1.0f / sqrtf(total[0] * a.inv_h + a.eps);
    if (t < n) {
      if (rt.tid == 0) {
        if (a.mean) a.mean[t] = on ? mean : 0.f;
        if (a.rstd) a.rstd[t] = on ? rstd : 0.f;
      }
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        F2 g[kPairs];
        gamma[i].get(g);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) v[i][j] = mul2(mul2(v[i][j], f2(rstd)), g[j]);
        if (a.beta) {
          beta[i].get(g);
#pragma unroll
          for (int j = 0; j < kPairs; ++j) v[i][j] = add2(v[i][j], g[j]);
        }
        if (!WIDE && !on) {
#pragma unroll
          for (int j = 0; j < kPairs; ++j) v[i][j] = f2(0.f);
        }
        cols.write(a.y + off, i, v[i]);
      }
    }
    on = on_ahead;
  }
  if constexpr (VEC) cp_async_wait<0>();
}

// Rows longer than the register form holds: the row is read again for each use (from L2), one row per block.  8,192 x 20,000
// bf16: RMS 295 us (0.34 of the copy rate), join 512 (0.39).
template <typename T, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(kLongThreads)
norm_fwd_long_kernel(const NormFwdArgs<T> a) {
  __shared__ float2 sh[kWarp];
  const long long t = blockIdx.x;
  const bool vec = a.vec != 0;
  const bool masked = a.row_mask && a.row_mask[t] == 0;
  T* y = a.y + t * a.h;
  T* r = JOIN ? a.r + t * a.h : nullptr;
  const T* x = JOIN ? r : a.x + t * a.h;
  const bool drop = JOIN && a.drop.rng != nullptr;
  PhiloxState ph;
  if (drop) ph.load(a.drop.rng);
  float s = 0.f;
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float v[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = 0.f;
    if (masked) {
      store_chunk(y, col, a.h, vec, v);
      if (JOIN) store_chunk(r, col, a.h, vec, v);
      continue;
    }
    load_chunk(a.x + t * a.h, col, a.h, vec, v);
    if constexpr (JOIN) {
      float res[kVec];
      load_chunk(a.residual + t * a.h, col, a.h, vec, res);
      if (drop) {
        bool keep[kVec];
        keep_bits(ph.draw(static_cast<uint32_t>(col / kVec), static_cast<uint32_t>(t)), a.drop.below, keep);
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[j] = drop_add(keep[j], v[j], a.drop.scale, res[j]);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[j] += res[j];
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[j] = as_stored<T>(v[j]);
      store_chunk(r, col, a.h, vec, v);
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) s += v[j];
  }
  if (masked) {
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[t] = 0.f;
      if (a.rstd) a.rstd[t] = 0.f;
    }
    return;
  }
  // each thread reads back only chunks that it wrote itself
  const float mean = LAYER ? block_sum2(s, 0.f, sh).x * a.inv_h : 0.f;
  float q = 0.f;
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float v[kVec];
    load_chunk(x, col, a.h, vec, v);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const float d = (col + j < a.h) ? v[j] - mean : 0.f;
      q = fmaf(d, d, q);
    }
  }
  const float rstd = 1.0f / sqrtf(block_sum2(q, 0.f, sh).x * a.inv_h + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[t] = mean;
    if (a.rstd) a.rstd[t] = rstd;
  }
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float v[kVec], g[kVec], b[kVec];
    load_chunk(x, col, a.h, vec, v);
    load_chunk(a.gamma, col, a.h, vec, g);
#pragma unroll
    for (int j = 0; j < kVec; ++j) b[j] = 0.f;
    if (a.beta) load_chunk(a.beta, col, a.h, vec, b);
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = fmaf((v[j] - mean) * rstd, g[j], b[j]);
    store_chunk(y, col, a.h, vec, v);
  }
}


template <typename T, int CPT, bool WIDE, int MAXT, bool VEC, bool LAYER, bool JOIN>
int launch(const NormFwdArgs<T>& a, int threads, int lanes, cudaStream_t stream) {
  auto kernel = norm_fwd_kernel<T, CPT, WIDE, MAXT, VEC, LAYER, JOIN>;
  const size_t smem = VEC ? static_cast<size_t>(threads) * CPT * ring_rows<T>(JOIN ? 2 : 1, CPT) * (JOIN ? 2 : 1) * sizeof(Raw<T>) : 0;
  static std::atomic<uint64_t> cached[64];
  const int per_sm = blocks_per_sm(kernel, threads, smem, 2048 / threads, cached);
  if (per_sm <= 0) return A3PO_ERR_CUDA;
  const int rows = WIDE ? 1 : threads / lanes;
  long long blocks = (a.n + rows - 1) / rows;
  // Long rows: a block per 16 rows once that is more than twice what fits at a time, so that the hardware hands them out as blocks
  // finish (65,536 x 1,536 and x 2,048 bf16, RMS norm: 82 -> 70 and 104 -> 88 us, with the join 157 -> 132 and 200 -> 169 us;
  // a layer norm gains little, narrow rows nothing).
  long long most = static_cast<long long>(sm_count()) * per_sm;
  if (WIDE && blocks / 16 > 2 * most) most = blocks / 16;
  if (blocks > most) blocks = most;
  const Turns turns{turn_shift((a.n + rows - 1) / rows, blocks)};
  A3PO_LAUNCH(kKNorm, stream, (kernel<<<static_cast<unsigned>(blocks), threads, smem, stream>>>(a, lanes, turns)));
  return after_launch();
}

// Rows of up to 512 columns share a block, 1 or 2 chunks per thread; longer ones take a block of as many warps as give
// every thread 2 chunks (up to 8,192 columns) or 4.  With 4, dropout and the sum spill (120-264 bytes a thread): 16,384 x
// 16,384 bf16, RMS: norm 180 us (0.91 of the copy rate), join 542 (0.61).
template <typename T, bool VEC, bool LAYER, bool JOIN>
int by_length(const NormFwdArgs<T>& a, cudaStream_t stream) {
  const int groups = (a.h + kVec - 1) / kVec;
  int lanes = 1;
  if (groups <= 32) {
    while (lanes < groups) lanes *= 2;
    return launch<T, 1, false, kNarrowThreads, VEC, LAYER, JOIN>(a, kNarrowThreads, lanes, stream);
  }
  if (groups <= 64) return launch<T, 2, false, kNarrowThreads, VEC, LAYER, JOIN>(a, kNarrowThreads, kWarp, stream);
  if (groups <= 2 * kNarrowThreads)
    return launch<T, 2, true, kNarrowThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up((groups + 1) / 2, kWarp)), 0, stream);
  if (groups <= 2 * kWideThreads)
    return launch<T, 2, true, kWideThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up((groups + 1) / 2, kWarp)), 0, stream);
  if (groups <= 4 * kWideThreads)
    return launch<T, 4, true, kWideThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up((groups + 3) / 4, kWarp)), 0, stream);
  A3PO_LAUNCH(kKNorm, stream, (norm_fwd_long_kernel<T, LAYER, JOIN>
                                   <<<static_cast<unsigned>(a.n), kLongThreads, 0, stream>>>(a)));
  return after_launch();
}

template <typename T, bool LAYER, bool JOIN>
int by_alignment(const NormFwdArgs<T>& a, cudaStream_t stream) {
  return a.vec ? by_length<T, true, LAYER, JOIN>(a, stream) : by_length<T, false, LAYER, JOIN>(a, stream);
}
template <typename T>
int by_kind(const NormFwdArgs<T>& a, bool layer, bool join, cudaStream_t stream) {
  if (layer) return join ? by_alignment<T, true, true>(a, stream) : by_alignment<T, true, false>(a, stream);
  return join ? by_alignment<T, false, true>(a, stream) : by_alignment<T, false, false>(a, stream);
}

}  // namespace

int launch_norm_fwd(const NormFwdArgs<float>& a, bool layer, bool join, cudaStream_t stream) {
  return by_kind(a, layer, join, stream);
}
int launch_norm_fwd(const NormFwdArgs<__nv_bfloat16>& a, bool layer, bool join, cudaStream_t stream) {
  return by_kind(a, layer, join, stream);
}

}  // namespace a3po
