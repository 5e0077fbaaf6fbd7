// Norm and dropout + add + norm, backward (mathematics in row_ops.cu).
//
// Bound by HBM: 3 (join: 4 or 5) elements moved per element.  Persistent blocks stream their rows through a ring in shared
// memory (row_ops.cuh) and keep their share of dgamma / dbeta in registers, one sum per column a thread owns; the
// blocks' shares are added up in index order by reduce_parts_kernel, so results do not depend on the order in which
// blocks run.  131,072 x 4,096 bf16 with 39 % of the rows masked: 376-392 us (6.1-6.3 TB/s with the zero rows that it writes);
// join on 65,536 x 4,096, five streams: 437-475 us (5.7-6.1 TB/s); layer norm on 5,001 x 1,003 bf16: 21 us, latency.

#include "row_ops.cuh"

namespace a3po {
namespace {

// MAXT: most threads of a block, and with it a register limit: two blocks of 256 threads on an SM, one of 512.  With three,
// a layer norm's sums spill (65,536 x 2,048 bf16: 194 us against 140) and an RMS norm gains nothing (8B-shaped batch,
// 39 % masked: 402 against 376, of the same run); only element-wise rows, which have no ring, want the third (5,001 x 1,003: 24.6 against 22.6).
template <typename T, int CPT, bool WIDE, int MAXT, bool VEC, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(MAXT, MAXT == 256 ? (VEC || JOIN || sizeof(T) == 4 ? 2 : 3) : 1)
norm_bwd_kernel(const NormBwdArgs<T> a, int lanes, Turns turns) {
  constexpr int kIn = JOIN ? 3 : 2;
  constexpr int kRing = ring_rows<T>(kIn, CPT);
  constexpr int kSums = LAYER ? 2 : 1;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float sums[4 * RowSum<WIDE>::kSlots];
  allow_next();
  const RowThreads<WIDE> rt(lanes);
  const Columns<T, CPT, WIDE, VEC> cols(rt, a.h);
  RowSum<WIDE> row_sum(sums);
  Ring<T, CPT, kIn, kRing> ring(smem);
  if constexpr (VEC) ring.clear();
  const bool drop = JOIN && a.drop.rng != nullptr;
  const bool past = JOIN && a.grad_r != nullptr;
  PhiloxState ph;
  if (drop) ph.load(a.drop.rng);
  Raw<T> gamma[CPT];
  F2 dg[CPT][kPairs], db[LAYER ? CPT : 1][kPairs];
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    gamma[i] = cols.read(a.gamma, i);
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      dg[i][j] = f2(0.f);
      if (LAYER) db[i][j] = f2(0.f);
    }
  }
  const uint32_t n = static_cast<uint32_t>(a.n);

  auto row_at = [&](uint32_t k) { return turns.unit(k) * static_cast<uint32_t>(rt.rows) + static_cast<uint32_t>(rt.slot); };
  auto row_on = [&](uint32_t t) { return t < n && (!a.row_mask || a.row_mask[t] != 0); };
  auto fetch = [&](uint32_t t, uint32_t st, bool on) {   // this thread's chunks of row t into the ring
    if (on) {
#pragma unroll
      for (int in = 0; in < kIn; ++in) {
        if (in == 2 && !past) continue;
        const T* src = (in == 0 ? a.x : in == 1 ? a.grad_y : a.grad_r) + static_cast<long long>(t) * a.h;
#pragma unroll
        for (int i = 0; i < CPT; ++i)
          if (cols.have[i]) ring.fetch(st, in, i, src + cols.at[i]);
      }
    }
    cp_async_commit();
  };
  // Masks and statistics are read ahead of their use: the mask of the row fetched next, all of the row after this one.
  // Without the ring the elements of the next row wait in registers.
  bool on_next = false;
  bool on = row_on(row_at(0));
  Raw<T> held[VEC ? 1 : kIn][VEC ? 1 : CPT];
  auto hold = [&](uint32_t t, bool have) {
    const long long off = static_cast<long long>(t) * a.h;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      held[0][VEC ? 0 : i] = cols.read(a.x + off, i, have);
      held[VEC ? 0 : 1][VEC ? 0 : i] = cols.read(a.grad_y + off, i, have);
      if constexpr (JOIN) held[VEC ? 0 : 2][VEC ? 0 : i] = cols.read(a.grad_r + off, i, have && past);
    }
  };
  if constexpr (VEC) {
#pragma unroll
    for (int k = 0; k < kRing; ++k) fetch(row_at(k), k, row_on(row_at(k)));
    on_next = row_on(row_at(kRing));
  } else {
    hold(row_at(0), on);
    on_next = row_on(row_at(1));
  }
  float rstd = on ? a.rstd[row_at(0)] : 0.f;
  float mean = LAYER && on ? a.mean[row_at(0)] : 0.f;
  for (uint32_t k = 0; turns.unit(k) * static_cast<uint32_t>(rt.rows) < n; ++k) {   // the same trips for the whole block
    const uint32_t t = row_at(k), ahead = row_at(k + 1);
    const long long off = static_cast<long long>(t) * a.h;
    const bool on_ahead = VEC ? row_on(ahead) : on_next;
    float rstd_ahead = 0.f, mean_ahead = 0.f;
    if (ahead < n) {   // a row masked out has statistics too (0, or anything): they meet zeros
      rstd_ahead = a.rstd[ahead];
      if (LAYER) mean_ahead = a.mean[ahead];
    }
    if (WIDE && !on) {   // the whole block: zeros
      Raw<T> z;
      z.clear();
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        if (JOIN) cols.write(a.grad_residual + off, i, z);
        if (!JOIN || a.grad_x) cols.write(a.grad_x + off, i, z);
      }
      if constexpr (VEC) {
        fetch(row_at(k + kRing), ring.stage, on_next);
        on_next = row_on(row_at(k + kRing + 1));
        ring.advance();
      } else {
        hold(ahead, on_ahead);
        on_next = row_on(row_at(k + 2));
      }
      on = on_ahead;
      rstd = rstd_ahead;
      mean = mean_ahead;
      continue;
    }
    F2 x[CPT][kPairs], gy[CPT][kPairs];
    Raw<T> gr[JOIN ? CPT : 1];
    if constexpr (VEC) {
      cp_async_wait<kRing - 1>();
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        ring.take(0, i, WIDE || on).get(x[i]);
        ring.take(1, i, WIDE || on).get(gy[i]);
        if constexpr (JOIN) gr[i] = ring.take(2, i, WIDE || on);
      }
      fetch(row_at(k + kRing), ring.stage, on_next);
      on_next = row_on(row_at(k + kRing + 1));
      ring.advance();
    } else {
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        held[0][i].get(x[i]);
        held[1][i].get(gy[i]);
        if constexpr (JOIN) gr[i] = held[2][i];
      }
      hold(ahead, on_ahead);
      on_next = row_on(row_at(k + 2));
    }
    if (!WIDE && !on) rstd = mean = 0.f;
    // with b = gy rstd:  dgamma += b x',  gx = b gamma,  grad = gx - [mean(gx)] - x' rstd mean(gx x'),  x' = x - mean
    F2 s0 = f2(0.f), s1 = f2(0.f);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      F2 g[kPairs];
      gamma[i].get(g);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        if (LAYER) {
          db[i][j] = add2(db[i][j], gy[i][j]);
          x[i][j] = add2(x[i][j], f2(-mean));   // columns past h: gy = gamma = 0
        }
        const F2 b = mul2(gy[i][j], f2(rstd));
        dg[i][j] = fma2(b, x[i][j], dg[i][j]);
        gy[i][j] = mul2(b, g[j]);
        if (LAYER) s0 = add2(s0, gy[i][j]);
        s1 = fma2(gy[i][j], x[i][j], s1);
      }
    }
    float s[kSums];
    s[kSums - 1] = parts(s1).x + parts(s1).y;
    if (LAYER) s[0] = parts(s0).x + parts(s0).y;
    row_sum(s, rt);
    const F2 m1 = f2(-s[kSums - 1] * a.inv_h * rstd * rstd), m0 = f2(LAYER ? -s[0] * a.inv_h : 0.f);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
#pragma unroll
      for (int j = 0; j < kPairs; ++j) gy[i][j] = fma2(x[i][j], m1, LAYER ? add2(gy[i][j], m0) : gy[i][j]);
      if constexpr (JOIN) {
        F2 g[kPairs];
        gr[i].get(g);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) gy[i][j] = add2(gy[i][j], g[j]);
        if (t < n) cols.write(a.grad_residual + off, i, gy[i]);
        if (!a.grad_x) continue;   // the same for all threads
        if (drop) {
          bool keep[kVec];
          keep_bits(ph.draw(static_cast<uint32_t>(i * rt.tpr + rt.tid), t), a.drop.below, keep);
          rt.template own_bits<VEC>(keep);
#pragma unroll
          for (int j = 0; j < kPairs; ++j) gy[i][j] = drop2(keep[2 * j], keep[2 * j + 1], gy[i][j], a.drop.scale);
        }
      }
      if (t < n) cols.write(a.grad_x + off, i, gy[i]);
    }
    on = on_ahead;
    rstd = rstd_ahead;
    mean = mean_ahead;
  }
  if constexpr (VEC) cp_async_wait<0>();

  // this block's share of the weight gradients
  float* out = a.part + static_cast<long long>(blockIdx.x) * kSums * a.h;
  auto share = [&](int which, int i, int j) {
    const F2 p = LAYER && which ? db[LAYER ? i : 0][j / 2] : dg[i][j / 2];
    return j & 1 ? parts(p).y : parts(p).x;
  };
  if constexpr (WIDE) {
#pragma unroll
    for (int which = 0; which < kSums; ++which)
#pragma unroll
      for (int i = 0; i < CPT; ++i)
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if (cols.col(i, j) < a.h) out[which * a.h + cols.col(i, j)] = share(which, i, j);
  } else {
    // the block's rows first: one slot after the other
    float* buf = reinterpret_cast<float*>(smem);   // [rows][tpr * CPT * 8]
    const int width = rt.tpr * CPT * kVec;
#pragma unroll
    for (int which = 0; which < kSums; ++which) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < CPT; ++i)
#pragma unroll
        for (int j = 0; j < kVec; ++j) buf[rt.slot * width + cols.col(i, j)] = share(which, i, j);
      __syncthreads();
      for (int c = threadIdx.x; c < a.h; c += blockDim.x) {
        float s = 0.f;
        for (int r = 0; r < rt.rows; ++r) s += buf[r * width + c];
        out[which * a.h + c] = s;
      }
    }
  }
}

// grad[c] (+)= sum over parts, in a fixed order: 1024 / COLS threads per column take every (1024 / COLS)-th part, then one in
// eight of them adds up eight of those sums, then one the rest.
constexpr int kReduceThreads = 1024;
template <int COLS>
__global__ void __launch_bounds__(kReduceThreads)
reduce_parts_kernel(const float* part, int parts, long long row_pitch, int h, int accumulate,
                    float* grad_gamma, float* grad_beta) {
  constexpr int kLanes = kReduceThreads / COLS, kFirst = kLanes / 8;
  wait_for_previous();
  const float* src = part + (blockIdx.y ? h : 0);
  float* dst = blockIdx.y ? grad_beta : grad_gamma;
  if (!dst) return;
  const int c = blockIdx.x * COLS + threadIdx.x;
  float s = 0.f;
  if (c < h)
#pragma unroll 8
    for (int p = threadIdx.y; p < parts; p += kLanes) s += src[p * row_pitch + c];
  __shared__ float sh[kLanes][COLS];
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y < kFirst) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sh[threadIdx.y * 8 + i][threadIdx.x];
  }
  __syncthreads();
  if (threadIdx.y < kFirst) sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y == 0 && c < h) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kFirst; ++i) t += sh[i][threadIdx.x];
    dst[c] = accumulate ? dst[c] + t : t;
  }
}

template <typename T, bool LAYER, bool JOIN>
__global__ void __launch_bounds__(kLongThreads)
norm_bwd_long_kernel(const NormBwdArgs<T> a) {
  __shared__ float2 sh[kWarp];
  const long long t = blockIdx.x;
  const bool vec = a.vec != 0;
  float z[kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) z[j] = 0.f;
  if (a.row_mask && a.row_mask[t] == 0) {
    for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
      if (!JOIN || a.grad_x) store_chunk(a.grad_x + t * a.h, col, a.h, vec, z);
      if (JOIN) store_chunk(a.grad_residual + t * a.h, col, a.h, vec, z);
    }
    return;
  }
  const float rstd = a.rstd[t];
  const float mean = LAYER ? a.mean[t] : 0.f;
  float s0 = 0.f, s1 = 0.f;
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float x[kVec], gy[kVec], g[kVec];
    load_chunk(a.x + t * a.h, col, a.h, vec, x);
    load_chunk(a.grad_y + t * a.h, col, a.h, vec, gy);
    load_chunk(a.gamma, col, a.h, vec, g);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const float gx = gy[j] * g[j];
      s0 += gx;
      s1 = fmaf(gx, (x[j] - mean) * rstd, s1);
    }
  }
  const float2 s = block_sum2(s0, s1, sh);
  const float m0 = LAYER ? s.x * a.inv_h : 0.f, m1 = s.y * a.inv_h;
  const bool drop = JOIN && a.drop.rng != nullptr;
  PhiloxState ph;
  if (drop) ph.load(a.drop.rng);
  for (int col = threadIdx.x * kVec; col < a.h; col += kLongThreads * kVec) {
    float x[kVec], gy[kVec], g[kVec];
    load_chunk(a.x + t * a.h, col, a.h, vec, x);
    load_chunk(a.grad_y + t * a.h, col, a.h, vec, gy);
    load_chunk(a.gamma, col, a.h, vec, g);
#pragma unroll
    for (int j = 0; j < kVec; ++j) gy[j] = (gy[j] * g[j] - m0 - (x[j] - mean) * rstd * m1) * rstd;
    if constexpr (JOIN) {
      if (a.grad_r) {
        load_chunk(a.grad_r + t * a.h, col, a.h, vec, g);
#pragma unroll
        for (int j = 0; j < kVec; ++j) gy[j] += g[j];
      }
      store_chunk(a.grad_residual + t * a.h, col, a.h, vec, gy);
      if (!a.grad_x) continue;
      if (drop) {
        bool keep[kVec];
        keep_bits(ph.draw(static_cast<uint32_t>(col / kVec), static_cast<uint32_t>(t)), a.drop.below, keep);
#pragma unroll
        for (int j = 0; j < kVec; ++j) gy[j] = drop_add(keep[j], gy[j], a.drop.scale, 0.f);
      }
    }
    store_chunk(a.grad_x + t * a.h, col, a.h, vec, gy);
  }
}

// Partial weight gradients of the long form: block (x: 256 columns, y: part), rows part, part + parts, ...
template <typename T, bool LAYER>
__global__ void __launch_bounds__(256)
norm_weight_long_kernel(const NormBwdArgs<T> a, int parts) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.h) return;
  float dg = 0.f, db = 0.f;
  for (long long t = blockIdx.y; t < a.n; t += parts) {
    if (a.row_mask && a.row_mask[t] == 0) continue;
    const float gy = to_float(a.grad_y[t * a.h + c]);
    const float x = to_float(a.x[t * a.h + c]);
    dg = fmaf(gy, (LAYER ? x - a.mean[t] : x) * a.rstd[t], dg);
    db += gy;
  }
  float* out = a.part + static_cast<long long>(blockIdx.y) * (LAYER ? 2 : 1) * a.h;
  out[c] = dg;
  if (LAYER) out[a.h + c] = db;
}

// Partial sums of dbeta for an RMS norm that has a beta, in a pass over grad_y of its own: block (x: 1024 columns, 8 per
// thread; y: part), rows part, part + parts, ...  Bound by that pass and its two launches: 65,536 x 2,048 bf16 144 -> 214 us,
// 5,001 x 1,003 21 -> 34.  Asked of the main kernel (a layer norm's form without means) it would cost every layer norm a
// branch: 4,000 x 12,001 bf16, whose registers spill, 384 -> 566 us.
constexpr int kBetaThreads = 128;
template <typename T>
__global__ void __launch_bounds__(kBetaThreads)
norm_beta_kernel(const NormBwdArgs<T> a, int parts) {
  const int col = (blockIdx.x * kBetaThreads + threadIdx.x) * kVec;
  if (col >= a.h) return;
  float sum[kVec] = {};
#pragma unroll 4
  for (long long t = blockIdx.y; t < a.n; t += parts) {
    if (a.row_mask && a.row_mask[t] == 0) continue;
    float gy[kVec];
    load_chunk(a.grad_y + t * a.h, col, a.h, a.vec != 0, gy);
#pragma unroll
    for (int j = 0; j < kVec; ++j) sum[j] += gy[j];
  }
  float* out = a.part + static_cast<long long>(blockIdx.y) * a.h;
#pragma unroll
  for (int j = 0; j < kVec; ++j)
    if (col + j < a.h) out[col + j] = sum[j];
}


template <typename T, int CPT, bool WIDE, int MAXT, bool VEC, bool LAYER, bool JOIN>
int launch(const NormBwdArgs<T>& a, int threads, int lanes, int* parts, cudaStream_t stream) {
  auto kernel = norm_bwd_kernel<T, CPT, WIDE, MAXT, VEC, LAYER, JOIN>;
  size_t smem = VEC ? static_cast<size_t>(threads) * CPT * ring_rows<T>(JOIN ? 3 : 2, CPT) * (JOIN ? 3 : 2) * sizeof(Raw<T>) : 0;
  if constexpr (!WIDE) {   // the block's rows are merged in the same memory at the end
    const size_t merge = static_cast<size_t>(threads) * CPT * kVec * sizeof(float);
    if (smem < merge) smem = merge;
  }
  static std::atomic<uint64_t> cached[64];
  const int per_sm = blocks_per_sm(kernel, threads, smem, a.h <= 2048 ? 8 : 4, cached);
  if (per_sm <= 0) return A3PO_ERR_CUDA;
  const int rows = WIDE ? 1 : threads / lanes;
  long long blocks = (a.n + rows - 1) / rows;
  long long most = static_cast<long long>(sm_count()) * per_sm;
  if (most > max_parts(a.h)) most = max_parts(a.h);
  if (blocks > most) blocks = most;
  *parts = static_cast<int>(blocks);
  const Turns turns{turn_shift((a.n + rows - 1) / rows, blocks)};
  A3PO_LAUNCH(kKNormBwd, stream, (kernel<<<static_cast<unsigned>(blocks), threads, smem, stream>>>(a, lanes, turns)));
  return after_launch();
}

// Threads by row length as in the forward.  The longest register forms spill (bytes a thread, bf16): 16-byte rows of 8,193 to
// 16,384 columns 52 (RMS) to 660 (layer norm of a join), element-wise rows of 4,097 to 8,192 columns up to 356 and of up to
// 16,384 columns 488 to 1,820.  Of the copy rate: 16,384 x 16,384 RMS 0.62 (400 us), layer 0.44, join 0.54, both 0.41; 8,192 x
// 6,001 0.12 to 0.27, 8,192 x 12,001 0.09 to 0.12.  The re-reading form, 8,192 x 20,000: 0.18 to 0.25.
template <typename T, bool VEC, bool LAYER, bool JOIN>
int by_length(const NormBwdArgs<T>& a, int* parts, cudaStream_t stream) {
  const int groups = (a.h + kVec - 1) / kVec;
  int lanes = 1;
  if (groups <= 32) {
    while (lanes < groups) lanes *= 2;
    return launch<T, 1, false, kNarrowThreads, VEC, LAYER, JOIN>(a, kNarrowThreads, lanes, parts, stream);
  }
  // 16-byte rows: two chunks per thread; element-wise rows: one as long as that fits, for more loads in flight
  if constexpr (VEC) {
    if (groups <= 64) return launch<T, 2, false, kNarrowThreads, VEC, LAYER, JOIN>(a, kNarrowThreads, kWarp, parts, stream);
    if (groups <= 2 * kNarrowThreads)
      return launch<T, 2, true, kNarrowThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up((groups + 1) / 2, kWarp)), 0, parts, stream);
  } else {
    if (groups <= kNarrowThreads)
      return launch<T, 1, true, kNarrowThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up(groups, kWarp)), 0, parts,
                                                                  stream);
    if (groups <= kWideThreads)
      return launch<T, 1, true, kWideThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up(groups, kWarp)), 0, parts, stream);
  }
  if (groups <= 2 * kWideThreads)
    return launch<T, 2, true, kWideThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up((groups + 1) / 2, kWarp)), 0, parts, stream);
  if (groups <= 4 * kWideThreads)
    return launch<T, 4, true, kWideThreads, VEC, LAYER, JOIN>(a, static_cast<int>(round_up((groups + 3) / 4, kWarp)), 0, parts, stream);
  A3PO_LAUNCH(kKNormBwd, stream, (norm_bwd_long_kernel<T, LAYER, JOIN>
                                      <<<static_cast<unsigned>(a.n), kLongThreads, 0, stream>>>(a)));
  A3PO_RETURN_IF(after_launch());
  *parts = a.n < 64 ? static_cast<int>(a.n) : 64;
  const dim3 grid(static_cast<unsigned>((a.h + 255) / 256), static_cast<unsigned>(*parts));
  A3PO_LAUNCH(kKNormBwd, stream, (norm_weight_long_kernel<T, LAYER><<<grid, 256, 0, stream>>>(a, *parts)));
  return after_launch();
}

// grad[c] (+)= the parts' sums: dgamma, and with `layer` dbeta behind it.
int reduce_parts(const float* part, int parts, int h, bool layer, int accumulate, float* grad_gamma, float* grad_beta,
                 cudaStream_t stream) {
  // 16 columns per block as long as that is a block per SM at most, else 32: 3,000 x 2,048, RMS norm, 14.4 us a call against 15.1,
  // 300 x 4,096 14.4 against 12.5 (inputs in L2).
  const bool fine = (h + 15) / 16 * (layer ? 2 : 1) <= sm_count();
  const int cols = fine ? 16 : 32;
  const dim3 grid(static_cast<unsigned>((h + cols - 1) / cols), layer ? 2u : 1u);
  A3PO_LAUNCH(kKNormBwd, stream, (launch_early(fine ? reduce_parts_kernel<16> : reduce_parts_kernel<32>, grid,
                                               dim3(cols, kReduceThreads / cols), 0, stream, 1, true, part, parts,
                                               static_cast<long long>(layer ? 2 : 1) * h, h, accumulate, grad_gamma,
                                               grad_beta)));
  return after_launch();
}

template <typename T, bool LAYER, bool JOIN>
int by_alignment(const NormBwdArgs<T>& a, float* grad_gamma, float* grad_beta, int accumulate, cudaStream_t stream) {
  int parts = 0;
  A3PO_RETURN_IF((a.vec ? by_length<T, true, LAYER, JOIN>(a, &parts, stream)
                        : by_length<T, false, LAYER, JOIN>(a, &parts, stream)));
  A3PO_RETURN_IF(reduce_parts(a.part, parts, a.h, LAYER, accumulate, grad_gamma, grad_beta, stream));
  if (LAYER || !grad_beta) return A3PO_OK;
  // a few blocks per SM; the workspace holds two sums of min(n, max_parts) rows
  const unsigned columns = static_cast<unsigned>((a.h + kBetaThreads * kVec - 1) / (kBetaThreads * kVec));
  long long want = (8ll * sm_count() + columns - 1) / columns;
  if (want > max_parts(a.h)) want = max_parts(a.h);
  if (want > a.n) want = a.n;
  parts = static_cast<int>(want);
  A3PO_LAUNCH(kKNormBwd, stream, (norm_beta_kernel<T><<<dim3(columns, static_cast<unsigned>(parts)), kBetaThreads, 0, stream>>>(
                                     a, parts)));
  A3PO_RETURN_IF(after_launch());
  return reduce_parts(a.part, parts, a.h, false, accumulate, grad_beta, nullptr, stream);
}
template <typename T>
int by_kind(const NormBwdArgs<T>& a, bool layer, bool join, float* gg, float* gb, int acc, cudaStream_t s) {
  if (layer) return join ? by_alignment<T, true, true>(a, gg, gb, acc, s) : by_alignment<T, true, false>(a, gg, gb, acc, s);
  return join ? by_alignment<T, false, true>(a, gg, gb, acc, s) : by_alignment<T, false, false>(a, gg, gb, acc, s);
}

}  // namespace

int launch_norm_bwd(const NormBwdArgs<float>& a, bool layer, bool join, float* grad_gamma, float* grad_beta,
                    int accumulate, cudaStream_t stream) {
  return by_kind(a, layer, join, grad_gamma, grad_beta, accumulate, stream);
}
int launch_norm_bwd(const NormBwdArgs<__nv_bfloat16>& a, bool layer, bool join, float* grad_gamma, float* grad_beta,
                    int accumulate, cudaStream_t stream) {
  return by_kind(a, layer, join, grad_gamma, grad_beta, accumulate, stream);
}

}  // namespace a3po
