// Layer norm, forward and backward (sm_100a).
//
// Bound by memory: each value is read once and written once, and a row stays in the registers of the threads that
// share it (OWN = 16 or 32 columns each) while its sums are taken.  A row's sums need barriers, during which its threads load
// nothing; so the next rows are already on their way into shared memory by asynchronous copies.  Each thread (where rows
// are not aligned, each warp) copies what it will itself read, so the copies need no barrier of their own.
#pragma once
#include "accept_rows.cuh"

namespace accept {

struct NormArgs {
  const void* x;
  const void* dy;        // backward
  const void* gamma;     // may be null
  const void* beta;      // forward, may be null
  void* y;               // forward
  float* mean_out;       // forward, may be null
  float* rstd_out;
  const float* mean;     // backward
  const float* rstd;
  void* dx;              // backward, may be null
  float* partials;       // backward: n_partials x 2 x cols, or null
  int joins;             // backward: the grid is one cluster, which adds up dgamma and dbeta itself
  float* dgamma;
  float* dbeta;
  uint64_t rows, ld_x, ld_y;
  uint32_t cols;
  uint32_t n_partials;
  uint32_t warps;        // that share a row
  float eps, inv_cols;
  int dtype_w;
  int whole_weights;     // gamma and beta start on 16-byte boundaries
};

extern __shared__ __align__(16) uint8_t norm_shared[];

// Forward.  The mean first, then the sum of the squared distances from it, so that an offset much larger than the spread
// costs no digits.  FULL: all columns of this warp exist (the warps of a group meet at the same barriers either way).
template <typename TX, typename TY, int V, bool FULL, int OWN, int L, int STAGES>
__device__ __forceinline__ void forward_rows(const NormArgs& a, const Group<L>& g, float (&slots)[2][16], uint32_t shared, uint32_t space, uint64_t first, uint32_t step) {
  const uint32_t t = g.t, shared_end = shared + STAGES * space;
  const Own<V, FULL, OWN, L> own(t, a.cols);
  bool ends_inside = false;
#pragma unroll
  for (int i = 0; i < OWN / V; ++i) ends_inside |= V > 2 && own.of(i) % V != 0;
  const TX* x = static_cast<const TX*>(a.x);
  const TX* end = x + (a.rows - 1) * a.ld_x + a.cols;
  const TX* row = x + first * a.ld_x;
  TY* out = static_cast<TY*>(a.y) + first * a.ld_y;
  const uint64_t stride_x = step * a.ld_x, stride_y = step * a.ld_y;
#pragma unroll
  for (int s = 0; s + 1 < STAGES; ++s) {
    if (first + (uint64_t)s * step < a.rows) start_row<TX, V, FULL, OWN, L>(shared + s * space, row + s * stride_x, a.cols, t, own, x, end);
    copy_commit();
  }
  Pair gamma[OWN / 2], beta[OWN / 2];
  load_weights<V, FULL, OWN, L>(a, a.gamma, own, 1.0f, t, gamma);
  load_weights<V, FULL, OWN, L>(a, a.beta, own, 0.0f, t, beta);
  uint32_t here = shared, ahead = shared + (STAGES - 1) * space;  // where this row lies, and where the one to start goes
  uint32_t left = (uint32_t)((a.rows - first + step - 1) / step);  // rows of this group from this one on
  float* mean_out = a.mean_out && t == 0 ? a.mean_out + first : nullptr;
  float* rstd_out = a.rstd_out && t == 0 ? a.rstd_out + first : nullptr;
  for (;;) {
    if (left > STAGES - 1) start_row<TX, V, FULL, OWN, L>(ahead, row + (STAGES - 1) * stride_x, a.cols, t, own, x, end);
    copy_commit();
    copy_wait<STAGES - 1>();
    if (V <= 2) __syncwarp(g.mask);  // other lanes of the warp have copied for this one
    Pair v[OWN / 2];
    take_row<TX, V, FULL, OWN, L>(here, row, t, own, v);
    Pair sums[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int i = 4; i < OWN / 2; ++i) sums[i % 4] = add2(sums[i % 4], v[i]);
    const Pair sum = add2(add2(sums[0], sums[1]), add2(sums[2], sums[3]));
    const float mean = g.sum(sum_of(sum), slots[0]) * a.inv_cols;
    Pair squares[2] = {both(0.0f), both(0.0f)};
#pragma unroll
    for (int i = 0; i < OWN / 2; ++i) {
      // a unit that does not exist stays zero; one that ends inside (one thread's) is masked value by value
      if (FULL || V > 2) v[i] = add2(v[i], both(own.of(2 * i / V) ? -mean : 0.0f));
      else v[i] = add2(v[i], pair_of(own.has(2 * i) ? -mean : 0.0f, own.has(2 * i + 1) ? -mean : 0.0f));
      if (!FULL && V > 2 && ends_inside) {
        const float2 f = split(v[i]);
        v[i] = pair_of(own.has(2 * i) ? f.x : 0.0f, own.has(2 * i + 1) ? f.y : 0.0f);
      }
      squares[i % 2] = fma2(v[i], v[i], squares[i % 2]);
    }
    squares[0] = add2(squares[0], squares[1]);
    const float rstd = rsqrtf(g.sum(sum_of(squares[0]), slots[1]) * a.inv_cols + a.eps);
#pragma unroll
    for (int i = 0; i < OWN / 2; ++i) v[i] = fma2(mul2(v[i], both(rstd)), gamma[i], beta[i]);
    store_row<TY, V, FULL, OWN, L>(out, t, own, v);
    if (mean_out) { st_c(mean_out, mean); mean_out += step; }
    if (rstd_out) { st_c(rstd_out, rstd); rstd_out += step; }
    if (--left == 0) break;
    row += stride_x;
    out += stride_y;
    ahead = here;
    here = here + space == shared_end ? shared : here + space;
  }
}

template <typename TX, typename TY, int V, int OWN, int L, int STAGES>
__global__ void __launch_bounds__(512) norm_forward_kernel(const NormArgs a) {
  __shared__ __align__(16) float slots[kMostGroups][2][16];
  const Group<L> g(a.warps);
  const uint32_t groups = blockDim.x / g.threads;
  const uint32_t space = row_space<TX>(V, OWN, L, a.warps);
  const uint32_t shared = (uint32_t)__cvta_generic_to_shared(norm_shared) + g.index * STAGES * space;
  const uint64_t first = (uint64_t)blockIdx.x * groups + g.index;
  const uint32_t step = gridDim.x * groups;
  const bool full = lanes_are_full<OWN, L>(g.t, a.cols);
  if (!full)
#pragma unroll
    for (int i = 0; i < STAGES; ++i) clear_row<TX, V, OWN, L>(shared + i * space, g.t, a.cols);
  if (L == 32 && a.warps > 1) {
    float* zero = &slots[g.index][0][0];
    for (uint32_t i = g.t; i < 32; i += g.threads) zero[i] = 0.0f;
    g.sync();
  }
  grid_dependency_handshake();
  if (first >= a.rows) return;
  if (full) forward_rows<TX, TY, V, true, OWN, L, STAGES>(a, g, slots[g.index % kMostGroups], shared, space, first, step);
  else forward_rows<TX, TY, V, false, OWN, L, STAGES>(a, g, slots[g.index % kMostGroups], shared, space, first, step);
}

// Backward.  dx needs two sums of a row, taken together; the gradients of gamma and beta are sums over the rows (SUMS),
// held in registers over all rows of a group, added up over the block's groups and joined by norm_join_kernel.
template <typename TX, typename TY, int V, bool FULL, int OWN, int L, int STAGES, bool SUMS>
__device__ __forceinline__ void backward_rows(const NormArgs& a, const Group<L>& g, float (&slots)[2][32], uint32_t shared, uint32_t space, uint32_t space_x,
                                              uint64_t first, uint32_t step, Pair (&dgamma)[SUMS ? OWN / 2 : 1], Pair (&dbeta)[SUMS ? OWN / 2 : 1]) {
  constexpr int kSums = SUMS ? OWN / 2 : 1;
  const uint32_t t = g.t, shared_end = shared + STAGES * space;
  const Own<V, FULL, OWN, L> own(t, a.cols);
  const TX* x = static_cast<const TX*>(a.x);
  const TY* dy = static_cast<const TY*>(a.dy);
  const TX* end_x = x + (a.rows - 1) * a.ld_x + a.cols;
  const TY* end_y = dy + (a.rows - 1) * a.ld_y + a.cols;
  Pair gamma[OWN / 2];
  const TX* row = x + first * a.ld_x;
  const TY* drow = dy + first * a.ld_y;
  TX* out = static_cast<TX*>(a.dx) + first * a.ld_x;
  const uint64_t stride_x = step * a.ld_x, stride_y = step * a.ld_y;
#pragma unroll
  for (int s = 0; s + 1 < STAGES; ++s) {
    if (first + (uint64_t)s * step < a.rows) {
      start_row<TX, V, FULL, OWN, L>(shared + s * space, row + s * stride_x, a.cols, t, own, x, end_x);
      start_row<TY, V, FULL, OWN, L>(shared + s * space + space_x, drow + s * stride_y, a.cols, t, own, dy, end_y);
    }
    copy_commit();
  }
  load_weights<V, FULL, OWN, L>(a, a.gamma, own, 1.0f, t, gamma);
  uint32_t here = shared, ahead = shared + (STAGES - 1) * space, turn = 0;
  uint32_t left = (uint32_t)((a.rows - first + step - 1) / step);
  const float* means = a.mean + first;
  const float* rstds = a.rstd + first;
  float mean_next = ld_c(means), rstd_next = ld_c(rstds);
  for (;;) {
    if (left > STAGES - 1) {
      start_row<TX, V, FULL, OWN, L>(ahead, row + (STAGES - 1) * stride_x, a.cols, t, own, x, end_x);
      start_row<TY, V, FULL, OWN, L>(ahead + space_x, drow + (STAGES - 1) * stride_y, a.cols, t, own, dy, end_y);
    }
    copy_commit();
    const float mean = mean_next, rstd = rstd_next;
    if (left > 1) { mean_next = ld_c(means += step); rstd_next = ld_c(rstds += step); }
    copy_wait<STAGES - 1>();
    if (V <= 2) __syncwarp(g.mask);  // other lanes of the warp have copied for this one
    Pair xhat[OWN / 2], h[OWN / 2];
    take_row<TX, V, FULL, OWN, L>(here, row, t, own, xhat);
    take_row<TY, V, FULL, OWN, L>(here + space_x, drow, t, own, h);
    Pair sum[2] = {both(0.0f), both(0.0f)}, along[2] = {both(0.0f), both(0.0f)};
#pragma unroll
    for (int i = 0; i < OWN / 2; ++i) {
      xhat[i] = mul2(add2(xhat[i], both(-mean)), both(rstd));
      // Zero in columns that do not exist: their x and dy are 0, but -mean rstd may pass the largest float where the row's own
      // xhat do not (a constant row of 2^120), and 0 times infinity would be NaN in the row's sum.  (Masked here: before the
      // multiplication, or in a branch for such rows alone, the fp32 kernels spill 180 bytes more.)
      if (!FULL) {
        const float2 f = split(xhat[i]);
        xhat[i] = pair_of(own.has(2 * i) ? f.x : 0.0f, own.has(2 * i + 1) ? f.y : 0.0f);
      }
      if (SUMS) {
        dbeta[i % kSums] = add2(dbeta[i % kSums], h[i]);
        dgamma[i % kSums] = fma2(h[i], xhat[i], dgamma[i % kSums]);
      }
      h[i] = mul2(h[i], gamma[i]);
      sum[i % 2] = add2(sum[i % 2], h[i]);
      along[i % 2] = fma2(h[i], xhat[i], along[i % 2]);
    }
    if (a.dx) {
      sum[0] = add2(sum[0], sum[1]);
      along[0] = add2(along[0], along[1]);
      const float2 s = g.sum_two(make_float2(sum_of(sum[0]), sum_of(along[0])), slots[turn]);
      turn ^= 1;
      const Pair less = both(-s.x * a.inv_cols), slope = both(-s.y * a.inv_cols);
#pragma unroll
      for (int i = 0; i < OWN / 2; ++i) h[i] = mul2(fma2(xhat[i], slope, add2(h[i], less)), both(rstd));
      store_row<TX, V, FULL, OWN, L>(out, t, own, h);
    } else if (V <= 2) {
      __syncwarp(g.mask);  // the row has been read: its place is free
    }
    if (--left == 0) break;
    row += stride_x;
    drow += stride_y;
    out += stride_x;
    ahead = here;
    here = here + space == shared_end ? shared : here + space;
  }
}

template <typename TX, typename TY, int V, int OWN, int L, int STAGES, bool SUMS>
__global__ void __launch_bounds__(512) norm_backward_kernel(const NormArgs a) {
  constexpr int kSums = SUMS ? OWN / 2 : 1;
  __shared__ __align__(16) float slots[kMostGroups][2][32];
  const Group<L> g(a.warps);
  const uint32_t groups = blockDim.x / g.threads, t = g.t, threads = g.threads;
  const uint32_t space_x = row_space<TX>(V, OWN, L, a.warps), space = space_x + row_space<TY>(V, OWN, L, a.warps);
  const uint32_t shared = (uint32_t)__cvta_generic_to_shared(norm_shared) + g.index * STAGES * space;
  const uint64_t first = (uint64_t)blockIdx.x * groups + g.index;
  const uint32_t step = gridDim.x * groups;
  const bool full = lanes_are_full<OWN, L>(t, a.cols);
  if (!full) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      clear_row<TX, V, OWN, L>(shared + i * space, t, a.cols);
      clear_row<TY, V, OWN, L>(shared + i * space + space_x, t, a.cols);
    }
  }
  if (L == 32 && a.warps > 1) {
    float* zero = &slots[g.index][0][0];
    for (uint32_t i = t; i < 64; i += threads) zero[i] = 0.0f;
    g.sync();
  }
  grid_dependency_handshake();
  Pair dgamma[kSums], dbeta[kSums];
#pragma unroll
  for (int i = 0; i < kSums; ++i) dgamma[i] = dbeta[i] = both(0.0f);
  if (first < a.rows) {
    if (full) backward_rows<TX, TY, V, true, OWN, L, STAGES, SUMS>(a, g, slots[g.index % kMostGroups], shared, space, space_x, first, step, dgamma, dbeta);
    else backward_rows<TX, TY, V, false, OWN, L, STAGES, SUMS>(a, g, slots[g.index % kMostGroups], shared, space, space_x, first, step, dgamma, dbeta);
  }
  if (!SUMS || !(a.partials || (a.joins && (a.dgamma || a.dbeta)))) return;
  float* out = a.partials + (uint64_t)blockIdx.x * 2 * a.cols;
  if (groups == 1 && !a.joins) {
    if (V > 2 && a.cols % 4 == 0) {
#pragma unroll
      for (int i = 0; i < OWN; i += 4) {
        const uint32_t c = column_of<V, OWN, L>(t, i);
        const float2 d0 = split(dgamma[i / 2 % kSums]), d1 = split(dgamma[(i / 2 + 1) % kSums]);
        const float2 e0 = split(dbeta[i / 2 % kSums]), e1 = split(dbeta[(i / 2 + 1) % kSums]);
        if (c < a.cols) {
          st_c(reinterpret_cast<float4*>(out + c), make_float4(d0.x, d0.y, d1.x, d1.y));
          st_c(reinterpret_cast<float4*>(out + a.cols + c), make_float4(e0.x, e0.y, e1.x, e1.y));
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const uint32_t c = column_of<V, OWN, L>(t, i);
      const float2 d = split(dgamma[i / 2 % kSums]), e = split(dbeta[i / 2 % kSums]);
      if (c < a.cols) { st_c(out + c, i % 2 ? d.y : d.x); st_c(out + a.cols + c, i % 2 ? e.y : e.x); }
    }
    return;
  }
  // the groups of the block lay their sums side by side in shared memory; all threads add them up, group after group
  const uint32_t width = a.warps * L * OWN;
  float* sums = reinterpret_cast<float*>(norm_shared);
  copy_wait<0>();
  __syncthreads();
  float* mine = sums + (uint64_t)g.index * 2 * width;
#pragma unroll
  for (int i = 0; i < OWN / 2; ++i) {
    const uint32_t c = column_of<V, OWN, L>(t, 2 * i);
    if (V > 1) {
      *reinterpret_cast<Pair*>(mine + c) = dgamma[i % kSums];
      *reinterpret_cast<Pair*>(mine + width + c) = dbeta[i % kSums];
    } else {
      const float2 d = split(dgamma[i % kSums]), e = split(dbeta[i % kSums]);
      mine[c] = d.x;
      mine[c + L] = d.y;
      mine[width + c] = e.x;
      mine[width + c + L] = e.y;
    }
  }
  __syncthreads();
#pragma unroll 2
  for (uint32_t c = threadIdx.x; c < a.cols && groups > 1; c += blockDim.x) {
    float d = 0.0f, e = 0.0f;
#pragma unroll 4
    for (uint32_t k = 0; k < groups; ++k) {
      d += sums[(uint64_t)k * 2 * width + c];
      e += sums[(uint64_t)k * 2 * width + width + c];
    }
    if (a.joins) {
      sums[c] = d;
      sums[width + c] = e;
    } else {
      st_c(out + c, d);
      st_c(out + a.cols + c, e);
    }
  }
  if (!a.joins) return;
  // few rows: the blocks of the one cluster take the columns in turn and add up what each of them has, in their order
  cluster_sync();
  const uint32_t from = smem_address(sums);
#pragma unroll 2
  for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < 2 * a.cols; i += gridDim.x * blockDim.x) {
    const uint32_t which = i >= a.cols ? 1 : 0, c = i - which * a.cols, at = from + 4 * (which * width + c);
    float v[8], d = 0.0f;
#pragma unroll
    for (uint32_t r = 0; r < 8; ++r) v[r] = r < gridDim.x ? ld_cluster_one(address_in(at, r)) : 0.0f;
#pragma unroll
    for (uint32_t r = 0; r < 8; ++r) d += v[r];
    float* result = which ? a.dbeta : a.dgamma;
    if (result) st_c(result + c, d);
  }
  cluster_sync();  // no block leaves while others read its sums
}

// Rows longer than the registers of a block: the same formulas, each row read again for each of its sums.
__device__ __forceinline__ float block_sum(float v, float* slot) {
  v = warp_sum(v);
  const uint32_t warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) slot[threadIdx.x >> 5] = v;
  __syncthreads();
  return warp_sum(lane < warps ? slot[lane] : 0.0f);
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(1024) norm_forward_long_kernel(const NormArgs a) {
  __shared__ float slots[2][32];
  grid_dependency_handshake();
  for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const TX* row = static_cast<const TX*>(a.x) + r * a.ld_x;
    TY* out = static_cast<TY*>(a.y) + r * a.ld_y;
    float sum = 0.0f, squares = 0.0f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) sum += to_float(ld_c(row + c));
    const float mean = block_sum(sum, slots[0]) * a.inv_cols;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float d = to_float(ld_c(row + c)) - mean;
      squares = fmaf(d, d, squares);
    }
    const float rstd = 1.0f / sqrtf(block_sum(squares, slots[1]) * a.inv_cols + a.eps);
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float g = weight_at(a.gamma, a.dtype_w, 1.0f, c), b = weight_at(a.beta, a.dtype_w, 0.0f, c);
      st_c(out + c, from_float<TY>(fmaf((to_float(ld_c(row + c)) - mean) * rstd, g, b)));
    }
    if (threadIdx.x == 0 && a.mean_out) st_c(a.mean_out + r, mean);
    if (threadIdx.x == 0 && a.rstd_out) st_c(a.rstd_out + r, rstd);
  }
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(1024) norm_backward_long_kernel(const NormArgs a) {
  __shared__ float slots[2][2][32];
  grid_dependency_handshake();
  int turn = 0;
  for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const TX* row = static_cast<const TX*>(a.x) + r * a.ld_x;
    const TY* drow = static_cast<const TY*>(a.dy) + r * a.ld_y;
    TX* out = static_cast<TX*>(a.dx) + r * a.ld_x;
    const float mean = ld_c(a.mean + r), rstd = ld_c(a.rstd + r);
    float sum = 0.0f, along = 0.0f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float h = to_float(ld_c(drow + c)) * weight_at(a.gamma, a.dtype_w, 1.0f, c);
      sum += h;
      along = fmaf(h, (to_float(ld_c(row + c)) - mean) * rstd, along);
    }
    sum = block_sum(sum, slots[turn][0]) * a.inv_cols;
    along = block_sum(along, slots[turn][1]) * a.inv_cols;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float h = to_float(ld_c(drow + c)) * weight_at(a.gamma, a.dtype_w, 1.0f, c);
      st_c(out + c, from_float<TX>(rstd * (h - sum - (to_float(ld_c(row + c)) - mean) * rstd * along)));
    }
  }
}

// C neighbouring values at p, in fp32; one read where C = 4.
template <typename T, int C>
__device__ __forceinline__ void ld_neighbours(const T* p, float (&v)[C]) {
  if constexpr (C == 1) {
    v[0] = to_float(ld_c(p));
  } else if constexpr (sizeof(T) == 4) {
    const float4 f = ld_c(reinterpret_cast<const float4*>(p));
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
    const uint2 w = ld_c(reinterpret_cast<const uint2*>(p));
    const float2 lo = split(word_to_pair<T>(w.x)), hi = split(word_to_pair<T>(w.y));
    v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
  }
}

// Sums over the rows where the pass over dx does not hold them (rows of more than 8192 values): 32 C columns a block (C = 4
// where rows start on 16-byte boundaries and their length divides by 4), the rows of its slab (blockIdx.y) dealt over
// eight warps, several rows on their way for each.  With one slab the sums are the results.
template <typename TX, typename TY, int C>
__global__ void __launch_bounds__(256) norm_column_sums_kernel(const NormArgs a) {
  __shared__ float part[2][8][32 * C + 1];
  constexpr int kAtOnce = C == 1 ? 8 : 4;
  grid_dependency_handshake();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = ((uint64_t)blockIdx.x * 32 + lane) * C;
  float dgamma[C], dbeta[C];
#pragma unroll
  for (int k = 0; k < C; ++k) dgamma[k] = dbeta[k] = 0.0f;
  if (c < a.cols) {
    const TX* x = static_cast<const TX*>(a.x) + c;
    const TY* dy = static_cast<const TY*>(a.dy) + c;
    const uint64_t step = 8ull * gridDim.y;
#pragma unroll 1
    for (uint64_t r = blockIdx.y * 8 + warp; r < a.rows; r += kAtOnce * step) {
      float u[kAtOnce][C], v[kAtOnce][C], mean[kAtOnce], rstd[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const uint64_t row = r + j * step;
        mean[j] = rstd[j] = 0.0f;
#pragma unroll
        for (int k = 0; k < C; ++k) u[j][k] = v[j][k] = 0.0f;
        if (row < a.rows) {
          ld_neighbours<TY, C>(dy + row * a.ld_y, u[j]);
          ld_neighbours<TX, C>(x + row * a.ld_x, v[j]);
          mean[j] = ld_c(a.mean + row);
          rstd[j] = ld_c(a.rstd + row);
        }
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
        for (int k = 0; k < C; ++k) {
          dbeta[k] += u[j][k];
          dgamma[k] = fmaf(u[j][k], (v[j][k] - mean[j]) * rstd[j], dgamma[k]);
        }
    }
  }
#pragma unroll
  for (int k = 0; k < C; ++k) {
    part[0][warp][lane * C + k] = dgamma[k];
    part[1][warp][lane * C + k] = dbeta[k];
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < 64 * C; i += 256) {
    const uint32_t which = i / (32 * C), at = i - which * (32 * C);
    const uint64_t col = (uint64_t)blockIdx.x * (32 * C) + at;
    if (col >= a.cols) continue;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[which][w][at];
    float* out = gridDim.y > 1 ? a.partials + (2ull * blockIdx.y + which) * a.cols : which == 0 ? a.dgamma : a.dbeta;
    if (out) st_c(out + col, s);
  }
}

// dgamma and dbeta from the blocks' partial sums: 32 columns a block, the partials dealt over its sixteen warps, all of a
// warp's loads on their way at once, and added in a fixed order.
constexpr int kJoinWarps = 16;
__global__ void __launch_bounds__(32 * kJoinWarps) norm_join_kernel(const NormArgs a) {
  __shared__ float part[kJoinWarps][33];
  grid_dependency_handshake();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;  // over dgamma, then dbeta
  const uint64_t width = 2ull * a.cols;
  float s = 0.0f;
  if (c < width) {
    const float* p = a.partials + c;
    constexpr int kAtOnce = 10;  // 148 blocks over 16 warps
    for (uint32_t i = warp; i < a.n_partials; i += kAtOnce * kJoinWarps) {
      float v[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) v[j] = i + j * kJoinWarps < a.n_partials ? ld_c(p + (uint64_t)(i + j * kJoinWarps) * width) : 0.0f;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) s += v[j];
    }
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < width) {
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) s += part[w][lane];
    float* out = c < a.cols ? a.dgamma : a.dbeta;
    if (out) st_c(out + (c < a.cols ? c : c - a.cols), s);
  }
}

}  // namespace accept
