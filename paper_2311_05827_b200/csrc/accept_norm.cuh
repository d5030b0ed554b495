// Layer norm, forward and backward (sm_100a).
//
// Bound by memory: each value is read once and written once, and a row stays in the registers of the threads that
// share it (16 columns each) while its sums are taken.  A row's sums need barriers, during which its threads load
// nothing; so the next rows are already on their way into shared memory by asynchronous copies.  Each thread copies what it
// will itself read, so the copies need no barrier of their own.
#pragma once
#include "accept_types.cuh"

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
  float* dgamma;
  float* dbeta;
  uint64_t rows, ld_x, ld_y;
  uint32_t cols;
  uint32_t n_partials;
  uint32_t warps;        // that share a row
  uint32_t stages;       // rows of a group in shared memory
  float eps, inv_cols;
  int dtype_w;
  int whole_weights;     // gamma and beta start on 16-byte boundaries
};

constexpr int kOwn = 16;  // columns of a row that a thread holds

// How the columns of a row lie over the threads that share it: units of V neighbours, thread t holding units t, t + T, ...
// V = 8 where both tensors are 16-bit types, 4 where one is fp32 (16 bytes at most for a thread, neighbours side by side),
// 1 where rows do not start on 16-byte boundaries.
template <int V>
__device__ __forceinline__ uint32_t column_of(uint32_t t, uint32_t threads, int own) {
  return V * (t + own / V * threads) + own % V;
}

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, uint32_t bytes) {  // the rest of BYTES is zero
  if (!bounds_ok(src, bytes, false)) bytes = 0;
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait(uint32_t pending) {  // all but the last `pending` groups have landed
  switch (pending) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
  }
}

// Bytes of shared memory that a row of T takes for `threads` threads (V = 1: the 16-byte pieces that hold it).
template <typename T>
__host__ __device__ constexpr uint32_t row_space(int v, uint32_t threads, uint32_t cols) {
  return v > 1 ? threads * kOwn * (uint32_t)sizeof(T) : (cols * (uint32_t)sizeof(T) + 30) / 16 * 16;
}

// Starts the copies of a row into `dst`.  `begin` and `end` bound the bytes of the matrix.
template <typename T, int V>
__device__ __forceinline__ void start_row(uint32_t dst, const T* row, uint32_t cols, uint32_t t, uint32_t threads, const T* begin, const T* end) {
  if (V > 1) {
    constexpr int kBytes = V * (int)sizeof(T) < 16 ? 8 : 16;
    constexpr int kCopies = V * (int)sizeof(T) / kBytes;  // of a unit: one, but for V = 8 of fp32, which does not occur
    static_assert(kCopies == 1 || V == 1, "a unit is one copy");
#pragma unroll
    for (int i = 0; i < kOwn / V; ++i) {
      const uint32_t c = V * (t + i * threads);
      const uint32_t bytes = c < cols ? min(cols - c, (uint32_t)V) * (uint32_t)sizeof(T) : 0;
      copy_async<kBytes>(dst + (i * threads + t) * kBytes, row + (bytes ? c : 0), bytes);
    }
  } else {
    // the 16-byte pieces that hold the row; what lies outside the matrix is not read
    const uintptr_t from = reinterpret_cast<uintptr_t>(row) & ~(uintptr_t)15, to = reinterpret_cast<uintptr_t>(row + cols);
    for (uint32_t i = t; from + 16ull * i < to; i += threads) {
      const uintptr_t at = from + 16ull * i;
      if (at >= reinterpret_cast<uintptr_t>(begin)) {
        const uint64_t left = reinterpret_cast<uintptr_t>(end) - at;
        copy_async<16>(dst + 16 * i, reinterpret_cast<const void*>(at), left < 16 ? (uint32_t)left : 16u);
      } else {  // the matrix starts inside this piece
        for (const T* p = begin; reinterpret_cast<uintptr_t>(p) < at + 16 && p < end; ++p) {
          const T v = ld_c(p);
          const uint32_t to_byte = dst + 16 * i + (uint32_t)(reinterpret_cast<uintptr_t>(p) - at);
          if (sizeof(T) == 4) {
            uint32_t w;
            memcpy(&w, &v, sizeof(T));
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(to_byte), "r"(w) : "memory");
          } else {
            uint16_t w;
            memcpy(&w, &v, 2);
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(to_byte), "h"(w) : "memory");
          }
        }
      }
    }
  }
}

// Takes a row that has landed at `src` into registers; columns past the last are zero.
template <typename T, int V>
__device__ __forceinline__ void take_row(const uint8_t* src, const T* row, uint32_t cols, uint32_t t, uint32_t threads, float (&v)[kOwn]) {
  if (V > 1) {
#pragma unroll
    for (int i = 0; i < kOwn / V; ++i) {
      T w[V];
      if (V * sizeof(T) == 16) {
        const uint4 raw = *reinterpret_cast<const uint4*>(src + (i * threads + t) * 16);
        memcpy(w, &raw, sizeof(w));
      } else {
        const uint2 raw = *reinterpret_cast<const uint2*>(src + (i * threads + t) * 8);
        memcpy(w, &raw, sizeof(w));
      }
#pragma unroll
      for (int j = 0; j < V; ++j) v[V * i + j] = to_float(w[j]);
    }
  } else {
    const T* p = reinterpret_cast<const T*>(src + (reinterpret_cast<uintptr_t>(row) & 15));
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const uint32_t c = t + i * threads;
      v[i] = c < cols ? to_float(p[c]) : 0.0f;
    }
  }
}

template <typename T, int V>
__device__ __forceinline__ void store_row(T* row, uint32_t cols, uint32_t t, uint32_t threads, const float (&v)[kOwn]) {
#pragma unroll
  for (int i = 0; i < kOwn / V; ++i) {
    const uint32_t c = V * (t + i * threads);
    if (V > 1 && c + V <= cols) {
      if (V * sizeof(T) == 16) {
        T w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = from_float<T>(v[V * i + j]);
        uint4 raw;
        memcpy(&raw, w, 16);
        if (bounds_ok(row + c, 16, true)) __stcs(reinterpret_cast<uint4*>(row + c), raw);
      } else {
        T w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = from_float<T>(v[V * i + j]);
        uint2 raw;
        memcpy(&raw, w, 8);
        if (bounds_ok(row + c, 8, true)) __stcs(reinterpret_cast<uint2*>(row + c), raw);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (c + j < cols) st_c(row + c + j, from_float<T>(v[V * i + j]));
    }
  }
}

// Value c of gamma or beta, in whichever type it has.
__device__ __forceinline__ float weight_at(const void* w, int dtype, float absent, uint32_t c) {
  if (!w) return absent;
  if (dtype == kF32) return ld_c(static_cast<const float*>(w) + c);
  if (dtype == kBf16) return to_float(ld_c(static_cast<const __nv_bfloat16*>(w) + c));
  return to_float(ld_c(static_cast<const __half*>(w) + c));
}

// gamma or beta for this thread's columns: read once for all rows that it takes.
template <int V>
__device__ __forceinline__ void load_weights(const NormArgs& a, const void* w, float absent, uint32_t t, uint32_t threads, float (&v)[kOwn]) {
#pragma unroll
  for (int i = 0; i < kOwn; i += V) {
    const uint32_t c = column_of<V>(t, threads, i);
    if (V > 1 && w && a.whole_weights && c + V <= a.cols) {
      if (a.dtype_w == kF32) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
          const float4 f = ld_c(reinterpret_cast<const float4*>(static_cast<const float*>(w) + c + j));
          v[i + j] = f.x; v[(i + j + 1) % kOwn] = f.y; v[(i + j + 2) % kOwn] = f.z; v[(i + j + 3) % kOwn] = f.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
          const uint2 raw = ld_c(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(w) + c + j));
          if (a.dtype_w == kBf16) {
            __nv_bfloat16 h[4];
            memcpy(h, &raw, 8);
#pragma unroll
            for (int l = 0; l < 4; ++l) v[(i + j + l) % kOwn] = to_float(h[l]);
          } else {
            __half h[4];
            memcpy(h, &raw, 8);
#pragma unroll
            for (int l = 0; l < 4; ++l) v[(i + j + l) % kOwn] = to_float(h[l]);
          }
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[i + j] = c + j < a.cols ? weight_at(w, a.dtype_w, absent, c + j) : absent;
    }
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// The threads that share a row: `warps` warps, one of the block's groups.
struct Group {
  uint32_t index, warps, threads, t;
  __device__ __forceinline__ explicit Group(uint32_t warps_) : warps(warps_), threads(32 * warps_) {
    index = (threadIdx.x >> 5) / warps;
    t = threadIdx.x - index * threads;
  }
  __device__ __forceinline__ void sync() const {
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(threads) : "memory");
  }
  // Sum over the group; `slot` holds a value of each warp and is used in turn with another (a barrier lies between).
  __device__ __forceinline__ float sum(float v, float* slot) const {
    v = warp_sum(v);
    if (warps == 1) return v;
    if ((t & 31) == 0) slot[t >> 5] = v;
    sync();
    return warp_sum((t & 31) < warps ? slot[t & 31] : 0.0f);
  }
};

extern __shared__ __align__(16) uint8_t norm_shared[];

// Forward.  The mean first, then the sum of the squared distances from it, so that an offset much larger than the spread
// costs no digits.
template <typename TX, typename TY, int V, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) norm_forward_kernel(const NormArgs a) {
  __shared__ float slots[2][32];
  const Group g(a.warps);
  const uint32_t groups = blockDim.x / g.threads, t = g.t, threads = g.threads;
  const uint32_t space = row_space<TX>(V, threads, a.cols);
  const uint32_t offset = g.index * a.stages * space, shared = (uint32_t)__cvta_generic_to_shared(norm_shared) + offset;
  const TX* x = static_cast<const TX*>(a.x);
  const TX* end = x + (a.rows - 1) * a.ld_x + a.cols;
  const uint64_t first = (uint64_t)blockIdx.x * groups + g.index, step = (uint64_t)gridDim.x * groups;
  grid_dependency_handshake();
  for (uint32_t s = 0; s + 1 < a.stages; ++s) {
    const uint64_t r = first + s * step;
    if (r < a.rows) start_row<TX, V>(shared + s * space, x + r * a.ld_x, a.cols, t, threads, x, end);
    copy_commit();
  }
  float gamma[kOwn], beta[kOwn];
  load_weights<V>(a, a.gamma, 1.0f, t, threads, gamma);
  load_weights<V>(a, a.beta, 0.0f, t, threads, beta);
  float* slot = slots[0] + g.index * a.warps;
  uint32_t stage = 0;
  for (uint64_t r = first; r < a.rows; r += step) {
    const uint64_t ahead = r + (a.stages - 1) * step;
    const uint32_t into = stage == 0 ? a.stages - 1 : stage - 1;  // where the row before lay (or this one, with one stage)
    if (ahead < a.rows) start_row<TX, V>(shared + into * space, x + ahead * a.ld_x, a.cols, t, threads, x, end);
    copy_commit();
    copy_wait(a.stages - 1);
    if (V == 1) g.sync();
    float v[kOwn];
    take_row<TX, V>(norm_shared + offset + stage * space, x + r * a.ld_x, a.cols, t, threads, v);
    stage = stage + 1 == a.stages ? 0 : stage + 1;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) sum += v[i];
    const float mean = g.sum(sum, slot) * a.inv_cols;
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      v[i] = column_of<V>(t, threads, i) < a.cols ? v[i] - mean : 0.0f;
      squares = fmaf(v[i], v[i], squares);
    }
    const float rstd = 1.0f / sqrtf(g.sum(squares, slot + 32) * a.inv_cols + a.eps);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) v[i] = fmaf(v[i] * rstd, gamma[i], beta[i]);
    store_row<TY, V>(static_cast<TY*>(a.y) + r * a.ld_y, a.cols, t, threads, v);
    if (t == 0 && a.mean_out) st_c(a.mean_out + r, mean);
    if (t == 0 && a.rstd_out) st_c(a.rstd_out + r, rstd);
  }
}

// Backward.  dx needs two sums of a row, taken together; the gradients of gamma and beta are sums over the rows (SUMS),
// held in registers over all rows of a group, added up over the block's groups and joined by norm_join_kernel.
template <typename TX, typename TY, int V, bool SUMS, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) norm_backward_kernel(const NormArgs a) {
  __shared__ float slots[4][32];
  const Group g(a.warps);
  const uint32_t groups = blockDim.x / g.threads, t = g.t, threads = g.threads;
  const uint32_t space_x = row_space<TX>(V, threads, a.cols), space = space_x + row_space<TY>(V, threads, a.cols);
  const uint32_t offset = g.index * a.stages * space, shared = (uint32_t)__cvta_generic_to_shared(norm_shared) + offset;
  const TX* x = static_cast<const TX*>(a.x);
  const TY* dy = static_cast<const TY*>(a.dy);
  const TX* end_x = x + (a.rows - 1) * a.ld_x + a.cols;
  const TY* end_y = dy + (a.rows - 1) * a.ld_y + a.cols;
  const uint64_t first = (uint64_t)blockIdx.x * groups + g.index, step = (uint64_t)gridDim.x * groups;
  grid_dependency_handshake();
  for (uint32_t s = 0; s + 1 < a.stages; ++s) {
    const uint64_t r = first + s * step;
    if (r < a.rows) {
      start_row<TX, V>(shared + s * space, x + r * a.ld_x, a.cols, t, threads, x, end_x);
      start_row<TY, V>(shared + s * space + space_x, dy + r * a.ld_y, a.cols, t, threads, dy, end_y);
    }
    copy_commit();
  }
  float gamma[kOwn], dgamma[SUMS ? kOwn : 1], dbeta[SUMS ? kOwn : 1];
  load_weights<V>(a, a.gamma, 1.0f, t, threads, gamma);
#pragma unroll
  for (int i = 0; i < (SUMS ? kOwn : 1); ++i) dgamma[i] = dbeta[i] = 0.0f;
  float* slot = slots[0] + g.index * a.warps;
  uint32_t stage = 0;
  for (uint64_t r = first; r < a.rows; r += step) {
    const uint64_t ahead = r + (a.stages - 1) * step;
    const uint32_t into = stage == 0 ? a.stages - 1 : stage - 1;
    const float mean = ld_c(a.mean + r), rstd = ld_c(a.rstd + r);
    if (ahead < a.rows) {
      start_row<TX, V>(shared + into * space, x + ahead * a.ld_x, a.cols, t, threads, x, end_x);
      start_row<TY, V>(shared + into * space + space_x, dy + ahead * a.ld_y, a.cols, t, threads, dy, end_y);
    }
    copy_commit();
    copy_wait(a.stages - 1);
    if (V == 1) g.sync();
    float xhat[kOwn], h[kOwn];
    const uint8_t* landed = norm_shared + offset + stage * space;
    take_row<TX, V>(landed, x + r * a.ld_x, a.cols, t, threads, xhat);
    take_row<TY, V>(landed + space_x, dy + r * a.ld_y, a.cols, t, threads, h);
    stage = stage + 1 == a.stages ? 0 : stage + 1;
    float sum = 0.0f, along = 0.0f;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      xhat[i] = (xhat[i] - mean) * rstd;  // columns past the last: dy = 0, so what stands here counts nowhere
      if (SUMS) {
        dbeta[i % kOwn] += h[i];
        dgamma[i % kOwn] = fmaf(h[i], xhat[i], dgamma[i % kOwn]);
      }
      h[i] *= gamma[i];
      sum += h[i];
      along = fmaf(h[i], xhat[i], along);
    }
    if (!a.dx) {
      if (V == 1) g.sync();  // the row has been read: its place is free
      continue;
    }
    // both sums with one barrier; the two pairs of slots are used in turn
    sum = warp_sum(sum);
    along = warp_sum(along);
    if (a.warps > 1) {
      const uint32_t lane = t & 31;
      if (lane == 0) { slot[t >> 5] = sum; slot[32 + (t >> 5)] = along; }
      g.sync();
      sum = warp_sum(lane < a.warps ? slot[lane] : 0.0f);
      along = warp_sum(lane < a.warps ? slot[32 + lane] : 0.0f);
      slot += slot >= slots[2] ? -64 : 64;
    }
    sum *= a.inv_cols;
    along *= a.inv_cols;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) h[i] = rstd * (h[i] - sum - xhat[i] * along);
    store_row<TX, V>(static_cast<TX*>(a.dx) + r * a.ld_x, a.cols, t, threads, h);
  }
  if (!SUMS || !a.partials) return;
  float* out = a.partials + (uint64_t)blockIdx.x * 2 * a.cols;
  if (groups > 1) {  // the block's groups add up their columns one after the other
    float* sums = reinterpret_cast<float*>(norm_shared);
    copy_wait(0);
    __syncthreads();
    for (uint32_t k = 0; k < groups; ++k) {
      if (g.index == k) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          float* p = sums + i * threads + t;  // a place of its own for each of the thread's columns
          float* q = p + kOwn * threads;
          dgamma[i % kOwn] = k ? *p + dgamma[i % kOwn] : dgamma[i % kOwn];
          dbeta[i % kOwn] = k ? *q + dbeta[i % kOwn] : dbeta[i % kOwn];
          *p = dgamma[i % kOwn];
          *q = dbeta[i % kOwn];
        }
      }
      __syncthreads();
    }
    if (g.index + 1 != groups) return;
  }
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const uint32_t c = column_of<V>(t, threads, i);
    if (c < a.cols) { st_c(out + c, dgamma[i % kOwn]); st_c(out + a.cols + c, dbeta[i % kOwn]); }
  }
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

// Sums over the rows where the pass over dx does not hold them (rows of more than 8192 values): one column for
// each thread; blockIdx.y takes every gridDim.y-th row into its own partial, eight rows in flight.
template <typename TX, typename TY>
__global__ void __launch_bounds__(128) norm_column_sums_kernel(const NormArgs a) {
  grid_dependency_handshake();
  const uint32_t c = blockIdx.x * 128 + threadIdx.x;
  if (c >= a.cols) return;
  float dgamma = 0.0f, dbeta = 0.0f;
#pragma unroll 8
  for (uint64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const float dy = to_float(ld_c(static_cast<const TY*>(a.dy) + r * a.ld_y + c));
    dbeta += dy;
    dgamma = fmaf(dy, (to_float(ld_c(static_cast<const TX*>(a.x) + r * a.ld_x + c)) - ld_c(a.mean + r)) * ld_c(a.rstd + r), dgamma);
  }
  float* out = a.partials + (uint64_t)blockIdx.y * 2 * a.cols;
  st_c(out + c, dgamma);
  st_c(out + a.cols + c, dbeta);
}

// dgamma and dbeta from the blocks' partial sums: 32 columns a block, the partials dealt over its eight warps and
// added in a fixed order.
__global__ void __launch_bounds__(256) norm_join_kernel(const NormArgs a) {
  __shared__ float part[8][33];
  grid_dependency_handshake();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;  // over dgamma, then dbeta
  const uint64_t width = 2ull * a.cols;
  float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
  if (c < width) {
    uint32_t i = warp;
    for (; i + 24 < a.n_partials; i += 32) {
      s0 += ld_c(a.partials + (uint64_t)i * width + c);
      s1 += ld_c(a.partials + (uint64_t)(i + 8) * width + c);
      s2 += ld_c(a.partials + (uint64_t)(i + 16) * width + c);
      s3 += ld_c(a.partials + (uint64_t)(i + 24) * width + c);
    }
    for (; i < a.n_partials; i += 8) s0 += ld_c(a.partials + (uint64_t)i * width + c);
  }
  part[warp][lane] = (s0 + s1) + (s2 + s3);
  __syncthreads();
  if (warp == 0 && c < width) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w][lane];
    float* out = c < a.cols ? a.dgamma : a.dbeta;
    if (out) st_c(out + (c < a.cols ? c : c - a.cols), s);
  }
}

}  // namespace accept
