// Layer norm, forward and backward (sm_100a).
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
  float eps, inv_cols;
  int dtype_w;
};

// How the columns of a row lie over the threads that share it.  Whole: thread t holds octets t, t + T, ... of eight
// neighbours, moved in 16-byte pieces.  Loose (rows that do not start on 16-byte boundaries): thread t holds
// columns t, t + T, ..., one at a time.
template <bool WHOLE>
__device__ __forceinline__ uint32_t column_of(uint32_t t, uint32_t threads, int i, int j) {
  return WHOLE ? 8 * (t + i * threads) + j : t + (8 * i + j) * threads;
}

// P octets of a row into registers; columns past the last are zero.
template <typename T, bool WHOLE, int P>
__device__ __forceinline__ void load_row(const T* row, uint32_t cols, uint32_t t, uint32_t threads, float (&v)[P][8]) {
  if (WHOLE) {
    Pack<T> raw[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint32_t c = column_of<true>(t, threads, i, 0);
      if (c + 8 <= cols) raw[i] = ld_pack(row + c);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint32_t c = column_of<true>(t, threads, i, 0);
      if (c + 8 <= cols) unpack(raw[i], v[i]);
      else ld_some(row + c, c < cols ? (int)(cols - c) : 0, v[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = column_of<false>(t, threads, i, j);
        v[i][j] = c < cols ? to_float(ld_c(row + c)) : 0.0f;
      }
  }
}

template <typename T, bool WHOLE, int P>
__device__ __forceinline__ void store_row(T* row, uint32_t cols, uint32_t t, uint32_t threads, const float (&v)[P][8]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (WHOLE) {
      const uint32_t c = column_of<true>(t, threads, i, 0);
      if (c + 8 <= cols) {
        Pack<T> raw;
        pack(v[i], raw);
        st_pack(row + c, raw);
      } else if (c < cols) {
        st_some(row + c, (int)(cols - c), v[i]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = column_of<false>(t, threads, i, j);
        if (c < cols) st_c(row + c, from_float<T>(v[i][j]));
      }
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

// gamma or beta for this thread's columns: read once for all rows of the block.
template <bool WHOLE, int P>
__device__ __forceinline__ void load_weights(const void* w, int dtype, float absent, uint32_t cols, uint32_t t, uint32_t threads, float (&v)[P][8]) {
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t c = column_of<WHOLE>(t, threads, i, j);
      v[i][j] = c < cols ? weight_at(w, dtype, absent, c) : absent;
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// Sum over the threads that share a row.  ONE_WARP: a warp has a row of its own; otherwise the whole block has one and
// `slot` is shared memory for a value of each warp, used in turn (no barrier is needed before its next use but one).
template <bool ONE_WARP>
__device__ __forceinline__ float row_sum(float v, float* slot) {
  v = warp_sum(v);
  if (ONE_WARP) return v;
  const uint32_t warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) slot[threadIdx.x >> 5] = v;
  __syncthreads();
  return warp_sum(lane < warps ? slot[lane] : 0.0f);
}

// Forward.  A row stays in the registers of the threads that share it: the mean first, then the sum of the squared
// distances from it, so that an offset much larger than the spread costs no digits.
template <typename TX, typename TY, bool WHOLE, bool ONE_WARP, int P, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) norm_forward_kernel(const NormArgs a) {
  __shared__ float slots[2][32];
  const uint32_t threads = ONE_WARP ? 32 : blockDim.x;
  const uint32_t t = ONE_WARP ? threadIdx.x & 31 : threadIdx.x;
  const uint32_t rows_per_block = ONE_WARP ? blockDim.x >> 5 : 1;
  grid_dependency_handshake();
  float gamma[P][8], beta[P][8];
  load_weights<WHOLE, P>(a.gamma, a.dtype_w, 1.0f, a.cols, t, threads, gamma);
  load_weights<WHOLE, P>(a.beta, a.dtype_w, 0.0f, a.cols, t, threads, beta);
  for (uint64_t r = (uint64_t)blockIdx.x * rows_per_block + (ONE_WARP ? threadIdx.x >> 5 : 0); r < a.rows;
       r += (uint64_t)gridDim.x * rows_per_block) {
    float v[P][8];
    load_row<TX, WHOLE, P>(static_cast<const TX*>(a.x) + r * a.ld_x, a.cols, t, threads, v);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += v[i][j];
    const float mean = row_sum<ONE_WARP>(sum, slots[0]) * a.inv_cols;
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = column_of<WHOLE>(t, threads, i, j) < a.cols ? v[i][j] - mean : 0.0f;
        squares = fmaf(v[i][j], v[i][j], squares);
      }
    const float var = row_sum<ONE_WARP>(squares, slots[1]) * a.inv_cols;
    const float rstd = 1.0f / sqrtf(var + a.eps);
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j] * rstd, gamma[i][j], beta[i][j]);
    store_row<TY, WHOLE, P>(static_cast<TY*>(a.y) + r * a.ld_y, a.cols, t, threads, v);
    if (t == 0 && a.mean_out) st_c(a.mean_out + r, mean);
    if (t == 0 && a.rstd_out) st_c(a.rstd_out + r, rstd);
  }
}

// Backward.  dx needs two sums of a row, taken together; the gradients of gamma and beta are sums over the rows, held
// in registers over all rows of a block and joined by norm_join_kernel.
template <typename TX, typename TY, bool WHOLE, bool ONE_WARP, int P, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) norm_backward_kernel(const NormArgs a) {
  __shared__ float slots[2][2][32];
  const uint32_t threads = ONE_WARP ? 32 : blockDim.x;
  const uint32_t t = ONE_WARP ? threadIdx.x & 31 : threadIdx.x;
  const uint32_t rows_per_block = ONE_WARP ? blockDim.x >> 5 : 1;
  grid_dependency_handshake();
  float gamma[P][8], dgamma[P][8], dbeta[P][8];
  load_weights<WHOLE, P>(a.gamma, a.dtype_w, 1.0f, a.cols, t, threads, gamma);
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dgamma[i][j] = dbeta[i][j] = 0.0f;
  int turn = 0;
  for (uint64_t r = (uint64_t)blockIdx.x * rows_per_block + (ONE_WARP ? threadIdx.x >> 5 : 0); r < a.rows; r += (uint64_t)gridDim.x * rows_per_block, turn ^= 1) {
    float x[P][8], dy[P][8];
    load_row<TX, WHOLE, P>(static_cast<const TX*>(a.x) + r * a.ld_x, a.cols, t, threads, x);
    load_row<TY, WHOLE, P>(static_cast<const TY*>(a.dy) + r * a.ld_y, a.cols, t, threads, dy);
    const float mean = ld_c(a.mean + r), rstd = ld_c(a.rstd + r);
    float sum = 0.0f, along = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[i][j] = (x[i][j] - mean) * rstd;  // columns past the last: dy = 0, so what stands here counts nowhere
        dbeta[i][j] += dy[i][j];
        dgamma[i][j] = fmaf(dy[i][j], x[i][j], dgamma[i][j]);
        dy[i][j] *= gamma[i][j];
        sum += dy[i][j];
        along = fmaf(dy[i][j], x[i][j], along);
      }
    if (!a.dx) continue;
    sum = row_sum<ONE_WARP>(sum, slots[turn][0]) * a.inv_cols;
    along = row_sum<ONE_WARP>(along, slots[turn][1]) * a.inv_cols;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = rstd * (dy[i][j] - sum - x[i][j] * along);
    store_row<TX, WHOLE, P>(static_cast<TX*>(a.dx) + r * a.ld_x, a.cols, t, threads, x);
  }
  if (!a.partials) return;
  float* out = a.partials + (uint64_t)blockIdx.x * 2 * a.cols;
  if (ONE_WARP) {  // the block's warps add up their columns one after the other
    __shared__ float sums[2][P * 256];
    for (uint32_t w = 0; w < rows_per_block; ++w) {
      if (threadIdx.x >> 5 == w) {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t c = (8 * i + j) * 32 + t;  // a place of its own for each of the lane's columns
            sums[0][c] = w ? sums[0][c] + dgamma[i][j] : dgamma[i][j];
            sums[1][c] = w ? sums[1][c] + dbeta[i][j] : dbeta[i][j];
          }
      }
      __syncthreads();
    }
    if (threadIdx.x >= 32) return;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dgamma[i][j] = sums[0][(8 * i + j) * 32 + t];
        dbeta[i][j] = sums[1][(8 * i + j) * 32 + t];
      }
  }
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t c = column_of<WHOLE>(t, threads, i, j);
      if (c < a.cols) { st_c(out + c, dgamma[i][j]); st_c(out + a.cols + c, dbeta[i][j]); }
    }
}

// Rows longer than the registers of a block: the same formulas, each row read again for each of its sums.
template <typename TX, typename TY>
__global__ void __launch_bounds__(1024) norm_forward_long_kernel(const NormArgs a) {
  __shared__ float slots[2][32];
  grid_dependency_handshake();
  for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const TX* row = static_cast<const TX*>(a.x) + r * a.ld_x;
    TY* out = static_cast<TY*>(a.y) + r * a.ld_y;
    float sum = 0.0f, squares = 0.0f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) sum += to_float(ld_c(row + c));
    const float mean = row_sum<false>(sum, slots[0]) * a.inv_cols;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float d = to_float(ld_c(row + c)) - mean;
      squares = fmaf(d, d, squares);
    }
    const float rstd = 1.0f / sqrtf(row_sum<false>(squares, slots[1]) * a.inv_cols + a.eps);
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float g = weight_at(a.gamma, a.dtype_w, 1.0f, c), b = weight_at(a.beta, a.dtype_w, 0.0f, c);
      st_c(out + c, from_float<TY>(fmaf((to_float(ld_c(row + c)) - mean) * rstd, g, b)));
    }
    if (threadIdx.x == 0 && a.mean_out) st_c(a.mean_out + r, mean);
    if (threadIdx.x == 0 && a.rstd_out) st_c(a.rstd_out + r, rstd);
  }
}

// The two sums of each row and dx; norm_backward_long_sums_kernel takes the sums over the rows.
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
    sum = row_sum<false>(sum, slots[turn][0]) * a.inv_cols;
    along = row_sum<false>(along, slots[turn][1]) * a.inv_cols;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float h = to_float(ld_c(drow + c)) * weight_at(a.gamma, a.dtype_w, 1.0f, c);
      st_c(out + c, from_float<TX>(rstd * (h - sum - (to_float(ld_c(row + c)) - mean) * rstd * along)));
    }
  }
}

// Sums over the rows for one column a thread; blockIdx.y takes every gridDim.y-th row into its own partial.
template <typename TX, typename TY>
__global__ void __launch_bounds__(256) norm_backward_long_sums_kernel(const NormArgs a) {
  grid_dependency_handshake();
  const uint32_t c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  float dgamma = 0.0f, dbeta = 0.0f;
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
