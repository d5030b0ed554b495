// Host side of layer norm (accept_layer_norm_*): argument checks, launch shapes, launches.
#include "accept_host.cuh"
#include "accept_norm.cuh"

namespace {

using accept::is_aligned;
using accept::launch_overlapped;
using accept::NormArgs;

constexpr unsigned kSms = 148;

// Launch shape of a pass: octets per thread, threads, whether each warp has a row of its own, blocks.
struct NormShape { int octets; unsigned threads; bool one_warp; bool longer; unsigned blocks; };

NormShape norm_shape(const accept_layer_norm_params* p, bool backward) {
  NormShape s{};
  const uint64_t octets = (p->cols + 7) / 8;
  if (octets <= 64) {
    s.one_warp = true;
    s.octets = octets <= 32 ? 1 : 2;
    s.threads = 256;
  } else {
    s.octets = octets <= 256 || (backward && octets > 512) ? 1 : 2;
    s.threads = (unsigned)(((octets + s.octets - 1) / s.octets + 31) / 32 * 32);
    if ((octets + s.octets - 1) / s.octets > 1024) s.longer = true;
  }
  if (s.longer) s.threads = 1024;
  const uint64_t units = s.one_warp ? (p->rows + 7) / 8 : p->rows;
  const uint64_t per_sm = backward ? (s.octets == 2 ? 512 : 1024) / s.threads : 1024 / s.threads;
  const uint64_t most = kSms * (per_sm ? per_sm : 1);
  s.blocks = (unsigned)(units < most ? units : most);
  return s;
}

// Partial sums of dgamma and dbeta that the backward pass leaves in the workspace.
unsigned long_partials(const accept_layer_norm_params* p) { return (unsigned)(p->rows < 64 ? p->rows : 64); }

uint64_t norm_partials(const accept_layer_norm_params* p) {
  const NormShape s = norm_shape(p, true);
  return s.longer ? long_partials(p) : s.blocks;
}

using KernelFn = void (*)(const NormArgs);

template <typename TX, typename TY, bool WHOLE>
KernelFn forward_for(const NormShape& s) {
  if (s.one_warp) return s.octets == 1 ? accept::norm_forward_kernel<TX, TY, WHOLE, true, 1, 256> : accept::norm_forward_kernel<TX, TY, WHOLE, true, 2, 256>;
  return s.octets == 1 ? accept::norm_forward_kernel<TX, TY, WHOLE, false, 1, 256>
                       : s.threads <= 512 ? accept::norm_forward_kernel<TX, TY, WHOLE, false, 2, 512> : accept::norm_forward_kernel<TX, TY, WHOLE, false, 2, 1024>;
}
template <typename TX, typename TY, bool WHOLE>
KernelFn backward_for(const NormShape& s) {
  if (s.one_warp) return s.octets == 1 ? accept::norm_backward_kernel<TX, TY, WHOLE, true, 1, 256> : accept::norm_backward_kernel<TX, TY, WHOLE, true, 2, 256>;
  return s.octets == 2 ? accept::norm_backward_kernel<TX, TY, WHOLE, false, 2, 256>
                       : s.threads <= 256 ? accept::norm_backward_kernel<TX, TY, WHOLE, false, 1, 256> : accept::norm_backward_kernel<TX, TY, WHOLE, false, 1, 1024>;
}

struct Kernels { KernelFn one, sums; };

template <typename TX, typename TY>
Kernels kernels_for(const NormShape& s, bool backward, bool whole) {
  if (s.longer) return backward ? Kernels{accept::norm_backward_long_kernel<TX, TY>, accept::norm_backward_long_sums_kernel<TX, TY>}
                                : Kernels{accept::norm_forward_long_kernel<TX, TY>, nullptr};
  if (backward) return {whole ? backward_for<TX, TY, true>(s) : backward_for<TX, TY, false>(s), nullptr};
  return {whole ? forward_for<TX, TY, true>(s) : forward_for<TX, TY, false>(s), nullptr};
}

template <typename TX>
Kernels kernels_for_y(const accept_layer_norm_params* p, const NormShape& s, bool backward, bool whole) {
  switch (p->dtype_y) {
    case ACCEPT_DTYPE_F32: return kernels_for<TX, float>(s, backward, whole);
    case ACCEPT_DTYPE_BF16: return kernels_for<TX, __nv_bfloat16>(s, backward, whole);
    default: return kernels_for<TX, __half>(s, backward, whole);
  }
}

Kernels select_kernels(const accept_layer_norm_params* p, const NormShape& s, bool backward, bool whole) {
  switch (p->dtype_x) {
    case ACCEPT_DTYPE_F32: return kernels_for_y<float>(p, s, backward, whole);
    case ACCEPT_DTYPE_BF16: return kernels_for_y<__nv_bfloat16>(p, s, backward, whole);
    default: return kernels_for_y<__half>(p, s, backward, whole);
  }
}

size_t value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == ACCEPT_DTYPE_F32 || d == ACCEPT_DTYPE_BF16 || d == ACCEPT_DTYPE_F16; }

// rows that all start on 16-byte boundaries
bool whole_rows(const void* p, uint64_t ld, int32_t dtype) { return is_aligned(p, 16) && ld * value_size(dtype) % 16 == 0; }

NormArgs norm_args(const accept_layer_norm_params* p) {
  NormArgs a{};
  a.rows = p->rows;
  a.cols = (uint32_t)p->cols;
  a.ld_x = p->ld_x;
  a.ld_y = p->ld_y;
  a.eps = p->eps;
  a.inv_cols = 1.0f / (float)p->cols;
  a.dtype_w = p->dtype_w;
  return a;
}

#ifdef ACCEPT_BOUNDS_CHECK
size_t matrix_bytes(uint64_t rows, uint64_t cols, uint64_t ld, int32_t dtype) { return rows ? ((rows - 1) * ld + cols) * value_size(dtype) : 0; }
#endif

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_norm_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_layer_norm_check_params(const accept_layer_norm_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  if (p->cols == 0 || p->cols > 0x7fffffffull || p->ld_x < p->cols || p->ld_y < p->cols) return ACCEPT_ERR_BAD_SIZE;
  // every offset of a value must be a 63-bit number of bytes
  if (p->rows > (1ull << 40) || p->ld_x > (1ull << 40) || p->ld_y > (1ull << 40) ||
      (p->rows && (p->ld_x > (1ull << 60) / p->rows || p->ld_y > (1ull << 60) / p->rows)))
    return ACCEPT_ERR_BAD_SIZE;
  if (!is_dtype(p->dtype_x) || !is_dtype(p->dtype_y) || !is_dtype(p->dtype_w)) return ACCEPT_ERR_BAD_ENUM;
  if (!(p->eps >= 0.0f) || p->eps > 3.402823466e38f) return ACCEPT_ERR_BAD_SIZE;
  return ACCEPT_OK;
}

size_t accept_layer_norm_workspace_size(const accept_layer_norm_params* p) {
  if (accept_layer_norm_check_params(p) != ACCEPT_OK) return 0;
  return 16 + (size_t)(norm_partials(p) * 8 * p->cols);
}

accept_status accept_layer_norm_forward(const accept_layer_norm_params* p, const void* d_x, const void* d_gamma,
                                        const void* d_beta, void* d_y, float* d_mean, float* d_rstd, void* cuda_stream) {
  if (!p) return ACCEPT_ERR_NULL;
  const accept_status st = accept_layer_norm_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (p->rows == 0) return ACCEPT_OK;
  if (!d_x || !d_y) return ACCEPT_ERR_NULL;
  if (!is_aligned(d_x, value_size(p->dtype_x)) || !is_aligned(d_y, value_size(p->dtype_y)) || !is_aligned(d_gamma, value_size(p->dtype_w)) ||
      !is_aligned(d_beta, value_size(p->dtype_w)) || !is_aligned(d_mean, 4) || !is_aligned(d_rstd, 4))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  NormArgs a = norm_args(p);
  a.x = d_x;
  a.gamma = d_gamma;
  a.beta = d_beta;
  a.y = d_y;
  a.mean_out = d_mean;
  a.rstd_out = d_rstd;
  ACCEPT_BOUNDS(s, bounds_list.add(d_x, matrix_bytes(p->rows, p->cols, p->ld_x, p->dtype_x), false);
                bounds_list.add(d_y, matrix_bytes(p->rows, p->cols, p->ld_y, p->dtype_y), true);
                bounds_list.add(d_gamma, p->cols * value_size(p->dtype_w), false);
                bounds_list.add(d_beta, p->cols * value_size(p->dtype_w), false);
                bounds_list.add(d_mean, 4 * p->rows, true); bounds_list.add(d_rstd, 4 * p->rows, true));
  const NormShape shape = norm_shape(p, false);
  const bool whole = whole_rows(d_x, p->ld_x, p->dtype_x) && whole_rows(d_y, p->ld_y, p->dtype_y);
  const Kernels k = select_kernels(p, shape, false, whole);
  ACCEPT_LAUNCH(launch_overlapped(k.one, dim3(shape.blocks), shape.threads, s, a));
  return ACCEPT_OK;
}

accept_status accept_layer_norm_backward(const accept_layer_norm_params* p, const void* d_dy, const void* d_x,
                                         const void* d_gamma, const float* d_mean, const float* d_rstd, void* d_dx,
                                         float* d_dgamma, float* d_dbeta, void* d_ws, size_t ws_bytes, void* cuda_stream) {
  if (!p || !d_ws) return ACCEPT_ERR_NULL;
  const accept_status st = accept_layer_norm_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (ws_bytes < accept_layer_norm_workspace_size(p)) return ACCEPT_ERR_TOO_SMALL;
  if (p->rows != 0 && (!d_dy || !d_x || !d_mean || !d_rstd)) return ACCEPT_ERR_NULL;
  const bool weights = d_dgamma || d_dbeta;
  if (!d_dx && !weights) return ACCEPT_ERR_NULL;
  if (!is_aligned(d_x, value_size(p->dtype_x)) || !is_aligned(d_dy, value_size(p->dtype_y)) || !is_aligned(d_dx, value_size(p->dtype_x)) ||
      !is_aligned(d_gamma, value_size(p->dtype_w)) || !is_aligned(d_mean, 4) || !is_aligned(d_rstd, 4) || !is_aligned(d_dgamma, 4) ||
      !is_aligned(d_dbeta, 4) || !is_aligned(d_ws, 16))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const NormShape shape = norm_shape(p, true);
  NormArgs a = norm_args(p);
  a.x = d_x;
  a.dy = d_dy;
  a.gamma = d_gamma;
  a.mean = d_mean;
  a.rstd = d_rstd;
  a.dx = d_dx;
  a.partials = weights ? reinterpret_cast<float*>(static_cast<uint8_t*>(d_ws) + 16) : nullptr;
  a.n_partials = (uint32_t)norm_partials(p);
  a.dgamma = d_dgamma;
  a.dbeta = d_dbeta;
  ACCEPT_BOUNDS(s, bounds_list.add(d_x, matrix_bytes(p->rows, p->cols, p->ld_x, p->dtype_x), false);
                bounds_list.add(d_dy, matrix_bytes(p->rows, p->cols, p->ld_y, p->dtype_y), false);
                bounds_list.add(d_dx, matrix_bytes(p->rows, p->cols, p->ld_x, p->dtype_x), true);
                bounds_list.add(d_gamma, p->cols * value_size(p->dtype_w), false);
                bounds_list.add(d_mean, 4 * p->rows, false); bounds_list.add(d_rstd, 4 * p->rows, false);
                bounds_list.add(d_dgamma, 4 * p->cols, true); bounds_list.add(d_dbeta, 4 * p->cols, true);
                bounds_list.add(d_ws, accept_layer_norm_workspace_size(p), true));
  if (p->rows != 0) {
    const bool whole = whole_rows(d_x, p->ld_x, p->dtype_x) && whole_rows(d_dy, p->ld_y, p->dtype_y) && is_aligned(d_dx, 16);
    const Kernels k = select_kernels(p, shape, true, whole);
    if (!shape.longer || d_dx) ACCEPT_LAUNCH(launch_overlapped(k.one, dim3(shape.blocks), shape.threads, s, a));
    if (shape.longer && weights) ACCEPT_LAUNCH(launch_overlapped(k.sums, dim3((a.cols + 255) / 256, a.n_partials), 256, s, a));
  }
  if (weights) ACCEPT_LAUNCH(launch_overlapped(accept::norm_join_kernel, dim3((unsigned)((2ull * a.cols + 31) / 32)), 256, s, a));
  return ACCEPT_OK;
}

}  // extern "C"
