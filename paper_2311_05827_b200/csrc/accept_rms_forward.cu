// Host side of the root-mean-square norm (accept_rms_norm_*): argument checks, sizes, and the forward pass.
#include "accept_rms_host.cuh"

namespace {

using namespace accept;

bool is_dtype(int32_t d) { return d == ACCEPT_DTYPE_F32 || d == ACCEPT_DTYPE_BF16 || d == ACCEPT_DTYPE_F16; }
uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

template <typename TX, typename TY, bool CODES>
struct ForwardTo {
  static constexpr int kStages = rms_stages_for((int)(sizeof(TX) + sizeof(TY)));
  template <int V, int L, bool LOOSE> static RmsKernel held() { return rms_forward_kernel<TX, TY, V, kRmsOwn, L, kStages, LOOSE, CODES>; }
  template <bool VEC> static RmsKernel wide() { return rms_forward_wide_kernel<TX, TY, VEC>; }
};
template <typename TX, typename TY> using Forward = ForwardTo<TX, TY, false>;
template <typename TX, typename TY> using ForwardToCodes = ForwardTo<TX, TY, true>;

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_rms_forward_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_rms_norm_check_params(const accept_rms_norm_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  if (p->cols == 0 || p->cols > 0x7fffffffull || p->ld_x < p->cols || p->ld_y < p->cols) return ACCEPT_ERR_BAD_SIZE;
  // every offset of a value must be a 63-bit number of bytes
  if (p->rows > (1ull << 38) || p->ld_x > (1ull << 40) || p->ld_y > (1ull << 40) ||
      (p->rows && (p->ld_x > (1ull << 60) / p->rows || p->ld_y > (1ull << 60) / p->rows)))
    return ACCEPT_ERR_BAD_SIZE;
  if (!is_dtype(p->dtype_x) || !is_dtype(p->dtype_y) || !is_dtype(p->dtype_w)) return ACCEPT_ERR_BAD_ENUM;
  if (p->format != ACCEPT_FORMAT_E4M3 && p->format != ACCEPT_FORMAT_E5M2) return ACCEPT_ERR_BAD_ENUM;
  if (!(p->eps >= 0.0f) || p->eps > 3.402823466e38f || !is_drop_rate(p->p)) return ACCEPT_ERR_BAD_SIZE;
  return ACCEPT_OK;
}

size_t accept_rms_norm_workspace_size(const accept_rms_norm_params* p) {
  if (accept_rms_norm_check_params(p) != ACCEPT_OK) return 0;
  const RmsShape s = rms_shape(p, true, true, 2, 1);  // the partials depend on the rows and columns alone
  return 16 + (size_t)(rms_partials(p, s) * 4 * p->cols);
}

accept_status accept_rms_norm_forward(const accept_rms_norm_params* p, const void* d_x, const void* d_branch, const void* d_gamma,
                                      void* d_sum, void* d_y, void* d_q, void* d_scale, float* d_rstd, void* d_ws, size_t ws_bytes,
                                      void* cuda_stream) {
  if (!p) return ACCEPT_ERR_NULL;
  const accept_status st = accept_rms_norm_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (!d_q != !d_scale || (d_q && !d_ws)) return ACCEPT_ERR_NULL;
  if (d_q && ws_bytes < 16) return ACCEPT_ERR_TOO_SMALL;
  if (d_q && p->rows > 0x7fffffffull) return ACCEPT_ERR_BAD_SIZE;
  if (p->rows == 0) return ACCEPT_OK;
  if (!d_x || (!d_y && !d_q && !d_sum && !d_rstd)) return ACCEPT_ERR_NULL;
  const size_t size_x = rms_value_size(p->dtype_x), size_y = rms_value_size(p->dtype_y);
  if (!is_aligned(d_x, size_x) || !is_aligned(d_sum, size_x) || !is_aligned(d_branch, size_y) || !is_aligned(d_y, size_y) ||
      !is_aligned(d_gamma, rms_value_size(p->dtype_w)) || !is_aligned(d_q, 16) || !is_aligned(d_scale, 16) || !is_aligned(d_rstd, 4) ||
      (d_q && !is_aligned(d_ws, 4)))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  RmsArgs a = rms_args(p, d_gamma);
  a.x = d_x;
  a.branch = d_branch;
  a.sum = d_sum;
  a.y = d_y;
  a.q = static_cast<uint8_t*>(d_q);
  a.scale = static_cast<uint8_t*>(d_scale);
  a.rstd_out = d_rstd;
  a.status = static_cast<uint32_t*>(d_ws);
  a.format = p->format;
  a.ldq = (uint32_t)up(p->cols, 16);
  a.blocks = (uint32_t)(up(p->cols, 128) / 128);
  a.atoms = (uint32_t)(up(p->rows, 128) / 128);
  if (!d_branch) a.drop.on = 0;
  ACCEPT_BOUNDS(s, bounds_list.add(d_x, rms_matrix_bytes(p, p->ld_x, p->dtype_x), false);
                bounds_list.add(d_branch, rms_matrix_bytes(p, p->ld_y, p->dtype_y), false);
                bounds_list.add(d_gamma, p->cols * rms_value_size(p->dtype_w), false);
                bounds_list.add(d_sum, rms_matrix_bytes(p, p->ld_x, p->dtype_x), true);
                bounds_list.add(d_y, rms_matrix_bytes(p, p->ld_y, p->dtype_y), true);
                bounds_list.add(d_q, p->rows * up(p->cols, 16), true);
                bounds_list.add(d_scale, 512 * (up(p->rows, 128) / 128) * (up(p->cols, 512) / 512), true);
                bounds_list.add(d_rstd, 4 * p->rows, true); if (d_q) bounds_list.add(d_ws, 16, true));
  const auto all = [&](auto rows) {
    return rows(d_x, p->ld_x, p->dtype_x) && rows(d_sum, p->ld_x, p->dtype_x) && rows(d_branch, p->ld_y, p->dtype_y) && rows(d_y, p->ld_y, p->dtype_y);
  };
  const bool whole = all(rms_whole_rows);
  const RmsShape shape = rms_shape(p, false, whole, 1, d_branch || !whole ? 1 : 0);
  ACCEPT_LAUNCH(launch_rms(d_q ? rms_kernel<ForwardToCodes>(p, shape, whole) : rms_kernel<Forward>(p, shape, whole), shape, a, s));
  return ACCEPT_OK;
}

}  // extern "C"
