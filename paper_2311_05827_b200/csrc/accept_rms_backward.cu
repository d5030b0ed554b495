// Host side of the root-mean-square norm's backward pass (accept_rms_norm_backward).
#include "accept_rms_host.cuh"

namespace {

using namespace accept;

template <typename TX, typename TY>
struct Backward {
  static constexpr int kStages = rms_stages_for((int)(2 * sizeof(TX) + sizeof(TY)));
  template <int V, int L, bool LOOSE> static RmsKernel held() { return rms_backward_kernel<TX, TY, V, kRmsOwn, L, kStages, LOOSE>; }
  template <bool VEC> static RmsKernel wide() { return rms_backward_wide_kernel<TX, TY, VEC>; }
};
template <typename TX, typename TY>
struct ColumnSums {  // of wide rows only
  template <int V, int L, bool LOOSE> static RmsKernel held() { return nullptr; }
  template <bool VEC> static RmsKernel wide() { return rms_column_sums_kernel<TX, TY, VEC>; }
};

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_rms_backward_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" accept_status accept_rms_norm_backward(const accept_rms_norm_params* p, const void* d_dy, const void* d_s, const void* d_gamma,
                                                  const float* d_rstd, const void* d_dsum, void* d_dx, void* d_dbranch, float* d_dgamma,
                                                  void* d_ws, size_t ws_bytes, void* cuda_stream) {
  if (!p || !d_ws) return ACCEPT_ERR_NULL;
  const accept_status st = accept_rms_norm_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (ws_bytes < accept_rms_norm_workspace_size(p)) return ACCEPT_ERR_TOO_SMALL;
  if (p->rows != 0 && (!d_dy || !d_s || !d_rstd)) return ACCEPT_ERR_NULL;
  if (!d_dx && !d_dbranch && !d_dgamma) return ACCEPT_ERR_NULL;
  const size_t size_x = rms_value_size(p->dtype_x), size_y = rms_value_size(p->dtype_y);
  if (!is_aligned(d_dy, size_y) || !is_aligned(d_s, size_x) || !is_aligned(d_gamma, rms_value_size(p->dtype_w)) || !is_aligned(d_rstd, 4) ||
      !is_aligned(d_dsum, size_x) || !is_aligned(d_dx, size_x) || !is_aligned(d_dbranch, size_y) || !is_aligned(d_dgamma, 4) || !is_aligned(d_ws, 16))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const auto all = [&](auto rows) {
    return rows(d_s, p->ld_x, p->dtype_x) && rows(d_dsum, p->ld_x, p->dtype_x) && rows(d_dx, p->ld_x, p->dtype_x) && rows(d_dy, p->ld_y, p->dtype_y) &&
           rows(d_dbranch, p->ld_y, p->dtype_y);
  };
  const bool whole = all(rms_whole_rows);
  const RmsShape shape = rms_shape(p, true, whole, d_dsum ? 2 : 1, 1);
  RmsArgs a = rms_args(p, d_gamma);
  a.x = d_s;
  a.dy = d_dy;
  a.rstd = d_rstd;
  a.dsum = d_dsum;
  a.dx = d_dx;
  a.dbranch = d_dbranch;
  a.dgamma = d_dgamma;
  a.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(d_ws) + 16);
  a.n_partials = p->rows ? (uint32_t)rms_partials(p, shape) : 0;
  ACCEPT_BOUNDS(s, bounds_list.add(d_dy, rms_matrix_bytes(p, p->ld_y, p->dtype_y), false);
                bounds_list.add(d_s, rms_matrix_bytes(p, p->ld_x, p->dtype_x), false);
                bounds_list.add(d_gamma, p->cols * rms_value_size(p->dtype_w), false); bounds_list.add(d_rstd, 4 * p->rows, false);
                bounds_list.add(d_dsum, rms_matrix_bytes(p, p->ld_x, p->dtype_x), false);
                bounds_list.add(d_dx, rms_matrix_bytes(p, p->ld_x, p->dtype_x), true);
                bounds_list.add(d_dbranch, rms_matrix_bytes(p, p->ld_y, p->dtype_y), true);
                bounds_list.add(d_dgamma, 4 * p->cols, true); bounds_list.add(d_ws, accept_rms_norm_workspace_size(p), true));
  if (p->rows != 0) {
    // the column sums of wide rows first: dx may take the place of the sum, dbranch that of dy
    if (shape.wide && d_dgamma)
      ACCEPT_LAUNCH(launch_overlapped(rms_kernel<ColumnSums>(p, shape, whole), dim3((a.cols + 255) / 256, a.n_partials), 256, s, a));
    if (!shape.wide || d_dx || d_dbranch) ACCEPT_LAUNCH(launch_rms(rms_kernel<Backward>(p, shape, whole), shape, a, s));
  }
  const bool summed = p->rows != 0 && (shape.joins || (shape.wide && a.n_partials == 1));
  if (d_dgamma && !summed)
    ACCEPT_LAUNCH(launch_overlapped(rms_join_kernel<kRmsJoinWarps>, dim3((a.cols + 31) / 32), 32 * kRmsJoinWarps, s, a));
  return ACCEPT_OK;
}
