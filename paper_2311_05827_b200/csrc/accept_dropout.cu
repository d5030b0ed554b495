// Host side of dropout (accept_dropout): argument checks, launches.
#include "accept_dropout.cuh"
#include "accept_drop_host.cuh"

namespace {

using accept::DropoutArgs;
using accept::is_aligned;

size_t value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == ACCEPT_DTYPE_F32 || d == ACCEPT_DTYPE_BF16 || d == ACCEPT_DTYPE_F16; }

using KernelFn = void (*)(const DropoutArgs);
constexpr int kUnits = 2, kFlatUnits = 4;
enum class Rows { kFlat, kWhole, kLoose };  // no gaps, every row on a 16-byte boundary, neither

template <typename TX, typename TY>
KernelFn select_rows(Rows rows) {
  return rows == Rows::kFlat    ? accept::dropout_flat_kernel<TX, TY, kFlatUnits>
         : rows == Rows::kWhole ? accept::dropout_kernel<TX, TY, true, kUnits> : accept::dropout_kernel<TX, TY, false, kUnits>;
}
template <typename TX>
KernelFn select_y(int32_t dtype_y, Rows rows) {
  switch (dtype_y) {
    case ACCEPT_DTYPE_F32: return select_rows<TX, float>(rows);
    case ACCEPT_DTYPE_BF16: return select_rows<TX, __nv_bfloat16>(rows);
    default: return select_rows<TX, __half>(rows);
  }
}
KernelFn select_kernel(int32_t dtype_x, int32_t dtype_y, Rows rows) {
  switch (dtype_x) {
    case ACCEPT_DTYPE_F32: return select_y<float>(dtype_y, rows);
    case ACCEPT_DTYPE_BF16: return select_y<__nv_bfloat16>(dtype_y, rows);
    default: return select_y<__half>(dtype_y, rows);
  }
}

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_dropout_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_dropout_check_params(const accept_dropout_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  // every offset of a value must be a 63-bit number of bytes
  if (p->ld_x < p->cols || p->ld_y < p->cols || p->rows > (1ull << 40) || p->cols > (1ull << 40) || p->ld_x > (1ull << 40) || p->ld_y > (1ull << 40) ||
      (p->rows && (p->ld_x > (1ull << 60) / p->rows || p->ld_y > (1ull << 60) / p->rows)))
    return ACCEPT_ERR_BAD_SIZE;
  if (p->rows * ((p->cols + 7) / 8) / (kUnits * accept::kDropThreads) >= 0x7fffffffull) return ACCEPT_ERR_BAD_SIZE;  // blocks of a grid
  if (!is_dtype(p->dtype_x) || !is_dtype(p->dtype_y) || p->reserved != 0) return ACCEPT_ERR_BAD_ENUM;
  if (!accept::is_drop_rate(p->p)) return ACCEPT_ERR_BAD_SIZE;
  return ACCEPT_OK;
}

accept_status accept_dropout(const accept_dropout_params* p, const void* d_x, const void* d_residual, void* d_y, void* cuda_stream) {
  if (!p) return ACCEPT_ERR_NULL;
  const accept_status st = accept_dropout_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (p->rows == 0 || p->cols == 0) return ACCEPT_OK;
  if (!d_x || !d_y) return ACCEPT_ERR_NULL;
  const size_t size_x = value_size(p->dtype_x), size_y = value_size(p->dtype_y);
  if (!is_aligned(d_x, size_x) || !is_aligned(d_residual, size_y) || !is_aligned(d_y, size_y)) return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  DropoutArgs a{};
  a.x = d_x;
  a.residual = d_residual;
  a.y = d_y;
  a.rows = p->rows;
  a.cols = p->cols;
  a.ld_x = p->ld_x;
  a.ld_y = p->ld_y;
  a.drop = accept::drop_of(p->p, p->seed, p->rng_offset);
  ACCEPT_BOUNDS(s, bounds_list.add(d_x, ((p->rows - 1) * p->ld_x + p->cols) * size_x, false);
                bounds_list.add(d_residual, ((p->rows - 1) * p->ld_y + p->cols) * size_y, false);
                bounds_list.add(d_y, ((p->rows - 1) * p->ld_y + p->cols) * size_y, true));
  const bool starts = is_aligned(d_x, 16) && is_aligned(d_residual, 16) && is_aligned(d_y, 16);
  Rows rows = starts && p->ld_x * size_x % 16 == 0 && p->ld_y * size_y % 16 == 0 ? Rows::kWhole : Rows::kLoose;
  if (p->rows == 1 || (p->ld_x == p->cols && p->ld_y == p->cols)) {
    a.cols = p->rows * p->cols;
    a.rows = 1;
    rows = starts ? Rows::kFlat : Rows::kLoose;
  }
  a.per_row = (a.cols + 7) / 8;
  a.units = a.rows * a.per_row;
  const uint64_t block = (rows == Rows::kFlat ? kFlatUnits : kUnits) * accept::kDropThreads;
  ACCEPT_LAUNCH(accept::launch_overlapped(select_kernel(p->dtype_x, p->dtype_y, rows), dim3((unsigned)((a.units + block - 1) / block)), accept::kDropThreads, s, a));
  return ACCEPT_OK;
}

}  // extern "C"
