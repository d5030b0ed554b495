// Host side of dropout (accept_dropout): argument checks, launches.
#include "accept_dropout.cuh"
#include "accept_drop_host.cuh"

namespace {

using accept::DropoutArgs;
using accept::is_aligned;

size_t value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == ACCEPT_DTYPE_F32 || d == ACCEPT_DTYPE_BF16 || d == ACCEPT_DTYPE_F16; }

using KernelFn = void (*)(const DropoutArgs);
constexpr int kRows = 2, kFlatUnits = 4;
enum class Rows { kFlat, kFew, kMany };  // no gaps; others

template <typename TX, typename TY>
KernelFn select_rows(Rows rows) {
  return rows == Rows::kFlat  ? accept::dropout_flat_kernel<TX, TY, kFlatUnits>
         : rows == Rows::kFew ? accept::dropout_kernel<TX, TY, kRows, true> : accept::dropout_kernel<TX, TY, kRows, false>;
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
  if (p->rows * ((p->cols + 14) / 8) / 32 >= 0x7fffffffull) return ACCEPT_ERR_BAD_SIZE;  // blocks of a grid
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
  bool flat = false;
  if (p->rows == 1 || (p->ld_x == p->cols && p->ld_y == p->cols)) {  // no gaps: one row
    a.cols = p->rows * p->cols;
    a.rows = 1;
    flat = is_aligned(d_x, 16) && is_aligned(d_residual, 16) && is_aligned(d_y, 16);
  }
  const KernelFn fn = select_kernel(p->dtype_x, p->dtype_y, flat ? Rows::kFlat : a.rows < 32 ? Rows::kFew : Rows::kMany);
  if (flat) {
    const uint64_t block = 8 * kFlatUnits * accept::kDropThreads;
    ACCEPT_LAUNCH(accept::launch_overlapped(fn, dim3((unsigned)((a.cols + block - 1) / block)), accept::kDropThreads, s, a));
    return ACCEPT_OK;
  }
  // Units start on y's 16-byte boundaries: one more than the columns fill where a row does not.  A warp takes neighbours of one row
  // where there are so many, more of a block where there are few rows.
  const bool on_boundaries = is_aligned(d_y, 16) && a.ld_y * size_y % 16 == 0;
  const uint64_t per_row = (a.cols + (on_boundaries ? 0 : 16 / size_y - 1) + 7) / 8;
  while (a.log_units < 8 && (1u << a.log_units) < per_row && (a.log_units < 5 || (uint64_t)kRows * (accept::kDropThreads >> a.log_units) > a.rows)) ++a.log_units;
  const uint64_t wide = (per_row + (1u << a.log_units) - 1) >> a.log_units, each = (uint64_t)kRows * (accept::kDropThreads >> a.log_units);
  // a few blocks for each SM, which take groups of rows in turn: what they work out once serves all of them
  const uint64_t high = (a.rows + each - 1) / each, most = wide < 8 * 148 ? 8 * 148 / wide : 1;
  ACCEPT_LAUNCH(accept::launch_overlapped(fn, dim3((unsigned)wide, (unsigned)(high < most ? high : most)), accept::kDropThreads, s, a));
  return ACCEPT_OK;
}

}  // extern "C"
