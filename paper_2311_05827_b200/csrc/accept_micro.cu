// Host side of the 4-bit quantiser (accept_micro_*): argument checks, sizes, launches.
#include "accept_host.cuh"
#include "accept_micro.cuh"

namespace {

using accept::is_aligned;
using accept::launch_overlapped;
using accept::MicroArgs;
using accept::MicroValueArgs;

size_t value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

using KernelFn = void (*)(const MicroArgs);
struct Kernel { KernelFn fn; unsigned threads; };
using accept::MicroRound;
template <typename T, MicroRound ROUND>
Kernel select_rows(bool whole) {
  return {whole ? accept::micro_quantize_kernel<T, ROUND, true> : accept::micro_quantize_kernel<T, ROUND, false>, (unsigned)accept::kMicroThreads<T, ROUND>};
}
template <typename T>
Kernel select_round(MicroRound round, bool whole) {
  return round == MicroRound::kNearest ? select_rows<T, MicroRound::kNearest>(whole)
         : round == MicroRound::kQuads ? select_rows<T, MicroRound::kQuads>(whole) : select_rows<T, MicroRound::kAnywhere>(whole);
}
Kernel select_kernel(const accept_micro_params* p, bool whole) {
  const MicroRound round = p->round == ACCEPT_ROUND_NEAREST ? MicroRound::kNearest
                           : p->cols % 4 == 0 && p->rng_offset % 4 == 0 ? MicroRound::kQuads : MicroRound::kAnywhere;
  switch (p->dtype) {
    case ACCEPT_DTYPE_F32: return select_round<float>(round, whole);
    case ACCEPT_DTYPE_BF16: return select_round<__nv_bfloat16>(round, whole);
    default: return select_round<__half>(round, whole);
  }
}

constexpr int kRows = 4;
using ValueFn = void (*)(const MicroValueArgs);
template <typename T>
ValueFn select_values(bool whole) { return whole ? accept::micro_dequantize_kernel<T, true, kRows> : accept::micro_dequantize_kernel<T, false, kRows>; }

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_micro_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_micro_check_params(const accept_micro_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  if (p->rows > 0x7fffffffull || p->cols > 0x7fffffffull || p->ld < p->cols || p->ld > (1ull << 40)) return ACCEPT_ERR_BAD_SIZE;
  // one block of threads for each tile must fit the grid's x dimension
  if ((up(p->rows, 128) / 128) * (up(p->cols, 128) / 128) > 0x7fffffffull) return ACCEPT_ERR_BAD_SIZE;
  if (p->dtype != ACCEPT_DTYPE_F32 && p->dtype != ACCEPT_DTYPE_BF16 && p->dtype != ACCEPT_DTYPE_F16) return ACCEPT_ERR_BAD_ENUM;
  if (p->round != ACCEPT_ROUND_NEAREST && p->round != ACCEPT_ROUND_STOCHASTIC) return ACCEPT_ERR_BAD_ENUM;
  if ((p->block != ACCEPT_BLOCK_ROW && p->block != ACCEPT_BLOCK_SQUARE) || p->reserved != 0) return ACCEPT_ERR_BAD_ENUM;
  return ACCEPT_OK;
}

size_t accept_micro_data_size(const accept_micro_params* p, int transposed) {
  if (accept_micro_check_params(p) != ACCEPT_OK) return 0;
  return transposed ? (size_t)(p->cols * (up(p->rows, 32) / 2)) : (size_t)(p->rows * (up(p->cols, 32) / 2));
}

size_t accept_micro_scale_size(const accept_micro_params* p, int transposed) {
  if (accept_micro_check_params(p) != ACCEPT_OK) return 0;
  return (size_t)(512 * (up(p->rows, 128) / 128) * (up(p->cols, 128) / 128));  // the same both ways
}

size_t accept_micro_workspace_size(const accept_micro_params* p) { return accept_micro_check_params(p) == ACCEPT_OK ? 16 : 0; }

accept_status accept_micro_quantize(const accept_micro_params* p, const void* d_x, void* d_q, void* d_scale, void* d_qt, void* d_scale_t,
                                  void* d_ws, size_t ws_bytes, void* cuda_stream) {
  if (!p || !d_ws) return ACCEPT_ERR_NULL;
  const accept_status st = accept_micro_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (ws_bytes < 16) return ACCEPT_ERR_TOO_SMALL;
  if (p->rows == 0 || p->cols == 0) return ACCEPT_OK;
  if (!d_x || (!d_q && !d_qt) || !d_q != !d_scale || !d_qt != !d_scale_t) return ACCEPT_ERR_NULL;
  if (!is_aligned(d_x, value_size(p->dtype)) || !is_aligned(d_q, 16) || !is_aligned(d_scale, 16) || !is_aligned(d_qt, 16) ||
      !is_aligned(d_scale_t, 16) || !is_aligned(d_ws, 4))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  MicroArgs a{};
  a.x = d_x;
  a.q = static_cast<uint8_t*>(d_q);
  a.scale = static_cast<uint8_t*>(d_scale);
  a.qt = static_cast<uint8_t*>(d_qt);
  a.scale_t = static_cast<uint8_t*>(d_scale_t);
  a.status = static_cast<uint32_t*>(d_ws);
  a.ld = p->ld;
  a.offset = p->rng_offset;
  a.rng.seed_lo = (uint32_t)p->seed;
  a.rng.seed_hi = (uint32_t)(p->seed >> 32);
  a.rows = (uint32_t)p->rows;
  a.cols = (uint32_t)p->cols;
  a.ldq = (uint32_t)(up(p->cols, 32) / 2);
  a.ldqt = (uint32_t)(up(p->rows, 32) / 2);
  a.tiles_r = (uint32_t)(up(p->rows, 128) / 128);
  a.tiles_c = (uint32_t)(up(p->cols, 128) / 128);
  a.square = p->block == ACCEPT_BLOCK_SQUARE;
  ACCEPT_BOUNDS(s, bounds_list.add(d_x, ((p->rows - 1) * p->ld + p->cols) * value_size(p->dtype), false);
                bounds_list.add(d_q, accept_micro_data_size(p, 0), true); bounds_list.add(d_scale, accept_micro_scale_size(p, 0), true);
                bounds_list.add(d_qt, accept_micro_data_size(p, 1), true); bounds_list.add(d_scale_t, accept_micro_scale_size(p, 1), true);
                bounds_list.add(d_ws, 16, true));
  const bool whole = is_aligned(d_x, 16) && p->ld * value_size(p->dtype) % 16 == 0;
  const Kernel kernel = select_kernel(p, whole);
  ACCEPT_LAUNCH(launch_overlapped(kernel.fn, dim3(a.tiles_r * a.tiles_c), kernel.threads, s, a));
  return ACCEPT_OK;
}

accept_status accept_micro_dequantize(const accept_micro_params* p, const void* d_q, const void* d_scale, void* d_x, void* cuda_stream) {
  if (!p) return ACCEPT_ERR_NULL;
  const accept_status st = accept_micro_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (p->rows == 0 || p->cols == 0) return ACCEPT_OK;
  if (!d_q || !d_scale || !d_x) return ACCEPT_ERR_NULL;
  if (!is_aligned(d_q, 16) || !is_aligned(d_scale, 16) || !is_aligned(d_x, value_size(p->dtype))) return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  MicroValueArgs a{};
  a.q = static_cast<const uint8_t*>(d_q);
  a.scale = static_cast<const uint8_t*>(d_scale);
  a.x = d_x;
  a.ld = p->ld;
  a.rows = (uint32_t)p->rows;
  a.cols = (uint32_t)p->cols;
  a.ldq = (uint32_t)(up(p->cols, 32) / 2);
  a.atoms = (uint32_t)(up(p->rows, 128) / 128);
  ACCEPT_BOUNDS(s, bounds_list.add(d_q, accept_micro_data_size(p, 0), false); bounds_list.add(d_scale, accept_micro_scale_size(p, 0), false);
                bounds_list.add(d_x, ((p->rows - 1) * p->ld + p->cols) * value_size(p->dtype), true));
  const bool whole = is_aligned(d_x, 16) && p->ld * value_size(p->dtype) % 16 == 0;
  const ValueFn fn = p->dtype == ACCEPT_DTYPE_F32 ? select_values<float>(whole) : p->dtype == ACCEPT_DTYPE_BF16 ? select_values<__nv_bfloat16>(whole) : select_values<__half>(whole);
  // Units start on x's 16-byte boundaries: one more than the columns fill where a row does not.  A warp takes neighbours of one row
  // where there are so many; a few blocks for each SM take groups of rows in turn.
  const uint64_t per_row = (p->cols + (whole ? 0 : 16 / value_size(p->dtype) - 1) + 7) / 8;
  while (a.log_units < 5 && (1u << a.log_units) < per_row) ++a.log_units;
  const uint64_t wide = (per_row + (1u << a.log_units) - 1) >> a.log_units, each = (uint64_t)kRows * (accept::kValueThreads >> a.log_units);
  const uint64_t high = (p->rows + each - 1) / each, most = wide < 16 * 148 ? 16 * 148 / wide : 1;
  ACCEPT_LAUNCH(launch_overlapped(fn, dim3((unsigned)wide, (unsigned)(high < most ? high : most)), accept::kValueThreads, s, a));
  return ACCEPT_OK;
}

}  // extern "C"
