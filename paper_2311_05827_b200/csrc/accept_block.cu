// Host side of the block quantiser (accept_block_*): argument checks, sizes, launches.
#include "accept_host.cuh"
#include "accept_block.cuh"

namespace {

using accept::BlockArgs;
using accept::is_aligned;
using accept::launch_overlapped;

size_t value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

using KernelFn = void (*)(const BlockArgs);

template <typename T>
KernelFn select_format(int32_t format, bool whole) {
  if (format == ACCEPT_FORMAT_E4M3)
    return whole ? accept::block_quantize_kernel<T, accept::kE4m3, true> : accept::block_quantize_kernel<T, accept::kE4m3, false>;
  return whole ? accept::block_quantize_kernel<T, accept::kE5m2, true> : accept::block_quantize_kernel<T, accept::kE5m2, false>;
}

KernelFn select_kernel(const accept_quantize_params* p, bool whole) {
  switch (p->dtype) {
    case ACCEPT_DTYPE_F32: return select_format<float>(p->format, whole);
    case ACCEPT_DTYPE_BF16: return select_format<__nv_bfloat16>(p->format, whole);
    default: return select_format<__half>(p->format, whole);
  }
}

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_block_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_block_check_params(const accept_quantize_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  if (p->rows > 0x7fffffffull || p->cols > 0x7fffffffull || p->ld < p->cols || p->ld > (1ull << 40)) return ACCEPT_ERR_BAD_SIZE;
  // one block of threads for each tile must fit the grid's x dimension
  if ((up(p->rows, 128) / 128) * (up(p->cols, 128) / 128) > 0x7fffffffull) return ACCEPT_ERR_BAD_SIZE;
  if (p->dtype != ACCEPT_DTYPE_F32 && p->dtype != ACCEPT_DTYPE_BF16 && p->dtype != ACCEPT_DTYPE_F16) return ACCEPT_ERR_BAD_ENUM;
  if (p->format != ACCEPT_FORMAT_E4M3 && p->format != ACCEPT_FORMAT_E5M2) return ACCEPT_ERR_BAD_ENUM;
  if ((p->block != ACCEPT_BLOCK_ROW && p->block != ACCEPT_BLOCK_SQUARE) || p->reserved != 0) return ACCEPT_ERR_BAD_ENUM;
  return ACCEPT_OK;
}

size_t accept_block_data_size(const accept_quantize_params* p, int transposed) {
  if (accept_block_check_params(p) != ACCEPT_OK) return 0;
  return transposed ? (size_t)(p->cols * up(p->rows, 16)) : (size_t)(p->rows * up(p->cols, 16));
}

size_t accept_block_scale_size(const accept_quantize_params* p, int transposed) {
  if (accept_block_check_params(p) != ACCEPT_OK) return 0;
  const uint64_t r = transposed ? p->cols : p->rows, c = transposed ? p->rows : p->cols;
  return (size_t)(512 * (up(r, 128) / 128) * (up(c, 512) / 512));
}

size_t accept_block_workspace_size(const accept_quantize_params* p) { return accept_block_check_params(p) == ACCEPT_OK ? 16 : 0; }

accept_status accept_block_quantize(const accept_quantize_params* p, const void* d_x, void* d_q, void* d_scale, void* d_qt,
                                    void* d_scale_t, void* d_ws, size_t ws_bytes, void* cuda_stream) {
  if (!p || !d_ws) return ACCEPT_ERR_NULL;
  const accept_status st = accept_block_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (ws_bytes < 16) return ACCEPT_ERR_TOO_SMALL;
  if (p->rows == 0 || p->cols == 0) return ACCEPT_OK;
  if (!d_x || (!d_q && !d_qt) || !d_q != !d_scale || !d_qt != !d_scale_t) return ACCEPT_ERR_NULL;
  if (!is_aligned(d_x, value_size(p->dtype)) || !is_aligned(d_q, 16) || !is_aligned(d_scale, 16) || !is_aligned(d_qt, 16) ||
      !is_aligned(d_scale_t, 16) || !is_aligned(d_ws, 4))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  BlockArgs a{};
  a.x = d_x;
  a.q = static_cast<uint8_t*>(d_q);
  a.scale = static_cast<uint8_t*>(d_scale);
  a.qt = static_cast<uint8_t*>(d_qt);
  a.scale_t = static_cast<uint8_t*>(d_scale_t);
  a.status = static_cast<uint32_t*>(d_ws);
  a.ld = p->ld;
  a.rows = (uint32_t)p->rows;
  a.cols = (uint32_t)p->cols;
  a.ldq = (uint32_t)up(p->cols, 16);
  a.ldqt = (uint32_t)up(p->rows, 16);
  a.tiles_r = (uint32_t)(up(p->rows, 128) / 128);
  a.tiles_c = (uint32_t)(up(p->cols, 128) / 128);
  a.square = p->block == ACCEPT_BLOCK_SQUARE;
  ACCEPT_BOUNDS(s, bounds_list.add(d_x, ((p->rows - 1) * p->ld + p->cols) * value_size(p->dtype), false);
                bounds_list.add(d_q, accept_block_data_size(p, 0), true); bounds_list.add(d_scale, accept_block_scale_size(p, 0), true);
                bounds_list.add(d_qt, accept_block_data_size(p, 1), true); bounds_list.add(d_scale_t, accept_block_scale_size(p, 1), true);
                bounds_list.add(d_ws, 16, true));
  const bool whole = is_aligned(d_x, 16) && p->ld * value_size(p->dtype) % 16 == 0;
  ACCEPT_LAUNCH(launch_overlapped(select_kernel(p, whole), dim3(a.tiles_r * a.tiles_c), 256, s, a));
  return ACCEPT_OK;
}

}  // extern "C"
