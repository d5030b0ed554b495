// Host side of the block-scaled matrix product (accept_block_matmul): argument checks.
#include "accept_matmul_host.cuh"

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_matmul_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_matmul_check_params(const accept_matmul_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  if (!accept::matmul_sizes_fit(p)) return ACCEPT_ERR_BAD_SIZE;
  for (int32_t f : {p->format_a, p->format_b})
    if (f != ACCEPT_FORMAT_E4M3 && f != ACCEPT_FORMAT_E5M2) return ACCEPT_ERR_BAD_ENUM;
  return accept::matmul_enums_fit(p) ? ACCEPT_OK : ACCEPT_ERR_BAD_ENUM;
}

size_t accept_matmul_workspace_size(const accept_matmul_params* p) {
  return accept_matmul_check_params(p) == ACCEPT_OK ? accept::matmul_workspace<accept::EightBit>(p) : 0;
}

accept_status accept_block_matmul(const accept_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b,
                                  const void* d_b_scale, const float* d_bias, void* d_d, void* d_ws, size_t ws_bytes,
                                  void* cuda_stream) {
  if (!p || !d_ws) return ACCEPT_ERR_NULL;
  const accept_status st = accept_matmul_check_params(p);
  if (st != ACCEPT_OK) return st;
  return accept::matmul<accept::EightBit>(p, d_a, d_a_scale, d_b, d_b_scale, d_bias, d_d, d_ws, ws_bytes, cuda_stream);
}

}  // extern "C"
