// Host side of the product of 4-bit operands (accept_micro_matmul): argument checks.
#include "accept_matmul_host.cuh"

namespace {

accept_matmul_params product_of(const accept_micro_matmul_params* p) {
  return {p->m, p->n, p->k, p->ldd, 0, 0, p->dtype_d, p->accumulate};
}

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_micro_matmul_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_micro_matmul_check_params(const accept_micro_matmul_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  const accept_matmul_params q = product_of(p);
  if (!accept::matmul_sizes_fit(&q)) return ACCEPT_ERR_BAD_SIZE;
  return accept::matmul_enums_fit(&q) ? ACCEPT_OK : ACCEPT_ERR_BAD_ENUM;
}

size_t accept_micro_matmul_workspace_size(const accept_micro_matmul_params* p) {
  if (accept_micro_matmul_check_params(p) != ACCEPT_OK) return 0;
  const accept_matmul_params q = product_of(p);
  return accept::matmul_workspace<accept::FourBit>(&q);
}

accept_status accept_micro_matmul(const accept_micro_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b,
                                const void* d_b_scale, const float* d_bias, void* d_d, void* d_ws, size_t ws_bytes, void* cuda_stream) {
  if (!p || !d_ws) return ACCEPT_ERR_NULL;
  const accept_status st = accept_micro_matmul_check_params(p);
  if (st != ACCEPT_OK) return st;
  const accept_matmul_params q = product_of(p);
  return accept::matmul<accept::FourBit>(&q, d_a, d_a_scale, d_b, d_b_scale, d_bias, d_d, d_ws, ws_bytes, cuda_stream);
}

}  // extern "C"
