// Host side of layer norm (accept_layer_norm_*): argument checks, launch shapes, launches.
#include "accept_host.cuh"
#include "accept_norm.cuh"

namespace {

using accept::is_aligned;
using accept::launch_overlapped;
using accept::NormArgs;

constexpr unsigned kSms = 148;
uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

size_t value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == ACCEPT_DTYPE_F32 || d == ACCEPT_DTYPE_BF16 || d == ACCEPT_DTYPE_F16; }

// rows that all start on 16-byte boundaries, or on 4-byte ones
bool whole_rows(const void* p, uint64_t ld, int32_t dtype) { return is_aligned(p, 16) && ld * value_size(dtype) % 16 == 0; }
bool word_rows(const void* p, uint64_t ld, int32_t dtype) { return is_aligned(p, 4) && ld * value_size(dtype) % 4 == 0; }

// Launch shape of a pass.  A row is shared by as many warps as hold it at `own` columns a thread; a block holds as many
// such groups as fit 512 threads, fewer where there are too few rows for every SM.  16 columns a thread, 32 for rows of more
// than 8192 (32 everywhere: 16384 x 4096 fp32 to bf16 62 -> 77 us, 8 x 4096 bf16 2.6 -> 3.7 us, for want of registers: those
// kernels spill 204 to 424 bytes; 16 columns a thread none in the forward pass, 0 to 20 bytes in the backward pass).  The
// backward pass over more than 8192 columns has no registers for the sums over the rows and leaves them to a pass of their
// own (kApart); rows of more than 16384 columns are not held (kLong).  Rows of up to 128 columns take eight lanes each: with
// a warp each, 14400 x 105 bf16 took 13.4 us.
enum class NormPath { kRegisters, kApart, kLong };
struct NormShape { NormPath path; int own, lanes; unsigned warps, groups, blocks; bool joins; size_t shared; };

// Rows of a group in shared memory: up to 192 KB for the block, and 16 bytes more for each row of a warp (of eight lanes where
// those share it) and stage where rows are not aligned: 8 KB at most, for 64 rows of eight lanes, two tensors and four stages.
constexpr int kRing = 196608, kMostShared = kRing + 64 * 16 * 2 * 4;
constexpr int stages_for(bool backward, int own, int size_x, int size_y) {
  const int row = 512 * own * (size_x + (backward ? size_y : 0));
  return kRing / row < 4 ? kRing / row : 4;
}
int stages_of(const accept_layer_norm_params* p, bool backward, int own) {
  return stages_for(backward, own, p->dtype_x == ACCEPT_DTYPE_F32 ? 4 : 2, p->dtype_y == ACCEPT_DTYPE_F32 ? 4 : 2);
}

NormShape norm_shape(const accept_layer_norm_params* p, bool backward, int v) {
  NormShape s{};
  if (p->cols > 16384) {
    s.path = NormPath::kLong;
    s.blocks = (unsigned)(p->rows < kSms ? p->rows : kSms);
    return s;
  }
  s.path = backward && p->cols > 8192 ? NormPath::kApart : NormPath::kRegisters;
  s.own = p->cols > 8192 ? 32 : 16;
  s.lanes = p->cols <= 128 ? 8 : 32;
  s.warps = (unsigned)((p->cols + s.lanes * s.own - 1) / (s.lanes * s.own));
  const uint64_t most = 512 / (s.lanes * s.warps);
  // So few rows that eight blocks take them in two turns: one cluster, which adds up dgamma and dbeta itself.  That saves the
  // launch that would join them (64 x 1024 fp32: 7.4 us a call with it, the host's time for two launches, 5.6 without); the
  // cluster's own adding up outweighs it for wider rows (5 x 4356 bf16: 8.3 us against 7.4) and for more groups (640 x 79 fp16:
  // 8.9 us).
  s.joins = backward && s.path == NormPath::kRegisters && p->cols <= 2048 && p->rows != 0 && p->rows <= 16 * most && p->rows <= 256;
  const uint64_t over = s.joins ? 8 : kSms, spread = (p->rows + over - 1) / over;
  s.groups = (unsigned)(spread < most ? (spread ? spread : 1) : most);
  if (s.lanes < 32) s.groups = (unsigned)up(s.groups, 32 / s.lanes);  // whole warps
  const auto space = [&](int32_t dtype) {
    return (size_t)(dtype == ACCEPT_DTYPE_F32 ? accept::row_space<float>(v, s.own, s.lanes, s.warps)
                                              : accept::row_space<uint16_t>(v, s.own, s.lanes, s.warps));
  };
  s.shared = s.groups * (size_t)stages_of(p, backward, s.own) * (space(p->dtype_x) + (backward ? space(p->dtype_y) : 0));
  // the column sums of the block's groups take the same memory
  const size_t sums = backward && s.path == NormPath::kRegisters ? 2 * 4 * (size_t)s.own * s.lanes * s.warps * s.groups : 0;
  if (s.shared < sums) s.shared = sums;
  const uint64_t units = (p->rows + s.groups - 1) / s.groups;
  s.blocks = (unsigned)(units < over ? units : over);
  return s;
}

// Partial sums of dgamma and dbeta that the backward pass leaves in the workspace: one for each block, or for each
// slab of rows (512 at least: a slab of its own costs a launch that joins them).
uint64_t norm_partials(const accept_layer_norm_params* p, const NormShape& s) {
  if (s.path == NormPath::kRegisters) return s.joins ? 0 : s.blocks;
  const uint64_t slabs = (p->rows + 511) / 512;
  return slabs < 32 ? slabs : 32;
}

using KernelFn = void (*)(const NormArgs);
struct Kernels { KernelFn rows, sums; };

template <typename TX, typename TY, int V>
KernelFn rows_kernel(const NormShape& s, bool backward) {
  constexpr int kX = (int)sizeof(TX), kY = (int)sizeof(TY);
  if (s.path == NormPath::kLong) return backward ? accept::norm_backward_long_kernel<TX, TY> : accept::norm_forward_long_kernel<TX, TY>;
  if (!backward)
    return s.own == 32     ? accept::norm_forward_kernel<TX, TY, V, 32, 32, stages_for(false, 32, kX, kY)>
           : s.lanes == 32 ? accept::norm_forward_kernel<TX, TY, V, 16, 32, stages_for(false, 16, kX, kY)>
                           : accept::norm_forward_kernel<TX, TY, V, 16, 8, stages_for(false, 16, kX, kY)>;
  return s.own == 32     ? accept::norm_backward_kernel<TX, TY, V, 32, 32, stages_for(true, 32, kX, kY), false>
         : s.lanes == 32 ? accept::norm_backward_kernel<TX, TY, V, 16, 32, stages_for(true, 16, kX, kY), true>
                         : accept::norm_backward_kernel<TX, TY, V, 16, 8, stages_for(true, 16, kX, kY), true>;
}

template <typename TX, typename TY>
KernelFn loose_kernel(const NormShape& s, bool backward) {
  if constexpr (sizeof(TX) + sizeof(TY) < 8) return rows_kernel<TX, TY, 1>(s, backward);
  else return nullptr;  // fp32 values start on 4-byte boundaries
}

// How rows lie: all tensors' on 16-byte boundaries, or the 16-bit tensors' on 4-byte boundaries, or neither.
enum class RowStarts { kWhole, kWords, kLoose };

template <typename TX, typename TY>
Kernels kernels_for(const NormShape& s, bool backward, RowStarts starts, bool wide_sums) {
  constexpr int kUnit = sizeof(TX) == 2 && sizeof(TY) == 2 ? 8 : 4;
  return {starts == RowStarts::kWhole   ? rows_kernel<TX, TY, kUnit>(s, backward)
          : starts == RowStarts::kWords ? rows_kernel<TX, TY, 2>(s, backward) : loose_kernel<TX, TY>(s, backward),
          wide_sums ? accept::norm_column_sums_kernel<TX, TY, 4> : accept::norm_column_sums_kernel<TX, TY, 1>};
}

template <typename TX>
Kernels kernels_for_y(const accept_layer_norm_params* p, const NormShape& s, bool backward, RowStarts starts) {
  switch (p->dtype_y) {
    case ACCEPT_DTYPE_F32: return kernels_for<TX, float>(s, backward, starts, p->cols % 4 == 0 && starts == RowStarts::kWhole);
    case ACCEPT_DTYPE_BF16: return kernels_for<TX, __nv_bfloat16>(s, backward, starts, p->cols % 4 == 0 && starts == RowStarts::kWhole);
    default: return kernels_for<TX, __half>(s, backward, starts, p->cols % 4 == 0 && starts == RowStarts::kWhole);
  }
}

Kernels select_kernels(const accept_layer_norm_params* p, const NormShape& s, bool backward, RowStarts starts) {
  switch (p->dtype_x) {
    case ACCEPT_DTYPE_F32: return kernels_for_y<float>(p, s, backward, starts);
    case ACCEPT_DTYPE_BF16: return kernels_for_y<__nv_bfloat16>(p, s, backward, starts);
    default: return kernels_for_y<__half>(p, s, backward, starts);
  }
}

// Columns that a thread takes side by side (see column_of).
int unit_of(const accept_layer_norm_params* p, RowStarts starts) {
  if (starts != RowStarts::kWhole) return starts == RowStarts::kWords ? 2 : 1;
  return p->dtype_x == ACCEPT_DTYPE_F32 || p->dtype_y == ACCEPT_DTYPE_F32 ? 4 : 8;
}

cudaError_t launch_norm(KernelFn fn, const NormShape& shape, NormArgs& a, cudaStream_t s) {
  a.warps = shape.warps;
  const unsigned threads = shape.path == NormPath::kLong ? 1024 : shape.lanes * shape.warps * shape.groups;
  if (shape.shared > 32 * 1024) {  // with the static part, more than a kernel gets without asking
    // the kernel's limit is the process': always the same, so that another thread's call of other sizes cannot lower it before
    // this one's launch
    const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    if (err != cudaSuccess) return err;
  }
  if (!shape.joins) return accept::launch_overlapped_shared(fn, dim3(shape.blocks), threads, shape.shared, s, a);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(shape.blocks, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = shape.shared;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = shape.blocks;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, fn, a);
}

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
  // every offset of a value must be a 63-bit number of bytes, and the turns of a group of threads a 31-bit number
  if (p->rows > (1ull << 38) || p->ld_x > (1ull << 40) || p->ld_y > (1ull << 40) ||
      (p->rows && (p->ld_x > (1ull << 60) / p->rows || p->ld_y > (1ull << 60) / p->rows)))
    return ACCEPT_ERR_BAD_SIZE;
  if (!is_dtype(p->dtype_x) || !is_dtype(p->dtype_y) || !is_dtype(p->dtype_w)) return ACCEPT_ERR_BAD_ENUM;
  if (!(p->eps >= 0.0f) || p->eps > 3.402823466e38f) return ACCEPT_ERR_BAD_SIZE;
  return ACCEPT_OK;
}

size_t accept_layer_norm_workspace_size(const accept_layer_norm_params* p) {
  if (accept_layer_norm_check_params(p) != ACCEPT_OK) return 0;
  const NormShape s = norm_shape(p, true, 4);  // the partials depend on the rows and columns alone, not on their alignment
  return 16 + (size_t)(norm_partials(p, s) * 8 * p->cols);
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
  const RowStarts starts = whole_rows(d_x, p->ld_x, p->dtype_x) && whole_rows(d_y, p->ld_y, p->dtype_y)  ? RowStarts::kWhole
                           : word_rows(d_x, p->ld_x, p->dtype_x) && word_rows(d_y, p->ld_y, p->dtype_y) ? RowStarts::kWords : RowStarts::kLoose;
  a.whole_weights = is_aligned(d_gamma, 16) && is_aligned(d_beta, 16);
  const NormShape shape = norm_shape(p, false, unit_of(p, starts));
  ACCEPT_LAUNCH(launch_norm(select_kernels(p, shape, false, starts).rows, shape, a, s));
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
  const RowStarts starts =
      whole_rows(d_x, p->ld_x, p->dtype_x) && whole_rows(d_dy, p->ld_y, p->dtype_y) && is_aligned(d_dx, 16) ? RowStarts::kWhole
      : word_rows(d_x, p->ld_x, p->dtype_x) && word_rows(d_dy, p->ld_y, p->dtype_y) && is_aligned(d_dx, 4) ? RowStarts::kWords : RowStarts::kLoose;
  const NormShape shape = norm_shape(p, true, unit_of(p, starts));
  NormArgs a = norm_args(p);
  a.x = d_x;
  a.dy = d_dy;
  a.gamma = d_gamma;
  a.mean = d_mean;
  a.rstd = d_rstd;
  a.dx = d_dx;
  a.joins = shape.joins;
  a.partials = weights && !shape.joins ? reinterpret_cast<float*>(static_cast<uint8_t*>(d_ws) + 16) : nullptr;
  a.n_partials = (uint32_t)norm_partials(p, shape);
  a.whole_weights = is_aligned(d_gamma, 16);
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
    const Kernels k = select_kernels(p, shape, true, starts);
    const unsigned columns = p->cols % 4 == 0 && starts == RowStarts::kWhole ? 128 : 32;  // a block of the sums
    const bool apart = shape.path != NormPath::kRegisters;
    // the column sums first: dx may take the place of x or dy
    if (apart && weights) ACCEPT_LAUNCH(launch_overlapped(k.sums, dim3((a.cols + columns - 1) / columns, a.n_partials), 256, s, a));
    if (!apart || d_dx) ACCEPT_LAUNCH(launch_norm(k.rows, shape, a, s));
  }
  const bool summed = shape.joins || (shape.path != NormPath::kRegisters && p->rows != 0 && a.n_partials == 1);
  if (weights && !summed) ACCEPT_LAUNCH(launch_overlapped(accept::norm_join_kernel, dim3((unsigned)((2ull * a.cols + 31) / 32)), 32 * accept::kJoinWarps, s, a));
  return ACCEPT_OK;
}

}  // extern "C"
