// What the host sides of the root-mean-square norm's two passes share: launch shapes, how rows lie, arguments.
#pragma once
#include "accept_drop_host.cuh"
#include "accept_rms.cuh"

namespace accept {

constexpr unsigned kRmsSms = 148;

inline size_t rms_value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
// rows that all start on 16-byte boundaries
inline bool rms_whole_rows(const void* p, uint64_t ld, int32_t dtype) { return is_aligned(p, 16) && (!p || ld * rms_value_size(dtype) % 16 == 0); }

// Launch shape of a pass, as layer norm's: a row is shared by as many warps as hold it at 16 columns a thread, a block holds
// as many such groups as fit 512 threads, fewer where there are too few rows for every SM.  Rows of up to 128 columns take
// eight lanes each, rows of more than 8192 a block that reads them twice (wide).
constexpr int kRmsOwn = 16;
struct RmsShape { bool wide; int lanes; unsigned warps, groups, blocks; bool joins; size_t shared; };

// Rows of a group in shared memory: up to 144 KB for the block, and 16 bytes more for each row of a warp (of eight lanes where
// those share it), tensor and stage where rows are not aligned: 64 rows of eight lanes, three tensors, four stages at most.
constexpr int kRmsRing = 147456, kRmsMostShared = kRmsRing + 64 * 16 * 3 * 4;
// Rows ahead of the one in work, and it.  Up to three of less than 64 KB; of longer ones (for 8192 columns) that one alone, while
// the block's other group computes: 16384 x 4096, fp32 both, forward 181 us with two, 166 with one; fp32 and bf16, backward 177 and
// 168.  fp32 and bf16, forward, with two, three and four (192 KB): dropped branch to codes 124, 125, 112, without dropout 132 each, without a
// branch 61, 61, 63; to bf16 140, 140, 140, without a branch 63, 62, 65.
constexpr int rms_stages_for(int bytes) {  // of a column in all tensors that a pass reads
  return 512 * kRmsOwn * bytes >= 65536 ? 1 : kRmsRing / (512 * kRmsOwn * bytes) < 4 ? kRmsRing / (512 * kRmsOwn * bytes) : 4;
}
inline int rms_column_bytes(const accept_rms_norm_params* p, bool backward) {
  return (int)((backward ? 2 : 1) * rms_value_size(p->dtype_x) + rms_value_size(p->dtype_y));
}

// whole: rows start on 16-byte boundaries; streams_x, streams_y: tensors of each type that the pass reads.
inline RmsShape rms_shape(const accept_rms_norm_params* p, bool backward, bool whole, int streams_x, int streams_y) {
  RmsShape s{};
  s.wide = p->cols > 8192;
  if (s.wide) {
    s.blocks = (unsigned)(p->rows < 2 * kRmsSms ? p->rows : 2 * kRmsSms);
    return s;
  }
  s.lanes = p->cols <= 128 ? 8 : 32;
  s.warps = (unsigned)((p->cols + s.lanes * kRmsOwn - 1) / (s.lanes * kRmsOwn));
  const uint64_t most = 512 / (s.lanes * s.warps);
  // so few rows that eight blocks take them in two turns: one cluster, which adds up dgamma itself and saves the launch that joins
  s.joins = backward && p->cols <= 2048 && p->rows != 0 && p->rows <= 16 * most && p->rows <= 256;
  const uint64_t over = s.joins ? 8 : kRmsSms, spread = (p->rows + over - 1) / over;
  s.groups = (unsigned)(spread < most ? (spread ? spread : 1) : most);
  if (s.lanes < 32) s.groups = (s.groups + 3) / 4 * 4;  // whole warps
  const int v = whole ? 4 : 2;  // as row_space has it
  const auto space = [&](int32_t dtype) {
    return (size_t)(dtype == ACCEPT_DTYPE_F32 ? row_space<float>(v, kRmsOwn, s.lanes, s.warps) : row_space<uint16_t>(v, kRmsOwn, s.lanes, s.warps));
  };
  s.shared = s.groups * (size_t)rms_stages_for(rms_column_bytes(p, backward)) * (streams_x * space(p->dtype_x) + streams_y * space(p->dtype_y));
  const size_t sums = backward ? 4 * (size_t)kRmsOwn * s.lanes * s.warps * s.groups : 0;  // the column sums of the block's groups take the same memory
  if (s.shared < sums) s.shared = sums;
  const uint64_t units = (p->rows + s.groups - 1) / s.groups;
  s.blocks = (unsigned)(units < over ? units : over);
  return s;
}

// Partial sums of dgamma that the backward pass leaves in the workspace: one for each block, or for each slab of 256 rows.
inline uint64_t rms_partials(const accept_rms_norm_params* p, const RmsShape& s) {
  if (!s.wide) return s.joins ? 0 : s.blocks;
  const uint64_t slabs = (p->rows + 255) / 256;
  return slabs < 32 ? slabs : 32;
}

using RmsKernel = void (*)(const RmsArgs);

// The kernel of the pass that Pass<TX, TY> has for these types, rows and widths.  A thread takes eight columns side by side, four
// where a tensor is fp32 (16 bytes at most).
template <template <typename, typename> class Pass, typename TX, typename TY>
RmsKernel rms_kernel_of(const RmsShape& s, bool whole) {
  using P = Pass<TX, TY>;
  constexpr int kUnit = sizeof(TX) == 2 && sizeof(TY) == 2 ? 8 : 4;
  if (s.wide) return whole ? P::template wide<true>() : P::template wide<false>();
  if (whole) return s.lanes == 32 ? P::template held<kUnit, 32, false>() : P::template held<kUnit, 8, false>();
  return s.lanes == 32 ? P::template held<kUnit, 32, true>() : P::template held<kUnit, 8, true>();
}
template <template <typename, typename> class Pass, typename TX>
RmsKernel rms_kernel_y(const accept_rms_norm_params* p, const RmsShape& s, bool whole) {
  switch (p->dtype_y) {
    case ACCEPT_DTYPE_F32: return rms_kernel_of<Pass, TX, float>(s, whole);
    case ACCEPT_DTYPE_BF16: return rms_kernel_of<Pass, TX, __nv_bfloat16>(s, whole);
    default: return rms_kernel_of<Pass, TX, __half>(s, whole);
  }
}
template <template <typename, typename> class Pass>
RmsKernel rms_kernel(const accept_rms_norm_params* p, const RmsShape& s, bool whole) {
  switch (p->dtype_x) {
    case ACCEPT_DTYPE_F32: return rms_kernel_y<Pass, float>(p, s, whole);
    case ACCEPT_DTYPE_BF16: return rms_kernel_y<Pass, __nv_bfloat16>(p, s, whole);
    default: return rms_kernel_y<Pass, __half>(p, s, whole);
  }
}

inline cudaError_t launch_rms(RmsKernel fn, const RmsShape& shape, RmsArgs& a, cudaStream_t s) {
  a.warps = shape.warps;
  a.joins = shape.joins;
  const unsigned threads = shape.wide ? kWideThreads : shape.lanes * shape.warps * shape.groups;
  if (shape.shared > 32 * 1024) {
    // with the static part, more than a kernel gets without asking; the kernel's limit is the process': always the same, so that
    // another thread's call of other sizes cannot lower it before this one's launch
    const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kRmsMostShared);
    if (err != cudaSuccess) return err;
  }
  if (!shape.joins) return launch_overlapped_shared(fn, dim3(shape.blocks), threads, shape.shared, s, a);
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

inline RmsArgs rms_args(const accept_rms_norm_params* p, const void* d_gamma) {
  RmsArgs a{};
  a.gamma = d_gamma;
  a.rows = p->rows;
  a.cols = (uint32_t)p->cols;
  a.ld_x = p->ld_x;
  a.ld_y = p->ld_y;
  a.eps = p->eps;
  a.inv_cols = 1.0f / (float)p->cols;
  a.dtype_w = p->dtype_w;
  a.whole_weights = is_aligned(d_gamma, 16);
  a.drop = drop_of(p->p, p->seed, p->rng_offset);
  return a;
}

inline uint64_t rms_matrix_bytes(const accept_rms_norm_params* p, uint64_t ld, int32_t dtype) {
  return p->rows ? ((p->rows - 1) * ld + p->cols) * rms_value_size(dtype) : 0;
}

}  // namespace accept
