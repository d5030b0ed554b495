// What the host sides of the products of 8-bit and of 4-bit operands share: plans, tensor maps, launches.
#pragma once
#include <chrono>

#include "accept_host.cuh"
#include "accept_matmul.cuh"

namespace accept {


constexpr unsigned kMatmulSms = 148;

inline size_t matmul_value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
inline uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// The driver's encoder of tensor maps, asked for once: the library does not link the driver.
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeFn tensor_map_encoder() {
  static std::atomic<EncodeFn> found{nullptr};
  EncodeFn fn = found.load(std::memory_order_acquire);
  if (fn) return fn;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult result;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &result) != cudaSuccess ||
      result != cudaDriverEntryPointSuccess)
    return nullptr;
  fn = reinterpret_cast<EncodeFn>(p);
  found.store(fn, std::memory_order_release);
  return fn;
}

// Groups of 512 bytes of scales along k.
template <typename Op> constexpr uint64_t scale_groups(uint64_t k) {
  const uint64_t each = Op::kValues * Op::kServes / Op::kGroups;
  return (k + each - 1) / each;
}
// Bytes of a coded row, and from one to the next.
template <typename Op> constexpr uint64_t row_bytes(uint64_t k) { return Op::kGroups == 1 ? k : up(k, 32) / 2; }
template <typename Op> constexpr uint64_t row_step(uint64_t k) { return Op::kGroups == 1 ? up(k, 16) : up(k, 32) / 2; }

// Boxes of 128 bytes of k by `box_rows` rows of a coded matrix, 128-byte swizzle, zeros outside.
template <typename Op>
bool operand_map(CUtensorMap* map, const void* codes, uint64_t rows, uint64_t k, uint32_t box_rows) {
  const EncodeFn encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {row_bytes<Op>(k), rows}, strides[1] = {row_step<Op>(k)};
  const cuuint32_t box[2] = {128, box_rows}, steps[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The scales of a coded matrix as rows of 512 bytes (128 rows and four scales of each), `box_rows` at a time.
inline bool scale_map(CUtensorMap* map, const void* scales, uint64_t atoms, uint32_t box_rows) {
  const EncodeFn encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {128, atoms}, strides[1] = {512};
  const cuuint32_t box[2] = {128, box_rows}, steps[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(scales), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pieces of 32 rows of 64 bytes of d, the span of the swizzle.
inline bool result_map(CUtensorMap* map, void* d, int32_t dtype, uint64_t m, uint64_t n, uint64_t ldd) {
  const EncodeFn encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {n, m}, strides[1] = {ldd * matmul_value_size(dtype)};
  const cuuint32_t box[2] = {64 / (cuuint32_t)matmul_value_size(dtype), 32}, steps[2] = {1, 1};
  const CUtensorMapDataType type = dtype == ACCEPT_DTYPE_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == ACCEPT_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encode(map, type, 2, d, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ---- large products: pairs of SMs ----
// Arrival counts at the start of the workspace, for 73 cut tiles of 16 warps at most.  What they hold before a call does not
// matter: a call counts from its own number on (see arrive), so a workspace can serve other calls and other entry
// points in between, without a launch that clears it.
constexpr size_t kArrivalBytes = 74 * 16 * sizeof(unsigned long long);

// A number for a call, a multiple of 8 and not 0: 61 bits that no other call of this process has and that what happens to lie
// in memory does not look like (a counter and the process' start, mixed one to one).
inline unsigned long long call_number() {
  static const uint64_t start = (uint64_t)std::chrono::system_clock::now().time_since_epoch().count() ^ (uint64_t)(uintptr_t)&start;
  static std::atomic<uint64_t> calls{0};
  constexpr uint64_t kMask = (1ull << 61) - 1;
  for (;;) {
    uint64_t v = (start + calls.fetch_add(1, std::memory_order_relaxed)) & kMask;
    v = v * 0x9e3779b97f4a7c15ull & kMask;  // odd factors and shifts to the right: one to one on 61 bits
    v ^= v >> 31;
    v = v * 0xd6e8feb86659fd93ull & kMask;
    v ^= v >> 29;
    if (v != 0) return v << 3;
  }
}

// How a product is dealt to the pairs of SMs: see matmul_pair_kernel.
struct PairPlan { unsigned nt; uint64_t tiles; unsigned pairs; uint32_t whole, parts, chunks; };

// The plan with tiles of 256 x nt, and about how many cycles it takes.
template <typename Op>
PairPlan pair_plan(const accept_matmul_params* p, unsigned nt, uint64_t* cycles) {
  PairPlan s{};
  const uint64_t blocks = up(p->k, Op::kValues) / Op::kValues, pairs = kMatmulSms / 2;
  s.nt = nt;
  s.tiles = (up(p->m, 256) / 256) * (up(p->n, nt) / nt);
  s.pairs = (unsigned)pairs;
  const uint64_t left = s.tiles % pairs;
  s.chunks = p->dtype_d == ACCEPT_DTYPE_F32 ? (uint32_t)((blocks + kChunk<Op> - 1) / kChunk<Op>) : 1;
  s.parts = 1;
  s.whole = (uint32_t)s.tiles;
  // Measured at 16 to 128 blocks of k, one to four rounds: a block of k takes about 600 cycles with 256 columns and 480
  // with 128 (whose operands' way into the SM binds it), a tile 2500 and 1500 more, the join of a cut tile 11000.  That was 8-bit operands.
  // With 4-bit ones, whose blocks are 256 values, every width, cut and the small kernel were timed on 24 products (k 171 to 40000): what these
  // figures choose was the fastest or within 4 % of it, but for four that the other kernel does sooner: 700 x 1100 x 24000 (fp32 and bf16) 30 us
  // here, 22 by small tiles; 500 x 700 x 40000 fp32 26 against 21; 512 x 512 x 4096 16 by small tiles, 11 here.
  const uint64_t block = nt == 256 ? 600 : 480, tile = nt == 256 ? 2500 : 1500, join = 11000;
  uint64_t last = left ? blocks * block + tile : 0;
  if (left != 0) {  // cut what is left so that all pairs share the last round, where the join costs less than that saves
    const uint64_t most = 6;  // parts that the join has room for
    for (uint64_t parts = s.chunks < 2 ? 2 : s.chunks; parts <= most && parts * left <= pairs && parts <= blocks; ++parts) {
      const uint64_t cost = (blocks + parts - 1) / parts * block + tile + join;
      if (cost >= last) continue;
      last = cost;
      s.parts = (uint32_t)parts;
      s.whole = (uint32_t)(s.tiles - left);
    }
  }
  if (s.tiles * s.parts < s.pairs) s.pairs = (unsigned)(s.tiles * s.parts);
  *cycles = s.tiles / pairs * (blocks * block + tile) + last;
  return s;
}
template <typename Op>
PairPlan pair_plan(const accept_matmul_params* p) {
  uint64_t large, small;
  const PairPlan a = pair_plan<Op>(p, 256, &large), b = pair_plan<Op>(p, 128, &small);
  return small < large ? b : a;
}

// ---- small products: a block for each tile of 128 x 128 (or 128 x m), or a cluster of blocks that share its k ----
inline uint64_t small_tiles(const accept_matmul_params* p) { return (up(p->m, 128) / 128) * (up(p->n, 128) / 128); }
template <typename Op>
unsigned small_parts(const accept_matmul_params* p) {
  unsigned parts = 1;
  while (parts < 8 && small_tiles(p) * parts * 2 <= kMatmulSms && up(p->k, Op::kValues) / Op::kValues >= parts * 4) parts *= 2;
  return parts;
}

// Products of up to 128 rows, whose bytes bind them, are small; others where one block for each tile does them sooner than
// the pairs.  Measured: 7500 cycles and 700 a block of k (where all SMs ask for operands; their way into the SM binds it)
// against 10000 and the plan's (1000 x 2048 x 1544: 9.0 us against 9.7; 237 x 270 x 171: 5.2 against 6.4).
template <typename Op>
bool uses_pairs(const accept_matmul_params* p) {
  if (p->k == 0 || p->m <= 128) return false;
  if (small_tiles(p) > kMatmulSms) return true;
  uint64_t large, small;
  pair_plan<Op>(p, 256, &large);
  pair_plan<Op>(p, 128, &small);
  const uint64_t parts = small_parts<Op>(p), blocks = up(p->k, Op::kValues) / Op::kValues;
  return 7500 + (blocks + parts - 1) / parts * 700 > 10000 + (small < large ? small : large);
}

inline size_t pair_partial_bytes(const PairPlan& s) { return (size_t)((s.tiles - s.whole) * s.parts * 256 * s.nt * 4); }

template <typename Op, int NT>
cudaError_t launch_pair_kernel(bool single, unsigned pairs, cudaStream_t s, const CUtensorMap& map_a, const CUtensorMap& map_b, const CUtensorMap& map_sa,
                               const CUtensorMap& map_sb, const CUtensorMap& map_d, const PairArgs& a) {
  constexpr int kBytes = PairShape<Op, NT>::kSharedBytes;
  auto fn = single ? matmul_pair_kernel<Op, NT, true> : matmul_pair_kernel<Op, NT, false>;
  const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  if (err != cudaSuccess) return err;
  return launch_overlapped_shared(fn, dim3(2 * pairs), PairShape<Op, NT>::kThreads, kBytes, s, map_a, map_b, map_sa, map_sb, map_d, a);
}

template <typename Op>
accept_status launch_pairs(const accept_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b, const void* d_b_scale,
                           const MatmulArgs& base, uint8_t* d_ws, cudaStream_t s) {
  const PairPlan plan = pair_plan<Op>(p);
  PairArgs a{};
  a.bias = base.bias;
  a.d = base.d;
  a.status = base.status;
  a.arrivals = reinterpret_cast<unsigned long long*>(d_ws + 16);
  a.call = plan.parts > 1 ? call_number() : 0;
  a.partials = reinterpret_cast<float*>(d_ws + 16 + kArrivalBytes);
  a.ldd = base.ldd;
  a.dtype_d = base.dtype_d;
  a.accumulate = base.accumulate;
  a.m = (uint32_t)p->m;
  a.n = (uint32_t)p->n;
  a.blocks = (uint32_t)(up(p->k, Op::kValues) / Op::kValues);
  a.atoms_a = (uint32_t)(up(p->m, 128) / 128);
  a.atoms_b = (uint32_t)(up(p->n, 128) / 128);
  a.tiles_m = (uint32_t)(up(p->m, 256) / 256);
  a.tiles_n = (uint32_t)(up(p->n, plan.nt) / plan.nt);
  a.whole = plan.whole;
  a.parts = plan.parts;
  a.chunks = plan.chunks;
  a.instruction = Op::instruction((uint32_t)p->format_a, (uint32_t)p->format_b, 256, plan.nt);
  const bool single = p->dtype_d == ACCEPT_DTYPE_F32;
  // Tile stores: 16-byte aligned rows, nothing to add but in fp32.  A tile store ends at a multiple of 16 bytes: where d's rows
  // do not, its last unit would go over what lies behind the row's n values, so the piece (64 bytes of a row) that holds the end of
  // the row is stored value by value.
  const uint64_t size = matmul_value_size(p->dtype_d);
  if (is_aligned(a.d, 16) && a.ldd * size % 16 == 0 && (single || !a.accumulate))
    a.tile_columns = (uint32_t)(p->n * size % 16 == 0 ? p->n : p->n / (64 / size) * (64 / size));
  a.word_stores = is_aligned(a.d, 4) && a.ldd % 2 == 0;
  const uint64_t groups = scale_groups<Op>(p->k);
  CUtensorMap map_a, map_b, map_sa, map_sb, map_d{};
  if (!operand_map<Op>(&map_a, d_a, p->m, p->k, 128) || !operand_map<Op>(&map_b, d_b, p->n, p->k, plan.nt / 2) ||
      !scale_map(&map_sa, d_a_scale, groups * a.atoms_a, 1) || !scale_map(&map_sb, d_b_scale, groups * a.atoms_b, plan.nt / 128) ||
      (a.tile_columns && !result_map(&map_d, a.d, p->dtype_d, p->m, p->n, a.ldd)))
    return ACCEPT_ERR_CUDA;
  if (plan.nt == 256) ACCEPT_LAUNCH((launch_pair_kernel<Op, 256>(single, plan.pairs, s, map_a, map_b, map_sa, map_sb, map_d, a)));
  else ACCEPT_LAUNCH((launch_pair_kernel<Op, 128>(single, plan.pairs, s, map_a, map_b, map_sa, map_sb, map_d, a)));
  return ACCEPT_OK;
}

template <typename Op, int NT>
cudaError_t launch_small(const CUtensorMap& map_a, const CUtensorMap& map_b, const MatmulArgs& a, unsigned tiles, unsigned parts, cudaStream_t s) {
  // 16-bit results are rounded by 2^-9 or 2^-12 in the end: one run does for them
  const bool chunks = a.dtype_d == ACCEPT_DTYPE_F32 && (a.blocks + parts - 1) / parts > kChunk<Op>;
  auto fn = chunks ? matmul_small_kernel<Op, NT, true> : matmul_small_kernel<Op, NT, false>;
  const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallShared);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles, parts, 1);
  cfg.blockDim = dim3(kSmallThreads, 1, 1);
  cfg.dynamicSmemBytes = kSmallShared;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = parts;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, fn, map_a, map_b, a);
}

inline bool matmul_sizes_fit(const accept_matmul_params* p) {
  if (p->m > 0x7fffffffull || p->n > 0x7fffffffull || p->k > 0x7fffffffull || p->ldd < p->n || p->ldd > (1ull << 40)) return false;
  return (up(p->m, 128) / 128) * (up(p->n, 128) / 128) <= 0x7fffffffull && p->m * p->n / 256 <= 0x7ffffff0ull;
}
inline bool matmul_enums_fit(const accept_matmul_params* p) {
  return (p->dtype_d == ACCEPT_DTYPE_F32 || p->dtype_d == ACCEPT_DTYPE_BF16 || p->dtype_d == ACCEPT_DTYPE_F16) && (p->accumulate == 0 || p->accumulate == 1);
}

// Of a valid p.
template <typename Op>
size_t matmul_workspace(const accept_matmul_params* p) {
  if (!uses_pairs<Op>(p)) return 16;
  const PairPlan s = pair_plan<Op>(p);
  return 16 + (s.parts > 1 ? kArrivalBytes + pair_partial_bytes(s) : 0);
}

// The product of a valid p: checks of the pointers, then the kernel.
template <typename Op>
accept_status matmul(const accept_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b, const void* d_b_scale, const float* d_bias,
                     void* d_d, void* d_ws, size_t ws_bytes, void* cuda_stream) {
  if (ws_bytes < matmul_workspace<Op>(p)) return ACCEPT_ERR_TOO_SMALL;
  if (p->m == 0 || p->n == 0) return ACCEPT_OK;
  if (!d_d || (p->k != 0 && (!d_a || !d_a_scale || !d_b || !d_b_scale))) return ACCEPT_ERR_NULL;
  if (!is_aligned(d_a, 16) || !is_aligned(d_a_scale, 16) || !is_aligned(d_b, 16) || !is_aligned(d_b_scale, 16) || !is_aligned(d_bias, 4) ||
      !is_aligned(d_d, matmul_value_size(p->dtype_d)) || !is_aligned(d_ws, 16))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  MatmulArgs a{};
  a.bias = d_bias;
  a.d = d_d;
  a.status = static_cast<uint32_t*>(d_ws);
  a.ldd = p->ldd;
  a.dtype_d = p->dtype_d;
  a.accumulate = p->accumulate;
  ACCEPT_BOUNDS(s, bounds_list.add(d_bias, 4 * p->n, false); bounds_list.add(d_d, ((p->m - 1) * p->ldd + p->n) * matmul_value_size(p->dtype_d), true);
                bounds_list.add(d_ws, matmul_workspace<Op>(p), true));
  a.m = (uint32_t)p->m;
  a.n = (uint32_t)p->n;
  if (p->k == 0) {
    ACCEPT_LAUNCH(launch_overlapped(matmul_empty_kernel<256>, dim3((unsigned)((p->m * p->n + 255) / 256)), 256, s, a));
    return ACCEPT_OK;
  }
  if (uses_pairs<Op>(p)) return launch_pairs<Op>(p, d_a, d_a_scale, d_b, d_b_scale, a, static_cast<uint8_t*>(d_ws), s);

  const unsigned nt = p->m <= 16 ? 16 : p->m <= 32 ? 32 : p->m <= 64 ? 64 : 128;
  a.scale_a = static_cast<const uint8_t*>(d_b_scale);
  a.scale_b = static_cast<const uint8_t*>(d_a_scale);
  a.blocks = (uint32_t)(up(p->k, Op::kValues) / Op::kValues);
  a.groups = (uint32_t)scale_groups<Op>(p->k);
  a.atoms_a = (uint32_t)(up(p->n, 128) / 128);
  a.atoms_b = (uint32_t)(up(p->m, 128) / 128);
  a.tiles = a.atoms_a;
  a.instruction = Op::instruction((uint32_t)p->format_b, (uint32_t)p->format_a, 128, nt);
  a.wide_stores = !a.accumulate && is_aligned(a.d, 4 * matmul_value_size(p->dtype_d)) && a.ldd % 4 == 0;
  CUtensorMap map_a, map_b;
  if (!operand_map<Op>(&map_a, d_b, p->n, p->k, 128) || !operand_map<Op>(&map_b, d_a, p->m, p->k, nt)) return ACCEPT_ERR_CUDA;
  const unsigned tiles = a.tiles * (unsigned)(up(p->m, nt) / nt);
  const unsigned parts = small_parts<Op>(p);
  if (nt == 16) ACCEPT_LAUNCH((launch_small<Op, 16>(map_a, map_b, a, tiles, parts, s)));
  else if (nt == 32) ACCEPT_LAUNCH((launch_small<Op, 32>(map_a, map_b, a, tiles, parts, s)));
  else if (nt == 64) ACCEPT_LAUNCH((launch_small<Op, 64>(map_a, map_b, a, tiles, parts, s)));
  else ACCEPT_LAUNCH((launch_small<Op, 128>(map_a, map_b, a, tiles, parts, s)));
  return ACCEPT_OK;
}

}  // namespace accept
