// Host side of the block-scaled matrix product (accept_block_matmul): argument checks, tensor maps, launches.
#include <chrono>

#include "accept_host.cuh"
#include "accept_matmul.cuh"

namespace {

using accept::is_aligned;
using accept::launch_overlapped;
using accept::MatmulArgs;

constexpr unsigned kSms = 148;

size_t value_size(int32_t dtype) { return dtype == ACCEPT_DTYPE_F32 ? 4 : 2; }
uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// The driver's encoder of tensor maps, asked for once: the library does not link the driver.
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn tensor_map_encoder() {
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

// Boxes of 128 values of k by `box_rows` rows of a coded matrix, 128-byte swizzle, zeros outside.
bool operand_map(CUtensorMap* map, const void* codes, uint64_t rows, uint64_t k, uint32_t box_rows) {
  const EncodeFn encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {k, rows}, strides[1] = {up(k, 16)};
  const cuuint32_t box[2] = {128, box_rows}, steps[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The scales of a coded matrix as rows of 512 bytes (128 rows and four blocks of it each), `box_rows` at a time.
bool scale_map(CUtensorMap* map, const void* scales, uint64_t atoms, uint32_t box_rows) {
  const EncodeFn encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {128, atoms}, strides[1] = {512};
  const cuuint32_t box[2] = {128, box_rows}, steps[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(scales), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pieces of 32 rows of 64 bytes of d, the span of the swizzle.
bool result_map(CUtensorMap* map, void* d, int32_t dtype, uint64_t m, uint64_t n, uint64_t ldd) {
  const EncodeFn encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {n, m}, strides[1] = {ldd * value_size(dtype)};
  const cuuint32_t box[2] = {64 / (cuuint32_t)value_size(dtype), 32}, steps[2] = {1, 1};
  const CUtensorMapDataType type = dtype == ACCEPT_DTYPE_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == ACCEPT_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encode(map, type, 2, d, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ---- large products: pairs of SMs ----
// Arrival counts at the start of the workspace, for 73 cut tiles of 16 warps at most.  What they hold before a call does not
// matter: a call counts from its own number on (see accept::arrive), so a workspace can serve other calls and other entry
// points in between, without a launch that clears it.
constexpr size_t kArrivalBytes = 74 * 16 * sizeof(unsigned long long);

// A number for a call, a multiple of 8 and not 0: 61 bits that no other call of this process has and that what happens to lie
// in memory does not look like (a counter and the process' start, mixed one to one).
unsigned long long call_number() {
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
PairPlan pair_plan(const accept_matmul_params* p, unsigned nt, uint64_t* cycles) {
  PairPlan s{};
  const uint64_t blocks = up(p->k, 128) / 128, pairs = kSms / 2;
  s.nt = nt;
  s.tiles = (up(p->m, 256) / 256) * (up(p->n, nt) / nt);
  s.pairs = (unsigned)pairs;
  const uint64_t left = s.tiles % pairs;
  s.chunks = p->dtype_d == ACCEPT_DTYPE_F32 ? (uint32_t)((blocks + accept::kChunk - 1) / accept::kChunk) : 1;
  s.parts = 1;
  s.whole = (uint32_t)s.tiles;
  // Measured at 16 to 128 blocks of k, one to four rounds: a block of k takes about 600 cycles with 256 columns and 480
  // with 128 (whose operands' way into the SM binds it), a tile 2500 and 1500 more, the join of a cut tile 11000.
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
PairPlan pair_plan(const accept_matmul_params* p) {
  uint64_t large, small;
  const PairPlan a = pair_plan(p, 256, &large), b = pair_plan(p, 128, &small);
  return small < large ? b : a;
}

// ---- small products: a block for each tile of 128 x 128 (or 128 x m), or a cluster of blocks that share its k ----
uint64_t small_tiles(const accept_matmul_params* p) { return (up(p->m, 128) / 128) * (up(p->n, 128) / 128); }
unsigned small_parts(const accept_matmul_params* p) {
  unsigned parts = 1;
  while (parts < 8 && small_tiles(p) * parts * 2 <= kSms && up(p->k, 128) / 128 >= parts * 4) parts *= 2;
  return parts;
}

// Products of up to 128 rows, whose bytes bind them, are small; others where one block for each tile does them sooner than
// the pairs.  Measured: 7500 cycles and 700 a block of k (where all SMs ask for operands; their way into the SM binds it)
// against 10000 and the plan's (1000 x 2048 x 1544: 9.0 us against 9.7; 237 x 270 x 171: 5.2 against 6.4).
bool uses_pairs(const accept_matmul_params* p) {
  if (p->k == 0 || p->m <= 128) return false;
  if (small_tiles(p) > kSms) return true;
  uint64_t large, small;
  pair_plan(p, 256, &large);
  pair_plan(p, 128, &small);
  const uint64_t parts = small_parts(p), blocks = up(p->k, 128) / 128;
  return 7500 + (blocks + parts - 1) / parts * 700 > 10000 + (small < large ? small : large);
}

size_t pair_partial_bytes(const PairPlan& s) { return (size_t)((s.tiles - s.whole) * s.parts * 256 * s.nt * 4); }

template <int NT>
cudaError_t launch_pair_kernel(bool single, unsigned pairs, cudaStream_t s, const CUtensorMap& map_a, const CUtensorMap& map_b, const CUtensorMap& map_sa,
                               const CUtensorMap& map_sb, const CUtensorMap& map_d, const accept::PairArgs& a) {
  constexpr int kBytes = accept::PairShape<NT>::kSharedBytes;
  auto fn = single ? accept::matmul_pair_kernel<NT, true> : accept::matmul_pair_kernel<NT, false>;
  const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  if (err != cudaSuccess) return err;
  return accept::launch_overlapped_shared(fn, dim3(2 * pairs), accept::PairShape<NT>::kThreads, kBytes, s, map_a, map_b, map_sa, map_sb, map_d, a);
}

accept_status launch_pairs(const accept_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b, const void* d_b_scale,
                           const MatmulArgs& base, uint8_t* d_ws, cudaStream_t s) {
  const PairPlan plan = pair_plan(p);
  accept::PairArgs a{};
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
  a.blocks = (uint32_t)(up(p->k, 128) / 128);
  a.atoms_a = (uint32_t)(up(p->m, 128) / 128);
  a.atoms_b = (uint32_t)(up(p->n, 128) / 128);
  a.tiles_m = (uint32_t)(up(p->m, 256) / 256);
  a.tiles_n = (uint32_t)(up(p->n, plan.nt) / plan.nt);
  a.whole = plan.whole;
  a.parts = plan.parts;
  a.chunks = plan.chunks;
  a.instruction = accept::scaled_instruction((uint32_t)p->format_a, (uint32_t)p->format_b, 256, plan.nt);
  const bool single = p->dtype_d == ACCEPT_DTYPE_F32;
  // Tile stores: 16-byte aligned rows, nothing to add but in fp32.  A tile store ends at a multiple of 16 bytes: where d's rows
  // do not, its last unit would go over what lies behind the row's n values, so the piece (64 bytes of a row) that holds the end of
  // the row is stored value by value.
  const uint64_t size = value_size(p->dtype_d);
  if (is_aligned(a.d, 16) && a.ldd * size % 16 == 0 && (single || !a.accumulate))
    a.tile_columns = (uint32_t)(p->n * size % 16 == 0 ? p->n : p->n / (64 / size) * (64 / size));
  a.word_stores = is_aligned(a.d, 4) && a.ldd % 2 == 0;
  const uint64_t groups = (a.blocks + 3) / 4;
  CUtensorMap map_a, map_b, map_sa, map_sb, map_d{};
  if (!operand_map(&map_a, d_a, p->m, p->k, 128) || !operand_map(&map_b, d_b, p->n, p->k, plan.nt / 2) ||
      !scale_map(&map_sa, d_a_scale, groups * a.atoms_a, 1) || !scale_map(&map_sb, d_b_scale, groups * a.atoms_b, plan.nt / 128) ||
      (a.tile_columns && !result_map(&map_d, a.d, p->dtype_d, p->m, p->n, a.ldd)))
    return ACCEPT_ERR_CUDA;
  if (plan.nt == 256) ACCEPT_LAUNCH(launch_pair_kernel<256>(single, plan.pairs, s, map_a, map_b, map_sa, map_sb, map_d, a));
  else ACCEPT_LAUNCH(launch_pair_kernel<128>(single, plan.pairs, s, map_a, map_b, map_sa, map_sb, map_d, a));
  return ACCEPT_OK;
}

template <int NT>
cudaError_t launch_small(const CUtensorMap& map_a, const CUtensorMap& map_b, const MatmulArgs& a, unsigned tiles, unsigned parts, cudaStream_t s) {
  // 16-bit results are rounded by 2^-9 or 2^-12 in the end: one run does for them
  const bool chunks = a.dtype_d == ACCEPT_DTYPE_F32 && (a.blocks + parts - 1) / parts > accept::kChunk;
  auto fn = chunks ? accept::matmul_small_kernel<NT, true> : accept::matmul_small_kernel<NT, false>;
  const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, accept::kSmallShared);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles, parts, 1);
  cfg.blockDim = dim3(accept::kSmallThreads, 1, 1);
  cfg.dynamicSmemBytes = accept::kSmallShared;
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

}  // namespace

#ifdef ACCEPT_BOUNDS_CHECK
bool accept::collect_matmul_bounds(uint32_t* violations, unsigned long long (&first)[2]) { return collect_bounds(violations, first); }
#endif

extern "C" {

accept_status accept_matmul_check_params(const accept_matmul_params* p) {
  if (!p) return ACCEPT_ERR_NULL;
  if (p->m > 0x7fffffffull || p->n > 0x7fffffffull || p->k > 0x7fffffffull || p->ldd < p->n || p->ldd > (1ull << 40)) return ACCEPT_ERR_BAD_SIZE;
  if ((up(p->m, 128) / 128) * (up(p->n, 128) / 128) > 0x7fffffffull || p->m * p->n / 256 > 0x7ffffff0ull) return ACCEPT_ERR_BAD_SIZE;
  for (int32_t f : {p->format_a, p->format_b})
    if (f != ACCEPT_FORMAT_E4M3 && f != ACCEPT_FORMAT_E5M2) return ACCEPT_ERR_BAD_ENUM;
  if (p->dtype_d != ACCEPT_DTYPE_F32 && p->dtype_d != ACCEPT_DTYPE_BF16 && p->dtype_d != ACCEPT_DTYPE_F16) return ACCEPT_ERR_BAD_ENUM;
  if (p->accumulate != 0 && p->accumulate != 1) return ACCEPT_ERR_BAD_ENUM;
  return ACCEPT_OK;
}

size_t accept_matmul_workspace_size(const accept_matmul_params* p) {
  if (accept_matmul_check_params(p) != ACCEPT_OK) return 0;
  if (!uses_pairs(p)) return 16;
  const PairPlan s = pair_plan(p);
  return 16 + (s.parts > 1 ? kArrivalBytes + pair_partial_bytes(s) : 0);
}

accept_status accept_block_matmul(const accept_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b,
                                  const void* d_b_scale, const float* d_bias, void* d_d, void* d_ws, size_t ws_bytes,
                                  void* cuda_stream) {
  if (!p || !d_ws) return ACCEPT_ERR_NULL;
  const accept_status st = accept_matmul_check_params(p);
  if (st != ACCEPT_OK) return st;
  if (ws_bytes < accept_matmul_workspace_size(p)) return ACCEPT_ERR_TOO_SMALL;
  if (p->m == 0 || p->n == 0) return ACCEPT_OK;
  if (!d_d || (p->k != 0 && (!d_a || !d_a_scale || !d_b || !d_b_scale))) return ACCEPT_ERR_NULL;
  if (!is_aligned(d_a, 16) || !is_aligned(d_a_scale, 16) || !is_aligned(d_b, 16) || !is_aligned(d_b_scale, 16) || !is_aligned(d_bias, 4) ||
      !is_aligned(d_d, value_size(p->dtype_d)) || !is_aligned(d_ws, 16))
    return ACCEPT_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  MatmulArgs a{};
  a.bias = d_bias;
  a.d = d_d;
  a.status = static_cast<uint32_t*>(d_ws);
  a.ldd = p->ldd;
  a.dtype_d = p->dtype_d;
  a.accumulate = p->accumulate;
  ACCEPT_BOUNDS(s, bounds_list.add(d_bias, 4 * p->n, false); bounds_list.add(d_d, ((p->m - 1) * p->ldd + p->n) * value_size(p->dtype_d), true);
                bounds_list.add(d_ws, accept_matmul_workspace_size(p), true));
  a.m = (uint32_t)p->m;
  a.n = (uint32_t)p->n;
  if (p->k == 0) {
    ACCEPT_LAUNCH(launch_overlapped(accept::matmul_empty_kernel, dim3((unsigned)((p->m * p->n + 255) / 256)), 256, s, a));
    return ACCEPT_OK;
  }
  if (uses_pairs(p)) return launch_pairs(p, d_a, d_a_scale, d_b, d_b_scale, a, static_cast<uint8_t*>(d_ws), s);

  const unsigned nt = p->m <= 16 ? 16 : p->m <= 32 ? 32 : p->m <= 64 ? 64 : 128;
  a.scale_a = static_cast<const uint8_t*>(d_b_scale);
  a.scale_b = static_cast<const uint8_t*>(d_a_scale);
  a.blocks = (uint32_t)(up(p->k, 128) / 128);
  a.atoms_a = (uint32_t)(up(p->n, 128) / 128);
  a.atoms_b = (uint32_t)(up(p->m, 128) / 128);
  a.tiles = a.atoms_a;
  a.instruction = accept::scaled_instruction((uint32_t)p->format_b, (uint32_t)p->format_a, 128, nt);
  a.wide_stores = !a.accumulate && is_aligned(a.d, 4 * value_size(p->dtype_d)) && a.ldd % 4 == 0;
  CUtensorMap map_a, map_b;
  if (!operand_map(&map_a, d_b, p->n, p->k, 128) || !operand_map(&map_b, d_a, p->m, p->k, nt)) return ACCEPT_ERR_CUDA;
  const unsigned tiles = a.tiles * (unsigned)(up(p->m, nt) / nt);
  const unsigned parts = small_parts(p);
  if (nt == 16) ACCEPT_LAUNCH(launch_small<16>(map_a, map_b, a, tiles, parts, s));
  else if (nt == 32) ACCEPT_LAUNCH(launch_small<32>(map_a, map_b, a, tiles, parts, s));
  else if (nt == 64) ACCEPT_LAUNCH(launch_small<64>(map_a, map_b, a, tiles, parts, s));
  else ACCEPT_LAUNCH(launch_small<128>(map_a, map_b, a, tiles, parts, s));
  return ACCEPT_OK;
}

}  // extern "C"
