// Matrix product of 8-bit operands with a power-of-two scale for each row and 128 values of k, and of 4-bit operands with one for
// each 32 (sm_100a).
//
// The tensor cores apply such scales themselves: the scale bytes go to tensor memory next to the sums, the sums stay
// there in fp32 over all of k, and a scale costs no instruction of its own.
#pragma once
#include "accept_tensor.cuh"
#include "accept_types.cuh"

namespace accept {

// What the operands are.  A block of k is 128 bytes of each row; scales lie in groups of 512 bytes, 128 rows and four scales of each.
struct EightBit {
  static constexpr uint32_t kValues = 128;  // of a block
  static constexpr uint32_t kServes = 4;    // blocks that a group of scales serves
  static constexpr uint32_t kGroups = 1;    // groups of a block
  static constexpr uint32_t instruction(uint32_t format_a, uint32_t format_b, uint32_t m, uint32_t n) { return scaled_instruction(format_a, format_b, m, n); }
};
struct FourBit {
  static constexpr uint32_t kValues = 256;
  static constexpr uint32_t kServes = 1;
  static constexpr uint32_t kGroups = 2;
  static constexpr uint32_t instruction(uint32_t, uint32_t, uint32_t m, uint32_t n) { return scaled4_instruction(m, n); }
};
// The first group of block b, and whether its scales come with it (they do for the first block of a sum too).
template <typename Op> __device__ __forceinline__ uint32_t first_group(uint32_t b) { return b * Op::kGroups / Op::kServes; }
template <typename Op> __device__ __forceinline__ bool brings_scales(uint32_t b) { return b % Op::kServes == 0; }
// The products of the 128 bytes of k at da and db, 32 bytes at a time (that much further in the swizzled rows); a group's scales of a
// lie in tensor memory at scale_a, those of b four columns on, the next group `stride` columns on.
template <typename Op, bool PAIR>
__device__ __forceinline__ void block_mma(uint32_t into, uint64_t da, uint64_t db, uint32_t instruction, uint32_t b, uint32_t scale_a, uint32_t stride, bool add) {
#pragma unroll
  for (uint32_t k = 0; k < 4; ++k) {
    if constexpr (Op::kGroups == 1) {
      if (PAIR) pair_scaled_mma(into, da + 2 * k, db + 2 * k, with_scale_byte(instruction, b & 3), scale_a, scale_a + 4, add || k > 0);
      else scaled_mma(into, da + 2 * k, db + 2 * k, with_scale_byte(instruction, b & 3), scale_a, scale_a + 4, add || k > 0);
    } else {
      const uint32_t at = scale_a + k / 2 * stride, with = with_scale_byte(instruction, k % 2 * 2);
      if (PAIR) pair_scaled4_mma(into, da + 2 * k, db + 2 * k, with, at, at + 4, add || k > 0);
      else scaled4_mma(into, da + 2 * k, db + 2 * k, with, at, at + 4, add || k > 0);
    }
  }
}

struct MatmulArgs {
  const uint8_t* scale_a;  // of the operand on the instruction's M side: b's rows, the columns of d
  const uint8_t* scale_b;  // of a
  const float* bias;       // may be null
  void* d;
  uint32_t* status;
  uint64_t ldd;
  uint32_t m, n;
  uint32_t blocks;            // of k
  uint32_t groups;            // of scales along k
  uint32_t atoms_a, atoms_b;  // groups of 128 rows in the scales
  uint32_t tiles;             // along n
  uint32_t instruction;
  int dtype_d, accumulate;
  int wide_stores;            // four neighbours of d are stored at once (aligned rows, nothing to add)
};

// How long the warps that read the sums may wait for those over `blocks` blocks of k: the limit of one copy and 2 us for each
// block (200 to 700 cycles, measured), so that long sums are not taken for lost ones.
__device__ __forceinline__ unsigned long long sums_wait_ns(uint32_t blocks) { return kCopyWaitNs + 2000ull * blocks; }

// After a wait that ran out in this block (one warp): waits until the products have read the `issued` copies, stage after stage
// (one that was never filled passes), or none has come for the limit of a wait.  So no copy and no product is under way when the
// block frees its tensor memory and leaves, also where the other warps went on after one had given up.  (Without such a wait
// the reading warps' own wait for the last sums says as much; asking every stage there too took 4 x 4096 x 4096 from 5.2 to 5.6 us.)
template <int STAGES>
__device__ __noinline__ void settle(uint32_t empty, uint32_t issued) {
  uint32_t stage = issued % STAGES, parity = 1 ^ (issued / STAGES & 1);
  for (int i = 0; i < STAGES; ++i) {
    if (!mbarrier_wait_warp(empty + 8 * stage, parity)) return;
    if (++stage == STAGES) { stage = 0; parity ^= 1; }
  }
}

__device__ __forceinline__ float load_value(const void* d, int dtype, uint64_t at) {
  if (dtype == kF32) return ld_c(static_cast<const float*>(d) + at);
  if (dtype == kBf16) return __bfloat162float(ld_c(static_cast<const __nv_bfloat16*>(d) + at));
  return __half2float(ld_c(static_cast<const __half*>(d) + at));
}
__device__ __forceinline__ void store_value(void* d, int dtype, uint64_t at, float v) {
  if (dtype == kF32) st_c(static_cast<float*>(d) + at, v);
  else if (dtype == kBf16) st_c(static_cast<__nv_bfloat16*>(d) + at, __float2bfloat16_rn(v));
  else st_c(static_cast<__half*>(d) + at, __float2half_rn(v));
}
__device__ __forceinline__ uint32_t two_values(int dtype, float x, float y) {  // 16-bit types
  return dtype == kBf16 ? pair_to_word<__nv_bfloat16>(pair_of(x, y)) : pair_to_word<__half>(pair_of(x, y));
}

// Blocks of k that fp32 results are summed over in one run of the tensor cores (see the pairs of SMs): 8192 values.
template <typename Op> constexpr uint32_t kChunk = 8192 / Op::kValues;

// ---- small products: single tokens, small batches, few tiles ---------------------------------------------------------
//
// Bound by the bytes of b, or by the time of a launch.  b's rows take the 128 lanes of the instruction's M side and a's rows
// its N side (NT = 16 to 128), so nothing is loaded or multiplied for rows that are not there.  Where there are few tiles
// the blocks of a cluster share k, up to eight ways, and add their sums through each other's shared memory in the order of
// their ranks.  Every block asks for as much of its share at once as shared memory holds.
//
// fp32 results of shares of more than kChunk blocks of k (CHUNKS) are summed as those of pairs are, a chunk at a time: the
// reading warps hold the sums so far in registers (64 at NT = 128) and add each chunk's, the next chunk's products start once
// they have read it: 0 to 4 % (16 x 9600 x 32768 73.8 -> 75.8 us, 128 x 9600 x 32768 85.5 -> 86.0).
constexpr int kTileA = 128;
constexpr int kSmallReaders = 8;  // warps that read the sums: two share 32 lanes
constexpr int kSmallThreads = 32 * (kSmallReaders + 2);
constexpr int kSmallShared = 224 * 1024;
template <typename Op> __host__ __device__ constexpr int small_stage_bytes(int nt) { return (kTileA + nt) * 128 + 1024 * (int)Op::kGroups; }  // both tiles and 1 KB of scales a group
template <typename Op> __host__ __device__ constexpr int small_stages(int nt) { return (kSmallShared - 1024) / small_stage_bytes<Op>(nt); }

// The finished rows to d, dealt over the cluster's blocks and their warps; several rows' reads are on their way at once.
template <bool WIDE, uint32_t PARTS>
__device__ __forceinline__ void small_store(const MatmulArgs& a, uint32_t tile, uint32_t col0, uint32_t row0, uint32_t rows, uint32_t rank,
                                            uint32_t warp, uint32_t lane) {
  constexpr uint32_t kWarps = kSmallThreads / 32, kAtOnce = PARTS < 4 ? 4 : 2, kPartsAtOnce = PARTS < 4 ? PARTS : 4;
  const uint32_t c = WIDE ? 4 * lane : lane, stride = PARTS * kWarps;
  float bias[4];
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    const uint32_t col = col0 + c + j * (WIDE ? 1 : 32);
    bias[j] = a.bias && col < a.n ? ldg_c(a.bias + col) : 0.0f;
  }
  for (uint32_t r0 = rank * kWarps + warp; r0 < rows; r0 += kAtOnce * stride) {
    float4 v[kAtOnce];
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i) v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (uint32_t p = 0; p < PARTS; p += kPartsAtOnce) {
      float4 f[kPartsAtOnce][kAtOnce];
#pragma unroll
      for (uint32_t q = 0; q < kPartsAtOnce; ++q) {
        const uint32_t from = address_in(tile, p + q);
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) {
          const uint32_t at = from + 4 * (min(r0 + i * stride, rows - 1) * kTileA + c);  // rows past the last are read and dropped
          if (WIDE) f[q][i] = ld_cluster(at);
          else f[q][i] = make_float4(ld_cluster_one(at), ld_cluster_one(at + 128), ld_cluster_one(at + 256), ld_cluster_one(at + 384));
        }
      }
#pragma unroll
      for (uint32_t q = 0; q < kPartsAtOnce; ++q)
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) { v[i].x += f[q][i].x; v[i].y += f[q][i].y; v[i].z += f[q][i].z; v[i].w += f[q][i].w; }
    }
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i) {
      const uint32_t r = r0 + i * stride;
      if (r >= rows) break;
      const uint64_t to = (uint64_t)(row0 + r) * a.ldd + col0 + c;
      const float out[4] = {v[i].x + bias[0], v[i].y + bias[1], v[i].z + bias[2], v[i].w + bias[3]};
      if (WIDE) {
        if (a.dtype_d == kF32) st_c(reinterpret_cast<float4*>(static_cast<float*>(a.d) + to), make_float4(out[0], out[1], out[2], out[3]));
        else st_c(reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.d) + to), make_uint2(two_values(a.dtype_d, out[0], out[1]), two_values(a.dtype_d, out[2], out[3])));
      } else {
        float old[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (a.accumulate)
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j)
            if (col0 + c + 32 * j < a.n) old[j] = load_value(a.d, a.dtype_d, to + 32 * j);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
          if (col0 + c + 32 * j < a.n) store_value(a.d, a.dtype_d, to + 32 * j, a.accumulate ? out[j] + old[j] : out[j]);
      }
    }
  }
}

template <typename Op, int NT, bool CHUNKS>
__global__ void __launch_bounds__(kSmallThreads) matmul_small_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                                 const MatmulArgs a) {
  constexpr int kStage = small_stage_bytes<Op>(NT), kStages = small_stages<Op>(NT);
  constexpr int kWords = 4;  // of scales in tensor memory, used in turn
  constexpr uint32_t kWordColumns = 8 * Op::kGroups;
  static_assert(Op::kServes == 1 || kStages <= 13, "a word comes round again thirteen blocks on, when the stage says that its products are done");
  static_assert(Op::kServes != 1 || kStages > kWords, "the products of the last use of a word belong to another stage");
  constexpr uint32_t kNeeded = NT + kWordColumns * kWords;  // the sums and the scales
  constexpr uint32_t kColumns = kNeeded <= 64 ? 64 : kNeeded <= 128 ? 128 : 256;
  constexpr uint32_t kScaleColumn = kColumns - kWordColumns * kWords;
  extern __shared__ uint8_t raw_shared[];
  __shared__ __align__(8) uint64_t barriers[2 * kStages + 2];
  __shared__ uint32_t tensor_base, failed, issued;
  const uint32_t base = (smem_address(raw_shared) + 1023) & ~1023u;  // 128-byte swizzle repeats every 1024 bytes
  const uint32_t full = smem_address(barriers), empty = full + 8 * kStages, done = empty + 8 * kStages, drained = done + 8;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t parts = gridDim.y, rank = blockIdx.y;
  const uint32_t first = (uint32_t)((uint64_t)a.blocks * rank / parts), last = (uint32_t)((uint64_t)a.blocks * (rank + 1) / parts);
  const uint32_t tile_b = blockIdx.x / a.tiles, tile_a = blockIdx.x - tile_b * a.tiles;
  const uint32_t row_a = tile_a * kTileA, row_b = tile_b * NT, rows = min(a.m - row_b, (uint32_t)NT);
  const uint32_t chunks = CHUNKS ? (last - first + kChunk<Op> - 1) / kChunk<Op> : 1;
  const auto chunk_start = [&](uint32_t chunk) { return first + (uint32_t)((uint64_t)(last - first) * chunk / chunks); };

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2 * kStages + 1; ++i) mbarrier_init(full + 8 * i, 1);
    mbarrier_init(drained, kSmallReaders);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    failed = issued = 0;
    prefetch_map(&map_a);
    prefetch_map(&map_b);
  }
  if (warp == 0) tensor_alloc(smem_address(&tensor_base), kColumns);
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  const uint32_t sums = tensor_base;
  grid_dependency_handshake();

  if (warp == kSmallReaders) {  // loads
    const bool leader = elect_one();
    uint32_t stage = 0, parity = 1;  // a fresh barrier passes for the phase before its first
    uint32_t b = first;
    for (; b < last; ++b) {
      if (!mbarrier_wait_warp(empty + 8 * stage, parity)) break;
      if (leader) {
        const uint32_t at = base + stage * kStage, bar = full + 8 * stage;
        // k may end before a block's second group: the group before it comes a second time, its codes there are zeros
        const uint32_t group = first_group<Op>(b), more = Op::kGroups > 1 && group + 1 < a.groups ? 1 : 0;
        const bool scales = b == first || brings_scales<Op>(b);
        mbarrier_expect_bytes(bar, (kTileA + NT) * 128 + (scales ? 1024 * Op::kGroups : 0) + kCopyAnnounceExtra);
        tile_load(at, &map_a, b * 128, row_a, bar);
        tile_load(at + kTileA * 128, &map_b, b * 128, row_b, bar);
        if (scales) {
#pragma unroll
          for (uint32_t g = 0; g < Op::kGroups; ++g) {
            const uint32_t to = at + (kTileA + NT) * 128 + 1024 * g, of = group + (g ? more : 0);
            bulk_copy_to_shared(to, a.scale_a + ((uint64_t)of * a.atoms_a + tile_a) * 512, 512, bar);
            bulk_copy_to_shared(to + 512, a.scale_b + ((uint64_t)of * a.atoms_b + tile_b) * 512, 512, bar);  // NT < 128: one tile
          }
        }
      }
      if (++stage == kStages) { stage = 0; parity ^= 1; }
    }
    if (leader) {
      issued = b - first;
      if (b < last) atomicExch(&failed, 1u);
    }
  } else if (warp == kSmallReaders + 1) {  // matrix instructions
    const bool leader = elect_one();
    const uint32_t tensor = __shfl_sync(0xffffffffu, sums, 0);
    uint32_t stage = 0, parity = 0, word = kWords - 1, b = first, chunk = 0, from = first;
    uint32_t stop = CHUNKS ? chunk_start(1) : last;
    for (; b < last; ++b) {
      if (CHUNKS && b == stop) {
        if (leader) mma_commit(done);
        if (!mbarrier_wait_warp(drained, chunk & 1)) break;
        tensor_fence_after();
        ++chunk;
        from = b;
        stop = chunk_start(chunk + 1);
      }
      if (!mbarrier_wait_warp(full + 8 * stage, parity)) break;
      tensor_fence_after();
      // A word of scales serves four blocks of k and comes round again after three others, thirteen blocks after the last
      // that used it (only a share's first and last word serve fewer); this stage was filled again, so the products of
      // kStages blocks back are done.
      const bool fresh = b == first || brings_scales<Op>(b);
      if (fresh) word = word + 1 == kWords ? 0 : word + 1;
      if (Op::kServes == 1 && b - first >= kWords) {  // a word of one block: wait for the products that used it last
        const uint32_t before = b - first - kWords;
        if (!mbarrier_wait_warp(empty + 8 * (before % kStages), before / kStages & 1)) break;
      }
      const uint32_t at = base + stage * kStage, scale_a = tensor + kScaleColumn + kWordColumns * word;
      const uint64_t da = operand_descriptor(at), db = operand_descriptor(at + kTileA * 128), ds = scale_descriptor(at + (kTileA + NT) * 128);
      if (leader) {
        if (fresh) {
#pragma unroll
          for (uint32_t g = 0; g < Op::kGroups; ++g) {
            scale_copy(scale_a + 8 * g, ds + 64 * g);
            scale_copy(scale_a + 8 * g + 4, ds + 64 * g + 32);
          }
        }
        block_mma<Op, false>(tensor, da, db, a.instruction, b, scale_a, 8, b > from);
        mma_commit(empty + 8 * stage);
      }
      if (++stage == kStages) { stage = 0; parity ^= 1; }
    }
    if (leader) {
      if (b == last) mma_commit(done);
      else atomicExch(&failed, 1u);
    }
  }
  __syncwarp();

  // The block's sums go through shared memory as fp32, a row of d (a row of a) in 128 floats.
  float* tile = reinterpret_cast<float*>(raw_shared + (base - smem_address(raw_shared)));
  constexpr int kPiece = NT < 32 ? 16 : 32;
  if (CHUNKS && warp < kSmallReaders) {
    constexpr int kPieces = NT > 2 * kPiece ? NT / (2 * kPiece) : 1;
    float total[kPieces][kPiece];
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
      for (int j = 0; j < kPiece; ++j) total[i][j] = 0.0f;
    bool ok = true;
    for (uint32_t chunk = 0; chunk < chunks && ok; ++chunk) {
      ok = mbarrier_wait_warp(done, chunk & 1, sums_wait_ns(kChunk<Op>));
      if (!ok) break;
      tensor_fence_after();
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const uint32_t c = kPiece * ((warp >> 2) + 2 * i);
        if (c < rows) {
          float v[kPiece];
          tensor_read(sums + (((warp & 3) * 32) << 16) + c, v);
          tensor_read_wait();
#pragma unroll
          for (int j = 0; j < kPiece; ++j) total[i][j] += v[j];
        }
      }
      tensor_fence_before();
      __syncwarp();
      if (lane == 0) mbarrier_arrive(drained);
    }
    if (!ok && lane == 0) atomicExch(&failed, 1u);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const uint32_t c = kPiece * ((warp >> 2) + 2 * i);
      if (ok && c < rows)
#pragma unroll
        for (int j = 0; j < kPiece; ++j) tile[(c + j) * kTileA + (warp & 3) * 32 + lane] = total[i][j];
    }
  } else if (warp < kSmallReaders) {
    const bool ok = mbarrier_wait_warp(done, 0, sums_wait_ns(last - first));
    if (!ok) atomicExch(&failed, 1u);
    tensor_fence_after();
    if (ok) {
#pragma unroll 1
      for (uint32_t c = kPiece * (warp >> 2); c < rows; c += 2 * kPiece) {
        float v[kPiece];
        tensor_read(sums + (((warp & 3) * 32) << 16) + c, v);
        tensor_read_wait();
#pragma unroll
        for (int j = 0; j < kPiece; ++j) tile[(c + j) * kTileA + (warp & 3) * 32 + lane] = first == last ? 0.0f : v[j];  // no share of k: nothing was summed
      }
    }
    tensor_fence_before();
  }
  if (parts > 1) cluster_sync();
  else __syncthreads();
  const bool failure = *reinterpret_cast<volatile uint32_t*>(&failed) != 0;
  if (warp == 0) {
    if (failure) {
      if (lane == 0) atomicOr(a.status, kDevCopyTimeout);
      settle<kStages>(empty, issued);
    }
    tensor_fence_after();
    tensor_free(sums, kColumns);
  }

  if (!failure) {
    // wide: a lane has four neighbours of a row; otherwise four columns 32 apart, so that a row leaves in runs
    const bool wide = a.wide_stores && row_a + kTileA <= a.n;
    const uint32_t at = smem_address(tile);
    if (parts == 1) wide ? small_store<true, 1>(a, at, row_a, row_b, rows, rank, warp, lane) : small_store<false, 1>(a, at, row_a, row_b, rows, rank, warp, lane);
    else if (parts == 2) wide ? small_store<true, 2>(a, at, row_a, row_b, rows, rank, warp, lane) : small_store<false, 2>(a, at, row_a, row_b, rows, rank, warp, lane);
    else if (parts == 4) wide ? small_store<true, 4>(a, at, row_a, row_b, rows, rank, warp, lane) : small_store<false, 4>(a, at, row_a, row_b, rows, rank, warp, lane);
    else wide ? small_store<true, 8>(a, at, row_a, row_b, rows, rank, warp, lane) : small_store<false, 8>(a, at, row_a, row_b, rows, rank, warp, lane);
  }
  if (parts > 1) cluster_sync();  // the other blocks may still be reading this one's tile
}

// ---- more rows: pairs of SMs, tiles of 256 x NT, persistent ---------------------------------------------------------
//
// Bound by the tensor cores.  A pair of blocks holds one tile (128 rows of it in each block's tensor memory); each
// block loads its own 128 rows of a and half of b, so an operand byte in shared memory feeds twice the products it would
// feed for one SM alone.  Each pair keeps taking units of work; the sums of the next one are formed while the last one's
// are read.  NT = 256 for large products; two tiles of sums (2 x 256 columns) and the scales do not fit 512 columns side by
// side, so the two overlap by 24 columns (48 with 4-bit operands): those are read first, and the next unit's products start once they are.
// NT = 128 where tiles of 256 would leave pairs without work.
// The products of unit i so wait twice: for the last read of unit i - 2, whose columns they take over (`drained`: all reading
// warps of both blocks), and, where the two tiles overlap, for the first reads of unit i - 1 by the warps that hold the shared
// columns (`shared_read`).  The second does not imply the first: the warps that hold no shared columns of unit i - 1 may still
// be storing what they read of unit i - 2.
//
// A unit is a tile over all of k; the tiles that are left when every pair has had the same number (whole tiles) are cut
// along k into `parts`, so that all pairs share the last round: one part at most for each pair, its last unit.  A part's
// sums go to the workspace; the warp that is the last to bring its rows and columns of a tile fetches the other parts' sums
// into the shared memory that the operands have left and adds all parts in their order.  No block waits for another pair.
//
// Sums that go out in fp32 are taken over at most kChunk blocks of k at a time and the chunks added one after the other
// (in d): the tensor cores' own sums are off by what grows with their length, 0.5e-6 of the result's norm over 8192 values of k,
// 1.5e-6 over 20001, 3.0e-6 over 32768.  In chunks of 8192 it is 0.5e-6 for any k (fp32 library sums: 0.1e-6 to 0.2e-6).
constexpr uint32_t kPairRows = 256;

template <typename Op, int NT>
struct PairShape {
  static constexpr int kReaders = 8;                                     // warps that read sums: two share 32 rows
  static constexpr int kThreads = 32 * (kReaders + 2);
  static constexpr int kStages = (NT == 256 ? 6 : 8) - (Op::kGroups - 1);
  static constexpr int kOperandBytes = (128 + NT / 2) * 128;             // a block's rows of a and of b, 128 bytes each
  static constexpr int kGroupBytes = 512 + 4 * NT;                       // a group of scales: of 128 rows of a, of NT of b
  static constexpr int kScaleBytes = Op::kGroups * kGroupBytes;
  static constexpr int kStaging = kReaders * 2048;                       // a piece of the result for each of those warps: 32 rows of 64 bytes
  static constexpr int kSharedBytes = 1024 + kStages * (kOperandBytes + kScaleBytes) + kStaging + kReaders * 4 * NT;  // and each warp's copy of the bias
  static constexpr uint32_t kGroupColumns = 4 + NT / 32;                 // a group of scales in tensor memory: of a, of b
  static constexpr uint32_t kWordColumns = Op::kGroups * kGroupColumns;  // a block's
  static constexpr uint32_t kScaleColumn = 512 - 2 * kWordColumns;       // two words in turn
  static constexpr uint32_t kSecond = kScaleColumn - NT < (uint32_t)NT ? kScaleColumn - NT : NT;  // the second tile of sums
  static constexpr bool kOverlap = kSecond < (uint32_t)NT;
  // Two pieces of 32 columns hold shared ones (48, with 4-bit operands): the two warps that share 32 rows read one each first, so
  // that the next unit waits for one read (16384 x 4096 x 4096: 112 -> 106 us).
  static constexpr bool kDealt = NT - kSecond > 32;
  static_assert(NT - kSecond <= 64, "one piece for each of two warps");
  static_assert(kStages * kScaleBytes % 1024 == 0, "the pieces lie on the boundaries that the tensor map's swizzle counts from");
  // pieces of other parts' sums (32 rows x 32 columns, 4 KB) that a reading warp can have in shared memory at the end
  static constexpr uint32_t kSlots = kStages * kOperandBytes / kReaders / 4096;
};

struct PairArgs {
  const float* bias;
  void* d;
  uint32_t* status;
  float* partials;     // parts of cut tiles: (tile, part) x 256 x NT values
  unsigned long long* arrivals;  // one for each reading warp of both blocks and each cut tile, see arrive()
  unsigned long long call;       // this call's number: a multiple of 8, never 0, another for each call
  uint64_t ldd;
  uint32_t m, n, blocks;
  uint32_t atoms_a, atoms_b;
  uint32_t tiles_m, tiles_n;
  uint32_t whole;      // tiles that are not cut
  uint32_t parts;      // of each of the others
  uint32_t chunks;     // of a whole tile, one after the other
  uint32_t instruction;
  int dtype_d, accumulate;
  uint32_t tile_columns;  // columns of d below this one are stored through its tensor map, piece by piece
  int word_stores;     // rows of a 16-bit d start on 4-byte boundaries
};

// One accumulation: blocks [first, last) of k of a tile.
struct Unit {
  uint32_t tile_m, tile_n, first, last;
  uint32_t chunk;  // of a whole tile
  uint32_t cut;    // index of the cut tile, or ~0
  uint32_t part;
};

// One arrival of `parts` (8 at most) at a count in the workspace: how many of this call came before it.  A count holds the
// call's number plus its arrivals; whatever else is there, left by anyone who used the workspace before, stands for none.  The
// last one leaves zero, which is what the first one of the next call expects.  At most parts + 1 turns: past the second, each
// turn follows another part's arrival.
__device__ __forceinline__ uint32_t arrive(unsigned long long* count, unsigned long long call, uint32_t parts) {
  unsigned long long held = 0;
  for (;;) {
    const uint32_t before = held - call < 8 ? (uint32_t)(held - call) : 0;
    if (before + 1 == parts) {
      *reinterpret_cast<volatile unsigned long long*>(count) = 0;  // all others have been here
      return before;
    }
    const unsigned long long found = atomicCAS(count, held, call + before + 1);
    if (found == held) return before;
    held = found;
  }
}

// The i-th unit of a pair; false if it has no more.  Tiles are taken in the order eight tiles of rows, then the next tile
// of columns: the tiles in flight at a time form a block that shares its operands in L2.
__device__ __forceinline__ bool pair_unit(const PairArgs& a, uint32_t pair, uint32_t pairs, uint32_t i, Unit& u) {
  const uint32_t turn = i / a.chunks;
  uint32_t tile;
  u.chunk = i - turn * a.chunks;
  uint64_t index = pair + (uint64_t)turn * pairs;
  if (index < a.whole) {
    tile = (uint32_t)index;
    u.cut = ~0u;
    u.part = 0;
    u.first = (uint32_t)((uint64_t)a.blocks * u.chunk / a.chunks);
    u.last = (uint32_t)((uint64_t)a.blocks * (u.chunk + 1) / a.chunks);
  } else {
    // the pair's turns at whole tiles are over: one unit for each turn from here on
    const uint32_t own = a.whole > pair ? (a.whole - pair + pairs - 1) / pairs : 0;
    index = pair + (uint64_t)(own + (i - own * a.chunks)) * pairs - a.whole;
    if (index >= (uint64_t)(a.tiles_m * a.tiles_n - a.whole) * a.parts) return false;
    u.chunk = 0;
    u.cut = (uint32_t)(index / a.parts);
    u.part = (uint32_t)(index - (uint64_t)u.cut * a.parts);
    tile = a.whole + u.cut;
    u.first = (uint32_t)((uint64_t)a.blocks * u.part / a.parts);
    u.last = (uint32_t)((uint64_t)a.blocks * (u.part + 1) / a.parts);
  }
  const uint32_t per_group = 8 * a.tiles_n, group = tile / per_group, inside = tile - group * per_group;
  const uint32_t rows = min(8u, a.tiles_m - 8 * group);
  u.tile_n = inside / rows;
  u.tile_m = 8 * group + inside - u.tile_n * rows;
  return true;
}

// For the checking build: what a tile store of a warp's 32 rows may write, 64 bytes of each row or up to the end of d's rows in
// units of 16 bytes, lies inside the call's buffers.
template <typename T>
__device__ __forceinline__ bool tile_inside(const PairArgs& a, uint32_t row, uint32_t col) {
#ifdef ACCEPT_BOUNDS_CHECK
  const uint32_t bytes = min(((a.n - col) * (uint32_t)sizeof(T) + 15) & ~15u, 64u);
  return __all_sync(0xffffffffu, row >= a.m || bounds_ok(static_cast<const T*>(a.d) + row * a.ldd + col, bytes, true));
#else
  return true;
#endif
}

// 32 columns of a warp's 32 rows to d, through the warp's 2 KB of shared memory (`piece`): 32 rows of 64 bytes, 16-byte units
// permuted as the tensor map's swizzle has them.
template <bool SINGLE>
__device__ __forceinline__ void pair_store(const PairArgs& a, const CUtensorMap* map_d, uint8_t* piece, uint32_t piece_address, uint32_t lane,
                                           uint32_t row0, uint32_t col, bool add, float (&v)[32]) {
  if (row0 >= a.m || col >= a.n) return;
  const uint32_t rows = min(a.m - row0, 32u);
  uint8_t* mine = piece + lane * 64;
  const uint32_t swap = (lane >> 1) & 3;
  if (!SINGLE && !add) {
    const bool by_tile = col < a.tile_columns;
    if (a.tile_columns) {  // the piece's last tile store has read it
      if (lane == 0) store_wait_read<0>();
      __syncwarp();
    }
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) {
      uint32_t w[4];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) w[j] = two_values(a.dtype_d, v[8 * u + 2 * j], v[8 * u + 2 * j + 1]);
      *reinterpret_cast<uint4*>(mine + 16 * (u ^ swap)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (by_tile) {
      shared_to_async();
      __syncwarp();
      const bool inside = tile_inside<uint16_t>(a, row0 + lane, col);
      if (lane == 0) {
        if (inside) tile_store(map_d, col, row0, piece_address);
        store_commit();
      }
      return;
    }
    __syncwarp();
    if (a.word_stores) {  // two rows at a time, a word for each lane
      const uint32_t c = 2 * (lane & 15), unit = c >> 3, in_unit = 2 * (c & 7);
      uint16_t* p = static_cast<uint16_t*>(a.d) + (uint64_t)(row0 + (lane >> 4)) * a.ldd + col + c;
#pragma unroll 8
      for (uint32_t r = lane >> 4; r < rows; r += 2, p += 2 * a.ldd) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(piece + r * 64 + 16 * (unit ^ ((r >> 1) & 3)) + in_unit);
        if (col + c + 1 < a.n) st_c(reinterpret_cast<uint32_t*>(p), w);
        else if (col + c < a.n) st_c(p, (uint16_t)w);
      }
    } else {
      uint16_t* p = static_cast<uint16_t*>(a.d) + (uint64_t)row0 * a.ldd + col + lane;
#pragma unroll 8
      for (uint32_t r = 0; r < rows; ++r, p += a.ldd) {
        const uint16_t w = *reinterpret_cast<const uint16_t*>(piece + r * 64 + 16 * ((lane >> 3) ^ ((r >> 1) & 3)) + 2 * (lane & 7));
        if (col + lane < a.n) st_c(p, w);
      }
    }
    __syncwarp();
    return;
  }
  // in fp32, sixteen columns at a time
#pragma unroll
  for (uint32_t half = 0; half < 32; half += 16) {
    if (col + half >= a.n) return;
    const bool by_tile = SINGLE && col + half < a.tile_columns;
    if (SINGLE && a.tile_columns) {
      if (lane == 0) store_wait_read<0>();
      __syncwarp();
    }
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u)
      *reinterpret_cast<float4*>(mine + 16 * (u ^ swap)) = make_float4(v[half + 4 * u], v[half + 4 * u + 1], v[half + 4 * u + 2], v[half + 4 * u + 3]);
    if (by_tile) {
      shared_to_async();
      __syncwarp();
      const bool inside = tile_inside<float>(a, row0 + lane, col + half);
      if (lane == 0 && inside) {
        if (add) tile_add(map_d, col + half, row0, piece_address);
        else tile_store(map_d, col + half, row0, piece_address);
        store_commit();
      }
      continue;
    }
    __syncwarp();
    const uint32_t c = col + half + (lane & 15);
    if (c < a.n) {  // two rows at a time; eight such pairs' sums, and the old values that they are added to, at once
      uint64_t at = (uint64_t)(row0 + (lane >> 4)) * a.ldd + c;
#pragma unroll 1
      for (uint32_t r = lane >> 4; r < rows; r += 16, at += 16 * a.ldd) {
        float x[8], old[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          x[j] = *reinterpret_cast<const float*>(piece + (r + 2 * j) * 64 + 16 * (((lane & 15) >> 2) ^ (((r >> 1) + j) & 3)) + 4 * (lane & 3));
          old[j] = 0.0f;
          if (add && r + 2 * j < rows) old[j] = SINGLE ? ld_c(static_cast<const float*>(a.d) + at + 2 * j * a.ldd) : load_value(a.d, a.dtype_d, at + 2 * j * a.ldd);
        }
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
          if (r + 2 * j < rows) {
            if (SINGLE) st_c(static_cast<float*>(a.d) + at + 2 * j * a.ldd, add ? x[j] + old[j] : x[j]);
            else store_value(a.d, a.dtype_d, at + 2 * j * a.ldd, x[j] + old[j]);
          }
      }
    }
    __syncwarp();
  }
}

template <typename Op, int NT, bool SINGLE>  // SINGLE: d is fp32
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairShape<Op, NT>::kThreads)
    matmul_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                       const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                       const __grid_constant__ CUtensorMap map_d, const PairArgs a) {
  using S = PairShape<Op, NT>;
  constexpr int kStages = S::kStages, kReaders = S::kReaders, kShare = kReaders / 4, kPer = NT / 32 / kShare;  // warps that share 32 rows, pieces of 32 columns for each
  extern __shared__ uint8_t raw_shared[];
  __shared__ __align__(8) uint64_t barriers[2 * kStages + 6 + kReaders];
  __shared__ uint32_t tensor_base, failed, issued;
  const uint32_t base = (smem_address(raw_shared) + 1023) & ~1023u;
  const uint32_t scales = base + kStages * S::kOperandBytes, staging = scales + kStages * S::kScaleBytes;
  const uint32_t full = smem_address(barriers), empty = full + 8 * kStages, done = empty + 8 * kStages, drained = done + 16, shared_read = drained + 16, joined = shared_read + 16;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();
  const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2 * kStages + 2; ++i) mbarrier_init(full + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {  // warps of both blocks
      mbarrier_init(drained + 8 * i, 2 * kReaders);
      mbarrier_init(shared_read + 8 * i, S::kDealt ? 2 * kReaders : 2 * 4);
    }
    for (int i = 0; i < kReaders; ++i) mbarrier_init(joined + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    failed = issued = 0;
    prefetch_map(&map_a);
    prefetch_map(&map_b);
    prefetch_map(&map_sa);
    prefetch_map(&map_sb);
    prefetch_map(&map_d);
  }
  if (warp == 0) pair_tensor_alloc(smem_address(&tensor_base), 512);
  tensor_fence_before();
  cluster_sync();
  tensor_fence_after();
  const uint32_t sums = tensor_base;
  grid_dependency_handshake();

  if (warp == kReaders) {  // loads, in both blocks; the even block's barrier counts the bytes of both
    const bool leader = elect_one();
    const uint32_t full_cluster = address_in(full, 0);
    uint32_t i = 0, stage = 0, parity = 1;  // a fresh barrier passes for the phase before its first
    bool ok = true;
    Unit u;
    for (uint32_t unit = 0; ok && pair_unit(a, pair, pairs, unit, u); ++unit) {
      const uint32_t row_a = u.tile_m * kPairRows + rank * 128, row_b = u.tile_n * NT + rank * (NT / 2);
      for (uint32_t b = u.first; b < u.last; ++b, ++i) {
        if (!mbarrier_wait_warp(empty + 8 * stage, parity)) { ok = false; break; }
        if (leader) {
          const bool with_scales = b == u.first || brings_scales<Op>(b);
          const uint32_t at = base + stage * S::kOperandBytes, at_scales = scales + stage * S::kScaleBytes, bar = full_cluster + 8 * stage;
          if (rank == 0) mbarrier_expect_bytes(full + 8 * stage, 2 * (S::kOperandBytes + (with_scales ? S::kScaleBytes : 0)) + kCopyAnnounceExtra);
          pair_tile_load(at, &map_a, b * 128, row_a, bar);
          pair_tile_load(at + 128 * 128, &map_b, b * 128, row_b, bar);
          if (with_scales) {
#pragma unroll
            for (uint32_t g = 0; g < Op::kGroups; ++g) {  // past the last group of k: zeros, and so are the codes there
              const uint32_t group = first_group<Op>(b) + g;
              pair_tile_load(at_scales + g * S::kGroupBytes, &map_sa, 0, group * a.atoms_a + u.tile_m * 2 + rank, bar);
              pair_tile_load(at_scales + g * S::kGroupBytes + 512, &map_sb, 0, group * a.atoms_b + u.tile_n * (NT / 128), bar);
            }
          }
        }
        if (++stage == kStages) { stage = 0; parity ^= 1; }
      }
    }
    if (leader) {
      issued = i;
      if (!ok) atomicExch(&failed, 1u);
    }
  } else if (warp == kReaders + 1 && rank == 0) {  // matrix instructions, for both blocks
    const bool leader = elect_one();
    const uint32_t tensor = __shfl_sync(0xffffffffu, sums, 0);
    uint32_t i = 0, stage = 0, parity = 0, word = 0;
    uint32_t used[2] = {0, 0};  // one past the last block of k that used each word of scales
    bool ok = true;
    Unit u;
    for (uint32_t unit = 0; ok && pair_unit(a, pair, pairs, unit, u); ++unit) {
      if (unit >= 2 && !mbarrier_wait_warp(drained + 8 * (unit & 1), ((unit - 2) >> 1) & 1)) { ok = false; break; }
      if (S::kOverlap && unit >= 1 && !mbarrier_wait_warp(shared_read + 8 * ((unit - 1) & 1), ((unit - 1) >> 1) & 1)) { ok = false; break; }
      tensor_fence_after();
      const uint32_t into = tensor + (unit & 1 ? S::kSecond : 0);
      for (uint32_t b = u.first; b < u.last; ++b) {
        if (!mbarrier_wait_warp(full + 8 * stage, parity)) { ok = false; break; }
        tensor_fence_after();
        const bool fresh = b == u.first || brings_scales<Op>(b);
        if (fresh) {
          // the products that used this word before must be done (at most five blocks back: that phase is the latest)
          word ^= 1;
          const uint32_t before = word ? used[1] : used[0];
          if (before != 0 && !mbarrier_wait_warp(empty + 8 * ((before - 1) % kStages), ((before - 1) / kStages) & 1)) { ok = false; break; }
        }
        ++i;
        if (word) used[1] = i;
        else used[0] = i;
        const uint32_t at = base + stage * S::kOperandBytes, scale_a = tensor + S::kScaleColumn + S::kWordColumns * word;
        const uint64_t da = operand_descriptor(at), db = operand_descriptor(at + 128 * 128), ds = scale_descriptor(scales + stage * S::kScaleBytes);
        if (leader) {
          if (fresh) {
#pragma unroll
            for (uint32_t g = 0; g < Op::kGroups; ++g) {
              const uint32_t to = scale_a + g * S::kGroupColumns;
              const uint64_t from = ds + g * (S::kGroupBytes / 16);
              pair_scale_copy(to, from);
              pair_scale_copy(to + 4, from + 32);
              if (NT == 256) pair_scale_copy(to + 8, from + 64);
            }
          }
          block_mma<Op, true>(into, da, db, a.instruction, b, scale_a, S::kGroupColumns, b > u.first);
          pair_mma_commit(empty + 8 * stage);
        }
        if (++stage == kStages) { stage = 0; parity ^= 1; }
      }
      if (ok && leader) pair_mma_commit(done + 8 * (unit & 1));
    }
    if (!ok && leader) atomicExch(&failed, 1u);
  } else if (warp < kReaders) {  // results
    const uint32_t piece_address = staging + warp * 2048;
    uint8_t* piece = raw_shared + (piece_address - smem_address(raw_shared));
    float* bias_tile = reinterpret_cast<float*>(raw_shared + (staging + S::kStaging - smem_address(raw_shared))) + warp * NT;
    const uint32_t drained_at = address_in(drained, 0), shared_read_at = address_in(shared_read, 0);
    // the i-th piece of 32 columns that a warp reads: of its half, or, where two pieces hold shared columns, of every kShare-th
    constexpr bool kDealt = S::kDealt;
    const auto piece_at = [&](uint32_t i) { return kDealt ? i * kShare + (warp >> 2) : (warp >> 2) * kPer + i; };
    Unit u;
    for (uint32_t unit = 0; pair_unit(a, pair, pairs, unit, u); ++unit) {
      const uint32_t row0 = u.tile_m * kPairRows + rank * 128 + (warp & 3) * 32, col0 = u.tile_n * NT;
      const bool with_bias = a.bias && u.chunk == 0;
      if (with_bias) {
        __syncwarp();
        for (uint32_t c = lane; c < NT; c += 32) bias_tile[c] = col0 + c < a.n ? ld_c(a.bias + col0 + c) : 0.0f;
        __syncwarp();
      }
      // by the whole warp: the reads of tensor memory that follow want all of its lanes, also where the wait runs out for some
      if (!mbarrier_wait_warp(done + 8 * (unit & 1), (unit >> 1) & 1, sums_wait_ns(u.last - u.first))) {
        if (lane == 0) atomicExch(&failed, 1u);
        break;
      }
      tensor_fence_after();
      const uint32_t from = sums + (unit & 1 ? S::kSecond : 0) + (((warp & 3) * 32) << 16);
      // a cut tile: this warp's 32 x NT values of each part, four neighbours of each lane's row side by side
      float4* partial = u.cut == ~0u ? nullptr : reinterpret_cast<float4*>(a.partials) + (((uint64_t)u.cut * a.parts * 2 + rank) * 4 + (warp & 3)) * (8 * NT);
      const uint64_t part_stride = 2 * 4 * (8 * NT);
      if (u.chunk > 0 && lane == 0) store_wait();  // the chunk before must lie in d
#pragma unroll 1
      for (uint32_t turn = 0; turn < kPer; ++turn) {  // 32 columns at a time, those shared with the next unit's sums first
        const uint32_t c = 32 * piece_at(unit & 1 || !S::kOverlap ? turn : kPer - 1 - turn);
        float v[32];
        tensor_read(from + c, v);
        tensor_read_wait();
        const bool shares = S::kOverlap && turn == 0 && (kDealt || (warp >> 2) == (unit & 1 ? 0 : kShare - 1)), last = turn + 1 == kPer;
        if (shares || last) {
          tensor_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (shares) mbarrier_arrive_cluster(shared_read_at + 8 * (unit & 1));
            if (last) mbarrier_arrive_cluster(drained_at + 8 * (unit & 1));
          }
        }
        if (partial) {
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j)
            st_c(partial + u.part * part_stride + (c / 4 + j) * 32 + lane, make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
        } else {
          if (with_bias)
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += bias_tile[c + j];
          pair_store<SINGLE>(a, &map_d, piece, piece_address, lane, row0, col0 + c, a.accumulate || u.chunk > 0, v);
        }
      }
      if (partial) {
        __threadfence();
        __syncwarp();
        uint32_t before = 0;
        if (lane == 0) before = arrive(a.arrivals + (u.cut * 2 + rank) * kReaders + warp, a.call, a.parts);
        before = __shfl_sync(0xffffffffu, before, 0);
        if (before + 1 == a.parts) {  // all parts are there: add them in their order, this one's from tensor memory (it is the pair's last unit)
          __threadfence();
          asm volatile("fence.proxy.async;" ::: "memory");
          const uint32_t others = a.parts - 1, batch = S::kSlots / others, slots = base + warp * S::kSlots * 4096, bar = joined + 8 * warp;
          bool landed = true;
          for (uint32_t start = 0, phase = 0; start < kPer && landed; start += batch, phase ^= 1) {
            const uint32_t stop = min(start + batch, (uint32_t)kPer);
            __syncwarp();
            if (lane == 0) {
              mbarrier_expect_bytes(bar, (stop - start) * others * 4096 + kCopyAnnounceExtra);
              for (uint32_t i = start; i < stop; ++i)
                for (uint32_t o = 0; o < others; ++o)
                  bulk_copy_to_shared(slots + ((i - start) * others + o) * 4096, partial + (o + (o >= u.part)) * part_stride + 8 * piece_at(i) * 32, 4096, bar);
            }
            landed = mbarrier_wait_warp(bar, phase);
            for (uint32_t i = start; i < stop && landed; ++i) {
              const uint32_t c = 32 * piece_at(i);
              float own[32], v[32];
              tensor_read(from + c, own);
              tensor_read_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = u.part == 0 ? own[j] : 0.0f;
              for (uint32_t o = 0; o < others; ++o) {
                if (o == u.part && o > 0)
#pragma unroll
                  for (int j = 0; j < 32; ++j) v[j] += own[j];
                const float4* w = reinterpret_cast<const float4*>(raw_shared + (slots + ((i - start) * others + o) * 4096 - smem_address(raw_shared))) + lane;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const float4 f = w[32 * j];
                  v[4 * j] += f.x; v[4 * j + 1] += f.y; v[4 * j + 2] += f.z; v[4 * j + 3] += f.w;
                }
              }
              if (u.part == others)
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += own[j];
              if (with_bias)
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += bias_tile[c + j];
              pair_store<SINGLE>(a, &map_d, piece, piece_address, lane, row0, col0 + c, a.accumulate, v);
            }
          }
          if (!landed) {
            if (lane == 0) atomicExch(&failed, 1u);
            break;
          }
        }
      }
    }
    if (lane == 0) store_wait_read<0>();  // the block may leave: its shared memory has been read
  }
  __syncwarp();
  __syncthreads();
  if (warp == 0 && *reinterpret_cast<volatile uint32_t*>(&failed)) {
    if (lane == 0) atomicOr(a.status, kDevCopyTimeout);
    settle<kStages>(empty, issued);
  }
  tensor_fence_before();
  cluster_sync();
  tensor_fence_after();
  if (warp == 0) pair_tensor_free(sums, 512);
}

// k = 0: the sum is empty.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) matmul_empty_kernel(const MatmulArgs a) {
  grid_dependency_handshake();
  const uint64_t i = (uint64_t)blockIdx.x * THREADS + threadIdx.x, row = i / a.n, col = i % a.n;
  if (row < a.m) {
    const float v = a.bias ? ld_c(a.bias + col) : 0.0f;
    store_value(a.d, a.dtype_d, row * a.ldd + col, a.accumulate ? v + load_value(a.d, a.dtype_d, row * a.ldd + col) : v);
  }
}

}  // namespace accept
