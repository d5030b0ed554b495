// Matrix product of 8-bit operands with a power-of-two scale for each row and block of 128 values of k (sm_100a).
//
// The tensor cores apply such scales themselves: the scale bytes go to tensor memory next to the sums, the sums stay
// there in fp32 over all of k, and a scale costs no instruction of its own.
#pragma once
#include "accept_tensor.cuh"
#include "accept_types.cuh"

namespace accept {

struct MatmulArgs {
  const uint8_t* scale_a;  // of the operand on the instruction's M side
  const uint8_t* scale_b;
  const float* bias;       // may be null
  void* d;
  uint32_t* status;
  uint64_t ldd;
  uint32_t rows_a, rows_b;    // rows of the two operands
  uint32_t blocks;            // ceil(k / 128)
  uint32_t atoms_a, atoms_b;  // groups of 128 rows in the scales
  uint32_t tiles_a;           // tiles along the M side
  uint32_t instruction;
  int dtype_d, accumulate;
};

constexpr int kTileA = 128;      // rows of the M side of a tile: one lane of tensor memory each
constexpr int kStageBlocks = 6;  // blocks of k in flight
constexpr int kMatmulThreads = 192;

// Shared memory of a block of threads: stages, each the two operand tiles and 1 KB of scales; the same memory holds the
// finished tile in fp32 afterwards.
__host__ __device__ constexpr int stage_bytes(int nt) { return (kTileA + nt) * 128 + 1024; }
__host__ __device__ constexpr int matmul_shared_bytes(int nt) { return 1024 + kStageBlocks * stage_bytes(nt); }

__device__ __forceinline__ void store_value(void* d, int dtype, uint64_t at, float v, bool accumulate) {
  if (dtype == kF32) {
    float* p = static_cast<float*>(d) + at;
    st_c(p, accumulate ? v + ld_c(p) : v);
  } else if (dtype == kBf16) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(d) + at;
    st_c(p, __float2bfloat16_rn(accumulate ? v + __bfloat162float(ld_c(p)) : v));
  } else {
    __half* p = static_cast<__half*>(d) + at;
    st_c(p, __float2half_rn(accumulate ? v + __half2float(ld_c(p)) : v));
  }
}

// One tile of 128 rows of the M-side operand by NT rows of the other, over this block's share of k; the blocks of a
// cluster (z) share k and add their sums in the order of their ranks.  TURNED: the M side is b (few rows of a), the
// tile's rows are columns of d.
template <int NT, bool TURNED>
__global__ void __launch_bounds__(kMatmulThreads) matmul_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                                const MatmulArgs a) {
  constexpr int kStage = stage_bytes(NT);
  constexpr int kScaleSlots = 4;             // words of scales in tensor memory, used in turn
  constexpr uint32_t kColumns = NT <= 32 ? 64 : NT <= 64 ? 128 : 256;  // NT sums and 32 columns of scales, a power of two
  constexpr uint32_t kScaleColumn = kColumns - 8 * kScaleSlots;
  extern __shared__ uint8_t raw_shared[];
  __shared__ __align__(8) uint64_t barriers[2 * kStageBlocks + 1];
  __shared__ uint32_t tensor_base, failed, issued;
  const uint32_t base = (smem_address(raw_shared) + 1023) & ~1023u;  // 128-byte swizzle repeats every 1024 bytes
  const uint32_t full = smem_address(barriers), empty = full + 8 * kStageBlocks, done = empty + 8 * kStageBlocks;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t parts = gridDim.z, rank = blockIdx.z;
  const uint32_t first = (uint32_t)((uint64_t)a.blocks * rank / parts), last = (uint32_t)((uint64_t)a.blocks * (rank + 1) / parts);
  const uint32_t row_a = blockIdx.x % a.tiles_a * kTileA, row_b = blockIdx.x / a.tiles_a * NT;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2 * kStageBlocks + 1; ++i) mbarrier_init(full + 8 * i, 1);
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

  if (warp == 4 && lane == 0) {  // loads
    uint32_t b = first;
    for (; b < last; ++b) {
      const uint32_t i = b - first, stage = i % kStageBlocks, round = i / kStageBlocks;
      if (round > 0 && !mbarrier_wait(empty + 8 * stage, (round - 1) & 1)) { atomicExch(&failed, 1u); break; }
      const uint32_t at = base + stage * kStage, bar = full + 8 * stage;
      const bool scales = i == 0 || (b & 3) == 0;  // a word of scales serves four blocks of k
      mbarrier_expect_bytes(bar, (kTileA + NT) * 128 + (scales ? 1024 : 0) + kCopyAnnounceExtra);
      tile_load(at, &map_a, b * 128, row_a, bar);
      tile_load(at + kTileA * 128, &map_b, b * 128, row_b, bar);
      if (scales) {
        bulk_copy_to_shared(at + (kTileA + NT) * 128, a.scale_a + ((uint64_t)(b >> 2) * a.atoms_a + row_a / 128) * 512, 512, bar);
        bulk_copy_to_shared(at + (kTileA + NT) * 128 + 512, a.scale_b + ((uint64_t)(b >> 2) * a.atoms_b + row_b / 128) * 512, 512, bar);
      }
    }
    issued = b - first;
  } else if (warp == 5 && lane == 0) {  // matrix instructions
    uint32_t slot = 0, scale_a = 0, scale_b = 0;
    bool ok = true;
    for (uint32_t b = first; b < last && ok; ++b) {
      const uint32_t i = b - first, stage = i % kStageBlocks, round = i / kStageBlocks;
      ok = mbarrier_wait(full + 8 * stage, round & 1);
      if (!ok) break;
      tensor_fence_after();
      const uint32_t at = base + stage * kStage;
      if (i == 0 || (b & 3) == 0) {
        scale_a = sums + kScaleColumn + 8 * slot;
        scale_b = scale_a + 4;
        slot = (slot + 1) % kScaleSlots;
        scale_copy(scale_a, scale_descriptor(at + (kTileA + NT) * 128));
        scale_copy(scale_b, scale_descriptor(at + (kTileA + NT) * 128 + 512));
      }
      const uint32_t instruction = with_scale_byte(a.instruction, b & 3);
      const uint64_t da = operand_descriptor(at), db = operand_descriptor(at + kTileA * 128);
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k)  // 32 values of k: 32 bytes further in the swizzled rows
        scaled_mma(sums, da + 2 * k, db + 2 * k, instruction, scale_a, scale_b + (row_b % 128) / 32, i > 0 || k > 0);
      mma_commit(empty + 8 * stage);
    }
    if (ok) mma_commit(done);
    else atomicExch(&failed, 1u);
  }
  __syncwarp();

  // The finished tile goes through shared memory as fp32, a row of d in a row of it.
  constexpr int kRows = TURNED ? NT : kTileA, kCols = TURNED ? kTileA : NT, kPitch = TURNED ? kTileA : NT + 4;
  float* tile = reinterpret_cast<float*>(raw_shared + (base - smem_address(raw_shared)));
  if (warp < 4) {
    const bool ok = mbarrier_wait(done, 0);
    if (!ok) atomicExch(&failed, 1u);
    tensor_fence_after();
    if (ok) {
      const uint32_t l = warp * 32 + lane;
#pragma unroll
      for (int c = 0; c < NT; c += 16) {
        float v[16];
        tensor_read(sums + ((warp * 32) << 16) + c, v);
        tensor_read_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (first == last) v[j] = 0.0f;  // no share of k: nothing was written there
          if (TURNED) tile[(c + j) * kPitch + l] = v[j];
        }
        if (!TURNED)
#pragma unroll
          for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4*>(tile + l * kPitch + c + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
      }
    }
    tensor_fence_before();
  }
  if (parts > 1) cluster_sync();
  else __syncthreads();
  if (warp == 0) {
    tensor_fence_after();
    tensor_free(sums, kColumns);
  }

  // Rows of the tile are dealt over the blocks of the cluster; each adds all blocks' sums and stores.
  const bool failure = *reinterpret_cast<volatile uint32_t*>(&failed) != 0;
  if (failure) {
    if (threadIdx.x == 0) {
      atomicOr(a.status, kDevCopyTimeout);
      // no copy of this block may still be on its way when it leaves
      for (uint32_t i = 0; i < issued && i < kStageBlocks; ++i) mbarrier_wait(full + 8 * i, ((issued - 1 - i) / kStageBlocks) & 1);
    }
  } else {
    const uint32_t d_rows = TURNED ? a.rows_b : a.rows_a, d_cols = TURNED ? a.rows_a : a.rows_b;
    const uint32_t row0 = TURNED ? row_b : row_a, col0 = TURNED ? row_a : row_b;
    const uint32_t tile_address = smem_address(tile);
    for (uint32_t r = rank + parts * warp; r < kRows && row0 + r < d_rows; r += parts * (kMatmulThreads / 32)) {
      for (uint32_t c = 4 * lane; c < kCols && col0 + c < d_cols; c += 128) {
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (uint32_t p = 0; p < parts; ++p) {
          const uint32_t at = tile_address + 4 * (r * kPitch + c);
          const float4 v = parts > 1 ? ld_cluster(address_in(at, p)) : *reinterpret_cast<const float4*>(tile + r * kPitch + c);
          s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const float out[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t col = col0 + c + j;
          if (col < d_cols) store_value(a.d, a.dtype_d, (uint64_t)(row0 + r) * a.ldd + col, out[j] + (a.bias ? ld_c(a.bias + col) : 0.0f), a.accumulate);
        }
      }
    }
  }
  if (parts > 1) cluster_sync();  // the other blocks may still be reading this one's tile
}

// ---- large products: pairs of SMs, tiles of 256 x 256, persistent -----------------------------------------------------
//
// Bound by the tensor cores.  A pair of blocks holds one tile (128 rows of it in each block's tensor memory); each
// block loads its own 128 rows of a and half of b, so an operand byte in shared memory feeds twice the products it would
// feed for one SM alone.  Each pair keeps taking units of work; the sums of the next one are formed while the last one's
// are read.  Two tiles of sums (2 x 256 columns) and the scales do not fit 512 columns side by side, so the two overlap by
// 24 columns: those are read first, and the next unit's products start once they are.
//
// A unit is a tile over all of k; the tiles that are left when every pair has had the same number (whole tiles) are cut
// along k into `parts`, so that all pairs share the last round.  A part's sums go to the workspace; the warp that
// is the last to bring its 32 rows of a tile adds all parts in their order.  No block waits for another pair.
//
// Sums that go out in fp32 are taken over at most kChunk blocks of k at a time and the chunks added one after the other
// (in d): the tensor cores' own sums over 16384 values of k are off by 1.1e-6 of the result's norm, over 8192 by 0.8e-6.
constexpr int kPairTile = 256;
constexpr int kPairStages = 6;
constexpr int kPairStageBytes = 2 * 128 * 128;            // 128 rows of a and 128 of b, 128 bytes each
constexpr int kPairScaleBytes = 512 + 1024;               // scales of 128 rows of a, of 256 of b, four blocks of k
constexpr int kPairStaging = 4 * 4096;                    // a piece of the result for each of four warps: 32 rows of 128 bytes
constexpr int kPairSharedBytes = 1024 + kPairStages * (kPairStageBytes + kPairScaleBytes) + kPairStaging + 4 * 4 * kPairTile;  // and each warp's copy of the bias
constexpr uint32_t kPairScaleColumn = 512 - 2 * 12;            // two words of scales in turn: 4 columns of a, 8 of b each
constexpr uint32_t kPairSecond = kPairScaleColumn - kPairTile; // where the second tile of sums starts
constexpr uint32_t kChunk = 64;

struct PairArgs {
  const float* bias;
  void* d;
  uint32_t* status;
  float* partials;     // parts of cut tiles: (tile, part) x 256 x 256 values
  uint32_t* arrivals;  // eight for each cut tile (two blocks of four warps), zero at the start
  uint64_t ldd;
  uint32_t m, n, blocks;
  uint32_t atoms_a, atoms_b;
  uint32_t tiles_m, tiles_n;
  uint32_t whole;      // tiles that are not cut
  uint32_t parts;      // of each of the others
  uint32_t chunks;     // of a whole tile, one after the other
  uint32_t instruction;
  int dtype_d, accumulate;
  int tile_stores;     // d is stored through its tensor map (16-byte aligned rows, nothing to add but in fp32)
};

// One accumulation: blocks [first, last) of k of a tile.
struct Unit {
  uint32_t tile_m, tile_n, first, last;
  uint32_t chunk;  // of a whole tile
  uint32_t cut;    // index of the cut tile, or ~0
  uint32_t part;
};

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

// 32 columns of a warp's 32 rows to d.  `piece`: the warp's 4 KB of shared memory.
template <bool SINGLE>
__device__ __forceinline__ void pair_store(const PairArgs& a, const CUtensorMap* map_d, uint8_t* piece, uint32_t piece_address, uint32_t lane,
                                           uint32_t row0, uint32_t col, bool add, uint32_t turn, float (&v)[32]) {
  if (a.tile_stores) {
    // row `lane` of the piece, its 16-byte units permuted as the tensor map's swizzle has them
    if (SINGLE) {
      if (lane == 0) store_wait_read<0>();
      __syncwarp();
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u)
        *reinterpret_cast<float4*>(piece + lane * 128 + 16 * (u ^ (lane & 7))) = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
    } else {
      if (lane == 0) store_wait_read<1>();  // two pieces of 2 KB in turn
      __syncwarp();
      piece += 2048 * (turn & 1);
      piece_address += 2048 * (turn & 1);
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u) {
        uint32_t w[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          const float x = v[8 * u + 2 * j], y = v[8 * u + 2 * j + 1];
          if (a.dtype_d == kBf16) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
            memcpy(&w[j], &h, 4);
          } else {
            const __half2 h = __floats2half2_rn(x, y);
            memcpy(&w[j], &h, 4);
          }
        }
        *reinterpret_cast<uint4*>(piece + lane * 64 + 16 * (u ^ ((lane >> 1) & 3))) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    shared_to_async();
    __syncwarp();
    if (lane == 0) {
      if (row0 < a.m && col < a.n) {
        if (SINGLE && add) tile_add(map_d, col, row0, piece_address);
        else tile_store(map_d, col, row0, piece_address);
      }
      store_commit();
    }
  } else {  // through shared memory so that a row's values leave side by side
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u)
      *reinterpret_cast<float4*>(piece + lane * 128 + 16 * (u ^ (lane & 7))) = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
    __syncwarp();
    if (col + lane < a.n)
      for (uint32_t r = 0; r < 32 && row0 + r < a.m; ++r)
        store_value(a.d, a.dtype_d, (uint64_t)(row0 + r) * a.ldd + col + lane,
                    *reinterpret_cast<const float*>(piece + r * 128 + 16 * ((lane >> 2) ^ (r & 7)) + 4 * (lane & 3)), add);
    __syncwarp();
  }
}

template <bool SINGLE>  // d is fp32
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMatmulThreads)
    matmul_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                       const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                       const __grid_constant__ CUtensorMap map_d, const PairArgs a) {
  extern __shared__ uint8_t raw_shared[];
  __shared__ __align__(8) uint64_t barriers[2 * kPairStages + 3];
  __shared__ uint32_t tensor_base, failed, issued;
  const uint32_t base = (smem_address(raw_shared) + 1023) & ~1023u;
  const uint32_t scales = base + kPairStages * kPairStageBytes, staging = scales + kPairStages * kPairScaleBytes;
  const uint32_t full = smem_address(barriers), empty = full + 8 * kPairStages, done = empty + 8 * kPairStages, drained = done + 16;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();
  const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2 * kPairStages + 2; ++i) mbarrier_init(full + 8 * i, 1);
    mbarrier_init(drained, 8);  // the four reading warps of both blocks
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

  if (warp == 4) {  // loads, in both blocks; the even block's barrier counts the bytes of both
    const bool leader = elect_one();
    const uint32_t full_cluster = address_in(full, 0);
    uint32_t i = 0, stage = 0, parity = 1;  // a fresh barrier passes for the phase before its first
    bool ok = true;
    Unit u;
    for (uint32_t unit = 0; ok && pair_unit(a, pair, pairs, unit, u); ++unit) {
      const uint32_t row_a = u.tile_m * kPairTile + rank * 128, row_b = u.tile_n * kPairTile + rank * 128;
      for (uint32_t b = u.first; b < u.last; ++b, ++i) {
        if (!mbarrier_wait_warp(empty + 8 * stage, parity)) { ok = false; break; }
        if (leader) {
          const bool with_scales = b == u.first || (b & 3) == 0;
          const uint32_t at = base + stage * kPairStageBytes, at_scales = scales + stage * kPairScaleBytes, bar = full_cluster + 8 * stage;
          if (rank == 0) mbarrier_expect_bytes(full + 8 * stage, 2 * (kPairStageBytes + (with_scales ? kPairScaleBytes : 0)) + kCopyAnnounceExtra);
          pair_tile_load(at, &map_a, b * 128, row_a, bar);
          pair_tile_load(at + 128 * 128, &map_b, b * 128, row_b, bar);
          if (with_scales) {
            pair_tile_load(at_scales, &map_sa, 0, (b >> 2) * a.atoms_a + u.tile_m * 2 + rank, bar);
            pair_tile_load(at_scales + 512, &map_sb, 0, (b >> 2) * a.atoms_b + u.tile_n * 2, bar);
          }
        }
        if (++stage == kPairStages) { stage = 0; parity ^= 1; }
      }
    }
    if (leader) {
      issued = i;
      if (!ok) atomicExch(&failed, 1u);
    }
  } else if (warp == 5 && rank == 0) {  // matrix instructions, for both blocks
    const bool leader = elect_one();
    const uint32_t tensor = __shfl_sync(0xffffffffu, sums, 0);
    uint32_t i = 0, stage = 0, parity = 0, word = 0;
    uint32_t used[2] = {0, 0};  // one past the last block of k that used each word of scales
    bool ok = true;
    Unit u;
    for (uint32_t unit = 0; ok && pair_unit(a, pair, pairs, unit, u); ++unit) {
      if (unit > 0 && !mbarrier_wait_warp(drained, (unit - 1) & 1)) { ok = false; break; }
      tensor_fence_after();
      const uint32_t into = tensor + (unit & 1 ? kPairSecond : 0);
      for (uint32_t b = u.first; b < u.last; ++b) {
        if (!mbarrier_wait_warp(full + 8 * stage, parity)) { ok = false; break; }
        tensor_fence_after();
        const bool fresh = b == u.first || (b & 3) == 0;  // a word of scales serves four blocks of k
        if (fresh) {
          // the products that used this word before must be done (at most five blocks back: that phase is the latest)
          word ^= 1;
          const uint32_t before = word ? used[1] : used[0];
          if (before != 0 && !mbarrier_wait_warp(empty + 8 * ((before - 1) % kPairStages), ((before - 1) / kPairStages) & 1)) { ok = false; break; }
        }
        ++i;
        if (word) used[1] = i;
        else used[0] = i;
        const uint32_t at = base + stage * kPairStageBytes, scale_a = tensor + kPairScaleColumn + 12 * word;
        const uint32_t instruction = with_scale_byte(a.instruction, b & 3);
        const uint64_t da = operand_descriptor(at), db = operand_descriptor(at + 128 * 128), ds = scale_descriptor(scales + stage * kPairScaleBytes);
        if (leader) {
          if (fresh) {
            pair_scale_copy(scale_a, ds);
            pair_scale_copy(scale_a + 4, ds + 32);
            pair_scale_copy(scale_a + 8, ds + 64);
          }
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k) pair_scaled_mma(into, da + 2 * k, db + 2 * k, instruction, scale_a, scale_a + 4, b > u.first || k > 0);
          pair_mma_commit(empty + 8 * stage);
        }
        if (++stage == kPairStages) { stage = 0; parity ^= 1; }
      }
      if (ok && leader) pair_mma_commit(done + 8 * (unit & 1));
    }
    if (!ok && leader) atomicExch(&failed, 1u);
  } else if (warp < 4) {  // results
    const uint32_t piece_address = staging + warp * 4096;
    uint8_t* piece = raw_shared + (piece_address - smem_address(raw_shared));
    float* bias_tile = reinterpret_cast<float*>(raw_shared + (staging + kPairStaging - smem_address(raw_shared))) + warp * kPairTile;
    const uint32_t drained_at = address_in(drained, 0);
    Unit u;
    for (uint32_t unit = 0; pair_unit(a, pair, pairs, unit, u); ++unit) {
      const uint32_t row0 = u.tile_m * kPairTile + rank * 128 + warp * 32, col0 = u.tile_n * kPairTile;
      const bool with_bias = a.bias && u.chunk == 0;
      if (with_bias) {
        __syncwarp();
        for (uint32_t c = lane; c < kPairTile; c += 32) bias_tile[c] = col0 + c < a.n ? ld_c(a.bias + col0 + c) : 0.0f;
        __syncwarp();
      }
      if (!mbarrier_wait(done + 8 * (unit & 1), (unit >> 1) & 1)) { atomicExch(&failed, 1u); break; }
      tensor_fence_after();
      const uint32_t from = sums + (unit & 1 ? kPairSecond : 0) + ((warp * 32) << 16);
      // a cut tile: this warp's 32 x 256 values of each part, as 8 x 8 x 32 pieces of four
      float4* partial = u.cut == ~0u ? nullptr : reinterpret_cast<float4*>(a.partials) + (((uint64_t)u.cut * a.parts * 2 + rank) * 4 + warp) * 2048;
      const uint64_t part_stride = 2 * 4 * 2048;
      if (u.chunk > 0 && lane == 0) store_wait();  // the chunk before must lie in d
#pragma unroll 1
      for (uint32_t turn = 0; turn < 8; ++turn) {  // 32 columns at a time, those shared with the next unit's sums first
        const uint32_t c = 32 * (unit & 1 ? turn : 7 - turn);
        float v[32];
        tensor_read(from + c, v);
        tensor_read_wait();
        if (turn == 0) {
          tensor_fence_before();
          __syncwarp();
          if (lane == 0) mbarrier_arrive_cluster(drained_at);
        }
        if (partial) {
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j)
            st_c(partial + u.part * part_stride + (c / 4 + j) * 32 + lane, make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
        } else {
          if (with_bias)
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += bias_tile[c + j];
          pair_store<SINGLE>(a, &map_d, piece, piece_address, lane, row0, col0 + c, a.accumulate || u.chunk > 0, turn, v);
        }
      }
      if (partial) {
        __threadfence();
        __syncwarp();
        uint32_t before = 0;
        if (lane == 0) before = atomicAdd(a.arrivals + (u.cut * 2 + rank) * 4 + warp, 1u);
        before = __shfl_sync(0xffffffffu, before, 0);
        if (before + 1 == a.parts) {  // all parts are there: add them in their order
          __threadfence();
#pragma unroll 1
          for (uint32_t turn = 0; turn < 8; ++turn) {
            const uint32_t c = 32 * turn;
            float v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.0f;
            for (uint32_t p = 0; p < a.parts; ++p)
#pragma unroll
              for (uint32_t j = 0; j < 8; ++j) {
                const float4 w = ld_c(partial + p * part_stride + (c / 4 + j) * 32 + lane);
                v[4 * j] += w.x; v[4 * j + 1] += w.y; v[4 * j + 2] += w.z; v[4 * j + 3] += w.w;
              }
            if (with_bias)
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] += bias_tile[c + j];
            pair_store<SINGLE>(a, &map_d, piece, piece_address, lane, row0, col0 + c, a.accumulate, turn, v);
          }
        }
      }
    }
    if (lane == 0) store_wait();
  }
  __syncwarp();
  __syncthreads();
  if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(&failed)) {
    atomicOr(a.status, kDevCopyTimeout);
    // no copy may still be on its way when a block of the pair leaves
    if (rank == 0)
      for (uint32_t i = 0; i < issued && i < kPairStages; ++i) mbarrier_wait(full + 8 * i, ((issued - 1 - i) / kPairStages) & 1);
  }
  tensor_fence_before();
  cluster_sync();
  tensor_fence_after();
  if (warp == 0) pair_tensor_free(sums, 512);
}

// k = 0: the sum is empty.
__global__ void __launch_bounds__(256) matmul_empty_kernel(const MatmulArgs a) {
  grid_dependency_handshake();
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = i / a.rows_b, col = i % a.rows_b;
  if (row < a.rows_a) store_value(a.d, a.dtype_d, row * a.ldd + col, a.bias ? ld_c(a.bias + col) : 0.0f, a.accumulate);
}

}  // namespace accept
