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

// k = 0: the sum is empty.
__global__ void __launch_bounds__(256) matmul_empty_kernel(const MatmulArgs a) {
  grid_dependency_handshake();
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = i / a.rows_b, col = i % a.rows_b;
  if (row < a.rows_a) store_value(a.d, a.dtype_d, row * a.ldd + col, a.bias ? ld_c(a.bias + col) : 0.0f, a.accumulate);
}

}  // namespace accept
