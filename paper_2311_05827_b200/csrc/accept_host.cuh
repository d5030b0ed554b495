// What the host sides of all entry points share: launching, counting launches, alignment tests, and the byte
// ranges that the checking build compares accesses with.
#pragma once
#include "../../include/accept.h"

#include <atomic>
#include <cstdint>
#include <cstdlib>
#include <utility>

#include <cuda_runtime.h>

#include "accept_device.cuh"

namespace accept {

extern std::atomic<uint64_t> g_launches;  // kernels launched by all entry points

inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Launch with programmatic stream serialization: every kernel of this library starts with
// grid_dependency_handshake(), so it may be scheduled while its predecessor in the stream drains.
template <typename... Params, typename... Args>
cudaError_t launch_overlapped_shared(void (*fn)(Params...), dim3 grid, unsigned block, size_t shared_bytes, cudaStream_t s,
                                     Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block, 1, 1);
  cfg.dynamicSmemBytes = shared_bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, fn, std::forward<Args>(args)...);
}

template <typename... Params, typename... Args>
cudaError_t launch_overlapped(void (*fn)(Params...), dim3 grid, unsigned block, cudaStream_t s, Args&&... args) {
  return launch_overlapped_shared(fn, grid, block, 0, s, std::forward<Args>(args)...);
}

// A launch (or any runtime call) that fails ends the entry point at once: later launches of the same call
// are not issued, and only launches that were issued are counted.  The result is the call's own return
// value; cudaGetLastError() is never consulted, so an error left behind by the caller's earlier work is
// neither reported as ours nor cleared.
#define ACCEPT_LAUNCH(call)                                         \
  do {                                                              \
    if ((call) != cudaSuccess) return ACCEPT_ERR_CUDA;              \
    accept::g_launches.fetch_add(1, std::memory_order_relaxed);             \
  } while (0)

// ---- tests-only build: byte ranges the kernels of a call may touch ------------------------------------
#ifdef ACCEPT_BOUNDS_CHECK
// ACCEPT_BOUNDS_TEST_SHRINK=<bytes> in the environment cuts that many bytes off the end of every writable
// range: the test of the checker itself, which shows that the last stores of a call are then counted and
// skipped (nothing is written there, nothing faults).
inline size_t bounds_test_shrink() {
  const char* text = std::getenv("ACCEPT_BOUNDS_TEST_SHRINK");
  return text ? (size_t)std::strtoull(text, nullptr, 10) : 0;
}

namespace {  // each source file has its own table on the device
struct BoundsList {
  BoundsTable table{};
  void add(const void* p, size_t bytes, bool writable) {
    if (!p || table.n >= kMaxBoundsRanges) return;
    if (writable) bytes -= bounds_test_shrink() < bytes ? bounds_test_shrink() : bytes;
    table.lo[table.n] = (unsigned long long)p;
    table.hi[table.n] = (unsigned long long)p + bytes;
    table.writable[table.n] = writable ? 1u : 0u;
    ++table.n;
  }
  // ordered with the call's kernels on its stream (the source is pageable host memory: staged before return)
  cudaError_t install(cudaStream_t s) const {
    return cudaMemcpyToSymbolAsync(g_bounds, &table, sizeof(table), 0, cudaMemcpyHostToDevice, s);
  }
};

// Adds this source file's tally of skipped accesses to the report (keeping the first one) and clears it.
inline bool collect_bounds(uint32_t* violations, unsigned long long (&first)[2]) {
  uint32_t count = 0;
  const uint32_t zero = 0;
  unsigned long long mine[2] = {0, 0};
  if (cudaMemcpyFromSymbol(&count, g_bounds_violations, sizeof(count)) != cudaSuccess) return false;
  if (cudaMemcpyFromSymbol(mine, g_bounds_first, sizeof(mine)) != cudaSuccess) return false;
  if (cudaMemcpyToSymbol(g_bounds_violations, &zero, sizeof(zero)) != cudaSuccess) return false;
  if (count != 0 && *violations == 0) { first[0] = mine[0]; first[1] = mine[1]; }
  *violations += count;
  return true;
}
}  // namespace
// the same for the files of the operators beside the codec
bool collect_norm_bounds(uint32_t* violations, unsigned long long (&first)[2]);
bool collect_block_bounds(uint32_t* violations, unsigned long long (&first)[2]);
bool collect_matmul_bounds(uint32_t* violations, unsigned long long (&first)[2]);
#define ACCEPT_BOUNDS(stream, ...)                                              \
  do {                                                                          \
    accept::BoundsList bounds_list;                                                     \
    __VA_ARGS__;                                                                \
    if (bounds_list.install(stream) != cudaSuccess) return ACCEPT_ERR_CUDA;     \
  } while (0)
#else
#define ACCEPT_BOUNDS(stream, ...) do { } while (0)
#endif

}  // namespace accept
