// row_ring.cuh — rows of a matrix on their way into shared memory by asynchronous
// copies, at any alignment.
#pragma once

#include "tma.cuh"
#include "vec_io.cuh"

namespace efs {

// A row in shared memory as it lies in memory: copies of 16 bytes from the
// 16-byte boundary at or before its start on, so that rows at any alignment are
// read by wide copies. (The bytes before the start lie in the same 16 as the
// row's first: within the allocation. Past the row's end nothing is read.)
__device__ __forceinline__ uint32_t row_lead(const void* row) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row)) & 15u;
}
__device__ __forceinline__ void fetch_row(char* to, const void* row, uint32_t bytes, uint32_t t,
                                          uint32_t group) {
  const uint32_t lead = row_lead(row), total = lead + bytes;
  const char* from = static_cast<const char*>(row) - lead;
  const uint32_t at = smem_u32(to);
  for (uint32_t c = t * 16; c < total; c += group * 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + c), "l"(from + c),
                 "r"(min(16u, total - c))
                 : "memory");
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the last N groups have landed.
template <int N>
__device__ __forceinline__ void fetch_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// Bytes of a row's place in the ring.
__host__ __device__ __forceinline__ uint32_t row_place(uint32_t d, uint32_t size) {
  return (d * size + 15u + 15u) / 16u * 16u;
}

// V values of a row in shared memory.
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> staged(const char* row, uint32_t c) {
  Vec<T, V> x;
  x.load_own(reinterpret_cast<const T*>(row) + c);
  return x;
}

}  // namespace efs
