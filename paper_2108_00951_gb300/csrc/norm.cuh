// norm.cuh — what layer norm's forward and backward kernels share: rows that come
// through a ring in shared memory, their columns over the lanes of a warp or the
// threads of a CTA, the weights, sums.
#pragma once

#include "internal.h"
#include "row_ring.cuh"

namespace efs {

constexpr uint32_t kNormThreads = 256;    // of a CTA that has several rows at once
constexpr uint32_t kNormRowWidth = 8192;  // longest row that threads hold

// The threads that have a row together: 1, 2, 4 or 8 warps of a CTA, with which no
// other threads of the CTA wait. ALL: the whole CTA.
template <bool ALL>
struct RowGroup {
  uint32_t warps, index, t;  // warps of the group, its number in the CTA, this thread's in the group
  __device__ __forceinline__ explicit RowGroup(uint32_t of_row) {
    warps = ALL ? blockDim.x >> 5 : of_row;
    index = ALL ? 0u : threadIdx.x / (warps * 32u);
    t = threadIdx.x - index * warps * 32u;
  }
  __device__ __forceinline__ uint32_t threads() const { return warps * 32u; }
  __device__ __forceinline__ void sync() const {
    if (ALL) __syncthreads();
    else if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(index + 1u), "r"(warps * 32u) : "memory");
  }
};
// Warps for rows of d values with `per` a thread: a power of two.
inline uint32_t row_warps(uint32_t d, uint32_t per) {
  uint32_t warps = 1;
  while (warps * 32 * per < d) warps *= 2;
  return warps;
}

// V values of a weight vector of either type, or `none` where there is no vector.
template <int V>
__device__ __forceinline__ void load_weights(const void* w, bool bf16, bool wide, uint32_t c,
                                             float none, float (&out)[V]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = none;
  } else if (bf16) {
    const bf16_t* p = static_cast<const bf16_t*>(w) + c;
    if (wide) {
      Vec<bf16_t, V> x;
      x.load(p);
#pragma unroll
      for (int j = 0; j < V; ++j) out[j] = x.get(j);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) out[j] = bf16_bits_to_f32(__ldg(p + j));
    }
  } else {
    const float* p = static_cast<const float*>(w) + c;
    constexpr int kPart = V > 4 ? 4 : V;
    if (wide) {
#pragma unroll
      for (int j = 0; j < V; j += kPart) {
        Vec<float, kPart> x;
        x.load(p + j);
#pragma unroll
        for (int i = 0; i < kPart; ++i) out[j + i] = x.get(i);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) out[j] = __ldg(p + j);
    }
  }
}

// Sums over the threads of a group, in a fixed order. `room`: 16 floats of the
// CTA's a sum, which no other sum uses before the group's next barrier but one.
template <bool ALL>
__device__ __forceinline__ float group_sum(const RowGroup<ALL>& g, float a, float* room) {
  a = warp_sum(a);
  if (g.warps == 1) return a;
  if ((threadIdx.x & 31u) == 0) room[threadIdx.x >> 5] = a;
  g.sync();
  const float* mine = room + g.index * g.warps;
  a = 0.0f;
  for (uint32_t i = 0; i < g.warps; i += 2) {
    const float2 x = *reinterpret_cast<const float2*>(mine + i);
    a += x.x + x.y;
  }
  return a;
}
// Two of them; `room`: 32 floats.
template <bool ALL>
__device__ __forceinline__ float2 group_sum2(const RowGroup<ALL>& g, float a, float b, float* room) {
  a = warp_sum(a);
  b = warp_sum(b);
  if (g.warps == 1) return make_float2(a, b);
  if ((threadIdx.x & 31u) == 0) *reinterpret_cast<float2*>(room + 2 * (threadIdx.x >> 5)) = make_float2(a, b);
  g.sync();
  const float* mine = room + 2 * g.index * g.warps;
  a = b = 0.0f;
  for (uint32_t i = 0; i < 2 * g.warps; i += 4) {
    const float4 x = *reinterpret_cast<const float4*>(mine + i);
    a += x.x + x.z;
    b += x.y + x.w;
  }
  return make_float2(a, b);
}

// The same over a CTA (of rows that no group's registers hold).
__device__ __forceinline__ float2 cta_sum2(float a, float b, float* room) {
  a = warp_sum(a);
  b = warp_sum(b);
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if (lane == 0) room[warp] = a, room[32 + warp] = b;
  __syncthreads();
  a = lane < warps ? room[lane] : 0.0f;
  b = lane < warps ? room[32 + lane] : 0.0f;
  return make_float2(warp_sum(a), warp_sum(b));
}

// (var + eps)^(-1/2): the approximate root and one Newton step. Infinity for 0, as the
// exact one is (the step would make it NaN).
__device__ __forceinline__ float inverse_root(float x) {
  const float y = rsqrtf(x);
  const float z = y * fmaf(-0.5f * x * y, y, 1.5f);
  return x > 1e-35f && x < 1e35f ? z : y;
}

// The widest vectors that rows of a type allow: as many values as every pointer
// and stride (in bytes) and the width are multiples of.
inline bool rows_allow(const void* at, uint64_t ld, uint64_t size, uint32_t v) {
  return (reinterpret_cast<uintptr_t>(at) | ld * size) % (size * v) == 0;
}

}  // namespace efs
