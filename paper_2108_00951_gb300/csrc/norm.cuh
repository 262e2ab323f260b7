// norm.cuh — what layer norm's forward and backward kernels share: rows that come
// through a ring in shared memory, their columns over the lanes of a warp or the
// threads of a CTA, the weights, sums.
#pragma once

#include "internal.h"
#include "row_ring.cuh"

namespace efs {

constexpr uint32_t kNormMaxThreads = 512;
constexpr uint32_t kNormPerThread = 16;   // values of a row that a thread of a CTA holds
constexpr uint32_t kNormCtaWidth = kNormMaxThreads * kNormPerThread;  // longest row in a CTA's registers
constexpr uint32_t kNormWarpWidth = 1024; // longest row of a warp

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

template <int V, int W>
__device__ __forceinline__ void load_weights(const void* w, bool bf16, bool wide, uint32_t c,
                                             float none, Lane<W> (&out)[V / W]) {
  float f[V];
  load_weights<V>(w, bf16, wide, c, none, f);
#pragma unroll
  for (int i = 0; i < V / W; ++i) out[i] = Lane<W>::of(f + i * W);
}

// The sum of `a` over the threads of a CTA, in a fixed order. `room`: 32 floats, zero from the
// last warp's on, that no other sum uses before the next barrier but one.
__device__ __forceinline__ float cta_sum(float a, float* room) {
  a = warp_sum(a);
  const uint32_t warps = (blockDim.x + 31) >> 5;
  if ((threadIdx.x & 31u) == 0) room[threadIdx.x >> 5] = a;
  __syncthreads();
  a = 0.0f;
  for (uint32_t i = 0; i < warps; i += 4) {
    const float4 x = *reinterpret_cast<const float4*>(room + i);
    a += (x.x + x.y) + (x.z + x.w);
  }
  return a;
}
// Two of them; `room` as above, 64 floats.
__device__ __forceinline__ float2 cta_sum2(float a, float b, float* room) {
  a = warp_sum(a);
  b = warp_sum(b);
  const uint32_t warps = (blockDim.x + 31) >> 5;
  if ((threadIdx.x & 31u) == 0) {
    room[threadIdx.x >> 5] = a;
    room[32 + (threadIdx.x >> 5)] = b;
  }
  __syncthreads();
  a = b = 0.0f;
  for (uint32_t i = 0; i < warps; i += 4) {
    const float4 x = *reinterpret_cast<const float4*>(room + i);
    const float4 y = *reinterpret_cast<const float4*>(room + 32 + i);
    a += (x.x + x.y) + (x.z + x.w);
    b += (y.x + y.y) + (y.z + y.w);
  }
  return make_float2(a, b);
}
// Zeros for a sum's room, seen by all after the CTA's next barrier.
__device__ __forceinline__ void clear_room(float* room, uint32_t floats) {
  if (threadIdx.x < floats) room[threadIdx.x] = 0.0f;
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
