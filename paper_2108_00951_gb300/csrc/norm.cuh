// norm.cuh — what layer norm's forward and backward kernels share: the row's
// columns over the lanes of a warp or the threads of a CTA, the weights, sums.
#pragma once

#include "internal.h"
#include "vec_io.cuh"

namespace efs {

constexpr int kNormMaxThreads = 512;

// V values of a weight vector of either type, or `none` where there is no vector. It lies in
// L1 after a CTA's first row, so a vector at any alignment is read value by value.
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

// Sums of `a` and `b` over the threads of a CTA, in a fixed order; `room`: 64
// floats that no other sum uses before the next barrier.
__device__ __forceinline__ float2 cta_sum2(float a, float b, float* room) {
  a = warp_sum(a);
  b = warp_sum(b);
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, warps = (blockDim.x + 31) >> 5;
  if (lane == 0) room[warp] = a, room[32 + warp] = b;
  __syncthreads();
  a = lane < warps ? room[lane] : 0.0f;
  b = lane < warps ? room[32 + lane] : 0.0f;
  return make_float2(warp_sum(a), warp_sum(b));
}
__device__ __forceinline__ float cta_sum(float a, float* room) {
  a = warp_sum(a);
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, warps = (blockDim.x + 31) >> 5;
  if (lane == 0) room[warp] = a;
  __syncthreads();
  a = lane < warps ? room[lane] : 0.0f;
  return warp_sum(a);
}

// The widest vectors that rows of a type allow: as many values as every pointer
// and stride (in bytes) and the width are multiples of.
inline bool rows_allow(uint64_t at, uint64_t ld, uint64_t size, uint32_t v) {
  return (at | ld * size) % (size * v) == 0;
}

}  // namespace efs
