// norm.cuh — what layer norm's forward and backward kernels share: a row's columns
// over lanes, warps, a CTA or a cluster; the weights; sums.
#pragma once

#include <algorithm>

#include "internal.h"
#include "row_ring.cuh"
#include "tensor.cuh"

namespace efs {

constexpr uint32_t kNormThreads = 256;      // of a CTA, at most
constexpr uint32_t kNormCluster = 8;        // CTAs that have a row together, at most
constexpr uint32_t kNormRowWidth = 65536;   // longest row that threads hold

// The threads of a CTA that have a row (or a CTA's part of one) together, with which no
// others wait: 1 to 32 lanes of a warp, a number of whole warps, or all.
enum RowKind { kRowLanes, kRowWarps, kRowAll };
template <RowKind KIND>
struct RowGroup {
  uint32_t threads, index, t;  // how many, the group's number in the CTA, this thread's in the group
  __device__ __forceinline__ explicit RowGroup(uint32_t of_row) {
    threads = KIND == kRowAll ? blockDim.x : of_row;
    index = KIND == kRowAll ? 0u : threadIdx.x / threads;
    t = threadIdx.x - index * threads;
  }
  __device__ __forceinline__ void sync() const {
    if (KIND == kRowAll) __syncthreads();
    else if (KIND == kRowLanes || threads == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(index + 1u), "r"(threads) : "memory");
  }
};
// Threads for `columns` with `values` a thread.
inline uint32_t row_threads(RowKind kind, uint32_t columns, uint32_t values) {
  const uint32_t least = (columns + values - 1) / values;
  if (kind != kRowLanes) return (least + 31) / 32 * 32;
  uint32_t lanes = 1;
  while (lanes < least) lanes *= 2;
  return lanes;
}

// What the CTAs of a cluster have of a row: `part` columns each.
struct RowPart {
  uint32_t first, columns;  // of this CTA
};
__device__ __forceinline__ RowPart row_part(uint32_t d, uint32_t part, uint32_t cluster) {
  if (cluster == 1) return {0u, d};
  const uint32_t first = blockIdx.x % cluster * part;
  return {first, min(part, d - first)};
}

// A thread's columns of a row, or of a CTA's part of one: K vectors of V, `step` apart. A warp's
// columns lie together, so that its steps are constants of the addresses.
template <RowKind KIND, int V>
struct RowColumns {
  uint32_t first, end, lanes;
  __device__ __forceinline__ RowColumns(const RowGroup<KIND>& g, uint32_t columns)
      : first(g.t * V), end(columns), lanes(g.threads) {
    if (KIND == kRowLanes) return;
    const uint32_t per = (columns + g.threads * V - 1) / (g.threads * V) * (32 * V), warp = g.t >> 5;
    first = warp * per + (g.t & 31u) * V;
    end = min(columns, (warp + 1) * per);
  }
  __device__ __forceinline__ uint32_t step() const { return KIND == kRowLanes ? lanes * V : 32u * V; }
  __device__ __forceinline__ uint32_t off(int k) const { return k * step(); }  // from the first
  __device__ __forceinline__ bool has(int k) const { return first + off(k) < end; }
};

// A thread's K vectors of V values, `step` columns apart, of a weight vector of either type, or
// `none` where there is no vector. (All are on their way before one is widened: with a vector
// at a time, both passes over 3 rows of 7398 with bf16 weights take 19.7 us, so 11.3.)
template <typename T, int V, int PART, int K>
__device__ __forceinline__ void load_vectors(const T* w, uint32_t c, uint32_t step, uint32_t columns,
                                             float (&out)[K][V]) {
  Vec<T, PART> x[K][V / PART];
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (c + k * step < columns)
#pragma unroll
      for (int i = 0; i < V / PART; ++i) x[k][i].load(w + c + k * step + i * PART);
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (c + k * step < columns)
#pragma unroll
      for (int j = 0; j < V; ++j) out[k][j] = x[k][j / PART].get(j % PART);
}
template <int V, int K>
__device__ __forceinline__ void load_weights(const void* w, bool bf16, bool wide, uint32_t first, uint32_t c,
                                             uint32_t step, uint32_t columns, float none, float (&out)[K][V]) {
  if (!w) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) out[k][j] = none;
  } else if (bf16) {
    const bf16_t* p = static_cast<const bf16_t*>(w) + first;
    if (wide) load_vectors<bf16_t, V, V>(p, c, step, columns, out);
    else load_vectors<bf16_t, V, 1>(p, c, step, columns, out);
  } else {
    const float* p = static_cast<const float*>(w) + first;
    if (wide) load_vectors<float, V, (V > 4 ? 4 : V)>(p, c, step, columns, out);
    else load_vectors<float, V, 1>(p, c, step, columns, out);
  }
}
// One value of it.
__device__ __forceinline__ float load_weight(const void* w, bool bf16, uint32_t c, float none) {
  if (!w) return none;
  return bf16 ? bf16_bits_to_f32(__ldg(static_cast<const bf16_t*>(w) + c)) : __ldg(static_cast<const float*>(w) + c);
}

// The sum of a value (or of TWO) over a row's threads, in a fixed order, across the CTAs of a
// cluster too. `Room` lies in shared memory; no sum writes what a thread may still read
// of the one before, as long as the group meets between two rows.
struct __align__(16) RowRoom {
  float2 warp[2][kNormThreads / 32];       // by the sum's number in the row
  float2 peer[2][kNormCluster];            // by the parity of the cluster's sums
};
template <RowKind KIND, bool TWO>
__device__ __forceinline__ float2 row_sum(const RowGroup<KIND>& g, float a, float b, RowRoom& room, uint32_t which,
                                          uint32_t cluster, uint32_t& parity) {
  if (KIND == kRowLanes) {
    for (uint32_t o = g.threads >> 1; o > 0; o >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      if (TWO) b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    return make_float2(a, b);
  }
  a = warp_sum(a);
  if (TWO) b = warp_sum(b);
  if (KIND == kRowAll || g.threads > 32) {
    const uint32_t warps = g.threads >> 5;
    float2* mine = room.warp[which] + g.index * warps;
    if ((threadIdx.x & 31u) == 0) mine[g.t >> 5] = make_float2(a, b);
    g.sync();
    a = b = 0.0f;
#pragma unroll 4
    for (uint32_t i = 0; i < warps; ++i) {
      const float2 x = mine[i];
      a += x.x;
      if (TWO) b += x.y;
    }
  }
  if (KIND == kRowAll && cluster > 1) {
    if (threadIdx.x < cluster)
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(
                       cluster_addr(&room.peer[parity][blockIdx.x % cluster], threadIdx.x)),
                   "f"(a), "f"(b)
                   : "memory");
    cluster_sync();
    a = b = 0.0f;
    for (uint32_t i = 0; i < cluster; ++i) {
      const float2 x = room.peer[parity][i];
      a += x.x;
      if (TWO) b += x.y;
    }
    parity ^= 1u;
  }
  return make_float2(a, b);
}

// The same over a CTA (of rows that no threads hold).
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

// How the rows of a call are spread.
struct RowPlan {
  const void* kernel;
  uint32_t threads;   // of a row in a CTA
  uint32_t cluster;   // CTAs of a row
  uint32_t part;      // columns of a row in a CTA
  uint32_t per_cta;   // rows that a CTA has at once
  uint32_t groups;    // rows that are had at once
  uint32_t smem;
};
// `values`: of a row in a thread; `most`: columns in a CTA.
inline void plan_row(RowPlan& p, const void* kernel, RowKind kind, uint32_t values, uint32_t d, uint32_t most) {
  p.kernel = kernel;
  p.cluster = (d + most - 1) / most;
  p.part = p.cluster == 1 ? d : ((d + p.cluster - 1) / p.cluster + 15) / 16 * 16;
  p.threads = row_threads(kind, p.part, values);
  p.per_cta = kind == kRowAll ? 1 : kNormThreads / p.threads;
}
// `ring`: bytes of shared memory of a row's threads.
inline cudaError_t plan_groups(RowPlan& p, uint32_t ring, uint32_t n, const DeviceInfo& dev) {
  p.smem = p.per_cta * ring;
  uint32_t resident = 0;
  const cudaError_t err = resident_ctas(p.kernel, p.per_cta * p.threads, p.smem, p.cluster, dev, &resident);
  p.groups = std::min((n + p.per_cta - 1) / p.per_cta, resident);
  return err;
}
inline cudaError_t launch_row(const RowPlan& p, void* params, cudaStream_t stream) {
  void* args[] = {params};
  const dim3 grid(p.groups * p.cluster), block(p.per_cta * p.threads);
  if (p.cluster == 1) return cudaLaunchKernel(p.kernel, grid, block, args, p.smem, stream);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = p.cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelExC(&cfg, p.kernel, args);
}

}  // namespace efs
