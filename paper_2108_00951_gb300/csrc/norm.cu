// norm.cu — layer norm's forward pass: y = (x - mean) rstd w + b over rows of d
// values, mean = sum x / d, rstd = (sum (x - mean)^2 / d + eps)^(-1/2).
//
// Both sums are fp32 over values that stay in registers, the second after the
// mean is known (a difference of squares would lose the variance of rows whose
// mean is large). rstd makes much of a last place of a large mean: of a row of
// 1000.0 it is 0.02 of y, of one near 1e5 all of it. So the product with 1 / d is
// corrected by its remainder, sum - mean d, and an fp32 row whose mean is beyond four
// deviations by the mean of its differences, which are exact there (bf16 values of
// one magnitude add up exactly); below, what the sum loses is at most
// 5 (depth + 2) 2^-24 deviations, depth its additions one after another.
//
// What bounds it: reading x and writing y once. A row of up to 256 values lies in
// lanes of a warp, of up to 2048 in warps, of up to 8192 in a CTA, of up to 65,536 in a
// cluster of CTAs; they take rows a stride apart, the next ones on their way into
// a ring in shared memory meanwhile, and the weights stay in registers. A longer
// row is read three times by one CTA, twice out of L2.
#include <algorithm>
#include <map>
#include <mutex>
#include <tuple>

#include "norm.cuh"

namespace efs {
namespace {

// Rows that a group has in its ring, with E values of a row a thread.
template <int E>
constexpr int kRing = E == 8 ? 8 : 4;

// The mean c of a row's differences from what its sum gave for a mean (divided: exact for a row of
// one value), and rstd without c^2 in the variance.
struct Correction {
  float c, rstd;
};
__device__ __forceinline__ Correction correction(float sum, float squares, uint32_t d, float inv, float eps) {
  const float c = sum / static_cast<float>(d), left = fmaf(-sum, c, squares);
  return {c, inverse_root((left < 0.0f ? 0.0f : left) * inv + eps)};  // (a NaN stays)
}

// (32 values a thread in 128 registers, narrow vectors with some of them spilled: 2000 x 9001 fp32
// 49 us, in 192 registers 75)
template <typename X, typename Y, int V, int K, RowKind KIND>
__global__ void __launch_bounds__(kNormThreads, V * K == 32 ? 2 : 0) norm_kernel(const NormCall a) {
  constexpr int S = kRing<V * K>;
  extern __shared__ __align__(16) char ring[];
  __shared__ RowRoom room;
  const RowGroup<KIND> g(a.threads);
  const RowPart part = row_part(a.d, a.part, a.cluster);
  const RowColumns<KIND, V> of(g, part.columns);
  const uint32_t per_cta = KIND == kRowAll ? 1u : blockDim.x / g.threads, t = g.t;
  const uint32_t groups = gridDim.x / a.cluster * per_cta;
  const uint32_t first = blockIdx.x / a.cluster * per_cta + g.index;
  const uint32_t place = row_place(a.part, sizeof(X));
  char* rows = ring + g.index * S * place;
  auto x_row = [&](uint32_t row) {
    return static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx + part.first;
  };
  auto fetch = [&](uint32_t row, uint32_t slot) {
    if (row < a.n) fetch_row(rows + slot * place, x_row(row), part.columns * sizeof(X), t, g.threads);
    fetch_commit();
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s) fetch(first + s * groups, s);
  float w[K][V], b[K][V];
  load_weights(a.w, a.w_bf16, a.w_wide, part.first, of.first, of.step(), of.end, 1.0f, w);
  load_weights(a.b, a.w_bf16, a.b_wide, part.first, of.first, of.step(), of.end, 0.0f, b);
  const float width = static_cast<float>(a.d), inv = 1.0f / width;
  if (KIND == kRowAll && a.cluster > 1) cluster_sync();  // (the others' shared memory is theirs)
  uint32_t slot = 0, parity = 0;
  // (the lanes of a warp go through its rows together: to the last round of the warp's first)
  const uint32_t ahead = KIND == kRowLanes ? g.index % (32u / g.threads) : 0u;
  for (uint32_t row = first; row - ahead < a.n; row += groups) {
    fetch_wait<S - 2>();
    g.sync();
    // (all threads are done with the row before: its place is free)
    fetch(row + (S - 1) * groups, slot == 0 ? S - 1 : slot - 1);
    const bool in = KIND != kRowLanes || row < a.n;
    const char* in_row = rows + slot * place + (in ? row_lead(x_row(row)) : 0u) + of.first * sizeof(X);
    slot = slot == S - 1 ? 0 : slot + 1;
    float x[K][V], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && of.has(k)) {
        const Vec<X, V> v = staged<X, V>(in_row, of.off(k));
#pragma unroll
        for (int j = 0; j < V; ++j) sum += x[k][j] = v.get(j);
      }
    }
    // (the fused product has the remainder exactly: of a row of one value, summed exactly, the
    // mean is that value)
    const float total = row_sum<KIND, false>(g, sum, 0.0f, room, 0, a.cluster, parity).x, near = total * inv;
    const float mean = fmaf(fmaf(-near, width, total), inv, near);
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && of.has(k))
#pragma unroll
        for (int j = 0; j < V; ++j) {
          x[k][j] -= mean;
          sum = fmaf(x[k][j], x[k][j], sum);
        }
    }
    const float squares = row_sum<KIND, false>(g, sum, 0.0f, room, 1, a.cluster, parity).x;
    const float var = squares * inv, rstd = inverse_root(var + a.eps);
    Y* y = static_cast<Y*>(a.y) + static_cast<uint64_t>(row) * a.ldy + part.first + of.first;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && of.has(k)) {
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = fmaf(x[k][j] * rstd, w[k][j], b[k][j]);
        Vec<Y, V> o;
        o.round(out);
        o.store(y + of.off(k));
      }
    }
    if (t == 0 && part.first == 0 && in) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    // A large mean: the row again, from its place in the ring. (All of a row's threads have the same
    // sums; the lanes of a warp go together. As a branch around the last pass, its values in
    // registers, it takes 2000 x 9001 from 42 to 50 us; for every row 32,768 x 4096 from 85 to 96.)
    const bool large = sizeof(X) == 4 && in && mean * mean > 16.0f * var;
    if (sizeof(X) == 4 && __builtin_expect(KIND == kRowLanes ? __any_sync(0xffffffffu, large) : large, 0)) {
      sum = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (in && of.has(k)) {
          const Vec<X, V> v = staged<X, V>(in_row, of.off(k));
#pragma unroll
          for (int j = 0; j < V; ++j) sum += x[k][j] = v.get(j) - mean;
        }
      }
      sum = row_sum<KIND, false>(g, sum, 0.0f, room, 0, a.cluster, parity).x;
      const Correction by = correction(sum, squares, a.d, inv, a.eps);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (large && of.has(k)) {
          float out[V];
#pragma unroll
          for (int j = 0; j < V; ++j) out[j] = fmaf((x[k][j] - by.c) * by.rstd, w[k][j], b[k][j]);
          Vec<Y, V> o;
          o.round(out);
          o.store(y + of.off(k));
        }
      }
      if (t == 0 && part.first == 0 && large) {
        if (a.mean) a.mean[row] = mean + by.c;
        if (a.rstd) a.rstd[row] = by.rstd;
      }
    }
  }
}

// Rows of any length, a CTA each.
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormCall a) {
  __shared__ float room[2][64];
  const X* x = static_cast<const X*>(a.x) + static_cast<uint64_t>(blockIdx.x) * a.ldx;
  Y* y = static_cast<Y*>(a.y) + static_cast<uint64_t>(blockIdx.x) * a.ldy;
  const float inv = 1.0f / static_cast<float>(a.d);
  float sum = 0.0f;
#pragma unroll 8
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) sum += widen(__ldg(x + c));
  const float mean = cta_sum2(sum, 0.0f, room[0]).x * inv;
  float squares = 0.0f;
  sum = 0.0f;
#pragma unroll 8
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    const float off = widen(__ldg(x + c)) - mean;
    sum += off;
    squares = fmaf(off, off, squares);
  }
  const float2 sums = cta_sum2(sum, squares, room[1]);
  const Correction by = correction(sums.x, sums.y, a.d, inv, a.eps);  // (of every row)
#pragma unroll 4
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    const float w = load_weight(a.w, a.w_bf16, c, 1.0f), b = load_weight(a.b, a.w_bf16, c, 0.0f);
    store_rounded(y + c, fmaf((widen(__ldg(x + c)) - mean - by.c) * by.rstd, w, b));
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[blockIdx.x] = mean + by.c;
    if (a.rstd) a.rstd[blockIdx.x] = by.rstd;
  }
}

template <typename X, typename Y, int V, int K, RowKind KIND>
cudaError_t launch_rows(NormCall c, uint32_t most, const DeviceInfo& dev, cudaStream_t stream) {
  RowPlan p;
  plan_row(p, reinterpret_cast<const void*>(norm_kernel<X, Y, V, K, KIND>), KIND, V * K, c.d, most);
  const cudaError_t err = plan_groups(p, kRing<V * K> * row_place(p.part, sizeof(X)), c.n, dev);
  if (err != cudaSuccess) return err;
  c.threads = p.threads;
  c.cluster = p.cluster;
  c.part = p.part;
  return launch_row(p, &c, stream);
}

template <typename X, typename Y, int V>
cudaError_t launch(const NormCall& c, const DeviceInfo& dev, cudaStream_t stream) {
  // Values of a row that a thread holds: fewer warps a row add up and wait less
  // (32,768 x 4096: 16 a thread 110 us, 32 85), more have more rows at once
  if (c.d <= 256) return launch_rows<X, Y, V, 8 / V, kRowLanes>(c, 256, dev, stream);
  if (c.d <= 2048) return launch_rows<X, Y, V, 16 / V, kRowWarps>(c, 2048, dev, stream);
  // Of a few long rows with narrow vectors, a thread's values are the wait: 255 x 24,209 fp32
  // 26.4 us with 32 a thread, 22.5 with 16 (30 x 9001 6.2 and 4.3; but 700 x 9001 23.5 and 25.1, and
  // 255 x 16,388, vectors of 4, 13.8 and 13.3: not worth their kernels)
  constexpr uint32_t kMany = 32 * kNormThreads, kFew = 16 * kNormThreads;
  if constexpr (V < 4)
    if (c.d > kMany && c.d <= kFew * kNormCluster && c.n <= 2u * dev.sm_count)
      return launch_rows<X, Y, V, 16 / V, kRowAll>(c, kFew, dev, stream);
  return launch_rows<X, Y, V, 32 / V, kRowAll>(c, kMany, dev, stream);
}

template <typename X, typename Y>
cudaError_t launch_typed(NormCall c, const DeviceInfo& dev, cudaStream_t stream) {
  if (c.d > kNormRowWidth) {
    norm_long_kernel<X, Y><<<c.n, 1024, 0, stream>>>(c);
    return cudaGetLastError();
  }
  constexpr bool kBoth16 = sizeof(X) == 2 && sizeof(Y) == 2;
  auto allow = [&](uint32_t v) {
    return c.d % v == 0 && rows_allow(c.x, c.n > 1 ? c.ldx : 0, sizeof(X), v) &&
           rows_allow(c.y, c.n > 1 ? c.ldy : 0, sizeof(Y), v);
  };
  const uint32_t v = kBoth16 && allow(8) ? 8 : allow(4) ? 4 : allow(2) ? 2 : 1;
  const uint64_t wsize = c.w_bf16 ? 2 : 4;
  const uint32_t vec = c.w_bf16 ? v : std::min(v, 4u);
  c.w_wide = rows_allow(c.w, 0, wsize, vec);
  c.b_wide = rows_allow(c.b, 0, wsize, vec);
  if constexpr (kBoth16)
    if (v == 8) return launch<X, Y, 8>(c, dev, stream);
  if (v == 4) return launch<X, Y, 4>(c, dev, stream);
  return v == 2 ? launch<X, Y, 2>(c, dev, stream) : launch<X, Y, 1>(c, dev, stream);
}

}  // namespace

cudaError_t resident_ctas(const void* kernel, uint32_t threads, uint32_t smem, uint32_t cluster,
                          const DeviceInfo& info, uint32_t* count) {
  using Key = std::tuple<int, const void*, uint32_t, uint32_t, uint32_t>;
  static std::mutex mu;
  static std::map<Key, uint32_t> known;
  struct Last {  // what a thread asked for last, by kernel
    Key key;
    uint32_t count;
  };
  static thread_local Last last[16] = {};
  int dev = 0, n = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const Key key(dev, kernel, threads, smem, cluster);
  Last& l = last[(reinterpret_cast<uintptr_t>(kernel) >> 4) % 16];
  if (l.count && l.key == key) {
    *count = l.count;
    return cudaSuccess;
  }
  std::lock_guard<std::mutex> lk(mu);
  const auto it = known.find(key);
  if (it != known.end()) {
    *count = it->second;
    l = {key, it->second};
    return cudaSuccess;
  }
  // (an opt-in stays: the largest asked for, whatever order sizes come in)
  err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  if (err != cudaSuccess) return err;
  if (cluster == 1) {
    err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem);
    n *= info.sm_count;
  } else {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster * static_cast<uint32_t>(info.sm_count));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    err = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
  }
  if (err != cudaSuccess) return err;
  if (n < 1) return cudaErrorLaunchOutOfResources;
  known.emplace(key, static_cast<uint32_t>(n));
  *count = static_cast<uint32_t>(n);
  return cudaSuccess;
}

cudaError_t launch_layer_norm(const NormCall& c, const DeviceInfo& dev, cudaStream_t stream) {
  count_launch();
  if (c.x_bf16)
    return c.y_bf16 ? launch_typed<bf16_t, bf16_t>(c, dev, stream) : launch_typed<bf16_t, float>(c, dev, stream);
  return c.y_bf16 ? launch_typed<float, bf16_t>(c, dev, stream) : launch_typed<float, float>(c, dev, stream);
}

}  // namespace efs
