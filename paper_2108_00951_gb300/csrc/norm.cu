// norm.cu — layer norm's forward pass: y = (x - mean) rstd w + b over rows of d
// values, mean = sum x / d, rstd = (sum (x - mean)^2 / d + eps)^(-1/2).
//
// Both sums are fp32 over values that stay in registers, the second after the
// mean is known (a difference of squares would lose the variance of rows whose
// mean is large). What bounds it: reading x and writing y once. A warp (rows of at
// most 1024 values, no barrier) or a CTA (at most 8192) takes rows a stride apart; the
// next ones are on their way into a ring in shared memory meanwhile, and the
// weights stay in registers. A longer row is read three times, twice out of L1
// and L2.
#include <algorithm>
#include <map>
#include <mutex>
#include <tuple>

#include "norm.cuh"

namespace efs {
namespace {

constexpr uint32_t kWarpsPerCta = 4;
// Rows that a group has in its ring, with K V values of a row a thread.
template <int E, bool WARP>
constexpr int kRing = !WARP ? 4 : E == 8 ? 8 : E == 16 ? 4 : 3;

template <typename X, typename Y, int V, int K, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kWarpsPerCta : kNormMaxThreads) norm_kernel(const NormCall a) {
  constexpr int S = kRing<V * K, WARP>, W = V > 1 ? 2 : 1;
  using L = Lane<W>;
  extern __shared__ __align__(16) char ring[];
  __shared__ __align__(16) float room[2][32];
  const uint32_t group = WARP ? 32u : blockDim.x;
  const uint32_t t = WARP ? threadIdx.x & 31u : threadIdx.x;
  const uint32_t groups = WARP ? gridDim.x * kWarpsPerCta : gridDim.x;
  const uint32_t first = WARP ? blockIdx.x * kWarpsPerCta + (threadIdx.x >> 5) : blockIdx.x;
  const uint32_t place = row_place(a.d, sizeof(X));
  char* rows = ring + (WARP ? (threadIdx.x >> 5) * S * place : 0u);
  auto x_row = [&](uint32_t row) { return static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx; };
  auto fetch = [&](uint32_t row, uint32_t slot) {
    if (row < a.n) fetch_row(rows + slot * place, x_row(row), a.d * sizeof(X), t, group);
    fetch_commit();
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s) fetch(first + s * groups, s);
  L w[K][V / W], b[K][V / W];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t c = (k * group + t) * V;
    if (c < a.d) {
      load_weights<V, W>(a.w, a.w_bf16, a.w_wide, c, 1.0f, w[k]);
      load_weights<V, W>(a.b, a.w_bf16, a.b_wide, c, 0.0f, b[k]);
    }
  }
  const float inv = 1.0f / static_cast<float>(a.d);
  if (!WARP) {
    clear_room(room[0], 64);
    __syncthreads();
  }
  uint32_t slot = 0;
  for (uint32_t row = first; row < a.n; row += groups) {
    fetch_wait<S - 2>();
    if (WARP) __syncwarp();
    else __syncthreads();
    // (all threads are done with the row before: its place is free)
    fetch(row + (S - 1) * groups, slot == 0 ? S - 1 : slot - 1);
    const char* in_row = rows + slot * place + row_lead(x_row(row));
    slot = slot == S - 1 ? 0 : slot + 1;
    L x[K][V / W], sums = L::all(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * group + t) * V;
      if (c < a.d) {
        const Vec<X, V> in = staged<X, V>(in_row, c);
#pragma unroll
        for (int j = 0; j < V / W; ++j) {
          x[k][j] = in.template lane<W>(j);
          sums = sums + x[k][j];
        }
      }
    }
    const float mean = (WARP ? warp_sum(sums.sum()) : cta_sum(sums.sum(), room[0])) * inv;
    const L minus = L::all(-mean);
    sums = L::all(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if ((k * group + t) * V < a.d)
#pragma unroll
        for (int j = 0; j < V / W; ++j) {
          x[k][j] = x[k][j] + minus;
          sums = fma(x[k][j], x[k][j], sums);
        }
    }
    const float var = (WARP ? warp_sum(sums.sum()) : cta_sum(sums.sum(), room[1])) * inv;
    const float rstd = inverse_root(var + a.eps);
    const L r = L::all(rstd);
    Y* y = static_cast<Y*>(a.y) + static_cast<uint64_t>(row) * a.ldy;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * group + t) * V;
      if (c < a.d) {
        L out[V / W];
#pragma unroll
        for (int j = 0; j < V / W; ++j) out[j] = fma(x[k][j] * r, w[k][j], b[k][j]);
        Vec<Y, V> o;
        o.template round<W>(out);
        o.store(y + c);
      }
    }
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

// Rows of any length, a CTA each.
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormCall a) {
  __shared__ __align__(16) float room[2][32];
  clear_room(room[0], 64);
  __syncthreads();
  const X* x = static_cast<const X*>(a.x) + static_cast<uint64_t>(blockIdx.x) * a.ldx;
  Y* y = static_cast<Y*>(a.y) + static_cast<uint64_t>(blockIdx.x) * a.ldy;
  const float inv = 1.0f / static_cast<float>(a.d);
  float sum = 0.0f;
#pragma unroll 8
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) sum += widen(__ldg(x + c));
  const float mean = cta_sum(sum, room[0]) * inv;
  sum = 0.0f;
#pragma unroll 8
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    const float off = widen(__ldg(x + c)) - mean;
    sum = fmaf(off, off, sum);
  }
  const float rstd = inverse_root(cta_sum(sum, room[1]) * inv + a.eps);
#pragma unroll 4
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    float w[1], b[1];
    load_weights<1>(a.w, a.w_bf16, true, c, 1.0f, w);
    load_weights<1>(a.b, a.w_bf16, true, c, 0.0f, b);
    store_rounded(y + c, fmaf((widen(__ldg(x + c)) - mean) * rstd, w[0], b[0]));
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[blockIdx.x] = mean;
    if (a.rstd) a.rstd[blockIdx.x] = rstd;
  }
}

template <typename X, typename Y, int V, int K, bool WARP>
cudaError_t launch_rows(const NormCall& c, const DeviceInfo& dev, cudaStream_t stream) {
  const uint32_t warps = WARP ? kWarpsPerCta : 1;  // groups of a CTA
  const uint32_t threads =
      WARP ? 32 * kWarpsPerCta : ((c.d + kNormPerThread - 1) / kNormPerThread + 31) / 32 * 32;
  const uint32_t smem = warps * kRing<V * K, WARP> * row_place(c.d, sizeof(X));
  const void* fn = reinterpret_cast<const void*>(norm_kernel<X, Y, V, K, WARP>);
  uint32_t per_sm = 0;
  const cudaError_t err = resident_ctas(fn, threads, smem, &per_sm);
  if (err != cudaSuccess) return err;
  const uint32_t grid = std::min((c.n + warps - 1) / warps, per_sm * static_cast<uint32_t>(dev.sm_count));
  norm_kernel<X, Y, V, K, WARP><<<grid, threads, smem, stream>>>(c);
  return cudaGetLastError();
}

template <typename X, typename Y, int V>
cudaError_t launch(const NormCall& c, const DeviceInfo& dev, cudaStream_t stream) {
  if (c.d <= 256) return launch_rows<X, Y, V, 8 / V, true>(c, dev, stream);
  if (c.d <= 512) return launch_rows<X, Y, V, 16 / V, true>(c, dev, stream);
  if (c.d <= kNormWarpWidth) return launch_rows<X, Y, V, 32 / V, true>(c, dev, stream);
  return launch_rows<X, Y, V, kNormPerThread / V, false>(c, dev, stream);
}

template <typename X, typename Y>
cudaError_t launch_typed(NormCall c, const DeviceInfo& dev, cudaStream_t stream) {
  if (c.d > kNormCtaWidth) {
    norm_long_kernel<X, Y><<<c.n, 1024, 0, stream>>>(c);
    return cudaGetLastError();
  }
  constexpr uint32_t kWide = sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
  auto allow = [&](uint32_t v) {
    return c.d % v == 0 && rows_allow(c.x, c.n > 1 ? c.ldx : 0, sizeof(X), v) &&
           rows_allow(c.y, c.n > 1 ? c.ldy : 0, sizeof(Y), v);
  };
  const uint32_t v = allow(kWide) ? kWide : allow(2) ? 2 : 1;
  const uint64_t wsize = c.w_bf16 ? 2 : 4;
  const uint32_t part = c.w_bf16 ? v : std::min(v, 4u);
  c.w_wide = rows_allow(c.w, 0, wsize, part);
  c.b_wide = rows_allow(c.b, 0, wsize, part);
  if (v == kWide) return launch<X, Y, kWide>(c, dev, stream);
  return v == 2 ? launch<X, Y, 2>(c, dev, stream) : launch<X, Y, 1>(c, dev, stream);
}

}  // namespace

cudaError_t resident_ctas(const void* kernel, uint32_t threads, uint32_t smem, uint32_t* ctas) {
  static std::mutex mu;
  static std::map<std::tuple<int, const void*, uint32_t, uint32_t>, uint32_t> known;
  struct Last {  // what a thread asked for last, by kernel
    const void* kernel;
    int dev;
    uint32_t threads, smem, ctas;
  };
  static thread_local Last last[16] = {};
  int dev = 0, n = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  Last& l = last[(reinterpret_cast<uintptr_t>(kernel) >> 4) % 16];
  if (l.kernel == kernel && l.dev == dev && l.threads == threads && l.smem == smem) {
    *ctas = l.ctas;
    return cudaSuccess;
  }
  std::lock_guard<std::mutex> lk(mu);
  const auto key = std::make_tuple(dev, kernel, threads, smem);
  const auto it = known.find(key);
  if (it != known.end()) {
    *ctas = it->second;
    l = {kernel, dev, threads, smem, it->second};
    return cudaSuccess;
  }
  // (an opt-in stays: the largest asked for, whatever order sizes come in)
  err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  if (err == cudaSuccess) err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem);
  if (err != cudaSuccess) return err;
  if (n < 1) return cudaErrorLaunchOutOfResources;
  known.emplace(key, static_cast<uint32_t>(n));
  *ctas = static_cast<uint32_t>(n);
  return cudaSuccess;
}

cudaError_t launch_layer_norm(const NormCall& c, const DeviceInfo& dev, cudaStream_t stream) {
  count_launch();
  if (c.x_bf16)
    return c.y_bf16 ? launch_typed<bf16_t, bf16_t>(c, dev, stream) : launch_typed<bf16_t, float>(c, dev, stream);
  return c.y_bf16 ? launch_typed<float, bf16_t>(c, dev, stream) : launch_typed<float, float>(c, dev, stream);
}

}  // namespace efs
