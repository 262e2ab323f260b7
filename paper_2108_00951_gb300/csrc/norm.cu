// norm.cu — layer norm's forward pass: y = (x - mean) rstd w + b over rows of d
// values, mean = sum x / d, rstd = (sum (x - mean)^2 / d + eps)^(-1/2).
//
// Both sums are fp32 over values that stay in registers, the second after the
// mean is known (a difference of squares would lose the variance of rows whose
// mean is large). What bounds it: reading x and writing y once. A row of at most
// 1024 values lies in a warp (no barrier), one of at most 8192 in a CTA's
// registers; a longer one is read three times, twice out of L1 and L2.
#include "norm.cuh"

namespace efs {
namespace {

template <typename X, typename Y, int V, int K, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : kNormMaxThreads)
    norm_kernel(const NormCall a) {
  __shared__ float room[2][32];
  const uint32_t group = WARP ? 32u : blockDim.x;
  const uint32_t t = WARP ? threadIdx.x & 31u : threadIdx.x;
  const uint32_t row = WARP ? blockIdx.x * 4u + (threadIdx.x >> 5) : blockIdx.x;
  if (row >= a.n) return;
  const X* x = static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx;
  Y* y = static_cast<Y*>(a.y) + static_cast<uint64_t>(row) * a.ldy;
  Vec<X, V> in[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t c = (k * group + t) * V;
    if (c < a.d) in[k].load(x + c);
    else in[k].clear();
  }
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) sum += in[k].get(j);
  const float inv = 1.0f / static_cast<float>(a.d);
  const float mean = (WARP ? warp_sum(sum) : cta_sum(sum, room[0])) * inv;
  sum = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if ((k * group + t) * V < a.d)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float off = in[k].get(j) - mean;
        sum = fmaf(off, off, sum);
      }
  }
  const float var = (WARP ? warp_sum(sum) : cta_sum(sum, room[1])) * inv;
  const float rstd = 1.0f / sqrtf(var + a.eps);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t c = (k * group + t) * V;
    if (c >= a.d) break;
    float w[V], b[V], out[V];
    load_weights<V>(a.w, a.w_bf16, a.w_wide, c, 1.0f, w);
    load_weights<V>(a.b, a.w_bf16, a.b_wide, c, 0.0f, b);
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = fmaf((in[k].get(j) - mean) * rstd, w[j], b[j]);
    Vec<Y, V> o;
    o.round(out);
    o.store(y + c);
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// Rows of any length, a CTA each.
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormCall a) {
  __shared__ float room[2][32];
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
  const float rstd = 1.0f / sqrtf(cta_sum(sum, room[1]) * inv + a.eps);
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

template <typename X, typename Y, int V>
cudaError_t launch(const NormCall& c, cudaStream_t stream) {
  const uint32_t rows4 = (c.n + 3) / 4;
  if (c.d <= 256) {
    norm_kernel<X, Y, V, 8 / V, true><<<rows4, 128, 0, stream>>>(c);
  } else if (c.d <= 512) {
    norm_kernel<X, Y, V, 16 / V, true><<<rows4, 128, 0, stream>>>(c);
  } else if (c.d <= 1024) {
    norm_kernel<X, Y, V, 32 / V, true><<<rows4, 128, 0, stream>>>(c);
  } else {
    const uint32_t threads = ((c.d + 15) / 16 + 31) / 32 * 32;
    norm_kernel<X, Y, V, 16 / V, false><<<c.n, threads, 0, stream>>>(c);
  }
  return cudaGetLastError();
}

template <typename X, typename Y>
cudaError_t launch_typed(NormCall c, cudaStream_t stream) {
  if (c.d > 16 * kNormMaxThreads) {
    norm_long_kernel<X, Y><<<c.n, 1024, 0, stream>>>(c);
    return cudaGetLastError();
  }
  constexpr uint32_t kWide = sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
  auto allow = [&](uint32_t v) {
    return c.d % v == 0 && rows_allow(reinterpret_cast<uintptr_t>(c.x), c.n > 1 ? c.ldx : 0, sizeof(X), v) &&
           rows_allow(reinterpret_cast<uintptr_t>(c.y), c.n > 1 ? c.ldy : 0, sizeof(Y), v);
  };
  const uint32_t v = allow(kWide) ? kWide : allow(2) ? 2 : 1;
  const uint64_t wsize = c.w_bf16 ? 2 : 4, part = c.w_bf16 ? v : (v > 4 ? 4 : v);
  c.w_wide = rows_allow(reinterpret_cast<uintptr_t>(c.w), 0, wsize, part);
  c.b_wide = rows_allow(reinterpret_cast<uintptr_t>(c.b), 0, wsize, part);
  if (v == kWide) return launch<X, Y, kWide>(c, stream);
  return v == 2 ? launch<X, Y, 2>(c, stream) : launch<X, Y, 1>(c, stream);
}

}  // namespace

cudaError_t launch_layer_norm(const NormCall& c, cudaStream_t stream) {
  count_launch();
  if (c.x_bf16)
    return c.y_bf16 ? launch_typed<bf16_t, bf16_t>(c, stream) : launch_typed<bf16_t, float>(c, stream);
  return c.y_bf16 ? launch_typed<float, bf16_t>(c, stream) : launch_typed<float, float>(c, stream);
}

}  // namespace efs
