// norm_grad.cu — layer norm's backward pass. With x' = (x - mean) rstd and
// q = dy w,
//
//   dx = rstd (q - sum q / d - x' sum(q x') / d),
//   dw = sum over rows of dy x',   db = sum over rows of dy.
//
// What bounds it: reading x and dy and writing dx once. A warp (rows of at most
// 1024 values) or a CTA takes rows a stride apart and keeps its columns' shares
// of dw and db in registers, or in shared memory for long rows; the CTAs' shares
// are joined by a second kernel in the order of the CTAs, so equal inputs give
// equal bits.
#include <algorithm>

#include "norm.cuh"

namespace efs {
namespace {

constexpr int kWarpsPerCta = 8;
constexpr uint32_t kJoinColumns = 32, kJoinRows = 8;

// A share of columns c of dw and db; the only one is the result.
__device__ __forceinline__ void write_share(const NormGradCall& a, uint32_t share, uint32_t parts,
                                            uint32_t c, float dw, float db) {
  if (parts > 1) {
    float* to = a.shares + static_cast<uint64_t>(share) * 2 * a.d + c;
    to[0] = dw;
    to[a.d] = db;
    return;
  }
  if (a.dw) {
    if (a.w_bf16) store_rounded(static_cast<bf16_t*>(a.dw) + c, dw);
    else static_cast<float*>(a.dw)[c] = dw;
  }
  if (a.db) {
    if (a.w_bf16) store_rounded(static_cast<bf16_t*>(a.db) + c, db);
    else static_cast<float*>(a.db)[c] = db;
  }
}

// Rows of at most 32 V K values, a warp each.
template <typename X, typename Y, int V, int K>
__global__ void __launch_bounds__(32 * kWarpsPerCta) norm_grad_warp_kernel(const NormGradCall a) {
  extern __shared__ float shares[];  // [kWarpsPerCta][d]
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const float inv = 1.0f / static_cast<float>(a.d);
  float dw[K][V] = {}, db[K][V] = {};
  for (uint32_t row = blockIdx.x * kWarpsPerCta + warp; row < a.n; row += gridDim.x * kWarpsPerCta) {
    const X* x = static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx;
    const Y* dy = static_cast<const Y*>(a.dy) + static_cast<uint64_t>(row) * a.lddy;
    Vec<X, V> xs[K];
    Vec<Y, V> dys[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * 32 + lane) * V;
      if (c < a.d) {
        xs[k].load(x + c);
        dys[k].load(dy + c);
      } else {
        xs[k].clear();
        dys[k].clear();
      }
    }
    const float mean = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * 32 + lane) * V;
      if (c < a.d) {
        float w[V];
        load_weights<V>(a.w, a.w_bf16, a.w_wide, c, 1.0f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float hat = (xs[k].get(j) - mean) * rstd, g = dys[k].get(j), q = g * w[j];
          s1 += q;
          s2 = fmaf(q, hat, s2);
          dw[k][j] = fmaf(g, hat, dw[k][j]);
          db[k][j] += g;
        }
      }
    }
    if (!a.dx) continue;
    s1 = warp_sum(s1) * inv;
    s2 = warp_sum(s2) * inv;
    X* dx = static_cast<X*>(a.dx) + static_cast<uint64_t>(row) * a.lddx;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * 32 + lane) * V;
      if (c < a.d) {
        float w[V], out[V];
        load_weights<V>(a.w, a.w_bf16, a.w_wide, c, 1.0f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float hat = (xs[k].get(j) - mean) * rstd;
          out[j] = rstd * (fmaf(dys[k].get(j), w[j], -s1) - hat * s2);
        }
        Vec<X, V> o;
        o.round(out);
        o.store(dx + c);
      }
    }
  }
  if (!a.dw && !a.db) return;
  // the warps' shares, summed in their order
  float sums[K * V * 32 / (32 * kWarpsPerCta)];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const uint32_t c = (k * 32 + lane) * V + j;
        if (c < a.d) shares[warp * a.d + c] = which ? db[k][j] : dw[k][j];
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K * V / kWarpsPerCta; ++i) {
      const uint32_t c = i * 32 * kWarpsPerCta + threadIdx.x;
      if (c < a.d) {
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < kWarpsPerCta; ++r) s += shares[r * a.d + c];
        if (which) write_share(a, blockIdx.x, gridDim.x, c, sums[i], s);
        else sums[i] = s;
      }
    }
  }
}

// Rows of at most V K times the threads, a CTA each; the next row is loaded
// before this one's sums are joined.
template <typename X, typename Y, int V, int K>
__global__ void __launch_bounds__(kNormMaxThreads) norm_grad_cta_kernel(const NormGradCall a) {
  __shared__ float room[2][64];
  const float inv = 1.0f / static_cast<float>(a.d);
  const uint32_t threads = blockDim.x, t = threadIdx.x;
  float dw[K][V] = {}, db[K][V] = {};
  Vec<X, V> xs[K];
  Vec<Y, V> dys[K];
  float mean = 0.0f, rstd = 0.0f;
  auto load = [&](uint32_t row) {
    const X* x = static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx;
    const Y* dy = static_cast<const Y*>(a.dy) + static_cast<uint64_t>(row) * a.lddy;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * threads + t) * V;
      if (c < a.d) {
        xs[k].load(x + c);
        dys[k].load(dy + c);
      } else {
        xs[k].clear();
        dys[k].clear();
      }
    }
    mean = __ldg(a.mean + row);
    rstd = __ldg(a.rstd + row);
  };
  uint32_t parity = 0;
  if (blockIdx.x < a.n) load(blockIdx.x);
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x, parity ^= 1u) {
    float hat[K][V], q[K][V], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * threads + t) * V;
      float w[V];
      if (c < a.d) {
        load_weights<V>(a.w, a.w_bf16, a.w_wide, c, 1.0f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float g = dys[k].get(j);
          hat[k][j] = (xs[k].get(j) - mean) * rstd;
          q[k][j] = g * w[j];
          s1 += q[k][j];
          s2 = fmaf(q[k][j], hat[k][j], s2);
          dw[k][j] = fmaf(g, hat[k][j], dw[k][j]);
          db[k][j] += g;
        }
      }
    }
    const float scale = rstd;
    if (row + gridDim.x < a.n) load(row + gridDim.x);
    if (!a.dx) continue;
    const float2 s = cta_sum2(s1, s2, room[parity]);
    X* dx = static_cast<X*>(a.dx) + static_cast<uint64_t>(row) * a.lddx;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * threads + t) * V;
      if (c < a.d) {
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = scale * (q[k][j] - s.x * inv - hat[k][j] * (s.y * inv));
        Vec<X, V> o;
        o.round(out);
        o.store(dx + c);
      }
    }
  }
  if (!a.dw && !a.db) return;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint32_t c = (k * threads + t) * V + j;
      if (c < a.d) write_share(a, blockIdx.x, gridDim.x, c, dw[k][j], db[k][j]);
    }
}

// Rows of any length, a CTA each, read twice (the second time out of L2). SHARES:
// the columns' shares of dw and db lie in shared memory, each the business of
// one thread.
template <typename X, typename Y, bool SHARES>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(const NormGradCall a) {
  extern __shared__ float shares[];  // [2][d]
  __shared__ float room[2][64];
  const float inv = 1.0f / static_cast<float>(a.d);
  if (SHARES)
    for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) shares[c] = shares[a.d + c] = 0.0f;
  uint32_t parity = 0;
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x, parity ^= 1u) {
    const X* x = static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx;
    const Y* dy = static_cast<const Y*>(a.dy) + static_cast<uint64_t>(row) * a.lddy;
    const float mean = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      float w[1];
      load_weights<1>(a.w, a.w_bf16, true, c, 1.0f, w);
      const float hat = (widen(__ldg(x + c)) - mean) * rstd, g = widen(__ldg(dy + c));
      s1 = fmaf(g, w[0], s1);
      s2 = fmaf(g * w[0], hat, s2);
      if (SHARES) {
        shares[c] = fmaf(g, hat, shares[c]);
        shares[a.d + c] += g;
      }
    }
    if (!a.dx) continue;
    const float2 s = cta_sum2(s1, s2, room[parity]);
    X* dx = static_cast<X*>(a.dx) + static_cast<uint64_t>(row) * a.lddx;
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      float w[1];
      load_weights<1>(a.w, a.w_bf16, true, c, 1.0f, w);
      const float hat = (widen(__ldg(x + c)) - mean) * rstd;
      store_rounded(dx + c, rstd * (widen(__ldg(dy + c)) * w[0] - s.x * inv - hat * (s.y * inv)));
    }
  }
  if (SHARES)
    for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x)
      write_share(a, blockIdx.x, gridDim.x, c, shares[c], shares[a.d + c]);
}

// dw and db of very long rows: 1024 columns and a part of the rows per CTA.
template <typename X, typename Y>
__global__ void __launch_bounds__(256) norm_grad_columns_kernel(const NormGradCall a, uint32_t parts) {
  const uint32_t part = blockIdx.y;
  const uint32_t per = (a.n + parts - 1) / parts;
  const uint32_t lo = min(part * per, a.n), hi = min(lo + per, a.n);
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = blockIdx.x * 1024 + i * 256 + threadIdx.x;
    if (c >= a.d) return;
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (uint32_t row = lo; row < hi; ++row) {
      const float g = widen(__ldg(static_cast<const Y*>(a.dy) + static_cast<uint64_t>(row) * a.lddy + c));
      const float v = widen(__ldg(static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx + c));
      dw = fmaf(g, (v - __ldg(a.mean + row)) * __ldg(a.rstd + row), dw);
      db += g;
    }
    write_share(a, part, parts, c, dw, db);
  }
}

// The sum of the CTAs' shares: 32 columns of dw or db per CTA, eight warps each
// taking every eighth share.
__global__ void __launch_bounds__(kJoinColumns * kJoinRows) norm_join_kernel(const NormGradCall a, uint32_t parts) {
  __shared__ float sums[kJoinRows][kJoinColumns];
  griddep_wait();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const uint32_t c = blockIdx.x * kJoinColumns + lane;  // of dw, then of db
  float s = 0.0f;
  if (c < 2 * a.d) {
    const float* from = a.shares + c;
#pragma unroll 8
    for (uint32_t p = warp; p < parts; p += kJoinRows) s += from[static_cast<uint64_t>(p) * 2 * a.d];
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= 2 * a.d) return;
  s = 0.0f;
#pragma unroll
  for (uint32_t r = 0; r < kJoinRows; ++r) s += sums[r][lane];
  void* out = c < a.d ? a.dw : a.db;
  const uint32_t at = c < a.d ? c : c - a.d;
  if (!out) return;
  if (a.w_bf16) store_rounded(static_cast<bf16_t*>(out) + at, s);
  else static_cast<float*>(out)[at] = s;
}

constexpr uint32_t kSharesWidth = 28000;  // columns whose shares fit shared memory

// How many CTAs take the rows, and how many shares of dw and db they leave.
struct Grid {
  uint32_t ctas, parts;
};
Grid grid_of(const NormGradCall& c, const DeviceInfo& dev) {
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count);
  if (c.n == 0) return {0, 0};
  if (c.d <= 1024) {
    const uint32_t grid = std::min((c.n + kWarpsPerCta - 1) / kWarpsPerCta, sms * (c.d <= 512 ? 2 : 1));
    return {grid, grid};
  }
  if (c.d <= 16 * kNormMaxThreads) {
    const uint32_t grid = std::min(c.n, sms * (c.d <= 2048 ? 4 : c.d <= 4096 ? 2 : 1));
    return {grid, grid};
  }
  const uint32_t grid = std::min(c.n, sms);
  if (c.d <= kSharesWidth) return {grid, grid};
  const uint32_t wide = (c.d + 1023) / 1024;
  return {grid, std::min((c.n + 15) / 16, (8 * sms + wide - 1) / wide)};
}

template <typename X, typename Y, int V>
cudaError_t launch(const NormGradCall& c, uint32_t grid, cudaStream_t stream) {
  const uint32_t smem = c.d * kWarpsPerCta * 4;
  if (c.d <= 256) {
    norm_grad_warp_kernel<X, Y, V, 8 / V><<<grid, 256, smem, stream>>>(c);
  } else if (c.d <= 512) {
    norm_grad_warp_kernel<X, Y, V, 16 / V><<<grid, 256, smem, stream>>>(c);
  } else if (c.d <= 1024) {
    norm_grad_warp_kernel<X, Y, V, 32 / V><<<grid, 256, smem, stream>>>(c);
  } else if (c.d <= 8 * kNormMaxThreads) {
    norm_grad_cta_kernel<X, Y, V, 8 / V><<<grid, ((c.d + 7) / 8 + 31) / 32 * 32, 0, stream>>>(c);
  } else {
    norm_grad_cta_kernel<X, Y, V, 16 / V><<<grid, ((c.d + 15) / 16 + 31) / 32 * 32, 0, stream>>>(c);
  }
  return cudaGetLastError();
}

template <typename X, typename Y>
cudaError_t launch_long(const NormGradCall& c, const Grid& grid, cudaStream_t stream) {
  cudaError_t err = cudaSuccess;
  const bool shares = c.dw || c.db;
  if (shares && c.d <= kSharesWidth) {
    err = cudaFuncSetAttribute(norm_grad_long_kernel<X, Y, true>,
                               cudaFuncAttributeMaxDynamicSharedMemorySize, kSharesWidth * 8);
    if (err != cudaSuccess) return err;
    count_launch();
    norm_grad_long_kernel<X, Y, true><<<grid.ctas, 1024, c.d * 8, stream>>>(c);
    return cudaGetLastError();
  }
  if (c.dx) {
    count_launch();
    norm_grad_long_kernel<X, Y, false><<<grid.ctas, 1024, 0, stream>>>(c);
    if ((err = cudaGetLastError()) != cudaSuccess) return err;
  }
  if (shares) {
    count_launch();
    norm_grad_columns_kernel<X, Y>
        <<<dim3((c.d + 1023) / 1024, grid.parts), 256, 0, stream>>>(c, grid.parts);
    err = cudaGetLastError();
  }
  return err;
}

template <typename X, typename Y>
cudaError_t launch_typed(NormGradCall c, const Grid& grid, cudaStream_t stream) {
  if (c.n == 0) return cudaSuccess;
  if (c.d > 16 * kNormMaxThreads) return launch_long<X, Y>(c, grid, stream);
  constexpr uint32_t kWide = sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
  const bool many = c.n > 1;
  auto allow = [&](uint32_t v) {
    return c.d % v == 0 &&
           rows_allow(reinterpret_cast<uintptr_t>(c.x), many ? c.ldx : 0, sizeof(X), v) &&
           rows_allow(reinterpret_cast<uintptr_t>(c.dy), many ? c.lddy : 0, sizeof(Y), v) &&
           rows_allow(reinterpret_cast<uintptr_t>(c.dx), many ? c.lddx : 0, sizeof(X), v);
  };
  const uint32_t v = allow(kWide) ? kWide : allow(2) ? 2 : 1;
  c.w_wide = rows_allow(reinterpret_cast<uintptr_t>(c.w), 0, c.w_bf16 ? 2 : 4,
                        c.w_bf16 ? v : (v > 4 ? 4 : v));
  count_launch();
  if (v == kWide) return launch<X, Y, kWide>(c, grid.ctas, stream);
  return v == 2 ? launch<X, Y, 2>(c, grid.ctas, stream) : launch<X, Y, 1>(c, grid.ctas, stream);
}

}  // namespace

size_t norm_grad_scratch(const NormGradCall& c, const DeviceInfo& dev) {
  if (!c.dw && !c.db) return 0;
  const uint32_t parts = grid_of(c, dev).parts;
  return parts > 1 ? static_cast<size_t>(parts) * 2 * c.d * sizeof(float) : 0;
}

cudaError_t launch_layer_norm_grad(NormGradCall c, Workspace* ws, cudaStream_t stream,
                                   const DeviceInfo& dev) {
  Grid grid = grid_of(c, dev);
  c.shares = ws ? reinterpret_cast<float*>(ws->model_scratch()) : nullptr;
  cudaError_t err;
  if (c.x_bf16)
    err = c.y_bf16 ? launch_typed<bf16_t, bf16_t>(c, grid, stream) : launch_typed<bf16_t, float>(c, grid, stream);
  else
    err = c.y_bf16 ? launch_typed<float, bf16_t>(c, grid, stream) : launch_typed<float, float>(c, grid, stream);
  if (err != cudaSuccess || (!c.dw && !c.db) || grid.parts == 1) return err;
  count_launch();
  void* params[] = {&c, &grid.parts};
  return launch_pdl(reinterpret_cast<const void*>(norm_join_kernel),
                    dim3((2 * c.d + kJoinColumns - 1) / kJoinColumns), kJoinColumns * kJoinRows, 0,
                    stream, params, false);
}

}  // namespace efs
