// norm_grad.cu — layer norm's backward pass. With x' = (x - mean) rstd and
// q = dy w,
//
//   dx = rstd (q - sum q / d - x' sum(q x') / d),
//   dw = sum over rows of dy x',   db = sum over rows of dy.
//
// What bounds it: reading x and dy and writing dx once. One to eight warps (rows of up to
// 8192 values) take rows a stride apart, the next ones on their way into a ring in
// shared memory, and keep their columns' shares of dw and db in registers (in shared
// memory for longer rows); the CTAs' shares are joined by a second kernel in the order
// of the CTAs, so equal inputs give equal bits.
#include <algorithm>

#include "norm.cuh"

namespace efs {
namespace {

constexpr uint32_t kJoinColumns = 32, kJoinRows = 16;
// Rows that a group has in its ring, with E values of a row a thread.
template <int E>
constexpr int kRing = E == 8 ? 6 : 3;

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

// Rows of at most K V times the threads of a group.
template <typename X, typename Y, int V, int K, bool ALL>
__global__ void __launch_bounds__(ALL || V * K < 16 ? kNormThreads : 2 * kNormThreads, ALL && V * K == 16 ? 2 : 1)
    norm_grad_kernel(const NormGradCall a) {
  constexpr int S = kRing<V * K>;
  extern __shared__ __align__(16) char ring[];
  __shared__ __align__(16) float room[32];
  const RowGroup<ALL> of(a.warps);
  const uint32_t group = of.threads(), t = of.t;
  const uint32_t per_cta = ALL ? 1u : blockDim.x / group, groups = gridDim.x * per_cta;
  const uint32_t first = blockIdx.x * per_cta + of.index;
  const uint32_t x_place = row_place(a.d, sizeof(X)), place = x_place + row_place(a.d, sizeof(Y));
  char* rows = ring + of.index * S * place;
  auto x_row = [&](uint32_t row) { return static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx; };
  auto dy_row = [&](uint32_t row) { return static_cast<const Y*>(a.dy) + static_cast<uint64_t>(row) * a.lddy; };
  auto fetch = [&](uint32_t row, uint32_t slot) {
    if (row < a.n) {
      fetch_row(rows + slot * place, x_row(row), a.d * sizeof(X), t, group);
      fetch_row(rows + slot * place + x_place, dy_row(row), a.d * sizeof(Y), t, group);
    }
    fetch_commit();
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s) fetch(first + s * groups, s);
  float mean = 0.0f, rstd = 0.0f;
  if (first < a.n) mean = __ldg(a.mean + first), rstd = __ldg(a.rstd + first);
  float w[K][V], dw[K][V] = {}, db[K][V] = {};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t c = (k * group + t) * V;
    if (c < a.d) load_weights<V>(a.w, a.w_bf16, a.w_wide, c, 1.0f, w[k]);
  }
  const float inv = 1.0f / static_cast<float>(a.d);
  uint32_t slot = 0;
  for (uint32_t row = first; row < a.n; row += groups) {
    fetch_wait<S - 2>();
    of.sync();
    // (all threads are done with the row before: its place is free)
    fetch(row + (S - 1) * groups, slot == 0 ? S - 1 : slot - 1);
    const float mu = mean, r = rstd;
    if (row + groups < a.n) mean = __ldg(a.mean + row + groups), rstd = __ldg(a.rstd + row + groups);
    const char* xs = rows + slot * place + row_lead(x_row(row));
    const char* dys = rows + slot * place + x_place + row_lead(dy_row(row));
    slot = slot == S - 1 ? 0 : slot + 1;
    float hat[K][V], q[K][V], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * group + t) * V;
      if (c < a.d) {
        const Vec<X, V> x = staged<X, V>(xs, c);
        const Vec<Y, V> dy = staged<Y, V>(dys, c);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float g = dy.get(j);
          hat[k][j] = (x.get(j) - mu) * r;
          q[k][j] = g * w[k][j];
          s1 += q[k][j];
          s2 = fmaf(q[k][j], hat[k][j], s2);
          dw[k][j] = fmaf(g, hat[k][j], dw[k][j]);
          db[k][j] += g;
        }
      }
    }
    if (!a.dx) continue;
    const float2 s = group_sum2(of, s1, s2, room);
    const float m1 = s.x * inv, m2 = s.y * inv;
    X* dx = static_cast<X*>(a.dx) + static_cast<uint64_t>(row) * a.lddx;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c = (k * group + t) * V;
      if (c < a.d) {
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = r * fmaf(-m2, hat[k][j], q[k][j] - m1);
        Vec<X, V> o;
        o.round(out);
        o.store(dx + c);
      }
    }
  }
  griddep_launch_dependents();  // (the join, which waits for this kernel's end)
  if (!a.dw && !a.db) return;
  if (per_cta == 1) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const uint32_t c = (k * group + t) * V + j;
        if (c < a.d) write_share(a, blockIdx.x, gridDim.x, c, dw[k][j], db[k][j]);
      }
    return;
  }
  // the groups' shares, summed in their order (in the ring's place, which is larger)
  fetch_wait<0>();
  float* shares = reinterpret_cast<float*>(ring);  // [2][per_cta][d]
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint32_t c = (k * group + t) * V + j;
      if (c < a.d) {
        shares[of.index * a.d + c] = dw[k][j];
        shares[(per_cta + of.index) * a.d + c] = db[k][j];
      }
    }
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    float w_sum = 0.0f, b_sum = 0.0f;
    for (uint32_t q = 0; q < per_cta; ++q) {
      w_sum += shares[q * a.d + c];
      b_sum += shares[(per_cta + q) * a.d + c];
    }
    write_share(a, blockIdx.x, gridDim.x, c, w_sum, b_sum);
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

// The sum of the CTAs' shares: 32 columns of dw or db per CTA, 16 warps each
// taking every 16th share.
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

// A call's kernel, its CTAs, and how many shares of dw and db they leave.
struct Plan {
  const void* kernel;
  uint32_t v, warps, ctas, threads, smem, parts;
};

template <typename X, typename Y, int V, int K, bool ALL>
cudaError_t plan_rows(const NormGradCall& c, const DeviceInfo& dev, Plan& p) {
  p.kernel = reinterpret_cast<const void*>(norm_grad_kernel<X, Y, V, K, ALL>);
  p.warps = row_warps(c.d, V * K);
  p.threads = ALL ? p.warps * 32 : kNormThreads;
  const uint32_t per_cta = p.threads / (p.warps * 32);
  p.smem = per_cta * kRing<V * K> * (row_place(c.d, sizeof(X)) + row_place(c.d, sizeof(Y)));
  uint32_t per_sm = 0;
  const cudaError_t err = resident_ctas(p.kernel, p.threads, p.smem, &per_sm);
  p.parts = p.ctas = std::min((c.n + per_cta - 1) / per_cta, per_sm * static_cast<uint32_t>(dev.sm_count));
  return err;
}
template <typename X, typename Y, int V>
cudaError_t plan_width(const NormGradCall& c, const DeviceInfo& dev, Plan& p) {
  if (c.d <= 256) return plan_rows<X, Y, V, 8 / V, false>(c, dev, p);
  if (c.d <= 2048) return plan_rows<X, Y, V, 16 / V, false>(c, dev, p);
  if (c.d <= 4096) return plan_rows<X, Y, V, 16 / V, true>(c, dev, p);
  return plan_rows<X, Y, V, 32 / V, true>(c, dev, p);
}
template <typename X, typename Y>
cudaError_t plan_typed(const NormGradCall& c, const DeviceInfo& dev, Plan& p) {
  constexpr uint32_t kWide = sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
  const bool many = c.n > 1;
  auto allow = [&](uint32_t v) {
    return c.d % v == 0 && rows_allow(c.x, many ? c.ldx : 0, sizeof(X), v) &&
           rows_allow(c.dy, many ? c.lddy : 0, sizeof(Y), v) &&
           rows_allow(c.dx, many && c.dx ? c.lddx : 0, sizeof(X), v);
  };
  p.v = allow(kWide) ? kWide : allow(2) ? 2 : 1;
  if (p.v == kWide) return plan_width<X, Y, kWide>(c, dev, p);
  return p.v == 2 ? plan_width<X, Y, 2>(c, dev, p) : plan_width<X, Y, 1>(c, dev, p);
}
cudaError_t plan_of(const NormGradCall& c, const DeviceInfo& dev, Plan& p) {
  p = {};
  if (c.n == 0) return cudaSuccess;
  if (c.d <= kNormRowWidth) {
    if (c.x_bf16) return c.y_bf16 ? plan_typed<bf16_t, bf16_t>(c, dev, p) : plan_typed<bf16_t, float>(c, dev, p);
    return c.y_bf16 ? plan_typed<float, bf16_t>(c, dev, p) : plan_typed<float, float>(c, dev, p);
  }
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count), wide = (c.d + 1023) / 1024;
  p.parts = p.ctas = std::min(c.n, sms);
  if (c.d > kSharesWidth) p.parts = std::min((c.n + 15) / 16, (8 * sms + wide - 1) / wide);
  return cudaSuccess;
}

template <typename X, typename Y>
cudaError_t launch_long(const NormGradCall& c, const Plan& p, cudaStream_t stream) {
  cudaError_t err = cudaSuccess;
  const bool shares = c.dw || c.db;
  if (shares && c.d <= kSharesWidth) {
    err = cudaFuncSetAttribute(norm_grad_long_kernel<X, Y, true>,
                               cudaFuncAttributeMaxDynamicSharedMemorySize, kSharesWidth * 8);
    if (err != cudaSuccess) return err;
    count_launch();
    norm_grad_long_kernel<X, Y, true><<<p.ctas, 1024, c.d * 8, stream>>>(c);
    return cudaGetLastError();
  }
  if (c.dx) {
    count_launch();
    norm_grad_long_kernel<X, Y, false><<<p.ctas, 1024, 0, stream>>>(c);
    if ((err = cudaGetLastError()) != cudaSuccess) return err;
  }
  if (shares) {
    count_launch();
    norm_grad_columns_kernel<X, Y>
        <<<dim3((c.d + 1023) / 1024, p.parts), 256, 0, stream>>>(c, p.parts);
    err = cudaGetLastError();
  }
  return err;
}

}  // namespace

cudaError_t norm_grad_scratch(const NormGradCall& c, const DeviceInfo& dev, size_t* bytes) {
  Plan p;
  const cudaError_t err = plan_of(c, dev, p);
  *bytes = (c.dw || c.db) && p.parts > 1 ? static_cast<size_t>(p.parts) * 2 * c.d * sizeof(float) : 0;
  return err;
}

cudaError_t launch_layer_norm_grad(NormGradCall c, Workspace* ws, cudaStream_t stream,
                                   const DeviceInfo& dev) {
  Plan p;
  cudaError_t err = plan_of(c, dev, p);
  if (err != cudaSuccess) return err;
  c.shares = ws ? reinterpret_cast<float*>(ws->model_scratch()) : nullptr;
  if (c.n == 0) {
  } else if (p.kernel) {
    c.warps = p.warps;
    c.w_wide = rows_allow(c.w, 0, c.w_bf16 ? 2 : 4, c.w_bf16 ? p.v : std::min(p.v, 4u));
    void* params[] = {&c};
    count_launch();
    err = cudaLaunchKernel(p.kernel, dim3(p.ctas), dim3(p.threads), params, p.smem, stream);
  } else if (c.x_bf16) {
    err = c.y_bf16 ? launch_long<bf16_t, bf16_t>(c, p, stream) : launch_long<bf16_t, float>(c, p, stream);
  } else {
    err = c.y_bf16 ? launch_long<float, bf16_t>(c, p, stream) : launch_long<float, float>(c, p, stream);
  }
  if (err != cudaSuccess || (!c.dw && !c.db) || p.parts == 1) return err;
  count_launch();
  void* params[] = {&c, &p.parts};
  return launch_pdl(reinterpret_cast<const void*>(norm_join_kernel),
                    dim3((2 * c.d + kJoinColumns - 1) / kJoinColumns), kJoinColumns * kJoinRows, 0,
                    stream, params, false);
}

}  // namespace efs
