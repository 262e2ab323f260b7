// norm_grad.cu — layer norm's backward pass. With x' = (x - mean) rstd and
// q = dy w,
//
//   dx = rstd (q - sum q / d - x' sum(q x') / d),
//   dw = sum over rows of dy x',   db = sum over rows of dy.
//
// What bounds it: reading x and dy and writing dx once. Rows are spread as in the
// forward pass (norm.cu), the next ones on their way into a ring in shared memory; a
// row's threads keep their columns' shares of dw and db in registers (of rows
// beyond 65,536 values a kernel of its own adds them up), and a second kernel joins
// the CTAs' shares in the order of the CTAs, so equal inputs give equal bits.
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

template <typename X, typename Y, int V, int K, RowKind KIND>
__global__ void __launch_bounds__(kNormThreads, V * K == 16 ? 2 : 1) norm_grad_kernel(const NormGradCall a) {
  constexpr int S = kRing<V * K>;
  extern __shared__ __align__(16) char ring[];
  __shared__ RowRoom room;
  const RowGroup<KIND> g(a.threads);
  const RowPart part = row_part(a.d, a.part, a.cluster);
  const RowColumns<KIND, V> of(g, part.columns);
  const uint32_t per_cta = KIND == kRowAll ? 1u : blockDim.x / g.threads, t = g.t;
  const uint32_t parts = gridDim.x / a.cluster, share = blockIdx.x / a.cluster;
  const uint32_t groups = parts * per_cta, first = share * per_cta + g.index;
  const uint32_t x_place = row_place(a.part, sizeof(X)), place = x_place + row_place(a.part, sizeof(Y));
  char* rows = ring + g.index * S * place;
  auto x_row = [&](uint32_t row) {
    return static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx + part.first;
  };
  auto dy_row = [&](uint32_t row) {
    return static_cast<const Y*>(a.dy) + static_cast<uint64_t>(row) * a.lddy + part.first;
  };
  auto fetch = [&](uint32_t row, uint32_t slot) {
    if (row < a.n) {
      fetch_row(rows + slot * place, x_row(row), part.columns * sizeof(X), t, g.threads);
      fetch_row(rows + slot * place + x_place, dy_row(row), part.columns * sizeof(Y), t, g.threads);
    }
    fetch_commit();
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s) fetch(first + s * groups, s);
  float mean = 0.0f, rstd = 0.0f;
  if (first < a.n) mean = __ldg(a.mean + first), rstd = __ldg(a.rstd + first);
  float w[K][V], dw[K][V] = {}, db[K][V] = {};
  load_weights(a.w, a.w_bf16, a.w_wide, part.first, of.first, of.step(), of.end, 1.0f, w);
  const float inv = 1.0f / static_cast<float>(a.d);
  if (KIND == kRowAll && a.cluster > 1) cluster_sync();  // (the others' shared memory is theirs)
  uint32_t slot = 0, parity = 0;
  // (the lanes of a warp go through its rows together: to the last round of the warp's first)
  const uint32_t ahead = KIND == kRowLanes ? g.index % (32u / g.threads) : 0u;
  for (uint32_t row = first; row - ahead < a.n; row += groups) {
    fetch_wait<S - 2>();
    g.sync();
    // (all threads are done with the row before: its place is free)
    fetch(row + (S - 1) * groups, slot == 0 ? S - 1 : slot - 1);
    const float mu = mean, r = rstd;
    if (row + groups < a.n) mean = __ldg(a.mean + row + groups), rstd = __ldg(a.rstd + row + groups);
    const bool in = KIND != kRowLanes || row < a.n;
    const char* xs = rows + slot * place + (in ? row_lead(x_row(row)) : 0u) + of.first * sizeof(X);
    const char* dys = rows + slot * place + x_place + (in ? row_lead(dy_row(row)) : 0u) + of.first * sizeof(Y);
    slot = slot == S - 1 ? 0 : slot + 1;
    float hat[K][V], q[K][V], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && of.has(k)) {
        const Vec<X, V> x = staged<X, V>(xs, of.off(k));
        const Vec<Y, V> dy = staged<Y, V>(dys, of.off(k));
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float dyj = dy.get(j);
          hat[k][j] = (x.get(j) - mu) * r;
          q[k][j] = dyj * w[k][j];
          s1 += q[k][j];
          s2 = fmaf(q[k][j], hat[k][j], s2);
          dw[k][j] = fmaf(dyj, hat[k][j], dw[k][j]);
          db[k][j] += dyj;
        }
      }
    }
    if (!a.dx) continue;
    const float2 s = row_sum<KIND, true>(g, s1, s2, room, 0, a.cluster, parity);
    const float m1 = s.x * inv, m2 = s.y * inv;
    X* dx = static_cast<X*>(a.dx) + static_cast<uint64_t>(row) * a.lddx + part.first + of.first;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && of.has(k)) {
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = r * fmaf(-m2, hat[k][j], q[k][j] - m1);
        Vec<X, V> o;
        o.round(out);
        o.store(dx + of.off(k));
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
        const uint32_t c = of.first + of.off(k) + j;
        if (of.has(k)) write_share(a, share, parts, part.first + c, dw[k][j], db[k][j]);
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
      const uint32_t c = of.first + of.off(k) + j;
      if (of.has(k)) {
        shares[g.index * a.d + c] = dw[k][j];
        shares[(per_cta + g.index) * a.d + c] = db[k][j];
      }
    }
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    float w_sum = 0.0f, b_sum = 0.0f;
    for (uint32_t q = 0; q < per_cta; ++q) {
      w_sum += shares[q * a.d + c];
      b_sum += shares[(per_cta + q) * a.d + c];
    }
    write_share(a, share, parts, c, w_sum, b_sum);
  }
}

// dx of rows of any length, a CTA each, read twice (the second time out of L2).
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(const NormGradCall a) {
  __shared__ float room[2][64];
  const float inv = 1.0f / static_cast<float>(a.d);
  uint32_t parity = 0;
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x, parity ^= 1u) {
    const X* x = static_cast<const X*>(a.x) + static_cast<uint64_t>(row) * a.ldx;
    const Y* dy = static_cast<const Y*>(a.dy) + static_cast<uint64_t>(row) * a.lddy;
    const float mean = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      const float w = load_weight(a.w, a.w_bf16, c, 1.0f);
      const float hat = (widen(__ldg(x + c)) - mean) * rstd, q = widen(__ldg(dy + c)) * w;
      s1 += q;
      s2 = fmaf(q, hat, s2);
    }
    const float2 s = cta_sum2(s1, s2, room[parity]);
    X* dx = static_cast<X*>(a.dx) + static_cast<uint64_t>(row) * a.lddx;
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      const float w = load_weight(a.w, a.w_bf16, c, 1.0f);
      const float hat = (widen(__ldg(x + c)) - mean) * rstd;
      store_rounded(dx + c, rstd * (widen(__ldg(dy + c)) * w - s.x * inv - hat * (s.y * inv)));
    }
  }
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

// A call's kernel, how its rows are spread, and how many shares of dw and db they leave.
struct Plan {
  RowPlan rows;  // (no kernel: rows that no threads hold)
  uint32_t v, parts;
};

template <typename X, typename Y, int V, int K, RowKind KIND>
cudaError_t plan_rows(const NormGradCall& c, uint32_t most, const DeviceInfo& dev, Plan& p) {
  plan_row(p.rows, reinterpret_cast<const void*>(norm_grad_kernel<X, Y, V, K, KIND>), KIND, V * K, c.d, most);
  const cudaError_t err = plan_groups(
      p.rows, kRing<V * K> * (row_place(p.rows.part, sizeof(X)) + row_place(p.rows.part, sizeof(Y))), c.n, dev);
  p.parts = p.rows.groups;
  return err;
}
template <typename X, typename Y, int V>
cudaError_t plan_width(const NormGradCall& c, const DeviceInfo& dev, Plan& p) {
  if (c.d <= 256) return plan_rows<X, Y, V, 8 / V, kRowLanes>(c, 256, dev, p);
  if (c.d <= 2048) return plan_rows<X, Y, V, 16 / V, kRowWarps>(c, 2048, dev, p);
  // 16 values a thread leave two CTAs an SM (both passes over 20,000 x 2501: 166 us, with 32 220; 20,000 x 3001
  // fp32 230 and 262; wide vectors lose less by 32, or nothing: 32,768 x 4096 250 with either, fp32 460 and
  // 423), but a CTA without a cluster waits less (16,384 x 8192: 264 with 32, 311 with 16 and two CTAs)
  constexpr uint32_t kFew = 16 * kNormThreads, kMany = 32 * kNormThreads;
  if (c.d <= kFew || (c.d > kMany && c.d <= kFew * kNormCluster))
    return plan_rows<X, Y, V, 16 / V, kRowAll>(c, kFew, dev, p);
  return plan_rows<X, Y, V, 32 / V, kRowAll>(c, kMany, dev, p);
}
template <typename X, typename Y>
cudaError_t plan_typed(const NormGradCall& c, const DeviceInfo& dev, Plan& p) {
  constexpr bool kBoth16 = sizeof(X) == 2 && sizeof(Y) == 2;
  const bool many = c.n > 1;
  auto allow = [&](uint32_t v) {
    return c.d % v == 0 && rows_allow(c.x, many ? c.ldx : 0, sizeof(X), v) &&
           rows_allow(c.dy, many ? c.lddy : 0, sizeof(Y), v) &&
           rows_allow(c.dx, many && c.dx ? c.lddx : 0, sizeof(X), v);
  };
  p.v = kBoth16 && allow(8) ? 8 : allow(4) ? 4 : allow(2) ? 2 : 1;
  if constexpr (kBoth16)
    if (p.v == 8) return plan_width<X, Y, 8>(c, dev, p);
  if (p.v == 4) return plan_width<X, Y, 4>(c, dev, p);
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
  p.rows.groups = std::min(c.n, sms);
  p.parts = std::min((c.n + 15) / 16, (8 * sms + wide - 1) / wide);
  return cudaSuccess;
}

template <typename X, typename Y>
cudaError_t launch_long(const NormGradCall& c, const Plan& p, cudaStream_t stream) {
  cudaError_t err = cudaSuccess;
  if (c.dx) {
    count_launch();
    norm_grad_long_kernel<X, Y><<<p.rows.groups, 1024, 0, stream>>>(c);
    if ((err = cudaGetLastError()) != cudaSuccess) return err;
  }
  if (c.dw || c.db) {
    count_launch();
    norm_grad_columns_kernel<X, Y><<<dim3((c.d + 1023) / 1024, p.parts), 256, 0, stream>>>(c, p.parts);
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
  } else if (p.rows.kernel) {
    c.threads = p.rows.threads;
    c.cluster = p.rows.cluster;
    c.part = p.rows.part;
    c.w_wide = rows_allow(c.w, 0, c.w_bf16 ? 2 : 4, c.w_bf16 ? p.v : std::min(p.v, 4u));
    count_launch();
    err = launch_row(p.rows, &c, stream);
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
