// embed.cu — rows of an embedding table by token: out_i = scale table[t_i], a row
// of zeros for padding (a negative token).
//
// What bounds it: writing out, and reading each different row once from memory
// (the others come out of L2). A warp takes a slice of a row, four vectors a lane, all
// loads before the first store (65,536 rows of 1024 bf16 values: 27.5 us, 89 % of the
// floor); with few rows the slices are short, so that the latency of one load after
// the token's is all there is. Rows of at most 32 vectors, which would leave lanes idle,
// go vector by vector over the threads (1,000,000 rows of 64 bf16 values: 144 us by slices, 32;
// fp32 139 and 62). Vectors need the width, too, to be whole ones: odd widths go value by value.
#include "internal.h"
#include "vec_io.cuh"

namespace efs {
namespace {

constexpr uint32_t kEmbedThreads = 256;

// How many times a row of `width` vectors goes into x, for x width < 2^32: `magic` is
// 2^32 / width, rounded up.
struct Rows {
  uint32_t width, magic;
  __device__ __forceinline__ uint32_t in(uint32_t x) const { return width == 1 ? x : __umulhi(x, magic); }
};

template <typename T, typename O, int V, int K>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedCall a, uint32_t slices, uint32_t* error) {
  const uint64_t item = static_cast<uint64_t>(blockIdx.x) * (kEmbedThreads / 32) + (threadIdx.x >> 5);
  const uint64_t row = item / slices;
  if (row >= a.n) return;
  const uint32_t lane = threadIdx.x & 31u, slice = static_cast<uint32_t>(item - row * slices);
  const int64_t token = __ldg(reinterpret_cast<const long long*>(a.token) + row);
  const bool in = token >= 0 && token < static_cast<int64_t>(a.v);
  if (token >= static_cast<int64_t>(a.v) && lane == 0) atomicOr(error, kDevErrBadInput);
  const T* from = static_cast<const T*>(a.table) + (in ? static_cast<uint64_t>(token) : 0ull) * a.ld_table;
  O* to = static_cast<O*>(a.out) + row * a.ld_out;
  Vec<T, V> x[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t c = ((slice * K + k) * 32 + lane) * V;
    if (in && c < a.d) x[k].load(from + c);
    else x[k].clear();
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t c = ((slice * K + k) * 32 + lane) * V;
    if (c < a.d) {
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = in ? x[k].get(j) * a.scale : 0.0f;
      Vec<O, V> o;
      o.round(f);
      o.store(to + c);
    }
  }
}

template <typename T, typename O, int V, int K>
__global__ void __launch_bounds__(kEmbedThreads) embed_short_kernel(const EmbedCall a, const Rows rows, uint32_t* error) {
  const uint64_t begin = static_cast<uint64_t>(blockIdx.x) * (kEmbedThreads * K);
  const uint64_t row0 = begin >> 32 ? begin / rows.width : static_cast<uint32_t>(begin) / rows.width;
  const uint32_t left = static_cast<uint32_t>(begin - row0 * rows.width);
  uint32_t c[K];
  int64_t token[K];
  uint64_t row[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t x = left + k * kEmbedThreads + threadIdx.x, down = rows.in(x);
    row[k] = row0 + down;
    c[k] = (x - down * rows.width) * V;
    token[k] = row[k] < a.n ? __ldg(reinterpret_cast<const long long*>(a.token) + row[k]) : -1;
  }
  Vec<T, V> v[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k].clear();
    if (token[k] >= 0 && token[k] < static_cast<int64_t>(a.v))
      v[k].load(static_cast<const T*>(a.table) + static_cast<uint64_t>(token[k]) * a.ld_table + c[k]);
    else if (token[k] >= static_cast<int64_t>(a.v) && c[k] == 0)
      atomicOr(error, kDevErrBadInput);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (row[k] >= a.n) continue;
    const bool in = token[k] >= 0 && token[k] < static_cast<int64_t>(a.v);
    float f[V];
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = in ? v[k].get(j) * a.scale : 0.0f;
    Vec<O, V> o;
    o.round(f);
    o.store(static_cast<O*>(a.out) + row[k] * a.ld_out + c[k]);
  }
}

template <typename T, typename O, int V>
cudaError_t launch(const EmbedCall& c, uint32_t* error, uint32_t sms, cudaStream_t stream) {
  const uint32_t width = c.d / V, one = (width + 31) / 32;  // vectors of a row; of a lane
  const bool few_vectors = width <= 32;
  // four vectors a lane where that leaves the GPU's warps busy
  const bool many = static_cast<uint64_t>(c.n) * (few_vectors ? width : 32 * one) >= 8192ull * sms;
  const uint32_t slices = many ? (one + 3) / 4 : one;
  const uint64_t items = few_vectors ? static_cast<uint64_t>(c.n) * width : static_cast<uint64_t>(c.n) * slices;
  const uint64_t per = few_vectors ? kEmbedThreads * (many ? 4 : 1) : kEmbedThreads / 32;
  const uint64_t ctas = (items + per - 1) / per;
  if (ctas > 0x7fffffffull) return cudaErrorInvalidValue;
  const uint32_t grid = static_cast<uint32_t>(ctas);
  count_launch();
  if (few_vectors) {
    const Rows rows = {width, width > 1 ? static_cast<uint32_t>(((1ull << 32) + width - 1) / width) : 0u};
    if (many) embed_short_kernel<T, O, V, 4><<<grid, kEmbedThreads, 0, stream>>>(c, rows, error);
    else embed_short_kernel<T, O, V, 1><<<grid, kEmbedThreads, 0, stream>>>(c, rows, error);
  } else if (many) {
    embed_kernel<T, O, V, 4><<<grid, kEmbedThreads, 0, stream>>>(c, slices, error);
  } else {
    embed_kernel<T, O, V, 1><<<grid, kEmbedThreads, 0, stream>>>(c, slices, error);
  }
  return cudaGetLastError();
}

template <typename T, typename O>
cudaError_t launch_typed(const EmbedCall& c, uint32_t* error, uint32_t sms, cudaStream_t stream) {
  constexpr uint32_t kWide = sizeof(T) == 2 && sizeof(O) == 2 ? 8 : 4;
  auto allow = [&](uint32_t v) {
    auto rows = [&](const void* p, uint64_t ld, uint64_t size) {
      return (reinterpret_cast<uintptr_t>(p) | ld * size) % (size * v) == 0;
    };
    return c.d % v == 0 && rows(c.table, c.v > 1 ? c.ld_table : 0, sizeof(T)) &&
           rows(c.out, c.n > 1 ? c.ld_out : 0, sizeof(O));
  };
  if (allow(kWide)) return launch<T, O, kWide>(c, error, sms, stream);
  return allow(2) ? launch<T, O, 2>(c, error, sms, stream) : launch<T, O, 1>(c, error, sms, stream);
}

}  // namespace

cudaError_t launch_embed(const EmbedCall& c, Workspace& ws, const DeviceInfo& dev) {
  uint32_t* error = ws.u32(kOffError);
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count);
  if (c.table_bf16)
    return c.out_bf16 ? launch_typed<bf16_t, bf16_t>(c, error, sms, ws.stream)
                      : launch_typed<bf16_t, float>(c, error, sms, ws.stream);
  return c.out_bf16 ? launch_typed<float, bf16_t>(c, error, sms, ws.stream)
                    : launch_typed<float, float>(c, error, sms, ws.stream);
}

}  // namespace efs
