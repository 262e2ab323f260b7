// embed.cu — rows of an embedding table by token: out_i = scale table[t_i], a row
// of zeros for padding (a negative token).
//
// What bounds it: writing out, and reading each different row once from memory
// (the others come out of L2). A warp takes a slice of a row, its loads issued
// together; with few rows the slices are short, so that the latency of one load
// after the token's is all there is.
#include "internal.h"
#include "vec_io.cuh"

namespace efs {
namespace {

constexpr int kEmbedWarps = 8;

template <typename T, typename O, int V, int K>
__global__ void __launch_bounds__(32 * kEmbedWarps) embed_kernel(const EmbedCall a, uint32_t slices, uint32_t* error) {
  const uint64_t item = static_cast<uint64_t>(blockIdx.x) * kEmbedWarps + (threadIdx.x >> 5);
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

template <typename T, typename O, int V>
cudaError_t launch(const EmbedCall& c, uint32_t* error, uint32_t sms, cudaStream_t stream) {
  // vectors of a row a lane takes: four where that leaves the GPU's warps busy
  const uint32_t one = (c.d + 32 * V - 1) / (32 * V);
  const bool many = static_cast<uint64_t>(c.n) * one >= 256ull * sms;
  const uint32_t slices = many ? (one + 3) / 4 : one;
  const uint64_t ctas = (static_cast<uint64_t>(c.n) * slices + kEmbedWarps - 1) / kEmbedWarps;
  if (ctas > 0x7fffffffull) return cudaErrorInvalidValue;
  count_launch();
  if (many) embed_kernel<T, O, V, 4><<<static_cast<uint32_t>(ctas), 32 * kEmbedWarps, 0, stream>>>(c, slices, error);
  else embed_kernel<T, O, V, 1><<<static_cast<uint32_t>(ctas), 32 * kEmbedWarps, 0, stream>>>(c, slices, error);
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
