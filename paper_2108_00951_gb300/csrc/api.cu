// api.cu — the extern "C" boundary declared in include/efsparse.h: host-side
// argument checks, the per-(device, stream) workspaces, and status reporting.
// Every compute step runs in the kernels of ht.cu, topk.cu, topk_layerwise.cu
// and aggregate.cu, of vocab.cu, vocab_few.cu, ortho.cu and ortho_small.cu, and of
// embed.cu, embed_grad.cu, norm.cu, norm_grad.cu and adamw.cu.
#include <algorithm>
#include <array>
#include <atomic>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <map>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "efsparse.h"
#include "internal.h"

namespace efs {
namespace {

std::mutex g_mu;
std::map<std::pair<int, cudaStream_t>, Workspace*> g_workspaces;
std::map<int, DeviceInfo> g_devices;
std::atomic<uint64_t> g_launches{0};
std::atomic<int64_t> g_withheld_tile{-1};
std::atomic<uint64_t> g_wait_limit_ns{2000000000ull};  // 2 s per wait
std::atomic<int> g_stream_kernel_mode{0};  // 0: by size, 1: chunks, 2: groups, 3: shallow ring

constexpr uint64_t kMaxD = 0xffffffffull;

bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || na == 0 || nb == 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

ef_status device_info(int dev, DeviceInfo* out) {
  std::lock_guard<std::mutex> lk(g_mu);
  auto it = g_devices.find(dev);
  if (it == g_devices.end()) {
    DeviceInfo info;
    if (cudaDeviceGetAttribute(&info.sm_count, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return EF_ERR_CUDA;
    ht_init_device(info);
    topk_init_device(info);
    topk_layerwise_init_device(info);
    aggregate_init_device(info);
    ortho_small_init_device(info);
    if (info.refine_blocks <= 0 || info.finalize_blocks <= 0) return EF_ERR_CUDA;
    it = g_devices.emplace(dev, info).first;
  }
  *out = it->second;
  return EF_OK;
}

// Whether calls on the stream are being captured into a graph. (The legacy
// stream answers with an error while another stream is: it is not itself.)
bool capturing(cudaStream_t stream) {
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(stream, &st) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return st != cudaStreamCaptureStatusNone;
}

// Frees an allocation that growth replaces, or keeps it for the graphs that
// refer to it.
void replace_block(char*& block, bool captured, std::vector<char*>& kept) {
  if (!captured) {
    cudaFree(block);
  } else {
    try {
      kept.push_back(block);
    } catch (const std::bad_alloc&) {  // kept all the same, until the process ends
    }
  }
  block = nullptr;
}

// Find or grow the workspace of (current device, stream). Growth
// synchronises the stream once; the new header and tile-status array start
// at zero.
ef_status acquire_workspace(cudaStream_t stream, uint32_t tiles, uint32_t cand_cap,
                            size_t offsets, size_t stage, Workspace** out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  const bool captured = capturing(stream);
  std::lock_guard<std::mutex> lk(g_mu);
  Workspace*& ws = g_workspaces[std::make_pair(dev, stream)];
  if (!ws) {
    ws = new Workspace;
    ws->device = dev;
    ws->stream = stream;
    // the density hint (no hint when mapped host memory is unavailable)
    void* h = nullptr;
    if (cudaHostAlloc(&h, sizeof(uint32_t), cudaHostAllocMapped) == cudaSuccess) {
      void* dp = nullptr;
      *static_cast<volatile uint32_t*>(h) = 0u;
      if (cudaHostGetDevicePointer(&dp, h, 0) == cudaSuccess) {
        ws->density_host = static_cast<uint32_t*>(h);
        ws->density_dev = static_cast<uint32_t*>(dp);
      } else {
        cudaFreeHost(h);
      }
    }
    cudaGetLastError();
  }
  if (!ws->base || tiles > ws->status_tiles || cand_cap > ws->cand_cap ||
      offsets > ws->offsets_cap || stage > ws->stage_cap) {
    if (ws->base) {
      if (cudaStreamSynchronize(stream) != cudaSuccess) return EF_ERR_CUDA;
      replace_block(ws->base, ws->base_captured, ws->old_bases);
      ws->base_captured = false;
    }
    Workspace grown = *ws;
    if (tiles > grown.status_tiles) grown.status_tiles = tiles;
    if (cand_cap > grown.cand_cap) grown.cand_cap = cand_cap;
    if (offsets > grown.offsets_cap) grown.offsets_cap = offsets;
    if (stage > grown.stage_cap) grown.stage_cap = stage;
    const size_t bytes = grown.total_bytes();
    void* p = nullptr;
    if (cudaMalloc(&p, bytes) != cudaSuccess) {
      cudaGetLastError();
      ws->status_tiles = ws->cand_cap = 0;
      ws->offsets_cap = ws->stage_cap = 0;
      return EF_ERR_NO_MEMORY;
    }
    grown.base = static_cast<char*>(p);
    grown.bytes = bytes;
    grown.dirty = true;
    *ws = grown;
  }
  if (ws->dirty) {
    // everything tagged with an epoch restarts from zero with the epochs
    const size_t clear = kHeaderBytes + sizeof(uint64_t) * ws->status_tiles;
    if (cudaMemsetAsync(ws->base, 0, clear, stream) != cudaSuccess ||
        cudaMemsetAsync(ws->chunks(), 0, sizeof(uint64_t) * kMaxChunks, stream) != cudaSuccess ||
        cudaMemsetAsync(ws->ht_chunks(0), 0, 2 * sizeof(uint64_t) * kMaxChunks, stream) !=
            cudaSuccess)
      return EF_ERR_CUDA;
    ws->epoch = 0;
    ws->ht_part_ready = false;  // no boundaries written for the next call
    ws->ht_last_tiles = 0;
    ws->dirty = false;
    if (ws->lw) ws->lw->valid = false;  // re-upload the tables, re-zero their counters
    if (ws->model_base &&
        cudaMemsetAsync(ws->model_base, 0, kModelArrivalBytes, stream) != cudaSuccess)
      return EF_ERR_CUDA;
  }
  ws->base_captured |= captured;
  *out = ws;
  return EF_OK;
}

// The workspace of (current device, stream) with `bytes` of model scratch.
// Growth synchronises the stream once; the arrival counters start at zero. A
// call that is being captured cannot grow it: its graph would zero the counters
// at each replay, not now.
ef_status acquire_model_scratch(cudaStream_t stream, size_t bytes, Workspace** out) {
  const bool captured = capturing(stream);
  if (captured) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
    std::lock_guard<std::mutex> lk(g_mu);
    const auto it = g_workspaces.find(std::make_pair(dev, stream));
    if (it == g_workspaces.end() || !it->second->base || !it->second->model_base ||
        it->second->model_bytes < bytes)
      return EF_ERR_NO_MEMORY;
    it->second->model_captured = true;
  }
  const ef_status st = acquire_workspace(stream, 0, 0, 0, 0, out);
  if (st != EF_OK) return st;
  Workspace* ws = *out;
  std::lock_guard<std::mutex> lk(g_mu);
  if (ws->model_base && ws->model_bytes >= bytes) return EF_OK;
  if (ws->model_base) {
    if (cudaStreamSynchronize(stream) != cudaSuccess) return EF_ERR_CUDA;
    replace_block(ws->model_base, ws->model_captured, ws->old_model_bases);
    ws->model_captured = false;
    ws->model_bytes = 0;
  }
  void* p = nullptr;
  if (cudaMalloc(&p, kModelArrivalBytes + bytes) != cudaSuccess) {
    cudaGetLastError();
    return EF_ERR_NO_MEMORY;
  }
  ws->model_base = static_cast<char*>(p);
  ws->model_bytes = bytes;
  return cudaMemsetAsync(p, 0, kModelArrivalBytes, stream) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
}

ef_status finish_launch(cudaError_t err, Workspace* ws) {
  if (err == cudaSuccess) return EF_OK;
  ws->dirty = true;  // a partial launch may leave the dispenser or barrier mid-way
  return EF_ERR_CUDA;
}

ef_status write_zero_count(uint32_t* count_out, cudaStream_t stream) {
  return cudaMemsetAsync(count_out, 0, sizeof(uint32_t), stream) == cudaSuccess ? EF_OK
                                                                                 : EF_ERR_CUDA;
}

ef_status write_err_zero(double* err_out, cudaStream_t stream) {
  if (!err_out) return EF_OK;
  return cudaMemsetAsync(err_out, 0, sizeof(double), stream) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
}

ef_status hard_threshold_entry(const void* g, bool bf16, float* e, float gamma, float lambda,
                               uint64_t d, uint32_t* idx_out, float* val_out,
                               uint32_t* count_out, double* err_out, uint32_t* tiles_out,
                               cudaStream_t stream) {
  const size_t gsz = bf16 ? 2 : 4;
  if (!count_out || !aligned(count_out, 4)) return EF_ERR_INVALID_ARG;
  if (!std::isfinite(gamma) || !(lambda >= 0.0f)) return EF_ERR_INVALID_ARG;
  if (d > kMaxD) return EF_ERR_INVALID_ARG;
  if (err_out && !aligned(err_out, 8)) return EF_ERR_INVALID_ARG;
  if (tiles_out && !aligned(tiles_out, 4)) return EF_ERR_INVALID_ARG;
  if (d == 0) {
    ef_status z = write_zero_count(count_out, stream);
    if (z == EF_OK && tiles_out) z = write_zero_count(tiles_out, stream);  // one entry: 0
    return z != EF_OK ? z : write_err_zero(err_out, stream);
  }
  if (!g || !e || !idx_out || !val_out) return EF_ERR_INVALID_ARG;
  if (!aligned(g, gsz) || !aligned(e, 4) || !aligned(idx_out, 4) || !aligned(val_out, 4))
    return EF_ERR_INVALID_ARG;
  const size_t nb = static_cast<size_t>(d) * 4;
  const void* outs[3] = {idx_out, val_out, count_out};
  const size_t out_n[3] = {nb, nb, 4};
  for (int o = 0; o < 3; ++o) {
    if (overlaps(outs[o], out_n[o], g, d * gsz) || overlaps(outs[o], out_n[o], e, nb))
      return EF_ERR_INVALID_ARG;
    for (int p = o + 1; p < 3; ++p)
      if (overlaps(outs[o], out_n[o], outs[p], out_n[p])) return EF_ERR_INVALID_ARG;
  }
  if (overlaps(g, d * gsz, e, nb)) return EF_ERR_INVALID_ARG;
  if (err_out && (overlaps(err_out, 8, e, nb) || overlaps(err_out, 8, g, d * gsz) ||
                  overlaps(err_out, 8, idx_out, nb) || overlaps(err_out, 8, val_out, nb) ||
                  overlaps(err_out, 8, count_out, 4)))
    return EF_ERR_INVALID_ARG;
  const size_t tb = (static_cast<size_t>(tiles_for(d)) + 1) * 4;
  if (tiles_out && (overlaps(tiles_out, tb, e, nb) || overlaps(tiles_out, tb, g, d * gsz) ||
                    overlaps(tiles_out, tb, idx_out, nb) || overlaps(tiles_out, tb, val_out, nb) ||
                    overlaps(tiles_out, tb, count_out, 4) ||
                    (err_out && overlaps(tiles_out, tb, err_out, 8))))
    return EF_ERR_INVALID_ARG;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  DeviceInfo info;
  ef_status st = device_info(dev, &info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_workspace(stream, stream_tiles_for(d), 0, 0,
                         static_cast<size_t>(stream_tiles_for(d)) * kTileElems, &ws);
  if (st != EF_OK) return st;
  return finish_launch(launch_hard_threshold(g, bf16, e, gamma, lambda, static_cast<uint32_t>(d),
                                             idx_out, val_out, count_out, err_out, tiles_out, *ws,
                                             info),
                       ws);
}

ef_status topk_entry(const void* g, bool bf16, float* e, float gamma, uint64_t k, uint64_t d,
                     uint32_t* idx_out, float* val_out, uint32_t* count_out, double* err_out,
                     cudaStream_t stream) {
  const size_t gsz = bf16 ? 2 : 4;
  if (!count_out || !aligned(count_out, 4)) return EF_ERR_INVALID_ARG;
  if (!std::isfinite(gamma)) return EF_ERR_INVALID_ARG;
  if (d > kMaxD || k > d) return EF_ERR_INVALID_ARG;
  if (err_out && !aligned(err_out, 8)) return EF_ERR_INVALID_ARG;
  if (d == 0) {
    const ef_status z = write_zero_count(count_out, stream);
    return z != EF_OK ? z : write_err_zero(err_out, stream);
  }
  if (!g || !e || (k > 0 && (!idx_out || !val_out))) return EF_ERR_INVALID_ARG;
  if (!aligned(g, gsz) || !aligned(e, 4) || !aligned(idx_out, 4) || !aligned(val_out, 4))
    return EF_ERR_INVALID_ARG;
  const size_t nb = static_cast<size_t>(d) * 4, kb = static_cast<size_t>(k) * 4;
  const void* outs[3] = {idx_out, val_out, count_out};
  const size_t out_n[3] = {kb, kb, 4};
  for (int o = 0; o < 3; ++o) {
    if (overlaps(outs[o], out_n[o], g, d * gsz) || overlaps(outs[o], out_n[o], e, nb))
      return EF_ERR_INVALID_ARG;
    for (int p = o + 1; p < 3; ++p)
      if (overlaps(outs[o], out_n[o], outs[p], out_n[p])) return EF_ERR_INVALID_ARG;
  }
  if (overlaps(g, d * gsz, e, nb)) return EF_ERR_INVALID_ARG;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  DeviceInfo info;
  ef_status st = device_info(dev, &info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_workspace(stream, stream_tiles_for(d), topk_candidate_capacity(d), 0,
                         static_cast<size_t>(stream_tiles_for(d)) * kTileElems, &ws);
  if (st != EF_OK) return st;
  if (err_out && (overlaps(err_out, 8, e, nb) || overlaps(err_out, 8, g, d * gsz) ||
                  overlaps(err_out, 8, idx_out, kb) || overlaps(err_out, 8, val_out, kb) ||
                  overlaps(err_out, 8, count_out, 4)))
    return EF_ERR_INVALID_ARG;
  return finish_launch(launch_topk(g, bf16, e, gamma, static_cast<uint32_t>(k),
                                   static_cast<uint32_t>(d), idx_out, val_out, count_out, err_out,
                                   *ws, info),
                       ws);
}

ef_status topk_layerwise_entry(const void* g, bool bf16, float* e, float gamma, uint32_t n_seg,
                               const uint64_t* seg_end, const uint64_t* seg_k, uint64_t d,
                               uint32_t* idx_out, float* val_out, uint32_t* count_out,
                               double* err_out, cudaStream_t stream) {
  const size_t gsz = bf16 ? 2 : 4;
  if (!count_out || !aligned(count_out, 4)) return EF_ERR_INVALID_ARG;
  if (!std::isfinite(gamma) || d > kMaxD) return EF_ERR_INVALID_ARG;
  if (n_seg == 0 || n_seg >= (1u << 31) || !seg_end || !seg_k) return EF_ERR_INVALID_ARG;
  uint64_t lo = 0, total_k = 0;
  for (uint32_t s = 0; s < n_seg; ++s) {
    if (seg_end[s] < lo || seg_end[s] > d || seg_k[s] > seg_end[s] - lo)
      return EF_ERR_INVALID_ARG;
    total_k += seg_k[s];
    lo = seg_end[s];
  }
  if (lo != d) return EF_ERR_INVALID_ARG;
  if (err_out && !aligned(err_out, 8)) return EF_ERR_INVALID_ARG;
  if (d == 0) {
    const ef_status z = write_zero_count(count_out, stream);
    return z != EF_OK ? z : write_err_zero(err_out, stream);
  }
  if (!g || !e || (total_k > 0 && (!idx_out || !val_out))) return EF_ERR_INVALID_ARG;
  if (!aligned(g, gsz) || !aligned(e, 4) || !aligned(idx_out, 4) || !aligned(val_out, 4))
    return EF_ERR_INVALID_ARG;
  const size_t nb = static_cast<size_t>(d) * 4, kb = static_cast<size_t>(total_k) * 4;
  const void* outs[3] = {idx_out, val_out, count_out};
  const size_t out_n[3] = {kb, kb, 4};
  for (int o = 0; o < 3; ++o) {
    if (overlaps(outs[o], out_n[o], g, d * gsz) || overlaps(outs[o], out_n[o], e, nb))
      return EF_ERR_INVALID_ARG;
    for (int p = o + 1; p < 3; ++p)
      if (overlaps(outs[o], out_n[o], outs[p], out_n[p])) return EF_ERR_INVALID_ARG;
  }
  if (overlaps(g, d * gsz, e, nb)) return EF_ERR_INVALID_ARG;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  DeviceInfo info;
  ef_status st = device_info(dev, &info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_workspace(stream, stream_tiles_for(d), topk_candidate_capacity(d), 0,
                         static_cast<size_t>(stream_tiles_for(d)) * kTileElems, &ws);
  if (st != EF_OK) return st;
  if (err_out && (overlaps(err_out, 8, e, nb) || overlaps(err_out, 8, g, d * gsz) ||
                  overlaps(err_out, 8, idx_out, kb) || overlaps(err_out, 8, val_out, kb) ||
                  overlaps(err_out, 8, count_out, 4)))
    return EF_ERR_INVALID_ARG;
  const cudaError_t perr = lw_prepare(*ws, seg_end, seg_k, n_seg, d, info);
  if (perr == cudaErrorMemoryAllocation) return EF_ERR_NO_MEMORY;
  if (perr != cudaSuccess) return EF_ERR_CUDA;
  return finish_launch(launch_topk_layerwise(g, bf16, e, gamma, static_cast<uint32_t>(d),
                                             idx_out, val_out, count_out, err_out, *ws, info),
                       ws);
}

// A matrix in memory, in bytes: rows of `width`, `stride` apart.
struct Rows {
  uintptr_t at;
  uint64_t rows, width, stride;
  // (2^57 bytes from there: past any address; and nothing overflows)
  uintptr_t end() const {
    const uint64_t most = 1ull << 57;
    return at + (rows - 1 > most / stride ? most : (rows - 1) * stride + width);
  }
};
Rows rows_of(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size) {
  return {reinterpret_cast<uintptr_t>(p), p && cols ? rows : 0, cols * size, ld * size};
}
Rows vector_of(const void* p, uint64_t bytes) { return rows_of(p, 1, bytes, bytes, 1); }

// Whether two matrices overlap: where their rows have one stride (column blocks
// of a buffer), whether they share a byte; else whether the ranges do that they
// lie in.
bool overlaps(const Rows& a, const Rows& b) {
  if (a.rows == 0 || b.rows == 0 || a.at >= b.end() || b.at >= a.end()) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  if (a.rows > 1 && b.rows > 1 && a.stride != b.stride) return true;
  const uint64_t stride = a.rows > 1 ? a.stride : b.stride;
  const uint64_t apart = b.at >= a.at ? (b.at - a.at) % stride : stride - (a.at - b.at - 1) % stride - 1;
  return apart < a.width || b.width > stride - apart;
}

constexpr uint64_t kMaxRows = 1u << 30, kMaxWords = 1u << 30, kMaxWidth = 1u << 20;
constexpr uint64_t kMaxLd = 1ull << 36;
constexpr uint64_t kMaxSide = 1u << 20;   // rows or columns of a matrix to orthogonalise
constexpr uint32_t kMaxMatrices = 4096;

// What the loss and its gradient check alike.
bool vocab_inputs_ok(const VocabCall& c, uint64_t n, uint64_t v, uint64_t d) {
  if (n > kMaxRows || v == 0 || v > kMaxWords || d == 0 || d > kMaxWidth) return false;
  if (c.ldh < d || c.ldw < d || c.ldh > kMaxLd || c.ldw > kMaxLd) return false;
  if (!c.w || !aligned(c.w, 2) || !aligned(c.bias, 2) || !aligned(c.lse, 4)) return false;
  if (n && (!c.h || !c.target || !c.lse || !aligned(c.h, 2) || !aligned(c.target, 8))) return false;
  return true;
}

ef_status vocab_entry(VocabCall c, uint64_t n, uint64_t v, uint64_t d, bool gradient,
                      cudaStream_t stream) {
  if (!vocab_inputs_ok(c, n, v, d)) return EF_ERR_INVALID_ARG;
  c.n = static_cast<uint32_t>(n);
  c.v = static_cast<uint32_t>(v);
  c.d = static_cast<uint32_t>(d);
  const Rows in[] = {rows_of(c.h, n, d, c.ldh, 2), rows_of(c.w, v, d, c.ldw, 2),
                     vector_of(c.bias, v * 2),     vector_of(c.target, n * 8),
                     vector_of(gradient ? c.lse : nullptr, n * 4), vector_of(c.row_scale, n * 4)};
  Rows outs[3];
  if (gradient) {
    if (!c.dw || !aligned(c.dw, 2) || c.lddw < d || c.lddw > kMaxLd) return EF_ERR_INVALID_ARG;
    if (!aligned(c.dbias, 2) || (c.dbias && !c.bias)) return EF_ERR_INVALID_ARG;
    if (n && (!c.dh || !aligned(c.dh, 2) || c.lddh < d || c.lddh > kMaxLd || !c.row_scale ||
              !aligned(c.row_scale, 4)))
      return EF_ERR_INVALID_ARG;
    outs[0] = rows_of(c.dh, n, d, c.lddh, 2);
    outs[1] = rows_of(c.dw, v, d, c.lddw, 2);
    outs[2] = vector_of(c.dbias, v * 2);
  } else {
    if (n == 0) return EF_OK;
    if (!c.loss || !aligned(c.loss, 4)) return EF_ERR_INVALID_ARG;
    outs[0] = vector_of(c.loss, n * 4);
    outs[1] = vector_of(c.lse, n * 4);
    outs[2] = vector_of(nullptr, 0);
  }
  for (int o = 0; o < 3; ++o) {
    for (const Rows& i : in)
      if (overlaps(outs[o], i)) return EF_ERR_INVALID_ARG;
    for (int q = o + 1; q < 3; ++q)
      if (overlaps(outs[o], outs[q])) return EF_ERR_INVALID_ARG;
  }
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  DeviceInfo info;
  ef_status st = device_info(dev, &info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_model_scratch(stream, vocab_scratch(c, gradient, info), &ws);
  if (st != EF_OK) return st;
  return finish_launch(gradient ? launch_vocab_loss_grad(c, *ws, info)
                                : launch_vocab_loss(c, *ws, info),
                       ws);
}

ef_status orthogonalize_entry(uint32_t n, const uint64_t* rows, const uint64_t* cols,
                              const void* const* u, const uint64_t* ld_u, bool bf16,
                              float* const* m, const uint64_t* ld_m, float momentum,
                              uint16_t* const* out, const uint64_t* ld_out,
                              cudaStream_t stream) {
  if (n > kMaxMatrices || !std::isfinite(momentum)) return EF_ERR_INVALID_ARG;
  if (n == 0) return EF_OK;
  if (!rows || !cols || !u || !ld_u || !out || !ld_out || (m && !ld_m)) return EF_ERR_INVALID_ARG;
  const size_t usz = bf16 ? 2 : 4;
  std::vector<OrthoMat> mats(n);
  struct Used {
    Rows rows;
    bool written;
  };
  std::vector<Used> used;
  used.reserve(3ull * n);
  for (uint32_t i = 0; i < n; ++i) {
    OrthoMat& t = mats[i];
    if (rows[i] > kMaxSide || cols[i] > kMaxSide) return EF_ERR_INVALID_ARG;
    t.rows = static_cast<uint32_t>(rows[i]);
    t.cols = static_cast<uint32_t>(cols[i]);
    t.u = u[i];
    t.m = m ? m[i] : nullptr;
    t.out = out[i];
    t.ld_u = ld_u[i];
    t.ld_m = m ? ld_m[i] : 0;
    t.ld_out = ld_out[i];
    if (t.rows == 0 || t.cols == 0) continue;
    if (!t.u || !t.out || (m && !t.m)) return EF_ERR_INVALID_ARG;
    if (!aligned(t.u, usz) || !aligned(t.m, 4) || !aligned(t.out, 2)) return EF_ERR_INVALID_ARG;
    if (t.ld_u < t.cols || t.ld_out < t.cols || (m && t.ld_m < t.cols)) return EF_ERR_INVALID_ARG;
    if (t.ld_u > kMaxLd || t.ld_out > kMaxLd || t.ld_m > kMaxLd) return EF_ERR_INVALID_ARG;
    used.push_back({rows_of(t.u, t.rows, t.cols, t.ld_u, usz), false});
    if (m) used.push_back({rows_of(t.m, t.rows, t.cols, t.ld_m, 4), true});
    used.push_back({rows_of(t.out, t.rows, t.cols, t.ld_out, 2), true});
  }
  if (used.empty()) return EF_OK;
  // nothing written may overlap anything else: by start, against those before that
  // reach that far
  std::sort(used.begin(), used.end(),
            [](const Used& x, const Used& y) { return x.rows.at < y.rows.at; });
  std::vector<Used> open;
  for (const Used& s : used) {
    size_t kept = 0;
    for (const Used& o : open) {
      if (o.rows.end() <= s.rows.at) continue;
      if ((o.written || s.written) && overlaps(o.rows, s.rows)) return EF_ERR_INVALID_ARG;
      open[kept++] = o;
    }
    open.resize(kept);
    open.push_back(s);
  }
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  DeviceInfo info;
  ef_status st = device_info(dev, &info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  std::shared_ptr<void> plan;
  st = acquire_model_scratch(stream, ortho_plan(mats.data(), n, info, &plan), &ws);
  if (st != EF_OK) return st;
  return finish_launch(
      launch_orthogonalize(mats.data(), n, bf16, momentum, plan.get(), *ws, info), ws);
}

// ---- the rest of a language-model training step ----
bool grad_type_ok(ef_grad_type t) { return t == EF_GRAD_F32 || t == EF_GRAD_BF16; }
uint64_t size_of(ef_grad_type t) { return t == EF_GRAD_BF16 ? 2 : 4; }

ef_status this_device(DeviceInfo* info) {
  int dev = 0;
  return cudaGetDevice(&dev) != cudaSuccess ? EF_ERR_CUDA : device_info(dev, info);
}

// Whether an output overlaps an input or another output.
template <int I, int O>
bool any_overlap(const Rows (&in)[I], const Rows (&out)[O]) {
  for (int o = 0; o < O; ++o) {
    for (const Rows& i : in)
      if (overlaps(out[o], i)) return true;
    for (int q = o + 1; q < O; ++q)
      if (overlaps(out[o], out[q])) return true;
  }
  return false;
}

bool matrix_ok(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size) {
  return ld >= cols && ld <= kMaxLd && (rows == 0 || (p && aligned(p, size)));
}

ef_status embed_entry(const void* table, uint64_t ld_table, ef_grad_type table_type,
                      const int64_t* token, uint64_t n, uint64_t v, uint64_t d, float scale,
                      void* out, uint64_t ld_out, ef_grad_type out_type, cudaStream_t stream) {
  if (!grad_type_ok(table_type) || !grad_type_ok(out_type) || !std::isfinite(scale) ||
      n > kMaxRows || v == 0 || v > kMaxWords || d == 0 || d > kMaxWidth ||
      !matrix_ok(table, v, d, ld_table, size_of(table_type)) ||
      !matrix_ok(out, n, d, ld_out, size_of(out_type)) || !aligned(token, 8))
    return EF_ERR_INVALID_ARG;
  if (n == 0) return EF_OK;
  if (!token) return EF_ERR_INVALID_ARG;
  const Rows in[] = {rows_of(table, v, d, ld_table, size_of(table_type)), vector_of(token, n * 8)};
  const Rows outs[] = {rows_of(out, n, d, ld_out, size_of(out_type))};
  if (any_overlap(in, outs)) return EF_ERR_INVALID_ARG;
  EmbedCall c = {};
  c.table = table;
  c.out = out;
  c.token = token;
  c.ld_table = ld_table;
  c.ld_out = ld_out;
  c.n = static_cast<uint32_t>(n);
  c.v = static_cast<uint32_t>(v);
  c.d = static_cast<uint32_t>(d);
  c.scale = scale;
  c.table_bf16 = table_type == EF_GRAD_BF16;
  c.out_bf16 = out_type == EF_GRAD_BF16;
  DeviceInfo info;
  ef_status st = this_device(&info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_model_scratch(stream, 0, &ws);
  return st != EF_OK ? st : finish_launch(launch_embed(c, *ws, info), ws);
}

ef_status embed_grad_entry(const void* dout, uint64_t ld_dout, ef_grad_type dout_type,
                           const int64_t* token, uint64_t n, uint64_t v, uint64_t d, float scale,
                           int accumulate, void* dtable, uint64_t ld_dtable,
                           ef_grad_type dtable_type, cudaStream_t stream) {
  if (!grad_type_ok(dout_type) || !grad_type_ok(dtable_type) || !std::isfinite(scale) ||
      n > kMaxRows || v == 0 || v > kMaxWords || d == 0 || d > kMaxWidth ||
      !matrix_ok(dout, n, d, ld_dout, size_of(dout_type)) ||
      !matrix_ok(dtable, v, d, ld_dtable, size_of(dtable_type)) || !aligned(token, 8) ||
      (n && !token))
    return EF_ERR_INVALID_ARG;
  const Rows in[] = {rows_of(dout, n, d, ld_dout, size_of(dout_type)), vector_of(token, n * 8)};
  const Rows outs[] = {rows_of(dtable, v, d, ld_dtable, size_of(dtable_type))};
  if (any_overlap(in, outs)) return EF_ERR_INVALID_ARG;
  if (n == 0 && accumulate) return EF_OK;
  EmbedGradCall c = {};
  c.dout = dout;
  c.dtable = dtable;
  c.token = token;
  c.ld_dout = ld_dout;
  c.ld_dtable = ld_dtable;
  c.n = static_cast<uint32_t>(n);
  c.v = static_cast<uint32_t>(v);
  c.d = static_cast<uint32_t>(d);
  c.scale = scale;
  c.dout_bf16 = dout_type == EF_GRAD_BF16;
  c.dtable_bf16 = dtable_type == EF_GRAD_BF16;
  c.add = accumulate != 0;
  DeviceInfo info;
  ef_status st = this_device(&info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_model_scratch(stream, embed_grad_scratch(c, info), &ws);
  return st != EF_OK ? st : finish_launch(launch_embed_grad(c, *ws, info), ws);
}

ef_status layer_norm_entry(const void* x, uint64_t ldx, ef_grad_type x_type, const void* weight,
                           const void* bias, ef_grad_type w_type, float eps, uint64_t n, uint64_t d,
                           void* y, uint64_t ldy, ef_grad_type y_type, float* mean, float* rstd,
                           cudaStream_t stream) {
  if (!grad_type_ok(x_type) || !grad_type_ok(w_type) || !grad_type_ok(y_type)) return EF_ERR_INVALID_ARG;
  const uint64_t xs = size_of(x_type), wsz = size_of(w_type), ys = size_of(y_type);
  if (!(eps >= 0.0f) || !std::isfinite(eps) || n > kMaxRows || d == 0 || d > kMaxWidth ||
      !matrix_ok(x, n, d, ldx, xs) || !matrix_ok(y, n, d, ldy, ys) || !aligned(weight, wsz) ||
      !aligned(bias, wsz) || !aligned(mean, 4) || !aligned(rstd, 4))
    return EF_ERR_INVALID_ARG;
  if (n == 0) return EF_OK;
  const Rows in[] = {rows_of(x, n, d, ldx, xs), vector_of(weight, d * wsz), vector_of(bias, d * wsz)};
  const Rows outs[] = {rows_of(y, n, d, ldy, ys), vector_of(mean, n * 4), vector_of(rstd, n * 4)};
  if (any_overlap(in, outs)) return EF_ERR_INVALID_ARG;
  NormCall c = {};
  c.x = x;
  c.y = y;
  c.w = weight;
  c.b = bias;
  c.mean = mean;
  c.rstd = rstd;
  c.ldx = ldx;
  c.ldy = ldy;
  c.eps = eps;
  c.n = static_cast<uint32_t>(n);
  c.d = static_cast<uint32_t>(d);
  c.x_bf16 = x_type == EF_GRAD_BF16;
  c.y_bf16 = y_type == EF_GRAD_BF16;
  c.w_bf16 = w_type == EF_GRAD_BF16;
  DeviceInfo info;
  const ef_status st = this_device(&info);
  if (st != EF_OK) return st;
  return launch_layer_norm(c, info, stream) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
}

ef_status layer_norm_grad_entry(const void* x, uint64_t ldx, ef_grad_type x_type,
                                const void* weight, ef_grad_type w_type, const float* mean,
                                const float* rstd, const void* dy, uint64_t lddy,
                                ef_grad_type dy_type, uint64_t n, uint64_t d, void* dx,
                                uint64_t lddx, void* dweight, void* dbias, cudaStream_t stream) {
  if (!grad_type_ok(x_type) || !grad_type_ok(w_type) || !grad_type_ok(dy_type)) return EF_ERR_INVALID_ARG;
  const uint64_t xs = size_of(x_type), wsz = size_of(w_type), ys = size_of(dy_type);
  if (n > kMaxRows || d == 0 || d > kMaxWidth || !matrix_ok(x, n, d, ldx, xs) ||
      !matrix_ok(dy, n, d, lddy, ys) || (dx && !matrix_ok(dx, n, d, lddx, xs)) ||
      !aligned(weight, wsz) || !aligned(dweight, wsz) || !aligned(dbias, wsz) ||
      !aligned(mean, 4) || !aligned(rstd, 4) || (n && (!mean || !rstd)))
    return EF_ERR_INVALID_ARG;
  const Rows in[] = {rows_of(x, n, d, ldx, xs), rows_of(dy, n, d, lddy, ys),
                     vector_of(weight, d * wsz), vector_of(mean, n * 4), vector_of(rstd, n * 4)};
  const Rows outs[] = {rows_of(dx, n, d, lddx, xs), vector_of(dweight, d * wsz),
                       vector_of(dbias, d * wsz)};
  if (any_overlap(in, outs)) return EF_ERR_INVALID_ARG;
  if (!dweight && !dbias && (!dx || n == 0)) return EF_OK;
  NormGradCall c = {};
  c.x = x;
  c.dy = dy;
  c.dx = dx;
  c.w = weight;
  c.dw = dweight;
  c.db = dbias;
  c.mean = mean;
  c.rstd = rstd;
  c.ldx = ldx;
  c.lddy = lddy;
  c.lddx = lddx;
  c.n = static_cast<uint32_t>(n);
  c.d = static_cast<uint32_t>(d);
  c.x_bf16 = x_type == EF_GRAD_BF16;
  c.y_bf16 = dy_type == EF_GRAD_BF16;
  c.w_bf16 = w_type == EF_GRAD_BF16;
  DeviceInfo info;
  ef_status st = this_device(&info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  size_t bytes = 0;
  if (norm_grad_scratch(c, info, &bytes) != cudaSuccess) return EF_ERR_CUDA;
  if (bytes && (st = acquire_model_scratch(stream, bytes, &ws)) != EF_OK) return st;
  const cudaError_t err = launch_layer_norm_grad(c, ws, stream, info);
  if (ws) return finish_launch(err, ws);
  return err == cudaSuccess ? EF_OK : EF_ERR_CUDA;
}

// Whether anything written overlaps anything else among the arrays of lists of tensors:
// range(l, i) is that of tensor i in list l. Lists as models have them, each ascending in
// its own stretch of memory, are seen to be apart in one pass; others by sorting.
struct Range {
  uintptr_t at;
  uint64_t bytes;  // 0: none
  bool written;
};
template <typename F>
bool lists_overlap(uint32_t lists, uint32_t n, F range) {
  struct Span {
    uintptr_t at, end;
  };
  std::array<Span, 10> spans;
  uint32_t used = 0;
  bool apart = true;
  for (uint32_t l = 0; l < lists && apart; ++l) {
    Span s = {UINTPTR_MAX, 0};
    for (uint32_t i = 0; i < n; ++i) {
      const Range r = range(l, i);
      if (r.bytes == 0) continue;
      apart &= r.at >= s.end;
      s.at = std::min(s.at, r.at);
      s.end = std::max(s.end, r.at + r.bytes);
    }
    for (uint32_t q = 0; q < used; ++q) apart &= s.at >= spans[q].end || spans[q].at >= s.end;
    if (s.end) spans[used++] = s;
  }
  if (apart) return false;
  std::vector<Range> all;
  all.reserve(static_cast<size_t>(lists) * n);
  for (uint32_t l = 0; l < lists; ++l)
    for (uint32_t i = 0; i < n; ++i) {
      const Range r = range(l, i);
      if (r.bytes) all.push_back(r);
    }
  std::sort(all.begin(), all.end(), [](const Range& x, const Range& y) { return x.at < y.at; });
  uintptr_t any = 0, write = 0;  // how far those before reach
  for (const Range& r : all) {
    if (r.at < write || (r.written && r.at < any)) return true;
    any = std::max(any, r.at + r.bytes);
    if (r.written) write = std::max(write, r.at + r.bytes);
  }
  return false;
}
Range range_of(const void* p, uint64_t bytes, bool written) {
  return {reinterpret_cast<uintptr_t>(p), p ? bytes : 0, written};
}
uint64_t blocks_of(uint64_t numel) { return (numel + 127) / 128; }

constexpr uint32_t kMaxTensors = 1u << 20;

ef_status adamw_entry(uint32_t n, const uint64_t* numel, float* const* p, const void* const* g,
                      ef_grad_type g_type, void* const* m, void* const* v, uint8_t* const* me,
                      uint8_t* const* ve, uint16_t* const* copy, AdamCall c, cudaStream_t stream) {
  if (n > kMaxTensors || !grad_type_ok(g_type) || !std::isfinite(c.lr) || !std::isfinite(c.decay) ||
      !(c.b1 >= 0.0 && c.b1 < 1.0) || !(c.b2 >= 0.0 && c.b2 < 1.0) || !std::isfinite(c.eps) ||
      !(c.eps == 0.0 || c.eps >= FLT_MIN) || (c.step == 0 && !c.step_dev) || !aligned(c.lr_dev, 4) ||
      !aligned(c.step_dev, 8) || !aligned(c.grad_scale, 4) || (me == nullptr) != (ve == nullptr))
    return EF_ERR_INVALID_ARG;
  if (n == 0) return EF_OK;
  if (!numel || !p || !g || !m || !v) return EF_ERR_INVALID_ARG;
  c.g_bf16 = g_type == EF_GRAD_BF16;
  c.eight = me != nullptr;
  const uint64_t state = c.eight ? 1 : 4;
  static thread_local std::vector<AdamTensor> t;  // (kept for its memory)
  t.assign(n, AdamTensor());
  bool any = false;
  for (uint32_t i = 0; i < n; ++i) {
    if (numel[i] > kMaxD - 4095) return EF_ERR_INVALID_ARG;
    t[i].numel = static_cast<uint32_t>(numel[i]);
    if (numel[i] == 0) continue;
    any = true;
    t[i].p = p[i];
    t[i].g = g[i];
    t[i].m = m[i];
    t[i].v = v[i];
    t[i].copy = copy ? copy[i] : nullptr;
    t[i].me = me ? me[i] : nullptr;
    t[i].ve = ve ? ve[i] : nullptr;
    if (!p[i] || !g[i] || !m[i] || !v[i] || (copy && !copy[i]) || (me && (!me[i] || !ve[i])) ||
        !aligned(p[i], 4) || !aligned(g[i], size_of(g_type)) || !aligned(m[i], state) ||
        !aligned(v[i], state) || !aligned(t[i].copy, 2))
      return EF_ERR_INVALID_ARG;
  }
  if (!any) return EF_OK;
  const uint64_t gsize = size_of(g_type);
  const auto range = [&](uint32_t l, uint32_t i) {
    const AdamTensor& x = t[i];
    const uint64_t k = x.numel;
    switch (l) {
      case 0: return range_of(x.p, k * 4, true);
      case 1: return range_of(x.g, k * gsize, false);
      case 2: return range_of(x.m, k * state, true);
      case 3: return range_of(x.v, k * state, true);
      case 4: return range_of(x.copy, k * 2, true);
      case 5: return range_of(x.me, blocks_of(k), true);
      case 6: return range_of(x.ve, blocks_of(k), true);
      case 7: return range_of(i ? nullptr : c.lr_dev, 4, false);
      case 8: return range_of(i ? nullptr : c.step_dev, 8, false);
      default: return range_of(i ? nullptr : c.grad_scale, 4, false);
    }
  };
  if (lists_overlap(10, n, range)) return EF_ERR_INVALID_ARG;
  return launch_adamw(t.data(), n, c, stream) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
}

ef_status adamw_states_entry(uint32_t n, const uint64_t* numel, const uint8_t* const* m,
                             const uint8_t* const* v, const uint8_t* const* me,
                             const uint8_t* const* ve, void* const* m_out, void* const* v_out,
                             ef_grad_type out_type, cudaStream_t stream) {
  if (n > kMaxTensors || !grad_type_ok(out_type)) return EF_ERR_INVALID_ARG;
  if (n == 0) return EF_OK;
  if (!numel || !m || !v || !me || !ve || !m_out || !v_out) return EF_ERR_INVALID_ARG;
  const uint64_t size = size_of(out_type);
  static thread_local std::vector<AdamStates> t;  // (kept for its memory)
  t.assign(n, AdamStates());
  for (uint32_t i = 0; i < n; ++i) {
    if (numel[i] > kMaxD - 4095) return EF_ERR_INVALID_ARG;
    t[i].numel = static_cast<uint32_t>(numel[i]);
    if (numel[i] == 0) continue;
    t[i].m = m[i];
    t[i].v = v[i];
    t[i].me = me[i];
    t[i].ve = ve[i];
    t[i].m_out = m_out[i];
    t[i].v_out = v_out[i];
    if (!m[i] || !v[i] || !me[i] || !ve[i] || !m_out[i] || !v_out[i] || !aligned(m_out[i], size) ||
        !aligned(v_out[i], size))
      return EF_ERR_INVALID_ARG;
  }
  const auto range = [&](uint32_t l, uint32_t i) {
    const AdamStates& x = t[i];
    const uint64_t k = x.numel;
    switch (l) {
      case 0: return range_of(x.m, k, false);
      case 1: return range_of(x.v, k, false);
      case 2: return range_of(x.me, blocks_of(k), false);
      case 3: return range_of(x.ve, blocks_of(k), false);
      case 4: return range_of(x.m_out, k * size, true);
      default: return range_of(x.v_out, k * size, true);
    }
  };
  if (lists_overlap(6, n, range)) return EF_ERR_INVALID_ARG;
  return launch_adamw_states(t.data(), n, out_type == EF_GRAD_BF16, stream) == cudaSuccess ? EF_OK
                                                                                            : EF_ERR_CUDA;
}

// An entry's body, with what it may throw as a status.
template <typename F>
ef_status guarded(F&& body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return EF_ERR_NO_MEMORY;
  } catch (...) {
    return EF_ERR_CUDA;
  }
}

}  // namespace

// A launch that may begin while the previous kernel on the stream finishes
// (programmatic dependent launch; every kernel here waits for its
// predecessor before reading what it wrote), optionally cooperative.
cudaError_t launch_pdl(const void* fn, dim3 grid, uint32_t block, uint32_t smem,
                       cudaStream_t stream, void** params, bool cooperative) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeCooperative;
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cooperative ? 2 : 1;
  return cudaLaunchKernelExC(&cfg, fn, params);
}

void count_launch() { g_launches.fetch_add(1, std::memory_order_relaxed); }
uint64_t wait_limit_ns() { return g_wait_limit_ns.load(); }
int64_t withheld_tile() { return g_withheld_tile.load(); }
int stream_kernel_mode() { return g_stream_kernel_mode.load(); }

ScanCtx next_scan_ctx(Workspace& ws, uint32_t num_tiles) {
  if (ws.epoch >= (1u << 30) - 1) {  // epoch wrap: old words must not match again
    cudaMemsetAsync(ws.status(), 0, sizeof(uint64_t) * ws.status_tiles, ws.stream);
    cudaMemsetAsync(ws.chunks(), 0, sizeof(uint64_t) * kMaxChunks, ws.stream);
    ws.epoch = 0;
  }
  ++ws.epoch;
  ScanCtx c;
  c.status = ws.status();
  c.error = ws.u32(kOffError);
  c.epoch = ws.epoch;
  c.num_tiles = num_tiles;
  c.withheld_tile = withheld_tile();
  c.wait_limit_ns = wait_limit_ns();
  c.tile_claim = nullptr;  // (the one-tile-per-CTA kernel's, on its own scratch)
  return c;
}

// The aggregate entries: the plain sum (dense_out set) or the fused update
// (x set); tiles optional.
ef_status aggregate_entry(uint32_t n, const uint32_t* const* idx, const float* const* val,
                          const uint32_t* const* tiles, const uint32_t* counts, uint64_t d,
                          float* dense_out, float alpha, float* x, float* m, float momentum,
                          float lr, cudaStream_t s) {
  if (n == 0 || n > kMaxWorkers || !idx || !val || !counts) return EF_ERR_INVALID_ARG;
  if (d > kMaxD) return EF_ERR_INVALID_ARG;
  const bool apply = x != nullptr;
  if (apply && (!std::isfinite(alpha) || !std::isfinite(momentum) || !std::isfinite(lr)))
    return EF_ERR_INVALID_ARG;
  if (d == 0) return EF_OK;
  const size_t nb = static_cast<size_t>(d) * 4;
  if (!aligned(counts, 4)) return EF_ERR_INVALID_ARG;
  if (apply) {
    if (!aligned(x, 4) || (m && !aligned(m, 4))) return EF_ERR_INVALID_ARG;
    if (m && overlaps(x, nb, m, nb)) return EF_ERR_INVALID_ARG;
  } else if (!dense_out || !aligned(dense_out, 4)) {
    return EF_ERR_INVALID_ARG;
  }
  for (uint32_t i = 0; i < n; ++i) {
    if (!idx[i] || !val[i] || !aligned(idx[i], 4) || !aligned(val[i], 4))
      return EF_ERR_INVALID_ARG;
    if (tiles && (!tiles[i] || !aligned(tiles[i], 4))) return EF_ERR_INVALID_ARG;
  }
  const uint32_t nt = agg_tiles_for(d);
  int dev = 0;  // the per-device set-up (kernel attributes) on first use
  DeviceInfo info;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  if (device_info(dev, &info) != EF_OK) return EF_ERR_CUDA;
  Workspace* ws = nullptr;
  const size_t offsets = tiles ? 0 : static_cast<size_t>(n) * (static_cast<size_t>(nt) + 1);
  const ef_status st = acquire_workspace(s, 0, 0, offsets, 0, &ws);
  if (st != EF_OK) return st;
  const uint32_t d32 = static_cast<uint32_t>(d);
  if (apply)
    return finish_launch(
        launch_aggregate_apply(n, idx, val, tiles, counts, d32, alpha, x, m, momentum, lr, *ws),
        ws);
  return finish_launch(launch_aggregate(n, idx, val, tiles, counts, d32, dense_out, *ws, info),
                       ws);
}

}  // namespace efs

using efs::Workspace;

extern "C" {

ef_status ef_hard_threshold(const float* g, float* e, float gamma, float lambda, uint64_t d,
                            uint32_t* idx_out, float* val_out, uint32_t* count_out,
                            ef_stream_t stream) {
  return efs::hard_threshold_entry(g, false, e, gamma, lambda, d, idx_out, val_out, count_out,
                                   nullptr, nullptr, reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_hard_threshold_bf16(const uint16_t* g, float* e, float gamma, float lambda,
                                 uint64_t d, uint32_t* idx_out, float* val_out,
                                 uint32_t* count_out, ef_stream_t stream) {
  return efs::hard_threshold_entry(g, true, e, gamma, lambda, d, idx_out, val_out, count_out,
                                   nullptr, nullptr, reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_topk(const float* g, float* e, float gamma, uint64_t k, uint64_t d,
                  uint32_t* idx_out, float* val_out, uint32_t* count_out, ef_stream_t stream) {
  return efs::topk_entry(g, false, e, gamma, k, d, idx_out, val_out, count_out, nullptr,
                         reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_topk_bf16(const uint16_t* g, float* e, float gamma, uint64_t k, uint64_t d,
                       uint32_t* idx_out, float* val_out, uint32_t* count_out,
                       ef_stream_t stream) {
  return efs::topk_entry(g, true, e, gamma, k, d, idx_out, val_out, count_out, nullptr,
                         reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_topk_layerwise(const float* g, float* e, float gamma, uint32_t n_seg,
                            const uint64_t* seg_end, const uint64_t* seg_k, uint64_t d,
                            uint32_t* idx_out, float* val_out, uint32_t* count_out,
                            ef_stream_t stream) {
  return efs::topk_layerwise_entry(g, false, e, gamma, n_seg, seg_end, seg_k, d, idx_out,
                                   val_out, count_out, nullptr,
                                   reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_topk_layerwise_bf16(const uint16_t* g, float* e, float gamma, uint32_t n_seg,
                                 const uint64_t* seg_end, const uint64_t* seg_k, uint64_t d,
                                 uint32_t* idx_out, float* val_out, uint32_t* count_out,
                                 ef_stream_t stream) {
  return efs::topk_layerwise_entry(g, true, e, gamma, n_seg, seg_end, seg_k, d, idx_out,
                                   val_out, count_out, nullptr,
                                   reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_hard_threshold_ex(const void* g, ef_grad_type g_type, float* e, float gamma,
                               float lambda, uint64_t d, uint32_t* idx_out, float* val_out,
                               uint32_t* count_out, double* err_sq_out, ef_stream_t stream) {
  if (g_type != EF_GRAD_F32 && g_type != EF_GRAD_BF16) return EF_ERR_INVALID_ARG;
  return efs::hard_threshold_entry(g, g_type == EF_GRAD_BF16, e, gamma, lambda, d, idx_out,
                                   val_out, count_out, err_sq_out, nullptr,
                                   reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_hard_threshold_tiled(const void* g, ef_grad_type g_type, float* e, float gamma,
                                  float lambda, uint64_t d, uint32_t* idx_out, float* val_out,
                                  uint32_t* count_out, uint32_t* tiles_out, double* err_sq_out,
                                  ef_stream_t stream) {
  if (g_type != EF_GRAD_F32 && g_type != EF_GRAD_BF16) return EF_ERR_INVALID_ARG;
  if (!tiles_out) return EF_ERR_INVALID_ARG;
  return efs::hard_threshold_entry(g, g_type == EF_GRAD_BF16, e, gamma, lambda, d, idx_out,
                                   val_out, count_out, err_sq_out, tiles_out,
                                   reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_topk_ex(const void* g, ef_grad_type g_type, float* e, float gamma, uint64_t k,
                     uint64_t d, uint32_t* idx_out, float* val_out, uint32_t* count_out,
                     double* err_sq_out, ef_stream_t stream) {
  if (g_type != EF_GRAD_F32 && g_type != EF_GRAD_BF16) return EF_ERR_INVALID_ARG;
  return efs::topk_entry(g, g_type == EF_GRAD_BF16, e, gamma, k, d, idx_out, val_out, count_out,
                         err_sq_out, reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_topk_layerwise_ex(const void* g, ef_grad_type g_type, float* e, float gamma,
                               uint32_t n_seg, const uint64_t* seg_end, const uint64_t* seg_k,
                               uint64_t d, uint32_t* idx_out, float* val_out,
                               uint32_t* count_out, double* err_sq_out, ef_stream_t stream) {
  if (g_type != EF_GRAD_F32 && g_type != EF_GRAD_BF16) return EF_ERR_INVALID_ARG;
  return efs::topk_layerwise_entry(g, g_type == EF_GRAD_BF16, e, gamma, n_seg, seg_end, seg_k,
                                   d, idx_out, val_out, count_out, err_sq_out,
                                   reinterpret_cast<cudaStream_t>(stream));
}

ef_status sparse_aggregate(uint32_t n, const uint32_t* const* idx, const float* const* val,
                           const uint32_t* counts, uint64_t d, float* dense_out,
                           ef_stream_t stream) {
  return efs::aggregate_entry(n, idx, val, nullptr, counts, d, dense_out, 0.0f, nullptr,
                              nullptr, 0.0f, 0.0f, reinterpret_cast<cudaStream_t>(stream));
}

ef_status sparse_aggregate_tiled(uint32_t n, const uint32_t* const* idx, const float* const* val,
                                 const uint32_t* const* tiles, const uint32_t* counts, uint64_t d,
                                 float* dense_out, ef_stream_t stream) {
  if (!tiles) return EF_ERR_INVALID_ARG;
  return efs::aggregate_entry(n, idx, val, tiles, counts, d, dense_out, 0.0f, nullptr, nullptr,
                              0.0f, 0.0f, reinterpret_cast<cudaStream_t>(stream));
}

ef_status sparse_aggregate_apply(uint32_t n, const uint32_t* const* idx, const float* const* val,
                                 const uint32_t* counts, uint64_t d, float alpha, float* x,
                                 float* m, float momentum, float lr, ef_stream_t stream) {
  if (!x) return EF_ERR_INVALID_ARG;
  return efs::aggregate_entry(n, idx, val, nullptr, counts, d, nullptr, alpha, x, m, momentum,
                              lr, reinterpret_cast<cudaStream_t>(stream));
}

ef_status sparse_aggregate_apply_tiled(uint32_t n, const uint32_t* const* idx,
                                       const float* const* val, const uint32_t* const* tiles,
                                       const uint32_t* counts, uint64_t d, float alpha, float* x,
                                       float* m, float momentum, float lr, ef_stream_t stream) {
  if (!tiles || !x) return EF_ERR_INVALID_ARG;
  return efs::aggregate_entry(n, idx, val, tiles, counts, d, nullptr, alpha, x, m, momentum, lr,
                              reinterpret_cast<cudaStream_t>(stream));
}

ef_status ef_scaled_round_ex(const void* g, ef_grad_type g_type, float* e, float gamma,
                             int32_t scale_log2, uint64_t d, int32_t* q_out,
                             uint32_t* unsent_out, double* err_sq_out, ef_stream_t stream) {
  using namespace efs;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (g_type != EF_GRAD_F32 && g_type != EF_GRAD_BF16) return EF_ERR_INVALID_ARG;
  const bool bf16 = g_type == EF_GRAD_BF16;
  const size_t gsz = bf16 ? 2 : 4;
  if (!std::isfinite(gamma) || scale_log2 < -100 || scale_log2 > 100) return EF_ERR_INVALID_ARG;
  if (d > kMaxD || !unsent_out || !aligned(unsent_out, 4)) return EF_ERR_INVALID_ARG;
  if (err_sq_out && !aligned(err_sq_out, 8)) return EF_ERR_INVALID_ARG;
  if (d == 0) {
    if (cudaMemsetAsync(unsent_out, 0, sizeof(uint32_t), s) != cudaSuccess) return EF_ERR_CUDA;
    return write_err_zero(err_sq_out, s);
  }
  if (!g || !e || !q_out || !aligned(g, gsz) || !aligned(e, 4) || !aligned(q_out, 4))
    return EF_ERR_INVALID_ARG;
  const size_t nb = static_cast<size_t>(d) * 4;
  if (overlaps(g, d * gsz, e, nb) || overlaps(q_out, nb, g, d * gsz) || overlaps(q_out, nb, e, nb) ||
      overlaps(unsent_out, 4, g, d * gsz) || overlaps(unsent_out, 4, e, nb) ||
      overlaps(unsent_out, 4, q_out, nb))
    return EF_ERR_INVALID_ARG;
  if (err_sq_out && (overlaps(err_sq_out, 8, g, d * gsz) || overlaps(err_sq_out, 8, e, nb) ||
                     overlaps(err_sq_out, 8, q_out, nb) || overlaps(err_sq_out, 8, unsent_out, 4)))
    return EF_ERR_INVALID_ARG;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  DeviceInfo info;
  ef_status st = device_info(dev, &info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_workspace(s, 0, 0, 0, 0, &ws);
  if (st != EF_OK) return st;
  return finish_launch(launch_scaled_round(g, bf16, e, gamma, scale_log2,
                                           static_cast<uint32_t>(d), q_out, unsent_out,
                                           err_sq_out, *ws, info),
                       ws);
}

ef_status int_aggregate(uint32_t n, const int32_t* const* q, uint64_t d, int32_t scale_log2,
                        float* dense_out, ef_stream_t stream) {
  using namespace efs;
  if (n == 0 || n > kMaxWorkers || !q) return EF_ERR_INVALID_ARG;
  if (d > kMaxD || scale_log2 < -100 || scale_log2 > 100) return EF_ERR_INVALID_ARG;
  if (d == 0) return EF_OK;
  if (!dense_out || !aligned(dense_out, 4)) return EF_ERR_INVALID_ARG;
  for (uint32_t i = 0; i < n; ++i) {
    if (!q[i] || !aligned(q[i], 4)) return EF_ERR_INVALID_ARG;
    if (overlaps(q[i], static_cast<size_t>(d) * 4, dense_out, static_cast<size_t>(d) * 4))
      return EF_ERR_INVALID_ARG;
  }
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  DeviceInfo info;
  ef_status st = device_info(dev, &info);
  if (st != EF_OK) return st;
  Workspace* ws = nullptr;
  st = acquire_workspace(s, 0, 0, 0, 0, &ws);
  if (st != EF_OK) return st;
  return finish_launch(
      launch_int_aggregate(n, q, static_cast<uint32_t>(d), scale_log2, dense_out, *ws), ws);
}

ef_status ef_vocab_loss(const uint16_t* h, uint64_t ldh, const uint16_t* w, uint64_t ldw,
                        const uint16_t* bias, const int64_t* target, uint64_t n, uint64_t v,
                        uint64_t d, float* loss_out, float* lse_out, ef_stream_t stream) {
  efs::VocabCall c = {};
  c.h = h;
  c.w = w;
  c.bias = bias;
  c.target = target;
  c.ldh = ldh;
  c.ldw = ldw;
  c.loss = loss_out;
  c.lse = lse_out;
  try {
    return efs::vocab_entry(c, n, v, d, false, reinterpret_cast<cudaStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return EF_ERR_NO_MEMORY;
  }
}

ef_status ef_vocab_loss_grad(const uint16_t* h, uint64_t ldh, const uint16_t* w, uint64_t ldw,
                             const uint16_t* bias, const int64_t* target, const float* lse,
                             const float* row_scale, uint64_t n, uint64_t v, uint64_t d,
                             uint16_t* dh_out, uint64_t lddh, uint16_t* dw_out, uint64_t lddw,
                             uint16_t* dbias_out, ef_stream_t stream) {
  efs::VocabCall c = {};
  c.h = h;
  c.w = w;
  c.bias = bias;
  c.target = target;
  c.ldh = ldh;
  c.ldw = ldw;
  c.lse = const_cast<float*>(lse);
  c.row_scale = row_scale;
  c.dh = dh_out;
  c.lddh = lddh;
  c.dw = dw_out;
  c.lddw = lddw;
  c.dbias = dbias_out;
  try {
    return efs::vocab_entry(c, n, v, d, true, reinterpret_cast<cudaStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return EF_ERR_NO_MEMORY;
  }
}

ef_status ef_orthogonalize(uint32_t n_mat, const uint64_t* rows, const uint64_t* cols,
                           const void* const* u, const uint64_t* ld_u, ef_grad_type u_type,
                           float* const* m, const uint64_t* ld_m, float momentum,
                           uint16_t* const* out, const uint64_t* ld_out, ef_stream_t stream) {
  if (u_type != EF_GRAD_F32 && u_type != EF_GRAD_BF16) return EF_ERR_INVALID_ARG;
  try {
    return efs::orthogonalize_entry(n_mat, rows, cols, u, ld_u, u_type == EF_GRAD_BF16, m, ld_m,
                                    momentum, out, ld_out, reinterpret_cast<cudaStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return EF_ERR_NO_MEMORY;
  }
}

ef_status ef_embed(const void* table, uint64_t ld_table, ef_grad_type table_type,
                   const int64_t* token, uint64_t n, uint64_t v, uint64_t d, float scale, void* out,
                   uint64_t ld_out, ef_grad_type out_type, ef_stream_t stream) {
  return efs::guarded([&] {
    return efs::embed_entry(table, ld_table, table_type, token, n, v, d, scale, out, ld_out,
                            out_type, reinterpret_cast<cudaStream_t>(stream));
  });
}

ef_status ef_embed_grad(const void* dout, uint64_t ld_dout, ef_grad_type dout_type,
                        const int64_t* token, uint64_t n, uint64_t v, uint64_t d, float scale,
                        int accumulate, void* dtable_out, uint64_t ld_dtable,
                        ef_grad_type dtable_type, ef_stream_t stream) {
  return efs::guarded([&] {
    return efs::embed_grad_entry(dout, ld_dout, dout_type, token, n, v, d, scale, accumulate,
                                 dtable_out, ld_dtable, dtable_type,
                                 reinterpret_cast<cudaStream_t>(stream));
  });
}

ef_status ef_layer_norm(const void* x, uint64_t ldx, ef_grad_type x_type, const void* weight,
                        const void* bias, ef_grad_type w_type, float eps, uint64_t n, uint64_t d,
                        void* y_out, uint64_t ldy, ef_grad_type y_type, float* mean_out,
                        float* rstd_out, ef_stream_t stream) {
  return efs::guarded([&] {
    return efs::layer_norm_entry(x, ldx, x_type, weight, bias, w_type, eps, n, d, y_out, ldy,
                                 y_type, mean_out, rstd_out, reinterpret_cast<cudaStream_t>(stream));
  });
}

ef_status ef_layer_norm_grad(const void* x, uint64_t ldx, ef_grad_type x_type, const void* weight,
                             ef_grad_type w_type, const float* mean, const float* rstd,
                             const void* dy, uint64_t lddy, ef_grad_type dy_type, uint64_t n,
                             uint64_t d, void* dx_out, uint64_t lddx, void* dweight_out,
                             void* dbias_out, ef_stream_t stream) {
  return efs::guarded([&] {
    return efs::layer_norm_grad_entry(x, ldx, x_type, weight, w_type, mean, rstd, dy, lddy, dy_type,
                                      n, d, dx_out, lddx, dweight_out, dbias_out,
                                      reinterpret_cast<cudaStream_t>(stream));
  });
}

ef_status ef_adamw(uint32_t n_tensors, const uint64_t* numel, float* const* p,
                   const void* const* g, ef_grad_type g_type, void* const* m, void* const* v,
                   uint8_t* const* m_exponents, uint8_t* const* v_exponents,
                   uint16_t* const* copies, double lr, double beta1, double beta2, double eps,
                   double weight_decay, uint64_t step, uint64_t seed, const float* lr_dev,
                   const int64_t* step_dev, const float* grad_scale, ef_stream_t stream) {
  efs::AdamCall c = {};
  c.lr = lr;
  c.b1 = beta1;
  c.b2 = beta2;
  c.eps = eps;
  c.decay = weight_decay;
  c.step = step;
  c.seed = seed;
  c.lr_dev = lr_dev;
  c.step_dev = step_dev;
  c.grad_scale = grad_scale;
  return efs::guarded([&] {
    return efs::adamw_entry(n_tensors, numel, p, g, g_type, m, v, m_exponents, v_exponents, copies,
                            c, reinterpret_cast<cudaStream_t>(stream));
  });
}

ef_status ef_adamw_states(uint32_t n_tensors, const uint64_t* numel, const uint8_t* const* m,
                          const uint8_t* const* v, const uint8_t* const* m_exponents,
                          const uint8_t* const* v_exponents, void* const* m_out,
                          void* const* v_out, ef_grad_type out_type, ef_stream_t stream) {
  return efs::guarded([&] {
    return efs::adamw_states_entry(n_tensors, numel, m, v, m_exponents, v_exponents, m_out, v_out,
                                   out_type, reinterpret_cast<cudaStream_t>(stream));
  });
}

ef_status ef_check_status(ef_stream_t stream) {
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (cudaStreamSynchronize(s) != cudaSuccess) return EF_ERR_CUDA;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  Workspace* ws = nullptr;
  {
    std::lock_guard<std::mutex> lk(efs::g_mu);
    auto it = efs::g_workspaces.find(std::make_pair(dev, s));
    if (it == efs::g_workspaces.end() || !it->second->base) return EF_OK;
    ws = it->second;
  }
  uint32_t bits = 0;
  auto take_bits = [&](char* base) {  // of a workspace's header, which is cleared
    uint32_t* word = reinterpret_cast<uint32_t*>(base + efs::kOffError);
    uint32_t x = 0;
    if (cudaMemcpyAsync(&x, word, sizeof x, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
        cudaStreamSynchronize(s) != cudaSuccess)
      return false;
    bits |= x;
    return x == 0 || (cudaMemsetAsync(word, 0, sizeof x, s) == cudaSuccess &&
                      cudaStreamSynchronize(s) == cudaSuccess);
  };
  if (!take_bits(ws->base)) return EF_ERR_CUDA;
  for (char* base : ws->old_bases)  // those that replays of graphs write
    if (!take_bits(base)) return EF_ERR_CUDA;
  if (bits == 0) return EF_OK;
  // replays clear nothing themselves: counters that a wait left mid-way start again
  for (char* base : ws->old_model_bases)
    if (cudaMemsetAsync(base, 0, efs::kModelArrivalBytes, s) != cudaSuccess) return EF_ERR_CUDA;
  if (ws->model_base &&
      cudaMemsetAsync(ws->model_base, 0, efs::kModelArrivalBytes, s) != cudaSuccess)
    return EF_ERR_CUDA;
  if (cudaStreamSynchronize(s) != cudaSuccess) return EF_ERR_CUDA;
  {
    // a wait that ran out, or a selection that stopped early, may leave
    // barrier counters or histograms mid-way: re-clear the workspace before
    // the next launch on this stream
    std::lock_guard<std::mutex> lk(efs::g_mu);
    ws->dirty = true;
  }
  return (bits & efs::kDevErrTimeout) ? EF_ERR_TIMEOUT : EF_ERR_BAD_INPUT;
}

const char* ef_status_string(ef_status status) {
  switch (status) {
    case EF_OK: return "EF_OK";
    case EF_ERR_INVALID_ARG: return "EF_ERR_INVALID_ARG";
    case EF_ERR_CUDA: return "EF_ERR_CUDA";
    case EF_ERR_TIMEOUT: return "EF_ERR_TIMEOUT";
    case EF_ERR_BAD_INPUT: return "EF_ERR_BAD_INPUT";
    case EF_ERR_NO_MEMORY: return "EF_ERR_NO_MEMORY";
  }
  return "EF_ERR_UNKNOWN";
}

ef_status ef_workspace_release(void) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
  if (cudaDeviceSynchronize() != cudaSuccess) return EF_ERR_CUDA;
  std::lock_guard<std::mutex> lk(efs::g_mu);
  for (auto it = efs::g_workspaces.begin(); it != efs::g_workspaces.end();) {
    if (it->first.first == dev) {
      if (it->second->base) cudaFree(it->second->base);
      if (it->second->model_base) cudaFree(it->second->model_base);
      for (char* old : it->second->old_bases) cudaFree(old);
      for (char* old : it->second->old_model_bases) cudaFree(old);
      if (it->second->density_host) cudaFreeHost(it->second->density_host);
      if (it->second->lw) {
        if (it->second->lw->dev) cudaFree(it->second->lw->dev);
        delete it->second->lw;
      }
      delete it->second;
      it = efs::g_workspaces.erase(it);
    } else {
      ++it;
    }
  }
  return EF_OK;
}

uint64_t ef_kernel_launches(void) { return efs::g_launches.load(); }

void ef_test_set_lookback_fault(int64_t withheld_tile, uint32_t spin_limit_us) {
  efs::g_withheld_tile.store(withheld_tile < 0 ? -1 : withheld_tile);
  efs::g_wait_limit_ns.store(withheld_tile < 0 ? 2000000000ull
                                               : static_cast<uint64_t>(spin_limit_us) * 1000ull);
}

void ef_test_set_stream_kernel(int mode) {
  efs::g_stream_kernel_mode.store(mode >= 1 && mode <= 3 ? mode : 0);
}

}  // extern "C"
