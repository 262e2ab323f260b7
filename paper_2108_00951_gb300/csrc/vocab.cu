// vocab.cu — softmax cross entropy of hidden states against a vocabulary,
// with its gradient, without the logits in memory.
//
//   z = h w^T + b,  lse_n = log sum_v exp z_nv,  loss_n = lse_n - z_n,t(n),
//   G_nv = r_n (exp(z_nv - lse_n) - [v = t(n)]),
//   dh = G w,  dw = G^T h,  db = sum_n G_n.
//
// Rows with a negative target take no part: the rows that do are gathered
// first (compaction, as everywhere in this library), so a batch of which a
// share carries no loss costs that share less, and nothing in a skipped row
// of h, not even a NaN, reaches a result.
//
// Loss: one product whose epilogue keeps, per row and tile of the vocabulary,
// the largest logit and the sum of exponentials below it; a row's pairs are
// then joined in order. Gradient: the vocabulary is taken in pieces; a piece's
// G is formed in a product's epilogue (logits again, then exp), rounded to
// bf16 as the tensor cores' operand (relative 2^-9, the outputs' own
// rounding), and used twice: dw's rows of that piece are final, dh adds up over
// the pieces in fp32. Products read h, w and G as they lie: K-major or
// MN-major, nothing is transposed.
#include <cstddef>

#include "product.cuh"

namespace efs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Rows that carry a loss, in their order: row_map[i], targets[i] (int32), and
// their number. One CTA: the targets are 8 bytes a row, against 2 v d
// operations. A target >= v is malformed input: latched, the row skipped.
constexpr int kRowsThreads = 1024;
__global__ void __launch_bounds__(kRowsThreads, 1)
    vocab_rows_kernel(const int64_t* __restrict__ target, uint32_t n, uint32_t v,
                      uint32_t* __restrict__ row_map, int32_t* __restrict__ targets,
                      uint32_t* __restrict__ count, float* loss, float* lse, uint32_t* error) {
  __shared__ uint32_t s_warp[32];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t base = 0;
  bool bad = false;
  griddep_wait();
  for (uint32_t n0 = 0; n0 < n; n0 += kRowsThreads) {
    const uint32_t i = n0 + threadIdx.x;
    const int64_t t = i < n ? target[i] : -1;
    const bool keep = t >= 0 && t < static_cast<int64_t>(v);
    bad |= t >= static_cast<int64_t>(v);
    const uint32_t ballot = __ballot_sync(0xffffffffu, keep);
    if (lane == 0) s_warp[warp] = __popc(ballot);
    __syncthreads();
    uint32_t before = base + __popc(ballot & lanemask_lt());
    uint32_t total = 0;
    for (uint32_t w = 0; w < 32; ++w) {
      const uint32_t c = s_warp[w];
      before += w < warp ? c : 0u;
      total += c;
    }
    if (keep) {
      row_map[before] = i;
      targets[before] = static_cast<int32_t>(t);
    } else if (i < n && loss) {
      loss[i] = 0.0f;
      lse[i] = 0.0f;
    }
    base += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) *count = base;
  if (bad) atomicOr(error, kDevErrBadInput);
}

// Copies rows of 16-bit elements to rows that TMA can read: dst[i] =
// src[row_map[i]] (or src[i]), zeros past `cols`, past *count and up to
// `rows_out`; with `one` the element after the last is 1.0 (bf16). zero_rows
// (optional): rows whose target is skipped are zeroed there.
__global__ void __launch_bounds__(256)
    vocab_pack_kernel(const uint16_t* __restrict__ src, uint64_t ld, uint32_t cols, uint32_t rows,
                      const uint32_t* __restrict__ row_map, const uint32_t* __restrict__ count,
                      uint16_t* __restrict__ dst, uint32_t ld_out, uint32_t rows_out, bool one,
                      uint16_t* zero_rows, uint64_t zero_ld, const int64_t* __restrict__ target,
                      uint32_t v) {
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t warps = static_cast<uint64_t>(gridDim.x) * 8;
  const bool vec = reinterpret_cast<uintptr_t>(src) % 16 == 0 && ld % 8 == 0;
  griddep_wait();
  const uint32_t have = count ? *count : rows;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5); i < rows_out;
       i += warps) {
    const bool real = i < have;
    const uint16_t* from = src + (real ? (row_map ? row_map[i] : i) : 0) * ld;
    uint16_t* to = dst + i * ld_out;
    for (uint32_t c = lane * 8; c < ld_out; c += 256) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (real && vec && c + 8 <= cols) {
        x = __ldg(reinterpret_cast<const uint4*>(from + c));
      } else if (real) {
        uint32_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          e[j] = c + j < cols ? __ldg(from + c + j) : (one && c + j == cols) ? 0x3f80u : 0u;
        x = make_uint4(e[0] | (e[1] << 16), e[2] | (e[3] << 16), e[4] | (e[5] << 16),
                       e[6] | (e[7] << 16));
      }
      *reinterpret_cast<uint4*>(to + c) = x;
    }
    if (zero_rows && i < rows) {
      const int64_t t = target[i];
      if (t < 0 || t >= static_cast<int64_t>(v))
        for (uint32_t c = lane; c < cols; c += 32) zero_rows[i * zero_ld + c] = 0;
    }
  }
}

// 32 logits of a row: accumulators plus the bias of their columns (through
// the warp's 32 floats of shared memory), -inf past the vocabulary.
__device__ __forceinline__ void add_bias(float (&v)[32], const uint16_t* bias, uint32_t col0,
                                         uint32_t n, float* s_bias) {
  if (bias) {
    const uint32_t lane = threadIdx.x & 31;
    __syncwarp();
    s_bias[lane] = col0 + lane < n ? bf16_bits_to_f32(__ldg(bias + col0 + lane)) : 0.0f;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float4 b = reinterpret_cast<const float4*>(s_bias)[j];
      v[4 * j] = __fadd_rn(v[4 * j], b.x);
      v[4 * j + 1] = __fadd_rn(v[4 * j + 1], b.y);
      v[4 * j + 2] = __fadd_rn(v[4 * j + 2], b.z);
      v[4 * j + 3] = __fadd_rn(v[4 * j + 3], b.w);
    }
  }
}

// Epilogue of the loss: (max, sum of exp(z - max)) of the row over the tile's
// columns, and the target's logit from the tile that holds it.
struct LossEpilogue {
  struct Params {
    const uint16_t* bias;
    const int32_t* targets;
    const uint32_t* count;
    float2* pairs;     // [row][tile]
    float* at_target;  // [row]
  };
  struct Smem {
    alignas(16) float bias[4][32];
  };
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, Smem& s,
                                              const ProductAcc& acc) {
    const uint32_t r = it.m0 + row;
    const bool real = r < *e.count;
    const int32_t target = real ? e.targets[r] : -1;
    float m = -INFINITY, sum = 0.0f;
    for (uint32_t c = 0; c < acc.chunks; ++c) {
      float v[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      add_bias(v, e.bias, col0, p.n, s.bias[(threadIdx.x >> 5) & 3u]);
      if (col0 + 32 > p.n) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = col0 + j < p.n ? v[j] : -INFINITY;
      }
      const uint32_t at = static_cast<uint32_t>(target) - col0;
      if (target >= 0 && at < 32u) {
        float z = 0.0f;
#pragma unroll
        for (int j = 0; j < 32; ++j) z = at == static_cast<uint32_t>(j) ? v[j] : z;
        e.at_target[r] = z;
      }
      float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
      for (int j = 4; j < 32; ++j) top[j & 3] = fmaxf(top[j & 3], v[j]);
      const float higher = fmaxf(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), m);
      const float shift = higher == -INFINITY ? 0.0f : __fmul_rn(higher, -kLog2e);
      float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 32; ++j)
        part[j & 3] = __fadd_rn(part[j & 3], exp2_fast(__fmaf_rn(v[j], kLog2e, shift)));
      const float rest = __fadd_rn(__fadd_rn(part[0], part[1]), __fadd_rn(part[2], part[3]));
      // m == higher also covers both -inf (nothing summed so far)
      const float scale = m == higher ? 1.0f : exp2_fast(__fmaf_rn(m, kLog2e, shift));
      sum = __fmaf_rn(sum, scale, rest);
      m = higher;
    }
    if (real) e.pairs[static_cast<uint64_t>(r) * p.tiles_n + it.tn] = make_float2(m, sum);
  }
};

// One warp per row: its tiles' pairs joined in a fixed order.
__global__ void __launch_bounds__(256)
    vocab_join_kernel(const float2* __restrict__ pairs, uint32_t tiles,
                      const float* __restrict__ at_target, const uint32_t* __restrict__ row_map,
                      const uint32_t* __restrict__ count, float* __restrict__ loss,
                      float* __restrict__ lse) {
  const uint32_t lane = threadIdx.x & 31;
  griddep_wait();
  const uint32_t r = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= *count) return;
  const float2* mine = pairs + static_cast<uint64_t>(r) * tiles;
  float m = -INFINITY;
  bool nan = false;
  for (uint32_t t = lane; t < tiles; t += 32) {
    const float2 x = __ldg(mine + t);
    m = fmaxf(m, x.x);
    nan |= x.y != x.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float sum = 0.0f;
  for (uint32_t t = lane; t < tiles; t += 32) {
    const float2 x = __ldg(mine + t);
    if (x.x > -INFINITY)
      sum = __fmaf_rn(x.y, x.x == m ? 1.0f : exp2_fast(__fmul_rn(__fsub_rn(x.x, m), kLog2e)), sum);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
  nan = __any_sync(0xffffffffu, nan);
  if (lane == 0) {
    float total = m == -INFINITY ? -INFINITY : __fadd_rn(m, logf(sum));
    if (nan) total = __int_as_float(0x7fffffff);
    const float z = at_target[r];
    lse[row_map[r]] = total;
    // a target that a bias of -inf rules out has probability 0: loss +inf
    loss[row_map[r]] = z == -INFINITY && !nan ? INFINITY : __fsub_rn(total, z);
  }
}

// Epilogue of the gradient's logits: G in bf16, one piece of the vocabulary.
struct GradEpilogue {
  struct Params {
    const uint16_t* bias;      // of the piece
    const int32_t* targets;
    const uint32_t* row_map;
    const uint32_t* count;
    const float* lse;          // by original row
    const float* row_scale;    // by original row
    uint16_t* g;               // [row][ld_g]
    uint32_t ld_g;
    uint32_t v0;               // the piece's first word
  };
  struct Smem {
    alignas(16) float bias[4][32];
  };
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, Smem& s,
                                              const ProductAcc& acc) {
    const uint32_t r = it.m0 + row;
    const bool real = r < *e.count;
    float scale = 0.0f, shift = 0.0f;
    uint32_t target = 0xffffffffu;
    bool dead = true;
    if (real) {
      const uint32_t src = e.row_map[r];
      const float lse = e.lse[src];
      scale = e.row_scale[src];
      shift = __fmul_rn(lse, -kLog2e);
      target = static_cast<uint32_t>(e.targets[r]) - e.v0;
      dead = lse == -INFINITY;  // no word has a probability
    }
    uint16_t* out = e.g + static_cast<uint64_t>(r) * e.ld_g + it.n0;
    for (uint32_t c = 0; c < acc.chunks; ++c) {
      float v[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      add_bias(v, e.bias, col0, p.n, s.bias[(threadIdx.x >> 5) & 3u]);
#pragma unroll
      for (int j = 0; j < 32; ++j)
        v[j] = __fmul_rn(exp2_fast(__fmaf_rn(v[j], kLog2e, shift)), scale);
      const uint32_t at = target - col0;
      if (at < 32u) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          v[j] = at == static_cast<uint32_t>(j) ? __fsub_rn(v[j], scale) : v[j];
      }
      if (dead) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = 0.0f;
      }
      // columns past the piece lie past the tensor map's extent: never read
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4*>(out + c * 32 + 8 * j) =
            make_uint4(pack_bf16(v[8 * j], v[8 * j + 1]), pack_bf16(v[8 * j + 2], v[8 * j + 3]),
                       pack_bf16(v[8 * j + 4], v[8 * j + 5]), pack_bf16(v[8 * j + 6], v[8 * j + 7]));
    }
  }
};

// Epilogue of dh and dw: rows of bf16 at any alignment, optionally through an
// fp32 sum over pieces, optionally one more column that goes elsewhere (db).
struct StoreEpilogue {
  struct Params {
    uint16_t* out;
    uint64_t ld;
    const uint32_t* row_map;  // or nullptr
    const uint32_t* count;    // rows that exist (with row_map)
    uint32_t rows, cols;
    uint16_t* extra;          // column `cols`, by row (or nullptr)
    float* sum;               // [row][ld_sum] (or nullptr)
    uint32_t ld_sum;
    uint32_t first, last;     // of the pieces
    uint32_t vec;             // rows start at 16-byte boundaries
  };
  struct Smem {
    uint32_t turn[4][32 * 17];
  };
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, Smem& s,
                                              const ProductAcc& acc) {
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t r = it.m0 + row;
    const bool real = r < (e.row_map ? *e.count : e.rows);
    const uint32_t dst = real ? (e.row_map ? e.row_map[r] : r) : 0xffffffffu;
    uint32_t* turn = s.turn[(threadIdx.x >> 5) & 3u];
    for (uint32_t c = 0; c < acc.chunks; ++c) {
      float v[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      if (e.sum) {
        float4* sum = reinterpret_cast<float4*>(e.sum + static_cast<uint64_t>(r) * e.ld_sum + col0);
        if (!e.first) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float4 x = __ldcg(sum + j);
            v[4 * j] = __fadd_rn(x.x, v[4 * j]);
            v[4 * j + 1] = __fadd_rn(x.y, v[4 * j + 1]);
            v[4 * j + 2] = __fadd_rn(x.z, v[4 * j + 2]);
            v[4 * j + 3] = __fadd_rn(x.w, v[4 * j + 3]);
          }
        }
        if (!e.last) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            __stcg(sum + j, make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
          continue;
        }
      }
      if (e.extra && real && e.cols - col0 < 32u) {
        float x = 0.0f;
#pragma unroll
        for (int j = 0; j < 32; ++j) x = e.cols - col0 == static_cast<uint32_t>(j) ? v[j] : x;
        e.extra[dst] = static_cast<uint16_t>(pack_bf16(x, 0.0f));
      }
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
      if (e.vec && col0 + 32 <= e.cols) {
        if (real) {
          uint4* to = reinterpret_cast<uint4*>(e.out + static_cast<uint64_t>(dst) * e.ld + col0);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            to[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
        }
        continue;
      }
      // through shared memory: a row's 32 columns are one store of the warp
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 16; ++j) turn[lane * 17 + j] = w[j];
      __syncwarp();
      const bool in = col0 + lane < e.cols;
      for (uint32_t i = 0; i < 32; ++i) {
        const uint32_t to = __shfl_sync(0xffffffffu, dst, i);
        if (to != 0xffffffffu && in)
          e.out[static_cast<uint64_t>(to) * e.ld + col0 + lane] =
              reinterpret_cast<const uint16_t*>(turn + i * 17)[lane];
      }
    }
  }
};

constexpr uint32_t round_up(uint32_t x, uint32_t to) { return (x + to - 1) / to * to; }
constexpr size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// Words per piece of the gradient's vocabulary: G stays within 1 GB (a piece
// has to be wide enough to fill the GPU twice, and its G, though larger than
// L2, costs less traffic than its products take), in whole tiles.
constexpr uint64_t kPieceBytes = 1ull << 30;
uint32_t piece_words(uint32_t rows, uint32_t v) {
  uint64_t words = kPieceBytes / (2ull * rows) / kTileNMax * kTileNMax;
  if (words < 8 * kTileNMax) words = 8 * kTileNMax;
  if (words >= v) return v;
  const uint64_t pieces = (v + words - 1) / words;  // of equal size
  return round_up(static_cast<uint32_t>((v + pieces - 1) / pieces), kTileNMax);
}

struct VocabLayout {
  uint32_t rows;    // rows of the gathered h: n rounded up to whole tiles
  uint32_t ld_h, ld_w, ld_g, piece, ld_sum;
  size_t row_map, targets, count, h, w, pairs, at_target, g, sum, parts, total;
  uint32_t pair_tiles;
};

VocabLayout vocab_layout(const VocabCall& c, bool gradient, size_t part_bytes,
                         uint32_t pair_tiles) {
  VocabLayout l = {};
  l.rows = round_up(c.n ? c.n : 1, kTileM);
  l.ld_h = round_up(c.d + (c.dbias ? 1 : 0), 8);
  l.ld_w = round_up(c.d, 8);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  l.row_map = take(4ull * l.rows);
  l.targets = take(4ull * l.rows);
  l.count = take(4);
  l.h = take(2ull * l.rows * l.ld_h);
  if (!tma_rows(c.w, c.ldw)) l.w = take(2ull * c.v * l.ld_w);
  if (gradient) {
    l.piece = piece_words(l.rows, c.v);
    l.ld_g = round_up(l.piece, kTileNMax);  // epilogues write whole tiles
    l.g = take(2ull * l.rows * l.ld_g);
    if (l.piece < c.v) {
      l.ld_sum = round_up(c.d, kTileNMax);
      l.sum = take(4ull * l.rows * l.ld_sum);
    }
  } else {
    l.pair_tiles = pair_tiles;
    l.pairs = take(8ull * l.rows * pair_tiles);
    l.at_target = take(4ull * l.rows);
  }
  l.parts = take(part_bytes);
  l.total = at;
  return l;
}

// The three products' plans. dh has few tiles and the whole piece as its K
// axis, dw the rows: both are cut along K where tiles are few.
struct VocabPlans {
  ProductShape logits, dh, dw;
  size_t part_bytes;
};
VocabPlans vocab_plans(const VocabCall& c, bool gradient, uint32_t words, const DeviceInfo& dev) {
  VocabPlans p = {};
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count), n = c.n ? c.n : 1;
  plan_product(p.logits, n, words, c.d, 1, false, sms, 1);
  if (gradient) {
    plan_product(p.dh, n, c.d, words, 1, false, sms, 32);
    plan_product(p.dw, words, c.d + (c.dbias ? 1 : 0), n, 1, false, sms, 8);
    // both run in one launch: scratch tiles of one size
    const uint32_t chunks = round_up(p.dh.bn > p.dw.bn ? p.dh.bn : p.dw.bn, 32) / 32;
    const size_t tiles = (p.dh.splits > 1 ? p.dh.tiles * p.dh.splits : 0) +
                         (p.dw.splits > 1 ? p.dw.tiles * p.dw.splits : 0);
    p.part_bytes = 4ull * kTileM * 32 * chunks * tiles;
  }
  return p;
}

cudaError_t launch_kernel(const void* fn, uint32_t grid, uint32_t block, cudaStream_t stream,
                          void** params) {
  const cudaError_t e = launch_pdl(fn, dim3(grid), block, 0, stream, params, false);
  if (e == cudaSuccess) count_launch();
  return e;
}

struct Gathered {
  const uint16_t* w;
  uint64_t ld_w;
};

// The rows that take part, h gathered, w copied where TMA cannot read it.
cudaError_t gather(const VocabCall& c, const VocabLayout& l, char* base, bool gradient,
                   Workspace& ws, const DeviceInfo& dev, Gathered* out) {
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count);
  uint32_t* row_map = reinterpret_cast<uint32_t*>(base + l.row_map);
  int32_t* targets = reinterpret_cast<int32_t*>(base + l.targets);
  uint32_t* count = reinterpret_cast<uint32_t*>(base + l.count);
  uint32_t* error = ws.u32(kOffError);
  uint32_t n = c.n, v = c.v, d = c.d;
  const int64_t* target = c.target;
  float* loss = gradient ? nullptr : c.loss;
  float* lse = c.lse;
  {
    void* params[] = {&target, &n, &v, &row_map, &targets, &count, &loss, &lse, &error};
    const cudaError_t e = launch_kernel(reinterpret_cast<const void*>(&vocab_rows_kernel), 1,
                                        kRowsThreads, ws.stream, params);
    if (e != cudaSuccess) return e;
  }
  auto pack = [&](const uint16_t* src, uint64_t ld, uint32_t rows, const uint32_t* map,
                  const uint32_t* cnt, uint16_t* dst, uint32_t ld_out, uint32_t rows_out, bool one,
                  uint16_t* zero, uint64_t zero_ld) {
    const uint32_t want = (rows_out + 7) / 8, grid = want < 8 * sms ? want : 8 * sms;
    void* params[] = {&src, &ld, &d, &rows, &map, &cnt, &dst, &ld_out, &rows_out, &one, &zero,
                      &zero_ld, &target, &v};
    return launch_kernel(reinterpret_cast<const void*>(&vocab_pack_kernel), grid, 256, ws.stream,
                         params);
  };
  cudaError_t e = pack(c.h, c.ldh, c.n, row_map, count, reinterpret_cast<uint16_t*>(base + l.h),
                       l.ld_h, l.rows, gradient && c.dbias, gradient ? c.dh : nullptr, c.lddh);
  if (e != cudaSuccess) return e;
  out->w = c.w;
  out->ld_w = c.ldw;
  if (!tma_rows(c.w, c.ldw)) {
    uint16_t* w = reinterpret_cast<uint16_t*>(base + l.w);
    e = pack(c.w, c.ldw, c.v, nullptr, nullptr, w, l.ld_w, c.v, false, nullptr, 0);
    out->w = w;
    out->ld_w = l.ld_w;
  }
  return e;
}

// Tile rows walked together: their h stays in L2 while the vocabulary passes.
uint32_t rows_in_l2(uint32_t tiles_m, uint32_t d) {
  const uint64_t tile = 2ull * kTileM * d, most = (48ull << 20) / tile;
  const uint32_t g = most < 1 ? 1 : most > tiles_m ? tiles_m : static_cast<uint32_t>(most);
  return g;
}

}  // namespace

size_t vocab_scratch(const VocabCall& c, bool gradient, const DeviceInfo& dev) {
  const uint32_t rows = round_up(c.n ? c.n : 1, kTileM);
  const VocabPlans p = vocab_plans(c, gradient, gradient ? piece_words(rows, c.v) : c.v, dev);
  return vocab_layout(c, gradient, p.part_bytes, p.logits.tiles_n).total;
}

cudaError_t launch_vocab_loss(const VocabCall& c, Workspace& ws, const DeviceInfo& dev) {
  char* base = ws.model_scratch();
  VocabPlans plan = vocab_plans(c, false, c.v, dev);
  const VocabLayout l = vocab_layout(c, false, 0, plan.logits.tiles_n);
  Gathered from;
  cudaError_t e = gather(c, l, base, false, ws, dev, &from);
  if (e != cudaSuccess) return e;
  const uint32_t* count = reinterpret_cast<const uint32_t*>(base + l.count);
  const uint16_t* h = reinterpret_cast<const uint16_t*>(base + l.h);
  ProductArgs<LossEpilogue, 1> args = {};
  ProductShape& p = args.shape[0];
  p = plan.logits;
  p.bf16 = 1;
  p.count = count;
  p.group_m = rows_in_l2(p.tiles_m, c.d);
  if (!make_map(&p.a, h, true, c.d, l.rows, l.ld_h, 1, static_cast<uint64_t>(l.rows) * l.ld_h,
                kTileM) ||
      !make_map(&p.b, from.w, true, c.d, c.v, from.ld_w, 1, from.ld_w * c.v, p.bn))
    return cudaErrorInvalidValue;
  args.epi[0] = {c.bias, reinterpret_cast<const int32_t*>(base + l.targets), count,
                 reinterpret_cast<float2*>(base + l.pairs),
                 reinterpret_cast<float*>(base + l.at_target)};
  args.problems = 1;
  e = launch_product(args, ws, dev);
  if (e != cudaSuccess) return e;
  const float2* pairs = args.epi[0].pairs;
  const float* at_target = args.epi[0].at_target;
  uint32_t tiles = p.tiles_n;
  const uint32_t* row_map = reinterpret_cast<const uint32_t*>(base + l.row_map);
  float *loss = c.loss, *lse = c.lse;
  void* params[] = {&pairs, &tiles, &at_target, &row_map, &count, &loss, &lse};
  return launch_kernel(reinterpret_cast<const void*>(&vocab_join_kernel), (l.rows + 7) / 8, 256,
                       ws.stream, params);
}

cudaError_t launch_vocab_loss_grad(const VocabCall& c, Workspace& ws, const DeviceInfo& dev) {
  char* base = ws.model_scratch();
  const uint32_t rows = round_up(c.n ? c.n : 1, kTileM);
  const uint32_t piece = piece_words(rows, c.v);
  const VocabPlans plan = vocab_plans(c, true, piece, dev);
  const VocabLayout l = vocab_layout(c, true, plan.part_bytes, 0);
  Gathered from;
  cudaError_t e = gather(c, l, base, true, ws, dev, &from);
  if (e != cudaSuccess) return e;
  const uint32_t* count = reinterpret_cast<const uint32_t*>(base + l.count);
  const uint32_t* row_map = reinterpret_cast<const uint32_t*>(base + l.row_map);
  const uint16_t* h = reinterpret_cast<const uint16_t*>(base + l.h);
  uint16_t* g = reinterpret_cast<uint16_t*>(base + l.g);
  const uint32_t dn = c.d + (c.dbias ? 1 : 0);
  const uint64_t h_all = static_cast<uint64_t>(l.rows) * l.ld_h;
  const uint64_t g_all = static_cast<uint64_t>(l.rows) * l.ld_g;
  for (uint32_t v0 = 0; v0 < c.v; v0 += piece) {
    const uint32_t words = c.v - v0 < piece ? c.v - v0 : piece;
    const uint16_t* w = from.w + static_cast<uint64_t>(v0) * from.ld_w;
    const uint64_t w_all = from.ld_w * words;
    {
      ProductArgs<GradEpilogue, 1> args = {};
      ProductShape& p = args.shape[0];
      p = plan.logits;
      p.n = words;
      p.tiles_n = (words + p.bn - 1) / p.bn;
      p.tiles = p.tiles_m * p.tiles_n;
      p.bf16 = 1;
      p.count = count;
      p.group_m = rows_in_l2(p.tiles_m, c.d);
      if (!make_map(&p.a, h, true, c.d, l.rows, l.ld_h, 1, h_all, kTileM) ||
          !make_map(&p.b, w, true, c.d, words, from.ld_w, 1, w_all, p.bn))
        return cudaErrorInvalidValue;
      args.epi[0] = {c.bias ? c.bias + v0 : nullptr,
                     reinterpret_cast<const int32_t*>(base + l.targets),
                     row_map,
                     count,
                     c.lse,
                     c.row_scale,
                     g,
                     l.ld_g,
                     v0};
      args.problems = 1;
      e = launch_product(args, ws, dev);
      if (e != cudaSuccess) return e;
    }
    ProductArgs<StoreEpilogue, 2> args = {};
    {
      ProductShape& p = args.shape[0];  // dw = G^T h
      p = plan.dw;
      p.m = words;
      p.tiles_m = (words + kTileM - 1) / kTileM;
      p.tiles = p.tiles_m * p.tiles_n;
      p.group_m = 1;
      p.a_mn = p.b_mn = p.bf16 = 1;
      p.count = count;
      p.count_is_k = 1;
      if (!make_map(&p.a, g, true, words, l.rows, l.ld_g, 1, g_all, 64) ||
          !make_map(&p.b, h, true, dn, l.rows, l.ld_h, 1, h_all, 64))
        return cudaErrorInvalidValue;
      uint16_t* out = c.dw + static_cast<uint64_t>(v0) * c.lddw;
      args.epi[0] = {out, c.lddw, nullptr, nullptr, words, c.d,
                     c.dbias ? c.dbias + v0 : nullptr, nullptr, 0, 1, 1,
                     tma_rows(out, c.lddw) ? 1u : 0u};
    }
    {
      ProductShape& p = args.shape[1];  // dh = G w
      p = plan.dh;
      p.k = words;
      p.group_m = 1;
      p.b_mn = p.bf16 = 1;
      p.count = count;
      if (!make_map(&p.a, g, true, words, l.rows, l.ld_g, 1, g_all, kTileM) ||
          !make_map(&p.b, w, true, c.d, words, from.ld_w, 1, w_all, 64))
        return cudaErrorInvalidValue;
      args.epi[1] = {c.dh, c.lddh, row_map, count, c.n, c.d, nullptr,
                     piece < c.v ? reinterpret_cast<float*>(base + l.sum) : nullptr, l.ld_sum,
                     v0 == 0 ? 1u : 0u, v0 + words == c.v ? 1u : 0u,
                     tma_rows(c.dh, c.lddh) ? 1u : 0u};
    }
    args.problems = 2;
    args.parts = reinterpret_cast<float*>(base + l.parts);
    e = launch_product(args, ws, dev);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace efs
