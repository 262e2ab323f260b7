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
// of h, not even a NaN, reaches a result. To the gradient a row whose
// log-sum-exp is -inf (no word has a probability) is such a row too: its G is 0,
// but 0 times an infinity of h or w would not be.
//
// Loss: one product whose epilogue keeps, per row and tile of the vocabulary,
// the largest logit and the sum of exponentials below it; a row's pairs are
// then joined in order. Gradient: the vocabulary is taken in pieces; a piece's
// G is formed in a product's epilogue (logits again, then exp), rounded to
// bf16 as the tensor cores' operand (relative 2^-8 at most, the outputs' own
// rounding), and used twice: dw's rows of that piece are final, dh adds up over
// the pieces in fp32. Products read h, w and G as they lie: K-major or
// MN-major, nothing is transposed. db is summed from G before it is rounded
// (its terms cancel: the rows of a frequent word's target against its
// probabilities elsewhere): over 32 rows in fp32, then in 64-bit fixed point,
// whose sums do not depend on the order of their atomics.
//
// What bounds it: the products. Each epilogue runs under the next tile's, so its
// 10 to 20 operations an entry are hidden from widths of about 2000 on (8192 x
// 128,000 x 4096: 4.9 ms, 92 % of the rate that a library product of that kind
// reaches in a burst; the board's power is at its limit), and show below (4096 x
// 50,001 x 1024: 275 us, 81 %). The gradient's three products: 8192 x 128,000 x
// 2048 7.9 ms, 86 %; 4096 x 50,001 x 1024 272 us for G and 484 for dh and dw. G
// (bf16, 2 n bytes a word) is written once and read twice, mostly from DRAM:
// 0.5 GB of traffic against 550 GFLOP at 4096 x 16,384 x 2048. Few rows (96 x
// 65,537 x 1021, 31 us) are bound by w at 5.4 TB/s and by two launches.
#include <cstddef>

#include "product.cuh"

namespace efs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// The scale of the fixed-point sums of G's columns: |G| <= |r| of its row, so a
// column's sum is at most sum |r|, which the scale (a power of two) takes to
// below 2^61.
__device__ __forceinline__ float fixed_scale(float sum) {
  if (!(sum > 0.0f) || !(sum < INFINITY)) return 1.0f;
  const int e = static_cast<int>(__float_as_uint(sum) >> 23) - 127;  // sum < 2^(e + 1)
  const int k = min(60 - e, 127);
  return __int_as_float((k + 127) << 23);
}
// Rows that carry a loss, in their order: row_map[i], targets[i] (int32), for the
// gradient soft[i] = (lse, scale), and their number. One CTA: the targets
// are 8 bytes a row, against 2 v d operations. A target >= v is malformed input:
// latched, the row skipped.
__device__ __forceinline__ bool takes_part(int64_t target, uint32_t v) {
  return target >= 0 && target < static_cast<int64_t>(v);
}
// `lse`: of the gradient's rows (nullptr in the loss call).
__device__ __forceinline__ bool takes_part(const int64_t* target, const float* lse, uint32_t i,
                                           uint32_t v) {
  const float x = lse ? lse[i] : 0.0f;
  return takes_part(__ldg(target + i), v) && x != -INFINITY;
}
constexpr int kRowsThreads = 1024;
__global__ void __launch_bounds__(kRowsThreads, 1)
    vocab_rows_kernel(const int64_t* __restrict__ target, uint32_t n, uint32_t v,
                      uint32_t* __restrict__ row_map, int32_t* __restrict__ targets,
                      uint32_t* __restrict__ count, float* loss, float* lse,
                      const float* __restrict__ row_scale, float2* __restrict__ soft,
                      float* __restrict__ fixed, uint32_t* error) {
  __shared__ uint32_t s_warp[32];
  __shared__ float s_abs[32];
  float abs_sum = 0.0f;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t base = 0;
  bool bad = false;
  griddep_wait();
  for (uint32_t n0 = 0; n0 < n; n0 += kRowsThreads) {
    const uint32_t i = n0 + threadIdx.x;
    const int64_t t = i < n ? target[i] : -1;
    const bool keep = i < n && takes_part(target, soft ? lse : nullptr, i, v);
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
      if (soft) {
        soft[before] = make_float2(lse[i], row_scale[i]);
        abs_sum = __fadd_rn(abs_sum, fabsf(row_scale[i]));
      }
    } else if (i < n && loss) {
      loss[i] = 0.0f;
      lse[i] = 0.0f;
    }
    base += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) *count = base;
  if (bad) atomicOr(error, kDevErrBadInput);
  if (fixed) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      abs_sum = __fadd_rn(abs_sum, __shfl_xor_sync(0xffffffffu, abs_sum, o));
    if (lane == 0) s_abs[warp] = abs_sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < 32; ++w) abs_sum = __fadd_rn(abs_sum, s_abs[w]);
      *fixed = fixed_scale(abs_sum);
    }
  }
}

// 8 elements of a row of `cols` from c on, zeros past its end.
__device__ __forceinline__ uint4 pack_8(const uint16_t* row, uint32_t c, uint32_t cols, bool vec) {
  if (c + 8 <= cols) {
    if (vec) return __ldg(reinterpret_cast<const uint4*>(row + c));
    if (reinterpret_cast<uintptr_t>(row) % 4 == 0) {
      const uint32_t* p = reinterpret_cast<const uint32_t*>(row + c);
      return make_uint4(__ldg(p), __ldg(p + 1), __ldg(p + 2), __ldg(p + 3));
    }
  }
  uint32_t e[8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
    e[j] = c + j < cols ? __ldg(row + c + j) : 0u;
  return make_uint4(e[0] | (e[1] << 16), e[2] | (e[3] << 16), e[4] | (e[5] << 16),
                    e[6] | (e[7] << 16));
}

// Copies rows of 16-bit elements to rows that TMA can read, a warp a row: dst[i]
// = src[row_map[i]] (or src[i]), zeros from `have` up to `rows_out`. Its rows lie
// on lines (kLine): TMA reads 128 bytes of a row at a time, which otherwise
// touch two (1230 x 50,001 x 1000 against 1024: the loss product 103 us, 86).
constexpr uint32_t kLine = 64;  // elements
struct PackArgs {
  const uint16_t* src;
  uint64_t ld;
  uint32_t cols;
  const uint32_t* row_map;
  uint16_t* dst;
  uint32_t ld_out, rows_out;
};
__device__ __forceinline__ void pack_row(const PackArgs& a, uint64_t i, uint32_t have, bool vec) {
  const uint32_t lane = threadIdx.x & 31;
  const bool real = i < have;
  const uint16_t* from = a.src + (real ? (a.row_map ? a.row_map[i] : i) : 0) * a.ld;
  uint16_t* to = a.dst + i * a.ld_out;
  for (uint32_t c = lane * 8; c < a.cols; c += 256) {
    const uint4 x = real ? pack_8(from, c, a.cols, vec) : make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(to + c) = x;
  }
}
__device__ __forceinline__ bool pack_wide(const PackArgs& a) {
  return reinterpret_cast<uintptr_t>(a.src) % 16 == 0 && a.ld % 8 == 0;
}
// zero_rows (optional): of the `rows` rows, those that take no part are zeroed
// there.
__global__ void __launch_bounds__(256)
    vocab_pack_kernel(const PackArgs a, uint32_t rows, const uint32_t* __restrict__ count,
                      uint16_t* zero_rows, uint64_t zero_ld, const int64_t* __restrict__ target,
                      const float* __restrict__ lse, uint32_t v) {
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t warps = static_cast<uint64_t>(gridDim.x) * 8;
  const bool vec = pack_wide(a);
  griddep_wait();
  const uint32_t have = count ? *count : rows;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5); i < a.rows_out;
       i += warps) {
    pack_row(a, i, have, vec);
    if (zero_rows && i < rows && !takes_part(target, lse, static_cast<uint32_t>(i), v))
      for (uint32_t c = lane; c < a.cols; c += 32) zero_rows[i * zero_ld + c] = 0;
  }
}

__device__ __forceinline__ float block_sum_8(float x, float* s8) {  // 8 warps, a fixed order
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xffffffffu, x, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s8[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.0f;
  for (int w = 0; w < 8; ++w) x = __fadd_rn(x, s8[w]);
  return x;
}
// Rows found and gathered in one launch, for batches whose targets every CTA can
// afford to count: a warp takes a row. Rows past the last gathered one are
// zeroed. CTAs past the first `ctas` copy w, where it has to be copied.
constexpr uint32_t kGatherRows = 4096;
struct GatherArgs {
  const int64_t* target;
  const uint16_t* h;
  uint64_t ld;
  uint32_t n, v, d;
  uint32_t* row_map;
  int32_t* targets;
  uint32_t* count;
  uint16_t* to;
  uint32_t ld_to, rows_to;
  float *loss, *lse;        // the loss call: zero for skipped rows
  const float* row_scale;   // the gradient's
  float2* soft;
  float* fixed;             // likewise: the scale of db's sums (or nullptr)
  uint32_t* zero;           // and those sums and their marks: 3 v words
  uint16_t* dh;             // likewise: zeroed rows
  uint64_t ld_dh;
  uint32_t* error;
  uint32_t ctas;
  PackArgs w;
};
__global__ void __launch_bounds__(256) vocab_gather_kernel(const GatherArgs a) {
  __shared__ uint32_t s_before[8], s_total[8];
  __shared__ float s_abs[8];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t first = blockIdx.x * 8, i = first + warp;
  griddep_wait();
  griddep_launch_dependents();  // the product's start needs nothing of this: 1 us less
  if (blockIdx.x >= a.ctas) {
    const bool wide = pack_wide(a.w);
    const uint64_t warps = static_cast<uint64_t>(gridDim.x - a.ctas) * 8;
    for (uint64_t r = i - a.ctas * 8; r < a.w.rows_out; r += warps)
      pack_row(a.w, r, a.w.rows_out, wide);
    return;
  }
  auto keeps = [&](uint32_t j) { return takes_part(a.target, a.soft ? a.lse : nullptr, j, a.v); };
  uint32_t before = 0, total = 0;
  bool bad = false;
#pragma unroll 4
  for (uint32_t j = threadIdx.x; j < a.n; j += 256) {
    const uint32_t k = keeps(j) ? 1u : 0u;
    bad |= __ldg(a.target + j) >= static_cast<int64_t>(a.v);
    before += j < first ? k : 0u;
    total += k;
  }
  before = warp_sum(before);
  total = warp_sum(total);
  if (lane == 0) {
    s_before[warp] = before;
    s_total[warp] = total;
  }
  __syncthreads();
  before = total = 0;
  for (int w = 0; w < 8; ++w) {
    before += s_before[w];
    total += s_total[w];
  }
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) *a.count = total;
    if (bad) atomicOr(a.error, kDevErrBadInput);
    if (a.fixed) {
      float x = 0.0f;
      for (uint32_t j = threadIdx.x; j < a.n; j += 256)
        if (keeps(j)) x = __fadd_rn(x, fabsf(a.row_scale[j]));
      x = block_sum_8(x, s_abs);
      if (threadIdx.x == 0) *a.fixed = fixed_scale(x);
    }
  }
  const bool vec = reinterpret_cast<uintptr_t>(a.h) % 16 == 0 && a.ld % 8 == 0;
  if (i < a.n) {
    const int64_t t = __ldg(a.target + i);
    // of this CTA's rows, those before this warp's
    const uint32_t mine = __ballot_sync(
        0xffffffffu, lane < warp && keeps(lane < warp ? first + lane : i));
    if (keeps(i)) {
      const uint32_t at = before + __popc(mine);
      if (lane == 0) {
        a.row_map[at] = i;
        a.targets[at] = static_cast<int32_t>(t);
        if (a.soft) a.soft[at] = make_float2(a.lse[i], a.row_scale[i]);
      }
      const uint16_t* from = a.h + i * a.ld;
      for (uint32_t c = lane * 8; c < a.d; c += 256)
        *reinterpret_cast<uint4*>(a.to + static_cast<uint64_t>(at) * a.ld_to + c) =
            pack_8(from, c, a.d, vec);
    } else {
      if (lane == 0 && a.loss) {
        a.loss[i] = 0.0f;
        a.lse[i] = 0.0f;
      }
      if (a.dh)
        for (uint32_t c = lane; c < a.d; c += 32) a.dh[i * a.ld_dh + c] = 0;
    }
  }
  if (a.fixed)
    for (uint64_t j = blockIdx.x * 256 + threadIdx.x; j < 3ull * a.v; j += a.ctas * 256) a.zero[j] = 0;
  for (uint32_t at = total + i; at < a.rows_to; at += a.ctas * 8)
    for (uint32_t c = lane * 8; c < a.d; c += 256)
      *reinterpret_cast<uint4*>(a.to + static_cast<uint64_t>(at) * a.ld_to + c) =
          make_uint4(0, 0, 0, 0);
}

// The biases of a warp's columns of a tile, at most 128, staged in its shared
// memory: loaded before the accumulators are ready.
struct BiasSmem {
  alignas(16) float bias[128];
};
__device__ __forceinline__ void stage_bias(const uint16_t* bias, uint32_t col0, uint32_t cols,
                                           uint32_t n, BiasSmem& s) {
  if (!bias) return;
  const uint32_t lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t c = i * 32 + lane;
    if (c < cols) s.bias[c] = col0 + c < n ? bf16_bits_to_f32(__ldg(bias + col0 + c)) : 0.0f;
  }
  __syncwarp();
}
// 32 logits of a row: accumulators plus the staged bias of their columns.
__device__ __forceinline__ void add_bias(float (&v)[32], const float* bias) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float4 b = reinterpret_cast<const float4*>(bias)[j];
    v[4 * j] = __fadd_rn(v[4 * j], b.x);
    v[4 * j + 1] = __fadd_rn(v[4 * j + 1], b.y);
    v[4 * j + 2] = __fadd_rn(v[4 * j + 2], b.z);
    v[4 * j + 3] = __fadd_rn(v[4 * j + 3], b.w);
  }
}

// exp(z - top) is taken as 2^(z log2e + shift), shift = -top log2e. A top beyond
// 2.35e38 (a mask of the type's lowest value on all the words looked at) takes
// that out of fp32's range: there z - top replaces z, and the shift is 0.
__device__ __forceinline__ bool out_of_range(float shift) { return fabsf(shift) == INFINITY; }
__device__ __forceinline__ void lower_by(float (&v)[32], float top) {
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = __fsub_rn(v[j], top);
}

// Epilogue of the loss: (max, sum of exp(z - max)) of the row over the tile's
// columns, and the target's logit from the tile that holds it.
struct LossEpilogue {
  static constexpr bool kTurns = false;
  struct Params {
    const uint16_t* bias;
    const int32_t* targets;
    float2* pairs;     // [row][half tile]
    float* at_target;  // [row]
    const int64_t* direct;  // != nullptr: nothing was gathered, all rows' targets
  };
  using Smem = BiasSmem;
  struct Row {
    int32_t target;
  };
  static __device__ __forceinline__ Row prepare(const ProductShape& p, const Params& e,
                                                const ProductItem& it, uint32_t row) {
    const uint32_t r = it.m0 + row;
    if (r >= it.rows) return {-1};
    if (!e.direct) return {__ldg(e.targets + r)};
    const int64_t t = __ldg(e.direct + r);
    return {t >= 0 && t < static_cast<int64_t>(p.n) ? static_cast<int32_t>(t) : -1};
  }
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row,
                                              uint32_t half, Smem& s, const ProductAcc& acc,
                                              uint32_t, Row state) {
    const uint32_t r = it.m0 + row;
    const bool real = r < it.rows;
    const int32_t target = state.target;
    float m = -INFINITY, sum = 0.0f;
    stage_bias(e.bias, it.n0 + acc.c0 * 32, (acc.c1 - acc.c0) * 32, p.n, s);
    for (uint32_t c = acc.c0; c < acc.c1; ++c) {
      float v[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      if (e.bias) add_bias(v, s.bias + (c - acc.c0) * 32);
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
      float shift = higher == -INFINITY ? 0.0f : __fmul_rn(higher, -kLog2e);
      if (out_of_range(shift)) {
        lower_by(v, higher);
        shift = 0.0f;
      }
      float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 32; ++j)
        part[j & 3] = __fadd_rn(part[j & 3], exp2_fast(__fmaf_rn(v[j], kLog2e, shift)));
      const float rest = __fadd_rn(__fadd_rn(part[0], part[1]), __fadd_rn(part[2], part[3]));
      // m == higher also covers both -inf (nothing summed so far)
      const float scale =
          m == higher ? 1.0f : exp2_fast(__fmul_rn(__fsub_rn(m, higher), kLog2e));
      sum = __fmaf_rn(sum, scale, rest);
      m = higher;
    }
    if (real)
      e.pairs[(static_cast<uint64_t>(r) * p.tiles_n + it.tn) * 2 + half] = make_float2(m, sum);
  }
};

// One warp per row: its tiles' pairs joined in a fixed order.
__global__ void __launch_bounds__(256)
    vocab_join_kernel(const float2* __restrict__ pairs, uint32_t tiles,
                      const float* __restrict__ at_target, const uint32_t* __restrict__ row_map,
                      const uint32_t* __restrict__ count, float* __restrict__ loss,
                      float* __restrict__ lse, const int64_t* __restrict__ direct, uint32_t n,
                      uint32_t v, uint32_t* error) {
  const uint32_t lane = threadIdx.x & 31;
  griddep_wait();
  const uint32_t r = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= (direct ? n : *count)) return;
  if (direct) {  // rows that take no part are here too
    const int64_t t = direct[r];
    if (t < 0 || t >= static_cast<int64_t>(v)) {
      if (lane == 0) {
        loss[r] = 0.0f;
        lse[r] = 0.0f;
        if (t >= 0) atomicOr(error, kDevErrBadInput);
      }
      return;
    }
  }
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
    const uint32_t to = direct ? r : row_map[r];
    lse[to] = total;
    // a target that a bias of -inf rules out has probability 0: loss +inf
    loss[to] = z == -INFINITY && !nan ? INFINITY : __fsub_rn(total, z);
  }
}

// The sum over the warp's rows of column `lane` of their 32: at every step half
// of the columns go to the lane that keeps them.
__device__ __forceinline__ float column_sum(const float (&v)[32]) {
  const uint32_t lane = threadIdx.x & 31;
  float x[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const bool up = lane & 16u;
    const float keep = up ? v[j + 16] : v[j], give = up ? v[j] : v[j + 16];
    x[j] = __fadd_rn(keep, __shfl_xor_sync(0xffffffffu, give, 16));
  }
#pragma unroll
  for (int w = 8; w > 0; w >>= 1) {
#pragma unroll
    for (int j = 0; j < w; ++j) {
      const bool up = lane & w;
      const float keep = up ? x[j + w] : x[j], give = up ? x[j] : x[j + w];
      x[j] = __fadd_rn(keep, __shfl_xor_sync(0xffffffffu, give, w));
    }
  }
  return x[0];
}

// Epilogue of the gradient's logits: G in bf16, one piece of the vocabulary.
struct GradEpilogue {
  static constexpr bool kTurns = false;
  struct Params {
    const uint16_t* bias;      // of the piece
    const int32_t* targets;
    const float2* soft;
    uint16_t* g;               // [row][ld_g]
    uint32_t ld_g;
    uint32_t v0;               // the piece's first word
    long long* db;             // of the piece: fixed-point sums of G's columns (or nullptr)
    uint32_t* spoilt;          // of the piece: columns whose sum is none
    const float* fixed;
  };
  struct Smem : BiasSmem {
    TurnSmem turn;
  };
  struct Row {
    float2 soft;
    uint32_t target;  // within the piece
  };
  static __device__ __forceinline__ Row prepare(const ProductShape&, const Params& e,
                                                const ProductItem& it, uint32_t row) {
    const uint32_t r = it.m0 + row;
    if (r >= it.rows) return {make_float2(0.0f, 0.0f), 0xffffffffu};
    return {__ldg(e.soft + r), static_cast<uint32_t>(__ldg(e.targets + r)) - e.v0};
  }
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, uint32_t,
                                              Smem& s, const ProductAcc& acc, uint32_t, Row state) {
    const uint32_t r = it.m0 + row, target = state.target;
    const float lse = state.soft.x, scale = state.soft.y;
    const bool far = out_of_range(__fmul_rn(lse, -kLog2e));
    const float shift = far ? 0.0f : __fmul_rn(lse, -kLog2e);
    const bool dead = scale == 0.0f;  // past the rows, or scaled by 0
    stage_bias(e.bias, it.n0 + acc.c0 * 32, (acc.c1 - acc.c0) * 32, p.n, s);
    for (uint32_t c = acc.c0; c < acc.c1; ++c) {
      float v[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      if (e.bias) add_bias(v, s.bias + (c - acc.c0) * 32);
      if (far) lower_by(v, lse);
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
      if (e.db && it.m0 + (row & ~31u) < it.rows) {
        const float x = __fmul_rn(column_sum(v), *e.fixed);
        const uint32_t col = col0 + (threadIdx.x & 31);
        if (col < p.n) {
          if (fabsf(x) < 4611686018427387904.0f)  // 2^62: an lse that is not these logits' exceeds it
            atomicAdd(reinterpret_cast<unsigned long long*>(e.db + col),
                      static_cast<unsigned long long>(__float2ll_rn(x)));
          else
            e.spoilt[col] = 1;
        }
      }
      // columns past the piece lie past the tensor map's extent: never read
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
      // in 64-byte runs: while G stays in L2, stores of one sector a row cost the
      // two products that read it 8 % (1230 x 50,001 x 1000: 354 us, not 328)
      uint16_t* out = e.g + static_cast<uint64_t>(r & ~31u) * e.ld_g + col0;
      store_block<8>(s.turn, w, 32, 16, [&](uint32_t i) { return out + i * e.ld_g; });
    }
  }
};

// Blocks of fp32 sums, 128 rows x 32 columns, four columns of all rows
// together: a warp's accesses are contiguous.
__device__ __forceinline__ float4* sum_block(float* sums, uint32_t row_tile, uint32_t chunks,
                                             uint32_t chunk, uint32_t row) {
  return reinterpret_cast<float4*>(sums) +
         (static_cast<uint64_t>(row_tile) * chunks + chunk) * (8 * kTileM) + row;
}

// Epilogue of dh and dw: rows of bf16 at any alignment; or fp32 sums, one set
// per K part, added to over the pieces of the vocabulary.
struct StoreEpilogue {
  static constexpr bool kTurns = true;
  struct Params {
    uint16_t* out;
    uint64_t ld;
    const uint32_t* row_map;  // or nullptr
    uint32_t cols;
    uint32_t align;           // of out's rows, in bytes
    float* sums;              // != nullptr: sums instead of out
    uint64_t part_floats;     // from one part's sums to the next
    uint32_t sum_chunks;      // 32-column chunks of a row
    uint32_t first;           // the sums start here
  };
  union Smem {
    TurnSmem turn;
    ShiftSmem shift;
  };
  struct Row {
    uint32_t dst;
  };
  static __device__ __forceinline__ Row prepare(const ProductShape&, const Params& e,
                                                const ProductItem& it, uint32_t row) {
    const uint32_t r = it.m0 + row;
    return {r >= it.rows ? 0xffffffffu : e.row_map ? __ldg(e.row_map + r) : r};
  }
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, uint32_t,
                                              Smem& s, const ProductAcc& acc, uint32_t, Row state) {
    const uint32_t r = it.m0 + row, dst = state.dst;
    const bool real = r < it.rows;
    uint4 carry = make_uint4(0, 0, 0, 0);
    for (uint32_t c = acc.c0; c < acc.c1; ++c) {
      float v[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      if (e.sums) {
        float4* sum = sum_block(e.sums + it.split * e.part_floats, it.m0 / kTileM, e.sum_chunks,
                                col0 / 32, row);
        if (real) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (!e.first) x = __ldcg(sum + j * kTileM);
            __stcg(sum + j * kTileM,
                   make_float4(__fadd_rn(x.x, v[4 * j]), __fadd_rn(x.y, v[4 * j + 1]),
                               __fadd_rn(x.z, v[4 * j + 2]), __fadd_rn(x.w, v[4 * j + 3])));
          }
        }
        continue;
      }
      if (col0 >= e.cols) continue;
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
      const uint32_t left = min(32u, e.cols - col0);
      if (e.align == 32 && left % 16 == 0) {
        if (real) store_row(e.out + static_cast<uint64_t>(dst) * e.ld + col0, w, left);
        continue;
      }
      const uint32_t r0 = r - (threadIdx.x & 31);
      auto to = [&](uint32_t i) -> uint16_t* {
        uint32_t at = r0 + i;
        if (e.row_map) at = __shfl_sync(0xffffffffu, dst, i);
        return r0 + i < it.rows ? e.out + static_cast<uint64_t>(at) * e.ld + col0 : nullptr;
      };
      if (e.align >= 4 && !(e.align >= 16 && left % 8 == 0))
        store_shifted(s.shift, w, carry, left, c == acc.c0, c + 1 == acc.c1 || col0 + 32 >= e.cols, to);
      else
        store_block<8>(s.turn, w, left, e.align, to);
    }
  }
};

// The gradient's last kernel. dh from its sums: parts added in order, rounded,
// rows scattered; a CTA takes 32 rows x 32 columns, a thread four columns of a
// row. CTAs past the first `ctas`: db from its fixed-point sums.
struct FinishArgs {
  uint32_t ctas;
  const float* sums;
  uint64_t part_floats;
  uint32_t parts, chunks;
  const uint32_t *row_map, *count;
  uint16_t* dh;
  uint64_t ld;
  uint32_t cols, wide;
  const long long* db_sums;
  const uint32_t* spoilt;
  const float* scale;
  uint32_t v;
  uint16_t* db;
};
__global__ void __launch_bounds__(256) vocab_finish_kernel(const FinishArgs a) {
  griddep_wait();
  if (blockIdx.x >= a.ctas) {
    const uint32_t i = (blockIdx.x - a.ctas) * 256 + threadIdx.x;
    if (i >= a.v) return;
    // (fp32 keeps 24 of the sum's bits; the division by a power of two is exact)
    const float x = a.spoilt[i] ? __int_as_float(0x7fffffff)
                                : __fdiv_rn(__ll2float_rn(a.db_sums[i]), *a.scale);
    a.db[i] = static_cast<uint16_t>(pack_bf16(x, 0.0f));
    return;
  }
  const uint32_t chunk = blockIdx.x % a.chunks, unit = threadIdx.x & 7u;
  const uint32_t r = blockIdx.x / a.chunks * 32 + (threadIdx.x >> 3), c = chunk * 32 + unit * 4;
  if (r >= *a.count || c >= a.cols) return;
  const float4* x = sum_block(const_cast<float*>(a.sums), r / kTileM, a.chunks, chunk, r % kTileM) +
                    unit * kTileM;
  uint16_t* to = a.dh + static_cast<uint64_t>(a.row_map[r]) * a.ld + c;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (uint32_t s = 0; s < a.parts; ++s) {
    const float4 y = __ldcg(x + s * (a.part_floats / 4));
    v = make_float4(__fadd_rn(v.x, y.x), __fadd_rn(v.y, y.y), __fadd_rn(v.z, y.z),
                    __fadd_rn(v.w, y.w));
  }
  const uint2 w = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  if (a.wide && c + 4 <= a.cols) {
    *reinterpret_cast<uint2*>(to) = w;
    return;
  }
  to[0] = static_cast<uint16_t>(w.x);
  if (c + 1 < a.cols) to[1] = static_cast<uint16_t>(w.x >> 16);
  if (c + 2 < a.cols) to[2] = static_cast<uint16_t>(w.y);
  if (c + 3 < a.cols) to[3] = static_cast<uint16_t>(w.y >> 16);
}

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

// Pairs of CTAs from more than one tile of 128 rows on: a pair's tile has 256
// rows, and with half of them empty it does half the work per SM.
bool use_pairs(const VocabCall& c) { return c.n > kTileM; }

// The loss of one tile row reads h as it lies where TMA can: gathering its rows
// would save nothing, and what a skipped row holds stays in that row (32 x 28,869
// x 656: 17.1 us, gathered 17.9; 96 x 65,537 x 1024: 32.1 and 37.2).
bool takes_rows(const VocabCall& c) {
  return c.n >= 1 && c.n <= 2 * kTileM && tma_rows(c.h, c.ldh) && tma_rows(c.w, c.ldw);
}

struct VocabPlan {
  uint32_t rows;    // rows of the gathered h: n rounded up to whole tiles
  uint32_t ld_h, ld_w, ld_g, piece;
  ProductShape logits, dh, dw;
  uint32_t sum_chunks, sum_parts;  // of dh's sums (0: dh is stored directly)
  uint64_t part_floats;
  // scratch offsets
  size_t row_map, targets, soft, fixed, db, count, h, w, pairs, at_target, g, sums, total;
};

// The products' plans and the scratch. dh has few tiles and the whole piece as
// its K axis: it is cut along K where tiles are few, the parts (and the
// pieces) added up in fp32 and joined by a kernel of their own.
VocabPlan vocab_plan(const VocabCall& c, bool gradient, const DeviceInfo& dev) {
  VocabPlan l = {};
  const double sms = dev.sm_count;
  const bool pair = use_pairs(c);
  const uint32_t n = c.n ? c.n : 1;
  l.rows = round_up(n, 2 * kTileM);
  l.ld_h = l.ld_w = round_up(c.d, kLine);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  if (gradient || !takes_rows(c)) {  // the gathered rows
    l.row_map = take(4ull * l.rows);
    l.targets = take(4ull * l.rows);
    l.count = take(4);
    l.h = take(2ull * l.rows * l.ld_h);
  }
  if (gradient) l.soft = take(8ull * l.rows);
  if (gradient && c.dbias) {
    l.fixed = take(4);
    l.db = take(12ull * c.v);  // sums, then marks
  }
  if (!tma_rows(c.w, c.ldw)) l.w = take(2ull * c.v * l.ld_w);
  l.piece = gradient ? piece_words(l.rows, c.v) : c.v;
  plan_product(l.logits, {n, l.piece, c.d, 1, false, pair, sms, 1, 1, 12.0, true});
  if (gradient) {
    l.ld_g = round_up(l.piece, kTileNMax);  // epilogues write whole tiles
    l.g = take(2ull * l.rows * l.ld_g);
    plan_product(l.dh, {n, c.d, l.piece, 1, false, pair, sms, 32, 1, 12.0, false});
    plan_product(l.dw, {l.piece, c.d, n, 1, false, pair, sms, 1, 1, 12.0, true});
    if (l.dh.splits > 1 || l.piece < c.v) {
      l.sum_parts = l.dh.splits;
      l.sum_chunks = round_up(c.d, 32) / 32;
      l.part_floats = static_cast<uint64_t>(l.rows) * l.sum_chunks * 32;
      l.sums = take(4ull * l.part_floats * l.sum_parts);
    }
  } else {
    l.pairs = take(16ull * l.rows * l.logits.tiles_n);
    l.at_target = take(4ull * l.rows);
  }
  l.total = at;
  return l;
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
cudaError_t gather(const VocabCall& c, const VocabPlan& l, char* base, bool gradient,
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
  const float* row_scale = c.row_scale;
  float2* soft = gradient ? reinterpret_cast<float2*>(base + l.soft) : nullptr;
  uint16_t* h = reinterpret_cast<uint16_t*>(base + l.h);
  float* fixed = gradient && c.dbias ? reinterpret_cast<float*>(base + l.fixed) : nullptr;
  auto pack = [&](PackArgs a, uint32_t rows, const uint32_t* cnt, uint16_t* zero, uint64_t zero_ld) {
    const uint32_t want = (a.rows_out + 7) / 8, grid = want < 8 * sms ? want : 8 * sms;
    void* params[] = {&a, &rows, &cnt, &zero, &zero_ld, &target, &lse, &v};
    return launch_kernel(reinterpret_cast<const void*>(&vocab_pack_kernel), grid, 256, ws.stream,
                         params);
  };
  out->w = c.w;
  out->ld_w = c.ldw;
  PackArgs copy_w = {};
  if (!tma_rows(c.w, c.ldw)) {
    copy_w = {c.w, c.ldw, d, nullptr, reinterpret_cast<uint16_t*>(base + l.w), l.ld_w, v};
    out->w = copy_w.dst;
    out->ld_w = l.ld_w;
  }
  if (n <= kGatherRows) {
    const uint32_t ctas = n ? (n + 7) / 8 : 1, rows = (v + 7) / 8;
    const uint32_t more = !copy_w.src ? 0 : rows < 8 * sms ? rows : 8 * sms;
    GatherArgs a = {target, c.h,    c.ldh, n,   v,         d,    row_map, targets,
                    count,  h,      l.ld_h, l.rows, loss,  lse,  row_scale, soft,
                    fixed,  reinterpret_cast<uint32_t*>(base + l.db), gradient ? c.dh : nullptr,
                    c.lddh, error,  ctas, copy_w};
    void* params[] = {&a};
    return launch_kernel(reinterpret_cast<const void*>(&vocab_gather_kernel), ctas + more, 256,
                         ws.stream, params);
  }
  void* params[] = {&target, &n, &v, &row_map, &targets, &count, &loss, &lse, &row_scale, &soft,
                    &fixed, &error};
  cudaError_t e = launch_kernel(reinterpret_cast<const void*>(&vocab_rows_kernel), 1, kRowsThreads,
                                ws.stream, params);
  if (e == cudaSuccess && fixed) e = cudaMemsetAsync(base + l.db, 0, 12ull * c.v, ws.stream);
  if (e == cudaSuccess)
    e = pack({c.h, c.ldh, d, row_map, h, l.ld_h, l.rows}, n, count, gradient ? c.dh : nullptr, c.lddh);
  if (e == cudaSuccess && copy_w.src) e = pack(copy_w, v, nullptr, nullptr, 0);
  return e;
}

// Tile rows walked together: their h stays in L2 while the vocabulary passes.
uint32_t rows_in_l2(const ProductShape& p, bool pair) {
  const uint64_t tile = 2ull * kTileM * (pair ? 2 : 1) * p.k, most = (48ull << 20) / tile;
  return most < 1 ? 1 : most > p.tiles_m ? p.tiles_m : static_cast<uint32_t>(most);
}

template <bool kPair>
cudaError_t loss_product(const VocabCall& c, const VocabPlan& l, const Gathered& from, char* base,
                         Workspace& ws, const DeviceInfo& dev) {
  ProductArgs<LossEpilogue, 1> args = {};
  ProductShape& p = args.shape[0];
  p = l.logits;
  p.bf16 = 1;
  const bool direct = takes_rows(c);
  if (!direct) {
    p.counts = 1;
    args.count = reinterpret_cast<const uint32_t*>(base + l.count);
  }
  p.group_m = rows_in_l2(p, kPair);
  if (!(direct ? make_map(&p.a, c.h, true, c.d, c.n, c.ldh, 1, c.ldh * c.n, kTileM)
               : make_map(&p.a, base + l.h, true, c.d, l.rows, l.ld_h, 1,
                          static_cast<uint64_t>(l.rows) * l.ld_h, kTileM)) ||
      !make_map(&p.b, from.w, true, c.d, c.v, from.ld_w, 1, from.ld_w * c.v, b_box(p, kPair)))
    return cudaErrorInvalidValue;
  args.epi[0] = {c.bias, reinterpret_cast<const int32_t*>(base + l.targets),
                 reinterpret_cast<float2*>(base + l.pairs),
                 reinterpret_cast<float*>(base + l.at_target), direct ? c.target : nullptr};
  args.phases = args.problems[0] = 1;
  number_items(args, kPair, kPartCounters);
  return launch_product<LossEpilogue, 1, kPair>(args, ws, dev);
}

// G of the words [v0, v0 + words), then dw's rows and dh's share of them.
template <bool kPair>
cudaError_t grad_piece(const VocabCall& c, const VocabPlan& l, const Gathered& from, char* base,
                       uint32_t v0, Workspace& ws, const DeviceInfo& dev) {
  const uint32_t words = c.v - v0 < l.piece ? c.v - v0 : l.piece;
  const uint32_t* count = reinterpret_cast<const uint32_t*>(base + l.count);
  const uint32_t* row_map = reinterpret_cast<const uint32_t*>(base + l.row_map);
  uint16_t* g = reinterpret_cast<uint16_t*>(base + l.g);
  const char* h = base + l.h;
  const uint16_t* w = from.w + static_cast<uint64_t>(v0) * from.ld_w;
  const uint64_t w_all = from.ld_w * words;
  const uint64_t h_all = static_cast<uint64_t>(l.rows) * l.ld_h;
  const uint64_t g_all = static_cast<uint64_t>(l.rows) * l.ld_g;
  const uint32_t tile_m = kPair ? 2 * kTileM : kTileM;
  long long* db = reinterpret_cast<long long*>(base + l.db);
  {
    ProductArgs<GradEpilogue, 1> args = {};
    ProductShape& p = args.shape[0];
    p = l.logits;
    p.n = words;
    p.tiles_n = (words + p.bn - 1) / p.bn;
    p.tiles = p.tiles_m * p.tiles_n;
    p.bf16 = 1;
    p.counts = 1;
    args.count = count;
    p.group_m = rows_in_l2(p, kPair);
    if (!make_map(&p.a, h, true, c.d, l.rows, l.ld_h, 1, h_all, kTileM) ||
        !make_map(&p.b, w, true, c.d, words, from.ld_w, 1, w_all, b_box(p, kPair)))
      return cudaErrorInvalidValue;
    args.epi[0] = {c.bias ? c.bias + v0 : nullptr,
                   reinterpret_cast<const int32_t*>(base + l.targets),
                   reinterpret_cast<const float2*>(base + l.soft), g, l.ld_g, v0,
                   c.dbias ? db + v0 : nullptr,
                   c.dbias ? reinterpret_cast<uint32_t*>(db + c.v) + v0 : nullptr,
                   reinterpret_cast<const float*>(base + l.fixed)};
    args.phases = args.problems[0] = 1;
    number_items(args, kPair, kPartCounters);
    const cudaError_t e = launch_product<GradEpilogue, 1, kPair>(args, ws, dev);
    if (e != cudaSuccess) return e;
  }
  ProductArgs<StoreEpilogue, 2> args = {};
  {
    ProductShape& p = args.shape[0];  // dh = G w: the deeper product first
    p = l.dh;
    p.k = words;
    p.group_m = 1;
    p.b_mn = p.bf16 = 1;
    p.counts = 1;
    if (!make_map(&p.a, g, true, words, l.rows, l.ld_g, 1, g_all, kTileM) ||
        !make_map(&p.b, w, true, c.d, words, from.ld_w, 1, w_all, kTileK))
      return cudaErrorInvalidValue;
    args.epi[0] = {c.dh, c.lddh, row_map, c.d, row_align(c.dh, c.lddh),
                   l.sum_parts ? reinterpret_cast<float*>(base + l.sums) : nullptr,
                   l.part_floats, l.sum_chunks, v0 == 0 ? 1u : 0u};
  }
  {
    ProductShape& p = args.shape[1];  // dw = G^T h
    p = l.dw;
    p.m = words;
    p.tiles_m = (words + tile_m - 1) / tile_m;
    p.tiles = p.tiles_m * p.tiles_n;
    p.group_m = 1;
    p.a_mn = p.b_mn = p.bf16 = 1;
    p.counts = 2;
    if (!make_map(&p.a, g, true, words, l.rows, l.ld_g, 1, g_all, kTileK) ||
        !make_map(&p.b, h, true, c.d, l.rows, l.ld_h, 1, h_all, kTileK))
      return cudaErrorInvalidValue;
    uint16_t* out = c.dw + static_cast<uint64_t>(v0) * c.lddw;
    args.epi[1] = {out, c.lddw, nullptr, c.d, row_align(out, c.lddw), nullptr, 0, 0, 1};
  }
  args.count = count;
  args.phases = 1;
  args.problems[0] = 2;
  // Of few rows dh reads and dw writes: half of the SMs begin with the one, half with
  // the other (gradient of 64 x 28,869 x 650 93 -> 80 us, 128 x 50,001 x 1024 124 ->
  // 107, 200 x 28,869 x 656 70 -> 66; 400 x 50,001 x 1024 154 both ways, 1230 x
  // 50,001 x 1000 299 -> 306).
  args.turn = c.n <= 2 * kTileM ? 1 : 0;
  number_items(args, kPair, kPartCounters);
  return launch_product<StoreEpilogue, 2, kPair>(args, ws, dev);
}

}  // namespace

size_t vocab_scratch(const VocabCall& c, bool gradient, const DeviceInfo& dev) {
  if (vocab_few(c)) return vocab_few_scratch(c, gradient, dev);
  return vocab_plan(c, gradient, dev).total;
}

cudaError_t launch_vocab_loss(const VocabCall& c, Workspace& ws, const DeviceInfo& dev) {
  if (vocab_few(c)) return launch_vocab_few_loss(c, ws, dev);
  char* base = ws.model_scratch();
  const VocabPlan l = vocab_plan(c, false, dev);
  Gathered from = {c.w, c.ldw};
  cudaError_t e = takes_rows(c) ? cudaSuccess : gather(c, l, base, false, ws, dev, &from);
  if (e != cudaSuccess) return e;
  e = use_pairs(c) ? loss_product<true>(c, l, from, base, ws, dev)
                   : loss_product<false>(c, l, from, base, ws, dev);
  if (e != cudaSuccess) return e;
  const float2* pairs = reinterpret_cast<const float2*>(base + l.pairs);
  const float* at_target = reinterpret_cast<const float*>(base + l.at_target);
  uint32_t tiles = 2 * l.logits.tiles_n;
  const uint32_t* count = reinterpret_cast<const uint32_t*>(base + l.count);
  const uint32_t* row_map = reinterpret_cast<const uint32_t*>(base + l.row_map);
  float *loss = c.loss, *lse = c.lse;
  const int64_t* direct = takes_rows(c) ? c.target : nullptr;
  uint32_t n = c.n, v = c.v, *error = ws.u32(kOffError);
  void* params[] = {&pairs, &tiles, &at_target, &row_map, &count,
                    &loss,  &lse,   &direct,    &n,       &v,     &error};
  return launch_kernel(reinterpret_cast<const void*>(&vocab_join_kernel), (c.n + 7) / 8, 256,
                       ws.stream, params);
}

cudaError_t launch_vocab_loss_grad(const VocabCall& c, Workspace& ws, const DeviceInfo& dev) {
  if (vocab_few(c)) return launch_vocab_few_grad(c, ws, dev);
  char* base = ws.model_scratch();
  const VocabPlan l = vocab_plan(c, true, dev);
  Gathered from;
  cudaError_t e = gather(c, l, base, true, ws, dev, &from);
  if (e != cudaSuccess) return e;
  for (uint32_t v0 = 0; v0 < c.v; v0 += l.piece) {
    e = use_pairs(c) ? grad_piece<true>(c, l, from, base, v0, ws, dev)
                     : grad_piece<false>(c, l, from, base, v0, ws, dev);
    if (e != cudaSuccess) return e;
  }
  FinishArgs f = {};
  uint32_t more = 0;
  if (l.sum_parts && c.n) {
    f.chunks = l.sum_chunks;
    f.ctas = (c.n + 31) / 32 * f.chunks;
    f.sums = reinterpret_cast<const float*>(base + l.sums);
    f.part_floats = l.part_floats;
    f.parts = l.sum_parts;
    f.row_map = reinterpret_cast<const uint32_t*>(base + l.row_map);
    f.count = reinterpret_cast<const uint32_t*>(base + l.count);
    f.dh = c.dh;
    f.ld = c.lddh;
    f.cols = c.d;
    f.wide = row_align(c.dh, c.lddh) >= 16 ? 1u : 0u;
  }
  if (c.dbias) {
    more = (c.v + 255) / 256;
    f.db_sums = reinterpret_cast<const long long*>(base + l.db);
    f.spoilt = reinterpret_cast<const uint32_t*>(f.db_sums + c.v);
    f.scale = reinterpret_cast<const float*>(base + l.fixed);
    f.v = c.v;
    f.db = c.dbias;
  }
  if (f.ctas + more == 0) return cudaSuccess;
  void* params[] = {&f};
  return launch_kernel(reinterpret_cast<const void*>(&vocab_finish_kernel), f.ctas + more, 256,
                       ws.stream, params);
}

}  // namespace efs
