// vocab_few.cu — the vocabulary loss and its gradient for at most 16 rows
// (scoring a token, a handful of training tokens): bound by reading w once
// (and, for the gradient, writing dw once), at any alignment, without the
// gathering and the tiles of 128 rows of vocab.cu.
//
// w goes through a ring of shared-memory tiles per warp, 16 words x 64 columns,
// by cp.async: a copy of the warp covers 128 consecutive bytes of a row (of 4
// rows, where rows start at 16-byte boundaries), and mma.sync operands are read
// back with ldmatrix. (Loading the operands straight from global memory touches
// 8 lines per load: 21 us for 28,869 words x 650, rows on 4-byte boundaries.)
// mma.sync rather than fp32 FMAs: those would need 8 or 16 per element of w,
// close to the CUDA cores' peak at the rate w arrives.
//
// Logits (words = M, tokens = N). The loss keeps (max, sum) per token in
// registers; the last CTA to finish joins all CTAs' pairs. One token against
// 28,869 words x 650 takes 12 us of which about 6 are w's 37.5 MB at the copy
// rate; the rest is the launch, the first loads and the joins.
//
// Gradient, G as bf16 hi + lo (16 bits: a handful of rows do not average
// roundings out). dw = G^T h has K = the tokens' hi and lo, dh = G w K = 16
// words; partial sums of dh are added in order by a kernel of their own.
// - Up to 1024 columns: one pass over w (vocab_few_once_kernel).
//   5 x 28,869 x 650: 24 us with w in L2, 32.5 without, 75 MB read and written.
// - Wider rows, whose columns do not fit an SM's warps: the logits leave G in
//   memory, 32 or 64 bytes a word, and a second pass over w (from L2 while w is
//   below about 100 MB) gives a warp 64 columns and a slice of the words. On
//   rows that both could take it was slower throughout (5 x 28,869 x 650: 34
//   against 24 us, 16 x 50,001 x 1024: 72 against 53, 3 x 1000 x 64: 14.8 against
//   12.5, the same inputs call after call).
// Measured on the one-pass kernel and not kept: dw stored along whole rows, 16
// bytes a lane, across the warps' tiles (650 columns: 39 us against 25); two
// teams per SM with 85 registers a thread (27); stores and copies moved between
// the sums and the products (26).
#include <algorithm>

#include "product.cuh"

namespace efs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kFewWarps = 16;        // per CTA, one CTA per SM
constexpr uint32_t kCols = 64;            // columns of a tile
constexpr uint32_t kTileLd = kCols + 8;   // its row stride in shared memory: no bank conflicts
constexpr uint32_t kRing = 4;             // tiles of a warp's ring
constexpr uint32_t kTileElemsFew = 16 * kTileLd;

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit elements, two per lane.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ void ldmatrix_4(uint32_t (&r)[4], const uint16_t* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(smem_u32(p))
               : "memory");
}
__device__ __forceinline__ void ldmatrix_4_trans(uint32_t (&r)[4], const uint16_t* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(smem_u32(p))
               : "memory");
}

// Two bf16 of a row that has `d` of them, zeros past its end.
template <int kAlign>
__device__ __forceinline__ uint32_t load_2(const uint16_t* row, uint32_t c, uint32_t d) {
  if (kAlign >= 4 && c + 2 <= d) return __ldg(reinterpret_cast<const uint32_t*>(row + c));
  uint32_t x = 0;
  if (c < d) x = __ldg(row + c);
  if (c + 1 < d) x |= static_cast<uint32_t>(__ldg(row + c + 1)) << 16;
  return x;
}
__device__ __forceinline__ void store_2(uint16_t* row, uint32_t c, uint32_t d, bool wide,
                                        uint32_t x) {
  if (wide && c + 2 <= d) {
    *reinterpret_cast<uint32_t*>(row + c) = x;
  } else {
    if (c < d) row[c] = static_cast<uint16_t>(x);
    if (c + 1 < d) row[c + 1] = static_cast<uint16_t>(x >> 16);
  }
}

// Starts copying 16 words from v0 x 64 columns from c0 into a tile (zeros past
// the columns; rows past the last word repeat it, their results are dropped).
// Rows on 2-byte boundaries go through registers.
template <int kAlign>
__device__ __forceinline__ void copy_tile(uint16_t* s, const uint16_t* w, uint64_t ld, uint32_t v0,
                                          uint32_t v, uint32_t c0, uint32_t d) {
  const uint32_t lane = threadIdx.x & 31;
  const bool whole = v0 + 16 <= v && c0 + kCols <= d;
  if constexpr (kAlign == 16) {
    const uint32_t r0 = lane >> 3, c = (lane & 7u) * 8;
    const uint32_t to = smem_u32(s + r0 * kTileLd + c);
    if (whole) {
      const uint16_t* p = w + (v0 + r0) * ld + c0 + c;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i, p += 4 * ld)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * (8 * kTileLd)),
                     "l"(p)
                     : "memory");
    } else {
      // bytes of this lane's 8 columns that exist
      const uint32_t bytes = c0 + c >= d ? 0 : min(16u, (d - c0 - c) * 2);
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const uint16_t* row = w + min(v0 + r0 + 4 * i, v - 1) * ld;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + i * (8 * kTileLd)),
                     "l"(row + (bytes ? c0 + c : 0)), "r"(bytes)
                     : "memory");
      }
    }
  } else if constexpr (kAlign == 4) {
    const uint32_t c = lane * 2, to = smem_u32(s + c);
    if (whole) {
      const uint16_t* p = w + v0 * ld + c0 + c;
#pragma unroll
      for (uint32_t i = 0; i < 16; ++i, p += ld)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + i * (2 * kTileLd)),
                     "l"(p)
                     : "memory");
    } else {
      const uint32_t bytes = c0 + c >= d ? 0 : min(4u, (d - c0 - c) * 2);
#pragma unroll
      for (uint32_t i = 0; i < 16; ++i) {
        const uint16_t* row = w + min(v0 + i, v - 1) * ld;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + i * (2 * kTileLd)),
                     "l"(row + (bytes ? c0 + c : 0)), "r"(bytes)
                     : "memory");
      }
    }
  } else {
    uint32_t x[16];
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) x[i] = load_2<2>(w + min(v0 + i, v - 1) * ld, c0 + lane * 2, d);
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i)
      *reinterpret_cast<uint32_t*>(s + i * kTileLd + lane * 2) = x[i];
  }
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the last `kOpen` groups of this thread's copies are done.
template <uint32_t kOpen>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kOpen) : "memory");
}

struct FewArgs {
  const uint16_t *h, *w, *bias;
  const int64_t* target;
  uint64_t ldh, ldw;
  uint32_t n, v, d;
  uint32_t ld_s;  // elements from one token's h to the next in shared memory
  float *loss, *lse;
  const float* row_scale;
  uint32_t* g;             // [word][tokens hi | tokens lo], two tokens a word
  uint16_t* dbias;
  float2* pairs;           // [cta][token]
  float* at_target;        // [token]
  uint32_t* done;          // CTAs that finished; zero between launches
  uint32_t* error;
};

// Two columns of every token's h, zeros past the tokens and columns. No load
// waits for another (rows start on any 2-byte boundary).
template <int kTokens>
__device__ __forceinline__ void load_tokens(uint32_t (&x)[kTokens], const uint16_t* h, uint64_t ld,
                                            uint32_t n, uint32_t c, uint32_t d) {
  const uint32_t c0 = min(c, d - 1), c1 = min(c + 1, d - 1);
  uint32_t lo[kTokens], hi[kTokens];
#pragma unroll
  for (uint32_t t = 0; t < kTokens; ++t) {
    lo[t] = hi[t] = 0;
    if (t < n) {
      lo[t] = __ldg(h + t * ld + c0);
      hi[t] = __ldg(h + t * ld + c1);
    }
  }
#pragma unroll
  for (uint32_t t = 0; t < kTokens; ++t) x[t] = (c < d ? lo[t] : 0u) | (c + 1 < d ? hi[t] << 16 : 0u);
}

// h into shared memory, zeros past the tokens and columns.
template <int kTokens>
__device__ __forceinline__ void stage_h(const FewArgs& a, uint16_t* s_h, uint32_t d_pad) {
  for (uint32_t c = threadIdx.x * 2; c < d_pad; c += kFewWarps * 64) {
    uint32_t x[kTokens];
    load_tokens<kTokens>(x, a.h, a.ldh, a.n, c, a.d);
#pragma unroll
    for (uint32_t t = 0; t < kTokens; ++t)
      *reinterpret_cast<uint32_t*>(s_h + t * a.ld_s + c) = x[t];
  }
}

// exp(z - top), for any finite z and top.
__device__ __forceinline__ float exp_below(float z, float top) {
  return exp2_fast(__fmul_rn(__fsub_rn(z, top), kLog2e));
}
// (max, sum of exp(z - max)) pairs joined; (-inf, 0) is empty.
__device__ __forceinline__ void join_pair(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  const float a = m == top ? 1.0f : exp_below(m, top);
  const float b = m2 == top ? 1.0f : exp_below(m2, top);
  // -inf on one side only: a factor 0; on both: factors 1 of empty sums
  s = __fmaf_rn(s, a, __fmul_rn(s2, b));
  m = top;
}

template <bool kGrad, int kNT, int kAlign>
__global__ void __launch_bounds__(kFewWarps * 32, 1) vocab_few_kernel(const FewArgs a) {
  constexpr int kTokens = 8 * kNT;
  extern __shared__ __align__(16) uint16_t s_dyn[];  // the warps' rings, then h
  __shared__ float2 s_pair[kFewWarps][kTokens];
  __shared__ int64_t s_target[kTokens];
  __shared__ float s_lse[kTokens], s_scale[kTokens];
  __shared__ uint32_t s_last;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t row = lane >> 2, quad = lane & 3u;
  const uint32_t d_pad = (a.d + kCols - 1) / kCols * kCols;
  griddep_wait();
  if (threadIdx.x < kTokens) {
    const uint32_t t = threadIdx.x;
    int64_t target = t < a.n ? a.target[t] : -1;
    if (target >= static_cast<int64_t>(a.v)) {
      target = -1;
      if (blockIdx.x == 0) atomicOr(a.error, kDevErrBadInput);
    }
    s_target[t] = target;
    if (kGrad) {
      float lse = t < a.n ? a.lse[t] : -INFINITY;  // (its load does not wait for the target's)
      if (target < 0) lse = -INFINITY;
      s_lse[t] = lse;
      // a row that is skipped, or has no word with a probability: no gradient
      s_scale[t] = lse == -INFINITY ? 0.0f : a.row_scale[t];
    }
  }
  // consecutive groups of 16 words go to different SMs; a warp's tiles are its
  // groups' columns one after another
  const uint32_t groups = (a.v + 15) / 16, warps = gridDim.x * kFewWarps;
  const uint32_t first = warp * gridDim.x + blockIdx.x;
  uint16_t* ring = s_dyn + warp * (kRing * kTileElemsFew);
  uint16_t* s_h = s_dyn + kFewWarps * kRing * kTileElemsFew;
  uint32_t next_grp = first, next_c = 0, next_slot = 0;
  auto fetch = [&]() {
    if (next_grp < groups) {
      copy_tile<kAlign>(ring + next_slot * kTileElemsFew, a.w, a.ldw, next_grp * 16, a.v, next_c, a.d);
      next_c += kCols;
      if (next_c >= d_pad) {
        next_c = 0;
        next_grp += warps;
      }
    }
    next_slot = next_slot + 1 == kRing ? 0 : next_slot + 1;
    copy_commit();
  };
#pragma unroll
  for (uint32_t i = 0; i < kRing - 1; ++i) fetch();
  stage_h<kTokens>(a, s_h, d_pad);
  __syncthreads();
  float m[2 * kNT], sum[2 * kNT];
#pragma unroll
  for (int i = 0; i < 2 * kNT; ++i) m[i] = -INFINITY, sum[i] = 0.0f;
  const uint16_t* frag_w = ring + (lane & 15u) * kTileLd + (lane >> 4) * 8;
  const uint16_t* frag_h = s_h + (lane & 7u) * a.ld_s + (lane >> 3) * 8;

  uint32_t slot = 0;
  for (uint32_t grp = first; grp < groups; grp += warps) {
    const uint32_t v0 = grp * 16 + row, v1 = v0 + 8;
    const float b0 = a.bias && v0 < a.v ? bf16_bits_to_f32(__ldg(a.bias + v0)) : 0.0f;
    const float b1 = a.bias && v1 < a.v ? bf16_bits_to_f32(__ldg(a.bias + v1)) : 0.0f;
    // two chains of sums per token tile: shorter, so their roundings add up less
    float acc[kNT][2][4];
#pragma unroll
    for (int t = 0; t < kNT; ++t)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[t][j >> 2][j & 3] = 0.0f;
    for (uint32_t c0 = 0; c0 < d_pad; c0 += kCols) {
      copy_wait<kRing - 2>();
      __syncwarp();
      fetch();  // into the tile that all lanes have finished reading
      const uint16_t* tile = frag_w + slot * kTileElemsFew;
      slot = slot + 1 == kRing ? 0 : slot + 1;
#pragma unroll
      for (uint32_t k = 0; k < kCols; k += 32) {
        uint32_t w0[4], w1[4];
        ldmatrix_4(w0, tile + k);
        ldmatrix_4(w1, tile + k + 16);
#pragma unroll
        for (int t = 0; t < kNT; ++t) {
          uint32_t h[4];
          ldmatrix_4(h, frag_h + t * 8 * a.ld_s + c0 + k);
          mma_16816(acc[t][0], w0[0], w0[1], w0[2], w0[3], h[0], h[1]);
          mma_16816(acc[t][1], w1[0], w1[1], w1[2], w1[3], h[2], h[3]);
        }
      }
    }
    float db0 = 0.0f, db1 = 0.0f;
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      float z[4];  // (word v0, token), (v0, token + 1), (v1, token), (v1, token + 1)
#pragma unroll
      for (int j = 0; j < 4; ++j) z[j] = __fadd_rn(__fadd_rn(acc[t][0][j], acc[t][1][j]), j < 2 ? b0 : b1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t token = t * 8 + quad * 2 + (j & 1), v = j < 2 ? v0 : v1;
        if (kGrad) {
          const float scale = s_scale[token];
          float g = 0.0f;
          if (scale != 0.0f && v < a.v) {
            g = __fmul_rn(exp_below(z[j], s_lse[token]), scale);
            if (static_cast<int64_t>(v) == s_target[token]) g = __fsub_rn(g, scale);
          }
          z[j] = g;
        } else if (v < a.v) {
          if (static_cast<int64_t>(v) == s_target[token]) a.at_target[token] = z[j];
          join_pair(m[2 * t + (j & 1)], sum[2 * t + (j & 1)], z[j],
                    z[j] == -INFINITY ? 0.0f : (z[j] - z[j]) + 1.0f);  // NaN, inf: NaN
        }
      }
      if (kGrad) {
        db0 = __fadd_rn(db0, __fadd_rn(z[0], z[1]));
        db1 = __fadd_rn(db1, __fadd_rn(z[2], z[3]));
        const uint32_t hi0 = pack_bf16(z[0], z[1]), hi1 = pack_bf16(z[2], z[3]);
        const uint32_t lo0 = pack_bf16(__fsub_rn(z[0], __uint_as_float(hi0 << 16)),
                                       __fsub_rn(z[1], __uint_as_float(hi0 & 0xffff0000u)));
        const uint32_t lo1 = pack_bf16(__fsub_rn(z[2], __uint_as_float(hi1 << 16)),
                                       __fsub_rn(z[3], __uint_as_float(hi1 & 0xffff0000u)));
        // words up to the group's end are written (zeros past the vocabulary)
        uint32_t* g0 = a.g + static_cast<uint64_t>(v0) * kTokens + t * 4 + quad;
        uint32_t* g1 = g0 + 8 * kTokens;
        g0[0] = hi0;
        g0[kTokens / 2] = lo0;
        g1[0] = hi1;
        g1[kTokens / 2] = lo1;
      }
    }
    if (kGrad && a.dbias) {
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        db0 = __fadd_rn(db0, __shfl_xor_sync(0xffffffffu, db0, o));
        db1 = __fadd_rn(db1, __shfl_xor_sync(0xffffffffu, db1, o));
      }
      if (quad == 0) {
        if (v0 < a.v) a.dbias[v0] = static_cast<uint16_t>(pack_bf16(db0, 0.0f));
        if (v1 < a.v) a.dbias[v1] = static_cast<uint16_t>(pack_bf16(db1, 0.0f));
      }
    }
  }
  if constexpr (!kGrad) {
    // the warps' pairs, the CTA's, and in the last CTA all of them
#pragma unroll
    for (int i = 0; i < 2 * kNT; ++i) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1)
        join_pair(m[i], sum[i], __shfl_xor_sync(0xffffffffu, m[i], o),
                  __shfl_xor_sync(0xffffffffu, sum[i], o));
      if (row == 0) s_pair[warp][(i >> 1) * 8 + quad * 2 + (i & 1)] = make_float2(m[i], sum[i]);
    }
    __syncthreads();
    if (threadIdx.x < kTokens) {
      float2 p = s_pair[0][threadIdx.x];
      for (uint32_t q = 1; q < kFewWarps; ++q)
        join_pair(p.x, p.y, s_pair[q][threadIdx.x].x, s_pair[q][threadIdx.x].y);
      a.pairs[blockIdx.x * kTokens + threadIdx.x] = p;
      __threadfence();
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      __threadfence();
      s_last = atomicAdd(a.done, 1u) == gridDim.x - 1 ? 1u : 0u;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    for (uint32_t t = warp; t < kTokens; t += kFewWarps) {
      float pm = -INFINITY, ps = 0.0f;
      for (uint32_t c = lane; c < gridDim.x; c += 32) {
        const float2 p = __ldcg(a.pairs + c * kTokens + t);
        join_pair(pm, ps, p.x, p.y);
      }
#pragma unroll
      for (int o = 1; o < 32; o <<= 1)
        join_pair(pm, ps, __shfl_xor_sync(0xffffffffu, pm, o), __shfl_xor_sync(0xffffffffu, ps, o));
      if (lane == 0 && t < a.n) {
        float lse = 0.0f, loss = 0.0f;
        if (s_target[t] >= 0) {
          const float z = __ldcg(a.at_target + t);
          lse = ps != ps ? ps : pm == -INFINITY ? -INFINITY : __fadd_rn(pm, logf(ps));
          loss = z == -INFINITY && ps == ps ? INFINITY : __fsub_rn(lse, z);
        }
        a.lse[t] = lse;
        a.loss[t] = loss;
      }
    }
    if (threadIdx.x == 0) *a.done = 0;
  }
}

// Whether a row has a gradient: a target, and a word with a probability. (Those
// that have none have G = 0, but their h, or w, may hold infinities.)
__device__ __forceinline__ bool has_gradient(int64_t target, float lse, uint32_t v) {
  return target >= 0 && target < static_cast<int64_t>(v) && lse != -INFINITY;
}

struct FewGradArgs {
  const uint16_t *h, *w;
  const int64_t* target;
  const float* lse;
  const uint32_t* g;
  uint64_t ldh, ldw, lddw;
  uint32_t n, v, d;
  uint32_t windows, slices, slice_groups;  // of columns; of words; groups of 16 words per slice
  uint16_t* dw;
  uint32_t align_dw;  // of dw's rows, in bytes
  float* sums;  // [slice][token][ld_sum]
  uint32_t ld_sum;
};

// A warp's ring of the second pass: tiles, each with G of its words (as many
// as fit an SM), and a tile of dw.
template <int kNT>
struct GradRing {
  static constexpr uint32_t kDeep = kNT == 1 ? 4 : 3;
  static constexpr uint32_t kSlot = kTileElemsFew + 16 * 2 * 8 * kNT;
  static constexpr uint32_t kBytes = (kDeep * kSlot + kTileElemsFew) * 2;
};

// dh += G w: words along K, two tiles of 8 columns at a time. G comes as the
// hi and lo of a word's tokens (fragments: words row, row + 8).
template <int kNT>
__device__ __forceinline__ void add_dh(float (&dh)[8][4], const uint32_t (&hi0)[kNT],
                                       const uint32_t (&hi1)[kNT], const uint32_t (&lo0)[kNT],
                                       const uint32_t (&lo1)[kNT], const uint16_t* words) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t a0, a1, a2, a3, l0 = 0, l1 = 0, l2 = 0, l3 = 0;
  if (kNT == 1) {  // rows: 8 tokens' hi, then lo
    a0 = transpose_8x8(hi0[0]), a1 = transpose_8x8(lo0[0]);
    a2 = transpose_8x8(hi1[0]), a3 = transpose_8x8(lo1[0]);
  } else {
    a0 = transpose_8x8(hi0[0]), a1 = transpose_8x8(hi0[kNT - 1]);
    a2 = transpose_8x8(hi1[0]), a3 = transpose_8x8(hi1[kNT - 1]);
    l0 = transpose_8x8(lo0[0]), l1 = transpose_8x8(lo0[kNT - 1]);
    l2 = transpose_8x8(lo1[0]), l3 = transpose_8x8(lo1[kNT - 1]);
  }
#pragma unroll
  for (int t = 0; t < 8; t += 2) {
    uint32_t w[4];  // words 0-7 and 8-15 of columns 8 t, then of 8 t + 8
    ldmatrix_4_trans(w, words + (lane & 15u) * kTileLd + t * 8 + (lane >> 4) * 8);
    if (kNT == 2) {
      mma_16816(dh[t], l0, l1, l2, l3, w[0], w[1]);
      mma_16816(dh[t + 1], l0, l1, l2, l3, w[2], w[3]);
    }
    mma_16816(dh[t], a0, a1, a2, a3, w[0], w[1]);
    mma_16816(dh[t + 1], a0, a1, a2, a3, w[2], w[3]);
  }
}
// dw = G^T h of 16 words x 64 columns, rounded, into a tile.
template <int kNT>
__device__ __forceinline__ void make_dw(const uint32_t (&hi0)[kNT], const uint32_t (&hi1)[kNT],
                                        const uint32_t (&lo0)[kNT], const uint32_t (&lo1)[kNT],
                                        const uint32_t (&ht)[kNT][8], uint16_t* tile) {
  const uint32_t lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3u;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (kNT == 1) {  // K = 8 tokens' hi, then lo
      mma_16816(f, hi0[0], hi1[0], lo0[0], lo1[0], ht[0][t], ht[0][t]);
    } else {
      mma_16816(f, lo0[0], lo1[0], lo0[kNT - 1], lo1[kNT - 1], ht[0][t], ht[kNT - 1][t]);
      mma_16816(f, hi0[0], hi1[0], hi0[kNT - 1], hi1[kNT - 1], ht[0][t], ht[kNT - 1][t]);
    }
    uint16_t* to = tile + row * kTileLd + t * 8 + quad * 2;
    *reinterpret_cast<uint32_t*>(to) = pack_bf16(f[0], f[1]);
    *reinterpret_cast<uint32_t*>(to + 8 * kTileLd) = pack_bf16(f[2], f[3]);
  }
}
// A tile to rows v0 .. of dw, columns c0 ..; `align` of its rows in bytes.
__device__ __forceinline__ void store_dw(const uint16_t* tile, uint16_t* dw, uint64_t ld, uint32_t align,
                                         uint32_t v0, uint32_t v, uint32_t c0, uint32_t d) {
  const uint32_t lane = threadIdx.x & 31;
  if (align == 16) {
    const uint32_t c = (lane & 7u) * 8;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      const uint32_t r = j * 4 + (lane >> 3);
      if (v0 + r >= v) break;
      uint16_t* to = dw + static_cast<uint64_t>(v0 + r) * ld;
      const uint4 x = *reinterpret_cast<const uint4*>(tile + r * kTileLd + c);
      if (c0 + c + 8 <= d) {
        *reinterpret_cast<uint4*>(to + c0 + c) = x;
      } else {
        store_2(to, c0 + c, d, true, x.x);
        store_2(to, c0 + c + 2, d, true, x.y);
        store_2(to, c0 + c + 4, d, true, x.z);
        store_2(to, c0 + c + 6, d, true, x.w);
      }
    }
  } else if (align >= 4 && v0 + 16 <= v) {
    const uint32_t c = c0 + lane * 2;
    uint16_t* to = dw + static_cast<uint64_t>(v0) * ld + c;
#pragma unroll
    for (uint32_t r = 0; r < 16; ++r, to += ld) {
      const uint32_t x = *reinterpret_cast<const uint32_t*>(tile + r * kTileLd + lane * 2);
      if (c + 2 <= d) *reinterpret_cast<uint32_t*>(to) = x;
    }
    if (c + 1 == d) {
#pragma unroll 1
      for (uint32_t r = 0; r < 16; ++r)
        dw[static_cast<uint64_t>(v0 + r) * ld + c] = tile[r * kTileLd + lane * 2];
    }
  } else {
#pragma unroll 1
    for (uint32_t r = 0; r < 16 && v0 + r < v; ++r)
      store_2(dw + static_cast<uint64_t>(v0 + r) * ld, c0 + lane * 2, d, align >= 4,
              *reinterpret_cast<const uint32_t*>(tile + r * kTileLd + lane * 2));
  }
}
// A warp's sums of dh: [token][ld], columns c0 ...
template <int kNT>
__device__ __forceinline__ void store_dh(const float (&dh)[8][4], float* to, uint32_t ld, uint32_t c0) {
  const uint32_t lane = threadIdx.x & 31;
  float* sums = to + (lane >> 2) * ld + c0 + (lane & 3u) * 2;
  float* more = sums + 8ull * ld;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    if (kNT == 1) {
      *reinterpret_cast<float2*>(sums + t * 8) =
          make_float2(__fadd_rn(dh[t][0], dh[t][2]), __fadd_rn(dh[t][1], dh[t][3]));
    } else {
      *reinterpret_cast<float2*>(sums + t * 8) = make_float2(dh[t][0], dh[t][1]);
      *reinterpret_cast<float2*>(more + t * 8) = make_float2(dh[t][2], dh[t][3]);
    }
  }
}

// dw and the slices' sums of dh: a warp takes a window of 64 columns and a
// slice of the words.
template <int kNT, int kAlign>
__global__ void __launch_bounds__(kFewWarps * 32, 1) vocab_few_grad_kernel(const FewGradArgs a) {
  constexpr int kTokens = 8 * kNT;
  extern __shared__ __align__(16) uint16_t s_dyn[];  // the warps' rings, then their dw tiles
  const uint32_t lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3u;
  const uint32_t warp = threadIdx.x >> 5;
  const uint32_t task = warp * gridDim.x + blockIdx.x;
  griddep_wait();
  if (task >= a.windows * a.slices) return;
  const uint32_t window = task % a.windows, slice = task / a.windows, c0 = window * kCols;
  const uint32_t groups = (a.v + 15) / 16;
  const uint32_t lo = slice * a.slice_groups, hi = min(lo + a.slice_groups, groups);
  using Slots = GradRing<kNT>;
  constexpr uint32_t kDeep = Slots::kDeep, kSlot = Slots::kSlot;
  uint16_t* ring = s_dyn + warp * (kDeep * kSlot + kTileElemsFew);
  uint16_t* tile = ring + kDeep * kSlot;  // h's, then dw's
  uint32_t next_grp = lo, next_slot = 0;
  auto fetch = [&]() {
    if (next_grp < hi) {
      uint16_t* to = ring + next_slot * kSlot;
      copy_tile<kAlign>(to, a.w, a.ldw, next_grp * 16, a.v, c0, a.d);
      const uint32_t* g = a.g + static_cast<uint64_t>(next_grp * 16) * kTokens + lane * 4;
#pragma unroll
      for (int i = 0; i < kNT; ++i)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                         smem_u32(to + kTileElemsFew + (i * 32 + lane) * 8)),
                     "l"(g + i * 128)
                     : "memory");
    }
    ++next_grp;
    next_slot = next_slot + 1 == kDeep ? 0 : next_slot + 1;
    copy_commit();
  };
#pragma unroll
  for (uint32_t i = 0; i < kDeep - 1; ++i) fetch();
  // h of the window as the operand of dw, tokens along K: through the tile
  uint32_t ht[kNT][8];
  {
    uint32_t x[kTokens];
    bool has[kTokens];
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
      has[t] = t < static_cast<int>(a.n) && has_gradient(a.target[t], a.lse[t], a.v);
    load_tokens<kTokens>(x, a.h, a.ldh, a.n, c0 + lane * 2, a.d);
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
      *reinterpret_cast<uint32_t*>(tile + t * kTileLd + lane * 2) = has[t] ? x[t] : 0u;
  }
  __syncwarp();
#pragma unroll
  for (int t = 0; t < kNT; ++t)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t r[4];
      ldmatrix_4_trans(r, tile + (t * 8 + (lane & 7u)) * kTileLd + j * 32 + (lane >> 3) * 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) ht[t][j * 4 + i] = r[i];
    }
  float dh[8][4];
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) dh[t][j] = 0.0f;
  uint32_t slot = 0;
  for (uint32_t grp = lo; grp < hi; ++grp) {
    copy_wait<kDeep - 2>();
    __syncwarp();
    fetch();  // into the tile that all lanes have finished reading
    const uint16_t* words = ring + slot * kSlot;
    slot = slot + 1 == kDeep ? 0 : slot + 1;
    uint32_t hi0[kNT], hi1[kNT], lo0[kNT], lo1[kNT];
    const uint32_t* g0 = reinterpret_cast<const uint32_t*>(words + kTileElemsFew) + row * kTokens + quad;
    const uint32_t* g1 = g0 + 8 * kTokens;
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      hi0[t] = g0[t * 4];
      hi1[t] = g1[t * 4];
      lo0[t] = g0[kTokens / 2 + t * 4];
      lo1[t] = g1[kTokens / 2 + t * 4];
    }
    add_dh<kNT>(dh, hi0, hi1, lo0, lo1, words);
    make_dw<kNT>(hi0, hi1, lo0, lo1, ht, tile);
    __syncwarp();
    store_dw(tile, a.dw, a.lddw, a.align_dw, grp * 16, a.v, c0, a.d);
  }
  store_dh<kNT>(dh, a.sums + static_cast<uint64_t>(slice) * kTokens * a.ld_sum, a.ld_sum, c0);
}

struct FewOnceArgs {
  const uint16_t *h, *w, *bias;
  const int64_t* target;
  const float *lse, *row_scale;
  uint64_t ldh, ldw, lddw;
  uint32_t n, v, d;
  uint32_t windows, teams;  // of columns, a warp each; of warps that share words
  uint32_t slice_groups;    // groups of 16 words per team
  uint16_t *dw, *dbias;
  uint32_t align_dw;  // of dw's rows, in bytes
  float* sums;        // [cta][token][ld_sum]
  uint32_t ld_sum;
  uint32_t* error;
};
constexpr uint32_t kOnceDeep = 5;  // tiles of a warp's ring: two in use, three on their way

// Shared memory of a team: the warps' rings, partial logits of two groups, G of
// two groups (hi, lo).
template <int kNT>
__host__ __device__ constexpr uint32_t team_bytes(uint32_t windows) {
  return windows * (kOnceDeep * kTileElemsFew * 2 + 2 * kNT * 512) + 2 * 2 * kNT * 256;
}
__device__ __forceinline__ void team_sync(uint32_t team, uint32_t warps) {
  if (warps == 1)
    __syncwarp();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(warps * 32) : "memory");
}

// The whole gradient in one pass over w, for up to 1024 columns: a team has a
// warp per 64 columns, and a group of 16 words that it has in shared memory
// serves all three products. Only the logits need the other warps' columns; the
// work on three groups is interleaved so that a group costs one barrier: between
// two of them the team sums the partial logits of group i and forms its G, takes
// the partial logits of group i + 1, and forms dw and dh from G of group i - 1.
template <int kNT, int kAlign>
__global__ void __launch_bounds__(kFewWarps * 32, 1) vocab_few_once_kernel(const FewOnceArgs a) {
  constexpr uint32_t kTokens = 8 * kNT, kPart = kNT * 128;
  extern __shared__ __align__(16) uint16_t s_dyn[];
  __shared__ int64_t s_target[kTokens];
  __shared__ float s_lse[kTokens], s_scale[kTokens];
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t warps = a.windows, team = (threadIdx.x >> 5) / warps, warp = (threadIdx.x >> 5) % warps;
  const uint32_t thread = warp * 32 + lane, threads = warps * 32, c0 = warp * kCols;
  uint16_t* s_team = s_dyn + team * (team_bytes<kNT>(warps) / 2);
  constexpr uint32_t ring_elems = kOnceDeep * kTileElemsFew;
  uint16_t* ring = s_team + warp * ring_elems;
  float* parts = reinterpret_cast<float*>(s_team + warps * ring_elems);
  uint16_t* s_g = reinterpret_cast<uint16_t*>(parts + 2 * warps * kPart);  // [parity][hi, lo], as fragments
  const uint32_t groups = (a.v + 15) / 16, lo = (blockIdx.x * a.teams + team) * a.slice_groups;
  const uint32_t count = lo < groups ? min(a.slice_groups, groups - lo) : 0u;
  griddep_wait();
  auto advance = [&](uint32_t slot) { return slot + 1 == kOnceDeep ? 0u : slot + 1; };
  uint32_t next = 0, next_slot = 0;
  auto fetch = [&]() {
    if (next < count)
      copy_tile<kAlign>(ring + next_slot * kTileElemsFew, a.w, a.ldw, (lo + next) * 16, a.v, c0, a.d);
    ++next;
    next_slot = advance(next_slot);
    copy_commit();
  };
  // (h's loads start ahead of the ring's copies, which fill the memory pipe; no
  // load waits for a target)
  int64_t targets[kTokens];
  float lses[kTokens];
  uint32_t x[kTokens];
#pragma unroll
  for (uint32_t t = 0; t < kTokens; ++t) {
    targets[t] = t < a.n ? a.target[t] : -1;
    lses[t] = t < a.n ? a.lse[t] : 0.0f;
  }
  load_tokens<kTokens>(x, a.h, a.ldh, a.n, c0 + lane * 2, a.d);
#pragma unroll
  for (uint32_t i = 0; i < kOnceDeep - 1; ++i) fetch();
  for (uint32_t t = threadIdx.x; t < kTokens; t += blockDim.x) {
    int64_t target = t < a.n ? a.target[t] : -1;
    float lse = t < a.n ? a.lse[t] : -INFINITY;
    const float scale = t < a.n ? a.row_scale[t] : 0.0f;
    if (target >= static_cast<int64_t>(a.v)) {
      target = -1;
      if (blockIdx.x == 0) atomicOr(a.error, kDevErrBadInput);
    }
    if (target < 0) lse = -INFINITY;
    s_target[t] = target;
    s_lse[t] = lse;
    // a row that is skipped, or has no word with a probability: no gradient
    s_scale[t] = lse == -INFINITY ? 0.0f : scale;
  }
  // h of the warp's columns as the operand of the logits (columns along K) and,
  // through the ring's last tile, of dw (tokens along K); nothing of a row without
  // a gradient
  uint32_t hk[kNT][8], ht[kNT][8];
  {
    uint16_t* tile = ring + (kOnceDeep - 1) * kTileElemsFew;
#pragma unroll
    for (uint32_t t = 0; t < kTokens; ++t)
      *reinterpret_cast<uint32_t*>(tile + t * kTileLd + lane * 2) =
          has_gradient(targets[t], lses[t], a.v) ? x[t] : 0u;
    __syncwarp();
#pragma unroll
    for (int t = 0; t < kNT; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint16_t* from = tile + (t * 8 + (lane & 7u)) * kTileLd + j * 32 + (lane >> 3) * 8;
        uint32_t r[4], q[4];
        ldmatrix_4_trans(r, from);
        ldmatrix_4(q, from);
#pragma unroll
        for (int i = 0; i < 4; ++i) ht[t][j * 4 + i] = r[i], hk[t][j * 4 + i] = q[i];
      }
  }
  __syncthreads();
  float dh[8][4];
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) dh[t][j] = 0.0f;

  // group i's logits over this warp's columns
  uint32_t slot_z = 0;
  auto logits = [&](uint32_t i) {
    const uint16_t* tile = ring + slot_z * kTileElemsFew + (lane & 15u) * kTileLd + (lane >> 4) * 8;
    slot_z = advance(slot_z);
    float acc[kNT][4];
#pragma unroll
    for (int t = 0; t < kNT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[t][j] = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t w[4];
      ldmatrix_4(w, tile + k * 16);
#pragma unroll
      for (int t = 0; t < kNT; ++t)
        mma_16816(acc[t], w[0], w[1], w[2], w[3], hk[t][2 * k], hk[t][2 * k + 1]);
    }
    float* to = parts + ((i & 1u) * warps + warp) * kPart + lane * 4;
#pragma unroll
    for (int t = 0; t < kNT; ++t)
      *reinterpret_cast<float4*>(to + t * 128) = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
  };
  copy_wait<kOnceDeep - 2>();
  __syncwarp();
  if (count) logits(0);

  // The partial logits of a value are summed by one lane, or by two in teams of
  // 8 warps and more. The bias of a lane's first value is loaded a group ahead.
  const uint32_t split = warps >= 8 ? 1 : 0;
  auto word = [&](uint32_t i, uint32_t e) { return (lo + i) * 16 + (e >> 4) + ((e & 2u) << 2); };
  auto load_bias = [&](uint32_t v) {
    return a.bias && v < a.v ? bf16_bits_to_f32(__ldg(a.bias + v)) : 0.0f;
  };
  float next_bias = thread < (128u << split) ? load_bias(word(0, thread >> split)) : 0.0f;
  uint32_t slot_g = 0;
  for (uint32_t i = 0; count && i <= count; ++i) {
    team_sync(team, warps);
    if (i < count) {
      // G of group i: value e is of word e / 16 + 8 (e / 2 % 2), token 2 (e / 4 % 4) + e % 2
      uint16_t* g_hi = s_g + (i & 1u) * (2 * kPart);
      for (uint32_t at = thread; at < (128u << split); at += threads) {
        const uint32_t e = at >> split, v = word(i, e);
        const float bias = at == thread ? next_bias : load_bias(v);
        if (at == thread) next_bias = load_bias(word(i + 1, e));
        const float* from = parts + (i & 1u) * (warps * kPart) + e;
        float z[kNT];
#pragma unroll
        for (int t = 0; t < kNT; ++t) z[t] = 0.0f;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          const uint32_t q = (j << split) + (at & split);
          if (q < warps) {
#pragma unroll
            for (int t = 0; t < kNT; ++t) z[t] = __fadd_rn(z[t], from[q * kPart + t * 128]);
          }
        }
        float db = 0.0f;
#pragma unroll
        for (int t = 0; t < kNT; ++t) {
          if (split) z[t] = __fadd_rn(z[t], __shfl_xor_sync(0xffffffffu, z[t], 1));
          z[t] = __fadd_rn(z[t], bias);
          const uint32_t token = t * 8 + ((e >> 2) & 3u) * 2 + (e & 1u);
          const float scale = s_scale[token];
          float g = 0.0f;
          if (scale != 0.0f && v < a.v) {
            g = __fmul_rn(exp_below(z[t], s_lse[token]), scale);
            if (static_cast<int64_t>(v) == s_target[token]) g = __fsub_rn(g, scale);
          }
          db = __fadd_rn(db, g);
          const uint32_t hi = pack_bf16(g, 0.0f) & 0xffffu;
          g_hi[t * 128 + e] = static_cast<uint16_t>(hi);
          g_hi[kPart + t * 128 + e] =
              static_cast<uint16_t>(pack_bf16(__fsub_rn(g, __uint_as_float(hi << 16)), 0.0f));
        }
        if (a.dbias) {
#pragma unroll
          for (int o : {1, 4, 8}) db = __fadd_rn(db, __shfl_xor_sync(0xffffffffu, db, o << split));
          if ((e & 13u) == 0 && (at & split) == 0 && v < a.v)
            a.dbias[v] = static_cast<uint16_t>(pack_bf16(db, 0.0f));
        }
      }
      copy_wait<kOnceDeep - 3>();
      __syncwarp();
      if (i + 1 < count) logits(i + 1);
    }
    if (i > 0) {
      uint16_t* tile = ring + slot_g * kTileElemsFew;
      slot_g = advance(slot_g);
      const uint16_t* g_hi = s_g + ((i & 1u) ^ 1u) * (2 * kPart) + lane * 4;
      uint32_t hi0[kNT], hi1[kNT], lo0[kNT], lo1[kNT];
#pragma unroll
      for (int t = 0; t < kNT; ++t) {
        const uint2 x = *reinterpret_cast<const uint2*>(g_hi + t * 128);
        const uint2 y = *reinterpret_cast<const uint2*>(g_hi + kPart + t * 128);
        hi0[t] = x.x, hi1[t] = x.y, lo0[t] = y.x, lo1[t] = y.y;
      }
      add_dh<kNT>(dh, hi0, hi1, lo0, lo1, tile);
      __syncwarp();
      make_dw<kNT>(hi0, hi1, lo0, lo1, ht, tile);  // in place of the words
      __syncwarp();
      store_dw(tile, a.dw, a.lddw, a.align_dw, (lo + i - 1) * 16, a.v, c0, a.d);
      __syncwarp();
    }
    fetch();  // group i + 4, into the tile of group i - 1
  }
  float* sums = a.sums + static_cast<uint64_t>(blockIdx.x) * kTokens * a.ld_sum;
  if (a.teams == 1) {
    store_dh<kNT>(dh, sums, a.ld_sum, c0);
  } else {  // the teams' sums in order, through the rings
    __syncthreads();
    float* all = reinterpret_cast<float*>(s_dyn);
    const uint32_t each = kTokens * a.ld_sum;
    store_dh<kNT>(dh, all + team * each, a.ld_sum, c0);
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < each; c += blockDim.x) {
      float x = all[c];
      for (uint32_t t = 1; t < a.teams; ++t) x = __fadd_rn(x, all[t * each + c]);
      sums[c] = x;
    }
  }
}

// dh: a CTA adds the slices of 32 columns of a token, in 8 runs of them.
__global__ void __launch_bounds__(256)
    vocab_few_dh_kernel(const float* __restrict__ sums, uint32_t slices, uint32_t tokens,
                        uint32_t ld_sum, uint32_t cols, uint16_t* __restrict__ dh, uint64_t ld,
                        const int64_t* __restrict__ target, const float* __restrict__ lse,
                        uint32_t v) {
  __shared__ float s_part[8][32];
  const uint32_t lane = threadIdx.x & 31, run = threadIdx.x >> 5;
  const uint32_t c = blockIdx.x * 32 + lane, token = blockIdx.y;
  griddep_wait();
  const uint32_t per = (slices + 7) / 8, lo = run * per, hi = min(lo + per, slices);
  const float* p = sums + static_cast<uint64_t>(token) * ld_sum + c;
  const uint64_t stride = static_cast<uint64_t>(tokens) * ld_sum;
  const bool has = has_gradient(target[token], lse[token], v);
  float x = 0.0f;
  for (uint32_t s0 = lo; s0 < hi; s0 += 10) {  // (151 slices: two rounds of loads)
    float y[10];
#pragma unroll
    for (uint32_t j = 0; j < 10; ++j) y[j] = __ldcg(p + min(s0 + j, hi - 1) * stride);
#pragma unroll
    for (uint32_t j = 0; j < 10; ++j)
      if (s0 + j < hi) x = __fadd_rn(x, y[j]);
  }
  s_part[run][lane] = x;
  __syncthreads();
  if (run == 0 && c < cols) {
    for (int r = 1; r < 8; ++r) x = __fadd_rn(x, s_part[r][lane]);
    if (!has) x = 0.0f;
    dh[token * ld + c] = static_cast<uint16_t>(pack_bf16(x, 0.0f));
  }
}

constexpr size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

constexpr uint32_t kOnceBytes = 225 * 1024;  // of shared memory, for a CTA's teams
struct FewPlan {
  uint32_t nt, ld_s, smem, ctas;
  uint32_t windows, slices, slice_groups;
  bool once;
  uint32_t teams, team_bytes;
  size_t pairs, at_target, g, sums, total;
};

FewPlan few_plan(const VocabCall& c, bool gradient, const DeviceInfo& dev) {
  FewPlan p = {};
  p.nt = c.n <= 8 ? 1 : 2;
  const uint32_t d_pad = (c.d + kCols - 1) / kCols * kCols, groups = (c.v + 15) / 16;
  const uint32_t tokens = 8 * p.nt, sms = static_cast<uint32_t>(dev.sm_count);
  p.ld_s = d_pad + 8;  // an odd number of 16 bytes: reads of h do not conflict
  p.smem = kFewWarps * kRing * kTileElemsFew * 2 + tokens * p.ld_s * 2;
  p.ctas = groups < sms ? groups : sms;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  p.windows = d_pad / kCols;
  // One pass where a CTA's warps cover the columns.
  p.once = gradient && p.windows <= kFewWarps;
  if (!gradient) {
    p.pairs = take(sizeof(float2) * p.ctas * tokens);
    p.at_target = take(sizeof(float) * tokens);
  }
  if (gradient) {
    if (p.once) {
      p.team_bytes = p.nt == 1 ? team_bytes<1>(p.windows) : team_bytes<2>(p.windows);
      p.teams = std::min(kFewWarps / p.windows, kOnceBytes / p.team_bytes);
      const uint32_t all = p.teams * sms;
      p.slice_groups = (groups + all - 1) / all;
      const uint32_t used = (groups + p.slice_groups - 1) / p.slice_groups;
      p.slices = (used + p.teams - 1) / p.teams;  // CTAs
    } else {
      const uint32_t slices = kFewWarps * sms / p.windows;  // 16 warps per SM, 17 to 71 windows
      p.slice_groups = (groups + slices - 1) / slices;
      p.slices = (groups + p.slice_groups - 1) / p.slice_groups;
    }
    if (!p.once) p.g = take(4ull * tokens * groups * 16);
    p.sums = take(4ull * p.slices * tokens * d_pad);
  }
  p.total = at;
  return p;
}

template <bool kGrad, int kNT, int kAlign>
cudaError_t few_logits(const FewArgs& a, const FewPlan& p, Workspace& ws) {
  auto fn = vocab_few_kernel<kGrad, kNT, kAlign>;
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(p.smem));
  if (e != cudaSuccess) return e;
  FewArgs copy = a;
  void* params[] = {&copy};
  e = launch_pdl(reinterpret_cast<const void*>(fn), dim3(p.ctas), kFewWarps * 32, p.smem, ws.stream,
                 params, false);
  if (e == cudaSuccess) count_launch();
  return e;
}
template <bool kGrad, int kNT>
cudaError_t few_logits(const FewArgs& a, const FewPlan& p, uint32_t align, Workspace& ws) {
  return align == 16  ? few_logits<kGrad, kNT, 16>(a, p, ws)
         : align == 4 ? few_logits<kGrad, kNT, 4>(a, p, ws)
                      : few_logits<kGrad, kNT, 2>(a, p, ws);
}

template <int kNT, int kAlign>
cudaError_t few_grad(FewGradArgs& a, const DeviceInfo& dev, Workspace& ws) {
  void* params[] = {&a};
  const uint32_t tasks = a.windows * a.slices, sms = static_cast<uint32_t>(dev.sm_count);
  const uint32_t want = (tasks + kFewWarps - 1) / kFewWarps;
  const uint32_t grid = want > sms ? want : tasks < sms ? tasks : sms;
  const void* fn = reinterpret_cast<const void*>(&vocab_few_grad_kernel<kNT, kAlign>);
  constexpr int smem = kFewWarps * GradRing<kNT>::kBytes;
  static_assert(smem <= 227 * 1024, "the rings fit an SM");
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(fn, dim3(grid), kFewWarps * 32, smem, ws.stream, params, false);
  if (e == cudaSuccess) count_launch();
  return e;
}
template <int kNT>
cudaError_t few_grad(FewGradArgs& a, uint32_t align, const DeviceInfo& dev, Workspace& ws) {
  return align == 16  ? few_grad<kNT, 16>(a, dev, ws)
         : align == 4 ? few_grad<kNT, 4>(a, dev, ws)
                      : few_grad<kNT, 2>(a, dev, ws);
}

template <int kNT, int kAlign>
cudaError_t few_once(FewOnceArgs& a, const FewPlan& p, Workspace& ws) {
  void* params[] = {&a};
  const void* fn = reinterpret_cast<const void*>(&vocab_few_once_kernel<kNT, kAlign>);
  cudaError_t e =
      cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnceBytes);
  if (e != cudaSuccess) return e;
  e = launch_pdl(fn, dim3(p.slices), p.teams * p.windows * 32, p.teams * p.team_bytes, ws.stream, params, false);
  if (e == cudaSuccess) count_launch();
  return e;
}
template <int kNT>
cudaError_t few_once(FewOnceArgs& a, const FewPlan& p, uint32_t align, Workspace& ws) {
  return align == 16  ? few_once<kNT, 16>(a, p, ws)
         : align == 4 ? few_once<kNT, 4>(a, p, ws)
                      : few_once<kNT, 2>(a, p, ws);
}

FewArgs few_args(const VocabCall& c, const FewPlan& p, char* base, Workspace& ws) {
  FewArgs a = {};
  a.h = c.h;
  a.w = c.w;
  a.bias = c.bias;
  a.target = c.target;
  a.ldh = c.ldh;
  a.ldw = c.ldw;
  a.n = c.n;
  a.v = c.v;
  a.d = c.d;
  a.ld_s = p.ld_s;
  a.loss = c.loss;
  a.lse = c.lse;
  a.row_scale = c.row_scale;
  a.g = reinterpret_cast<uint32_t*>(base + p.g);
  a.dbias = c.dbias;
  a.pairs = reinterpret_cast<float2*>(base + p.pairs);
  a.at_target = reinterpret_cast<float*>(base + p.at_target);
  a.done = ws.model_arrivals();
  a.error = ws.u32(kOffError);
  return a;
}

}  // namespace

// h of all tokens fits an SM's shared memory beside the rings.
bool vocab_few(const VocabCall& c) {
  return c.n >= 1 && c.n <= 16 && (c.n <= 8 ? 8u : 16u) * (c.d + 72) * 2ull <= 72 * 1024;
}

size_t vocab_few_scratch(const VocabCall& c, bool gradient, const DeviceInfo& dev) {
  return few_plan(c, gradient, dev).total;
}

cudaError_t launch_vocab_few_loss(const VocabCall& c, Workspace& ws, const DeviceInfo& dev) {
  const FewPlan p = few_plan(c, false, dev);
  const FewArgs a = few_args(c, p, ws.model_scratch(), ws);
  const uint32_t align = std::min(row_align(c.w, c.ldw), 16u);
  return p.nt == 1 ? few_logits<false, 1>(a, p, align, ws) : few_logits<false, 2>(a, p, align, ws);
}

cudaError_t launch_vocab_few_grad(const VocabCall& c, Workspace& ws, const DeviceInfo& dev) {
  const FewPlan p = few_plan(c, true, dev);
  char* base = ws.model_scratch();
  const uint32_t align = std::min(row_align(c.w, c.ldw), 16u);
  const uint32_t align_dw = std::min(row_align(c.dw, c.lddw), 16u), ld = p.windows * kCols;
  float* sums = reinterpret_cast<float*>(base + p.sums);
  cudaError_t e;
  if (p.once) {
    FewOnceArgs g = {c.h,       c.w,        c.bias,         c.target,  c.lse,     c.row_scale, c.ldh,
                     c.ldw,     c.lddw,     c.n,            c.v,       c.d,       p.windows,   p.teams,
                     p.slice_groups,        c.dw,           c.dbias,   align_dw,  sums,        ld,
                     ws.u32(kOffError)};
    e = p.nt == 1 ? few_once<1>(g, p, align, ws) : few_once<2>(g, p, align, ws);
  } else {
    const FewArgs a = few_args(c, p, base, ws);
    e = p.nt == 1 ? few_logits<true, 1>(a, p, align, ws) : few_logits<true, 2>(a, p, align, ws);
    if (e != cudaSuccess) return e;
    FewGradArgs g = {c.h, c.w, c.target, c.lse, a.g, c.ldh, c.ldw, c.lddw, c.n, c.v, c.d,
                     p.windows, p.slices, p.slice_groups, c.dw, align_dw, sums, ld};
    e = p.nt == 1 ? few_grad<1>(g, align, dev, ws) : few_grad<2>(g, align, dev, ws);
  }
  if (e != cudaSuccess) return e;
  uint32_t slices = p.slices, tokens = 8 * p.nt, ld_sum = ld, cols = c.d;
  uint16_t* dh = c.dh;
  uint64_t ld_dh = c.lddh;
  const int64_t* target = c.target;
  const float* lse = c.lse;
  uint32_t v = c.v;
  void* params[] = {&sums, &slices, &tokens, &ld_sum, &cols, &dh, &ld_dh, &target, &lse, &v};
  e = launch_pdl(reinterpret_cast<const void*>(&vocab_few_dh_kernel), dim3((c.d + 31) / 32, c.n), 256, 0,
                 ws.stream, params, false);
  if (e == cudaSuccess) count_launch();
  return e;
}

}  // namespace efs
