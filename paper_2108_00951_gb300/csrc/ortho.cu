// ortho.cu — the orthogonalised update: momentum, then five Newton-Schulz
// steps on each weight matrix's update.
//
//   m <- mu m + u, U = u + m (the direction of the library's momentum step;
//   without m: U = u);  X = U / |U|_F;  on the shorter side, A = X X^T (or
//   X^T X),  B = b A + c A A,  X <- a X + B X  (X B),
//   a = 3.4445, b = -4.7750, c = 2.0315,
//
// which drives every singular value of U towards 1 (into about [0.7, 1.2])
// and leaves the singular vectors.
//
// All fifteen products of a call run in one cooperative launch, a grid barrier
// between, each over the tiles of every matrix. A and B are symmetric: only
// tiles that reach the diagonal are formed, entries above it are mirrored.
//
// Operands are fp16 with power-of-two scales (X 2^14, A and B 2^13: |X| <= 1.3
// throughout, so nothing overflows), which keeps 11 bits where bf16 keeps 8:
// the steps amplify small singular values up to 485 times, and with them any
// rounding. For the linear term a X the rounding that the fp16 operand leaves is
// kept too, 8 more bits of each entry (X phases are bound by the bytes they
// move: 6 an entry, where an fp32 copy beside the operand made it 10), so that
// directions the products hardly touch keep their bits; and B is kept as
// B + 2 I, whose diagonal (-0.8 to 2 instead of -2.8 to 0) rounds finer, the
// term -2 X moving into the linear one. Relative error of the result against
// 64 bits about 1e-3 (bf16 operands: 1e-2), below the rounding of the bf16
// output. A matrix whose shorter side is at most kExactSide has fewer
// roundings to average over: its operands are pairs hi + lo of fp16 (22 bits)
// and its products three (hi hi + hi lo + lo hi), within 1e-4; they are small
// enough for that to cost little. (Sums along a side of some 10^5 entries and more
// lose that again, as the tensor cores' additions truncate: 4e-4 at 128 x 200,000,
// 1.4e-3 at 1 x 2^20.)
//
// What bounds it: matrices of a few thousand a side the tensor cores and the
// power they draw (VGG-16's three fully connected ones 6.8 ms, 63 % of the burst
// rate of a library product, at the board's cap: 1358 W, 1.61 GHz). Smaller ones the phases: a grid barrier and the
// start of the pipeline take 3 us each, the join of K parts 4; and where the
// shorter side is a few hundred, L2: an X tile of 256 x 256 x 512 moves 450 KB
// through each SM in 4.9 us. 256 x 2304: 151 us, ten a phase; ResNet-18's 21
// matrices 370 (A 19.5, B 12, X 32.7 a step); six of 2600 x 650 375.
#include "product.cuh"

#include <algorithm>
#include <memory>
#include <vector>

#include <cuda_fp16.h>

namespace efs {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f, kNsShift = 2.0f;
constexpr float kScaleX = 16384.0f, kScaleA = 8192.0f;
constexpr int kSteps = 5;
constexpr uint32_t kExactSide = 128;

// The 8 bits that fp16 leaves of an fp32 value x: the difference of the two bit
// patterns, in units of 2^5 (x = its fp16 value, widened, + 32 rest, as
// integers). Where fp16 is subnormal the difference saturates; those entries
// are below 2^-14 2^-14 of the largest.
__device__ __forceinline__ int rest_of(float x, float half) {
  return (__float_as_int(x) - __float_as_int(half) + 16) >> 5;
}
__device__ __forceinline__ uint32_t pack_rest(int a, int b, int c, int d) {
  uint32_t r;
  asm("{\n\t.reg .b32 t;\n\t"
      "cvt.pack.sat.s8.s32.b32 t, %4, %3, 0;\n\t"
      "cvt.pack.sat.s8.s32.b32 %0, %2, %1, t;\n\t}"
      : "=r"(r)
      : "r"(a), "r"(b), "r"(c), "r"(d));
  return r;
}
template <int kByte>
__device__ __forceinline__ float with_rest(float half, uint32_t word) {
  uint32_t rest;  // the byte, its sign extended
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(rest) : "r"(word), "n"(0x8880 | 0x1111 * kByte));
  return __int_as_float(__float_as_int(half) + static_cast<int>(rest << 5));
}
// Rests lie in blocks of 128 rows x 32 columns, 16 columns of all rows
// together, as the epilogues read and write them: contiguous per warp. Unit of
// (row, col / 16), in 16 bytes.
__device__ __forceinline__ uint64_t rest_at(uint32_t row, uint32_t col, uint32_t chunks) {
  return ((static_cast<uint64_t>(row / kTileM) * chunks + col / 32) * 2 + col % 32 / 16) * kTileM +
         row % kTileM;
}

// ---- momentum, norm, and the first X
constexpr uint32_t kMaxParts = 512;  // partial sums of squares per matrix
constexpr uint32_t kPrepMats = 48;   // matrices per launch
constexpr uint32_t kPrepCols = 64;   // a CTA takes blocks of 128 rows x 64 columns

struct PrepMat {
  const void* u;
  float* m;
  uint16_t* out;  // where the last step writes
  uint16_t* hi;   // X in fp16, scaled, rows ld_x apart
  uint16_t* lo;   // what hi leaves in fp16 (exact matrices), or nullptr
  uint4* rest;    // else its rests
  uint64_t ld_u, ld_m, ld_out;
  uint32_t rows, cols, ld_x;
  uint32_t chunks;         // 32-column blocks of a row
  uint32_t blocks, blocks_n;
  uint32_t blocks_per_cta;
  uint32_t index;          // in the groups' order
  uint32_t cta0;           // its first CTA of the launch
  uint32_t part0;          // its first partial sum
  uint32_t parts;
};
struct PrepArgs {
  PrepMat mat[kPrepMats];
  uint32_t mats;
  float mu;
  FF* parts;
  uint16_t** outs;     // tables of the results, by index
  uint64_t* ld_outs;
};

__device__ __forceinline__ uint32_t prep_mat(const PrepArgs& a) {
  uint32_t i = 0;
  while (i + 1 < a.mats && blockIdx.x >= a.mat[i + 1].cta0) ++i;
  return i;
}

// The direction U at four columns of a row (zeros past the matrix).
// kFirst: also writes the momentum back.
template <bool kBf16, bool kFirst>
__device__ __forceinline__ float4 direction(const PrepMat& t, float mu, uint32_t row, uint32_t col,
                                            bool vec) {
  float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (row >= t.rows || col >= t.cols) return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const uint16_t* ub = static_cast<const uint16_t*>(t.u) + row * t.ld_u + col;
  const float* uf = static_cast<const float*>(t.u) + row * t.ld_u + col;
  float* m = t.m ? t.m + row * t.ld_m + col : nullptr;
  if (vec && col + 4 <= t.cols) {
    if (kBf16) {
      const uint2 w = __ldg(reinterpret_cast<const uint2*>(ub));
      x[0] = __uint_as_float(w.x << 16), x[1] = __uint_as_float(w.x & 0xffff0000u);
      x[2] = __uint_as_float(w.y << 16), x[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
      const float4 p = __ldg(reinterpret_cast<const float4*>(uf));
      x[0] = p.x, x[1] = p.y, x[2] = p.z, x[3] = p.w;
    }
    if (m) {
      const float4 q = *reinterpret_cast<const float4*>(m);
      float mv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (kFirst) mv[j] = __fmaf_rn(mu, mv[j], x[j]);
        x[j] = __fadd_rn(x[j], mv[j]);
      }
      if (kFirst) *reinterpret_cast<float4*>(m) = make_float4(mv[0], mv[1], mv[2], mv[3]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (col + j >= t.cols) continue;
      x[j] = kBf16 ? bf16_bits_to_f32(__ldg(ub + j)) : __ldg(uf + j);
      if (m) {
        float mv = m[j];
        if (kFirst) {
          mv = __fmaf_rn(mu, mv, x[j]);
          m[j] = mv;
        }
        x[j] = __fadd_rn(x[j], mv);
      }
    }
  }
  return make_float4(x[0], x[1], x[2], x[3]);
}

template <bool kBf16>
__device__ __forceinline__ bool prep_vec(const PrepMat& t) {
  constexpr uint32_t size = kBf16 ? 2 : 4;
  return reinterpret_cast<uintptr_t>(t.u) % (4 * size) == 0 && t.ld_u % 4 == 0 &&
         reinterpret_cast<uintptr_t>(t.m) % 16 == 0 && t.ld_m % 4 == 0;
}

// Momentum and the sum of squares: fp32 over 8 rows' four entries, float-float
// from there (fixed order). A warp takes two rows of 64 columns at a time.
template <bool kBf16>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const __grid_constant__ PrepArgs a) {
  __shared__ FF s_ff[32];
  griddep_wait();
  const PrepMat& t = a.mat[prep_mat(a)];
  const uint32_t cta = blockIdx.x - t.cta0, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t lo = cta * t.blocks_per_cta, hi = min(lo + t.blocks_per_cta, t.blocks);
  const bool vec = prep_vec<kBf16>(t);
  FF total{0.0f, 0.0f};
  for (uint32_t b = lo; b < hi; ++b) {
    const uint32_t row0 = b / t.blocks_n * kTileM + warp * 16 + (lane >> 4);
    const uint32_t col = b % t.blocks_n * kPrepCols + (lane & 15u) * 4;
    float s = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const float4 x = direction<kBf16, true>(t, a.mu, row0 + 2 * i, col, vec);
      s = __fmaf_rn(x.x, x.x, __fmaf_rn(x.y, x.y, __fmaf_rn(x.z, x.z, __fmaf_rn(x.w, x.w, s))));
    }
    total = ff_add(total, FF{s, 0.0f});
  }
  total = block_sum_ff(total, s_ff);
  if (threadIdx.x == 0) {
    a.parts[t.part0 + cta] = total;
    if (cta == 0) {
      a.outs[t.index] = t.out;
      a.ld_outs[t.index] = t.ld_out;
    }
  }
}

__device__ __forceinline__ uint16_t half_bits(float x) {
  return __half_as_ushort(__float2half_rn(x));
}
__device__ __forceinline__ float half_of(float x) { return __half2float(__float2half_rn(x)); }
__device__ __forceinline__ float half_rest(float x) { return __fsub_rn(x, half_of(x)); }

// X = U / |U|_F, scaled: fp16 rows and what they leave.
template <bool kBf16>
__global__ void __launch_bounds__(256) ortho_start_kernel(const __grid_constant__ PrepArgs a) {
  __shared__ FF s_ff[32];
  __shared__ float s_inv;
  __shared__ float4 s_x[kPrepCols / 4][kTileM + 1];
  griddep_wait();
  const PrepMat& t = a.mat[prep_mat(a)];
  const uint32_t cta = blockIdx.x - t.cta0, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t lo = cta * t.blocks_per_cta, hi = min(lo + t.blocks_per_cta, t.blocks);
  const bool vec = prep_vec<kBf16>(t);
  const FF sum = sum_parts_ff(a.parts + t.part0, t.parts, s_ff);
  if (threadIdx.x == 0) {
    const double n = sqrt(ff_to_double(sum));
    s_inv = n == 0.0 ? 0.0f : static_cast<float>(static_cast<double>(kScaleX) / n);
  }
  __syncthreads();
  const float inv = s_inv;
  for (uint32_t b = lo; b < hi; ++b) {
    const uint32_t tile = b / t.blocks_n, col0 = b % t.blocks_n * kPrepCols;
    const uint32_t unit = lane & 15u, col = col0 + unit * 4;
    float4 x[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      x[i] = direction<kBf16, false>(t, a.mu, tile * kTileM + warp * 16 + (lane >> 4) + 2 * i, col, vec);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const uint32_t r = warp * 16 + (lane >> 4) + 2 * i, row = tile * kTileM + r;
      const float4 y = make_float4(__fmul_rn(x[i].x, inv), __fmul_rn(x[i].y, inv),
                                   __fmul_rn(x[i].z, inv), __fmul_rn(x[i].w, inv));
      s_x[unit][r] = y;
      if (row < t.rows && col < t.ld_x) {  // rows are padded
        const uint64_t at = static_cast<uint64_t>(row) * t.ld_x + col;
        *reinterpret_cast<uint2*>(t.hi + at) = make_uint2(pack_f16(y.x, y.y), pack_f16(y.z, y.w));
        if (t.lo)
          *reinterpret_cast<uint2*>(t.lo + at) =
              make_uint2(pack_f16(half_rest(y.x), half_rest(y.y)),
                         pack_f16(half_rest(y.z), half_rest(y.w)));
      }
    }
    if (t.lo) continue;  // (uniform)
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kPrepCols / 16 * kTileM; i += 256) {
      const uint32_t u = i / kTileM, r = i % kTileM;
      if (col0 + u * 16 >= t.chunks * 32) break;
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 y = s_x[u * 4 + j][r];
        w[j] = pack_rest(rest_of(y.x, half_of(y.x)), rest_of(y.y, half_of(y.y)),
                         rest_of(y.z, half_of(y.z)), rest_of(y.w, half_of(y.w)));
      }
      t.rest[rest_at(tile * kTileM + r, col0 + u * 16, t.chunks)] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncthreads();
  }
}

// ---- the products' epilogues
enum : uint32_t { kFormA = 0, kFormB = 1, kFormX = 2 };

__device__ __forceinline__ float2 unpack_f16(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ void pack_row(const float (&v)[32], uint32_t (&w)[16]) {
#pragma unroll
  for (int j = 0; j < 16; ++j) w[j] = pack_f16(v[2 * j], v[2 * j + 1]);
}
// 32 fp16 of a row (rows are padded to 32 bytes), from L2: other SMs wrote them
// in this launch.
__device__ __forceinline__ void load_row(const uint16_t* p, uint32_t left, uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (static_cast<uint32_t>(16 * i) < left)
      asm volatile("ld.relaxed.gpu.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(w[8 * i]), "=r"(w[8 * i + 1]), "=r"(w[8 * i + 2]), "=r"(w[8 * i + 3]),
                     "=r"(w[8 * i + 4]), "=r"(w[8 * i + 5]), "=r"(w[8 * i + 6]), "=r"(w[8 * i + 7])
                   : "l"(p + 16 * i)
                   : "memory");
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) w[8 * i + j] = 0;
  }
}

struct StepEpilogue {
  static constexpr bool kTurns = false;
  struct Params {
    uint32_t form;
    uint32_t exact;         // operands have a second plane
    uint32_t ld;            // of the fp16 result: rows padded to 16 columns
    uint32_t chunks;        // 32-column blocks of a row of `rest`
    uint64_t plane;         // fp16 elements of a plane of the result
    uint64_t rest_units;    // of a matrix in `rest`
    uint16_t* to;           // the fp16 result [batch][planes][rows][ld]
    const uint16_t* from;   // likewise: A (kFormB) or X (kFormX), of to's shape
    uint4* rest;            // kFormX: what `from` leaves; rewritten for `to`
    uint16_t* const* outs;  // the last step's results, by batch
    const uint64_t* ld_outs;
    uint32_t last_phase;
  };
  struct Smem {
    TurnSmem turn;
  };
  struct Row {};
  static __device__ __forceinline__ Row prepare(const ProductShape&, const Params&,
                                                const ProductItem&, uint32_t) {
    return {};
  }

  // A 32 x 32 block of a symmetric matrix on or below the diagonal, and its
  // mirror image.
  static __device__ __forceinline__ void store_symmetric(uint16_t* out, uint32_t ld, uint32_t n,
                                                         uint32_t r, uint32_t col0,
                                                         const float (&v)[32], Smem& s) {
    const uint32_t lane = threadIdx.x & 31, r0 = r - lane;
    if (r0 >= n) return;  // (uniform)
    uint32_t w[16];
    pack_row(v, w);
    if (col0 == r0) mirror_block(s.turn, w);
    if (r < n) store_row(out + static_cast<uint64_t>(r) * ld + col0, w, min(ld - col0, 32u));
    if (col0 < r0 && r < n) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        out[static_cast<uint64_t>(col0 + j) * ld + r] = half_bits(v[j]);
    }
  }

  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, uint32_t,
                                              Smem& s, const ProductAcc& acc, uint32_t phase, Row) {
    const uint32_t r = it.m0 + row, r0 = it.m0 + (row & ~31u);
    const uint32_t planes = e.exact ? 2 : 1;
    const uint16_t* from = e.from + it.batch * planes * e.plane + static_cast<uint64_t>(r) * e.ld;
    uint4* rests = e.rest + it.batch * e.rest_units +
                   static_cast<uint64_t>(it.m0 / kTileM) * e.chunks * (2 * kTileM) + row;
    uint16_t* to = e.to + it.batch * planes * e.plane;
    const bool last = e.form == kFormX && phase == e.last_phase;
    uint16_t* out = nullptr;
    uint64_t ld_out = 0;
    uint32_t align = 0;
    if (last) {
      out = e.outs[it.batch];
      ld_out = e.ld_outs[it.batch];
      const uint64_t low = reinterpret_cast<uintptr_t>(out) | (ld_out * 2);
      align = low % 32 == 0 ? 32 : low % 16 == 0 ? 16 : low % 4 == 0 ? 4 : 2;
    }
    const bool rows_exist = r0 < p.m;
    auto alive = [&](uint32_t c) {  // the warp's block has entries to store
      const uint32_t col0 = it.n0 + c * 32;
      return rows_exist && col0 < p.n && (e.form == kFormX || col0 <= r0 + 31);
    };
    uint32_t h[16], l[16];  // of `from`: fp16, and lo or rests; a block ahead of their use
    auto fetch = [&](uint32_t c) {
      if (e.form == kFormA || c >= acc.c1 || !alive(c)) return;
      const uint32_t col0 = it.n0 + c * 32, left = r < p.m ? e.ld - col0 : 0;
      load_row(from + col0, left, h);
      if (e.exact) {
        load_row(from + e.plane + col0, left, l);
      } else if (e.form == kFormX) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 y = __ldcg(rests + (static_cast<uint64_t>(col0 / 32) * 2 + i) * kTileM);
          l[4 * i] = y.x, l[4 * i + 1] = y.y, l[4 * i + 2] = y.z, l[4 * i + 3] = y.w;
        }
      }
    };
    fetch(acc.c0);
    for (uint32_t c = acc.c0; c < acc.c1; ++c) {
      const uint32_t col0 = it.n0 + c * 32;
      const bool live = alive(c);
      float v[32];
      acc.load(c, v);
      if (!live) {  // (uniform)
        fetch(c + 1);
        continue;
      }
      if (e.form == kFormX) {
        // the operand's rounding of x stands in the term that B + 2 I took over
        constexpr float kOp = -kNsShift;
        if (e.exact) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float2 hi = unpack_f16(h[j]), lo = unpack_f16(l[j]);
            const float x0 = __fadd_rn(hi.x, lo.x), x1 = __fadd_rn(hi.y, lo.y);
            v[2 * j] = __fmaf_rn(v[2 * j], 1.0f / kScaleA, __fmul_rn(kNsA + kOp, x0));
            v[2 * j + 1] = __fmaf_rn(v[2 * j + 1], 1.0f / kScaleA, __fmul_rn(kNsA + kOp, x1));
          }
        } else {
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            const float2 a = unpack_f16(h[j]), b = unpack_f16(h[j + 1]);
            const uint32_t w = l[j / 2];
            const float x0 = with_rest<0>(a.x, w), x1 = with_rest<1>(a.y, w);
            const float x2 = with_rest<2>(b.x, w), x3 = with_rest<3>(b.y, w);
            v[2 * j] = __fmaf_rn(v[2 * j], 1.0f / kScaleA, __fmaf_rn(kNsA, x0, __fmul_rn(kOp, a.x)));
            v[2 * j + 1] = __fmaf_rn(v[2 * j + 1], 1.0f / kScaleA, __fmaf_rn(kNsA, x1, __fmul_rn(kOp, a.y)));
            v[2 * j + 2] = __fmaf_rn(v[2 * j + 2], 1.0f / kScaleA, __fmaf_rn(kNsA, x2, __fmul_rn(kOp, b.x)));
            v[2 * j + 3] = __fmaf_rn(v[2 * j + 3], 1.0f / kScaleA, __fmaf_rn(kNsA, x3, __fmul_rn(kOp, b.y)));
          }
        }
        fetch(c + 1);
        uint32_t w[16];
        if (last) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            w[j] = pack_bf16(__fmul_rn(v[2 * j], 1.0f / kScaleX), __fmul_rn(v[2 * j + 1], 1.0f / kScaleX));
          const uint32_t cols = min(p.n - col0, 32u);
          if (align == 32 && cols % 16 == 0) {
            if (r < p.m) store_row(out + r * ld_out + col0, w, cols);
          } else {
            store_block<4>(s.turn, w, cols, align, [&](uint32_t i) -> uint16_t* {
              return r0 + i < p.m ? out + (r0 + i) * ld_out + col0 : nullptr;
            });
          }
          continue;
        }
        const uint32_t cols = min(e.ld - col0, 32u);
        uint16_t* row_to = to + static_cast<uint64_t>(r) * e.ld + col0;
        pack_row(v, w);
        if (!e.exact) {
          uint32_t q[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 a = unpack_f16(w[2 * j]), b = unpack_f16(w[2 * j + 1]);
            q[j] = pack_rest(rest_of(v[4 * j], a.x), rest_of(v[4 * j + 1], a.y),
                             rest_of(v[4 * j + 2], b.x), rest_of(v[4 * j + 3], b.y));
          }
          uint4* mine = rests + static_cast<uint64_t>(col0 / 32) * (2 * kTileM);
          __stcg(mine, make_uint4(q[0], q[1], q[2], q[3]));
          __stcg(mine + kTileM, make_uint4(q[4], q[5], q[6], q[7]));
        }
        if (r < p.m) store_row(row_to, w, cols);
        if (e.exact) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = half_rest(v[j]);
          pack_row(v, w);
          if (r < p.m) store_row(row_to + e.plane, w, cols);
        }
        continue;
      }
      if (e.form == kFormA) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __fmul_rn(v[j], kScaleA / (kScaleX * kScaleX));
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          // A as its products read it: errors of b A and c A A cancel in part
          float2 a = unpack_f16(h[j]);
          if (e.exact) {
            const float2 lo = unpack_f16(l[j]);
            a = make_float2(__fadd_rn(a.x, lo.x), __fadd_rn(a.y, lo.y));
          }
          v[2 * j] = __fmaf_rn(kNsB, a.x, __fmul_rn(v[2 * j], kNsC / kScaleA));
          v[2 * j + 1] = __fmaf_rn(kNsB, a.y, __fmul_rn(v[2 * j + 1], kNsC / kScaleA));
        }
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (col0 + j == r) v[j] = __fmaf_rn(kNsShift, kScaleA, v[j]);
        fetch(c + 1);
      }
      store_symmetric(to, e.ld, p.n, r, col0, v, s);
      if (e.exact) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = half_rest(v[j]);
        store_symmetric(to + e.plane, e.ld, p.n, r, col0, v, s);
      }
    }
  }
};

constexpr size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
constexpr uint32_t round_up(uint32_t x, uint32_t to) { return (x + to - 1) / to * to; }

// Entries of a launch, per group: A from either X, B, and X from either X.
enum : uint32_t { kEntryA = 0, kEntryB = 2, kEntryX = 3, kEntries = 5 };
constexpr uint32_t kOrthoGroups = 12;  // shapes per launch, at most

// Matrices of one shape: consecutive in scratch.
struct Group {
  uint32_t rows = 0, cols = 0, side = 0, ld_x = 0, ld_s = 0, planes = 1;
  std::vector<uint32_t> mats;
  size_t half[2] = {0, 0}, rest = 0, a = 0, b = 0;  // scratch offsets
  uint64_t rest_units = 0;              // of one matrix, 16 bytes each
  uint32_t first = 0;                   // its first matrix, in the groups' order
  ProductShape shape[3] = {};           // by form
  bool left() const { return rows <= cols; }
};

struct Plan {
  std::vector<Group> groups;
  size_t parts = 0, outs = 0, ld_outs = 0, join = 0, total = 0;
  bool pair = false;
};

// The products' shapes of groups [g0, g0 + count), which share a launch: each
// is planned for its share of the SMs.
void plan_groups(Plan& plan, size_t g0, size_t count, double sms) {
  double work[3] = {0.0, 0.0, 0.0};
  auto cost = [](const Group& g, int form) {
    const double s = g.side, x = static_cast<double>(g.rows) * g.cols;
    return g.mats.size() * (g.planes * 2 - 1) *
           (form == kFormA ? x * s * 0.5 : form == kFormB ? s * s * s * 0.5 : x * s);
  };
  for (size_t i = g0; i < g0 + count; ++i)
    for (int f = 0; f < 3; ++f) work[f] += cost(plan.groups[i], f);
  for (size_t i = g0; i < g0 + count; ++i) {
    Group& g = plan.groups[i];
    const uint32_t batch = static_cast<uint32_t>(g.mats.size()), terms = g.planes * 2 - 1;
    const uint32_t deep = g.left() ? g.cols : g.rows;
    const ProductWant want[3] = {
        {g.side, g.side, deep, batch, true, plan.pair, 0.0, 16, terms, 20.0, true},
        {g.side, g.side, g.side, batch, true, plan.pair, 0.0, 8, terms, 20.0, true},
        {g.rows, g.cols, g.side, batch, false, plan.pair, 0.0, 1, terms, 40.0, true}};
    for (int f = 0; f < 3; ++f) {
      ProductWant w = want[f];
      w.sms = cost(g, f) / work[f] * sms;
      if (w.sms < 1.0) w.sms = 1.0;
      plan_product(g.shape[f], w);
    }
  }
}

// Lays them out as a launch's entries and phases; returns the bytes of the
// scratch that joining K parts takes.
template <class Args>
size_t shape_products(Args& args, const Plan& plan, size_t g0, uint32_t count) {
  for (uint32_t i = 0; i < count; ++i) {
    const ProductShape* s = plan.groups[g0 + i].shape;
    args.shape[kEntryA * count + i] = args.shape[(kEntryA + 1) * count + i] = s[kFormA];
    args.shape[kEntryB * count + i] = s[kFormB];
    args.shape[kEntryX * count + i] = args.shape[(kEntryX + 1) * count + i] = s[kFormX];
  }
  args.phases = 3 * kSteps;
  for (uint32_t ph = 0; ph < args.phases; ++ph) {
    const uint32_t form = ph % 3, from = (ph / 3) & 1u;
    const uint32_t entry = form == kFormA ? kEntryA + from : form == kFormB ? kEntryB : kEntryX + from;
    args.first[ph] = entry * count;
    args.problems[ph] = count;
  }
  return number_items(args, plan.pair, kPartCounters);
}

// Kernel parameters for 1, 4 or kOrthoGroups shapes: a launch copies them.
template <int kGroups>
using StepArgs = ProductArgs<StepEpilogue, static_cast<int>(kEntries) * kGroups>;

Plan make_plan(const OrthoMat* mats, uint32_t n, const DeviceInfo& dev) {
  Plan p;
  const double sms = dev.sm_count;
  double items = 0.0;
  for (uint32_t i = 0; i < n; ++i) {
    if (mats[i].rows == 0 || mats[i].cols == 0) continue;
    Group* g = nullptr;
    for (Group& x : p.groups)
      if (x.rows == mats[i].rows && x.cols == mats[i].cols) g = &x;
    if (!g) {
      p.groups.emplace_back();
      g = &p.groups.back();
      g->rows = mats[i].rows;
      g->cols = mats[i].cols;
      g->side = g->rows < g->cols ? g->rows : g->cols;
      // rows on lines of 128 bytes, which TMA reads whole (650 columns: 383 -> 371 us)
      g->ld_x = round_up(g->cols, 64);
      g->ld_s = round_up(g->side, 64);
      g->planes = g->side <= kExactSide ? 2 : 1;
    }
    g->mats.push_back(i);
    const double pairs = (g->side + 255) / 256;
    items += pairs * (pairs + 1) / 2;
  }
  // Pairs of CTAs (256 x 256 tiles) once the symmetric products, which have the
  // fewest tiles, fill them.
  p.pair = items >= sms / 2;
  // the deepest products first: their tiles take longest
  std::stable_sort(p.groups.begin(), p.groups.end(), [](const Group& x, const Group& y) {
    return x.side != y.side ? x.side > y.side
                            : static_cast<uint64_t>(x.rows) * x.cols >
                                  static_cast<uint64_t>(y.rows) * y.cols;
  });
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  uint32_t all = 0;
  for (Group& g : p.groups) {
    const size_t batch = g.mats.size();
    const size_t x = 2ull * batch * g.planes * g.rows * g.ld_x;
    const size_t s = 2ull * batch * g.planes * g.side * g.ld_s;
    for (int i = 0; i < 2; ++i) g.half[i] = take(x);
    if (g.planes == 1) {
      g.rest_units = static_cast<uint64_t>(round_up(g.rows, kTileM)) * round_up(g.cols, 32) / 16;
      g.rest = take(16 * batch * g.rest_units);
    }
    g.a = take(s);
    g.b = take(s);
    g.first = all;
    all += static_cast<uint32_t>(batch);
  }
  p.parts = take(sizeof(FF) * kMaxParts * all);
  p.outs = take(8ull * all);
  p.ld_outs = take(8ull * all);
  size_t join = 0;
  for (size_t g0 = 0; g0 < p.groups.size(); g0 += kOrthoGroups) {
    const size_t left = p.groups.size() - g0;
    const uint32_t count = static_cast<uint32_t>(left < kOrthoGroups ? left : kOrthoGroups);
    plan_groups(p, g0, count, sms);
    std::unique_ptr<StepArgs<kOrthoGroups>> args(new StepArgs<kOrthoGroups>);
    args->phases = args->entries = 0;
    const size_t bytes = shape_products(*args, p, g0, count);
    if (bytes > join) join = bytes;
  }
  p.join = take(join);
  p.total = at;
  return p;
}

template <class Fn>
cudaError_t launch_prep(Fn fn, PrepArgs& a, uint32_t ctas, cudaStream_t stream) {
  void* params[] = {&a};
  const cudaError_t e = launch_pdl(reinterpret_cast<const void*>(fn), dim3(ctas), 256, 0, stream,
                                   params, false);
  if (e == cudaSuccess) count_launch();
  return e;
}

// Momentum, norms and the first X of every matrix.
cudaError_t prepare(const OrthoMat* mats, const Plan& plan, bool bf16, float mu, char* base,
                    Workspace& ws) {
  PrepArgs prep = {};
  prep.mu = mu;
  prep.parts = reinterpret_cast<FF*>(base + plan.parts);
  prep.outs = reinterpret_cast<uint16_t**>(base + plan.outs);
  prep.ld_outs = reinterpret_cast<uint64_t*>(base + plan.ld_outs);
  uint32_t ctas = 0, index = 0;
  auto flush = [&]() {
    if (prep.mats == 0) return cudaSuccess;
    cudaError_t e = bf16 ? launch_prep(&ortho_norm_kernel<true>, prep, ctas, ws.stream)
                         : launch_prep(&ortho_norm_kernel<false>, prep, ctas, ws.stream);
    if (e == cudaSuccess)
      e = bf16 ? launch_prep(&ortho_start_kernel<true>, prep, ctas, ws.stream)
               : launch_prep(&ortho_start_kernel<false>, prep, ctas, ws.stream);
    prep.mats = ctas = 0;
    return e;
  };
  for (const Group& g : plan.groups) {
    for (size_t b = 0; b < g.mats.size(); ++b, ++index) {
      const OrthoMat& m = mats[g.mats[b]];
      PrepMat& t = prep.mat[prep.mats++];
      t.u = m.u;
      t.m = m.m;
      t.out = m.out;
      t.ld_u = m.ld_u;
      t.ld_m = m.ld_m;
      t.ld_out = m.ld_out;
      t.rest = reinterpret_cast<uint4*>(base + g.rest) + b * g.rest_units;
      t.hi = reinterpret_cast<uint16_t*>(base + g.half[0]) +
             b * g.planes * g.rows * static_cast<uint64_t>(g.ld_x);
      t.lo = g.planes == 2 ? t.hi + g.rows * static_cast<uint64_t>(g.ld_x) : nullptr;
      t.rows = m.rows;
      t.cols = m.cols;
      t.ld_x = g.ld_x;
      t.chunks = round_up(g.cols, 32) / 32;
      t.blocks_n = (m.cols + kPrepCols - 1) / kPrepCols;
      t.blocks = (m.rows + kTileM - 1) / kTileM * t.blocks_n;
      t.blocks_per_cta = (t.blocks + kMaxParts - 1) / kMaxParts;
      t.index = index;
      t.cta0 = ctas;
      t.part0 = index * kMaxParts;
      t.parts = (t.blocks + t.blocks_per_cta - 1) / t.blocks_per_cta;
      ctas += t.parts;
      if (prep.mats == kPrepMats) {
        const cudaError_t e = flush();
        if (e != cudaSuccess) return e;
      }
    }
  }
  return flush();
}

// The products of `count` groups from `g0`, all steps.
template <int kGroups>
cudaError_t steps(const Plan& plan, size_t g0, uint32_t count, char* base, Workspace& ws,
                  const DeviceInfo& dev) {
  std::unique_ptr<StepArgs<kGroups>> held(new StepArgs<kGroups>());
  StepArgs<kGroups>& args = *held;
  shape_products(args, plan, g0, count);
  const bool pair = plan.pair;
  bool ok = true;
  for (uint32_t i = 0; i < count; ++i) {
    const Group& g = plan.groups[g0 + i];
    const bool left = g.left();
    const uint64_t batch = g.mats.size() * g.planes;
    struct {
      size_t at;
      uint32_t box;
      const CUtensorMap* map;
    } known[8];
    int maps = 0;
    auto map = [&](CUtensorMap* to, size_t at, bool square, uint32_t box) {
      for (int k = 0; k < maps; ++k)
        if (known[k].at == at && known[k].box == box) {  // encoding one costs more than a copy
          *to = *known[k].map;
          return;
        }
      if (maps < 8) known[maps++] = {at, box, to};
      const uint32_t rows = square ? g.side : g.rows, cols = square ? g.side : g.cols;
      const uint32_t ld = square ? g.ld_s : g.ld_x;
      ok = ok && make_map(to, base + at, false, cols, rows, ld, batch,
                          static_cast<uint64_t>(rows) * ld, box);
    };
    StepEpilogue::Params e = {};
    e.exact = g.planes == 2 ? 1u : 0u;
    e.last_phase = 3 * kSteps - 1;
    e.outs = reinterpret_cast<uint16_t* const*>(base + plan.outs) + g.first;
    e.ld_outs = reinterpret_cast<const uint64_t*>(base + plan.ld_outs) + g.first;
    for (uint32_t from = 0; from < 2; ++from) {
      {
        ProductShape& s = args.shape[(kEntryA + from) * count + i];
        s.a_mn = s.b_mn = left ? 0u : 1u;
        map(&s.a, g.half[from], false, kTileM);
        map(&s.b, g.half[from], false, left ? b_box(s, pair) : kTileK);
        e.form = kFormA;
        e.ld = g.ld_s;
        e.plane = static_cast<uint64_t>(g.side) * g.ld_s;
        e.to = reinterpret_cast<uint16_t*>(base + g.a);
        e.from = e.to;  // (not read)
        args.epi[(kEntryA + from) * count + i] = e;
      }
      if (from == 0) {
        ProductShape& s = args.shape[kEntryB * count + i];
        map(&s.a, g.a, true, kTileM);
        map(&s.b, g.a, true, b_box(s, pair));
        e.form = kFormB;
        e.from = e.to;
        e.to = reinterpret_cast<uint16_t*>(base + g.b);
        args.epi[kEntryB * count + i] = e;
      }
      ProductShape& s = args.shape[(kEntryX + from) * count + i];
      if (left) {  // B X: X is MN-major
        s.b_mn = 1;
        map(&s.a, g.b, true, kTileM);
        map(&s.b, g.half[from], false, kTileK);
      } else {  // X B: B is symmetric, its rows are its columns
        map(&s.a, g.half[from], false, kTileM);
        map(&s.b, g.b, true, b_box(s, pair));
      }
      e.form = kFormX;
      e.ld = g.ld_x;
      e.chunks = round_up(g.cols, 32) / 32;
      e.plane = static_cast<uint64_t>(g.rows) * g.ld_x;
      e.rest_units = g.rest_units;
      e.from = reinterpret_cast<const uint16_t*>(base + g.half[from]);
      e.to = reinterpret_cast<uint16_t*>(base + g.half[from ^ 1u]);
      e.rest = reinterpret_cast<uint4*>(base + g.rest);
      args.epi[(kEntryX + from) * count + i] = e;
    }
  }
  if (!ok) return cudaErrorInvalidValue;
  args.parts = reinterpret_cast<float*>(base + plan.join);
  return pair ? launch_product<StepEpilogue, kEntries * kGroups, true>(args, ws, dev)
              : launch_product<StepEpilogue, kEntries * kGroups, false>(args, ws, dev);
}

}  // namespace

size_t ortho_plan(const OrthoMat* mats, uint32_t n, const DeviceInfo& dev,
                  std::shared_ptr<void>* plan) {
  if (ortho_small(mats, n, dev)) return 0;  // no plan, no scratch
  auto p = std::make_shared<Plan>(make_plan(mats, n, dev));
  *plan = p;
  return p->total;
}

cudaError_t launch_orthogonalize(const OrthoMat* mats, uint32_t n, bool bf16, float mu,
                                 const void* made, Workspace& ws, const DeviceInfo& dev) {
  if (!made) return launch_ortho_small(mats, n, bf16, mu, ws, dev);
  const Plan& plan = *static_cast<const Plan*>(made);
  char* base = ws.model_scratch();
  cudaError_t e = prepare(mats, plan, bf16, mu, base, ws);
  for (size_t g0 = 0; g0 < plan.groups.size() && e == cudaSuccess; g0 += kOrthoGroups) {
    const size_t left = plan.groups.size() - g0;
    const uint32_t count = static_cast<uint32_t>(left < kOrthoGroups ? left : kOrthoGroups);
    e = count == 1 ? steps<1>(plan, g0, count, base, ws, dev)
        : count <= 4 ? steps<4>(plan, g0, count, base, ws, dev)
                     : steps<kOrthoGroups>(plan, g0, count, base, ws, dev);
  }
  return e;
}

}  // namespace efs
