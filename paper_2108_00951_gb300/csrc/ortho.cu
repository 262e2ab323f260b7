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
// All matrices of a call go through each product together: a launch holds
// the tiles of every matrix. A and B are symmetric: only tiles that reach the
// diagonal are formed, entries above it are mirrored.
//
// Operands are fp16 with power-of-two scales (X 2^14, A and B 2^13: |X| <= 1,
// so nothing overflows), which keeps 11 bits where bf16 keeps 8: the steps
// amplify small singular values up to 485 times, and with them any rounding.
// X is kept as a pair H + L of fp16 (22 bits): the products read H, the
// linear term a X reads both, so that directions the products hardly touch
// keep their bits. B's diagonal, -2.8 to 0, is kept as B + 2 I, whose entries
// round finer; the term -2 I moves into the linear term. Relative error of the result
// against 64 bits about 1e-3 (bf16 operands: 1e-2), below the rounding of the
// bf16 output.
#include "product.cuh"

#include <algorithm>
#include <vector>

#include <cuda_fp16.h>

namespace efs {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f, kNsShift = 2.0f;
constexpr float kScaleX = 16384.0f, kScaleA = 8192.0f;
constexpr int kSteps = 5;

// ---- momentum, norm, and the first H + L
constexpr uint32_t kSegment = 256;   // columns of a row that a warp takes at a time
constexpr uint32_t kMaxParts = 512;  // partial sums of squares per matrix
constexpr uint32_t kPrepMats = 48;   // matrices per launch

struct PrepMat {
  const void* u;
  float* m;
  uint16_t* hi;   // fp16, rows ld_x apart
  uint16_t* lo;
  uint16_t* out;  // where the last step writes
  uint64_t ld_u, ld_m, ld_out;
  uint32_t rows, cols, ld_x;
  uint32_t index;          // in the groups' order
  uint32_t units_per_cta;  // (row, segment) units
  uint32_t cta0;           // its first CTA of the launch
  uint32_t part0;          // its first partial sum
  uint32_t parts;
};
struct PrepArgs {
  PrepMat mat[kPrepMats];
  uint32_t mats;
  uint32_t bf16;
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

// The direction U at 8 columns of a row: 8 in a row per lane where the rows
// allow 16-byte accesses (col0 = first column of the lane's 8), else 32 apart.
// kFirst: also writes the momentum back.
template <bool kBf16, bool kFirst>
__device__ __forceinline__ void direction(const PrepMat& t, float mu, uint32_t row, uint32_t seg,
                                          bool vec, float (&x)[8], uint32_t (&col)[8]) {
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t c0 = seg * kSegment;
#pragma unroll
  for (int j = 0; j < 8; ++j) col[j] = vec ? c0 + lane * 8 + j : c0 + j * 32 + lane;
  const uint64_t base_u = row * t.ld_u, base_m = row * t.ld_m;
  const uint16_t* ub = static_cast<const uint16_t*>(t.u) + base_u;
  const float* uf = static_cast<const float*>(t.u) + base_u;
  if (vec && col[0] + 8 <= t.cols) {
    if (kBf16) {
      const uint4 w = __ldg(reinterpret_cast<const uint4*>(ub + col[0]));
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(ws[j] << 16);
        x[2 * j + 1] = __uint_as_float(ws[j] & 0xffff0000u);
      }
    } else {
      const float4 p = __ldg(reinterpret_cast<const float4*>(uf + col[0]));
      const float4 q = __ldg(reinterpret_cast<const float4*>(uf + col[0]) + 1);
      x[0] = p.x, x[1] = p.y, x[2] = p.z, x[3] = p.w;
      x[4] = q.x, x[5] = q.y, x[6] = q.z, x[7] = q.w;
    }
    if (t.m) {
      float4* mp = reinterpret_cast<float4*>(t.m + base_m + col[0]);
      float4 p = mp[0], q = mp[1];
      float mv[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (kFirst) mv[j] = __fmaf_rn(mu, mv[j], x[j]);
        x[j] = __fadd_rn(x[j], mv[j]);
      }
      if (kFirst) {
        mp[0] = make_float4(mv[0], mv[1], mv[2], mv[3]);
        mp[1] = make_float4(mv[4], mv[5], mv[6], mv[7]);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = 0.0f;
      if (col[j] < t.cols) {
        x[j] = kBf16 ? bf16_bits_to_f32(__ldg(ub + col[j])) : __ldg(uf + col[j]);
        if (t.m) {
          float* mp = t.m + base_m + col[j];
          float mv = *mp;
          if (kFirst) {
            mv = __fmaf_rn(mu, mv, x[j]);
            *mp = mv;
          }
          x[j] = __fadd_rn(x[j], mv);
        }
      }
    }
  }
}

__device__ __forceinline__ bool prep_vec(const PrepMat& t, bool bf16) {
  const uint32_t size = bf16 ? 2 : 4;
  return reinterpret_cast<uintptr_t>(t.u) % 16 == 0 && t.ld_u * size % 16 == 0 &&
         reinterpret_cast<uintptr_t>(t.m) % 16 == 0 && t.ld_m % 4 == 0;
}

// Momentum and the sum of squares: fp32 over 8 entries, float-float from there
// (fixed order).
template <bool kBf16>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const __grid_constant__ PrepArgs a) {
  __shared__ FF s_ff[32];
  griddep_wait();
  const PrepMat& t = a.mat[prep_mat(a)];
  const uint32_t cta = blockIdx.x - t.cta0, segs = (t.cols + kSegment - 1) / kSegment;
  const uint64_t units = static_cast<uint64_t>(t.rows) * segs;
  const uint64_t lo = static_cast<uint64_t>(cta) * t.units_per_cta;
  const uint64_t hi = lo + t.units_per_cta < units ? lo + t.units_per_cta : units;
  const bool vec = prep_vec(t, kBf16);
  FF total{0.0f, 0.0f};
  for (uint64_t i = lo + (threadIdx.x >> 5); i < hi; i += 8) {
    float x[8];
    uint32_t col[8];
    direction<kBf16, true>(t, a.mu, static_cast<uint32_t>(i / segs),
                           static_cast<uint32_t>(i % segs), vec, x, col);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __fmaf_rn(x[j], x[j], s);
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

// X = U / |U|_F as H + L, scaled by 2^14.
template <bool kBf16>
__global__ void __launch_bounds__(256) ortho_start_kernel(const __grid_constant__ PrepArgs a) {
  __shared__ FF s_ff[32];
  __shared__ float s_inv;
  griddep_wait();
  const PrepMat& t = a.mat[prep_mat(a)];
  const uint32_t cta = blockIdx.x - t.cta0, segs = (t.cols + kSegment - 1) / kSegment;
  const uint64_t units = static_cast<uint64_t>(t.rows) * segs;
  const uint64_t lo = static_cast<uint64_t>(cta) * t.units_per_cta;
  const uint64_t hi = lo + t.units_per_cta < units ? lo + t.units_per_cta : units;
  const bool vec = prep_vec(t, kBf16);
  const FF sum = sum_parts_ff(a.parts + t.part0, t.parts, s_ff);
  if (threadIdx.x == 0) {
    const double n = sqrt(ff_to_double(sum));
    s_inv = n == 0.0 ? 0.0f : static_cast<float>(static_cast<double>(kScaleX) / n);
  }
  __syncthreads();
  const float inv = s_inv;
  for (uint64_t i = lo + (threadIdx.x >> 5); i < hi; i += 8) {
    float x[8];
    uint32_t col[8];
    const uint32_t row = static_cast<uint32_t>(i / segs);
    direction<kBf16, false>(t, a.mu, row, static_cast<uint32_t>(i % segs), vec, x, col);
    uint16_t h[8], l[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float y = __fmul_rn(x[j], inv);
      const __half hh = __float2half_rn(y);
      h[j] = __half_as_ushort(hh);
      l[j] = __half_as_ushort(__float2half_rn(__fsub_rn(y, __half2float(hh))));
    }
    uint16_t* to_h = t.hi + static_cast<uint64_t>(row) * t.ld_x;
    uint16_t* to_l = t.lo + static_cast<uint64_t>(row) * t.ld_x;
    if (vec && col[0] + 8 <= t.cols) {
      *reinterpret_cast<uint4*>(to_h + col[0]) =
          make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
      *reinterpret_cast<uint4*>(to_l + col[0]) =
          make_uint4(l[0] | (l[1] << 16), l[2] | (l[3] << 16), l[4] | (l[5] << 16), l[6] | (l[7] << 16));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col[j] < t.cols) {
          to_h[col[j]] = h[j];
          to_l[col[j]] = l[j];
        }
    }
  }
}

// ---- the three products' epilogues
__device__ __forceinline__ float2 half2_at(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// 32 fp16 of a row from scratch (rows padded to 8 columns: 16-byte accesses;
// columns past the padding are left alone).
__device__ __forceinline__ void load_half_row(const uint16_t* p, uint32_t left, float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (static_cast<uint32_t>(8 * j) < left) w = __ldcg(reinterpret_cast<const uint4*>(p) + j);
    const float2 a = half2_at(w.x), b = half2_at(w.y), c = half2_at(w.z), d = half2_at(w.w);
    v[8 * j] = a.x, v[8 * j + 1] = a.y, v[8 * j + 2] = b.x, v[8 * j + 3] = b.y;
    v[8 * j + 4] = c.x, v[8 * j + 5] = c.y, v[8 * j + 6] = d.x, v[8 * j + 7] = d.y;
  }
}
__device__ __forceinline__ void store_half_row(uint16_t* p, uint32_t left, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (static_cast<uint32_t>(8 * j) < left)
      *(reinterpret_cast<uint4*>(p) + j) =
          make_uint4(pack_f16(v[8 * j], v[8 * j + 1]), pack_f16(v[8 * j + 2], v[8 * j + 3]),
                     pack_f16(v[8 * j + 4], v[8 * j + 5]), pack_f16(v[8 * j + 6], v[8 * j + 7]));
}

// The symmetric products: out = A (kSecond: out = B + 2 I), entries on and
// below the diagonal stored as computed, those below also mirrored.
template <bool kSecond>
struct SymmetricEpilogue {
  struct Params {
    const uint16_t* a;  // kSecond: A
    uint16_t* out;
    uint32_t ld;
    uint64_t batch_ld;
  };
  struct Smem {};
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, Smem&,
                                              const ProductAcc& acc) {
    const uint32_t r = it.m0 + row;
    const uint64_t base = it.batch * e.batch_ld;
    uint16_t* out = e.out + base;
    for (uint32_t c = 0; c < acc.chunks; ++c) {
      float v[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      if (r >= p.m || col0 > r) continue;
      if (kSecond) {
        float a[32];
        load_half_row(e.a + base + static_cast<uint64_t>(r) * e.ld + col0, e.ld - col0, a);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          v[j] = __fmaf_rn(kNsB, a[j], __fmul_rn(v[j], kNsC / kScaleA));
          if (col0 + j == r) v[j] = __fmaf_rn(kNsShift, kScaleA, v[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __fmul_rn(v[j], kScaleA / (kScaleX * kScaleX));
      }
      if (col0 + 31 <= r) {
        store_half_row(out + static_cast<uint64_t>(r) * e.ld + col0, 32, v);
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (col0 + j <= r)
            out[static_cast<uint64_t>(r) * e.ld + col0 + j] = __half_as_ushort(__float2half_rn(v[j]));
      }
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (col0 + j < r)
          out[static_cast<uint64_t>(col0 + j) * e.ld + r] = __half_as_ushort(__float2half_rn(v[j]));
    }
  }
};

constexpr uint32_t kOrthoGroups = 16;  // shapes per launch

// X <- a X + B X, as H + L; the last step writes the result in bf16.
struct StepEpilogue {
  struct Params {
    const uint16_t *h, *l;
    uint16_t *h_out, *l_out;
    uint32_t ld;
    uint64_t batch_ld;
    uint16_t* const* outs;  // the last step: device table of the results, by batch
    const uint64_t* ld_outs;
  };
  struct Smem {
    uint32_t turn[4][32 * 17];
  };
  static __device__ __forceinline__ void tile(const ProductShape& p, const Params& e,
                                              const ProductItem& it, uint32_t row, Smem& s,
                                              const ProductAcc& acc) {
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t r = it.m0 + row;
    const bool real = r < p.m;
    const uint64_t base = it.batch * e.batch_ld + static_cast<uint64_t>(real ? r : 0) * e.ld;
    uint16_t* out = nullptr;
    uint64_t ld_out = 0;
    if (e.outs) {
      out = e.outs[it.batch];
      ld_out = e.ld_outs[it.batch];
    }
    const bool vec = reinterpret_cast<uintptr_t>(out) % 16 == 0 && ld_out % 8 == 0;
    uint32_t* turn = s.turn[(threadIdx.x >> 5) & 3u];
    for (uint32_t c = 0; c < acc.chunks; ++c) {
      float v[32], x[32];
      acc.load(c, v);
      const uint32_t col0 = it.n0 + c * 32;
      if (col0 >= p.n) continue;  // (uniform: the last chunk may lie past the columns)
      const uint32_t left = real ? e.ld - col0 : 0;
      load_half_row(e.l + base + col0, left, x);
#pragma unroll
      for (int j = 0; j < 32; ++j)
        v[j] = __fmaf_rn(kNsA, x[j], __fmul_rn(v[j], 1.0f / kScaleA));
      load_half_row(e.h + base + col0, left, x);
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = __fmaf_rn(kNsA - kNsShift, x[j], v[j]);
      if (!e.outs) {
        if (real) {
          store_half_row(e.h_out + base + col0, left, v);
#pragma unroll
          for (int j = 0; j < 32; ++j)
            v[j] = __fsub_rn(v[j], __half2float(__float2half_rn(v[j])));
          store_half_row(e.l_out + base + col0, left, v);
        }
        continue;
      }
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        w[j] = pack_bf16(__fmul_rn(v[2 * j], 1.0f / kScaleX), __fmul_rn(v[2 * j + 1], 1.0f / kScaleX));
      if (vec && col0 + 32 <= p.n) {
        if (real) {
          uint4* to = reinterpret_cast<uint4*>(out + r * ld_out + col0);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            to[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
        }
        continue;
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 16; ++j) turn[lane * 17 + j] = w[j];
      __syncwarp();
      const uint32_t r0 = r - lane, rows = p.m - min(p.m, r0);
      if (col0 + lane < p.n)
        for (uint32_t i = 0; i < 32 && i < rows; ++i)
          out[(r0 + i) * ld_out + col0 + lane] = reinterpret_cast<const uint16_t*>(turn + i * 17)[lane];
    }
  }
};

constexpr size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
constexpr uint32_t round_up(uint32_t x, uint32_t to) { return (x + to - 1) / to * to; }

// Matrices of one shape: consecutive in scratch, one entry of a launch.
struct Group {
  uint32_t rows = 0, cols = 0, side = 0, ld_x = 0, ld_s = 0;
  std::vector<uint32_t> mats;
  size_t hi[2] = {0, 0}, lo[2] = {0, 0}, a = 0, b = 0;  // scratch offsets
  uint32_t first = 0;  // its first matrix, in the groups' order
};

struct Plan {
  std::vector<Group> groups;
  // of each phase and group: A, B, X
  std::vector<ProductShape> shape[3];
  size_t parts = 0, outs = 0, ld_outs = 0, join = 0, total = 0;
};

Plan make_plan(const OrthoMat* mats, uint32_t n, uint32_t sms) {
  Plan p;
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
      g->ld_x = round_up(g->cols, 8);
      g->ld_s = round_up(g->side, 8);
    }
    g->mats.push_back(i);
  }
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
  double work[3] = {0.0, 0.0, 0.0};
  auto cost = [](const Group& g, int phase) {
    const double s = g.side, x = static_cast<double>(g.rows) * g.cols;
    return g.mats.size() * (phase == 0 ? x * s * 0.5 : phase == 1 ? s * s * s * 0.5 : x * s);
  };
  for (Group& g : p.groups) {
    const size_t batch = g.mats.size();
    const size_t x = 2ull * batch * g.rows * g.ld_x, s = 2ull * batch * g.side * g.ld_s;
    for (int i = 0; i < 2; ++i) {
      g.hi[i] = take(x);
      g.lo[i] = take(x);
    }
    g.a = take(s);
    g.b = take(s);
    g.first = all;
    all += static_cast<uint32_t>(batch);
    for (int ph = 0; ph < 3; ++ph) work[ph] += cost(g, ph);
  }
  p.parts = take(sizeof(FF) * kMaxParts * all);
  p.outs = take(8ull * all);
  p.ld_outs = take(8ull * all);
  size_t join = 0;
  for (int ph = 0; ph < 3; ++ph) {
    size_t slots = 0, chunks = 0, most = 0;
    for (size_t i = 0; i < p.groups.size(); ++i) {
      const Group& g = p.groups[i];
      ProductShape s = {};
      const double share = cost(g, ph) / work[ph] * sms;
      const uint32_t mine = share < 1.0 ? 1u : static_cast<uint32_t>(share);
      const uint32_t batch = static_cast<uint32_t>(g.mats.size());
      const uint32_t splits = 8;
      if (ph == 0)
        plan_product(s, g.side, g.side, g.rows < g.cols ? g.cols : g.rows, batch, true, mine, splits);
      else if (ph == 1)
        plan_product(s, g.side, g.side, g.side, batch, true, mine, splits);
      else
        plan_product(s, g.rows, g.cols, g.side, batch, false, mine, splits);
      if (s.splits > 1) {
        slots += static_cast<size_t>(s.tiles) * s.batch * s.splits;
        if ((s.bn + 31) / 32 > chunks) chunks = (s.bn + 31) / 32;
      }
      p.shape[ph].push_back(s);
      if (i % kOrthoGroups == kOrthoGroups - 1 || i + 1 == p.groups.size()) {  // one launch
        const size_t bytes = 4ull * kTileM * 32 * chunks * slots;
        if (bytes > most) most = bytes;
        slots = chunks = 0;
      }
    }
    if (most > join) join = most;
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

bool operand(CUtensorMap* map, const char* base, uint64_t cols, uint64_t rows, uint64_t ld,
             uint64_t batch, uint32_t box) {
  return make_map(map, base, false, cols, rows, ld, batch, rows * ld, box);
}

}  // namespace

size_t ortho_scratch(const OrthoMat* mats, uint32_t n, const DeviceInfo& dev) {
  return make_plan(mats, n, static_cast<uint32_t>(dev.sm_count)).total;
}

cudaError_t launch_orthogonalize(const OrthoMat* mats, uint32_t n, bool bf16, float mu,
                                 Workspace& ws, const DeviceInfo& dev) {
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count);
  const Plan plan = make_plan(mats, n, sms);
  if (plan.groups.empty()) return cudaSuccess;
  char* base = ws.model_scratch();
  auto half = [&](size_t off) { return reinterpret_cast<uint16_t*>(base + off); };
  cudaError_t err = cudaSuccess;

  // momentum, norms, X
  PrepArgs prep = {};
  prep.bf16 = bf16 ? 1u : 0u;
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
      const uint64_t units = static_cast<uint64_t>(m.rows) * ((m.cols + kSegment - 1) / kSegment);
      uint64_t per = (units + kMaxParts - 1) / kMaxParts;
      if (per < 32) per = 32;  // 4 a warp
      t.u = m.u;
      t.m = m.m;
      t.out = m.out;
      t.ld_out = m.ld_out;
      t.index = index;
      t.hi = half(g.hi[0]) + b * g.rows * g.ld_x;
      t.lo = half(g.lo[0]) + b * g.rows * g.ld_x;
      t.ld_u = m.ld_u;
      t.ld_m = m.ld_m;
      t.rows = m.rows;
      t.cols = m.cols;
      t.ld_x = g.ld_x;
      t.units_per_cta = static_cast<uint32_t>(per);
      t.cta0 = ctas;
      t.part0 = index * kMaxParts;
      t.parts = static_cast<uint32_t>((units + per - 1) / per);
      ctas += t.parts;
      if (prep.mats == kPrepMats && (err = flush()) != cudaSuccess) return err;
    }
  }
  if ((err = flush()) != cudaSuccess) return err;

  const size_t groups = plan.groups.size();
  for (int step = 0; step < kSteps; ++step) {
    const int from = step & 1, to = from ^ 1;
    const bool last = step == kSteps - 1;
    for (int ph = 0; ph < 3; ++ph) {
      for (size_t g0 = 0; g0 < groups; g0 += kOrthoGroups) {
        const size_t g1 = g0 + kOrthoGroups < groups ? g0 + kOrthoGroups : groups;
        ProductArgs<SymmetricEpilogue<false>, kOrthoGroups> pa = {};
        ProductArgs<SymmetricEpilogue<true>, kOrthoGroups> pb = {};
        ProductArgs<StepEpilogue, kOrthoGroups> px = {};
        for (size_t i = g0; i < g1; ++i) {
          const Group& g = plan.groups[i];
          const bool left = g.rows <= g.cols;
          const uint64_t batch = g.mats.size();
          const char *x = base + g.hi[from], *a = base + g.a, *b = base + g.b;
          ProductShape s = plan.shape[ph][i];
          bool ok;
          if (ph == 0) {
            s.a_mn = s.b_mn = left ? 0u : 1u;
            ok = operand(&s.a, x, g.cols, g.rows, g.ld_x, batch, left ? kTileM : 64) &&
                 operand(&s.b, x, g.cols, g.rows, g.ld_x, batch, left ? s.bn : 64);
            pa.shape[i - g0] = s;
            pa.epi[i - g0] = {nullptr, half(g.a), g.ld_s, static_cast<uint64_t>(g.side) * g.ld_s};
          } else if (ph == 1) {
            ok = operand(&s.a, a, g.side, g.side, g.ld_s, batch, kTileM) &&
                 operand(&s.b, a, g.side, g.side, g.ld_s, batch, s.bn);
            pb.shape[i - g0] = s;
            pb.epi[i - g0] = {half(g.a), half(g.b), g.ld_s, static_cast<uint64_t>(g.side) * g.ld_s};
          } else {
            if (left) {  // B X: X is MN-major
              s.b_mn = 1;
              ok = operand(&s.a, b, g.side, g.side, g.ld_s, batch, kTileM) &&
                   operand(&s.b, x, g.cols, g.rows, g.ld_x, batch, 64);
            } else {  // X B: B is symmetric, its rows are its columns
              ok = operand(&s.a, x, g.cols, g.rows, g.ld_x, batch, kTileM) &&
                   operand(&s.b, b, g.side, g.side, g.ld_s, batch, s.bn);
            }
            px.shape[i - g0] = s;
            px.epi[i - g0] = {half(g.hi[from]), half(g.lo[from]), half(g.hi[to]), half(g.lo[to]),
                              g.ld_x, static_cast<uint64_t>(g.rows) * g.ld_x,
                              last ? prep.outs + g.first : nullptr,
                              last ? prep.ld_outs + g.first : nullptr};
          }
          if (!ok) return cudaErrorInvalidValue;
        }
        float* join = reinterpret_cast<float*>(base + plan.join);
        const uint32_t count = static_cast<uint32_t>(g1 - g0);
        pa.problems = pb.problems = px.problems = count;
        pa.parts = pb.parts = px.parts = join;
        err = ph == 0 ? launch_product(pa, ws, dev)
                      : ph == 1 ? launch_product(pb, ws, dev) : launch_product(px, ws, dev);
        if (err != cudaSuccess) return err;
      }
    }
  }
  return cudaSuccess;
}

}  // namespace efs
