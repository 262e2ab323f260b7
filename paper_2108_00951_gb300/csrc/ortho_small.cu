// ortho_small.cu — the orthogonalised update (ortho.cu) of matrices whose
// shorter side is at most 128, on chip: one thread-block cluster per matrix,
// from the update to the result in one launch.
//
// What bounds such a matrix is latency: fifteen products that depend on each
// other, of a microsecond or less. Through global memory and grid barriers
// each costs about 10 us (64 x 576: 151 us; here 45, 128 x 1152: 184 and 78);
// here a step's three products have their operands in shared memory throughout,
// and the CTAs of a cluster exchange only the small square A = X X^T.
//
// X (the long side along its columns; a tall matrix is turned on the way in
// and out) is split by columns, up to four blocks of 64 per CTA, each a pair
// hi + lo of fp16 tiles of 128 rows (22 bits; products are hi hi + hi lo +
// lo hi, as in ortho.cu for these sides). A tile serves as a K-major operand
// of X X^T and as the MN-major operand of B X. Per step:
//   1. each CTA's share of A, its rows sent to their owners (st.shared::cluster);
//   2. an owner adds the shares in rank order and sends A as fp16 hi + lo to all;
//   3. every CTA forms B = b A + c A A + 2 I for itself;
//   4. and its columns of X <- (a - 2) X + B X.
// Scales and constants are those of ortho.cu.
#include "product.cuh"

#include <vector>

#include <cuda_fp16.h>

namespace efs {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f, kNsShift = 2.0f;
constexpr float kScaleX = 16384.0f, kScaleA = 8192.0f;
constexpr int kSteps = 5;
constexpr uint32_t kSmallThreads = 256;
constexpr uint32_t kSmallMats = 64;     // per launch
constexpr uint32_t kMaxCluster = 16;  // beyond the portable 8 where a GPU takes it
constexpr uint32_t kTileBytes = 128 * 128;  // 128 rows of 64 fp16
constexpr uint32_t kSmallSmem = 200 * 1024;
// At least this much is asked for, so that one CTA runs per SM: a second one's
// allocation of tensor memory would wait for the first to end, which may be
// waiting for a CTA of its cluster that waits likewise elsewhere.
constexpr uint32_t kSmallSmemMin = 120 * 1024;

struct SmallMat {
  const void* u;
  float* m;
  uint16_t* out;
  uint64_t ld_u, ld_m, ld_out;
  uint32_t side, len;  // shorter and longer side
  uint32_t tall;       // stored [len][side]
};
struct SmallArgs {
  SmallMat mat[kSmallMats];
  float mu;
  uint32_t blocks;      // of 64 columns per CTA
  uint32_t shares_off, square_off;  // in dynamic shared memory
  uint32_t* error;
  uint64_t wait_ns;
};

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
  return n;
}
// Stores to a shared::cluster address: another CTA's shared memory.
__device__ __forceinline__ void st_cluster_f4(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(v.x), "f"(v.y),
               "f"(v.z), "f"(v.w)
               : "memory");
}
__device__ __forceinline__ void st_cluster_u2(uint32_t addr, uint2 v) {
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1,%2};" ::"r"(addr), "r"(v.x), "r"(v.y)
               : "memory");
}

// Byte offset of (row, col) in a swizzled tile of 64 columns; col within it.
__device__ __forceinline__ uint32_t tile_at(uint32_t row, uint32_t col) {
  return row * 128 + ((col * 2) ^ ((row & 7u) << 4));
}
__device__ __forceinline__ float rest(float x) {
  return __fsub_rn(x, __half2float(__float2half_rn(x)));
}
// 8 columns of a row (16 bytes of a tile) of a pair, added.
__device__ __forceinline__ void load_pair_8(const uint8_t* hi, const uint8_t* lo, float* v) {
  const uint4 h = *reinterpret_cast<const uint4*>(hi), l = *reinterpret_cast<const uint4*>(lo);
  const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&hw[j]));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&lw[j]));
    v[2 * j] = __fadd_rn(a.x, b.x);
    v[2 * j + 1] = __fadd_rn(a.y, b.y);
  }
}
__device__ __forceinline__ void store_pair_8(uint8_t* hi, uint8_t* lo, const float* v) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = pack_f16(v[2 * j], v[2 * j + 1]);
    l[j] = pack_f16(rest(v[2 * j]), rest(v[2 * j + 1]));
  }
  *reinterpret_cast<uint4*>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
}

// Four entries of the matrix, X's row r, columns c .. c + 3 of which `n` exist:
// of u (kU) or of the momentum.
template <bool kBf16, bool kU>
__device__ __forceinline__ void load_4(const SmallMat& t, uint32_t r, uint32_t c, uint32_t n,
                                       bool vec, float (&x)[4]) {
  const uint64_t ld = kU ? t.ld_u : t.ld_m;
  const uint64_t at = t.tall ? static_cast<uint64_t>(c) * ld + r : r * ld + c;
  const uint64_t step = t.tall ? ld : 1;
  if (vec && n == 4) {
    if (kU && kBf16) {
      const uint2 w = __ldg(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(t.u) + at));
      x[0] = __uint_as_float(w.x << 16), x[1] = __uint_as_float(w.x & 0xffff0000u);
      x[2] = __uint_as_float(w.y << 16), x[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
      const float4 y = kU ? __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(t.u) + at))
                          : *reinterpret_cast<const float4*>(t.m + at);
      x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
    }
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    x[j] = 0.0f;
    if (j < n) {
      if (!kU) x[j] = t.m[at + j * step];
      else if (kBf16) x[j] = bf16_bits_to_f32(__ldg(static_cast<const uint16_t*>(t.u) + at + j * step));
      else x[j] = __ldg(static_cast<const float*>(t.u) + at + j * step);
    }
  }
}
__device__ __forceinline__ void store_m(const SmallMat& t, uint32_t r, uint32_t c, uint32_t n,
                                        bool vec, const float (&x)[4]) {
  const uint64_t at = t.tall ? static_cast<uint64_t>(c) * t.ld_m + r : r * t.ld_m + c;
  const uint64_t step = t.tall ? t.ld_m : 1;
  if (vec && n == 4) {
    *reinterpret_cast<float4*>(t.m + at) = make_float4(x[0], x[1], x[2], x[3]);
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j)
    if (j < n) t.m[at + j * step] = x[j];
}

template <bool kBf16>
__global__ void __launch_bounds__(kSmallThreads, 1)
    ortho_small_kernel(const __grid_constant__ SmallArgs args) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_done, s_drained;
  __shared__ uint32_t s_tmem;
  __shared__ FF s_ff[32];
  __shared__ alignas(16) float2 s_norm[kMaxCluster];  // written as 8 bytes by the other CTAs
  uint8_t* xs = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank(), ranks = cluster_size();
  const SmallMat& t = args.mat[blockIdx.x / ranks];
  const uint32_t blocks = args.blocks, width = blocks * 64, c_first = rank * width;
  const uint32_t cols = t.len > c_first ? min(width, t.len - c_first) : 0;  // this CTA's
  const uint32_t side16 = (t.side + 15) & ~15u, side32 = (t.side + 31) & ~31u;
  const uint32_t squares = (t.side + 63) / 64;  // 64-column tiles of A and B
  uint8_t* xh = xs;
  uint8_t* xl = xs + blocks * kTileBytes;
  float* shares = reinterpret_cast<float*>(xs + args.shares_off);
  uint8_t* qh = xs + args.square_off;  // A, then B
  uint8_t* ql = qh + squares * kTileBytes;
  if (tid == 0) {
    mbar_init(&s_done, 1);
    mbar_init(&s_drained, 1);
    mbar_init_fence();
  }
  if (warp == 0) tmem_alloc<false>(&s_tmem, 512);
  for (uint32_t i = tid * 16; i < args.square_off + 2 * squares * kTileBytes; i += kSmallThreads * 16)
    *reinterpret_cast<uint4*>(xs + i) = make_uint4(0, 0, 0, 0);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  cluster_arrive();
  const uint32_t tmem = s_tmem, d_sq = tmem, d_x = tmem + 256;
  griddep_wait();

  // Momentum and |U|^2, four columns of X at a time (lanes along the matrix's
  // rows as they lie in memory). U waits in X's place, the high and the low
  // halves of its fp32 words where hi and lo will be.
  const uint32_t c_units = (cols + 3) / 4, units = t.side * c_units;
  const bool vec_u = !t.tall && t.ld_u % 4 == 0 && c_first % 4 == 0 &&
                     reinterpret_cast<uintptr_t>(t.u) % (kBf16 ? 8 : 16) == 0;
  const bool vec_m = !t.tall && t.ld_m % 4 == 0 && reinterpret_cast<uintptr_t>(t.m) % 16 == 0;
  FF total{0.0f, 0.0f};
  for (uint32_t i0 = tid; i0 < units; i0 += 4 * kSmallThreads) {
    float x[4][4];
    uint32_t r[4], c[4], n[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = i0 + j * kSmallThreads, by = t.tall ? t.side : c_units, q = i / by;
      r[j] = t.tall ? i - q * by : q;
      c[j] = (t.tall ? q : i - q * by) * 4;
      n[j] = i < units ? min(4u, cols - c[j]) : 0;
      load_4<kBf16, true>(t, r[j], c_first + c[j], n[j], vec_u, x[j]);
    }
    if (t.m) {
      float m[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) load_4<kBf16, false>(t, r[j], c_first + c[j], n[j], vec_m, m[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          m[j][k] = __fmaf_rn(args.mu, m[j][k], x[j][k]);
          x[j][k] = __fadd_rn(x[j][k], m[j][k]);
        }
        store_m(t, r[j], c_first + c[j], n[j], vec_m, m[j]);
      }
    }
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (n[j] == 0) continue;
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s = __fmaf_rn(x[j][k], x[j][k], s);
        w[k] = __float_as_uint(x[j][k]);
      }
      const uint32_t at = c[j] / 64 * kTileBytes + tile_at(r[j], c[j] % 64);
      *reinterpret_cast<uint2*>(xh + at) =
          make_uint2(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
      *reinterpret_cast<uint2*>(xl + at) =
          make_uint2(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410));
    }
    total = ff_add(total, FF{s, 0.0f});
  }
  total = block_sum_ff(total, s_ff);
  cluster_wait();  // the other CTAs have started: their shared memory may be written
  if (tid == 0)
    for (uint32_t q = 0; q < ranks; ++q)
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(cluster_addr(&s_norm[rank], q)),
                   "f"(total.hi), "f"(total.lo)
                   : "memory");
  cluster_sync();
  FF sum{s_norm[0].x, s_norm[0].y};
  for (uint32_t q = 1; q < ranks; ++q) sum = ff_add(sum, FF{s_norm[q].x, s_norm[q].y});
  const double norm = sqrt(ff_to_double(sum));
  const float inv = norm == 0.0 ? 0.0f : static_cast<float>(static_cast<double>(kScaleX) / norm);

  // X as hi + lo, in place (zeros where there is no entry)
  for (uint32_t i = tid; i < t.side * blocks * 8; i += kSmallThreads) {
    const uint32_t block = i / (t.side * 8), r = i / 8 - block * t.side;
    const uint32_t at = block * kTileBytes + tile_at(r, i % 8 * 8);
    const uint4 h = *reinterpret_cast<const uint4*>(xh + at);
    const uint4 l = *reinterpret_cast<const uint4*>(xl + at);
    const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
    float v[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __fmul_rn(__uint_as_float(__byte_perm(lw[j], hw[j], 0x5410)), inv);
      v[2 * j + 1] = __fmul_rn(__uint_as_float(__byte_perm(lw[j], hw[j], 0x7632)), inv);
    }
    store_pair_8(xh + at, xl + at, v);
  }

  // Products: one thread issues, all wait. An operand pair is taken as
  // hi hi + hi lo + lo hi.
  uint32_t parity = 0;
  bool ok = true;
  auto finish = [&]() {
    if (ok) ok = mbar_wait(&s_done, parity, args.wait_ns);
    parity ^= 1u;
    tc_fence_after();
    __syncwarp();
  };
  auto ready = [&]() {  // shared memory written by all threads, accumulators read
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  };
  const uint32_t quarter = warp & 3u, half = warp >> 2;
  const uint32_t row = quarter * 32 + lane, r0 = quarter * 32;
  const uint32_t lanes = r0 << 16;
  const uint32_t rows_per = (side32 + ranks - 1) / ranks;  // of A an owner adds up
  const uint32_t row_units = side32 / 4;

  for (int step = 0; step < kSteps; ++step) {
    // 1. this CTA's share of A = X X^T
    ready();
    if (tid == 0 && cols) {
      const uint32_t idesc = mma_idesc(0, 0, 0, kTileM, side16);
      bool more = false;
      for (uint32_t term = 0; term < 3; ++term)
        for (uint32_t b = 0; b * 64 < cols; ++b) {
          const uint32_t ah = smem_u32(xh) + b * kTileBytes, al = smem_u32(xl) + b * kTileBytes;
          const uint64_t da = smem_desc(term == 2 ? al : ah, 16, 1024);
          const uint64_t db = smem_desc(term == 1 ? al : ah, 16, 1024);
          for (uint32_t j = 0; j < 4 && b * 64 + j * 16 < cols; ++j) {
            mma_f16<false>(d_sq, da + j * 2, db + j * 2, idesc, more);
            more = true;
          }
        }
      mma_commit<false>(&s_done);
    }
    if (cols) finish();
    if (r0 < side32) {
      const uint32_t owner = row / rows_per, at = row - owner * rows_per;
      for (uint32_t c = half; c < side32 / 32; c += 2) {
        float v[32];
        __syncwarp();
        if (cols) {
          tmem_load_32(d_sq + lanes + c * 32, v);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0.0f;
        }
        // columns past the product's width hold nothing
#pragma unroll
        for (int j = 16; j < 32; ++j) v[j] = c * 32 + j < side16 ? v[j] : 0.0f;
        const uint32_t base = cluster_addr(
            shares + (static_cast<uint64_t>(rank) * rows_per + at) * side32, owner);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
          st_cluster_f4(base + (((c * 8 + j) ^ (row & 7u)) << 4),
                        make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
      }
    }
    tc_fence_before();
    cluster_sync();
    // 2. an owner's rows of A, in rank order, to every CTA
    const uint32_t mine = rank * rows_per < side32 ? min(rows_per, side32 - rank * rows_per) : 0;
    for (uint32_t i = tid; i < mine * row_units; i += kSmallThreads) {
      const uint32_t at = i / row_units, u = i - at * row_units, r = rank * rows_per + at;
      float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (uint32_t q = 0; q < ranks; ++q) {
        const float4 x = *reinterpret_cast<const float4*>(
            shares + (q * rows_per + at) * side32 + ((u ^ (r & 7u)) << 2));
        s = make_float4(__fadd_rn(s.x, x.x), __fadd_rn(s.y, x.y), __fadd_rn(s.z, x.z),
                        __fadd_rn(s.w, x.w));
      }
      constexpr float k = kScaleA / (kScaleX * kScaleX);
      s = make_float4(__fmul_rn(s.x, k), __fmul_rn(s.y, k), __fmul_rn(s.z, k), __fmul_rn(s.w, k));
      const uint2 h = make_uint2(pack_f16(s.x, s.y), pack_f16(s.z, s.w));
      const uint2 l = make_uint2(pack_f16(rest(s.x), rest(s.y)), pack_f16(rest(s.z), rest(s.w)));
      const uint32_t c = u * 4, to = c / 64 * kTileBytes + tile_at(r, c % 64);
      for (uint32_t q = 0; q < ranks; ++q) {
        st_cluster_u2(cluster_addr(qh + to, q), h);
        st_cluster_u2(cluster_addr(ql + to, q), l);
      }
    }
    fence_proxy_async();
    cluster_sync();
    tc_fence_after();
    // 3. B = b A + c A A + 2 I
    if (tid == 0) {
      fence_proxy_async();
      const uint32_t idesc = mma_idesc(0, 0, 0, kTileM, side16);
      for (uint32_t term = 0; term < 3; ++term)
        for (uint32_t j = 0; j * 16 < t.side; ++j) {
          const uint32_t off = j / 4 * kTileBytes;
          const uint64_t da = smem_desc(smem_u32(term == 2 ? ql : qh) + off, 16, 1024);
          const uint64_t db = smem_desc(smem_u32(term == 1 ? ql : qh) + off, 16, 1024);
          mma_f16<false>(d_sq, da + (j & 3u) * 2, db + (j & 3u) * 2, idesc, term > 0 || j > 0);
        }
      mma_commit<false>(&s_done);
    }
    finish();
    if (r0 < side32) {
      for (uint32_t c = half; c < side32 / 32; c += 2) {
        float v[32], a[8];
        __syncwarp();
        tmem_load_32(d_sq + lanes + c * 32, v);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          const uint32_t col = c * 32 + u * 8, at = col / 64 * kTileBytes + tile_at(row, col % 64);
          load_pair_8(qh + at, ql + at, a);
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j) {
            float x = __fmaf_rn(kNsB, a[j], __fmul_rn(v[u * 8 + j], kNsC / kScaleA));
            if (col + j == row) x = __fmaf_rn(kNsShift, kScaleA, x);
            // rows and columns past the side stay zero
            a[j] = row < t.side && col + j < t.side ? x : 0.0f;
          }
          store_pair_8(qh + at, ql + at, a);
        }
      }
    }
    // 4. X <- (a - 2) X + B X
    ready();
    if (tid == 0 && cols) {
      const uint32_t n = (cols + 15) & ~15u;
      const uint32_t idesc = mma_idesc(0, 0, 1, kTileM, n);
      for (uint32_t term = 0; term < 3; ++term)
        for (uint32_t j = 0; j * 16 < t.side; ++j) {
          const uint64_t da = smem_desc(smem_u32(term == 2 ? ql : qh) + j / 4 * kTileBytes, 16, 1024);
          const uint64_t db = smem_desc(smem_u32(term == 1 ? xl : xh), kTileBytes, 1024);
          mma_f16<false>(d_x, da + (j & 3u) * 2, db + j * (2048 >> 4), idesc, term > 0 || j > 0);
        }
      mma_commit<false>(&s_done);
    }
    if (cols) finish();
    const bool last = step == kSteps - 1;
    if (r0 < t.side) {
      for (uint32_t c = half; c * 32 < cols; c += 2) {
        float v[32];
        __syncwarp();
        tmem_load_32(d_x + lanes + c * 32, v);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          const uint32_t col = c * 32 + u * 8, at = col / 64 * kTileBytes + tile_at(row, col % 64);
          float x[8];
          load_pair_8(xh + at, xl + at, x);
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j)
            x[j] = row < t.side && col + j < cols
                       ? __fmaf_rn(v[u * 8 + j], 1.0f / kScaleA, __fmul_rn(kNsA - kNsShift, x[j]))
                       : 0.0f;
          if (!last) {
            store_pair_8(xh + at, xl + at, x);
          } else if (row < t.side) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
              w[j] = pack_bf16(__fmul_rn(x[2 * j], 1.0f / kScaleX), __fmul_rn(x[2 * j + 1], 1.0f / kScaleX));
            const uint32_t gc = c_first + col;
            if (t.tall) {
#pragma unroll
              for (uint32_t j = 0; j < 8; ++j)
                if (col + j < cols)
                  t.out[static_cast<uint64_t>(gc + j) * t.ld_out + row] =
                      static_cast<uint16_t>(j & 1u ? w[j / 2] >> 16 : w[j / 2]);
            } else {
              uint16_t* to = t.out + static_cast<uint64_t>(row) * t.ld_out + gc;
              if (col + 8 <= cols && (reinterpret_cast<uintptr_t>(t.out) | (t.ld_out * 2)) % 16 == 0) {
                *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
              } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                  if (col + j < cols) to[j] = static_cast<uint16_t>(j & 1u ? w[j / 2] >> 16 : w[j / 2]);
              }
            }
          }
        }
      }
    }
  }
  if (!ok) {
    atomicOr(args.error, kDevErrTimeout);
    if (tid == 0) {  // a wait ran out: no product may run after the CTA's end
      mma_commit<false>(&s_drained);
      mbar_wait(&s_drained, 0, kDrainNs);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_free<false>(tmem, 512);
  cluster_sync();  // no CTA ends while another may still write to it
}

struct SmallShape {
  uint32_t blocks, ranks, shares_off, square_off, smem;
  bool fits;
};
// Shared memory for a shorter side of `side` with `blocks` blocks per CTA.
SmallShape small_shape(uint32_t side, uint32_t len, uint32_t most) {
  SmallShape s = {};
  const uint32_t all = (len + 63) / 64, side32 = (side + 31) & ~31u;
  // up to 8 CTAs while they hold the matrix: a larger cluster exchanges more
  const uint32_t blocks = side <= 64 ? 4 : side <= 96 ? 3 : 2;
  if (most > 8 && all <= 8 * blocks) most = 8;
  s.blocks = (all + most - 1) / most;
  s.ranks = (all + s.blocks - 1) / s.blocks;
  const uint32_t rows_per = (side32 + s.ranks - 1) / s.ranks;
  s.shares_off = s.blocks * 2 * kTileBytes;
  s.square_off = s.shares_off + (s.ranks * rows_per * side32 * 4 + 1023) / 1024 * 1024;
  s.smem = s.square_off + (side + 63) / 64 * 2 * kTileBytes + 1024;
  if (s.smem < kSmallSmemMin) s.smem = kSmallSmemMin;
  s.fits = side <= 128 && s.blocks <= 4 && s.smem <= kSmallSmem;
  return s;
}

bool same_layout(const SmallShape& x, const SmallShape& y) {
  return x.blocks == y.blocks && x.ranks == y.ranks && x.square_off == y.square_off && x.smem == y.smem;
}

}  // namespace

void ortho_small_init_device(DeviceInfo& info) {
  info.ortho_cluster = 8;
  const void* fns[] = {reinterpret_cast<const void*>(&ortho_small_kernel<true>),
                       reinterpret_cast<const void*>(&ortho_small_kernel<false>)};
  int fit = 0;
  for (const void* fn : fns) {
    cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmallSmem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kMaxCluster);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = kSmallSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kMaxCluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
        cudaOccupancyMaxActiveClusters(&clusters, fn, &cfg) == cudaSuccess && clusters > 0)
      ++fit;
  }
  cudaGetLastError();
  if (fit == 2) info.ortho_cluster = kMaxCluster;
}

// Whether every matrix is one that a cluster holds, in launches (one after
// another, a layout each) that take less time together than the phases of
// ortho.cu, which are one set for all matrices: 64 x 27 and 64 x 576 take 76 us
// here and 151 there, three layouts of side 128 188 and 190, six of side 64 293
// and 158.
constexpr size_t kMaxLayouts = 3;
bool ortho_small(const OrthoMat* mats, uint32_t n, const DeviceInfo& dev) {
  std::vector<SmallShape> layouts;
  for (uint32_t i = 0; i < n; ++i) {
    const uint32_t r = mats[i].rows, c = mats[i].cols;
    if (!r || !c) continue;
    const SmallShape s = small_shape(r < c ? r : c, r < c ? c : r, dev.ortho_cluster);
    if (!s.fits) return false;
    bool known = false;
    for (const SmallShape& x : layouts) known |= same_layout(x, s);
    if (known) continue;
    layouts.push_back(s);
    if (layouts.size() > kMaxLayouts) return false;
  }
  return true;
}

cudaError_t launch_ortho_small(const OrthoMat* mats, uint32_t n, bool bf16, float mu,
                               Workspace& ws, const DeviceInfo& dev) {
  auto fn = bf16 ? ortho_small_kernel<true> : ortho_small_kernel<false>;
  // matrices of one layout go into one launch
  std::vector<bool> done(n, false);
  for (uint32_t i = 0; i < n; ++i) {
    if (done[i] || !mats[i].rows || !mats[i].cols) continue;
    SmallArgs args = {};
    args.mu = mu;
    args.error = ws.u32(kOffError);
    args.wait_ns = wait_limit_ns();
    uint32_t count = 0;
    SmallShape layout = {};
    for (uint32_t j = i; j < n && count < kSmallMats; ++j) {
      const OrthoMat& m = mats[j];
      if (done[j] || !m.rows || !m.cols) continue;
      const bool tall = m.rows > m.cols;
      const uint32_t side = tall ? m.cols : m.rows, len = tall ? m.rows : m.cols;
      const SmallShape s = small_shape(side, len, dev.ortho_cluster);
      if (count == 0) {
        layout = s;
        args.blocks = s.blocks;
        args.shares_off = s.shares_off;
        args.square_off = s.square_off;
      } else if (!same_layout(s, layout)) {
        continue;
      }
      args.mat[count++] = {m.u, m.m, m.out, m.ld_u, m.ld_m, m.ld_out, side, len, tall ? 1u : 0u};
      done[j] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(count * layout.ranks);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = layout.smem;
    cfg.stream = ws.stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = layout.ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t l = cudaLaunchKernelEx(&cfg, fn, args);
    if (l != cudaSuccess) return l;
    count_launch();
  }
  return cudaSuccess;
}

}  // namespace efs
