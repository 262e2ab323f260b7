// product.cuh — tiled matrix products D = A B^T on the tensor cores with an
// epilogue of the caller's: persistent CTAs, one per SM, each a TMA producer
// warp, an MMA warp and four epilogue warps.
//
// A CTA walks over the work items of up to a few products ("problems") in one
// launch. An item is one 128 x bn tile of D, or one of `splits` parts of its
// K axis. The producer fills a ring of shared-memory stages (64 of K each)
// with 128-byte-swizzled tiles; the MMA warp multiplies them into one of two
// accumulators in tensor memory, so the epilogue of one tile runs under the
// products of the next. Either operand may be stored K-major (rows along K)
// or MN-major (rows along M or N), so no operand is ever transposed in
// memory.
//
// Parts of K are joined without waiting: each part writes its fp32
// accumulators to scratch and counts itself in; the last part to arrive adds
// all parts in their order (so the sum does not depend on which was last) and
// runs the epilogue.
//
// Every wait on an mbarrier is bounded (tma.cuh); one that runs out latches a
// timeout, and the CTA ends without its results.
#pragma once

#include "internal.h"
#include "tensor.cuh"

namespace efs {

constexpr int kTileM = 128;        // rows of a tile: lanes of tensor memory
constexpr int kTileNMax = 256;     // columns of a tile, at most
constexpr int kTileK = 64;         // one 128-byte swizzle row of 16-bit elements
constexpr int kProductStages = 4;  // 48 KB each: 192 KB in flight per SM
constexpr int kProductThreads = 192;
constexpr uint32_t kStageABytes = kTileM * kTileK * 2;
constexpr uint32_t kStageBBytes = kTileNMax * kTileK * 2;
constexpr uint32_t kStageBytes = kStageABytes + kStageBBytes;
constexpr uint32_t kBoxMnBytes = 64 * kTileK * 2;  // an MN-major box: 64 elements x 64 k

// One product of a launch. The tensor maps are 3-D (innermost, rows, batch);
// a K-major operand's box is {64, rows of the tile}, an MN-major one's {64, 64}.
struct ProductShape {
  CUtensorMap a, b;
  uint32_t m, n, k;
  uint32_t a_mn, b_mn, bf16;
  uint32_t bn;                // columns per tile: a multiple of 16 (MN-major B: of 64)
  uint32_t tiles_m, tiles_n, batch, splits;
  uint32_t group_m;           // tiles are walked in groups of this many tile rows
  uint32_t lower;             // only tiles that reach the diagonal or below it
  uint32_t tiles;             // per batch entry
  uint32_t item0;             // this problem's first work item of the launch
  uint32_t slot0;             // its first scratch tile (splits > 1)
  const uint32_t* count;      // device: rows that exist (nullptr: all)
  uint32_t count_is_k;        // the count bounds K (else M)
};

struct ProductItem {
  uint32_t batch, tm, tn, m0, n0, n_eff, k0, kt, slot, split;
  bool skip;
};

__device__ __forceinline__ ProductItem product_item(const ProductShape& p, uint32_t item) {
  ProductItem it;
  uint32_t r = item - p.item0;
  it.split = r % p.splits;
  r /= p.splits;
  it.batch = r / p.tiles;
  r -= it.batch * p.tiles;
  if (p.lower) {
    // row group g (bn / 128 tile rows) holds q (g + 1) tiles, after q g (g + 1) / 2 others
    const uint32_t q = p.bn / kTileM;
    uint32_t g = static_cast<uint32_t>(sqrtf(2.0f * static_cast<float>(r / q) + 0.25f) - 0.5f);
    while (q * (g + 1) * (g + 2) / 2 <= r) ++g;
    while (q * g * (g + 1) / 2 > r) --g;
    const uint32_t rem = r - q * g * (g + 1) / 2;
    it.tm = q * g + rem / (g + 1);
    it.tn = rem % (g + 1);
  } else {
    const uint32_t per = p.group_m * p.tiles_n;
    const uint32_t g = r / per, in = r - g * per;
    const uint32_t rows = min(p.group_m, p.tiles_m - g * p.group_m);
    it.tn = in / rows;
    it.tm = g * p.group_m + in % rows;
  }
  it.m0 = it.tm * kTileM;
  it.n0 = it.tn * p.bn;
  it.n_eff = min(p.bn, (p.n - min(p.n, it.n0) + 15u) & ~15u);
  it.skip = it.tm >= p.tiles_m;
  uint32_t k = p.k;
  if (p.count) {
    const uint32_t c = *p.count;
    if (p.count_is_k) k = min(k, c);
    else it.skip |= it.m0 >= c;
  }
  const uint32_t kts = (k + kTileK - 1) / kTileK;
  const uint32_t lo = static_cast<uint32_t>(static_cast<uint64_t>(kts) * it.split / p.splits);
  const uint32_t hi = static_cast<uint32_t>(static_cast<uint64_t>(kts) * (it.split + 1) / p.splits);
  it.k0 = lo * kTileK;
  it.kt = hi - lo;
  it.slot = p.slot0 + (it.batch * p.tiles + r) * p.splits;  // its parts: slot .. slot + splits - 1
  return it;
}

template <class Epi, int kMaxProblems>
struct ProductArgs {
  ProductShape shape[kMaxProblems];
  typename Epi::Params epi[kMaxProblems];
  uint32_t problems, items;
  float* parts;         // scratch tiles of split items
  uint32_t* arrivals;   // by the tile's first scratch tile; zero between launches
  uint32_t part_chunks; // 32-column chunks per scratch tile
  uint32_t* error;
  uint64_t wait_ns;
};

struct ProductSmem {
  uint64_t full[kProductStages], empty[kProductStages], acc_full[2], acc_empty[2];
  uint32_t tmem, last;
};

// What an epilogue reads its accumulators through: 32 columns of the thread's
// row at a time, in order, from tensor memory or as the sum of the K parts.
struct ProductAcc {
  uint32_t tmem;            // address of the accumulator, the warp's lanes
  uint64_t* release;        // arrived on after the last chunk was read
  const float* parts;       // != nullptr: sum `splits` scratch tiles instead
  uint64_t part_stride;     // floats from one part to the next
  uint32_t splits, chunks;
  bool none;                // K is empty: zeros

  // All lanes of the warp call it alike.
  __device__ __forceinline__ void load(uint32_t c, float (&v)[32]) const {
    __syncwarp();
    if (none) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = 0.0f;
    } else if (parts) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = 0.0f;
      for (uint32_t s = 0; s < splits; ++s) {
        const float* src = parts + s * part_stride + static_cast<uint64_t>(c) * (32 * kTileM);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float4 x = __ldcg(reinterpret_cast<const float4*>(src) + j * kTileM);
          v[4 * j] = __fadd_rn(v[4 * j], x.x);
          v[4 * j + 1] = __fadd_rn(v[4 * j + 1], x.y);
          v[4 * j + 2] = __fadd_rn(v[4 * j + 2], x.z);
          v[4 * j + 3] = __fadd_rn(v[4 * j + 3], x.w);
        }
      }
    } else {
      tmem_load_32(tmem + c * 32, v);
      if (c + 1 == chunks) {
        tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(release);
      }
    }
  }
};

template <class Epi, int kMaxProblems>
__global__ void __launch_bounds__(kProductThreads, 1)
    product_kernel(const __grid_constant__ ProductArgs<Epi, kMaxProblems> args) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ ProductSmem s;
  __shared__ typename Epi::Smem epi_smem;
  uint8_t* stages = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kProductStages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 4);
    }
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc(&s.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s.tmem;
  griddep_wait();
  bool ok = true;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0, prob = 0;
      for (uint32_t item = blockIdx.x; item < args.items && ok; item += gridDim.x) {
        while (prob + 1 < args.problems && item >= args.shape[prob + 1].item0) ++prob;
        const ProductShape& p = args.shape[prob];
        const ProductItem it = product_item(p, item);
        if (it.skip) continue;
        const uint32_t b_boxes = (it.n_eff + 63) / 64;
        const uint32_t bytes = kStageABytes + (p.b_mn ? b_boxes * kBoxMnBytes : p.bn * kTileK * 2);
        for (uint32_t kt = 0; kt < it.kt; ++kt) {
          if (!mbar_wait(&s.empty[stage], phase ^ 1u, args.wait_ns)) {
            ok = false;
            break;
          }
          uint8_t* a = stages + stage * kStageBytes;
          uint8_t* b = a + kStageABytes;
          const uint32_t k = it.k0 + kt * kTileK;
          mbar_arrive_expect_tx(&s.full[stage], bytes);
          if (p.a_mn) {
            tma_load_3d(a, &p.a, it.m0, k, it.batch, &s.full[stage]);
            tma_load_3d(a + kBoxMnBytes, &p.a, it.m0 + 64, k, it.batch, &s.full[stage]);
          } else {
            tma_load_3d(a, &p.a, k, it.m0, it.batch, &s.full[stage]);
          }
          if (p.b_mn) {
            for (uint32_t x = 0; x < b_boxes; ++x)
              tma_load_3d(b + x * kBoxMnBytes, &p.b, it.n0 + 64 * x, k, it.batch, &s.full[stage]);
          } else {
            tma_load_3d(b, &p.b, k, it.n0, it.batch, &s.full[stage]);
          }
          if (++stage == kProductStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0, prob = 0, acc = 0, acc_phase = 0;
      for (uint32_t item = blockIdx.x; item < args.items && ok; item += gridDim.x) {
        while (prob + 1 < args.problems && item >= args.shape[prob + 1].item0) ++prob;
        const ProductShape& p = args.shape[prob];
        const ProductItem it = product_item(p, item);
        if (it.skip || it.kt == 0) continue;
        if (!mbar_wait(&s.acc_empty[acc], acc_phase ^ 1u, args.wait_ns)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t idesc = mma_idesc(p.bf16, p.a_mn, p.b_mn, kTileM, it.n_eff);
        const uint32_t d = tmem + acc * kTileNMax;
        // 16 of K: 32 bytes along a K-major row, 16 rows of an MN-major tile
        const uint32_t a_step = (p.a_mn ? 2048u : 32u) >> 4, b_step = (p.b_mn ? 2048u : 32u) >> 4;
        for (uint32_t kt = 0; kt < it.kt; ++kt) {
          if (!mbar_wait(&s.full[stage], phase, args.wait_ns)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a = smem_u32(stages + stage * kStageBytes);
          const uint64_t da = smem_desc(a, p.a_mn ? kBoxMnBytes : 16, 1024);
          const uint64_t db = smem_desc(a + kStageABytes, p.b_mn ? kBoxMnBytes : 16, 1024);
#pragma unroll
          for (uint32_t j = 0; j < kTileK / 16; ++j)
            mma_f16(d, da + j * a_step, db + j * b_step, idesc, kt > 0 || j > 0);
          mma_commit(&s.empty[stage]);
          if (++stage == kProductStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        mma_commit(&s.acc_full[acc]);
        if (++acc == 2) {
          acc = 0;
          acc_phase ^= 1u;
        }
      }
    }
  } else {
    const uint32_t quarter = warp & 3u;  // the lanes of tensor memory this warp may read
    const uint32_t row = quarter * 32 + lane;
    uint32_t prob = 0, acc = 0, acc_phase = 0;
    for (uint32_t item = blockIdx.x; item < args.items; item += gridDim.x) {
      while (prob + 1 < args.problems && item >= args.shape[prob + 1].item0) ++prob;
      const ProductShape& p = args.shape[prob];
      const ProductItem it = product_item(p, item);
      if (it.skip) continue;
      ProductAcc from;
      from.chunks = (it.n_eff + 31) / 32;
      from.none = it.kt == 0;
      from.parts = nullptr;
      from.splits = p.splits;
      from.tmem = tmem + acc * kTileNMax + ((quarter * 32) << 16);
      from.release = &s.acc_empty[acc];
      if (!from.none && ok) {
        ok = __all_sync(0xffffffffu, mbar_wait(&s.acc_full[acc], acc_phase, args.wait_ns));
        tc_fence_after();
        if (++acc == 2) {
          acc = 0;
          acc_phase ^= 1u;
        }
      }
      // a warp whose wait ran out stays for the barriers of the others, with
      // zeros (the call's results are void: the timeout is latched)
      from.none |= !ok;
      if (p.splits > 1) {
        const uint64_t tile_floats = static_cast<uint64_t>(args.part_chunks) * 32 * kTileM;
        float* mine = args.parts + static_cast<uint64_t>(it.slot) * tile_floats + row * 4;
        float* dst = mine + it.split * tile_floats;
        for (uint32_t c = 0; c < from.chunks; ++c) {
          float v[32];
          from.load(c, v);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            __stcg(reinterpret_cast<float4*>(dst + static_cast<uint64_t>(c) * (32 * kTileM)) + j * kTileM,
                   make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
        }
        __threadfence();
        asm volatile("bar.sync 2, 128;" ::: "memory");
        if (warp == 2 && lane == 0) {
          const uint32_t before = atomicAdd(&args.arrivals[it.slot], 1u);
          s.last = before == p.splits - 1 ? 1u : 0u;
          if (s.last) args.arrivals[it.slot] = 0;  // ready for the next launch
          __threadfence();
        }
        asm volatile("bar.sync 2, 128;" ::: "memory");
        const bool last = s.last != 0;
        asm volatile("bar.sync 2, 128;" ::: "memory");  // s.last is read before it is written again
        if (!last) continue;
        __threadfence();
        from.parts = mine;
        from.part_stride = tile_floats;
        from.none = false;
      }
      Epi::tile(p, args.epi[prob], it, row, epi_smem, from);
    }
  }
  if (!ok) atomicOr(args.error, kDevErrTimeout);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_free(tmem, 512);
}

// ------------------------------------------------------------- host side
// A tensor map over [batch][rows][cols] 16-bit elements, row stride `ld` and
// batch stride `batch_ld` in elements; boxes of 64 x box_rows, 128-byte
// swizzle, zeros outside. False: refused by the driver.
bool make_map(CUtensorMap* map, const void* base, bool bf16, uint64_t cols, uint64_t rows,
              uint64_t ld, uint64_t batch, uint64_t batch_ld, uint32_t box_rows);

// Whether TMA can read rows of 16-bit elements at this address and stride.
inline bool tma_rows(const void* p, uint64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0;
}

// Fills bn, tiles, splits of a product of m x n x k (batch of them) on `sms` SMs.
void plan_product(ProductShape& p, uint32_t m, uint32_t n, uint32_t k, uint32_t batch,
                  bool lower, uint32_t sms, uint32_t max_splits);

template <class Epi, int kMaxProblems>
cudaError_t launch_product(ProductArgs<Epi, kMaxProblems>& args, Workspace& ws,
                           const DeviceInfo& dev) {
  uint32_t items = 0, slots = 0, chunks = 0;
  for (uint32_t i = 0; i < args.problems; ++i) {
    ProductShape& p = args.shape[i];
    p.item0 = items;
    p.slot0 = slots;
    items += p.tiles * p.batch * p.splits;
    if (p.splits > 1) {
      // slots are indexed slot * splits within the problem's share of the scratch
      slots += p.tiles * p.batch * p.splits;
      chunks = (p.bn + 31) / 32 > chunks ? (p.bn + 31) / 32 : chunks;
    }
  }
  if (items == 0) return cudaSuccess;
  if (slots > kModelArrivals) return cudaErrorInvalidValue;
  args.items = items;
  args.part_chunks = chunks;
  args.arrivals = ws.model_arrivals();
  args.error = ws.u32(kOffError);
  args.wait_ns = wait_limit_ns();
  auto fn = product_kernel<Epi, kMaxProblems>;
  constexpr uint32_t smem = kProductStages * kStageBytes + 1024;
  static_assert(smem <= 220 * 1024, "stages fit beside the static shared memory");
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count);
  void* params[] = {&args};
  e = launch_pdl(reinterpret_cast<const void*>(fn), dim3(items < sms ? items : sms),
                 kProductThreads, smem, ws.stream, params, false);
  if (e == cudaSuccess) count_launch();
  return e;
}

}  // namespace efs
