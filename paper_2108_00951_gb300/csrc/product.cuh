// product.cuh — tiled matrix products D = A B^T on the tensor cores with an
// epilogue of the caller's: persistent CTAs, one per SM, each a TMA producer
// warp, an MMA warp and eight epilogue warps; two CTAs can work as a pair.
//
// A CTA (or pair) walks over the work items of a few products ("problems") in
// one launch. An item is one tile of D, 128 (a pair: 256) x bn, or one of
// `splits` parts of its K axis. The producer fills a ring of shared-memory
// stages (128 of K each) with 128-byte-swizzled tiles; the MMA warp multiplies
// them into one of two accumulators in tensor memory, so the epilogue of one
// tile runs under the products of the next. Either operand may be stored
// K-major (rows along K) or MN-major (rows along M or N), so no operand is
// ever transposed in memory.
//
// What bounds it: an SM takes about 64 bytes a cycle from L2 (measured on a
// GB300: 130 GB/s in boxes of 16 KB; in boxes of 8 KB, 104 to 108), and a
// 128 x 256 tile needs 96 a cycle at the tensor cores' full rate (8192
// operations a cycle, 512 cycles per 64 of K). A pair shares its B tile, each
// CTA loading half: 64 bytes a cycle. Stages are 128 of K deep so that every
// box has 16 KB, K-major (64 k x 128 rows) or MN-major (64 x 128 k).
//
// Parts of K (cooperative launches only): each part's CTA writes its fp32
// accumulators to scratch, counts itself in, waits for the others and then adds
// all parts, in their order, of its share of the tile's 32 x 32 blocks, whose
// epilogue it runs. (One CTA joining a tile of 8 parts alone takes 4 us at the
// 120 GB/s an SM reads.) The parts of a tile are consecutive items, and a CTA
// takes its items in ascending order, so the lowest unfinished tile never waits
// for a higher one.
//
// A launch may have several phases with a grid barrier between (a cooperative
// launch): what one phase's epilogues write the next one's TMA reads.
//
// Every wait on an mbarrier is bounded (tma.cuh); one that runs out latches a
// timeout, and the CTA ends without its results, after the copies that it has
// under way have landed and its products are done (bounded likewise).
#pragma once

#include <atomic>

#include "internal.h"
#include "product_items.h"
#include "tensor.cuh"

namespace efs {

constexpr uint32_t kTileNMax = 256; // columns of a tile, at most
constexpr uint32_t kTileK = 128;    // per stage: two 128-byte swizzle rows of 16-bit elements
constexpr uint32_t kEpilogueWarps = 8;
constexpr uint32_t kProductThreads = (2 + kEpilogueWarps) * 32;
constexpr uint32_t kBoxMnBytes = 64 * kTileK * 2;  // an MN-major box: 64 elements x 128 k

// Stages of the ring: 192 KB either way (a pair's are smaller, and more).
template <bool kPair>
struct Ring {
  static constexpr uint32_t kStages = kPair ? 3 : 2;
  static constexpr uint32_t kABytes = kTileM * kTileK * 2;
  static constexpr uint32_t kBBytes = (kPair ? kTileNMax / 2 : kTileNMax) * kTileK * 2;
  static constexpr uint32_t kStageBytes = kABytes + kBBytes;
  static constexpr uint32_t kBytes = kStages * kStageBytes;
};

// One product of a launch. The tensor maps are 3-D (innermost, rows, batch);
// a K-major operand's box is {64, rows a CTA loads}, an MN-major one's {64, 128}.
// With terms = 3 each operand is a sum hi + lo of two planes (batch entries
// 2 i and 2 i + 1 of its map), and D = hi hi + hi lo + lo hi.
struct ProductShape {
  CUtensorMap a, b;
  uint32_t m, n, k;
  uint32_t a_mn, b_mn, bf16, terms;
  uint32_t bn;                // columns per tile: a multiple of 64
  uint32_t tiles_m, tiles_n, batch, splits;
  uint32_t group_m;           // tiles are walked in groups of this many tile rows
  uint32_t lower;             // square tiles on and below the diagonal only
  uint32_t tiles;             // per batch entry
  uint32_t item0;             // this problem's first work item of its phase
  uint32_t part0;             // its first scratch tile (splits > 1)
  uint32_t join;              // parts are joined here (else the epilogue gets each)
  uint32_t counts;            // the launch's count bounds M (1) or K (2), or nothing (0)
};

struct ProductItem {
  uint32_t batch, tn, m0, n0, n_eff, rows, k, k0, kt, kts, part, split;
  bool skip;
};

template <bool kPair>
__device__ __forceinline__ ProductItem product_item(const ProductShape& p, uint32_t item,
                                                    uint32_t rank, uint32_t count) {
  constexpr uint32_t kRows = kPair ? 2 * kTileM : kTileM;
  // (divisions only where there is something to divide: an item's warps all wait
  // for this)
  ProductItem it;
  uint32_t r = item - p.item0;
  it.split = 0;
  it.batch = 0;
  if (p.splits > 1) {
    const uint32_t q = r / p.splits;
    it.split = r - q * p.splits;
    r = q;
  }
  if (p.batch > 1) {
    it.batch = r / p.tiles;
    r -= it.batch * p.tiles;
  }
  const uint32_t tile = r;
  uint32_t tm;
  if (p.lower) {  // tile row i holds i + 1 tiles
    uint32_t i = static_cast<uint32_t>(sqrtf(2.0f * static_cast<float>(r) + 0.25f) - 0.5f);
    while ((i + 1) * (i + 2) / 2 <= r) ++i;
    while (i * (i + 1) / 2 > r) --i;
    tm = i;
    it.tn = r - i * (i + 1) / 2;
  } else if (p.group_m == 1) {
    tm = r / p.tiles_n;
    it.tn = r - tm * p.tiles_n;
  } else {
    const uint32_t per = p.group_m * p.tiles_n;
    uint32_t g = 0, rows = p.tiles_m;
    if (p.group_m < p.tiles_m) {
      g = r / per;
      r -= g * per;
      rows = min(p.group_m, p.tiles_m - g * p.group_m);
    }
    it.tn = r / rows;
    tm = g * p.group_m + (r - it.tn * rows);
  }
  it.m0 = tm * kRows;
  it.n0 = it.tn * p.bn;
  it.n_eff = min(p.bn, (p.n - min(p.n, it.n0) + 31u) & ~31u);
  const uint32_t k = p.counts == 2 ? min(p.k, count) : p.k;
  it.skip = p.counts == 1 && it.m0 >= count;
  it.rows = p.counts == 1 ? min(p.m, count) : p.m;
  it.m0 += rank * kTileM;
  it.k = k;
  it.kts = (k + kTileK - 1) / kTileK;
  const uint32_t all = it.kts * p.terms;  // times splits: below 2^32 for any K of this library
  it.k0 = 0;
  it.kt = all;
  if (p.splits > 1) {
    it.k0 = all * it.split / p.splits;
    it.kt = all * (it.split + 1) / p.splits - it.k0;
  }
  it.part = p.part0 + ((it.batch * p.tiles + tile) * (kPair ? 2 : 1) + rank) * p.splits;
  return it;
}

constexpr uint32_t kMaxPhases = 16;

template <class Epi, int kMaxProblems>
struct ProductArgs {
  ProductShape shape[kMaxProblems];
  typename Epi::Params epi[kMaxProblems];
  uint32_t phases;
  uint32_t first[kMaxPhases], problems[kMaxPhases], items[kMaxPhases];  // of each phase
  const uint32_t* count;  // device: rows that exist (nullptr: all)
  float* parts;         // scratch tiles of split items
  uint32_t* arrivals;   // by the tile's first scratch tile; zero between tiles
  uint32_t part_chunks; // 32-column chunks per scratch tile
  uint32_t* error;
  uint32_t entries;     // problems in shape[]
  uint32_t turn;        // every other unit takes its items backwards (nothing joined)
  uint32_t* barrier;    // grid barrier: arrivals, CTAs finished (zero between launches)
  uint64_t wait_ns;
};

struct ProductSmem {
  uint64_t full[Ring<true>::kStages], empty[Ring<true>::kStages], acc_full[2], acc_empty[2], drained;
  uint32_t tmem, joined;
  uint32_t failed;  // an epilogue warp's wait ran out
};

// What an epilogue reads its accumulators through: 32 columns of the thread's
// row at a time, in order, from tensor memory or as the sum of the K parts.
struct ProductAcc {
  uint32_t tmem;            // address of the accumulator, the warp's lanes
  uint32_t release;         // barrier arrived on after the warp's last chunk was read
  uint32_t c0, c1;          // the warp's chunks
  const float* parts;       // != nullptr: sum `splits` scratch tiles instead
  uint64_t part_stride;     // floats from one part to the next
  uint32_t splits;
  bool none;                // K is empty: zeros

  __device__ __forceinline__ void arrive() const {
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive_cluster(release);
  }
  // All lanes of the warp call it alike.
  __device__ __forceinline__ void load(uint32_t c, float (&v)[32]) const {
    __syncwarp();
    if (none) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = 0.0f;
    } else if (parts) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = 0.0f;
      const float* src = parts + static_cast<uint64_t>(c) * (32 * kTileM);
#pragma unroll 2
      for (uint32_t s = 0; s < splits; ++s) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float4 x = __ldcg(reinterpret_cast<const float4*>(src + s * part_stride) + j * kTileM);
          v[4 * j] = __fadd_rn(v[4 * j], x.x);
          v[4 * j + 1] = __fadd_rn(v[4 * j + 1], x.y);
          v[4 * j + 2] = __fadd_rn(v[4 * j + 2], x.z);
          v[4 * j + 3] = __fadd_rn(v[4 * j + 3], x.w);
        }
      }
    } else {
      tmem_load_32(tmem + c * 32, v);
      if (c + 1 == c1) arrive();
    }
  }
};

// Parts of a joined block summed by several warps, kUnits of its eight groups of
// four columns each (a lane a row), in the place of the first part: one warp has
// registers for two parts on their way at a time, and sixteen parts took it 8 us.
template <int kUnits>
__device__ __forceinline__ void sum_parts(float4* first, uint64_t stride, uint32_t splits) {
  float4 sum[kUnits];
#pragma unroll
  for (int j = 0; j < kUnits; ++j) sum[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll (16 / kUnits)
  for (uint32_t s = 0; s < splits; ++s)
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      const float4 x = __ldcg(first + s * (stride / 4) + j * kTileM);
      sum[j] = make_float4(__fadd_rn(sum[j].x, x.x), __fadd_rn(sum[j].y, x.y),
                           __fadd_rn(sum[j].z, x.z), __fadd_rn(sum[j].w, x.w));
    }
#pragma unroll
  for (int j = 0; j < kUnits; ++j) __stcg(first + j * kTileM, sum[j]);
}

// How long a CTA that gives up waits for what it has under way.
constexpr uint64_t kDrainNs = 10000000;

// Waits until a counter has reached `target` (modulo 2^32).
__device__ __forceinline__ bool wait_count(const uint32_t* word, uint32_t target, uint64_t limit_ns) {
  const uint64_t t0 = global_timer_ns();
  uint32_t polls = 0;
  while (static_cast<int32_t>(ld_acquire_u32(word) - target) < 0)
    if ((++polls & 63u) == 0 && (polls > (1u << 26) || global_timer_ns() - t0 > limit_ns)) return false;
  return true;
}

// Barrier of all CTAs of a cooperative launch: `target` arrivals since the
// launch began. One word is counted up and polled.
__device__ __forceinline__ bool phase_barrier(uint32_t* word, uint32_t target, uint64_t limit_ns) {
  __syncthreads();
  bool ok = true;
  if (threadIdx.x == 0) {
    __threadfence();
    atomicAdd(word, 1u);
    ok = wait_count(word, target, limit_ns);
    __threadfence();
  }
  return __syncthreads_and(ok);
}

template <class Epi, int kMaxProblems, bool kPair>
__global__ void __launch_bounds__(kProductThreads, 1)
    product_kernel(const __grid_constant__ ProductArgs<Epi, kMaxProblems> args) {
  using R = Ring<kPair>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ ProductSmem s;
  __shared__ typename Epi::Smem epi_smem[kEpilogueWarps];
  uint8_t* stages = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = kPair ? cluster_rank() : 0u;
  const uint32_t unit = kPair ? blockIdx.x >> 1 : blockIdx.x;
  const uint32_t units = kPair ? gridDim.x >> 1 : gridDim.x;
  if (threadIdx.x == 0) {
    s.failed = 0;
    for (uint32_t i = 0; i < R::kStages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], kEpilogueWarps * (kPair ? 2 : 1));
    }
    mbar_init(&s.drained, 1);
    mbar_init_fence();
  }
  if (warp == 0)
    for (uint32_t i = lane; i < args.entries; i += 32) {
      prefetch_tensormap(&args.shape[i].a);
      prefetch_tensormap(&args.shape[i].b);
    }
  if (warp == 1) tmem_alloc<kPair>(&s.tmem, 512);
  tc_fence_before();
  __syncthreads();
  if (kPair) cluster_sync();
  tc_fence_after();
  const uint32_t tmem = s.tmem;
  griddep_wait();
  const uint32_t count = args.count ? *args.count : 0xffffffffu;
  bool ok = true;
  uint32_t stage = 0, phase = 0;    // ring position (producer, MMA)
  uint32_t acc = 0, acc_phase = 0;  // accumulator (MMA, epilogue)

  for (uint32_t ph = 0; ph < args.phases; ++ph) {
    const uint32_t prob0 = args.first[ph], prob1 = prob0 + args.problems[ph];
    const uint32_t items = args.items[ph];
    uint32_t prob = prob0;
    // (backwards, the index passes 0 to end above `items`)
    const bool back = Epi::kTurns && args.turn && (unit & 1u) && unit < items;
    const uint32_t first = back ? unit + (items - unit - 1) / units * units : unit;
    const uint32_t step = back ? 0u - units : units;
    if (warp == 0) {
      if (lane == 0) {
        fence_proxy_async();  // operands of this phase may come from the last one's epilogues
        for (uint32_t item = first; item < items && ok; item += step) {
          if (Epi::kTurns)
            while (item < args.shape[prob].item0) --prob;
          while (prob + 1 < prob1 && item >= args.shape[prob + 1].item0) ++prob;
          const ProductShape& p = args.shape[prob];
          const ProductItem it = product_item<kPair>(p, item, rank, count);
          if (it.skip) continue;
          const uint32_t half = kPair ? it.n_eff / 2 : it.n_eff;  // columns of B this CTA loads
          const uint32_t b_boxes = (half + 63) / 64, n0 = it.n0 + rank * half;
          const uint32_t b_rows = p.bn / (kPair ? 2 : 1);
          const uint32_t planes = p.terms > 1 ? 2 : 1;
          uint32_t term = it.k0 / max(it.kts, 1u), kk = it.k0 - term * it.kts;
          for (uint32_t kt = 0; kt < it.kt; ++kt) {
            if (!mbar_wait(&s.empty[stage], phase ^ 1u, args.wait_ns)) {
              ok = false;
              break;
            }
            uint8_t* a = stages + stage * R::kStageBytes;
            uint8_t* b = a + R::kABytes;
            const uint32_t k = kk * kTileK;
            const bool second = k + 64 < it.k;  // a K-major operand's other 64 of K
            const uint32_t za = it.batch * planes + (term == 2), zb = it.batch * planes + (term == 1);
            const uint32_t bar = kPair ? cluster_addr(&s.full[stage], 0) : smem_u32(&s.full[stage]);
            if (rank == 0) {
              const uint32_t a_bytes = p.a_mn || second ? R::kABytes : R::kABytes / 2;
              const uint32_t b_bytes = p.b_mn ? b_boxes * kBoxMnBytes : b_rows * (second ? 256u : 128u);
              mbar_arrive_expect_tx(&s.full[stage], (a_bytes + b_bytes) * (kPair ? 2 : 1));
            }
            if (p.a_mn) {
              tma_load_3d<kPair>(a, &p.a, it.m0, k, za, bar);
              tma_load_3d<kPair>(a + kBoxMnBytes, &p.a, it.m0 + 64, k, za, bar);
            } else {
              tma_load_3d<kPair>(a, &p.a, k, it.m0, za, bar);
              if (second) tma_load_3d<kPair>(a + R::kABytes / 2, &p.a, k + 64, it.m0, za, bar);
            }
            if (p.b_mn) {
              for (uint32_t x = 0; x < b_boxes; ++x)
                tma_load_3d<kPair>(b + x * kBoxMnBytes, &p.b, n0 + 64 * x, k, zb, bar);
            } else {
              tma_load_3d<kPair>(b, &p.b, k, n0, zb, bar);
              if (second) tma_load_3d<kPair>(b + b_rows * 128, &p.b, k + 64, n0, zb, bar);
            }
            if (++stage == R::kStages) {
              stage = 0;
              phase ^= 1u;
            }
            if (++kk == it.kts) {
              kk = 0;
              ++term;
            }
          }
        }
      }
    } else if (warp == 1) {
      if (lane == 0 && rank == 0) {
        for (uint32_t item = first; item < items && ok; item += step) {
          if (Epi::kTurns)
            while (item < args.shape[prob].item0) --prob;
          while (prob + 1 < prob1 && item >= args.shape[prob + 1].item0) ++prob;
          const ProductShape& p = args.shape[prob];
          const ProductItem it = product_item<kPair>(p, item, rank, count);
          if (it.skip || it.kt == 0) continue;
          if (!mbar_wait(&s.acc_empty[acc], acc_phase ^ 1u, args.wait_ns)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t idesc =
              mma_idesc(p.bf16, p.a_mn, p.b_mn, kPair ? 2 * kTileM : kTileM, it.n_eff);
          const uint32_t d = tmem + acc * kTileNMax;
          // 16 of K: 32 bytes along a K-major row (the second 64 of K follow the
          // first 64's rows), 16 rows of an MN-major tile
          const uint32_t a_step = (p.a_mn ? 2048u : 32u) >> 4, b_step = (p.b_mn ? 2048u : 32u) >> 4;
          const uint32_t b_rows = p.bn / (kPair ? 2 : 1);
          const uint32_t a_half = (p.a_mn ? 4 * 2048u : R::kABytes / 2) >> 4;
          const uint32_t b_half = (p.b_mn ? 4 * 2048u : b_rows * 128) >> 4;
          uint32_t kk = it.k0 % max(it.kts, 1u);
          for (uint32_t kt = 0; kt < it.kt; ++kt) {
            if (!mbar_wait(&s.full[stage], phase, args.wait_ns)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t a = smem_u32(stages + stage * R::kStageBytes);
            const uint64_t da = smem_desc(a, p.a_mn ? kBoxMnBytes : 16, 1024);
            const uint64_t db = smem_desc(a + R::kABytes, p.b_mn ? kBoxMnBytes : 16, 1024);
            const uint32_t steps = min(kTileK / 16, (it.k - kk * kTileK + 15) / 16);
            for (uint32_t j = 0; j < steps; ++j)
              mma_f16<kPair>(d, da + (j >> 2) * a_half + (j & 3u) * a_step,
                             db + (j >> 2) * b_half + (j & 3u) * b_step, idesc, kt > 0 || j > 0);
            if (++kk == it.kts) kk = 0;
            mma_commit<kPair>(&s.empty[stage]);
            if (++stage == R::kStages) {
              stage = 0;
              phase ^= 1u;
            }
          }
          mma_commit<kPair>(&s.acc_full[acc]);
          if (++acc == 2) {
            acc = 0;
            acc_phase ^= 1u;
          }
        }
      }
    } else {
      const uint32_t quarter = warp & 3u;  // the lanes of tensor memory this warp may read
      const uint32_t half = (warp - 2) >> 2;
      const uint32_t row = quarter * 32 + lane;
      for (uint32_t item = first; item < items; item += step) {
        if (Epi::kTurns)
          while (item < args.shape[prob].item0) --prob;
        while (prob + 1 < prob1 && item >= args.shape[prob + 1].item0) ++prob;
        const ProductShape& p = args.shape[prob];
        const ProductItem it = product_item<kPair>(p, item, rank, count);
        if (it.skip) continue;
        const uint32_t chunks = it.n_eff / 32, mid = (chunks + 1) / 2;
        ProductAcc from;
        from.c0 = half ? mid : 0;
        from.c1 = half ? chunks : mid;
        from.none = it.kt == 0;
        from.parts = nullptr;
        from.splits = p.splits;
        from.tmem = tmem + acc * kTileNMax + ((quarter * 32) << 16);
        from.release = kPair ? cluster_addr(&s.acc_empty[acc], 0) : smem_u32(&s.acc_empty[acc]);
        const typename Epi::Row state = Epi::prepare(p, args.epi[prob], it, row);
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
        if (!from.none && from.c0 == from.c1) from.arrive();
        uint32_t block = 0, blocks = 1;
        if (p.splits > 1 && p.join) {
          const uint64_t tile_floats = static_cast<uint64_t>(args.part_chunks) * 32 * kTileM;
          float* mine = args.parts + static_cast<uint64_t>(it.part) * tile_floats;
          float* dst = mine + it.split * tile_floats + row * 4;
          for (uint32_t c = from.c0; c < from.c1; ++c) {
            float v[32];
            from.load(c, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              __stcg(reinterpret_cast<float4*>(dst + static_cast<uint64_t>(c) * (32 * kTileM)) + j * kTileM,
                     make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
          }
          if (!ok) s.failed = 1;
          asm volatile("bar.sync 2, 256;" ::: "memory");
          if (warp == 2 && lane == 0) {
            __threadfence();
            // every part counts once more when it has seen all of them; the last
            // of those readies the counter for its next tile
            uint32_t* counter = &args.arrivals[it.part];
            atomicAdd(counter, 1u);
            const bool here = wait_count(counter, p.splits, ok ? args.wait_ns : 0);
            s.joined = here && !s.failed ? 1u : 0u;  // (all warps go on alike)
            if (here && atomicAdd(counter, 1u) == 2 * p.splits - 1) atomicExch(counter, 0u);
            __threadfence();
          }
          asm volatile("bar.sync 2, 256;" ::: "memory");
          ok = ok && s.joined != 0;
          asm volatile("bar.sync 2, 256;" ::: "memory");  // read before it is written again
          if (!ok) continue;
          block = it.split + (warp - 2) * p.splits;
          blocks = chunks * 4;
          from.none = false;
          from.part_stride = tile_floats;
          from.parts = mine;
          // from 8 parts on a CTA has at most half as many blocks as warps: two or
          // four warps sum a block, and the first of them runs its epilogue
          if (p.splits >= 8) {
            const uint32_t share = p.splits >= 16 ? 4 : 2, e = warp - 2;
            block = it.split + e / share * p.splits;
            if (block < blocks) {
              float4* first = reinterpret_cast<float4*>(mine) +
                              ((block >> 2) * 8 + e % share * (8 / share)) * kTileM +
                              (block & 3u) * 32 + lane;
              if (share == 4)
                sum_parts<2>(first, tile_floats, p.splits);
              else
                sum_parts<4>(first, tile_floats, p.splits);
            }
            asm volatile("bar.sync 2, 256;" ::: "memory");
            from.splits = 1;
            if (e % share) block = blocks;
          }
        }
        // the warp's half of the tile at once, or its 32 x 32 blocks of a joined one
        for (; block < blocks; block += kEpilogueWarps * p.splits) {
          uint32_t tile_row = row;
          ProductAcc at = from;
          if (from.parts) {
            at.c0 = block >> 2;
            at.c1 = at.c0 + 1;
            tile_row = (block & 3u) * 32 + lane;
            at.parts = from.parts + tile_row * 4;
          }
          Epi::tile(p, args.epi[prob], it, tile_row, half, epi_smem[warp - 2], at, ph, state);
        }
      }
    }
    __syncwarp();
    if (ph + 1 < args.phases) {
      ok = __syncthreads_and(ok);
      fence_proxy_async();
      if (!phase_barrier(args.barrier, gridDim.x * (ph + 1), args.wait_ns)) ok = false;
      if (!ok) break;
    }
  }
  griddep_launch_dependents();  // (they wait for this grid's end; their launch need not)
  if (!ok) atomicOr(args.error, kDevErrTimeout);
  if (args.phases > 1 && threadIdx.x == 0 &&
      atomicAdd(&args.barrier[1], 1u) == gridDim.x - 1) {  // all are past the last barrier
    args.barrier[0] = 0;
    args.barrier[1] = 0;
  }
  __syncwarp();
  tc_fence_before();
  if (!__syncthreads_and(ok)) {
    // a wait ran out: no copy may land and no product run after the CTA's end
    if (warp == 0 && lane == 0) {
      const uint64_t t0 = global_timer_ns();
      if (rank == 0)  // the last fill of every stage
        for (uint32_t i = 0; i < R::kStages; ++i)
          mbar_wait(&s.full[i], i < stage ? phase : phase ^ 1u, kDrainNs);
      // A pair's copies all count on rank 0's barriers, whose phases stay open where
      // the two CTAs stopped at different ones: there the time has to do.
      if (kPair)
        for (uint32_t i = 0; i < (1u << 20) && global_timer_ns() - t0 < kDrainNs; ++i)
          __nanosleep(1000);
    }
    if (warp == 1 && lane == 0 && rank == 0) {
      mma_commit<kPair>(&s.drained);
      mbar_wait(&s.drained, 0, kDrainNs);
    }
    __syncthreads();
  }
  if (kPair) cluster_sync();  // the other CTA's shared memory may be in use until here
  tc_fence_after();
  if (warp == 1) tmem_free<kPair>(tmem, 512);
}

// ------------------------------------------- epilogues' stores of 16-bit rows
// A lane's 32 columns of its row, at an address on a 32-byte boundary: two
// stores of a sector each (`cols` a multiple of 16).
__device__ __forceinline__ void store_row(uint16_t* p, const uint32_t (&w)[16], uint32_t cols) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (static_cast<uint32_t>(16 * i) < cols)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p + 16 * i),
                   "r"(w[8 * i]), "r"(w[8 * i + 1]), "r"(w[8 * i + 2]), "r"(w[8 * i + 3]),
                   "r"(w[8 * i + 4]), "r"(w[8 * i + 5]), "r"(w[8 * i + 6]), "r"(w[8 * i + 7])
                   : "memory");
}
// Other rows. A warp's 32 x 32 block of 16-bit values, each lane holding one row as 16
// words, through 2 KB of shared memory, so that stores cover whole sectors:
// 4 lanes per row with 16-byte rows (kVec16), 16 lanes per row with 4-byte
// rows, 32 with 2-byte ones. `rows(i)` gives the destination of block row i
// (nullptr: none).
struct TurnSmem {
  alignas(16) uint4 unit[32 * 4];
};
// `cols` of the 32 columns exist. kBatch: how many of the narrower stores are
// read ahead (registers).
template <int kBatch, class RowFn>
__device__ __forceinline__ void store_block(TurnSmem& t, const uint32_t (&w)[16], uint32_t cols,
                                            uint32_t align, RowFn rows) {
  const uint32_t lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (uint32_t u = 0; u < 4; ++u)
    t.unit[lane * 4 + (u ^ ((lane >> 1) & 3u))] =
        make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
  __syncwarp();
  // (everything is read before the first store: a store might alias)
  if (align >= 16 && cols % 8 == 0) {
    const uint32_t r0 = lane >> 2, u = lane & 3u;
    uint4 x[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t r = i * 8 + r0;
      x[i] = t.unit[r * 4 + (u ^ ((r >> 1) & 3u))];
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      uint16_t* to = rows(i * 8 + r0);
      if (to && u * 8 < cols) *reinterpret_cast<uint4*>(to + u * 8) = x[i];
    }
  } else if (align >= 4) {
    const uint32_t r0 = lane >> 4, col = (lane & 15u) * 2;
    const bool both = col + 1 < cols, one = col < cols;
#pragma unroll 1
    for (uint32_t i0 = 0; i0 < 16; i0 += kBatch) {
      uint32_t x[kBatch];
#pragma unroll
      for (uint32_t i = 0; i < kBatch; ++i) {
        const uint32_t r = (i0 + i) * 2 + r0;
        x[i] = reinterpret_cast<const uint32_t*>(
            &t.unit[r * 4 + ((col >> 3) ^ ((r >> 1) & 3u))])[(col >> 1) & 3u];
      }
#pragma unroll
      for (uint32_t i = 0; i < kBatch; ++i) {
        uint16_t* to = rows((i0 + i) * 2 + r0);
        if (to && both) *reinterpret_cast<uint32_t*>(to + col) = x[i];
        else if (to && one) to[col] = static_cast<uint16_t>(x[i]);
      }
    }
  } else {
    const bool in = lane < cols;
#pragma unroll 1
    for (uint32_t i0 = 0; i0 < 32; i0 += kBatch) {
      uint16_t x[kBatch];
#pragma unroll
      for (uint32_t i = 0; i < kBatch; ++i) {
        const uint32_t r = i0 + i;
        x[i] = reinterpret_cast<const uint16_t*>(
            &t.unit[r * 4 + ((lane >> 3) ^ ((r >> 1) & 3u))])[lane & 7u];
      }
#pragma unroll
      for (uint32_t i = 0; i < kBatch; ++i) {
        uint16_t* to = rows(i0 + i);
        if (to && in) to[lane] = x[i];
      }
    }
  }
}

// Rows on 4-byte boundaries whose blocks of 32 columns a warp stores one after
// another: 16 bytes at a time from the row's 16-byte boundaries on, the words
// past the last of them kept for the next block (`carry`: the lane's row). With
// 4-byte stores dw of 28,869 x 650 over 700 rows took 71 us with dh, so 62.
struct ShiftSmem {
  alignas(16) uint32_t word[32 * 20];  // a row: 4 words of the block before, then its own
};
template <class RowFn>
__device__ __forceinline__ void store_shifted(ShiftSmem& t, const uint32_t (&w)[16], uint4& carry,
                                              uint32_t cols, bool first, bool last, RowFn rows) {
  const uint32_t lane = threadIdx.x & 31;
  __syncwarp();
  uint4* mine = reinterpret_cast<uint4*>(t.word + lane * 20);
  mine[0] = carry;
#pragma unroll
  for (uint32_t u = 0; u < 4; ++u) mine[u + 1] = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
  carry = make_uint4(w[12], w[13], w[14], w[15]);
  __syncwarp();
  const int32_t full = static_cast<int32_t>(cols >> 1);  // whole words; an odd column follows
  const bool odd = cols & 1u;
  auto store_word = [&](uint16_t* to, int32_t at, uint32_t x) {
    if (at < full)
      *reinterpret_cast<uint32_t*>(to + 2 * at) = x;
    else if (at == full && odd)
      to[2 * at] = static_cast<uint16_t>(x);
  };
#pragma unroll
  for (uint32_t i0 = 0; i0 < 4; i0 += 2) {
    uint32_t x[2][4];
    uint16_t* to[2];
    int32_t from[2];
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
      const uint32_t r = (i0 + i) * 8 + (lane >> 2);
      to[i] = rows(r);
      const int32_t shift = static_cast<int32_t>((reinterpret_cast<uintptr_t>(to[i]) >> 2) & 3u);
      from[i] = static_cast<int32_t>(4 * (lane & 3u)) - shift;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) x[i][j] = t.word[r * 20 + 4 + from[i] + j];
    }
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
      if (!to[i]) continue;
      if ((from[i] >= 0 || !first) && from[i] + 4 <= full) {
        *reinterpret_cast<uint4*>(to[i] + 2 * from[i]) = make_uint4(x[i][0], x[i][1], x[i][2], x[i][3]);
      } else {
#pragma unroll
        for (int32_t j = 0; j < 4; ++j)
          if (from[i] + j >= 0 || !first) store_word(to[i], from[i] + j, x[i][j]);
      }
    }
  }
  if (last) {  // a row's words past its last 16-byte boundary
    uint16_t* to = rows(lane);
    const int32_t shift = static_cast<int32_t>((reinterpret_cast<uintptr_t>(to) >> 2) & 3u);
#pragma unroll
    for (int32_t j = 13; j < 16; ++j)
      if (to && j >= 16 - shift) store_word(to, j, w[j]);
  }
}

// A lane's row of a symmetric 32 x 32 block of which entries up to the diagonal
// are given: the others are read from the rows that mirror them.
__device__ __forceinline__ void mirror_block(TurnSmem& t, uint32_t (&w)[16]) {
  const uint32_t lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (uint32_t u = 0; u < 4; ++u)
    t.unit[lane * 4 + (u ^ ((lane >> 1) & 3u))] =
        make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
  __syncwarp();
#pragma unroll
  for (uint32_t j = 0; j < 32; ++j) {
    const uint32_t x = reinterpret_cast<const uint16_t*>(
        &t.unit[j * 4 + ((lane >> 3) ^ ((j >> 1) & 3u))])[lane & 7u];
    if (j > lane) w[j / 2] = j & 1u ? (w[j / 2] & 0xffffu) | (x << 16) : (w[j / 2] & 0xffff0000u) | x;
  }
}
// The largest of 32, 16, 4, 2 that every row of 16-bit elements starts on.
inline uint32_t row_align(const void* p, uint64_t ld) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p) | (ld * 2);
  return x % 32 == 0 ? 32 : x % 16 == 0 ? 16 : x % 4 == 0 ? 4 : 2;
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

// Fills bn, tiles, splits of a product of m x n x k (batch of them) on `sms`
// SMs, by CTAs or pairs.
struct ProductWant {
  uint32_t m, n, k, batch;
  bool lower, pair;
  double sms;
  uint32_t max_splits, terms;
  double epilogue;  // cycles per column of a tile (about: 128 rows, 8 warps)
  bool join;        // K parts are joined by the launch
};
void plan_product(ProductShape& p, const ProductWant& w);
// Rows and columns of B a CTA loads at a time (the box of a K-major operand).
inline uint32_t b_box(const ProductShape& p, bool pair) { return pair ? p.bn / 2 : p.bn; }

// Arrival counters of joined K parts; two words after them are the grid barrier.
constexpr uint32_t kPartCounters = kModelArrivals - 2;

// The caller has numbered the items and set args.parts.
template <class Epi, int kMaxProblems, bool kPair>
cudaError_t launch_product(ProductArgs<Epi, kMaxProblems>& args, Workspace& ws,
                           const DeviceInfo& dev) {
  uint32_t items = 0;
  for (uint32_t ph = 0; ph < args.phases; ++ph)
    items = args.items[ph] > items ? args.items[ph] : items;
  if (items == 0) return cudaSuccess;
  args.arrivals = ws.model_arrivals();
  args.error = ws.u32(kOffError);
  args.barrier = ws.model_arrivals() + kPartCounters;
  args.wait_ns = wait_limit_ns();
  auto fn = product_kernel<Epi, kMaxProblems, kPair>;
  constexpr uint32_t smem = Ring<kPair>::kBytes + 1024;
  static_assert(smem + sizeof(typename Epi::Smem) * kEpilogueWarps + 512 <= 227 * 1024,
                "stages and epilogue buffers fit an SM");
  static_assert(sizeof(args) <= 32764, "kernel parameters");
  // per device: opted into the ring's shared memory (by any of its threads)
  static std::atomic<bool> ready[64] = {};
  if (ws.device >= 64 || !ready[ws.device]) {
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (ws.device < 64) ready[ws.device] = true;
  }
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count), per = kPair ? 2 : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((items < sms / per ? items : sms / per) * per);
  cfg.blockDim = dim3(kProductThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = ws.stream;
  cudaLaunchAttribute attr[3];
  uint32_t n = 0;
  attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[n++].val.programmaticStreamSerializationAllowed = 1;
  if (args.phases > 1) {
    attr[n].id = cudaLaunchAttributeCooperative;
    attr[n++].val.cooperative = 1;
  }
  if (kPair) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = 2;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, args);
  if (e == cudaSuccess) count_launch();
  return e;
}

}  // namespace efs
