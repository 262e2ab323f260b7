// embed_grad.cu — the gradient of an embedding table: row w is the scaled sum of
// the rows of dout whose token is w, in fp32.
//
// What bounds it: reading dout once and writing the table's gradient once (or, where
// it is added to, the rows that occur). Sums run in a fixed order, without
// floating-point atomics: by groups of positions (every few-th occurrence, or those in
// one piece of the sorted list), each in the order of its positions, then over the groups. The sizes, the
// tokens, whether sums are added and the number of SMs fix the groups.
//
// Up to kFewTokens tokens of kFewValues values: one launch. A CTA per position looks through all
// tokens; if its own occurs before, another CTA has it, else it sums the rows of
// all its occurrences. Further CTAs write the rows that do not occur.
//
// More: the positions are sorted by token (stable, least digit first: for each digit
// a launch that counts it by parts of the positions, and one in which each CTA
// finds where its part goes from the counts of the parts before it). Then a warp
// takes 256 or 512 columns of a piece of the sorted positions, adds up rows and writes a
// row's sum when the token changes. A token that goes on past its piece leaves a
// share; the warp that leaves a token's last one joins them, in their order.
#include <algorithm>

#include "internal.h"
#include "vec_io.cuh"

namespace efs {
namespace {

// A CTA adds up a frequent word's rows by itself: of wide rows, fewer (of 350 words with 2164
// columns, 1024 positions take 12 us, sorted 14; 2000 take 19, sorted 15; 2000 of 650 columns
// 12 and 15).
constexpr uint32_t kFewTokens = 2048;
constexpr uint64_t kFewValues = uint64_t{9} << 18;
constexpr int kThreadsFew = 256;
constexpr int kLane = 8, kLaneMany = 16;  // columns a lane takes of a row: slices of 256, or 512
constexpr uint32_t kSlice = 32 * kLane;
constexpr uint32_t kSumWarps = 8;       // of a summing CTA
constexpr uint32_t kZeroRows = 64;       // rows that a CTA of zeros takes beside sums
constexpr uint32_t kRowsCta = 8192;     // and of a few tokens, at most
constexpr int kSortThreads = 512;
constexpr int kMaxBins = 512;
constexpr uint32_t kMaxParts = 296;     // sorting CTAs, at most
constexpr uint32_t kJoin = 16;          // shares that are joined at a time
constexpr uint32_t kPieceMost = 128;    // sorted positions that a warp adds up, at most

// A lane's L columns of a slice: vectors of V, 32 V apart.
template <int V, int L>
__device__ __forceinline__ uint32_t column(uint32_t slice, int k, uint32_t lane) {
  return slice * (32 * L) + (k * 32 + lane) * V;
}

template <typename T, int V, int L>
struct RowPart {
  Vec<T, V> x[L / V];
  __device__ __forceinline__ void load(const T* row, uint32_t slice, uint32_t lane, uint32_t d) {
#pragma unroll
    for (int k = 0; k < L / V; ++k) {
      const uint32_t c = column<V, L>(slice, k, lane);
      if (c < d) x[k].load(row + c);
      else x[k].clear();
    }
  }
  // Of a row that the kernel writes.
  __device__ __forceinline__ void load_own(const T* row, uint32_t slice, uint32_t lane, uint32_t d) {
#pragma unroll
    for (int k = 0; k < L / V; ++k) {
      const uint32_t c = column<V, L>(slice, k, lane);
      if (c < d) x[k].load_own(row + c);
    }
  }
  __device__ __forceinline__ void add_to(float (&sum)[L]) const {
#pragma unroll
    for (int k = 0; k < L / V; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) sum[k * V + j] += x[k].get(j);
  }
};

// scale sum, or (ADD) that added to what was there; rounded once.
template <typename T, int V, int L, bool ADD>
__device__ __forceinline__ void write_row(const EmbedGradCall& a, uint64_t row, uint32_t slice, uint32_t lane,
                                          const float (&sum)[L], const RowPart<T, V, L>& there) {
  T* to = static_cast<T*>(a.dtable) + row * a.ld_dtable;
#pragma unroll
  for (int k = 0; k < L / V; ++k) {
    const uint32_t c = column<V, L>(slice, k, lane);
    if (c < a.d) {
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j)
        f[j] = ADD ? fmaf(sum[k * V + j], a.scale, there.x[k].get(j)) : sum[k * V + j] * a.scale;
      Vec<T, V> o;
      o.round(f);
      o.store(to + c);
    }
  }
}

// Zeros over a row, 16 bytes at a time between its first and last boundary.
template <typename T>
__device__ __forceinline__ void zero_row(const EmbedGradCall& a, uint64_t row, uint32_t lane) {
  T* to = static_cast<T*>(a.dtable) + row * a.ld_dtable;
  constexpr uint32_t kPer = 16 / sizeof(T);
  const uint32_t lead = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(to) % 16 / sizeof(T));
  const uint32_t head = min(lead ? kPer - lead : 0u, a.d), body = (a.d - head) / kPer * kPer;
  if (lane < head) to[lane] = 0;
#pragma unroll 4
  for (uint32_t c = head + lane * kPer; c < head + body; c += 32 * kPer)
    *reinterpret_cast<uint4*>(to + c) = make_uint4(0u, 0u, 0u, 0u);
  if (head + body + lane < a.d) to[head + body + lane] = 0;
}

// ------------------------------------------------------------- few tokens
// CTAs by position, `chunks` of the columns each (566 positions of 350 words, 2164 columns:
// 16.5 us with all columns in one, 10.2 in three). The others: rows of the table, `rows` each.
template <typename D, typename T, int V, bool ADD>
__global__ void __launch_bounds__(kThreadsFew) embed_grad_few_kernel(const EmbedGradCall a, uint32_t rows, uint32_t chunks, uint32_t* error) {
  constexpr uint32_t kWarps = kThreadsFew / 32;
  constexpr int kAhead = V > 1 ? 8 : 4;  // rows on their way
  __shared__ uint32_t mask[kRowsCta / 32 > kFewTokens / 32 ? kRowsCta / 32 : kFewTokens / 32];
  __shared__ uint16_t list[kFewTokens];
  __shared__ float part[kWarps][kSlice];
  __shared__ uint32_t total;
  const uint32_t t = threadIdx.x, lane = t & 31u, warp = t >> 5;
  if (blockIdx.x >= a.n * chunks) {  // zeros
    const uint64_t lo = static_cast<uint64_t>(blockIdx.x - a.n * chunks) * rows;
    const uint64_t hi = min(lo + rows, static_cast<uint64_t>(a.v));
    for (uint32_t i = t; i < (rows + 31) / 32; i += kThreadsFew) mask[i] = 0u;
    __syncthreads();
    for (uint32_t i = t; i < a.n; i += kThreadsFew) {
      const int64_t w = __ldg(reinterpret_cast<const long long*>(a.token) + i);
      if (w >= static_cast<int64_t>(lo) && w < static_cast<int64_t>(hi))
        atomicOr(&mask[(w - lo) / 32], 1u << ((w - lo) & 31));
    }
    __syncthreads();
    for (uint64_t r = lo + warp; r < hi; r += kWarps)
      if (!(mask[(r - lo) / 32] >> ((r - lo) & 31) & 1u)) zero_row<T>(a, r, lane);
    return;
  }
  const uint32_t i = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const int64_t own = __ldg(reinterpret_cast<const long long*>(a.token) + i);
  const uint32_t words = (a.n + 31u) / 32u;
  constexpr uint32_t kLooks = kFewTokens / kThreadsFew;
  int64_t other[kLooks];
#pragma unroll
  for (uint32_t k = 0; k < kLooks; ++k) {
    const uint32_t j = k * kThreadsFew + t;
    other[k] = j < a.n ? __ldg(reinterpret_cast<const long long*>(a.token) + j) : -1;
  }
  if (__syncthreads_or(t < i && other[0] == own)) return;  // (frequent words are soon met)
  bool before = false;
#pragma unroll
  for (uint32_t k = 0; k < kLooks; ++k) {
    const uint32_t j = k * kThreadsFew + t;
    if (j < words * 32u) {
      const bool same = j < a.n && other[k] == own;
      before |= same && j < i;
      const uint32_t m = __ballot_sync(0xffffffffu, same);
      if (lane == 0) mask[j / 32] = m;
    }
  }
  if (own >= static_cast<int64_t>(a.v) && t == 0) atomicOr(error, kDevErrBadInput);
  if (own < 0 || own >= static_cast<int64_t>(a.v)) return;
  if (__syncthreads_or(before)) return;
  if (warp == 0) {  // the positions, in order
    uint32_t at = 0;
    for (uint32_t base = 0; base < words; base += 32) {
      uint32_t m = base + lane < words ? mask[base + lane] : 0u;
      const uint32_t count = __popc(m);
      uint32_t scan = count;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= static_cast<uint32_t>(o)) scan += x;
      }
      for (uint32_t k = at + scan - count; m; m &= m - 1)
        list[k++] = static_cast<uint16_t>((base + lane) * 32 + __ffs(m) - 1);
      at += __shfl_sync(0xffffffffu, scan, 31);
    }
    if (lane == 0) total = at;
  }
  __syncthreads();
  // the chunk's slices of columns over the warps; with fewer slices than warps, groups of
  // warps have all of them, each taking every groups-th occurrence
  const uint64_t all = (a.d + kSlice - 1) / kSlice;
  const uint32_t from = static_cast<uint32_t>(chunk * all / chunks);
  const uint32_t slices = static_cast<uint32_t>((chunk + 1) * all / chunks) - from;
  const uint32_t groups = slices < kWarps ? min(kWarps / slices, total) : 1u;
  const uint32_t group = slices < kWarps ? warp / slices : 0u;
  for (uint32_t s0 = 0; s0 < slices; s0 += kWarps) {
    const uint32_t at = slices < kWarps ? warp % slices : s0 + warp, slice = from + at;
    const bool work = group < groups && at < slices;
    float sum[kLane] = {};
    RowPart<T, V, kLane> there;
    if (ADD && work && group == 0)
      there.load_own(static_cast<T*>(a.dtable) + own * a.ld_dtable, slice, lane, a.d);
    if (work) {
      for (uint32_t k = group; k < total; k += groups * kAhead) {
        RowPart<D, V, kLane> row[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
          if (k + q * groups < total)
            row[q].load(static_cast<const D*>(a.dout) + static_cast<uint64_t>(list[k + q * groups]) * a.ld_dout,
                        slice, lane, a.d);
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
          if (k + q * groups < total) row[q].add_to(sum);
      }
    }
    if (groups > 1) {  // (then all slices are had at once)
      if (work && group > 0) {
#pragma unroll
        for (int j = 0; j < kLane; ++j) part[warp][j * 32 + lane] = sum[j];
      }
      __syncthreads();
      if (work && group == 0) {
        for (uint32_t g = 1; g < groups; ++g)
#pragma unroll
          for (int j = 0; j < kLane; ++j) sum[j] += part[g * slices + warp][j * 32 + lane];
      }
    }
    if (work && group == 0) write_row<T, V, kLane, ADD>(a, static_cast<uint64_t>(own), slice, lane, sum, there);
  }
}

// ------------------------------------------------------------------ sorting
struct Sort {
  uint32_t n, v, bits, passes, parts, per;  // per: positions a part takes (tiles of 512 R)
  uint32_t* hist;         // [parts][bins] of a digit
  uint32_t *key[2], *pos[2];
  uint32_t* error;
  const int64_t* token;
  uint32_t *arrived, arrivals;  // of the shares: see Sum
};

__device__ __forceinline__ uint32_t digit_of(const Sort& s, uint32_t key, uint32_t pass) {
  return (key >> (pass * s.bits)) & ((1u << s.bits) - 1u);
}

// Counts of a digit by part. The first launch makes the keys of the tokens, too, and
// zeros for the arrivals of shares.
__global__ void __launch_bounds__(kSortThreads) embed_count_kernel(const Sort s, uint32_t pass) {
  __shared__ uint32_t hist[kMaxBins];
  const uint32_t bins = 1u << s.bits, t = threadIdx.x;
  for (uint32_t b = t; b < bins; b += kSortThreads) hist[b] = 0u;
  if (pass == 0)
    for (uint32_t i = blockIdx.x * kSortThreads + t; i < s.arrivals; i += gridDim.x * kSortThreads) s.arrived[i] = 0u;
  griddep_wait();
  __syncthreads();
  const uint32_t lo = blockIdx.x * s.per, hi = min(lo + s.per, s.n);
  bool bad = false;
#pragma unroll 4
  for (uint32_t i0 = lo; i0 < hi; i0 += kSortThreads) {
    const uint32_t i = i0 + t;
    uint32_t key = s.v;
    if (i < hi) {
      if (pass == 0) {
        const int64_t w = __ldg(reinterpret_cast<const long long*>(s.token) + i);
        bad |= w >= static_cast<int64_t>(s.v);
        if (w >= 0 && w < static_cast<int64_t>(s.v)) key = static_cast<uint32_t>(w);
        s.key[0][i] = key;
      } else {
        key = __ldcg(s.key[pass & 1u] + i);
      }
    }
    // (131,072 x 1024: 118 us, with 95 % of it padding, one digit, 87; with a warp's equal digits matched to be
    // one addition 121 and 88)
    if (i < hi) atomicAdd(&hist[digit_of(s, key, pass)], 1u);
  }
  griddep_launch_dependents();  // (the scatter, which waits for this kernel's end)
  if (bad) atomicOr(s.error, kDevErrBadInput);
  __syncthreads();
  for (uint32_t b = t; b < bins; b += kSortThreads) s.hist[blockIdx.x * bins + b] = hist[b];
}

// One digit. Positions keep their order: a warp takes consecutive ones, and a
// position's rank is the number of equal digits before it in its warp, in the
// warps before, in the tiles before and in the parts before.
template <int kPer>
__global__ void __launch_bounds__(kSortThreads) embed_scatter_kernel(const Sort s, uint32_t pass) {
  constexpr int kWarps = kSortThreads / 32;
  constexpr uint32_t kSortTile = kSortThreads * kPer;
  __shared__ uint32_t base[kMaxBins];           // where the part's next position of a digit goes
  __shared__ __align__(16) uint16_t count[kWarps][kMaxBins];
  __shared__ uint32_t sums[kWarps];
  griddep_wait();
  const uint32_t bins = 1u << s.bits, t = threadIdx.x, lane = t & 31u, warp = t >> 5;
  const uint32_t* hist = s.hist;
  const uint32_t* keys = s.key[pass & 1u];
  const uint32_t* from = s.pos[pass & 1u];
  uint32_t *keys_out = s.key[(pass + 1u) & 1u], *to = s.pos[(pass + 1u) & 1u];
  {  // a thread a digit: the parts before, then all parts; and the digits before
    uint32_t before = 0, all = 0;
    if (t < bins) {
      constexpr int kAhead = 32;  // (a load takes half a microsecond: few rounds of many)
      for (uint32_t p0 = 0; p0 < s.parts; p0 += kAhead) {
        uint32_t c[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) c[q] = p0 + q < s.parts ? __ldcg(hist + (p0 + q) * bins + t) : 0u;
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          before += p0 + q < blockIdx.x ? c[q] : 0u;
          all += c[q];
        }
      }
    }
    uint32_t scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= static_cast<uint32_t>(o)) scan += x;
    }
    if (lane == 31) sums[warp] = scan;
    __syncthreads();
    uint32_t under = 0;
    for (uint32_t w = 0; w < warp; ++w) under += sums[w];
    if (t < bins) base[t] = under + scan - all + before;
  }
  griddep_launch_dependents();
  const uint32_t lo = blockIdx.x * s.per, hi = min(lo + s.per, s.n);
  for (uint32_t tile = lo; tile < hi; tile += kSortTile) {
    for (uint32_t i = t; i < kWarps * kMaxBins / 8; i += kSortThreads)
      reinterpret_cast<uint4*>(&count[0][0])[i] = make_uint4(0u, 0u, 0u, 0u);
    uint32_t key[kPer], rank[kPer], digit[kPer], pos[kPer];
    const uint32_t at = tile + warp * (32 * kPer) + lane;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const uint32_t i = at + 32 * k;
      key[k] = i < hi ? keys[i] : 0u;
      pos[k] = i < hi ? (pass ? from[i] : i) : 0u;
      digit[k] = i < hi ? digit_of(s, key[k], pass) : bins;  // (no digit)
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const uint32_t same = __match_any_sync(0xffffffffu, digit[k]);
      const bool in = digit[k] < bins;
      const uint32_t had = in ? count[warp][digit[k]] : 0u;
      rank[k] = had + __popc(same & lanemask_lt());
      __syncwarp();
      if (in && (same & lanemask_lt()) == 0u) count[warp][digit[k]] = static_cast<uint16_t>(had + __popc(same));
      __syncwarp();
    }
    __syncthreads();
    uint32_t total = 0;
    if (t < bins) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const uint32_t c = count[w][t];
        count[w][t] = static_cast<uint16_t>(total);
        total += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (digit[k] < bins) {
        const uint32_t out = base[digit[k]] + count[warp][digit[k]] + rank[k];
        keys_out[out] = key[k];
        to[out] = pos[k];
      }
    }
    __syncthreads();
    if (t < bins) base[t] += total;
  }
}

// ------------------------------------------------------------------ summing
struct Sum {
  // (read by ordinary loads: the launch that writes them may still run when the sums' begins)
  const uint32_t *key, *pos;
  float* shares;          // [pieces][2][d]: a token from the piece before, one that goes on
  // [pieces][3][slices]: shares of a join whose first is the piece's, from the piece before
  // or going on; joins of the token that begins and goes on there
  uint32_t* arrived;
  uint32_t piece, pieces, slices, warps;  // positions a piece; warps that sum
  uint32_t rows;          // rows a CTA of zeros takes
};

// The first position whose token is at least `key`.
__device__ __forceinline__ uint32_t first_of(const uint32_t* keys, uint32_t n, uint32_t key) {
  uint32_t lo = 0, hi = n;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (keys[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// A sum's columns to a share's place, and from it (which this kernel writes, too).
template <int V, int L>
__device__ __forceinline__ void write_share(float* to, uint32_t slice, uint32_t lane, uint32_t d, const float (&sum)[L]) {
#pragma unroll
  for (int k = 0; k < L / V; ++k) {
    const uint32_t c = column<V, L>(slice, k, lane);
    if (c < d) {
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = sum[k * V + j];
      Vec<float, V> x;
      x.round(f);
      x.store(to + c);
    }
  }
}
template <int V, int L>
__device__ __forceinline__ void read_share(const float* from, uint32_t slice, uint32_t lane, uint32_t d, float (&x)[L]) {
#pragma unroll
  for (int k = 0; k < L / V; ++k) {
    const uint32_t c = column<V, L>(slice, k, lane);
    if (c < d) {
      if constexpr (V == 8) {
#pragma unroll
        for (int h = 0; h < V; h += 4) {
          const float4 f = __ldcg(reinterpret_cast<const float4*>(from + c + h));
          x[k * V + h] = f.x, x[k * V + h + 1] = f.y, x[k * V + h + 2] = f.z, x[k * V + h + 3] = f.w;
        }
      } else if constexpr (V == 2) {
        const float2 f = __ldcg(reinterpret_cast<const float2*>(from + c));
        x[k * V] = f.x, x[k * V + 1] = f.y;
      } else {
        x[k] = __ldcg(from + c);
      }
    }
  }
}

// A warp's share of a token that several pieces have: slot 0 of its piece where it
// has come from the piece before, else slot 1.
__device__ __forceinline__ float* share_at(const Sum& s, uint32_t piece, uint32_t slot, uint32_t d) {
  return s.shares + (static_cast<uint64_t>(piece) * 2 + slot) * d;
}

// The pieces that begin with the token from piece q + 1 on, or (back) those before q that
// end with it: how many there are without a gap. Most runs end within a look at 32
// pieces; the ends of long ones are searched.
__device__ __forceinline__ uint32_t run_of(const Sum& s, uint32_t n, uint32_t token, uint32_t q, uint32_t lane,
                                           bool back) {
  const uint32_t step = 1 + lane;
  bool same = false;
  if (back) same = step <= q && s.key[(q - step + 1) * s.piece - 1] == token;
  else same = q + step < s.pieces && s.key[(q + step) * s.piece] == token;
  const uint32_t m = __ballot_sync(0xffffffffu, same);
  if (m != 0xffffffffu) return __ffs(~m) - 1;
  return back ? q - first_of(s.key, n, token) / s.piece : (first_of(s.key, n, token + 1) - 1) / s.piece - q;
}

// Whether this warp is the last of `of` at a counter. It then sees what the others have left.
__device__ __forceinline__ bool last_of(uint32_t* arrived, uint32_t of, uint32_t lane) {
  uint32_t had = 0;
  if (lane == 0) {
    had = atomicAdd(arrived, 1u);
    __threadfence();
  }
  had = __shfl_sync(0xffffffffu, had, 0);
  __syncwarp();  // (what lane 0 has seen, all have)
  return had + 1 == of;
}

// Where a token's shares are all there with this warp's: their sum, in order of the
// pieces, kJoin at a time; the sums of kJoin, left in the place of their first, likewise
// (one after another, the 150 shares of a word that 48,135 have 4800 times take 10 us more).
// (Lane 0 has made the warp's shares visible.)
template <typename T, int V, int L, bool ADD>
__device__ __forceinline__ void join_shares(const EmbedGradCall& a, const Sum& s, uint32_t token, uint32_t piece,
                                            uint32_t slice, uint32_t lane, bool came, bool on) {
  const uint32_t before = came ? run_of(s, a.n, token, piece, lane, true) : 0u;
  const uint32_t after = on ? run_of(s, a.n, token, piece, lane, false) : 0u;
  uint32_t first = piece - before, shares = before + 1 + after;  // of the run
  const uint32_t head = first, joins = (shares + kJoin - 1) / kJoin, join = before / kJoin;
  auto counter = [&](uint32_t at, uint32_t of) { return s.arrived + (static_cast<uint64_t>(at) * 3 + of) * s.slices + slice; };
  first += join * kJoin;  // of the join
  shares = min(shares - join * kJoin, kJoin);
  uint32_t step = 1;
  if (!last_of(counter(first, join ? 0 : 1), shares, lane)) return;
  RowPart<T, V, L> there;
  if (ADD && joins == 1)
    there.load_own(static_cast<T*>(a.dtable) + static_cast<uint64_t>(token) * a.ld_dtable, slice, lane, a.d);
  constexpr uint32_t kAhead = 32 / L;  // shares on their way
  while (true) {
    float sum[L] = {};
    for (uint32_t q0 = 0; q0 < shares; q0 += kAhead) {
      float x[kAhead][L];
#pragma unroll
      for (uint32_t q = 0; q < kAhead; ++q) {
        const uint32_t at = first + (q0 + q) * step;
        if (q0 + q < shares) read_share<V, L>(share_at(s, at, at == head ? 1 : 0, a.d), slice, lane, a.d, x[q]);
      }
#pragma unroll
      for (uint32_t q = 0; q < kAhead; ++q)
        if (q0 + q < shares)
#pragma unroll
          for (int j = 0; j < L; ++j) sum[j] += x[q][j];
    }
    if (step > 1 || joins == 1) {
      write_row<T, V, L, ADD>(a, token, slice, lane, sum, there);
      return;
    }
    write_share<V, L>(share_at(s, first, first == head ? 1 : 0, a.d), slice, lane, a.d, sum);
    __syncwarp();
    if (lane == 0) __threadfence();
    if (!last_of(counter(head, 2), joins, lane)) return;
    if (ADD)
      there.load_own(static_cast<T*>(a.dtable) + static_cast<uint64_t>(token) * a.ld_dtable, slice, lane, a.d);
    first = head;
    shares = joins;
    step = kJoin;
  }
}

template <typename D, typename T, int V, int L, bool ADD>
__global__ void __launch_bounds__(32 * kSumWarps) embed_sum_kernel(const EmbedGradCall a, const Sum s) {
  __shared__ uint32_t room[kSumWarps][2][kPieceMost];
  griddep_wait();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const uint32_t sum_ctas = (s.warps + kSumWarps - 1) / kSumWarps;
  if (blockIdx.x >= sum_ctas) {  // zeros, where a row's token does not occur
    const uint64_t lo = static_cast<uint64_t>(blockIdx.x - sum_ctas) * s.rows;
    const uint64_t hi = min(lo + s.rows, static_cast<uint64_t>(a.v));
    __shared__ uint8_t occurs[kZeroRows];
    if (lo + threadIdx.x < hi && threadIdx.x < kZeroRows) {
      const uint32_t row = static_cast<uint32_t>(lo) + threadIdx.x, at = first_of(s.key, a.n, row);
      occurs[threadIdx.x] = at < a.n && s.key[at] == row;
    }
    __syncthreads();
    for (uint64_t r = lo + warp; r < hi; r += kSumWarps)
      if (!occurs[r - lo]) zero_row<T>(a, r, lane);
    return;
  }
  const uint32_t item = blockIdx.x * kSumWarps + warp;
  if (item >= s.warps) return;
  const uint32_t slice = item % s.slices, piece = item / s.slices;
  const uint32_t lo = piece * s.piece, count = min(s.piece, a.n - lo);
  uint32_t *keys = room[warp][0], *at = room[warp][1];
  for (uint32_t i = lane; i < count; i += 32) {
    keys[i] = s.key[lo + i];
    at[i] = s.pos[lo + i];
  }
  const uint32_t last = lo > 0 ? s.key[lo - 1] : a.v, next = lo + count < a.n ? s.key[lo + count] : a.v;
  __syncwarp();
  // rows on their way; and (ADD) the rows of the table that sums end in meanwhile
  constexpr uint32_t kAhead = sizeof(D) == 2 && V > 2 && L == kLane && !ADD ? 8 : L == kLane || sizeof(D) == 2 ? 4 : 2;
  RowPart<D, V, L> rows[kAhead];
  RowPart<T, V, L> there[ADD ? kAhead : 1];
  float sum[L] = {};
  const uint32_t first = keys[0], end = keys[count - 1];
  const bool came = first < a.v && last == first;  // the first token has come from the piece before
  const bool on = end < a.v && next == end;        // the last one goes on in the next piece
  bool share = came;                               // the sum at hand is a share
  uint32_t token = first;
  auto finish = [&](bool goes_on, const RowPart<T, V, L>& was) {
    if (share || goes_on) write_share<V, L>(share_at(s, piece, share ? 0 : 1, a.d), slice, lane, a.d, sum);
    else if (token < a.v) write_row<T, V, L, ADD>(a, token, slice, lane, sum, was);
  };
  for (uint32_t i0 = 0; i0 < count; i0 += kAhead) {
#pragma unroll
    for (uint32_t q = 0; q < kAhead; ++q) {
      const uint32_t i = i0 + q;
      if (i < count && keys[i] < a.v) {
        rows[q].load(static_cast<const D*>(a.dout) + static_cast<uint64_t>(at[i]) * a.ld_dout, slice, lane, a.d);
        if (ADD && (i + 1 == count || keys[i + 1] != keys[i]))
          there[ADD ? q : 0].load_own(static_cast<const T*>(a.dtable) + static_cast<uint64_t>(keys[i]) * a.ld_dtable,
                                      slice, lane, a.d);
      }
    }
    // A sum is written at its last row where the table's row has come for it (ADD), else
    // when the next one begins (131,075 x 1024: 153 us; at the last row 167).
#pragma unroll
    for (uint32_t q = 0; q < kAhead; ++q) {
      const uint32_t i = i0 + q;
      if (i < count) {
        const uint32_t key = keys[i];
        if (!ADD && key != token) finish(false, there[0]);
        if (key != token) {
          token = key;
          share = false;
#pragma unroll
          for (int j = 0; j < L; ++j) sum[j] = 0.0f;
        }
        if (key < a.v) {
          rows[q].add_to(sum);
          if (ADD && (i + 1 == count || keys[i + 1] != key)) finish(i + 1 == count && on, there[ADD ? q : 0]);
        }
      }
    }
  }
  if (!ADD) finish(on, there[0]);
  if (!came && !on) return;
  __syncwarp();
  if (lane == 0) __threadfence();
  const bool whole = came && first == end;  // one token, with one share
  if (came) join_shares<T, V, L, ADD>(a, s, first, piece, slice, lane, true, whole && on);
  if (on && !whole) join_shares<T, V, L, ADD>(a, s, end, piece, slice, lane, false, true);
}

// ------------------------------------------------------------------ planning
struct Plan {
  bool few;
  uint32_t v;       // values per vector
  uint32_t rounds;  // positions that a sorting thread ranks at a time
  uint32_t lane;    // columns that a summing lane takes
  uint32_t chunks;  // of the columns, of few tokens
  Sort sort;
  Sum sum;
  size_t hist, key, shares, bytes;  // sizes, in bytes
};

Plan plan_of(const EmbedGradCall& c, const DeviceInfo& dev) {
  Plan p = {};
  const uint32_t dsize = c.dout_bf16 ? 2 : 4, tsize = c.dtable_bf16 ? 2 : 4;
  auto allow = [&](uint32_t v) {
    auto rows = [&](const void* q, uint64_t ld, uint64_t size) {
      return (reinterpret_cast<uintptr_t>(q) | ld * size) % (size * v) == 0;
    };
    return c.d % v == 0 && rows(c.dout, c.n > 1 ? c.ld_dout : 0, dsize) &&
           rows(c.dtable, c.v > 1 ? c.ld_dtable : 0, tsize);
  };
  p.v = allow(8) ? 8 : allow(2) ? 2 : 1;
  p.few = c.n <= kFewTokens && static_cast<uint64_t>(c.n) * c.d <= std::max(kFewValues, uint64_t{256} * c.d);
  const uint32_t sms = static_cast<uint32_t>(dev.sm_count);
  p.sum.rows = std::max(8u, std::min((c.v + 4 * sms - 1) / (4 * sms), kRowsCta));
  if (p.few) {
    // Each chunk's CTAs look through all tokens: up to 32 CTAs an SM, and narrow chunks only where
    // words are met often (2000 x 650: of 350 words 11.8 us with 2 slices, 17.3 with 4; of 33,278
    // 23.9 and 19.3).
    const uint32_t slices = (c.d + kSlice - 1) / kSlice, span = c.n >= c.v ? 2 : 4;
    p.chunks = std::max(1u, std::min((slices + span - 1) / span, 32 * sms / std::max(c.n, 1u)));
    return p;
  }
  p.sum.rows = kZeroRows;
  Sort& s = p.sort;
  uint32_t bits = 1;
  while (bits < 31 && (c.v >> bits) != 0) ++bits;  // of the keys, v itself among them
  s.passes = (bits + 8) / 9;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.n = c.n;
  s.v = c.v;
  p.rounds = c.n <= 32768 ? 1 : 4;
  const uint32_t tile = kSortThreads * p.rounds;
  s.per = ((c.n + kMaxParts - 1) / kMaxParts + tile - 1) / tile * tile;
  s.parts = (c.n + s.per - 1) / s.per;
  Sum& m = p.sum;
  // (16 columns a lane, and the rows that they are added to, would leave a CTA an SM)
  p.lane = c.n >= 65536 && p.v == 8 && c.d > 2 * kSlice && !c.add ? kLaneMany : kLane;
  m.slices = (c.d + 32 * p.lane - 1) / (32 * p.lane);
  // positions a piece: many warps of short lists, few shares of long ones (131,075 x 1024:
  // 149 us with 128, 154 with 64; added, 131,072 x 1001 154 with 64, 157 with 32)
  m.piece = c.n <= 16384 ? 16 : c.n < 65536 ? 32 : c.add ? kPieceMost / 2 : kPieceMost;
  m.pieces = (c.n + m.piece - 1) / m.piece;
  m.warps = m.pieces * m.slices;
  auto round = [](size_t x) { return (x + 255) & ~static_cast<size_t>(255); };
  p.hist = round(static_cast<size_t>(s.parts) * (4u << s.bits));
  p.key = round(static_cast<size_t>(c.n) * 4);
  p.shares = round(static_cast<size_t>(m.pieces) * 2 * c.d * 4);
  s.arrivals = 3 * m.warps;
  p.bytes = p.hist + 4 * p.key + p.shares + round(static_cast<size_t>(s.arrivals) * 4);
  return p;
}

template <typename D, typename T, int V, bool ADD>
cudaError_t launch(const EmbedGradCall& c, const Plan& p, cudaStream_t stream) {
  uint32_t zeros = c.add ? 0 : (c.v + p.sum.rows - 1) / p.sum.rows;
  EmbedGradCall a = c;
  if (p.few) {
    if (c.n + zeros == 0) return cudaSuccess;
    count_launch();
    embed_grad_few_kernel<D, T, V, ADD>
        <<<c.n * p.chunks + zeros, kThreadsFew, 0, stream>>>(a, p.sum.rows, p.chunks, p.sort.error);
    return cudaGetLastError();
  }
  Sum s = p.sum;
  void* params[] = {&a, &s};
  count_launch();
  const void* kernel = reinterpret_cast<const void*>(embed_sum_kernel<D, T, V, kLane, ADD>);
  if constexpr (V == 8 && !ADD)  // (as planned)
    if (p.lane == kLaneMany) kernel = reinterpret_cast<const void*>(embed_sum_kernel<D, T, V, kLaneMany, ADD>);
  return launch_pdl(kernel,
                    dim3((s.warps + kSumWarps - 1) / kSumWarps + zeros), 32 * kSumWarps, 0, stream, params, false);
}

template <typename D, typename T, int V>
cudaError_t launch(const EmbedGradCall& c, const Plan& p, cudaStream_t stream) {
  return c.add ? launch<D, T, V, true>(c, p, stream) : launch<D, T, V, false>(c, p, stream);
}
template <typename D, typename T>
cudaError_t launch_typed(const EmbedGradCall& c, const Plan& p, cudaStream_t stream) {
  if (p.v == 8) return launch<D, T, 8>(c, p, stream);
  return p.v == 2 ? launch<D, T, 2>(c, p, stream) : launch<D, T, 1>(c, p, stream);
}

}  // namespace

size_t embed_grad_scratch(const EmbedGradCall& c, const DeviceInfo& dev) { return plan_of(c, dev).bytes; }

cudaError_t launch_embed_grad(const EmbedGradCall& c, Workspace& ws, const DeviceInfo& dev) {
  Plan p = plan_of(c, dev);
  p.sort.error = ws.u32(kOffError);
  cudaError_t err = cudaSuccess;
  if (!p.few) {
    Sort& s = p.sort;
    char* at = ws.model_scratch();
    s.hist = reinterpret_cast<uint32_t*>(at);
    at += p.hist;
    for (int i = 0; i < 2; ++i) {
      s.key[i] = reinterpret_cast<uint32_t*>(at);
      s.pos[i] = reinterpret_cast<uint32_t*>(at + p.key);
      at += 2 * p.key;
    }
    p.sum.shares = reinterpret_cast<float*>(at);
    p.sum.arrived = s.arrived = reinterpret_cast<uint32_t*>(at + p.shares);
    p.sum.key = s.key[s.passes & 1u];
    p.sum.pos = s.pos[s.passes & 1u];
    s.token = c.token;
    for (uint32_t pass = 0; pass < s.passes; ++pass) {
      void* params[] = {&s, &pass};
      const void* scatter = p.rounds == 1 ? reinterpret_cast<const void*>(embed_scatter_kernel<1>)
                                          : reinterpret_cast<const void*>(embed_scatter_kernel<4>);
      count_launch();
      if (pass == 0) embed_count_kernel<<<s.parts, kSortThreads, 0, ws.stream>>>(s, pass);
      else err = launch_pdl(reinterpret_cast<const void*>(embed_count_kernel), dim3(s.parts), kSortThreads, 0,
                            ws.stream, params, false);
      if (err == cudaSuccess) err = cudaGetLastError();
      if (err != cudaSuccess) return err;
      count_launch();
      err = launch_pdl(scatter, dim3(s.parts), kSortThreads, 0, ws.stream, params, false);
      if (err != cudaSuccess) return err;
    }
  }
  if (c.dout_bf16)
    return c.dtable_bf16 ? launch_typed<bf16_t, bf16_t>(c, p, ws.stream) : launch_typed<bf16_t, float>(c, p, ws.stream);
  return c.dtable_bf16 ? launch_typed<float, bf16_t>(c, p, ws.stream) : launch_typed<float, float>(c, p, ws.stream);
}

}  // namespace efs
