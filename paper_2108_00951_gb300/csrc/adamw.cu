// adamw.cu — an AdamW step over a list of tensors in one launch:
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2,
//   p <- p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
//
// What bounds it: p, m and v are read and written, g is read, once: 28 bytes an
// entry, 16 with states in 8 bits. A CTA takes a piece of one tensor; it finds
// its tensor in the kernel's parameters, so a list of many small tensors costs
// one launch.
//
// States in 8 bits. Blocks of 128 entries share a byte E + 127, E the exponent of
// the block's largest magnitude (at least -92). A code is an exponent field f and
// three bits k (in m under a sign and with 4 bits of f, in v with 5) and stands for
// (8 + k) 2^(E - top + f - 3), or k 2^(E - top - 2) where f = 0; top is 14 in m and 30 in v, so
// the largest entry has room to round up. In steps of at least 2^-4 of its value a
// moving average that changes by a thousandth a step would never change at all
// when rounded to nearest; the rounding is stochastic, so it moves by the right
// amount on the average. A positive v is never held as zero: the update divides by
// its root. 16 random bits for each state come from the entry's number, the
// tensor's, the step and the seed, so equal calls give equal bits.
//
// A code's bits, 20 places up, are the fp32 number of value times 2^(top - 127 - E)
// (small codes are its subnormal numbers): coding is two exact products by powers
// of two, one addition of the random bits below the last place and a shift.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "vec_io.cuh"

namespace efs {
namespace {

constexpr int kAdamThreads = 256;
constexpr uint32_t kBlock = 128;           // entries that share an exponent
constexpr uint32_t kPiece = 4096;          // entries per CTA
constexpr int kTopM = 14, kTopV = 30, kLeast = -92;

__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

struct Entry {
  AdamTensor t;
  uint32_t first;   // CTA of the tensor's first piece
  uint32_t wide;    // all its pointers on 16 bytes (codes 4, bf16 8)
};
template <int N>
struct AdamArgs {
  float b1, c1, b2, c2, eps;
  float step_size, root, keep;   // lr / (1 - b1^t), (1 - b2^t)^(-1/2), 1 - lr wd
  double log_b1, log_b2;         // with step_dev
  float lr, decay;               // with lr_dev or step_dev
  uint32_t seed, step, first_tensor, n;
  const float* lr_dev;
  const int64_t* step_dev;
  const float* grad_scale;
  Entry entry[N];
};

__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

struct Hyper {
  float b1, c1, b2, c2, eps, step_size, root, keep, scale;
};

// One entry: m and v as they are kept in fp32 (each operation rounded by itself),
// p by approximate root and quotient (2^-22 of the update, lr times which is far
// below p's last place). (Packed in pairs the operations would be half as many, but
// the assembler fuses packed products and sums, whatever rounding they name.)
__device__ __forceinline__ void update(const Hyper& h, float& p, float g, float& m, float& v) {
  g *= h.scale;
  m = m * h.b1 + g * h.c1;
  v = v * h.b2 + g * g * h.c2;
  float root, inverse;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
  // (of 2^-75 or more, or 0: nothing to flush)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(fmaf(root, h.root, h.eps)));
  p = fmaf(-h.step_size, m * inverse, p * h.keep);
}

// A code's value from byte j of a word, in units of f: 2^(127 + E - top), which is
// in fp32's range for E up to top; above, the rest of it comes after.
__device__ __forceinline__ float decode_m(uint32_t word, int j, float f) {
  const int t = static_cast<int>(__byte_perm(word, 0u, 0x0444u | (j << 12)));  // the byte on top
  return __int_as_float((t >> 4) & 0x87f00000) * f;
}
__device__ __forceinline__ float decode_v(uint32_t word, int j, float f) {
  return __uint_as_float(__byte_perm(word, 0u, 0x4044u | (j << 8)) << 4) * f;
}
// What few blocks hold (NaN, or E above top), out of the way of the others' registers.
struct States {
  float m[4], v[4];
};
__device__ __noinline__ States decode_rare(uint32_t mc, uint32_t vc, int em, int ev) {
  States s;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s.m[j] = decode_m(mc, j, power(127 + min(em, kTopM) - kTopM)) * power(max(em - kTopM, 0));
    s.v[j] = decode_v(vc, j, power(127 + min(ev, kTopV) - kTopV)) * power(max(ev - kTopV, 0));
    if (((mc >> (8 * j)) & 127u) == 127u) s.m[j] = __int_as_float(0x7fffffff);
    if (((vc >> (8 * j)) & 255u) == 255u) s.v[j] = __int_as_float(0x7fffffff);
  }
  return s;
}
__device__ __forceinline__ void decode(uint32_t mc, uint32_t vc, int em, int ev, float (&m)[4], float (&v)[4]) {
  // a byte of m with seven ones, or one of v with eight
  const uint32_t nan = (((mc & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) | ((~vc - 0x01010101u) & vc & 0x80808080u);
  if (nan || em > kTopM || ev > kTopV) {
    const States s = decode_rare(mc, vc, em, ev);
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = s.m[j], v[j] = s.v[j];
    return;
  }
  const float fm = power(127 + em - kTopM), fv = power(127 + ev - kTopV);
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = decode_m(mc, j, fm), v[j] = decode_v(vc, j, fv);
}
__device__ __forceinline__ int exponent_of(uint32_t e) { return max(static_cast<int>(e) - 127, kLeast); }

constexpr uint32_t kTooLarge = 0x7f000000u;  // the bits of 2^127: not held from there on
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t held_bits(float x) { return magnitude(x) < kTooLarge ? magnitude(x) : 0u; }

// The code of x >= 0 in the top byte; f: 2^(top - 127 - E); `random`: 16 bits, 8 places up, and a
// half below them. (The product is truncated, so that a small code rounds up for
// the right random numbers exactly.)
__device__ __forceinline__ uint32_t encode(float x, float f, uint32_t random) {
  return __float_as_uint(__fmul_rz(x, f)) * 16u + random;
}
__device__ __forceinline__ uint32_t encode_m(float m, float scaled, float f, uint32_t r) {
  return (encode(fabsf(scaled), f, __byte_perm(r, 0x80u, 0x5104u)) & 0x7f000000u) |
         (__float_as_uint(m) & 0x80000000u);
}
__device__ __forceinline__ uint32_t encode_v(float scaled, float f, uint32_t r) {
  return encode(scaled, f, __byte_perm(r, 0x80u, 0x5324u));
}
// The top bytes of four words.
__device__ __forceinline__ uint32_t top_bytes(const uint32_t (&x)[4]) {
  return __byte_perm(__byte_perm(x[0], x[1], 0x0073u), __byte_perm(x[2], x[3], 0x0073u), 0x5410u);
}

// Codes and exponents of a block's states: a lane has four entries from `at` on, `gap`
// apart, those below hi.
struct Codes {
  uint32_t m, v;
  int em, ev;
};
// Any block: values too large to be held, and an E for which f is no normal number
// (the block is scaled down first; its entries stay normal numbers, or are far too
// small to be held).
__device__ __noinline__ Codes encode_rare(States s, uint32_t at, uint32_t gap, uint32_t hi, uint32_t key) {
  uint32_t top_m = 0u, top_v = 0u, ms[4], vs[4];
  for (int j = 0; j < 4; ++j) {
    if (gap == 1u || at + gap * j < hi) {
      top_m = max(top_m, held_bits(s.m[j]));
      top_v = max(top_v, held_bits(s.v[j]));
    }
  }
  Codes c;
  c.em = max(static_cast<int>(__reduce_max_sync(0xffffffffu, top_m) >> 23) - 127, kLeast);
  c.ev = max(static_cast<int>(__reduce_max_sync(0xffffffffu, top_v) >> 23) - 127, kLeast);
  const int down_m = c.em >= kTopM ? 114 : 0, down_v = c.ev >= kTopV ? 98 : 0;
  const float fm = power(kTopM - 127 - (c.em - down_m)), fv = power(kTopV - 127 - (c.ev - down_v));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t r = mix32(at + gap * j + key);
    ms[j] = encode_m(s.m[j], s.m[j] * power(-down_m), fm, r);
    vs[j] = max(encode_v(s.v[j] * power(-down_v), fv, r), s.v[j] > 0.0f ? 1u << 24 : 0u);
    if (magnitude(s.m[j]) >= kTooLarge) ms[j] = 0x7f000000u | (__float_as_uint(s.m[j]) & 0x80000000u);
    if (magnitude(s.v[j]) >= kTooLarge) vs[j] = 0xff000000u;
  }
  c.m = top_bytes(ms);
  c.v = top_bytes(vs);
  return c;
}
__device__ __forceinline__ Codes encode(const float (&m)[4], const float (&v)[4], uint32_t at, uint32_t gap,
                                        uint32_t hi, uint32_t key) {
  uint32_t top_m = 0u, top_v = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (gap == 1u || at + gap * j < hi) {
      top_m = max(top_m, magnitude(m[j]));
      top_v = max(top_v, __float_as_uint(v[j]));  // (never negative)
    }
  }
  top_m = __reduce_max_sync(0xffffffffu, top_m);
  top_v = __reduce_max_sync(0xffffffffu, top_v);
  if (top_m >= (127u + kTopM) << 23 || top_v >= (127u + kTopV) << 23) {  // of the whole block
    States s;
#pragma unroll
    for (int j = 0; j < 4; ++j) s.m[j] = m[j], s.v[j] = v[j];
    return encode_rare(s, at, gap, hi, key);
  }
  Codes c;
  c.em = max(static_cast<int>(top_m >> 23) - 127, kLeast);
  c.ev = max(static_cast<int>(top_v >> 23) - 127, kLeast);
  const float fm = power(kTopM - 127 - c.em), fv = power(kTopV - 127 - c.ev);
  uint32_t ms[4], vs[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t r = mix32(at + gap * j + key);
    ms[j] = encode_m(m[j], m[j], fm, r);
    vs[j] = encode_v(v[j], fv, r);
  }
  if (min(min(vs[0], vs[1]), min(vs[2], vs[3])) < 1u << 24) {  // a positive v is held as one
#pragma unroll
    for (int j = 0; j < 4; ++j) vs[j] = max(vs[j], v[j] > 0.0f ? 1u << 24 : 0u);
  }
  c.m = top_bytes(ms);
  c.v = top_bytes(vs);
  return c;
}

template <typename A>
__device__ __forceinline__ uint32_t find_entry(const A& a, uint32_t cta) {
  uint32_t lo = 0, hi = a.n;  // entry lo begins at or before the CTA, hi after it
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.entry[mid].first <= cta) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <typename A>
__device__ __forceinline__ Hyper hyper_of(const A& a, uint32_t& step) {
  Hyper h = {a.b1, a.c1, a.b2, a.c2, a.eps, a.step_size, a.root, a.keep, 1.0f};
  step = a.step;
  if (a.lr_dev || a.step_dev) {
    const float lr = a.lr_dev ? __ldg(a.lr_dev) : a.lr;
    if (a.lr_dev) h.keep = 1.0f - lr * a.decay;
    if (a.step_dev) {
      const int64_t t = max(__ldg(reinterpret_cast<const long long*>(a.step_dev)), 1ll);
      step = static_cast<uint32_t>(t);
      const double n = static_cast<double>(t);
      h.step_size = lr / -expm1f(static_cast<float>(n * a.log_b1));
      h.root = 1.0f / sqrtf(-expm1f(static_cast<float>(n * a.log_b2)));
    } else {
      h.step_size = lr * a.step_size;  // (then 1 / (1 - b1^t))
    }
  }
  if (a.grad_scale) h.scale = __ldg(a.grad_scale);
  return h;
}

template <typename G, int N>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamArgs<N> a) {
  const uint32_t which = find_entry(a, blockIdx.x);
  const Entry& e = a.entry[which];
  const uint32_t lo = (blockIdx.x - e.first) * kPiece, hi = min(lo + kPiece, e.t.numel);
  float* p = e.t.p;
  const G* g = static_cast<const G*>(e.t.g);
  float *m = static_cast<float*>(e.t.m), *v = static_cast<float*>(e.t.v);
  uint32_t step;
  const Hyper h = hyper_of(a, step);
  uint32_t i = lo;
  if (e.wide) {
#pragma unroll 2
    for (uint32_t at = lo + threadIdx.x * 4; at + 4 <= hi; at += kAdamThreads * 4) {
      Vec<float, 4> ps, ms, vs;
      Vec<G, 4> gs;
      ps.load_own(p + at);
      gs.load(g + at);
      ms.load_own(m + at);
      vs.load_own(v + at);
      float po[4], go[4], mo[4], vo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) po[j] = ps.get(j), go[j] = gs.get(j), mo[j] = ms.get(j), vo[j] = vs.get(j);
#pragma unroll
      for (int j = 0; j < 4; ++j) update(h, po[j], go[j], mo[j], vo[j]);
      ps.round(po);
      ms.round(mo);
      vs.round(vo);
      ps.store(p + at);
      ms.store(m + at);
      vs.store(v + at);
      if (e.t.copy) {
        Vec<bf16_t, 4> c;
        c.round(po);
        c.store(e.t.copy + at);
      }
    }
    i = hi & ~3u;
  }
#pragma unroll 4
  for (uint32_t at = i + threadIdx.x; at < hi; at += kAdamThreads) {
    float po = p[at], mo = m[at], vo = v[at];
    update(h, po, widen(g[at]), mo, vo);
    p[at] = po;
    m[at] = mo;
    v[at] = vo;
    if (e.t.copy) e.t.copy[at] = round_bf16(po);
  }
}

// A warp takes four blocks of 128 entries, eight apart, and a lane four entries of each:
// consecutive where the pointers allow vectors, else 32 apart. Everything is
// loaded before the first store. The piece's exponents are read by each warp at
// once and written by the CTA at once: bytes of one sector, read and written one
// by one from several SMs, took most of the time (25.6 M entries: 317 us).
constexpr int kBlocksWarp = kPiece / kBlock / (kAdamThreads / 32);
static_assert(kPiece / kBlock == 32, "a lane an exponent");

template <typename G, int N>
__global__ void __launch_bounds__(kAdamThreads) adamw8_kernel(const __grid_constant__ AdamArgs<N> a) {
  __shared__ uint8_t exponents[2][kPiece / kBlock];
  const uint32_t which = find_entry(a, blockIdx.x);
  const Entry& e = a.entry[which];
  const uint32_t lo = (blockIdx.x - e.first) * kPiece, hi = min(lo + kPiece, e.t.numel);
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  float* p = e.t.p;
  const G* g = static_cast<const G*>(e.t.g);
  uint8_t *m = static_cast<uint8_t*>(e.t.m), *v = static_cast<uint8_t*>(e.t.v);
  const uint32_t first = lo / kBlock, blocks = (hi - lo + kBlock - 1) / kBlock;
  const uint32_t my_em = lane < blocks ? e.t.me[first + lane] : 0u;
  const uint32_t my_ev = lane < blocks ? e.t.ve[first + lane] : 0u;
  float po[kBlocksWarp][4], go[kBlocksWarp][4];
  uint32_t mc[kBlocksWarp], vc[kBlocksWarp];
#pragma unroll
  for (int q = 0; q < kBlocksWarp; ++q) {
    const uint32_t base = lo + (q * (kAdamThreads / 32) + warp) * kBlock;
    mc[q] = vc[q] = 0u;
    if (e.wide && base + kBlock <= hi) {
      const uint32_t at = base + lane * 4;
      Vec<float, 4> ps;
      Vec<G, 4> gs;
      ps.load_own(p + at);
      gs.load(g + at);
      mc[q] = *reinterpret_cast<const uint32_t*>(m + at);
      vc[q] = *reinterpret_cast<const uint32_t*>(v + at);
#pragma unroll
      for (int j = 0; j < 4; ++j) po[q][j] = ps.get(j), go[q][j] = gs.get(j);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = base + lane + 32u * j;
        const bool in = i < hi;
        po[q][j] = in ? p[i] : 0.0f;
        go[q][j] = in ? widen(g[i]) : 0.0f;
        mc[q] |= (in ? m[i] : 0u) << (8 * j);
        vc[q] |= (in ? v[i] : 0u) << (8 * j);
      }
    }
  }
  uint32_t step;
  const Hyper h = hyper_of(a, step);
  const uint32_t key = mix32(mix32(a.seed + step) + 0x9E3779B9u * (a.first_tensor + which));
#pragma unroll
  for (int q = 0; q < kBlocksWarp; ++q) {
    const uint32_t block = q * (kAdamThreads / 32) + warp, base = lo + block * kBlock;
    const int em = exponent_of(__shfl_sync(0xffffffffu, my_em, block));
    const int ev = exponent_of(__shfl_sync(0xffffffffu, my_ev, block));
    if (base >= hi) break;
    const bool wide = e.wide && base + kBlock <= hi;
    const uint32_t at = wide ? base + lane * 4 : base + lane, gap = wide ? 1u : 32u;
    float mo[4], vo[4];
    decode(mc[q], vc[q], em, ev, mo, vo);
#pragma unroll
    for (int j = 0; j < 4; ++j) update(h, po[q][j], go[q][j], mo[j], vo[j]);
    const Codes c = encode(mo, vo, at, gap, hi, key);
    if (wide) {
      Vec<float, 4> ps;
      ps.round(po[q]);
      ps.store(p + at);
      *reinterpret_cast<uint32_t*>(m + at) = c.m;
      *reinterpret_cast<uint32_t*>(v + at) = c.v;
      if (e.t.copy) {
        Vec<bf16_t, 4> rounded;
        rounded.round(po[q]);
        rounded.store(e.t.copy + at);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = at + 32u * j;
        if (i < hi) {
          p[i] = po[q][j];
          m[i] = static_cast<uint8_t>(c.m >> (8 * j));
          v[i] = static_cast<uint8_t>(c.v >> (8 * j));
          if (e.t.copy) e.t.copy[i] = round_bf16(po[q][j]);
        }
      }
    }
    if (lane == 0) {
      exponents[0][block] = static_cast<uint8_t>(c.em + 127);
      exponents[1][block] = static_cast<uint8_t>(c.ev + 127);
    }
  }
  // (each warp has read the old ones before it stored its own)
  __syncthreads();
  if (warp == 0 && lane < blocks) {
    e.t.me[first + lane] = exponents[0][lane];
    e.t.ve[first + lane] = exponents[1][lane];
  }
}

struct StateEntry {
  AdamStates t;
  uint32_t first, wide;
};
template <int N>
struct StatesArgs {
  uint32_t n;
  StateEntry entry[N];
};

template <typename T, int N>
__global__ void __launch_bounds__(kAdamThreads) adamw_states_kernel(const __grid_constant__ StatesArgs<N> a) {
  const StateEntry& e = a.entry[find_entry(a, blockIdx.x)];
  const uint32_t lo = (blockIdx.x - e.first) * kPiece, hi = min(lo + kPiece, e.t.numel);
  T *m = static_cast<T*>(e.t.m_out), *v = static_cast<T*>(e.t.v_out);
  uint32_t i = lo;
  if (e.wide) {
    // eight entries a thread at a time
#pragma unroll
    for (uint32_t q = 0; q < kPiece / (8 * kAdamThreads); ++q) {
      const uint32_t at = lo + (q * kAdamThreads + threadIdx.x) * 8;
      if (at + 8 > hi) break;
      const uint2 mc = __ldg(reinterpret_cast<const uint2*>(e.t.m + at));
      const uint2 vc = __ldg(reinterpret_cast<const uint2*>(e.t.v + at));
      const int em = exponent_of(__ldg(e.t.me + at / kBlock)), ev = exponent_of(__ldg(e.t.ve + at / kBlock));
      float mo[2][4], vo[2][4];
      decode(mc.x, vc.x, em, ev, mo[0], vo[0]);
      decode(mc.y, vc.y, em, ev, mo[1], vo[1]);
      constexpr int kVec = 16 / sizeof(T);  // values of 16 bytes
#pragma unroll
      for (int j = 0; j < 8; j += kVec) {
        float f[kVec], h[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) f[k] = mo[(j + k) / 4][(j + k) % 4], h[k] = vo[(j + k) / 4][(j + k) % 4];
        Vec<T, kVec> ms, vs;
        ms.round(f);
        vs.round(h);
        ms.store(m + at + j);
        vs.store(v + at + j);
      }
    }
    i = hi & ~7u;
  }
#pragma unroll 2
  for (uint32_t at = i + threadIdx.x; at < hi; at += kAdamThreads) {
    float mo[4], vo[4];
    decode(__ldg(e.t.m + at), __ldg(e.t.v + at), exponent_of(__ldg(e.t.me + at / kBlock)),
           exponent_of(__ldg(e.t.ve + at / kBlock)), mo, vo);
    store_rounded(m + at, mo[0]);
    store_rounded(v + at, vo[0]);
  }
}

bool on(const void* p, uintptr_t size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

// Fills a launch's entries from `list` on; returns its CTAs.
template <typename A, typename T, typename Wide>
uint32_t fill(A& a, int most, const T* list, uint32_t n, uint32_t& next, Wide wide) {
  uint32_t ctas = 0;
  a.n = 0;
  for (; next < n && static_cast<int>(a.n) < most; ++next) {
    const uint32_t pieces = (list[next].numel + (kPiece - 1ull)) / kPiece;
    if (ctas + static_cast<uint64_t>(pieces) > 0x7fffffffu) break;
    auto& e = a.entry[a.n++];
    e.t = list[next];
    e.first = ctas;
    e.wide = wide(list[next]);
    ctas += pieces;
  }
  return ctas;
}

// Kernel parameters for 8, 64 or 400 tensors: a launch copies them.
template <typename G, int N>
cudaError_t adamw_in(const AdamTensor* t, uint32_t n, const AdamCall& c, cudaStream_t stream) {
  AdamArgs<N> a;
  const double t1 = 1.0 - std::pow(c.b1, static_cast<double>(c.step));
  const double t2 = 1.0 - std::pow(c.b2, static_cast<double>(c.step));
  a.b1 = static_cast<float>(c.b1);
  a.c1 = static_cast<float>(1.0 - c.b1);
  a.b2 = static_cast<float>(c.b2);
  a.c2 = static_cast<float>(1.0 - c.b2);
  a.eps = static_cast<float>(c.eps);
  a.step_size = static_cast<float>((c.lr_dev ? 1.0 : c.lr) / t1);
  a.root = static_cast<float>(1.0 / std::sqrt(t2));
  a.keep = static_cast<float>(1.0 - c.lr * c.decay);
  a.log_b1 = std::log(c.b1);
  a.log_b2 = std::log(c.b2);
  a.lr = static_cast<float>(c.lr);
  a.decay = static_cast<float>(c.decay);
  a.seed = mix32(mix32(static_cast<uint32_t>(c.seed)) ^ static_cast<uint32_t>(c.seed >> 32));
  a.step = static_cast<uint32_t>(c.step);
  a.lr_dev = c.lr_dev;
  a.step_dev = c.step_dev;
  a.grad_scale = c.grad_scale;
  auto wide = [&](const AdamTensor& x) -> uint32_t {
    const uintptr_t state = c.eight ? 4 : 16;
    return on(x.p, 16) && on(x.g, sizeof(G) * 4) && on(x.m, state) && on(x.v, state) && on(x.copy, 8);
  };
  for (uint32_t next = 0; next < n;) {
    a.first_tensor = next;
    const uint32_t ctas = fill(a, N, t, n, next, wide);
    if (ctas == 0) continue;
    count_launch();
    if (c.eight) adamw8_kernel<G, N><<<ctas, kAdamThreads, 0, stream>>>(a);
    else adamw_kernel<G, N><<<ctas, kAdamThreads, 0, stream>>>(a);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}
template <typename G>
cudaError_t adamw_typed(const AdamTensor* t, uint32_t n, const AdamCall& c, cudaStream_t stream) {
  if (n <= 8) return adamw_in<G, 8>(t, n, c, stream);
  return n <= 64 ? adamw_in<G, 64>(t, n, c, stream) : adamw_in<G, 400>(t, n, c, stream);
}

template <typename T, int N>
cudaError_t states_in(const AdamStates* t, uint32_t n, cudaStream_t stream) {
  StatesArgs<N> a;
  auto wide = [&](const AdamStates& x) -> uint32_t {
    return on(x.m, 8) && on(x.v, 8) && on(x.m_out, 16) && on(x.v_out, 16);
  };
  for (uint32_t next = 0; next < n;) {
    const uint32_t ctas = fill(a, N, t, n, next, wide);
    if (ctas == 0) continue;
    count_launch();
    adamw_states_kernel<T, N><<<ctas, kAdamThreads, 0, stream>>>(a);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}
template <typename T>
cudaError_t states_typed(const AdamStates* t, uint32_t n, cudaStream_t stream) {
  if (n <= 8) return states_in<T, 8>(t, n, stream);
  return n <= 64 ? states_in<T, 64>(t, n, stream) : states_in<T, 400>(t, n, stream);
}

}  // namespace

cudaError_t launch_adamw(const AdamTensor* t, uint32_t n, const AdamCall& c, cudaStream_t stream) {
  return c.g_bf16 ? adamw_typed<bf16_t>(t, n, c, stream) : adamw_typed<float>(t, n, c, stream);
}

cudaError_t launch_adamw_states(const AdamStates* t, uint32_t n, bool out_bf16, cudaStream_t stream) {
  return out_bf16 ? states_typed<bf16_t>(t, n, stream) : states_typed<float>(t, n, stream);
}

}  // namespace efs
