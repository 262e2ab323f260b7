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
// below p's last place).
__device__ __forceinline__ void update(const Hyper& h, float& p, float g, float& m, float& v) {
  m = m * h.b1 + g * h.c1;
  v = v * h.b2 + g * g * h.c2;
  float root;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
  const float u = __fdividef(m, fmaf(root, h.root, h.eps));
  p = fmaf(-h.step_size, u, p * h.keep);
}

template <bool SIGNED>
__device__ __forceinline__ float decode(uint32_t code, float f) {
  const uint32_t a = SIGNED ? code & 127u : code;
  float x = __uint_as_float(a << 20) * power(126) * f;
  if (a == (SIGNED ? 127u : 255u)) x = __int_as_float(0x7fffffff);
  return SIGNED && (code & 128u) ? -x : x;
}
// The factor of a block's values: 2^(E - top + 1).
__device__ __forceinline__ float decode_factor(uint32_t e, int top) {
  return power(max(static_cast<int>(e) - 127, kLeast) - top + 1);
}

// The bits of |x| where it can be held, 0 elsewhere (NaN, or 2^127 and more).
__device__ __forceinline__ uint32_t held_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f000000u ? b : 0u;
}
// f: 2^(top - 1 - E).
template <bool SIGNED>
__device__ __forceinline__ uint32_t encode(float x, float f, uint32_t random16) {
  // (truncated, so that a small code rounds up for the right random numbers exactly)
  const float z = __fmul_rz(fabsf(x) * f, power(-126));
  uint32_t code = (__float_as_uint(z) + (random16 << 4) + 8u) >> 20;
  if (!SIGNED && x > 0.0f && code == 0u) code = 1u;
  if (!(fabsf(x) < 0x1p127f)) code = SIGNED ? 127u : 255u;
  return SIGNED ? code | (__float_as_uint(x) >> 31 << 7) : code;
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
      float po[4], mo[4], vo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        po[j] = ps.get(j), mo[j] = ms.get(j), vo[j] = vs.get(j);
        update(h, po[j], gs.get(j) * h.scale, mo[j], vo[j]);
      }
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
    update(h, po, widen(g[at]) * h.scale, mo, vo);
    p[at] = po;
    m[at] = mo;
    v[at] = vo;
    if (e.t.copy) e.t.copy[at] = round_bf16(po);
  }
}

// A warp takes a block of 128 entries at a time, four a lane: consecutive where
// the pointers allow vectors, else 32 apart.
template <typename G, int N>
__global__ void __launch_bounds__(kAdamThreads) adamw8_kernel(const __grid_constant__ AdamArgs<N> a) {
  const uint32_t which = find_entry(a, blockIdx.x);
  const Entry& e = a.entry[which];
  const uint32_t lo = (blockIdx.x - e.first) * kPiece, hi = min(lo + kPiece, e.t.numel);
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  float* p = e.t.p;
  const G* g = static_cast<const G*>(e.t.g);
  uint8_t *m = static_cast<uint8_t*>(e.t.m), *v = static_cast<uint8_t*>(e.t.v);
  uint32_t step;
  const Hyper h = hyper_of(a, step);
  const uint32_t key = mix32(mix32(a.seed + step) + 0x9E3779B9u * (a.first_tensor + which));
#pragma unroll 2
  for (uint32_t b = lo / kBlock + warp; b * kBlock < hi; b += kAdamThreads / 32) {
    const uint32_t base = b * kBlock;
    const bool wide = e.wide && base + kBlock <= hi;
    const uint32_t at = wide ? base + lane * 4 : base + lane, gap = wide ? 1u : 32u;
    float po[4], go[4], mo[4], vo[4];
    uint32_t mc = 0u, vc = 0u;
    if (wide) {
      Vec<float, 4> ps;
      Vec<G, 4> gs;
      ps.load_own(p + at);
      gs.load(g + at);
      mc = *reinterpret_cast<const uint32_t*>(m + at);
      vc = *reinterpret_cast<const uint32_t*>(v + at);
#pragma unroll
      for (int j = 0; j < 4; ++j) po[j] = ps.get(j), go[j] = gs.get(j);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = at + 32u * j;
        const bool in = i < hi;
        po[j] = in ? p[i] : 0.0f;
        go[j] = in ? widen(g[i]) : 0.0f;
        mc |= (in ? m[i] : 0u) << (8 * j);
        vc |= (in ? v[i] : 0u) << (8 * j);
      }
    }
    const float fm = decode_factor(e.t.me[b], kTopM), fv = decode_factor(e.t.ve[b], kTopV);
    uint32_t top_m = 0u, top_v = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      mo[j] = decode<true>((mc >> (8 * j)) & 255u, fm);
      vo[j] = decode<false>((vc >> (8 * j)) & 255u, fv);
      update(h, po[j], go[j] * h.scale, mo[j], vo[j]);
      if (wide || at + 32u * j < hi) {
        top_m = max(top_m, held_bits(mo[j]));
        top_v = max(top_v, held_bits(vo[j]));
      }
    }
    const int em = max(static_cast<int>(__reduce_max_sync(0xffffffffu, top_m) >> 23) - 127, kLeast);
    const int ev = max(static_cast<int>(__reduce_max_sync(0xffffffffu, top_v) >> 23) - 127, kLeast);
    const float dm = power(kTopM - 1 - em), dv = power(kTopV - 1 - ev);
    mc = vc = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t r = mix32(at + gap * j + key);
      mc |= encode<true>(mo[j], dm, r & 0xffffu) << (8 * j);
      vc |= encode<false>(vo[j], dv, r >> 16) << (8 * j);
    }
    if (wide) {
      Vec<float, 4> ps;
      ps.round(po);
      ps.store(p + at);
      *reinterpret_cast<uint32_t*>(m + at) = mc;
      *reinterpret_cast<uint32_t*>(v + at) = vc;
      if (e.t.copy) {
        Vec<bf16_t, 4> c;
        c.round(po);
        c.store(e.t.copy + at);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = at + 32u * j;
        if (i < hi) {
          p[i] = po[j];
          m[i] = static_cast<uint8_t>(mc >> (8 * j));
          v[i] = static_cast<uint8_t>(vc >> (8 * j));
          if (e.t.copy) e.t.copy[i] = round_bf16(po[j]);
        }
      }
    }
    if (lane == 0) {
      e.t.me[b] = static_cast<uint8_t>(em + 127);
      e.t.ve[b] = static_cast<uint8_t>(ev + 127);
    }
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
#pragma unroll 2
    for (uint32_t at = lo + threadIdx.x * 4; at + 4 <= hi; at += kAdamThreads * 4) {
      const uint32_t mc = __ldg(reinterpret_cast<const uint32_t*>(e.t.m + at));
      const uint32_t vc = __ldg(reinterpret_cast<const uint32_t*>(e.t.v + at));
      const float fm = decode_factor(__ldg(e.t.me + at / kBlock), kTopM);
      const float fv = decode_factor(__ldg(e.t.ve + at / kBlock), kTopV);
      float mo[4], vo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        mo[j] = decode<true>((mc >> (8 * j)) & 255u, fm);
        vo[j] = decode<false>((vc >> (8 * j)) & 255u, fv);
      }
      Vec<T, 4> ms, vs;
      ms.round(mo);
      vs.round(vo);
      ms.store(m + at);
      vs.store(v + at);
    }
    i = hi & ~3u;
  }
#pragma unroll 4
  for (uint32_t at = i + threadIdx.x; at < hi; at += kAdamThreads) {
    store_rounded(m + at, decode<true>(__ldg(e.t.m + at), decode_factor(__ldg(e.t.me + at / kBlock), kTopM)));
    store_rounded(v + at, decode<false>(__ldg(e.t.v + at), decode_factor(__ldg(e.t.ve + at / kBlock), kTopV)));
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
    return on(x.m, 4) && on(x.v, 4) && on(x.m_out, sizeof(T) * 4) && on(x.v_out, sizeof(T) * 4);
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
