// product.cu — host side of the tensor-core products: tensor maps and the
// choice of tile width and K parts.
#include "product.cuh"

namespace efs {

namespace {
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                              const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}
}  // namespace

bool make_map(CUtensorMap* map, const void* base, bool bf16, uint64_t cols, uint64_t rows,
              uint64_t ld, uint64_t batch, uint64_t batch_ld, uint32_t box_rows) {
  const EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cols, rows, batch};
  const cuuint64_t strides[2] = {ld * 2, batch_ld * 2};
  const cuuint32_t box[3] = {64, box_rows, 1};
  const cuuint32_t step[3] = {1, 1, 1};
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
            const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The time of a launch is its longest CTA's: whole tiles per CTA, each of its
// 64-deep steps (2 cycles per column on the tensor cores, or the cycles that
// filling shared memory takes for narrow tiles) plus a start that does not
// overlap, and for K parts the join by one CTA (8 cycles per column and part).
void plan_product(ProductShape& p, uint32_t m, uint32_t n, uint32_t k, uint32_t batch,
                  bool lower, uint32_t sms, uint32_t max_splits) {
  p.m = m;
  p.n = n;
  p.k = k;
  p.batch = batch;
  p.lower = lower ? 1u : 0u;
  p.tiles_m = (m + kTileM - 1) / kTileM;
  p.group_m = p.tiles_m ? p.tiles_m : 1;
  const uint64_t kts = (k + kTileK - 1) / kTileK;
  double best = 0.0;
  uint32_t best_bn = 0, best_splits = 1;
  const uint32_t widths[] = {256, 192, 128, 64};
  for (uint32_t bn : widths) {
    if (lower && bn % kTileM) continue;  // rows of tiles pair up to a tile's width
    if (bn > (lower ? 128u : 64u) && bn >= 2 * n) continue;
    const uint64_t tiles_n = (n + bn - 1) / bn, q = bn / kTileM ? bn / kTileM : 1;
    const uint64_t groups = (p.tiles_m + q - 1) / q;
    const uint64_t tiles = (lower ? q * groups * (groups + 1) / 2 : p.tiles_m * tiles_n) * batch;
    const double step = bn * 2.0 > (kTileM + bn) * 1.5 ? bn * 2.0 : (kTileM + bn) * 1.5;
    for (uint32_t s = 1; s <= max_splits && s <= (kts ? kts : 1); ++s) {
      if (s > 1 && tiles > 4 * sms) break;  // nothing to gain (and scratch tiles stay few)
      const double waves = static_cast<double>((tiles * s + sms - 1) / sms);
      const double deep = static_cast<double>((kts + s - 1) / s);
      const double t = waves * (deep * step + 1500.0 + 4.0 * bn) + (s > 1 ? (s + 1) * 8.0 * bn + 2000.0 : 0.0);
      if (best_bn == 0 || t < best * 0.999) {
        best = t;
        best_bn = bn;
        best_splits = s;
      }
    }
  }
  p.bn = best_bn;
  p.splits = best_splits;
  p.tiles_n = (n + p.bn - 1) / p.bn;
  if (lower) {
    const uint32_t q = p.bn / kTileM, groups = (p.tiles_m + q - 1) / q;
    p.tiles = q * groups * (groups + 1) / 2;
  } else {
    p.tiles = p.tiles_m * p.tiles_n;
  }
}

}  // namespace efs
