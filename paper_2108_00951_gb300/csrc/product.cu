// product.cu — host side of the tensor-core products: tensor maps and the
// choice of tile width and K parts.
#include <cmath>

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

// The time of a launch is its longest CTA's (or pair's): whole tiles, each the
// longer of its 128-deep steps (4 cycles per column on the tensor cores, or the
// cycles that a CTA's share of A and B takes from L2 at 64 bytes a cycle) and
// its epilogue, which runs under the next tile's products; and for K parts the
// join, or (not joined here) writing and reading their sums.
void plan_product(ProductShape& p, const ProductWant& w) {
  const uint32_t rows = w.pair ? 2 * kTileM : kTileM;
  p.m = w.m;
  p.n = w.n;
  p.k = w.k;
  p.batch = w.batch;
  p.lower = w.lower ? 1u : 0u;
  p.terms = w.terms;
  p.join = w.join ? 1u : 0u;
  p.tiles_m = (w.m + rows - 1) / rows;
  p.group_m = p.tiles_m ? p.tiles_m : 1;
  const double units = w.pair ? w.sms / 2 : w.sms;
  const uint32_t kts = (w.k + kTileK - 1) / kTileK * w.terms;
  double best = 0.0;
  p.bn = 0;
  const uint32_t widths[] = {256, 192, 128, 64};
  for (uint32_t bn : widths) {
    if (w.lower ? bn != rows : bn > 64 && bn >= 2 * w.n) continue;
    const double tiles = (w.lower ? p.tiles_m * (p.tiles_m + 1.0) / 2.0
                                  : p.tiles_m * static_cast<double>((w.n + bn - 1) / bn)) * w.batch;
    const double mma = 4.0 * bn, load = 4.0 * (kTileM + (w.pair ? bn / 2 : bn));
    const double step = mma > load ? mma : load;
    for (uint32_t s : {1u, 2u, 3u, 4u, 6u, 8u, 12u, 16u, 24u, 32u}) {
      if (s > 1 && (s > w.max_splits || s > kts)) break;
      if (s > 1 && tiles > 2 * units) break;  // nothing to gain
      const double waves = ceil(tiles * s / units);
      const double deep = static_cast<double>((kts + s - 1) / s);
      // an epilogue runs under the next tile's products
      const double products = deep * step, epilogue = w.epilogue * bn;
      const double t = waves * (products > epilogue ? products : epilogue) + 600.0 * waves +
                       (products > epilogue ? epilogue : products) +
                       (s == 1 ? 0.0 : w.join ? 16.0 * bn + 5000.0
                                              : s * (8.0 * w.m) * w.n / (20.0 * w.sms) + 4000.0);
      if (p.bn == 0 || t < best * 0.999) {
        best = t;
        p.bn = bn;
        p.splits = s;
      }
    }
  }
  p.tiles_n = (w.n + p.bn - 1) / p.bn;
  p.tiles = w.lower ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
}

}  // namespace efs
