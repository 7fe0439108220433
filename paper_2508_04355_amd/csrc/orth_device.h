// What the kernels of the orthogonalised update share: U from the gradient and the momentum, alignment rules.
#pragma once
#include "ops_internal.h"
#include "ops_device.h"

namespace gecc {
namespace {

template <bool BF16G, bool VEC>
__device__ __forceinline__ void load_g(const OrthPrepArgs& a, int b, int64_t row, int c, bool ok, float (&g)[8]) {
  load8<!BF16G, VEC>(static_cast<const char*>(a.G) + (int64_t)b * a.p.stride_g * (BF16G ? 2 : 4), row * a.p.ld_g + c, c, a.p.cols, ok, g);
}

// U from G and the momentum after its update
__device__ __forceinline__ float update_of(const OrthPrepArgs& a, float g, float m) { return a.p.nesterov ? fmaf(a.p.mu, m, g) : m; }

// rows of the gradient and of the momentum in whole vectors of eight elements
bool vectors_ok(const OrthPrepArgs& a) {
  const int64_t es = a.p.dtype == GECC_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(a.G) % 16 || a.p.ld_g * es % 16 || (a.p.batch > 1 && a.p.stride_g * es % 16)) return false;
  if (!a.M) return true;
  return reinterpret_cast<uintptr_t>(a.M) % 16 == 0 && a.p.ld_m % 4 == 0 && (a.p.batch == 1 || a.p.stride_m % 4 == 0);
}

// rows of the output in vectors of four elements
inline bool orth_vec_out(const OrthPrepArgs& a, const void* out) {
  const int es = a.p.out_dtype == GECC_F32 ? 4 : 2;
  return reinterpret_cast<uintptr_t>(out) % (4 * es) == 0 && a.p.ld_o % 4 == 0 && (a.p.batch == 1 || a.p.stride_o % 4 == 0);
}

}  // namespace
}  // namespace gecc
