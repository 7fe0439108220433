// The elementwise passes of the orthogonalised update (formulas: gecc_ops.h): the momentum with the sum of squares, and
// the normalised matrix X in two halves, transposed where it is tall.  Both are bound by memory: G and M are read twice
// (the second time out of the memory-side cache where they fit it), M and the two halves of X written once.
#include "ops_internal.h"
#include "ops_device.h"

namespace gecc {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;

constexpr int CHUNK = 2048;     // columns of a workgroup's piece of a row: eight a thread

template <bool BF16G, bool VEC>
__device__ __forceinline__ void load_g(const OrthPrepArgs& a, int b, int64_t row, int c, bool ok, float (&g)[8]) {
  load8<!BF16G, VEC>(static_cast<const char*>(a.G) + (int64_t)b * a.p.stride_g * (BF16G ? 2 : 4), row * a.p.ld_g + c, c, a.p.cols, ok, g);
}

// U from G and the momentum after its update
__device__ __forceinline__ float update_of(const OrthPrepArgs& a, float g, float m) { return a.p.nesterov ? fmaf(a.p.mu, m, g) : m; }

// M <- mu M + G; the sum of U^2 of this workgroup's pieces, in fp64 (squares of fp32 neither overflow nor vanish there)
template <bool BF16G, bool VEC>
__global__ __launch_bounds__(256) void orth_norm_kernel(OrthPrepArgs a) {
  __shared__ double red[4];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int64_t per_row = (a.p.cols + CHUNK - 1) / CHUNK, pieces = a.p.rows * per_row;
  float* M = a.M ? a.M + (int64_t)b * a.p.stride_m : nullptr;
  double sum = 0.0;
  for (int64_t q = blockIdx.x; q < pieces; q += gridDim.x) {
    const int64_t row = q / per_row;
    const int c = (int)(q - row * per_row) * CHUNK + tid * 8;
    if (c >= a.p.cols) continue;
    float g[8], m[8];
    load_g<BF16G, VEC>(a, b, row, c, true, g);
    if (M) {
      load8<true, VEC>(M, row * a.p.ld_m + c, c, a.p.cols, true, m);
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = fmaf(a.p.mu, m[i], g[i]);
      float* o = M + row * a.p.ld_m + c;
      if (VEC && c + 8 <= a.p.cols) {
        reinterpret_cast<f32x4_t*>(o)[0] = f32x4_t{m[0], m[1], m[2], m[3]};
        reinterpret_cast<f32x4_t*>(o)[1] = f32x4_t{m[4], m[5], m[6], m[7]};
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (c + i < a.p.cols) o[i] = m[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = update_of(a, g[i], m[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (c + i < a.p.cols) sum = fma((double)g[i], (double)g[i], sum);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((tid & 63) == 0) red[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0) a.parts[(int64_t)b * a.nparts + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// times / (|U| + eps), the same for every workgroup of a batch item
__device__ __forceinline__ float normaliser(const OrthPrepArgs& a, int b, float times, double* red) {
  const int tid = threadIdx.x;
  double s = tid < a.nparts ? a.parts[(int64_t)b * a.nparts + tid] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  s = (red[0] + red[1]) + (red[2] + red[3]);
  return (float)((double)times / (sqrt(s) + (double)a.p.eps));
}

// X = x_scale U / (|U| + eps) as hi + lo, 64 x 64 elements a workgroup
template <bool BF16G, bool VEC, bool TALL>
__global__ __launch_bounds__(256) void orth_start_kernel(OrthPrepArgs a, int col_tiles) {
  __shared__ double red[4];
  __shared__ float tile[TALL ? 64 * 65 : 1];
  const int b = blockIdx.y, tid = threadIdx.x;
  const float f = normaliser(a, b, a.x_scale, red);
  const int64_t r0 = (int64_t)(blockIdx.x / col_tiles) * 64;
  const int c0 = (blockIdx.x % col_tiles) * 64;
  const float* M = a.M ? a.M + (int64_t)b * a.p.stride_m : nullptr;
  const int64_t base = (int64_t)b * a.s * a.lp;
  auto put = [&](int64_t at, const float (&x)[8]) {
    f16x8_t h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[i] = (_Float16)x[i];
      l[i] = (_Float16)(x[i] - (float)h[i]);
    }
    *reinterpret_cast<f16x8_t*>(a.hi + base + at) = h;
    *reinterpret_cast<f16x8_t*>(a.lo + base + at) = l;
  };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = h * 32 + (tid >> 3), c = (tid & 7) * 8;
    const int64_t row = r0 + r;
    float g[8], m[8];
    load_g<BF16G, VEC>(a, b, row, c0 + c, row < a.p.rows, g);
    if (M) {
      load8<true, VEC>(M, row * a.p.ld_m + c0 + c, c0 + c, a.p.cols, row < a.p.rows, m);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = update_of(a, g[i], m[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = c0 + c + i < a.p.cols && row < a.p.rows ? g[i] * f : 0.f;
    if (!TALL) {
      if (row < a.s && c0 + c < a.lp) put(row * a.lp + c0 + c, g);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) tile[r * 65 + c + i] = g[i];
    }
  }
  if (TALL) {
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = h * 32 + (tid >> 3), r = (tid & 7) * 8;
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = tile[(r + i) * 65 + c];
      if (c0 + c < a.s && r0 + r < a.lp) put((int64_t)(c0 + c) * a.lp + r0 + r, x);
    }
  }
}

// no steps: O = scale U / (|U| + eps)
template <bool BF16G>
__global__ __launch_bounds__(256) void orth_store_kernel(OrthPrepArgs a, void* out) {
  __shared__ double red[4];
  const int b = blockIdx.y;
  const float f = normaliser(a, b, a.p.scale, red);
  const int64_t n = (int64_t)a.p.rows * a.p.cols;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < n; q += (int64_t)gridDim.x * 256) {
    const int64_t row = q / a.p.cols, c = q - row * a.p.cols;
    const int64_t at = (int64_t)b * a.p.stride_g + row * a.p.ld_g + c;
    float g = BF16G ? bf16_of(static_cast<const uint16_t*>(a.G)[at]) : static_cast<const float*>(a.G)[at];
    if (a.M) g = update_of(a, g, a.M[(int64_t)b * a.p.stride_m + row * a.p.ld_m + c]);
    const int64_t to = (int64_t)b * a.p.stride_o + row * a.p.ld_o + c;
    if (a.p.out_dtype == GECC_F32) static_cast<float*>(out)[to] = g * f;
    else static_cast<uint16_t*>(out)[to] = to_bf16(g * f);
  }
}

bool vectors_ok(const OrthPrepArgs& a) {
  const int64_t es = a.p.dtype == GECC_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(a.G) % 16 || a.p.ld_g * es % 16 || (a.p.batch > 1 && a.p.stride_g * es % 16)) return false;
  if (!a.M) return true;
  return reinterpret_cast<uintptr_t>(a.M) % 16 == 0 && a.p.ld_m % 4 == 0 && (a.p.batch == 1 || a.p.stride_m % 4 == 0);
}

template <bool BF16G, bool VEC>
hipError_t start(const OrthPrepArgs& a, hipStream_t st) {
  const int64_t row_tiles = (a.p.rows + 63) / 64, col_tiles = (a.p.cols + 63) / 64;
  if (row_tiles * col_tiles > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(row_tiles * col_tiles), a.p.batch);
  if (a.tall) hipLaunchKernelGGL((orth_start_kernel<BF16G, VEC, true>), grid, dim3(256), 0, st, a, (int)col_tiles);
  else hipLaunchKernelGGL((orth_start_kernel<BF16G, VEC, false>), grid, dim3(256), 0, st, a, (int)col_tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_orth_norm(const OrthPrepArgs& a, hipStream_t st) {
  const dim3 grid(a.nparts, a.p.batch), block(256);
  const bool vec = vectors_ok(a);
  if (a.p.dtype == GECC_BF16) {
    if (vec) hipLaunchKernelGGL((orth_norm_kernel<true, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((orth_norm_kernel<true, false>), grid, block, 0, st, a);
  } else {
    if (vec) hipLaunchKernelGGL((orth_norm_kernel<false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((orth_norm_kernel<false, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

hipError_t launch_orth_start(const OrthPrepArgs& a, hipStream_t st) {
  const bool vec = vectors_ok(a);
  if (a.p.dtype == GECC_BF16) return vec ? start<true, true>(a, st) : start<true, false>(a, st);
  return vec ? start<false, true>(a, st) : start<false, false>(a, st);
}

hipError_t launch_orth_store(const OrthPrepArgs& a, void* out, hipStream_t st) {
  const int64_t n = (int64_t)a.p.rows * a.p.cols;
  const dim3 grid((unsigned)(n < 256 * 2048 ? (n + 255) / 256 : 2048), a.p.batch);
  if (a.p.dtype == GECC_BF16) hipLaunchKernelGGL((orth_store_kernel<true>), grid, dim3(256), 0, st, a, out);
  else hipLaunchKernelGGL((orth_store_kernel<false>), grid, dim3(256), 0, st, a, out);
  return hipGetLastError();
}

}  // namespace gecc
