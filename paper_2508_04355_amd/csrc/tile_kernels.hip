// Tiled products on fp16 and on microscaled 4-bit operands, D[i][j] = sum_k A(i, k) B(j, k), for the operators of
// gecc_ops.h: tiles of 64 x 64 or 128 x 128, k shared out over several workgroups where there are few tiles.
//
// Both kinds of operand are 128 bytes of k a row and stage (64 fp16 or 256 four-bit values), and a fragment of either
// kind is 16 bytes a lane (16 rows x 32 fp16 or x 128 four-bit values), so that one kernel serves both: the matrix
// instructions take the same 16 cycles.  Operands travel HBM -> LDS directly, one stage ahead of the one in use.
//
// LDS of a stage, an operand: k-contiguous: [row][128 bytes], the eight 16-byte chunks of a row XOR-swizzled with
// (row >> 1) & 7, so that the 16 rows of a fragment read meet in no bank.  A stored with its rows contiguous (fp16, tiles
// of 128): [k][128 rows], read by the transposing LDS read, the 64-byte chunks XOR-swizzled with k & 3 and the 32-byte
// halves of a chunk swapped when k & 8.  Scales of 4-bit operands: every second stage 16 bytes a row, the four bytes of
// a lane (its block of four consecutive instructions) in one 32-bit read.
//
// A lane ends up with D[4 g .. 4 g + 3][l16] of every 16 x 16 block, so D is stored transposed: four consecutive values.
#include <type_traits>
#include "ops_internal.h"
#include "dma_device.h"
#include "ops_device.h"
#include "lds_limit.h"
#include "tile_epilogue.h"
#include "tile_order.h"

namespace gecc {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(8))) short s16x8_t;
typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

constexpr int THREADS = 256;

// ---- operands --------------------------------------------------------------------------------------------------------
// KC: k-contiguous.  Otherwise (fp16): element (row, k) at P[k * ld + row].
template <bool KC, int T>
struct TileOperand {
  static constexpr int NV = T * 128 / (THREADS * 16);     // DMA instructions of a wavefront per stage
  const uint8_t* base;
  int64_t step;                 // bytes from stage to stage
  int64_t left;                 // bytes from `base` to the end of the operand
  unsigned voff[NV];
  int frag[T / 32];

  // place of 16-byte unit p of k-row `krow` in the LDS row (and the other way round): a transposing read takes 32 bytes of
  // eight rows (k & 3, k & 8) in one cycle, which have to lie in different banks (rows are 256 or 128 bytes long)
  static __device__ __forceinline__ int unit(int krow, int p) {
    if (T == 128) return p ^ ((krow & 3) << 2) ^ (((krow >> 3) & 1) << 1);
    return p ^ (((krow >> 1) & 1) << 1) ^ (((krow >> 3) & 1) << 2);
  }
  __device__ __forceinline__ void init(const uint8_t* P, int64_t ld, int r0, int rows, int cols, int stage0, int sub) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
    if (KC) {
      base = P + (int64_t)r0 * ld + (int64_t)stage0 * 128;
      step = 128;
      left = rows > r0 ? (int64_t)(rows - r0) * ld - (int64_t)stage0 * 128 : 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = (wave * NV + i) * 64 + lane, row = s >> 3, c = (s & 7) ^ ((row >> 1) & 7);
        voff[i] = r0 + row < rows ? (unsigned)(row * ld + c * 16) : OOB;
      }
#pragma unroll
      for (int i = 0; i < T / 32; ++i) {
        const int row = sub + i * 16 + l16;
        frag[i] = row * 128 + ((g ^ ((row >> 1) & 7)) << 4);
      }
    } else {
      base = P + (int64_t)stage0 * 64 * ld + (int64_t)r0 * 2;
      step = 64 * ld;
      left = (int64_t)(rows - stage0 * 64) * ld - (int64_t)r0 * 2;      // (rows: the valid k)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = (wave * NV + i) * 64 + lane, krow = s / (T / 8), u = unit(krow, s % (T / 8));
        voff[i] = r0 + u * 8 < cols ? (unsigned)(krow * ld + u * 16) : OOB;
      }
      const int j = (lane >> 2) & 3, q = lane & 3;
#pragma unroll
      for (int i = 0; i < T / 32; ++i) {
        const int col = sub + i * 16 + 4 * q, krow = 8 * g + j;
        frag[i] = krow * (T * 2) + (unit(krow, col >> 3) << 4) + (col & 7) * 2;
      }
    }
  }
  // stage number t (from the range's first) into the LDS region at `lds`
  __device__ __forceinline__ void issue(unsigned lds, int wave_u, int t) const {
    const int64_t off = (int64_t)t * step, rest = left - off;
    const i32x4_t rsrc = make_rsrc(base + off, rest <= 0 ? 0u : rest > 0x7fffffff ? 0x7fffffffu : (unsigned)rest);
#pragma unroll
    for (int i = 0; i < NV; ++i) dma16(lds + (wave_u * NV + i) * 1024, voff[i], rsrc, 0);
  }
  // the 16 bytes a lane of fragment i (16 rows), instruction ks (0, 1) of the stage
  __device__ __forceinline__ s16x8_t fragment(const char* region, int i, int ks) const {
    if (KC) return *reinterpret_cast<const s16x8_t*>(region + (frag[i] ^ (ks << 6)));
    const char* p = region + frag[i] + ks * 32 * (T * 2);
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(p));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(p + 4 * (T * 2)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

template <int T>
__device__ __forceinline__ void tile_at(const TileArgs& a, int t, int& tm, int& tn) {
  if (a.symmetric) { triangle(t, tm, tn); return; }
  const int ntm = (a.m_rows + T - 1) / T;
  tm = t % ntm;
  tn = t / ntm;
}

// RING: stages of LDS, RING - 1 of them on their way while one is in use
template <int KIND, bool KCA, int T, int RING, int EPI>
__global__ __launch_bounds__(THREADS, 2) void tile_kernel(TileArgs a, bool vec_out) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int F = T / 32;                       // 16-row fragments of a wavefront, an operand
  constexpr int STAGE = T * 128;                  // bytes of a stage, an operand
  constexpr int SCALES = KIND == KIND_MX4 ? T * 16 : 0;
  constexpr int SLOT = 2 * STAGE;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int wr = wave >> 1, wc = wave & 1, l16 = lane & 15, g = lane >> 4;
  const int b = blockIdx.z;
  int tm, tn;
  tile_at<T>(a, blockIdx.x, tm, tn);
  const int r0 = tm * T, c0 = tn * T;
  // this workgroup's stages: a range of whole pairs (a scale tile is two stages long)
  const int pairs = (a.stages + 1) / 2;
  const int first = (int)((int64_t)pairs * blockIdx.y / a.split) * 2;
  const int last = min((int)((int64_t)pairs * (blockIdx.y + 1) / a.split) * 2, a.stages);
  const int count = last - first;

  TileOperand<KCA, T> oa;
  TileOperand<true, T> ob;
  oa.init(a.A + b * a.sa, a.lda, r0, KCA ? a.m_rows : a.k_rows, a.a_cols, first, wr * (T / 2));
  ob.init(a.B + b * a.sb, a.ldb, c0, a.n_rows, 0, first, wc * (T / 2));

  // scales: instruction number `wave` of the 2 T / 64 of a pair (64 rows each); wavefronts beyond them repeat the last
  const uint8_t* sbase = nullptr;
  unsigned svoff = 0, slds = 0;
  int64_t sleft = 0;
  if (KIND == KIND_MX4) {
    const int q = min(wave_u, 2 * T / 64 - 1), per = T / 64;
    const bool is_b = q >= per;
    const int row = (is_b ? q - per : q) * 64 + lane;
    const int64_t units = pairs, row0 = is_b ? c0 : r0, rows16 = ((is_b ? a.n_rows : a.m_rows) + 15) / 16;
    sbase = (is_b ? a.scale_b : a.scale_a) + (row0 / 16 * units + first / 2) * 256;
    sleft = (rows16 - row0 / 16) * units * 256 - (int64_t)(first / 2) * 256;
    svoff = (unsigned)((row >> 4) * units * 256 + (row & 15) * 16);
    if (row0 / 16 + (row >> 4) >= rows16) svoff = OOB;
    slds = (is_b ? SCALES : 0) + (unsigned)(is_b ? q - per : q) * 1024;
  }

  f32x4_t acc[F][F];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  auto issue = [&](int t) {
    const unsigned at = lds0 + (t & (RING - 1)) * SLOT;
    if (KIND == KIND_MX4 && (t & 1) == 0) {
      const int64_t off = (int64_t)(t >> 1) * 256, rest = sleft - off;
      const i32x4_t rsrc = make_rsrc(sbase + off, rest <= 0 ? 0u : rest > 0x7fffffff ? 0x7fffffffu : (unsigned)rest);
      dma16(lds0 + RING * SLOT + ((t >> 1) & (RING / 2 - 1)) * 2 * SCALES + slds, svoff, rsrc, 0);
    }
    oa.issue(at, wave_u, t);
    ob.issue(at + STAGE, wave_u, t);
  };
  int sa[F], sb[F];
#pragma unroll
  for (int i = 0; i < F; ++i) sa[i] = sb[i] = 0;
  auto multiply = [&](int t, auto odd_c) {
    constexpr bool ODD = decltype(odd_c)::value;
    const char* ra = smem + (t & (RING - 1)) * SLOT;
    const char* rb = ra + STAGE;
    if (KIND == KIND_MX4 && !ODD) {
      const char* rs = smem + RING * SLOT + ((t >> 1) & (RING / 2 - 1)) * 2 * SCALES;
#pragma unroll
      for (int i = 0; i < F; ++i) {
        sa[i] = *reinterpret_cast<const int*>(rs + (wr * (T / 2) + i * 16 + l16) * 16 + g * 4);
        sb[i] = *reinterpret_cast<const int*>(rs + SCALES + (wc * (T / 2) + i * 16 + l16) * 16 + g * 4);
      }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      s16x8_t fa[F], fb[F];
#pragma unroll
      for (int i = 0; i < F; ++i) fa[i] = oa.fragment(ra, i, ks);
#pragma unroll
      for (int j = 0; j < F; ++j) fb[j] = ob.fragment(rb, j, ks);
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) {
          if (KIND == KIND_F16) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, fa[i]), __builtin_bit_cast(f16x8_t, fb[j]), acc[i][j], 0, 0, 0);
          } else {
            const i32x4_t xa = __builtin_bit_cast(i32x4_t, fa[i]), xb = __builtin_bit_cast(i32x4_t, fb[j]);
            const i32x8_t va = {xa[0], xa[1], xa[2], xa[3], 0, 0, 0, 0}, vb = {xb[0], xb[1], xb[2], xb[3], 0, 0, 0, 0};
            // (the byte of the scale registers, 2 ODD + ks, is a constant of the instruction)
            if (ks == 0) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, acc[i][j], 4, 4, ODD ? 2 : 0, sa[i], ODD ? 2 : 0, sb[j]);
            else         acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, acc[i][j], 4, 4, ODD ? 3 : 1, sa[i], ODD ? 3 : 1, sb[j]);
          }
        }
    }
  };
  // Stage t has landed when no more instructions are pending than the stages behind it have (a stage's scales go out first)
  constexpr int PER = TileOperand<KCA, T>::NV + TileOperand<true, T>::NV;
  auto step = [&](int t, auto odd_c) {
    const int behind = min(RING - 2, count - 1 - t);
    if (RING > 3 && behind == 2) wait_vm<(RING > 3 ? 2 : 0) * PER>();
    else if (RING > 2 && behind == 1) wait_vm<(RING > 2 ? 1 : 0) * PER>();
    else wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wavefront's reads of stage t - 1 are back
    __builtin_amdgcn_s_barrier();                        // stage t complete for everyone, the slot of stage t - 1 free
    asm volatile("" ::: "memory");
    if (t + RING - 1 < count) issue(t + RING - 1);
    multiply(t, odd_c);
  };
  for (int t = 0; t < min(RING - 1, count); ++t) issue(t);
  for (int t = 0; t < count; t += 2) {
    step(t, std::false_type{});
    if (t + 1 < count) step(t + 1, std::true_type{});
  }

  if (a.split > 1) {
    // [batch][tile][range][fragment pair][lane] in the order of the registers; tile_finish_kernel adds the ranges up
    f32x4_t* p = reinterpret_cast<f32x4_t*>(a.part) + (((int64_t)b * gridDim.x + blockIdx.x) * a.split + blockIdx.y) * (T * T / 4) + wave * (F * F * 64) + lane;
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) p[(i * F + j) * 64] = acc[i][j];
    return;
  }
  __syncthreads();               // the stages are done with: their LDS holds rows of the result now
  static_assert(4 * store_floats<F>() * 4 <= RING * SLOT, "room for the epilogue");
  store_tile<EPI, F, F>(a, b, acc, reinterpret_cast<float*>(smem) + wave * store_floats<F>(), r0 + wr * (T / 2), c0 + wc * (T / 2), r0 + T, c0 + T,
                         a.symmetric && tm != tn, vec_out);
}

// Adds the ranges of a split product up, in their order, and stores the result: a wavefront per fragment pair.
template <int T, int EPI>
__global__ __launch_bounds__(256) void tile_finish_kernel(TileArgs a, bool vec_out, int shared) {
  constexpr int F = T / 32;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int piece = blockIdx.x * 4 + (threadIdx.x >> 6);        // of shared * 4 F F
  const int b = blockIdx.y;
  const int t = piece / (4 * F * F), r = piece % (4 * F * F);   // t: of the `shared` tiles from number a.whole on
  if (t >= shared) return;
  int tm, tn;
  if (T == 256 && !a.symmetric) tile_of(a.whole + t, (a.m_rows + T - 1) / T, (a.n_rows + T - 1) / T, 0, 0, tm, tn);
  else tile_at<T>(a, a.whole + t, tm, tn);
  const int wave = r / (F * F), i = r % (F * F) / F, j = r % F;
  const f32x4_t* p = reinterpret_cast<const f32x4_t*>(a.part) + ((int64_t)b * shared + t) * a.split * (T * T / 4) + r * 64 + lane;
  f32x4_t s = p[0];
  for (int q = 1; q < a.split; ++q) {
    const f32x4_t x = p[q * (T * T / 4)];
#pragma unroll
    for (int v = 0; v < 4; ++v) s[v] += x[v];
  }
  const float x[4] = {s[0], s[1], s[2], s[3]};
  store_elements<EPI, 4>(a, b, tm * T + (wave >> 1) * (T / 2) + i * 16 + 4 * g, tn * T + (wave & 1) * (T / 2) + j * 16 + l16, a.symmetric && tm != tn, x, vec_out);
}

int64_t tiles_of(int64_t m_rows, int64_t n_rows, int T, bool symmetric) {
  const int64_t tm = (m_rows + T - 1) / T, tn = (n_rows + T - 1) / T;
  return symmetric ? tm * (tm + 1) / 2 : tm * tn;
}

template <int T, int EPI>
hipError_t launch_finish(const TileArgs& a, int64_t tiles, hipStream_t st) {
  constexpr int F = T / 32;
  const int64_t shared = tiles - a.whole;
  hipLaunchKernelGGL((tile_finish_kernel<T, EPI>), dim3((unsigned)(shared * F * F), a.batch), dim3(256), 0, st, a, vectors_out(a, 4), (int)shared);
  return hipGetLastError();
}

template <int KIND, bool KCA, int T, int RING, int EPI>
hipError_t launch(const TileArgs& a, hipStream_t st) {
  static_assert(RING == 2 || RING == 4, "the waits of tile_kernel");
  const int64_t tiles = tiles_of(a.m_rows, a.n_rows, T, a.symmetric);
  if (tiles > 0x7fffffff || a.batch > 65535) return hipErrorInvalidValue;
  constexpr int lds = RING * 2 * T * 128 + (KIND == KIND_MX4 ? RING / 2 * 2 * T * 16 : 0);
  auto kern = tile_kernel<KIND, KCA, T, RING, EPI>;
  if (lds > 65536) {
    static LdsLimit limit;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)tiles, a.split, a.batch), dim3(THREADS), lds, st, a, vectors_out(a, 8));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.split == 1) return e;
  return launch_finish<T, EPI>(a, tiles, st);
}

}  // namespace

TilePlan plan_tiles(TileKind kind, TileEpi epi, int64_t m_rows, int64_t n_rows, int stages, int batch, bool symmetric, bool big_ok) {
  TilePlan p;
  p.symmetric = symmetric;
  p.split = 1;
  p.part_bytes = 0;
  const int pairs = (stages + 1) / 2;
  int64_t tiles;
  if (big_ok && tiles_of(m_rows, n_rows, 256, false) * batch >= 256) {
    p.tile = 256;
    const int64_t all = tiles_of(m_rows, n_rows, 256, false), half = tiles_of(m_rows, n_rows, 256, true);
    // one triangle alone only where that saves a round of workgroups, one a compute unit
    if (symmetric && (half * batch + 255) / 256 == (all * batch + 255) / 256 && pairs < 3 * 16) p.symmetric = false;
    tiles = p.symmetric ? half : all;
    p.whole = (int)tiles;
    if (batch == 1) {
      const int64_t tail = tiles % 256;
      if (p.symmetric && tiles < 256 && pairs >= 3 * 16) { p.split = 3; p.whole = 0; }
      else if (tiles > 256 && tail > 0 && tail <= 128 && pairs >= 16) { p.split = 2; p.whole = (int)(tiles - tail); }
    }
  } else {
    p.tile = tiles_of(m_rows, n_rows, 128, symmetric) * batch >= 256 ? 128 : 64;
    tiles = tiles_of(m_rows, n_rows, p.tile, symmetric);
    int64_t s = 512 / (tiles * batch);
    if (s > 16) s = 16;
    if (s > pairs / 8) s = pairs / 8;
    p.split = s < 1 ? 1 : (int)s;
    p.whole = p.split > 1 ? 0 : (int)tiles;
  }
  if (p.split > 1) p.part_bytes = (size_t)(tiles - p.whole) * batch * p.split * p.tile * p.tile * 4;
  (void)kind; (void)epi;
  return p;
}

namespace {
template <int KIND, bool KCA, int EPI>
hipError_t launch_any(const TileArgs& a, const TilePlan& plan, hipStream_t st) {
  if (plan.tile == 256) {
    const hipError_t e = launch_tiles_256((TileKind)KIND, (TileEpi)EPI, a, st);
    const int64_t tiles = tiles_of(a.m_rows, a.n_rows, 256, a.symmetric);
    return e != hipSuccess || a.whole == tiles ? e : launch_finish<256, EPI>(a, tiles, st);
  }
  // (64 KiB of LDS either way, two workgroups a compute unit)
  return plan.tile == 128 ? launch<KIND, KCA, 128, 2, EPI>(a, st) : launch<KIND, KCA, 64, 4, EPI>(a, st);
}
}  // namespace

hipError_t launch_tiles(TileKind kind, TileEpi epi, const TileArgs& a0, const TilePlan& plan, hipStream_t st) {
  TileArgs a = a0;
  a.split = plan.split;
  a.whole = plan.whole;
  a.symmetric = plan.symmetric;
  if (kind == KIND_MX4) return launch_any<KIND_MX4, true, EPI_OUT>(a, plan, st);
  switch (epi) {
    case EPI_GRAM: return launch_any<KIND_F16, true, EPI_GRAM>(a, plan, st);
    case EPI_POLY: return launch_any<KIND_F16, true, EPI_POLY>(a, plan, st);
    case EPI_UPDATE: return launch_any<KIND_F16, false, EPI_UPDATE>(a, plan, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace gecc
