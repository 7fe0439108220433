// The main loop of the products on tiles of 256 x 256 (gfx950): four wavefronts (2 x 2), each 128 x 128 as 8 x 8 matrix
// instructions of 16 x 16, operands through LDS by direct loads several k-tiles ahead.  A k-tile is 64 bytes of k a row,
// one matrix instruction: 32 bf16 or fp16 values, or 128 microscaled 4-bit ones, at the same 16 cycles; LDS layout, loads
// and reads do not know the type.  The reasons for the schedule stand at the bf16 product (gemm_bf16_kernels.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include "dma_device.h"
#include "tile_order.h"

namespace gecc {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(8))) short s16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

constexpr int THREADS = 256;
constexpr int BM = 256, BN = 256, BK = 32;
constexpr int TILE_BYTES = BM * BK * 2;            // 16 KiB: one k-tile of one operand
constexpr int NSTAGE = 4;                          // k-tiles of one operand resident in LDS
constexpr int REGION_BYTES = NSTAGE * TILE_BYTES;  // 64 KiB per operand
constexpr int SMEM_BYTES = 2 * REGION_BYTES;       // 128 KiB
// DMA spread (see the schedule in the kernel): the 8 instructions of a pair go out as early as its
// slot allows (all in the half after the slot is released when there is one k-contiguous operand,
// 5 + 3 over two halves when there are two: a burst of 16 makes the address unit push back); the
// 4 instructions of a single k-tile go into its first half
constexpr int MX = 0;
constexpr int SKEW_M = 1, SKEW_N = 1;              // k start offset (pairs of k-tiles) per tile row / column

// The same in two parts, for the main loop, where an MFMA goes between them (M0 must be written
// at least one instruction before the load that reads it; nothing else in the loop writes M0)
template <unsigned LDS_OFF>
__device__ __forceinline__ void dma16_dest(unsigned lds_base) {
  asm volatile("s_add_u32 m0, %0, %1" :: "s"(lds_base), "n"(LDS_OFF) : "memory", "scc");
}
__device__ __forceinline__ void dma16_load(unsigned voff, i32x4_t rsrc, unsigned soff) {
  asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds" :: "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}

// ---- per-operand addressing ---------------------------------------------------------------
// KC = true : element (r, kk) at P[r * ld + kk]  (k contiguous);  LDS: 2 slots x pair of k-tiles
// KC = false: element (r, kk) at P[kk * ld + r]  (r contiguous);  LDS: 4 slots x one k-tile
template <bool KC>
struct Operand {
  static constexpr int NV = KC ? 8 : 4;   // DMA instructions of this wavefront per pair / per k-tile
  i32x4_t rsrc;
  unsigned voff[NV];    // byte offsets of this lane's 16-byte slots, loop invariant
  unsigned sstep;       // soffset advance per pair (KC) / per k-tile
  int frag[8];          // LDS byte offset of this lane's fragment address for i = 0..7 (16 rows each)

  // P: operand base for this batch item; r0: first row (m- or n-index) of the tile;
  // rlim: number of valid rows; sub: first row of this wavefront's sub-tile inside the tile
  __device__ __forceinline__ void init(const uint16_t* P, int64_t ld, int r0, int rlim, int klim, int sub) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (KC) {
      const int64_t rows_left = rlim - r0;
      const int64_t bytes = rows_left > 0 ? rows_left * ld * 2 : 0;
      rsrc = make_rsrc(P + (int64_t)r0 * ld, (unsigned)(bytes > 0x7fffffff ? 0x7fffffff : bytes));
      sstep = 2 * BK * 2;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = (wave * NV + i) * 64 + lane;          // slot in the pair tile
        const int row = s >> 3, c = (s & 7) ^ ((row >> 1) & 7);   // 8 lanes = one 128-byte line
        voff[i] = (unsigned)(row * ld * 2 + c * 16);
      }
      const int l16 = lane & 15, g = lane >> 4;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = sub + i * 16 + l16;
        // chunk = 4 (k-tile parity) + g: lane group g holds k = 8 g .. 8 g + 7 of the k-tile; the
        // parity toggles bit 6 of the offset
        frag[i] = row * 128 + ((g ^ ((row >> 1) & 7)) << 4);
      }
    } else {
      const int64_t bytes = ((int64_t)klim * ld - r0) * 2;
      rsrc = make_rsrc(P + r0, (unsigned)(bytes > 0x7fffffff ? 0x7fffffff : (bytes > 0 ? bytes : 0)));
      sstep = (unsigned)(BK * ld * 2);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = (wave * NV + i) * 64 + lane;
        const int krow = s >> 5, p = s & 31;
        const int u = ((((p >> 2) ^ (krow & 3)) << 2) | ((p & 3) ^ (((krow >> 3) & 1) << 1)));   // logical 16-byte unit along r
        voff[i] = (r0 + u * 8 < rlim) ? (unsigned)(krow * ld * 2 + u * 16) : OOB;
      }
      // transposing read: in each group of 16 lanes, lane 4 j + q supplies k-row j, columns
      // 4 q..4 q + 3, and lane t receives the 4 k-values of column t; group g reads k-rows 8 g + j
      // (+ 4 for the second read), which makes lane (t, g) hold k = 8 g .. 8 g + 7 of row t
      const int g = lane >> 4, j = (lane >> 2) & 3, q = lane & 3;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int col = sub + i * 16 + 4 * q;                       // first of the 4 columns
        const int krow = 8 * g + j;
        const int u = col >> 3;
        frag[i] = krow * 512 + (((((u >> 2) ^ j) << 2) | ((u & 3) ^ ((g & 1) << 1))) << 4) + (col & 7) * 2;
      }
    }
  }

  // LDS byte offset (inside this operand's region) of the slot that holds k-tile kt
  static __device__ __forceinline__ int slot_of(int kt) {
    return KC ? ((kt >> 1) & 1) * (2 * TILE_BYTES) : (kt & (NSTAGE - 1)) * TILE_BYTES;
  }

  // DMA instruction i (0 .. NV-1) of this wavefront: unit (pair or k-tile) number `src` into the
  // slot that unit number `unit` owns
  __device__ __forceinline__ void issue_one(unsigned lds_region, int wave_u, int unit, int src, int i) const {
    const unsigned slot = KC ? (unit & 1) * (2 * TILE_BYTES) : (unit & (NSTAGE - 1)) * TILE_BYTES;
    dma16(lds_region + slot + (wave_u * NV + i) * 1024, voff[i], rsrc, src * sstep);
  }
  // ... in two parts (PART 0: destination into M0, PART 1: the load)
  // UNIT: the unit's number modulo the slots (a compile-time constant in the main loop)
  template <int PART, int UNIT>
  __device__ __forceinline__ void issue_part(unsigned lds_region, int wave_u, int src, int i) const {
    constexpr unsigned slot = KC ? (UNIT & 1) * (2 * TILE_BYTES) : (UNIT & (NSTAGE - 1)) * TILE_BYTES;
    if (PART == 0) dma16_dest<slot>(lds_region + (wave_u * NV + i) * 1024);
    else if (PART == 1) dma16_load(voff[i], rsrc, src * sstep);
    else dma16(lds_region + slot + (wave_u * NV + i) * 1024, voff[i], rsrc, src * sstep);
  }
  __device__ __forceinline__ void issue_range(unsigned lds_region, int wave_u, int unit, int src, int first, int count) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i >= first && i < first + count) issue_one(lds_region, wave_u, unit, src, i);
  }

  // fragment i (16 rows x the 32 k) of k-tile kt, as two halves of 4 k-values per lane (a
  // transposing read fetches one half; the main loop puts them behind different MFMAs);
  // region = this operand's LDS region
  struct Frag {
    s16x4_t lo, hi;
    __device__ __forceinline__ bf16x8_t get() const {
      return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  // PART 0: all of a k-contiguous operand's fragment (one ds_read_b128), else the first half;
  // PART 1: the second half of the other kind
  // KT4: the k-tile's number modulo 4 (a compile-time constant in the main loop, so that slot
  // and fragment become the immediate offset of the read: the address registers are loop invariant)
  template <int PART, int KT4>
  __device__ __forceinline__ void fragment_part(Frag& f, const char* region, int i) const {
    if (KC) {
      if (PART == 0) {
        // frag[i] = frag[0] + 2048 i, and the parity only toggles bit 6 of frag[0]
        const char* p = region + (frag[0] ^ ((KT4 & 1) << 6)) + (((KT4 >> 1) & 1) * (2 * TILE_BYTES) + i * 2048);
        const s16x8_t v = *reinterpret_cast<const s16x8_t*>(p);
        f.lo = __builtin_shufflevector(v, v, 0, 1, 2, 3);
        f.hi = __builtin_shufflevector(v, v, 4, 5, 6, 7);
      }
    } else {
      const char* p = region + frag[i] + (KT4 & (NSTAGE - 1)) * TILE_BYTES;
      if (PART == 0) f.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(p));
      else           f.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(p + 4 * 512));
    }
  }
  // k-tile 0 (prologue)
  __device__ __forceinline__ void fragment(Frag& f, const char* region, int i) const {
    fragment_part<0, 0>(f, region, i);
    fragment_part<1, 0>(f, region, i);
  }
};

// f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>), in order
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<N, I + 1>(f);
  }
}

// What goes behind each of the 32 MFMAs of a half.  Measured on the chip with one wavefront per
// SIMD: behind a 16-cycle MFMA one other instruction issues for free, a second costs 4 cycles,
// a third 8 more.  So the D DMA instructions of the half (two instructions each: destination
// into M0, then -- behind the next MFMA, which also is the wait state M0 needs -- the load) and
// its R LDS reads are dealt out one per MFMA, DMA instructions evenly over the half, reads from
// MFMA number G0 on and over the first four fifths of it (their data is needed when the half ends).
// With more than 32 of them some MFMAs get two.  S further scalar instructions (the bookkeeping
// of the cyclic k order) go behind MFMAs that have nothing yet, from the end of the half
// backwards, then next to LDS reads (a read and a scalar instruction together still cost nothing).
enum { OP_NONE = 0, OP_READ = 1, OP_DEST = 2, OP_LOAD = 3, OP_DMA = 4 /* both parts, with the wait state */ };
struct HalfPlan {
  signed char kind[32][2], idx[32][2], scalar[32];
};
template <int D, int R, int G0, int S>
constexpr HalfPlan make_half_plan() {
  HalfPlan p{};
  for (int g = 0; g < 32; ++g) p.scalar[g] = -1;
  int sk[80] = {}, si[80] = {}, T = 0;
  int d = 0, r = 0;
  while (d < D || r < R) {   // merge by position: DMA d at (d + 1/2) / D, read r at 4/5 (r + 1/2) / R
    const bool dma = d < D && (r >= R || 5 * (2 * d + 1) * R <= 4 * (2 * r + 1) * D);
    if (dma) { sk[T] = OP_DEST; si[T] = d; ++T; sk[T] = OP_LOAD; si[T] = d; ++T; ++d; }
    else { sk[T] = OP_READ; si[T] = r; ++T; ++r; }
  }
  const int cap = 32 - G0, den = T > cap ? T : cap;
  int fill[32] = {};
  for (int k = 0; k < T; ++k) {
    int g = G0 + k * cap / den;
    while (fill[g] >= 2) ++g;                       // (never past 31: T <= 64 - 2 G0 is asserted by the caller)
    if (fill[g] == 1 && p.kind[g][0] == OP_DEST && sk[k] == OP_LOAD) { p.kind[g][0] = OP_DMA; continue; }
    p.kind[g][fill[g]] = (signed char)sk[k];
    p.idx[g][fill[g]] = (signed char)si[k];
    ++fill[g];
  }
  int left = S;     // scalar instruction number S - left goes ...
  for (int g = 31; g >= 0 && left > 0; --g)
    if (fill[g] == 0) { p.scalar[g] = (signed char)(left - 1); --left; }
  for (int g = 31; g >= 0 && left > 0; --g)
    if (p.scalar[g] < 0 && fill[g] == 1 && p.kind[g][0] == OP_READ) { p.scalar[g] = (signed char)(left - 1); --left; }
  for (int g = 31; g >= 0 && left > 0; --g)
    if (p.scalar[g] < 0) { p.scalar[g] = (signed char)(left - 1); --left; }
  return p;
}
// What the kernel relies on: every read and every scalar instruction once and in order of their
// numbers (the scalar ones depend on each other); every DMA instruction once, its load behind a
// later MFMA than its destination (or both together, with the wait state), and no other
// destination in between (there is one M0)
template <int D, int R, int G0, int S>
constexpr bool half_plan_ok(const HalfPlan& p) {
  int next_read = 0, next_scalar = 0, next_dest = 0, next_load = 0;
  for (int g = 0; g < 32; ++g) {
    for (int sl = 0; sl < 2; ++sl) {
      const int k = p.kind[g][sl], i = p.idx[g][sl];
      if (k == OP_NONE) continue;
      if (g < G0) return false;
      if (k == OP_READ) { if (i != next_read) return false; ++next_read; }
      else if (k == OP_DEST) { if (i != next_dest || next_load != next_dest) return false; ++next_dest; }
      else if (k == OP_LOAD) { if (i != next_load || next_dest != next_load + 1 || (sl != 0 && p.kind[g][0] == OP_DEST)) return false; ++next_load; }
      else if (k == OP_DMA) { if (i != next_dest || next_load != next_dest) return false; ++next_dest; ++next_load; }
      else return false;
    }
    if (p.scalar[g] >= 0) { if (p.scalar[g] != next_scalar) return false; ++next_scalar; }
  }
  return next_read == R && next_dest == D && next_load == D && next_scalar == S;
}
template <int D, int R, int G0, int S>
inline constexpr HalfPlan kHalfPlan = make_half_plan<D, R, G0, S>();

// What the operands hold
enum { T256_BF16 = 0, T256_F16 = 1, T256_MX4 = 2 };

// Scales of 4-bit operands: 16 bytes a row for four k-tiles (the byte of k-tile t is byte t & 3 of the 32-bit word of a
// lane's block), 256 rows of each operand behind the operands' LDS, in two slots.  A wavefront brings 128 rows of one
// operand (two instructions), once in four k-tiles, and reads the 8 + 8 words of its fragments one period ahead.
constexpr int SCALE_REGION = 256 * 16;                 // one operand
constexpr int SCALE_SLOT = 2 * SCALE_REGION;
constexpr int SMEM_MX_BYTES = SMEM_BYTES + 2 * SCALE_SLOT;
struct Scales256 {
  i32x4_t rsrc;
  unsigned voff[2];
  // sa, sb: scale tiles of the operands; r0, c0: first rows; units: scale tiles along k; unit0: first of this range
  __device__ __forceinline__ void init(const uint8_t* sa, const uint8_t* sb, int r0, int c0, int rows_a, int rows_b, int units, int unit0) {
    const int lane = threadIdx.x & 63, wave_u = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_b = wave_u >= 2;
    // (rows beyond the operand read the scales of its last ones: no offset leaves the buffer, whatever is added for k)
    const int tile0 = (is_b ? c0 : r0) / 16, left = ((is_b ? rows_b : rows_a) + 15) / 16 - tile0;     // row tiles from the tile's first on
    const uint8_t* base = (is_b ? sb : sa) + ((int64_t)tile0 * units + unit0) * 256;
    const int64_t bytes = ((int64_t)left * units - unit0) * 256;
    rsrc = make_rsrc(base, (unsigned)(bytes > 0x7fffffff ? 0x7fffffff : bytes));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = (wave_u & 1) * 128 + i * 64 + lane;
      voff[i] = (unsigned)(min(row >> 4, left - 1) * units * 256 + (row & 15) * 16);
    }
  }
};

template <int KIND, int BYTE>
__device__ __forceinline__ void mfma_256(f32x4_t& acc, const bf16x8_t& fa, const bf16x8_t& fb, int sa, int sb) {
  // (inline, with the accumulator tied to the accumulation registers: left to itself the
  // compiler moves hundreds of accumulators between register files in every round of the loop)
  if constexpr (KIND == T256_BF16) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(fa), "v"(fb));
  else if constexpr (KIND == T256_F16) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(fa), "v"(fb));
  else if constexpr (BYTE == 0) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(fa), "v"(fb), "v"(sa), "v"(sb));
  else if constexpr (BYTE == 1) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(fa), "v"(fb), "v"(sa), "v"(sb));
  else if constexpr (BYTE == 2) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(fa), "v"(fb), "v"(sa), "v"(sb));
  else asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(fa), "v"(fb), "v"(sa), "v"(sb));
}

// acc[i][j][v] += the tile's product over KT k-tiles (even), in element (16 i + 4 g + v, 16 j + l16) of the wavefront's
// 128 x 128 (g = lane >> 4, l16 = lane & 15).  p0: the pair of k-tiles to start from (cyclic order); 4-bit operands: even, and
// 0 unless KT is a multiple of 4.  smem is free again when it returns.  ZERO: acc is set, not added to (while the first loads
// are on their way).
template <int KIND, bool KCA, bool KCB, bool ZERO>
__device__ __forceinline__ void multiply_256(f32x4_t (&acc)[8][8], const Operand<KCA>& oa, const Operand<KCB>& ob, const Scales256& sc,
                                             char* smem, int KT, int p0) {
  static_assert(KIND != T256_MX4 || (KCA && KCB), "4-bit operands are k-contiguous");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // LDS byte addresses of the two operand regions (address-space-3 values, not flat addresses)
  const unsigned ldsA = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const unsigned ldsB = ldsA + REGION_BYTES;
  const char* regA = smem;
  const char* regB = smem + REGION_BYTES;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);

  // ---- DMA schedule ---------------------------------------------------------------------------
  // A "unit" is what one LDS slot holds: a pair of k-tiles for a k-contiguous operand (nK of
  // them, 8 instructions per wavefront and unit), one k-tile otherwise (nM of them, 4
  // instructions).  An iteration (one k-tile) has two halves of 16 steps (two MFMAs each) with
  // the workgroup barrier between them; that barrier releases the slot of k-tile kt (and of its pair when kt
  // is odd) and is where k-tile kt+1 must have landed.  Where the loads go is a trade between
  // lead time (a pair's slot is free from the barrier of k-tile 2q+1 on and its data is needed
  // at the barrier of 2q+3; with two k-contiguous operands the wavefronts used to wait there for
  // a sixth of the loop) and bursts (the address unit takes one instruction per 16 cycles):
  //   pair q+2:      PA instructions in the 2nd half of k-tile 2q+1, PB in the 1st half of
  //                  2q+2, PC = 8 - PA - PB in the 2nd half of 2q+2   (needed at barrier 2q+3)
  //   k-tile kt+4:   MX instructions in the 2nd half of kt, the rest in the 1st half of kt+1
  // Inside a half the k-contiguous operands go first.  The memory counter retires in order, so
  // "k-tile kt+1 has landed" becomes "at most W instructions are pending", W = at most what the
  // schedule issues after the last instruction of that k-tile's units (for any PA, PB, PC):
  //   kt even: (PA + PB) nK + 8 nM        kt odd: 4 nM  (8 nM without a k-contiguous operand)
  // Units past the end of k wrap around to the start of the tile's cyclic order (a harmless
  // reload into a free slot that nobody reads), which keeps every iteration identical.
  constexpr int nK = (KCA ? 1 : 0) + (KCB ? 1 : 0), nM = 2 - nK;
  constexpr int PA = nK == 2 ? 5 : 8, PB = 8 - PA, PC = 8 - PA - PB;
  constexpr int W_EVEN = (PA + PB) * nK + 8 * nM, W_ODD = nK > 0 ? 4 * nM : 8 * nM;
  const int NP = KT / 2;
  auto src_pair = [&](int pair) { int x = pair + p0; x -= x >= NP ? NP : 0; x -= x >= NP ? NP : 0; return x; };
  auto src_kt = [&](int t) { int x = t + 2 * p0; x -= x >= KT ? KT : 0; x -= x >= KT ? KT : 0; return x; };

  // Sources (cyclic k order) of what the loop requests next, kept as running scalars: cp = pair
  // kt/2 + 1 and cn = pair kt/2 + 2 of the current even kt, cm0 = k-tile kt + 3, cm1 = kt + 4
  int cp = src_pair(1), cn = src_pair(2), cm0 = src_kt(3), cm1 = src_kt(4);
  // scales: the unit (four k-tiles) whose loads go out next, its LDS slot, and the words of this period and the next
  constexpr bool MX4 = KIND == T256_MX4;
  const int units = (KT + 3) / 4;
  int su = 0;
  unsigned s_lds = 0, s_read = 0;
  int sa_now[8], sb_now[8], sa_next[8], sb_next[8];
  if constexpr (MX4) {
    su = p0 / 2 + 1;
    su = su >= units ? 0 : su;
    s_lds = ldsA + SMEM_BYTES + SCALE_SLOT + (wave_u >> 1) * SCALE_REGION + (wave_u & 1) * 2048;
    s_read = SMEM_BYTES + (lane & 15) * 16 + (lane >> 4) * 4;
  }
  // DMA instructions of half PH (0: 1st of even kt, 1: 2nd of even, 2: 1st of odd, 3: 2nd of odd)
  // that belong behind step number `step` of the half
  // DMA instruction number ORD of half PH of the main loop (PH = 0..3: the halves of k-tiles kt,
  // kt + 1 with kt = 0 mod 4; 4..7: those of kt + 2, kt + 3), PART 0: destination, 1: load, 2: both
  auto dma_op = [&](auto ph_c, auto part_c, auto ord_c) {
    constexpr int PH8 = decltype(ph_c)::value, PH = PH8 & 3, KT0 = (PH8 >> 2) * 2 + (PH >> 1);   // k-tile mod 4
    constexpr int PART = decltype(part_c)::value, ORD = decltype(ord_c)::value;
    constexpr int k_cnt = PH == 3 ? PA : PH == 0 ? PB : PH == 1 ? PC : 0;       // per operand
    constexpr int k_first = PH == 3 ? 0 : PH == 0 ? PA : PA + PB;
    constexpr int m_cnt = (PH & 1) ? MX : 4 - MX;
    constexpr int m_first = (PH & 1) ? 0 : MX;
    constexpr int pair = PH == 3 ? (KT0 + 3) >> 1 : (KT0 + 2) >> 1;   // slot
    constexpr int mt = (PH & 1) ? KT0 + 4 : KT0 + 3;
    static_assert(MX == 0, "the running sources cover the k-tiles requested in first halves only");
    const int spair = PH == 3 ? cn : cp, smt = PH == 2 ? cm1 : cm0;
    if constexpr (MX4 && PH8 == 0 && ORD >= 2 * PB) {
      constexpr int i = ORD - 2 * PB;
      if constexpr (PART == 0) dma16_dest<i * 1024>(s_lds);
      else if constexpr (PART == 1) dma16_load(sc.voff[i], sc.rsrc, su * 256);
      else dma16(s_lds + i * 1024, sc.voff[i], sc.rsrc, su * 256);
      return;
    }
    int r = 0;
#pragma unroll
    for (int x = 0; x < k_cnt; ++x) {
      if (KCA) { if (r == ORD) oa.template issue_part<PART, pair>(ldsA, wave_u, spair, k_first + x); ++r; }
      if (KCB) { if (r == ORD) ob.template issue_part<PART, pair>(ldsB, wave_u, spair, k_first + x); ++r; }
    }
#pragma unroll
    for (int x = 0; x < m_cnt; ++x) {
      if (!KCA) { if (r == ORD) oa.template issue_part<PART, mt>(ldsA, wave_u, smt, m_first + x); ++r; }
      if (!KCB) { if (r == ORD) ob.template issue_part<PART, mt>(ldsB, wave_u, smt, m_first + x); ++r; }
    }
  };

  // prologue, in the order the waits assume: pair 0, k-tile 0 | k-tile 1 | start of pair 1,
  // k-tile 2, start of k-tile 3
  if constexpr (MX4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) dma16(s_lds - SCALE_SLOT + i * 1024, sc.voff[i], sc.rsrc, (p0 / 2) * 256);
  }
  if (KCA) oa.issue_range(ldsA, wave_u, 0, src_pair(0), 0, 8);
  if (KCB) ob.issue_range(ldsB, wave_u, 0, src_pair(0), 0, 8);
  if (!KCA) oa.issue_range(ldsA, wave_u, 0, src_kt(0), 0, 4);
  if (!KCB) ob.issue_range(ldsB, wave_u, 0, src_kt(0), 0, 4);
  if (!KCA) oa.issue_range(ldsA, wave_u, 1, src_kt(1), 0, 4);
  if (!KCB) ob.issue_range(ldsB, wave_u, 1, src_kt(1), 0, 4);
  if (KCA) oa.issue_range(ldsA, wave_u, 1, src_pair(1), 0, PA);
  if (KCB) ob.issue_range(ldsB, wave_u, 1, src_pair(1), 0, PA);
  if (!KCA) oa.issue_range(ldsA, wave_u, 2, src_kt(2), 0, 4);
  if (!KCB) ob.issue_range(ldsB, wave_u, 2, src_kt(2), 0, 4);
  if (!KCA) oa.issue_range(ldsA, wave_u, 3, src_kt(3), 0, MX);
  if (!KCB) ob.issue_range(ldsB, wave_u, 3, src_kt(3), 0, MX);
  if constexpr (ZERO) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  wait_vm<PA * nK + (8 + MX) * nM>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  // Software pipeline.  A k-tile is 8 x 8 MFMA 16x16x32 per wavefront (the 16-row shape runs at
  // a higher sustained clock than 32x32x16 at the same flops per cycle), in two halves of 32:
  // rows 0..63 of the sub-tile (A fragments 0..3), then rows 64..127 (fragments 4..7), each
  // against the 8 B fragments of the k-tile.  A "step" is two MFMAs.  1st half of kt: the reads
  // of A fragments 4..7 of kt behind its first four steps; barrier; 2nd half: the reads of the 8
  // B fragments (into the other of two sets) and of A fragments 0..3 of k-tile kt+1 behind its
  // first twelve.  A step carries at most one fragment read and one DMA instruction, dealt out
  // over its two MFMAs in exactly the order written below (every position is fenced), so each
  // of them has an MFMA in flight as cover.
  typename Operand<KCA>::Frag fal[4], fah[4];     // A low / high rows
  typename Operand<KCB>::Frag fbe[8], fbo[8];     // B of the even / odd k-tile
#pragma unroll
  for (int i = 0; i < 4; ++i) oa.fragment(fal[i], regA, i);
#pragma unroll
  for (int j = 0; j < 8; ++j) ob.fragment(fbe[j], regB, j);
  // word number op of the wavefront's scales in the slot that s_read points at: A's eight, then B's
  auto scale_word = [&](auto op_c) {
    constexpr int op = decltype(op_c)::value, f = op & 7;
    const char* p = smem + s_read + (op < 8 ? (wave >> 1) * 2048 : SCALE_REGION + (wave & 1) * 2048);
    (op < 8 ? sa_next : sb_next)[f] = *reinterpret_cast<const int*>(p + f * 256);
  };
  if constexpr (MX4) {
    static_for<16>(scale_word);
#pragma unroll
    for (int i = 0; i < 8; ++i) { sa_now[i] = sa_next[i]; sb_now[i] = sb_next[i]; }
    s_read += SCALE_SLOT;
  }

  // The sources of the next two k-tiles' requests, one scalar instruction at a time (x + 1
  // modulo N as min(x + 1, x + 1 - N) in unsigned arithmetic); they replace cp, cn, cm0, cm1
  // when the two k-tiles are done
  unsigned nx0 = 0, nx1 = 0, ncn = 0, ncm0 = 0, ncm1 = 0;
  constexpr int N_SCALAR = 9;
  auto scalar_op = [&](auto op_c) {
    constexpr int op = decltype(op_c)::value;
    if constexpr (op == 0) nx0 = (unsigned)cn + 1u;
    else if constexpr (op == 1) nx1 = nx0 - (unsigned)NP;
    else if constexpr (op == 2) ncn = nx0 < nx1 ? nx0 : nx1;
    else if constexpr (op == 3) nx0 = (unsigned)cm1 + 1u;
    else if constexpr (op == 4) nx1 = nx0 - (unsigned)KT;
    else if constexpr (op == 5) ncm0 = nx0 < nx1 ? nx0 : nx1;
    else if constexpr (op == 6) nx0 = ncm0 + 1u;
    else if constexpr (op == 7) nx1 = nx0 - (unsigned)KT;
    else if constexpr (op == 8) ncm1 = nx0 < nx1 ? nx0 : nx1;
  };
  auto half = [&](auto ph_c) {
    constexpr int PH8 = decltype(ph_c)::value, PH = PH8 & 3, KT0 = (PH8 >> 2) * 2 + (PH >> 1);   // k-tile mod 4
    constexpr bool SECOND = PH & 1, ODD = (PH >> 1) & 1;
    constexpr int OA = KCA ? 1 : 2, OB = KCB ? 1 : 2;     // LDS instructions per fragment
    constexpr int D = (PH == 3 ? PA : PH == 0 ? PB : PH == 1 ? PC : 0) * nK + ((PH & 1) ? MX : 4 - MX) * nM + (MX4 && PH8 == 0 ? 2 : 0);
    constexpr int R_FRAG = SECOND ? 8 * OB + 4 * OA : 4 * OA;
    constexpr int R = R_FRAG + (MX4 && PH8 == 5 ? 16 : 0);     // (the next period's scales: they landed by the barrier of k-tile 1)
    constexpr int G0 = SECOND ? 0 : 2;   // (1st half: not behind the first MFMAs, or the wait for the previous half's reads takes them along)
    static_assert(2 * D + R <= 64 - 2 * G0, "two instructions per MFMA at most");
    constexpr int S = PH == 1 ? N_SCALAR : 0;   // the 2nd half of the even k-tile requests nothing: room for the bookkeeping
    static_assert(half_plan_ok<D, R, G0, S>(kHalfPlan<D, R, G0, S>), "instruction plan of the half");
    // LDS instruction number OP of the half: 2nd half: the 8 B fragments, then A fragments 0..3, of
    // the next k-tile (past the last k-tile this reads a slot nobody filled: in range, never
    // used); 1st half: A fragments 4..7 of this k-tile
    auto read_op = [&](auto op_c) {
      constexpr int op = decltype(op_c)::value;
      if constexpr (op >= R_FRAG) {
        scale_word(std::integral_constant<int, op - R_FRAG>{});
      } else if constexpr (SECOND) {
        if constexpr (op < 8 * OB) {
          constexpr int f = op / OB, part = op % OB;
          if (ODD) ob.template fragment_part<part, (KT0 + 1) & 3>(fbe[f], regB, f);
          else     ob.template fragment_part<part, (KT0 + 1) & 3>(fbo[f], regB, f);
        } else {
          constexpr int f = (op - 8 * OB) / OA, part = (op - 8 * OB) % OA;
          oa.template fragment_part<part, (KT0 + 1) & 3>(fal[f], regA, f);
        }
      } else {
        constexpr int f = op / OA, part = op % OA;
        oa.template fragment_part<part, KT0>(fah[f], regA, 4 + f);
      }
    };
    static_for<32>([&](auto g_c) {
      constexpr int g = decltype(g_c)::value, i = g >> 3, j = g & 7;
      const bf16x8_t fb = ODD ? fbo[j].get() : fbe[j].get();
      if constexpr (SECOND) mfma_256<KIND, KT0>(acc[4 + i][j], fah[i].get(), fb, MX4 ? sa_now[4 + i] : 0, MX4 ? sb_now[j] : 0);
      else                  mfma_256<KIND, KT0>(acc[i][j], fal[i].get(), fb, MX4 ? sa_now[i] : 0, MX4 ? sb_now[j] : 0);
      __builtin_amdgcn_sched_barrier(0);
      static_for<2>([&](auto s_c) {
        constexpr int sl = decltype(s_c)::value;
        constexpr int kind = kHalfPlan<D, R, G0, S>.kind[g][sl], idx = kHalfPlan<D, R, G0, S>.idx[g][sl];
        if constexpr (kind == OP_READ) read_op(std::integral_constant<int, idx>{});
        else if constexpr (kind == OP_DEST) dma_op(ph_c, std::integral_constant<int, 0>{}, std::integral_constant<int, idx>{});
        else if constexpr (kind == OP_LOAD) dma_op(ph_c, std::integral_constant<int, 1>{}, std::integral_constant<int, idx>{});
        else if constexpr (kind == OP_DMA)  dma_op(ph_c, std::integral_constant<int, 2>{}, std::integral_constant<int, idx>{});
      });
      if constexpr (kHalfPlan<D, R, G0, S>.scalar[g] >= 0) scalar_op(std::integral_constant<int, kHalfPlan<D, R, G0, S>.scalar[g]>{});
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto barrier = [&](auto w_c) {
    wait_vm<decltype(w_c)::value>();                     // k-tile kt+1 of this wavefront's loads
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // own reads of k-tile kt are back
    __builtin_amdgcn_s_barrier();        // k-tile kt+1 complete for everyone; k-tile kt released
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // two k-tiles, the first of them number 2 Q modulo 4
  auto two_ktiles = [&](auto q_c) {
    constexpr int Q = decltype(q_c)::value;
    half(std::integral_constant<int, 4 * Q + 0>{});
    barrier(std::integral_constant<int, W_EVEN>{});
    half(std::integral_constant<int, 4 * Q + 1>{});
    half(std::integral_constant<int, 4 * Q + 2>{});
    barrier(std::integral_constant<int, W_ODD>{});
    half(std::integral_constant<int, 4 * Q + 3>{});
    cp = cn;
    cn = (int)ncn;
    cm0 = (int)ncm0;
    cm1 = (int)ncm1;
  };
  // four k-tiles per round of the loop, so that every LDS slot is a compile-time constant (KT is even)
  for (int kt = 0; kt + 4 <= KT; kt += 4) {
    two_ktiles(std::integral_constant<int, 0>{});
    two_ktiles(std::integral_constant<int, 1>{});
    if constexpr (MX4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) { sa_now[i] = sa_next[i]; sb_now[i] = sb_next[i]; }
      su = su + 1 >= units ? 0 : su + 1;
      // the slots of the next loads and reads: the others
      s_lds = 2 * (ldsA + SMEM_BYTES + (wave_u >> 1) * SCALE_REGION + (wave_u & 1) * 2048) + SCALE_SLOT - s_lds;
      s_read = 2 * (SMEM_BYTES + (lane & 15) * 16 + (lane >> 4) * 4) + SCALE_SLOT - s_read;
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 7" ::: "memory");
    }
  }
  if (KT & 2) two_ktiles(std::integral_constant<int, 0>{});
  // (the wait states between the last MFMA and the first read of its result: the compiler does
  // not see the instruction inside the assembly statement)
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();            // nobody's clamped reloads still land in LDS

}

}  // namespace
}  // namespace gecc
