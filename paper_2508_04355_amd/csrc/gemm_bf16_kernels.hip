// bf16 x bf16 -> fp32 data block of the encoded product (Section III, C = A B), the kernel
// that holds nearly all flops of the path.
//
// Workgroup: 256 x 256 tile of C, 4 wavefronts (2 x 2), each owning a 128 x 128 sub-tile as
// 8 x 8 MFMA 16x16x32 accumulators (256 fp32 registers per lane).  k advances in tiles of 32.
// (Both bf16 MFMA shapes deliver 1024 flop per cycle and SIMD, but the chip is power-limited
// under this load and sustains a 15 % higher clock on 16x16x32 than on 32x32x16.)
// Operand tiles travel HBM -> LDS directly (buffer loads with the LDS bit set: no registers in
// between, out-of-range rows read as zero) and several k-tiles ahead of the one the MFMA units
// are consuming, which is what hides the memory latency with one workgroup per compute unit.
// Every request asks L2 for whole 128-byte lines: the L2 request rate, not its bandwidth, is
// what 32 compute units per XCD saturate first.
//
// LDS (64 KiB per operand), laid out so that neither the DMA writes (64 consecutive 16-byte
// slots per wavefront instruction) nor the fragment reads hit a bank twice:
// (the LDS serves 256 bytes per cycle from 64 banks: 16 lanes of a 16-byte read, 32 lanes of
// an 8-byte read):
//   operand contiguous along k in memory:  two slots, each a PAIR of k-tiles: tile[row][64 k],
//     128 bytes per row (one full line per row and request), the eight 16-byte chunks of a row
//     XOR-swizzled with (row >> 1) & 7; fragments (16 rows x 32 k) by ds_read_b128.
//   operand contiguous along m (or n):     four slots of one k-tile: tile[32 k][256 m], 512
//     bytes per k-row, the eight 64-byte chunks of a row XOR-swizzled with k & 3 and the two
//     32-byte halves of a chunk swapped when k & 8; fragments by the transposing LDS read (two
//     ds_read_b64_tr_b16 per fragment: 16 lanes fetch 4 k-rows x 16 columns and each lane
//     receives the 4 k-values of its own column).
//
// Epilogue, from the accumulators (C itself never passes through LDS): one branch-free pass that
// stores C through a range-checked raw buffer (rows and columns outside C are dropped by the
// hardware) and forms, per 128 x 128 sub-tile, the column sums (in-lane) and row sums (through
// a small LDS transpose) for Section V's syndromes.  Test faults, when a list is given, are
// planted into the accumulators first.
//
// Every tile walks k cyclically from its own start (a few k-tiles apart for neighbouring
// tiles), so that the compute units sharing an operand panel do not ask L2 for the same line
// in the same cycle: the first one misses, the others hit.
#include <mutex>
#include "gecc_internal.h"
#include "tile256_device.h"

namespace gecc {
namespace {

constexpr int EPI_SMEM_BYTES = 4 * 2 * 128 * 17 * 4;  // 68 KiB: row-sum transpose of the epilogue

// The k-split tail (see launch_one): a tile of the last, at most half filled round is computed
// by two workgroups, one per half of k, which add their halves into C and into the partial sums.
// Both are zeroed first, by the first workgroups of the launch that computes the full rounds
// (one tail tile each, before their own tile: that launch ends before the split one starts).
__device__ __forceinline__ void zero_tail_tile(const GemmArgs& a, int tile) {
  const int ntm = (a.n + BM - 1) / BM, ntn = (a.m + BN - 1) / BN;
  int tm, tn;
  tile_of(tile, ntm, ntn, a.map_sr, a.map_sc, tm, tn);
  const int r0 = tm * BM, c0 = tn * BN;
  const int rows = min(BM, a.n - r0), cols = min(BN, a.m - c0);
  for (int o = threadIdx.x; o < rows * BN; o += 256) {
    const int r = o / BN, c = o % BN;
    if (c < cols) a.C[(int64_t)(r0 + r) * a.ldc + c0 + c] = 0.f;
  }
  if (a.rowpart) {
    for (int o = threadIdx.x; o < 2 * BM; o += 256) {          // two 128-column slabs x 256 rows
      const int tn128 = 2 * tn + o / BM, row = r0 + o % BM;
      if (row < a.n && tn128 * 128 < a.m) {
        float2* rp = reinterpret_cast<float2*>(a.rowpart + ((int64_t)tn128 * a.rp_ld + row) * 2);
        *rp = make_float2(0.f, 0.f);
      }
    }
    for (int o = threadIdx.x; o < 2 * BN; o += 256) {
      const int tm128 = 2 * tm + o / BN, col = c0 + o % BN;
      if (col < a.m && tm128 * 128 < a.n) {
        float2* cp = reinterpret_cast<float2*>(a.colpart + ((int64_t)tm128 * a.cp_ld + col) * 2);
        *cp = make_float2(0.f, 0.f);
      }
    }
  }
}

template <bool KCA, bool KCB, bool EPI, bool SP>
__global__ __launch_bounds__(THREADS, 1) void gemm_bf16_256(GemmArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wr = wave >> 1, wc = wave & 1;
  const int l16 = lane & 15, lg = lane >> 4;
  const int b = blockIdx.y;
  if (!SP && a.split_first >= 0) {
    const int ntiles_all = ((a.n + BM - 1) / BM) * ((a.m + BN - 1) / BN);
    if (a.split_first + (int)blockIdx.x < ntiles_all) zero_tail_tile(a, a.split_first + (int)blockIdx.x);
  }

  const int ntm = (a.n + BM - 1) / BM, ntn = (a.m + BN - 1) / BN;
  // SP (the k-split launch, see launch_one): the workgroups share the tiles from split_first on
  // in pairs, khalf = 0 / 1 takes the first / second half of k.  Otherwise: one tile, all of k.
  const int khalf = SP ? (int)(blockIdx.x & 1) : -1;
  int tm, tn;
  tile_of(SP ? a.split_first + (int)(blockIdx.x >> 1) : (int)blockIdx.x, ntm, ntn, a.map_sr, a.map_sc, tm, tn);
  const int tile_r0 = tm * BM, tile_c0 = tn * BN;
  const int KT = SP ? a.k / (2 * BK) : a.k / BK;                 // even (checked by the launcher)
  const int k0 = khalf == 1 ? KT * BK : 0;

  const uint16_t* A = reinterpret_cast<const uint16_t*>(a.A) + (int64_t)b * a.sa + (KCA ? (int64_t)k0 : (int64_t)k0 * a.lda);
  const uint16_t* B = reinterpret_cast<const uint16_t*>(a.B) + (int64_t)b * a.sb + (KCB ? (int64_t)k0 : (int64_t)k0 * a.ldb);
  float* C = a.C + (int64_t)b * a.sc;

  Operand<KCA> oa;
  Operand<KCB> ob;
  oa.init(A, a.lda, tile_r0, a.n, KT * BK, wr * 128);
  ob.init(B, a.ldb, tile_c0, a.m, KT * BK, wc * 128);

  // acc[i][j][v] = C[16 i + 4 g + v][16 j + l16] of the sub-tile (g = lane >> 4, l16 = lane & 15)
  f32x4_t acc[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[i][j][v] = 0.f;

  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  // k order of this tile: cyclic, starting at pair p0 (see SKEW_M, SKEW_N)
  const int p0 = __builtin_amdgcn_readfirstlane(((tm & 7) * SKEW_M + (tn & 3) * SKEW_N) % (KT / 2));
  multiply_256<T256_BF16, KCA, KCB, false>(acc, oa, ob, Scales256{}, smem, KT, p0);

  // ---- epilogue -------------------------------------------------------------------------------
  const int R0 = tile_r0 + wr * 128, C0 = tile_c0 + wc * 128;   // origin of this wavefront's sub-tile
  // Test faults (none in production calls: then this is one scalar compare).
  if (khalf <= 0) {     // (of a split tile: planted into the first half)
    for (int f = 0; f < a.n_faults; ++f) {
      const gecc_fault ft = a.faults[f];
      if (ft.batch != b + a.fault_bias || ft.row < R0 || ft.row >= R0 + 128 || ft.col < C0 || ft.col >= C0 + 128) continue;
      const int dr = ft.row - R0, dc = ft.col - C0;
      const int fi = dr >> 4, fv = dr & 3, fj = dc >> 4;
      const bool mine = (((dr >> 2) & 3) == lg) && ((dc & 15) == l16);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (mine && i == fi && j == fj && v == fv) acc[i][j][v] += ft.offset;
    }
  }

  // One pass over the accumulators, no branches.  C goes straight to memory through a raw
  // buffer whose base is the sub-tile origin and whose size ends with the last valid row: rows
  // beyond n fail the hardware range check and are dropped, and a lane whose column is beyond m
  // carries an offset that is out of range by itself.  An accumulator register holds 4 rows x
  // 16 columns (64-byte pieces, which the memory system takes a third slower than whole
  // lines), so the registers of two neighbouring column blocks first trade their odd / even
  // groups of 16 lanes (v_permlane16_swap): each then holds 2 rows x 32 consecutive columns, two
  // full lines per store.  (Stores are marked non-temporal: C is written once and is larger
  // than the memory-side cache, which is better spent on the operands the parity kernels read
  // again.)
  // The accumulators of such rows and columns are exact zeros (their
  // operand rows were read as zeros), so the sums below need no predicates.
  // Column sums build up in 16 registers with the lane-independent part of the row weight (the
  // lane part, 4 g, is added at the end); of every row the lane keeps the sum of its 8
  // columns (one per 16-wide block) and u = x1 + 2 x2 + .. + 7 x7, the block part of the column
  // weight -- both go through LDS, where the 16 lanes of a group are added and the lane part of
  // the weight is applied.
  // (SP: this workgroup has one half of k of a split tile; its partner has the other.  Both add
  // into zeroed memory instead of storing: two terms, so the result does not depend on who is
  // first.)
  {
    const int tm128 = R0 >> 7, tn128 = C0 >> 7;
    const int R0u = tile_r0 + (wave_u >> 1) * 128, C0u = tile_c0 + (wave_u & 1) * 128;   // scalar copies
    const int rows_left = min(a.n - R0u, 128), cols_left = a.m - C0u;
    const __amdgpu_buffer_rsrc_t crsrc = __builtin_amdgcn_make_buffer_rsrc(
        C + (int64_t)R0u * a.ldc + C0u, 0, rows_left > 0 && cols_left > 0 ? rows_left * a.ldc * 4 : 0, 0x00020000);
    auto put = [&](float x, int off) {
      if (SP) __builtin_amdgcn_raw_ptr_buffer_atomic_fadd_f32(x, crsrc, off, 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, x), crsrc, off, 0, 2);
    };
    // after the swap lane (l16, g) of the first register of a pair has row 8 (g >> 1), column
    // 16 (g & 1) + l16 of the 32-wide block (the second register: 4 rows further down)
    int vo[4];   // byte offset of this lane in the sub-tile, per 32-wide block
#pragma unroll
    for (int jp = 0; jp < 4; ++jp) {
      const int col = jp * 32 + (lg & 1) * 16 + l16;
      vo[jp] = col < cols_left ? ((lg >> 1) * 8 * a.ldc + col) * 4 : (int)OOB;
    }
    float cs[8], cw[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) cs[j] = cw[j] = 0.f;
    float2* red2 = reinterpret_cast<float2*>(smem) + wave_u * (128 * 17) + (lg * 4) * 17 + l16;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int ru = i * 16 + v;                        // row inside the sub-tile, without 4 g
        const int rowoff = ru * a.ldc * 4;                // scalar; < 2^31 (ldc < 2^22, checked by the launcher)
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = acc[i][j][v];
#pragma unroll
        for (int jp = 0; jp < 4; ++jp) {
          // (inline: this compiler's builtin for the swap loses its second result; the wait
          // states are the ones a swap needs after a vector instruction wrote its operands)
          float t0 = x[2 * jp], t1 = x[2 * jp + 1];
          asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(t0), "+v"(t1));
          put(t0, vo[jp] + rowoff);
          put(t1, vo[jp] + rowoff + 4 * a.ldc * 4);
        }
        if (EPI) {
          // s = x0 + .. + x7 and u = x1 + 2 x2 + .. + 7 x7 from suffix sums: u = t1 + t2 + .. + t7
          const float t7 = x[7], t6 = x[6] + t7, t5 = x[5] + t6, t4 = x[4] + t5;
          const float t3 = x[3] + t4, t2 = x[2] + t3, t1 = x[1] + t2;
          red2[ru * 17] = make_float2(x[0] + t1, ((t1 + t2) + (t3 + t4)) + ((t5 + t6) + t7));
          const float wr_ = (float)(ru + 1);
#pragma unroll
          for (int j = 0; j < 8; ++j) { cs[j] += x[j]; cw[j] = fmaf(x[j], wr_, cw[j]); }
        }
      }
    }
    if (EPI) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w1 = fmaf((float)(lg * 4), cs[j], cw[j]);
        float s = cs[j] + __shfl_xor(cs[j], 16, 64), w = w1 + __shfl_xor(w1, 16, 64);
        s += __shfl_xor(s, 32, 64);
        w += __shfl_xor(w, 32, 64);
        const int col = C0 + j * 16 + l16;
        if (lg == 0 && col < a.m && R0 < a.n) {
          float* cp = a.colpart + (((int64_t)b * a.ntm + tm128) * a.cp_ld + col) * 2;
          if (SP) { atomicAdd(cp, s); atomicAdd(cp + 1, w); }
          else *reinterpret_cast<float2*>(cp) = make_float2(s, w);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the region is this wavefront's own
      const float2* mine = reinterpret_cast<const float2*>(smem) + wave_u * (128 * 17);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = lane + 64 * h;
        float s = 0.f, w = 0.f, u = 0.f;
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const float2 t = mine[r * 17 + c];
          s += t.x;
          w = fmaf((float)(c + 1), t.x, w);
          u += t.y;
        }
        const int row = R0 + r;
        if (row < a.n && C0 < a.m) {
          float* rp = a.rowpart + (((int64_t)b * a.ntn + tn128) * a.rp_ld + row) * 2;
          if (SP) { atomicAdd(rp, s); atomicAdd(rp + 1, fmaf(16.f, u, w)); }
          else *reinterpret_cast<float2*>(rp) = make_float2(s, fmaf(16.f, u, w));
        }
      }
    if (!SP && blockIdx.x == 0 && a.pg_out) form_pg(a, b, reinterpret_cast<double*>(smem));   // P_g, once per batch item
    }
  }
}

constexpr int MAX_DEVICES = 64;
// compute units of a device, asked once per device
int device_cus(int dev) {
  static std::mutex mu;
  static int cus_of[MAX_DEVICES] = {};
  std::lock_guard<std::mutex> lock(mu);
  if (cus_of[dev] == 0) {
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1) cus = 256;
    cus_of[dev] = cus;
  }
  return cus_of[dev];
}

template <bool KCA, bool KCB, bool EPI>
hipError_t launch_one(const GemmArgs& a0, hipStream_t st) {
  constexpr int lds_bytes = EPI && EPI_SMEM_BYTES > SMEM_BYTES ? EPI_SMEM_BYTES : SMEM_BYTES;
  auto kern = gemm_bf16_256<KCA, KCB, EPI, false>;
  auto kern_split = gemm_bf16_256<KCA, KCB, EPI, true>;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return hipErrorInvalidDevice;
  {
    // the LDS limit of the two kernels of this instantiation and the CU count, once per device,
    // whichever host thread comes first
    static std::mutex mu;
    static bool configured[MAX_DEVICES] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (!configured[dev]) {
      hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                         hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes);
      if (e != hipSuccess) return e;
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern_split),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes);
      if (e != hipSuccess) return e;
      configured[dev] = true;
    }
  }
  GemmArgs a = a0;
  const int ntm = (a.n + BM - 1) / BM, ntn = (a.m + BN - 1) / BN, ntiles = ntm * ntn;
  // Tiles run in rounds of one per compute unit.  When the last round is at most half full, its
  // tiles go to a launch of their own in which two workgroups share a tile, one per half of k,
  // so that the round takes half as long (cfg4-wgrad: 896 tiles on 256 CUs -> the time of 3.5
  // rounds instead of 4).  The halves add into C and the partial sums, zeroed beforehand.
  const int cus = a.cu_hint > 0 ? a.cu_hint : device_cus(dev);
  // rounds as blocks of tiles (see tile_of): 16 x 16 or 32 x 8, whichever fits
  // exactly -- where the panels a round of the default order touches (64 tile rows + 4 tile
  // columns) would not fit the 256 MiB memory-side cache; where they do, the default order is as
  // fast or a little faster
  a.map_sr = a.map_sc = 0;
  const int64_t default_round_bytes = (int64_t)((ntm < 64 ? ntm : 64) + 4) * BM * a.k * 2;
  if (cus == 256 && a.batch == 1 && default_round_bytes > ((int64_t)192 << 20)) {
    if (ntm % 16 == 0 && ntn % 16 == 0) { a.map_sr = 16; a.map_sc = 16; }
    else if (ntm % 32 == 0 && ntn % 8 == 0) { a.map_sr = 32; a.map_sc = 8; }
  }
  const int tail = ntiles % cus;
  a.split_first = -1;
  if (a.batch == 1 && ntiles > cus && tail > 0 && 2 * tail <= cus && a.k % (4 * BK) == 0) {
    a.split_first = ntiles - tail;      // (tail <= ntiles - tail: every tail tile has a workgroup to zero it)
    hipLaunchKernelGGL(kern, dim3(ntiles - tail, 1), dim3(THREADS), lds_bytes, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern_split, dim3(2 * tail, 1), dim3(THREADS), lds_bytes, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(kern, dim3(ntiles, a.batch), dim3(THREADS), lds_bytes, st, a);
  return hipGetLastError();
}

template <bool EPI>
hipError_t launch_layout(const GemmArgs& a, hipStream_t st) {
  const bool kca = a.trans_a == 0, kcb = a.trans_b != 0;
  if (kca && kcb) return launch_one<true, true, EPI>(a, st);
  if (kca && !kcb) return launch_one<true, false, EPI>(a, st);
  if (!kca && kcb) return launch_one<false, true, EPI>(a, st);
  return launch_one<false, false, EPI>(a, st);
}

}  // namespace

// The fast kernel needs 16-byte aligned operand rows, whole 16-byte chunks and whole pairs of
// k-tiles: k % 64 == 0, leading dimensions % 8 == 0, n (m) % 8 == 0 for an operand stored with n (m)
// contiguous, and operand panels that 32-bit byte offsets can address.  Partial sums are
// produced per 128 x 128 sub-tile.  Everything else goes to gemm_tile.
bool gemm_bf16_fast_ok(const GemmArgs& a) {
  if (a.dtype != GECC_BF16 || a.tile_m != 128 || a.tile_n != 128) return false;
  if (a.k % (2 * BK) || a.lda % 8 || a.ldb % 8) return false;
  if (reinterpret_cast<uintptr_t>(a.A) % 16 || reinterpret_cast<uintptr_t>(a.B) % 16) return false;
  if (a.batch > 1 && (a.sa % 8 || a.sb % 8)) return false;
  if (a.trans_a && a.n % 8) return false;
  if (!a.trans_b && a.m % 8) return false;
  // byte offsets inside a tile panel (k-contiguous: 256 rows; otherwise the whole k extent)
  const int64_t span_a = (a.trans_a ? (int64_t)a.k : (int64_t)BM) * a.lda * 2;
  const int64_t span_b = (a.trans_b ? (int64_t)BN : (int64_t)a.k) * a.ldb * 2;
  if (span_a >= 0x7fffffff || span_b >= 0x7fffffff || a.ldc >= (1 << 22)) return false;
  return (int64_t)a.n * a.m >= (int64_t)BM * BN;   // smaller problems: gemm_tile
}

hipError_t launch_gemm_bf16_fast(const GemmArgs& a, hipStream_t st) {
  return a.rowpart ? launch_layout<true>(a, st) : launch_layout<false>(a, st);
}

}  // namespace gecc
