// Loads from HBM straight into LDS (gfx950): no registers in between, rows beyond a buffer's end read as zero.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gecc {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4_t;
constexpr unsigned OOB = 0x80000000u;              // offset beyond any num_records: reads zero

// one LDS-DMA instruction: 64 lanes x 16 bytes from buffer `rsrc` at (voff + soff) into the
// 1 KiB of LDS starting at lds_addr (lane L lands at lds_addr + 16 L).  Invisible to the
// compiler's memory-counter bookkeeping on purpose: the waits are placed by hand.
__device__ __forceinline__ void dma16(unsigned lds_addr, unsigned voff, i32x4_t rsrc, unsigned soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :: "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}

__device__ __forceinline__ i32x4_t make_rsrc(const void* base, unsigned bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  i32x4_t r;
  r[0] = (int)(p & 0xffffffffu);
  r[1] = (int)((p >> 32) & 0xffffu);       // stride 0: raw buffer, offsets in bytes
  r[2] = (int)bytes;
  r[3] = 0x00020000;
  return r;
}

// s_waitcnt vmcnt(N), N a compile-time constant below 64
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}

}  // namespace
}  // namespace gecc
