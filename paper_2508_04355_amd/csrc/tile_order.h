// Which tile a workgroup takes.
#pragma once
#include <hip/hip_runtime.h>

namespace gecc {
namespace {

constexpr int GROUP_M = 8;                         // tile rows per L2-sharing group

// ---- tile order: consecutive workgroups land on different XCDs (round robin), so give every
// XCD a contiguous range of the tile sequence; inside it walk GROUP_M tile rows at a time, column
// by column, so that co-resident tiles share A row panels and B column panels.
// Where the tile counts allow it (sr > 0, chosen by the launcher), a whole round of 256 workgroups
// takes a block of sr x sc tiles instead, XCD x an 8 x 4 sub-block of it: sr + sc operand
// panels per round instead of 64 + 4, which keeps a round's panels inside the 256 MiB memory-side
// cache when k is long (cfg4-dgrad: 234 MB instead of 500 MB per round, product +6 %).
__device__ __forceinline__ void tile_of(int pid, int ntm, int ntn, int sr, int sc, int& tm, int& tn) {
  const int ntiles = ntm * ntn;
  if (sr > 0) {
    const int q = pid >> 8, w = pid & 255, x = w & 7, idx = w >> 3;
    const int nsn = ntn / sc, xc = sc >> 2;
    const int sbm = q / nsn, sbn = q - sbm * nsn;
    tm = sbm * sr + (x / xc) * 8 + (idx & 7);
    tn = sbn * sc + (x % xc) * 4 + (idx >> 3);
    return;
  }
  {
    const int per = ntiles / 8, rem = ntiles - per * 8;     // XCD x gets per (+1 if x < rem)
    const int x = pid & 7, idx = pid >> 3;
    pid = x * per + min(x, rem) + idx;
  }
  const int gsz = GROUP_M * ntn;
  const int grp = pid / gsz;
  const int first_m = grp * GROUP_M;
  const int gm = min(GROUP_M, ntm - first_m);
  tm = first_m + (pid - grp * gsz) % gm;
  tn = (pid - grp * gsz) / gm;
}

// the index of a tile in the lower triangle: tm >= tn
__device__ __forceinline__ void triangle(int t, int& tm, int& tn) {
  tm = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
  while (tm * (tm + 1) / 2 > t) --tm;
  while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
  tn = t - tm * (tm + 1) / 2;
}

// Batches of eight items or more: workgroup number `linear` of `groups` an item.  Workgroups go round the eight XCDs; all of an
// item's go to one of them, in whose L2 they share its operands (256 x 512 x 512 in chunks of 64: 2025 -> 1739 us).
__device__ __forceinline__ void batch_place(unsigned groups, unsigned batch, unsigned linear, unsigned& group, unsigned& item) {
  if (linear < groups * (batch & ~7u)) {
    const unsigned xcd = linear & 7, n = linear >> 3;
    item = n / groups * 8 + xcd;
    group = n % groups;
  } else {
    item = linear / groups;
    group = linear % groups;
  }
}

}  // namespace
}  // namespace gecc
