// The attention kernels' work slots: tile and block sizes, the block order without
// a plan, and halves of slots.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace scope {

constexpr int kBN = 64;          // keys per tile
constexpr int kNW = 8;           // waves per block
constexpr int kQB = 1;           // 32-query column blocks per wave
constexpr int kBM = 32 * kQB * kNW;

// Work slots run in list order: heads one after the other and, within a
// head, by estimated cost, largest first, with a cluster's row chunks
// adjacent.  All XCDs work on the same head at a time, so one head's K/V
// (60 MB at 118800 x 128 bf16) is what the 256 MB memory-side cache has to
// hold.  (Where several heads' fit there, attn_plan_kernel gives the order.)
//
// Block b runs on XCD b mod 8.  Runs of kRun consecutive work slots (the
// chunks of one cluster, which gather the same K/V rows) go to one XCD so
// that they share its L2; windows of 8 * kRun slots still follow the list
// order.  A partial last window keeps the identity map.
constexpr int kXcds = 8, kRun = 4;
__device__ __forceinline__ int xcd_item(int b, int total) {
  constexpr int W = kXcds * kRun;
  const int w0 = b / W * W;
  if (w0 + W > total) return b;
  const int r = b - w0;
  return w0 + (r % kXcds) * kRun + r / kXcds;
}

// Half a slot: the queries of its waves 0 .. kNW/2 - 1 (half 1) or of the others
// (half 2).  A query's result depends neither on its wave nor on its block, so
// halves give the slot's results bit for bit.
__device__ __forceinline__ void take_half(int4 *a, int4 *b, int half) {
  const int first = half == 2 ? kNW / 2 : 0;
  // the rows of an entry, whose first wave is w0, that the half's waves hold
  auto cut = [&](int4 *e, int w0) {
    const int from = min(max(32 * (first - w0), 0), e->z);
    const int to = min(max(32 * (first + kNW / 2 - w0), 0), e->z);
    e->y += from;
    e->z = to - from;
  };
  const int wa = (a->z + 31) >> 5;
  cut(a, 0);
  cut(b, wa);
  if (a->z <= 0) {
    *a = *b;
    b->z = 0;
  }
}

}  // namespace scope
