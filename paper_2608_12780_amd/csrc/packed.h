// Device side shared by the kernels of attention over packed sequences.
#pragma once

#include "attention_slots.h"
#include "common.h"
#include "kernels.h"

namespace scope {

constexpr float kPackLn2 = 0.6931471805599453f;

// Items as the XCDs take them.  Block b runs on XCD b mod 8 whatever the loads there,
// so each is given an equal share by construction: a key head's list, which falls in
// cost, is dealt out in eight classes (rank mod 8), and an XCD runs kv_heads
// neighbouring (head, class) pairs, heads one after the other: its L2 then holds the
// rows of one or two key heads.  False: nothing for this block.
__device__ __forceinline__ bool pack_place(int block, int kv_heads, int count, int *head, int *rank) {
  const int x = block % kXcds, per = (count + kXcds - 1) / kXcds;
  int j = block / kXcds;
  if (per == 0 || j >= kv_heads * per) return false;
  const int u0 = x * kv_heads, u1 = u0 + kv_heads;
  const int h0 = u0 / kXcds, c0 = u0 % kXcds, n0 = min(kXcds - c0, kv_heads);
  int i, c;
  if (j < n0 * per) {
    *head = h0;
    i = j / n0;
    c = c0 + j % n0;
  } else {
    j -= n0 * per;
    const int skip = j / (kXcds * per);
    *head = h0 + 1 + skip;
    j -= skip * kXcds * per;
    const int n = min(kXcds, u1 - kXcds * *head);
    i = j / n;
    c = j % n;
  }
  *rank = kXcds * i + c;
  return *rank < count;
}

// Keys that row `row` of a sequence's (query, head of the group) rows sees.
__device__ __forceinline__ int keys_seen(int row, int group, int lq, int lk, int causal) {
  return causal ? min(max(row / group + lk - lq + 1, 0), lk) : lk;
}

// Where row `row` of a key head lies, in bytes from the sequence's first query of the
// group's first head.
__device__ __forceinline__ uint32_t row_offset(int row, int group, const PackRows &r) {
  const int query = row / group;
  return static_cast<uint32_t>(query) * static_cast<uint32_t>(r.row) +
         static_cast<uint32_t>(row - query * group) * static_cast<uint32_t>(r.head);
}
// Base of a sequence's query rows of a key head's group, or of its key rows.
__device__ __forceinline__ char *rows_base(const PackRows &r, int first, int head) {
  return r.base + first * r.row + head * r.head;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t pack_resource(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), static_cast<short>(0), static_cast<int>(bytes), 0x00020000);
}
// Bytes from a base to the end of its last row.
__device__ __forceinline__ uint32_t span(const PackRows &r, int rows, int heads, int row_bytes) {
  return static_cast<uint32_t>((rows - 1) * r.row + (heads - 1) * r.head + row_bytes);
}

// Sequence s's place, from offsets that may be bad: each is the largest of those so
// far within [0, rows].
struct PackSequence {
  int q0, lq, k0, lk;
};

}  // namespace scope
