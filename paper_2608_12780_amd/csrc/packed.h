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
// rows of one or two key heads.  The parts of an item are neighbours in the list, so
// that it falls in cost with them too.  False: nothing for this block.
__device__ __forceinline__ bool pack_place(int block, int kv_heads, int items, int parts, int *head, int *rank, int *part) {
  const int count = items * parts, x = block % kXcds, per = (count + kXcds - 1) / kXcds;
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
  const int at = kXcds * i + c;
  *rank = at / parts;
  *part = at - *rank * parts;
  return at < count;
}

// Keys that row `row` of a sequence's (query, head of the group) rows sees.
__device__ __forceinline__ int keys_seen(int row, int group, int lq, int lk, int causal) {
  return causal ? min(max(row / group + lk - lq + 1, 0), lk) : lk;
}

// Where row `row` of a key head lies, in bytes from row 0 of the group's first head: rows
// of one tile, so that 32 bits hold it.
__device__ __forceinline__ uint32_t row_offset(int row, int group, const PackRows &r) {
  const int query = row / group;
  return static_cast<uint32_t>(query) * static_cast<uint32_t>(r.row) +
         static_cast<uint32_t>(row - query * group) * static_cast<uint32_t>(r.head);
}
// Base of a sequence's query rows of a key head's group, or of its key rows.
__device__ __forceinline__ char *rows_base(const PackRows &r, int first, int head) {
  return r.base + first * r.row + head * r.head;
}

// A value that is the same in all lanes, for a scalar register: a quotient lies in a
// vector register, and one in the address of a load through a buffer resource makes
// that load a loop.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t pack_resource(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), static_cast<short>(0), scalar(static_cast<int>(bytes)), 0x00020000);
}
// Bytes from a base to the end of its last row.
__device__ __forceinline__ uint32_t span(const PackRows &r, int rows, int heads, int row_bytes) {
  return static_cast<uint32_t>((rows - 1) * r.row + (heads - 1) * r.head + row_bytes);
}

constexpr int kStatusBadOffsets = 16;
constexpr int kCostKeys = 64, kCostRows = 32;  // units of an item's cost, by rows and by keys

// Sum of the lanes' values up to each lane's (the last lane: all of them).
__device__ __forceinline__ int lane_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // lanes 1, 2, 4, 8 to
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // the left, in rows of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // a row's last to the next
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // and lane 31 to the upper half
  return v;
}
__device__ __forceinline__ int lane_sum(int v) { return __builtin_amdgcn_readlane(lane_scan(v), 63); }

// The sequence of each lane, of at most 64: (first query row, queries, first key row,
// keys), of bad offsets too: each is the largest of those so far within [0, rows].
__device__ __forceinline__ int4 lane_sequence(const PackArgs &a, int lane, bool *bad) {
  const int S = a.sequences, s = min(lane, S), n = min(lane + 1, S);
  int q0 = a.offsets_q[s], q1 = a.offsets_q[n], k0 = a.offsets_k[s], k1 = a.offsets_k[n];
  const int length = a.lengths_k ? a.lengths_k[min(lane, S - 1)] : 0;
  const bool wrong = q0 < 0 || q1 < q0 || q1 > a.rows_q || k0 < 0 || k1 < k0 || k1 > a.rows_k;
  const bool any = __ballot(wrong) != 0;
  if (any) {
    auto up_to = [&](int &first, int &last, int rows) {
      const int own = min(max(first, 0), rows);
      int v = max(own, min(max(last, 0), rows));
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(v, o);
        if (lane >= o) v = max(v, x);
      }
      const int before = __shfl_up(v, 1);
      first = lane ? before : own;
      last = v;
    };
    up_to(q0, q1, a.rows_q);
    up_to(k0, k1, a.rows_k);
  }
  int lk = k1 - k0;
  bool cut = false;
  if (a.lengths_k && lane < S) {
    cut = length < 0 || length > lk;
    lk = min(max(length, 0), lk);
  }
  *bad = any || __ballot(cut) != 0;
  return make_int4(q0, q1 - q0, k0, lk);
}

// The item of this block: its key head, its part, its sequence and its first row (KEYS:
// key) there; and the first and last query (key) row of all sequences, set only for a call
// that clears the others.  Items run by falling cost, the keys that a block of ROWS rows sees (KEYS: the
// rows that see a block of ROWS keys).  Up to 64 sequences, a wave holds one per lane
// and finds the item of a rank from how many cost more, for which there is a formula:
// no list, and no launch to make one (that took 10 us); more sequences have a list.
template <bool KEYS, int ROWS>
__device__ __forceinline__ bool find_item(const PackArgs &a, int *head, int *part, int4 *seq, int *at, int2 *ends) {
  int rank;
  if (a.sequences > 64) {
    if (a.clear) *ends = make_int2(a.ends[KEYS ? 2 : 0], a.ends[KEYS ? 3 : 1]);
    if (!pack_place(static_cast<int>(blockIdx.x), a.kv_heads, a.count[0], a.splits, head, &rank, part)) return false;
    *seq = a.list.items[2 * rank];
    *at = a.list.items[2 * rank + 1].x;
    return true;
  }
  const int lane = static_cast<int>(threadIdx.x) & 63;
  bool bad;
  const int4 s = lane_sequence(a, lane, &bad);
  if (bad && a.status && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, kStatusBadOffsets);
  if (a.clear) {  // backward passes, which have no lengths, where KEYS
    const int first = KEYS ? s.z : s.x, end = first + (KEYS ? s.w : s.y);
    *ends = make_int2(__builtin_amdgcn_readlane(first, 0), __builtin_amdgcn_readlane(end, 63));
  }
  const int rows = s.y * a.group, ahead = s.w - s.y;
  const int tiles = ((KEYS ? s.w : rows) + ROWS - 1) / ROWS;
  const int total = lane_sum(tiles);
  if (!pack_place(static_cast<int>(blockIdx.x), a.kv_heads, total, a.splits, head, &rank, part)) return false;
  // this lane's items of cost c or more
  auto costing = [&](int c) {
    if (c == 0) return tiles;
    if constexpr (KEYS) {
      const int need = kCostRows * (c - 1) + 1;
      if (need > rows) return 0;
      if (!a.causal) return tiles;
      const int last = ahead + (rows - need) / a.group;  // key that so many rows see
      return last < 0 ? 0 : min(tiles, last / ROWS + 1);
    } else {
      const int need = kCostKeys * (c - 1) + 1;
      if (need > s.w) return 0;
      if (!a.causal) return tiles;
      return tiles - max(need - 1 - ahead, 0) * a.group / ROWS;
    }
  };
  int lo = 0, hi = 1, below = 0;  // items of cost lo or more: over rank; of hi: at most it
  int at_lo = tiles, at_hi = 0;
  for (;; hi *= 2) {
    at_hi = costing(hi);
    below = lane_sum(at_hi);
    if (below <= rank) break;
    lo = hi;
    at_lo = at_hi;
  }
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2, n = costing(mid), sum = lane_sum(n);
    if (sum > rank) {
      lo = mid;
      at_lo = n;
    } else {
      hi = mid;
      at_hi = n;
      below = sum;
    }
  }
  const int mine = at_lo - at_hi, incl = lane_scan(mine), left = rank - below;
  const int found = __ffsll(__ballot(incl > left)) - 1;
  const int tile = (KEYS ? at_hi : tiles - at_lo) + left - (incl - mine);
  auto of = [&](int x) { return __builtin_amdgcn_readlane(x, found); };
  *at = of(tile) * ROWS;
  *seq = make_int4(of(s.x), of(s.y), of(s.z), of(s.w));
  return true;
}

template <bool KEYS, int ROWS>
__device__ __forceinline__ bool pack_item(const PackArgs &a, int *head, int *part, int4 *seq, int *at, int2 *ends) {
  if (!find_item<KEYS, ROWS>(a, head, part, seq, at, ends)) return false;
  *head = scalar(*head);
  *part = scalar(*part);
  *at = scalar(*at);
  *seq = make_int4(scalar(seq->x), scalar(seq->y), scalar(seq->z), scalar(seq->w));
  return true;
}

// First and last row of all sequences, of queries or keys.
__device__ __forceinline__ int2 pack_ends(const PackArgs &a, bool keys) {
  if (a.sequences > 64) return make_int2(a.ends[keys ? 2 : 0], a.ends[keys ? 3 : 1]);
  const int32_t *off = keys ? a.offsets_k : a.offsets_q;
  const int rows = keys ? a.rows_k : a.rows_q, lane = static_cast<int>(threadIdx.x) & 63, S = a.sequences;
  const int first = min(max(off[0], 0), rows);
  int v = max(off[min(lane, S)], off[S]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o));
  return make_int2(first, min(max(v, first), rows));
}

// Rows of `out` in no sequence, as 0 (lse, where given: -inf), by all blocks of a launch, so
// that it takes no other: backward of 256 tokens, d = 64, 23.5 us, leaving them 23.2.  Only
// a call that clears them comes here, and without parts: their join does it.
template <typename T, int D, int THREADS>
__device__ __forceinline__ void clear_rows(const PackRows &out, int heads, int rows, const int2 &ends, float *lse) {
  constexpr uint32_t LANES = D * sizeof(T) / 16, PER = THREADS / LANES;  // 16 bytes a lane
  const uint32_t rest = static_cast<uint32_t>(rows - (ends.y - ends.x));
  if (rest == 0) return;
  const uint32_t all = rest * static_cast<uint32_t>(heads), lane = threadIdx.x % LANES;  // heads * rows < 2^31
  for (uint32_t i = blockIdx.x * PER + threadIdx.x / LANES; i < all; i += gridDim.x * PER) {
    const uint32_t head = i / rest;
    int row = static_cast<int>(i - head * rest);
    if (row >= ends.x) row += ends.y - ends.x;
    reinterpret_cast<uint4 *>(rows_base(out, row, static_cast<int>(head)))[lane] = make_uint4(0, 0, 0, 0);
    if (lse && lane == 0) lse[static_cast<size_t>(head) * rows + row] = -INFINITY;
  }
}

}  // namespace scope
