// Tiles of gathered bf16 rows in LDS, as the gradient kernels read them: row by
// row for products over channels, transposed for products over rows.
#pragma once

#include "common.h"
#include "kernels.h"
#include "mfma.h"

namespace scope {

// 16-byte slot of a row's chunk 0 (chunk c: slot ^ c): distinct for 16 (d = 64:
// 8 pairs of) consecutive rows, which the row-major reads take together, and four
// chunks apart for the four rows of a transposing read.
template <int D>
__device__ __forceinline__ int tile_swizzle(int row) {
  return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

// Operand whose lane holds channel l32 of a 32-channel group and 16 tile rows 4 hf +
// 8 (j / 4) + j % 4, from transposing reads of two groups of four rows.
__device__ __forceinline__ bf16x8 transposed(const char *lo, const char *hi) {
  const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lo)));
  const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(hi)));
  return as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
}

__device__ __forceinline__ bf16x8 pack8(const float *w) {
  return as_bf16x8(make_uint4(pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])));
}

// Where a lane reads a tile of D-channel rows, in bytes: of row lane % 32, and
// transposing of row 4 (lane / 32) + (lane % 16) / 4.  16 channels on is the first
// xor 32, 32 channels on the second xor 64, eight rows down the second xor 32 plus
// eight rows.
template <int D>
struct TileReader {
  int row_at, col_at;
  __device__ __forceinline__ explicit TileReader(int lane) {
    const int l32 = lane & 31, hf = lane >> 5;
    const int row = 4 * hf + ((lane & 15) >> 2), chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    row_at = 2 * D * l32 + 16 * (hf ^ tile_swizzle<D>(l32));
    col_at = 2 * D * row + 16 * (chunk ^ tile_swizzle<D>(row)) + 8 * (lane & 1);
  }
  // channels 16 x .. of 32 rows
  __device__ __forceinline__ bf16x8 row(const uint16_t *tile, int x) const {
    return as_bf16x8(*reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(tile) + (row_at ^ (x << 5))));
  }
  // 16 rows of channels 32 db ..
  __device__ __forceinline__ bf16x8 columns(const uint16_t *tile, int db) const {
    const char *t = reinterpret_cast<const char *>(tile);
    return transposed(t + (col_at ^ (db << 6)), t + 16 * D + (col_at ^ (db << 6) ^ 32));
  }
};

// Scheduling of one phase's matrix instructions: MFMAs with LDS reads and vector
// instructions between them, so that neither waits for the other.
template <int N, int READS, int VALU>
__device__ __forceinline__ void interleave() {
  __builtin_amdgcn_sched_group_barrier(0x100, 2 * READS, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    if (VALU) __builtin_amdgcn_sched_group_barrier(0x002, VALU, 0);
  }
}

// Whether dK and dV take head h's keys in the order of attention_order.hip: where
// that leaves 3% fewer (32 keys, tile) pairs.  By whole waves.
__device__ __forceinline__ bool keys_by_position(const KeyOrder &order, int h, int lane) {
  static_assert(kOrderSlots == 64, "a slot per lane");
  if (!order.cost) return false;
  const unsigned long long *cost = order.cost + (static_cast<size_t>(h) * kOrderSlots + lane) * 2;
  const unsigned long long by_key = wave_sum(cost[0]);
  return wave_sum(cost[1]) + by_key / 32 < by_key;
}

}  // namespace scope
