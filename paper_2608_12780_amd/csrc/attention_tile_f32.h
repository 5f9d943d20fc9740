// Tiles of gathered fp32 rows in LDS and their products, as the training attention's
// and the packed attention's fp32 kernels use them.
#pragma once

#include "common.h"
#include "kernels.h"

namespace scope {

constexpr int kThreads = 256;   // of a block
constexpr int kRows = 16 * kThreads / 64;   // rows (queries or keys) per block
constexpr int kTile = 32;                   // gathered rows per step
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Tiles of kTile gathered rows in LDS, written there by the buffer unit while the
// tile before is computed; 16-byte slots are XOR-swizzled by the row, so that 16
// rows' reads of a slot, and one row's of 16 slots, take distinct banks.
template <int D>
struct TileF32 {
  static constexpr int kFloats = kTile * D;
  static constexpr int CH = D / 4;          // 16-byte chunks per row
  static constexpr int RPL = 64 / CH;       // rows per gather load
  static constexpr int NG = kTile / (kThreads / 64) / RPL;  // gather loads per wave and tile
  int row_at, col_at;  // bytes: of row l16, chunk g; of row 4 g, chunk l16
  __device__ __forceinline__ TileF32(int l16, int g)
      : row_at(4 * D * l16 + 16 * (g ^ l16)), col_at(16 * D * g + 16 * (l16 ^ (4 * g))) {}
  static __device__ __forceinline__ float4 at(const float *tile, int bytes) {
    return *reinterpret_cast<const float4 *>(reinterpret_cast<const char *>(tile) + bytes);
  }
  // 16 rows of a tile . columns^T, of two tiles (or halves of one) at a time: one
  // accumulator alone would wait for itself.  Element r of a lane is row 4 g + r.
  __device__ __forceinline__ void scores(const float *t0, const float4 (&f0)[D / 16], f32x4 &s0, const float *t1,
                                         const float4 (&f1)[D / 16], f32x4 &s1) const {
    s0 = s1 = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const float4 x = at(t0, row_at ^ (s << 6)), y = at(t1, row_at ^ (s << 6));
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, f0[s].x, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(y.x, f1[s].x, s1, 0, 0, 0);
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, f0[s].y, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(y.y, f1[s].y, s1, 0, 0, 0);
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, f0[s].z, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(y.z, f1[s].z, s1, 0, 0, 0);
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, f0[s].w, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(y.w, f1[s].w, s1, 0, 0, 0);
    }
  }
  // out += (rows 16 b .. of the tile)^T . w, w in the layout of scores(); row m of
  // out[cb] is channel 64 (cb / 4) + 4 m + cb % 4, so that a lane reads 16 bytes
  __device__ __forceinline__ void accumulate(const float *tile, f32x4 (&out)[D / 16], const float (&w)[4], int b) const {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const float4 t = at(tile + (16 * b + r) * D + 64 * c, col_at ^ (r << 4));
        out[4 * c] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.x, w[r], out[4 * c], 0, 0, 0);
        out[4 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.y, w[r], out[4 * c + 1], 0, 0, 0);
        out[4 * c + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.z, w[r], out[4 * c + 2], 0, 0, 0);
        out[4 * c + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.w, w[r], out[4 * c + 3], 0, 0, 0);
      }
  }
  // this wave's rows of a tile, of the indices in `row`
  static __device__ __forceinline__ void gather(const __amdgpu_buffer_rsrc_t &from, float *tile, const int (&row)[NG],
                                                int w, int lane) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int r0 = (RPL * NG) * w + RPL * i, r = r0 + lane / CH;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(from, tile + r0 * D, 16, row[i] * (4 * D) + 16 * ((lane % CH) ^ (r & 15)), 0, 0, 0);
    }
  }
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), static_cast<short>(0), static_cast<int>(bytes), 0x00020000);
}

// This lane's fragments of a row (zeros where there is none), and its share of the
// results times `f` into the row of its column.
template <int D>
__device__ __forceinline__ void load_row(float4 (&f)[D / 16], const float *row, bool valid, int g) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    f[s] = valid ? *reinterpret_cast<const float4 *>(row + 16 * s + 4 * g) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}
template <int D>
__device__ __forceinline__ void store_row(float *row, const f32x4 (&acc)[D / 16], float f, int g) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<float4 *>(row + 64 * c + 4 * (4 * g + r)) =
          make_float4(acc[4 * c][r] * f, acc[4 * c + 1][r] * f, acc[4 * c + 2][r] * f, acc[4 * c + 3][r] * f);
}

}  // namespace scope
