// dK and dV of the training attention for bf16 inputs (attention_train.hip has
// the formulas, and the kernel for fp32).
//
// A block owns 128 keys, a wave 32 of them, whose K rows stay in registers as
// matrix operands (V rows too at d = 64; at d = 128, where dK and dV take half of
// the registers, they stay in LDS) and whose dK and dV in accumulators; the
// clusters' queries stream through LDS in tiles of 32, Q and dO rows gathered by
// the buffer unit while the tile before is computed.  Per tile a wave runs
//   S = Q_tile . K^T, dP = dO_tile . V^T   (queries x keys, row-major tile reads)
//   p = exp2(scale log2(e) S - lse), ds = p (m dP - D)
//   dV^T += dO_tile^T . (m p), dK^T += Q_tile^T . ds    (transposing tile reads)
// with p and ds going from the accumulator layout straight into the operand of
// the second products, as the forward's weights do: rounded to bf16 there, the sums
// in fp32.
//
// Bound by the matrix products it runs, which with sparse sets are more than those
// that count: a wave computes a tile if its cluster keeps one of its 32 keys, and a
// block takes the time of its busiest waves.  Dense (3 heads x 32760, d = 128) 3.04
// ms, 1.08 PFLOP/s of its four products, matrix pipe 52% busy.  Two blocks share a CU (d = 64: three), so that one computes
// where the other's waves have nothing to do or wait: blocks of 256 keys and tiles
// of 64 queries, one block per CU, took 2.9 ms dense, but on the sparse layer's own
// sets 5.09 for 4.79 ms (5 heads x 32760, 54% of the keys kept) and 3.38 for 3.22
// (15%); d = 64, 8 heads x 19721, 1040 for 804 us.
#include "attention_tile.h"
#include "common.h"
#include "kernels.h"
#include "mfma.h"
#include "noise.h"

namespace scope {

namespace {

constexpr int kList = 1024;        // active tiles listed at a time
static_assert(kTrainKeyTile == 32, "a tile is one matrix product's rows");

constexpr int kWaves = kTrainKeyBlock / 32;  // a wave owns 32 keys

template <int D, bool DROP>
__global__ __launch_bounds__(64 * kWaves)
__attribute__((amdgpu_waves_per_eu(D == 64 && !DROP ? 3 : 2))) void grad_keys_kernel(TrainArgs a, uint16_t *dk, uint16_t *dv) {
  constexpr int kPlane = 64;  // a row value's plane: a lane each
  constexpr int CH = D / 8;              // 16-byte chunks per row
  constexpr int RPL = 64 / CH;           // rows per gather load
  constexpr int NG = kTrainKeyTile / kWaves / RPL; // gather loads per wave, tile and matrix
  // a tile of Q, followed by four values per row: -lse (exp2 domain), D, and with
  // dropout the query's two words (in the tile's array: the compiler does not see
  // the buffer unit write to an array of their own, and folds its reads away)
  constexpr int kStats = kTrainKeyTile * D;
  __shared__ __attribute__((aligned(256))) uint16_t Q0[kStats + 8 * kPlane], Q1[kStats + 8 * kPlane], G0[kTrainKeyTile * D], G1[kTrainKeyTile * D];
  // d = 128: the block's V rows (each wave reads its own), for registers' sake
  constexpr bool VLDS = D == 128;
  __shared__ __attribute__((aligned(16))) uint16_t Vs[VLDS ? kTrainKeyBlock * D : 8];
  __shared__ int2 list[kList];
  __shared__ int found[kWaves];
  const int splits = a.splits, blocks = (a.n + kTrainKeyBlock - 1) / kTrainKeyBlock;
  const int kb = static_cast<int>(blockIdx.x) % blocks, part = static_cast<int>(blockIdx.x) / blocks % splits;
  const int h = static_cast<int>(blockIdx.x) / blocks / splits;
  const int t = threadIdx.x, lane = t & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const size_t first = static_cast<size_t>(h) * a.n;

  TileReader<D> at(lane);
  bf16x8 kf[D / 16], vf[VLDS ? 1 : D / 16];
  const int own_row = 32 * w + l32, place = kb * kTrainKeyBlock + own_row;
  const bool by_position = keys_by_position(a.order, h, lane);
  const int key = place >= a.n ? a.n : by_position ? a.order.key[first + place] : place;
  {
    const size_t from = (first + min(key, a.n - 1)) * D;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      kf[x] = as_bf16x8(key < a.n ? load8<true>(a.k, from + 16 * x + 8 * hf) : make_uint4(0, 0, 0, 0));
      const uint4 v = key < a.n ? load8<true>(a.v, from + 16 * x + 8 * hf) : make_uint4(0, 0, 0, 0);
      if constexpr (VLDS)
        *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(Vs + 32 * w * D) + (at.row_at ^ (x << 5))) = v;
      else
        vf[x] = as_bf16x8(v);
    }
  }
  const uint32_t *wk = a.words + (4 * static_cast<size_t>(h) + 2) * a.n + min(key, a.n - 1);
  const uint2 mine = DROP ? make_uint2(wk[0], wk[a.n]) : make_uint2(0, 0);
  f32x16 dka[D / 32], dva[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) dka[db][e] = dva[db][e] = 0.0f;

  const int nbytes = static_cast<int>(static_cast<uint32_t>(a.n) * (D * 2));
  auto rsrc = [](const void *p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), static_cast<short>(0), bytes, 0x00020000);
  };
  const __amdgpu_buffer_rsrc_t rq = rsrc(static_cast<const uint16_t *>(a.q) + first * D, nbytes);
  const __amdgpu_buffer_rsrc_t rg = rsrc(static_cast<const uint16_t *>(a.d_o) + first * D, nbytes);
  const __amdgpu_buffer_rsrc_t rp = rsrc(a.perm + first, a.n * 4);
  // plane w < 4 of the rows' values: statistics, then words
  const __amdgpu_buffer_rsrc_t rs = rsrc(w < 2 ? static_cast<const void *>(a.stats + (2 * static_cast<size_t>(h) + w) * (a.n + 1))
                                               : static_cast<const void *>(a.words + (4 * static_cast<size_t>(h) + (w & 1)) * a.n),
                                         w < 2 ? (a.n + 1) * 4 : DROP ? a.n * 4 : 0);
  constexpr int WORDS = kTrainMaskKeys / 32, SHARE = kTrainMaskKeys / kTrainKeyBlock;
  const uint32_t *masks = (by_position ? a.order.masks : a.masks) + (static_cast<size_t>(h) * ((a.n + kTrainMaskKeys - 1) / kTrainMaskKeys) + kb / SHARE) * a.c_q * WORDS +
                          kWaves * (kb % SHARE);

  // Rows past a tile's end repeat its last one, with the statistics of row n,
  // which give it no weight.
  struct Idx {
    int row[NG], own;   // gathered rows, and row `lane` for the statistics
    uint32_t m;         // the wave's key bits of the tile's cluster
  };
  auto entry_of = [&](int i) {
    const int2 e = list[i];
    return make_int2(__builtin_amdgcn_readfirstlane(e.x), __builtin_amdgcn_readfirstlane(e.y));
  };
  auto load_idx = [&](int i, int count, Idx &ix) {
    if (i >= count) return;
    const int2 e = entry_of(i);
    const int rows = e.y & 255, c = e.y >> 8;
#pragma unroll
    for (int x = 0; x < NG; ++x) {
      const int row = (kTrainKeyTile / kWaves) * w + RPL * x + lane / CH;
      ix.row[x] = __builtin_amdgcn_raw_buffer_load_b32(rp, (e.x + min(row, rows - 1)) * 4, 0, 0);
    }
    const int j = __builtin_amdgcn_raw_buffer_load_b32(rp, (e.x + min(lane, rows - 1)) * 4, 0, 0);
    ix.own = lane < rows ? j : a.n;
    ix.m = masks[c * WORDS + w];
  };
  auto gather = [&](uint16_t *q, uint16_t *g, const Idx &ix) {
#pragma unroll
    for (int x = 0; x < NG; ++x) {
      const int r0 = (kTrainKeyTile / kWaves) * w + RPL * x, row = r0 + lane / CH;
      const int at = ix.row[x] * (D * 2) + 16 * ((lane % CH) ^ tile_swizzle<D>(row));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, q + r0 * D, 16, at, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rg, g + r0 * D, 16, at, 0, 0, 0);
    }
    if (w < (DROP ? 4 : 2)) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, q + kStats + 2 * kPlane * w, 4, ix.own * 4, 0, 0, 0);
  };

  auto compute = [&](const uint16_t *qt, const uint16_t *gt, uint32_t m) {
    const float *st = reinterpret_cast<const float *>(qt + kStats);
    // a key that the cluster does not keep has no weight, whatever its K and V
    // rows hold: the bits of its operands are cleared
    const uint32_t keep = (m >> l32) & 1u ? ~0u : 0u;
    auto operand = [&](const float *x) {
      const uint4 u = __builtin_bit_cast(uint4, pack8(x));
      return as_bf16x8(make_uint4(u.x & keep, u.y & keep, u.z & keep, u.w & keep));
    };
    // The empty asm statements end a phase: its products stay before them (the
    // compiler would sink them past a scheduling barrier, and spill what they
    // read), and the places are formed anew after them (kept over the loop they
    // would be a register for each place and buffer instead of an offset).
    f32x16 s, dp;
    asm volatile("" : "+v"(at.row_at));
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = dp[e] = 0.0f;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          at.row(qt, x), kf[x], s, 0, 0, 0);
    interleave<D / 16, 1, 0>();
    asm volatile("" : "+v"(s), "+v"(at.row_at));
    // p, with its sign bit set where dropout drops it, and the kept ones' operands
    float p[16];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      const bf16x8 g = at.row(gt, x);
      bf16x8 v;
      if constexpr (VLDS)
        v = at.row(Vs + 32 * w * D, x);
      else
        v = vf[x];
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g, v, dp, 0, 0, 0);
    }
    bf16x8 pk[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r0 = 8 * i + 4 * hf;
      const float4 nl = *reinterpret_cast<const float4 *>(&st[r0]);
      const float nls[4] = {nl.x, nl.y, nl.z, nl.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) p[4 * i + j] = __builtin_amdgcn_exp2f(fmaf(s[4 * i + j], a.scale_log2, nls[j]));
    }
    if constexpr (DROP) {
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        float kept[8];
#pragma unroll
        for (int i = 2 * s2; i < 2 * s2 + 2; ++i) {
          const int r0 = 8 * i + 4 * hf;
          const uint4 wx = *reinterpret_cast<const uint4 *>(&st[2 * kPlane + r0]);
          const uint4 wy = *reinterpret_cast<const uint4 *>(&st[3 * kPlane + r0]);
          const uint32_t wxs[4] = {wx.x, wx.y, wx.z, wx.w}, wys[4] = {wy.x, wy.y, wy.z, wy.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = 4 * i + j;
            const bool k = pair_kept(make_uint2(wxs[j], wys[j]), mine, a.drop);
            kept[4 * (i & 1) + j] = k ? p[e] : 0.0f;
            p[e] = k ? p[e] : -p[e];
          }
        }
        pk[s2] = operand(kept);
      }
    } else {
      pk[0] = operand(p);
      pk[1] = operand(p + 8);
    }
    interleave<D / 16, VLDS ? 2 : 1, D == 128 ? 6 : 12>();
    asm volatile("" : "+v"(dp), "+v"(pk[0]), "+v"(pk[1]), "+v"(at.col_at));
    float ds[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 dl = *reinterpret_cast<const float4 *>(&st[kPlane + 8 * i + 4 * hf]);
      const float dls[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = 4 * i + j;
        const float g = DROP ? (p[e] > 0.0f ? dp[e] * a.kept_scale : 0.0f) : dp[e];
        ds[e] = fabsf(p[e]) * (g - dls[j]);
      }
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        dva[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.columns(gt + 16 * s2 * D, db), pk[s2], dva[db], 0, 0, 0);
    bf16x8 dsk[2] = {operand(ds), operand(ds + 8)};
    interleave<D / 16, 2, D == 128 ? 6 : 12>();
#pragma unroll
    for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(dva[db]));
    asm volatile("" : "+v"(dsk[0]), "+v"(dsk[1]), "+v"(at.col_at));
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        dka[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.columns(qt + 16 * s2 * D, db), dsk[s2], dka[db], 0, 0, 0);
    interleave<D / 16, 2, 0>();
#pragma unroll
    for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(dka[db]));
  };

  // the part's tiles of the head's list, those whose cluster keeps a key of the
  // block listed in LDS, up to kList at a time
  const int per = (a.items_per_head + splits - 1) / splits;
  int next = part * per;
  const int end = min(next + per, a.items_per_head);
  const int4 *items = a.items + static_cast<size_t>(h) * a.items_per_head;
  while (next < end) {
    int count = 0;
    while (next < end && count + 64 * kWaves <= kList) {
      int2 e = make_int2(0, 0);
      bool active = false;
      if (next + t < end) {
        const int4 it = items[next + t];
        if (it.z > 0) {
          const uint4 *m = reinterpret_cast<const uint4 *>(masks + it.x * WORDS);
          uint32_t any = 0;
#pragma unroll
          for (int i = 0; i < kWaves / 4; ++i) any |= (m[i].x | m[i].y) | (m[i].z | m[i].w);
          active = any != 0;
          e = make_int2(a.offsets[static_cast<size_t>(h) * (a.c_q + 1) + it.x] + it.y, it.x << 8 | it.z);
        }
      }
      const unsigned long long votes = __ballot(active);
      if (lane == 0) found[w] = __popcll(votes);
      __syncthreads();
      int slot = count + __popcll(votes & ((1ull << lane) - 1ull));
      for (int i = 0; i < kWaves; ++i) {
        if (i < w) slot += found[i];
        count += found[i];
      }
      if (active) list[slot] = e;
      next += 64 * kWaves;
      __syncthreads();
    }
    count = __builtin_amdgcn_readfirstlane(count);
    // step T: indices of tile T + 2 requested, tile T + 1 gathered, tile T
    // computed; every wave's gathers land before the barrier
    Idx now{}, ahead{};
    uint32_t m = 0;
    load_idx(0, count, now);
    load_idx(1, count, ahead);
    if (count > 0) gather(Q0, G0, now);
    m = now.m;
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
    auto step = [&](int i, uint16_t *qc, uint16_t *gc, uint16_t *qn, uint16_t *gn) {
      now = ahead;
      if (i + 1 < count) gather(qn, gn, now);
      load_idx(i + 2, count, ahead);
      if (m) compute(qc, gc, m);
      m = now.m;
      __builtin_amdgcn_s_waitcnt(0x0F70);
      __syncthreads();
    };
    for (int i = 0; i < count; i += 2) {
      step(i, Q0, G0, Q1, G1);
      if (i + 1 < count) step(i + 1, Q1, G1, Q0, G0);
    }
  }

  if (key >= a.n) return;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const size_t at = (first + key) * D + 32 * db + 8 * i + 4 * hf;
      const f32x16 &x = dka[db], &y = dva[db];
      if (splits > 1) {
        float *p = a.parts + static_cast<size_t>(part) * 2 * a.rows * D;
        *reinterpret_cast<float4 *>(p + at) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        *reinterpret_cast<float4 *>(p + a.rows * D + at) = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
      } else {
        *reinterpret_cast<uint2 *>(dk + at) = make_uint2(pack_bf16(x[4 * i] * a.scale, x[4 * i + 1] * a.scale),
                                                         pack_bf16(x[4 * i + 2] * a.scale, x[4 * i + 3] * a.scale));
        *reinterpret_cast<uint2 *>(dv + at) = make_uint2(pack_bf16(y[4 * i] * a.kept_scale, y[4 * i + 1] * a.kept_scale),
                                                         pack_bf16(y[4 * i + 2] * a.kept_scale, y[4 * i + 3] * a.kept_scale));
      }
    }
}

template <int D>
hipError_t run(const TrainArgs &a, int heads, uint16_t *dk, uint16_t *dv, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(heads) * a.splits * ((a.n + kTrainKeyBlock - 1) / kTrainKeyBlock));
  if (a.drop)
    hipLaunchKernelGGL((grad_keys_kernel<D, true>), grid, dim3(64 * kWaves), 0, s, a, dk, dv);
  else
    hipLaunchKernelGGL((grad_keys_kernel<D, false>), grid, dim3(64 * kWaves), 0, s, a, dk, dv);
  return hipGetLastError();
}

}  // namespace

hipError_t train_keys(int d, const TrainArgs &a, int heads, uint16_t *dk, uint16_t *dv, hipStream_t s) {
  return d == 128 ? run<128>(a, heads, dk, dv, s) : run<64>(a, heads, dk, dv, s);
}

}  // namespace scope
