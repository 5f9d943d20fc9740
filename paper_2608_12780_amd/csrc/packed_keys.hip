// dK and dV of attention over packed sequences, bf16 inputs (packed_plan.hip has the
// formulas).
//
// A block owns 128 keys of a sequence, a wave 32 of them, whose K rows stay in
// registers as matrix operands (V rows too at d = 64; at d = 128, where dK and dV take
// half of the registers, they stay in LDS) and whose dK and dV in accumulators.  The
// rows (query, head of the group) that see the block's first key stream through LDS in
// tiles of 32, Q and dO brought by the buffer unit while the tile before is computed:
//   S = Q_tile . K^T, dP = dO_tile . V^T   (rows x keys)
//   p = exp2(scale log2(e) S - lse), ds = p (dP - D)
//   dV^T += dO_tile^T . p, dK^T += Q_tile^T . ds    (transposing tile reads)
// with p and ds going from the accumulator layout straight into the operand of the
// second products, rounded to bf16 there; the sums are fp32.
//
// 5 heads x 32760, d = 128: 4.95 ms, 1.11 PFLOP/s of its four products, matrix pipe 60%
// busy at 1.85 GHz, LDS 47%; d = 64, 10 heads: 5.3 ms, 1.04 PFLOP/s.
#include "attention_tile.h"
#include "packed.h"

namespace scope {

namespace {

constexpr int kWaves = kPackKeys / 32;  // a wave owns 32 keys
static_assert(64 * kWaves == kPackThreads, "threads of a block");

// A tile's rows, 32 of them: 64 at d = 64 took as long, and at d = 128 would leave a CU
// one block.
template <int D>
struct RowTile {
  static constexpr int kRows = 32;
  static constexpr int CH = D / 8;              // 16-byte chunks per row
  static constexpr int RPL = 64 / CH;           // rows per load
  static constexpr int NG = kRows / kWaves / RPL; // loads per wave
  // row and 16-byte column (in bytes) that load x of a wave brings for a lane
  static __device__ __forceinline__ int row(int x, int w, int lane) { return kRows / kWaves * w + RPL * x + lane / CH; }
  static __device__ __forceinline__ int column(int r, int lane) { return 16 * ((lane % CH) ^ tile_swizzle<D>(r)); }
  static __device__ __forceinline__ void bring(const __amdgpu_buffer_rsrc_t &from, uint16_t *tile, int x, int w, uint32_t at) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, tile + (kRows / kWaves * w + RPL * x) * D, 16, at, 0, 0, 0);
  }
};

template <int D>
__global__ __launch_bounds__(64 * kWaves)
__attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2))) void packed_keys_kernel(PackArgs a, PackRows dk, PackRows dv) {
  typedef RowTile<D> T;
  constexpr int kRowTile = T::kRows;
  constexpr int kPlane = 64;             // a row value's plane: a lane each
  // a tile of Q, followed by two values per row: -lse (exp2 domain) and D (in the
  // tile's array: the compiler does not see the buffer unit write to an array of their
  // own, and folds its reads away)
  constexpr int kStats = kRowTile * D;
  __shared__ __attribute__((aligned(256))) uint16_t Q0[kStats + 4 * kPlane], Q1[kStats + 4 * kPlane], G0[kRowTile * D], G1[kRowTile * D];
  constexpr bool VLDS = D == 128;
  __shared__ __attribute__((aligned(16))) uint16_t Vs[VLDS ? kPackKeys * D : 8];
  int h, part, key0;
  int4 sq;
  int2 ends;
  const bool item = pack_item<true, kPackKeys>(a, &h, &part, &sq, &key0, &ends);
  if (a.clear && a.splits == 1) {
    clear_rows<uint16_t, D, 64 * kWaves>(dk, a.kv_heads, a.rows_k, ends, nullptr);
    clear_rows<uint16_t, D, 64 * kWaves>(dv, a.kv_heads, a.rows_k, ends, nullptr);
  }
  if (!item) return;
  const int q0 = sq.x, lq = sq.y, k0 = sq.z, lk = sq.w, rows = lq * a.group;
  const int t = threadIdx.x, lane = t & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);

  TileReader<D> at(lane);
  bf16x8 kf[D / 16], vf[VLDS ? 1 : D / 16];
  const int own = key0 + 32 * w + l32, key = min(own, lk - 1);
  const bool valid = own < lk, active = key0 + 32 * w < lk;
  {
    const uint16_t *k = reinterpret_cast<const uint16_t *>(rows_base(a.k, k0 + key, h));
    const uint16_t *v = reinterpret_cast<const uint16_t *>(rows_base(a.v, k0 + key, h));
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      kf[x] = as_bf16x8(valid ? load8<true>(k, 16 * x + 8 * hf) : make_uint4(0, 0, 0, 0));
      const uint4 u = valid ? load8<true>(v, 16 * x + 8 * hf) : make_uint4(0, 0, 0, 0);
      if constexpr (VLDS)
        *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(Vs + 32 * w * D) + (at.row_at ^ (x << 5))) = u;
      else
        vf[x] = as_bf16x8(u);
    }
  }
  // the first row that sees this key (query >= key - (lk - lq)), and the wave's least
  // and greatest
  const int sees = a.causal ? max(key - (lk - lq), 0) * a.group : 0;
  const int sees_least = __builtin_amdgcn_readlane(sees, 0), sees_most = __builtin_amdgcn_readlane(sees, 31);
  f32x16 dka[D / 32], dva[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) dka[db][e] = dva[db][e] = 0.0f;

  // the part's tiles, from the first row that sees the block's first key
  const int tiles_all = (rows + kRowTile - 1) / kRowTile;
  const int from_tile = min((a.causal ? max(key0 - (lk - lq), 0) * a.group : 0) / kRowTile, tiles_all);
  const int per = (tiles_all - from_tile + a.splits - 1) / a.splits;
  const int first = scalar(min(from_tile + part * per, tiles_all)), last = scalar(min(first + per, tiles_all));
  // this wave's first tile
  const int first_own = scalar(active ? sees_least / kRowTile : last);

  // plane w < 2 of the rows' values
  const __amdgpu_buffer_rsrc_t rs = pack_resource(
      a.stats + ((static_cast<size_t>(w & 1) * a.kv_heads + h) * a.rows_q + q0) * a.group, 4u * rows);

  // A tile's rows are addressed from the first query that it holds a row of (a sequence
  // may be longer than 32-bit offsets reach).  Where every tile starts with a query's first
  // row, at the same offsets in all whole tiles (a quotient for each row and tile: 796 us
  // for 756, 16 heads in groups of 4, 30011 tokens of 24 prompts, d = 64).
  const bool even = kRowTile % a.group == 0;
  const int queries = kRowTile / a.group;
  char *const q_base = rows_base(a.q, q0, h * a.group), *const g_base = rows_base(a.d_o, q0, h * a.group);
  uint32_t at_q[T::NG], at_g[T::NG];
#pragma unroll
  for (int x = 0; x < T::NG; ++x) {
    const int r = T::row(x, w, lane);
    at_q[x] = row_offset(r, a.group, a.q) + T::column(r, lane);
    at_g[x] = row_offset(r, a.group, a.d_o) + T::column(r, lane);
  }
  // Rows past the last repeat it, with no weight.
  auto bring = [&](uint16_t *q, uint16_t *g, int index) {
    const int first_query = even ? index * queries : scalar(index * kRowTile / a.group);
    const int before = index * kRowTile - first_query * a.group;  // rows of that query before the tile
    const int held = min(lq - first_query, kRowTile / a.group + 2);
    const __amdgpu_buffer_rsrc_t rq = pack_resource(q_base + first_query * a.q.row, span(a.q, held, a.group, 2 * D));
    const __amdgpu_buffer_rsrc_t rg = pack_resource(g_base + first_query * a.d_o.row, span(a.d_o, held, a.group, 2 * D));
    if (even && (index + 1) * kRowTile <= rows) {
#pragma unroll
      for (int x = 0; x < T::NG; ++x) {
        T::bring(rq, q, x, w, at_q[x]);
        T::bring(rg, g, x, w, at_g[x]);
      }
    } else {
#pragma unroll
      for (int x = 0; x < T::NG; ++x) {
        const int r = T::row(x, w, lane), row = min(before + r, rows - 1 - first_query * a.group);
        T::bring(rq, q, x, w, row_offset(row, a.group, a.q) + T::column(r, lane));
        T::bring(rg, g, x, w, row_offset(row, a.group, a.d_o) + T::column(r, lane));
      }
    }
    if (w < 2)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, q + kStats + 2 * kPlane * w, 4, 4u * static_cast<uint32_t>(min(index * kRowTile + lane, rows - 1)), 0, 0, 0);
  };

  // 32 rows of a tile
  auto compute = [&](const uint16_t *qt, const uint16_t *gt, const float *st, int row0) {
    // The empty asm statements end a phase: its products stay before them, and the
    // places are formed anew after them (as in attention_keys.hip).
    f32x16 s, dp;
    asm volatile("" : "+v"(at.row_at));
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = dp[e] = 0.0f;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.row(qt, x), kf[x], s, 0, 0, 0);
    interleave<D / 16, 1, 0>();
    asm volatile("" : "+v"(s), "+v"(at.row_at));
    if (row0 < sees_most || row0 + 32 > rows) {  // rows that do not see this lane's key
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = row0 + 8 * (e >> 2) + 4 * hf + (e & 3);
        if (row < sees || row >= rows) s[e] = -INFINITY;
      }
    }
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
      const float4 nl = *reinterpret_cast<const float4 *>(&st[8 * i + 4 * hf]);
      const float nls[4] = {nl.x, nl.y, nl.z, nl.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) p[4 * i + j] = __builtin_amdgcn_exp2f(fmaf(s[4 * i + j], a.scale_log2, nls[j]));
    }
    pk[0] = pack8(p);
    pk[1] = pack8(p + 8);
    interleave<D / 16, VLDS ? 2 : 1, D == 128 ? 6 : 12>();
    asm volatile("" : "+v"(dp), "+v"(pk[0]), "+v"(pk[1]), "+v"(at.col_at));
    float ds[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 dl = *reinterpret_cast<const float4 *>(&st[kPlane + 8 * i + 4 * hf]);
      const float dls[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) ds[4 * i + j] = p[4 * i + j] * (dp[4 * i + j] - dls[j]);
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        dva[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.columns(gt + 16 * s2 * D, db), pk[s2], dva[db], 0, 0, 0);
    bf16x8 dsk[2] = {pack8(ds), pack8(ds + 8)};
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

  // step T: tile T + 1 brought, tile T computed; every wave's loads land before the
  // barrier
  auto step = [&](int index, const uint16_t *qc, const uint16_t *gc, uint16_t *qn, uint16_t *gn) {
    if (index + 1 < last) bring(qn, gn, index + 1);
    if (index >= first_own) {
      const float *st = reinterpret_cast<const float *>(qc + kStats);
#pragma unroll
      for (int b = 0; b < kRowTile / 32; ++b) compute(qc + 32 * b * D, gc + 32 * b * D, st + 32 * b, index * kRowTile + 32 * b);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
  };
  if (first < last) bring(Q0, G0, first);
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  for (int index = first; index < last; index += 2) {
    step(index, Q0, G0, Q1, G1);
    if (index + 1 < last) step(index + 1, Q1, G1, Q0, G0);
  }

  if (!valid) return;
  if (a.splits > 1) {
    const size_t all = static_cast<size_t>(a.kv_heads) * a.rows_k;
    float *to = a.parts + (2 * static_cast<size_t>(part) * all + static_cast<size_t>(h) * a.rows_k + k0 + key) * D + 4 * hf;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x16 &x = dka[db], &y = dva[db];
        *reinterpret_cast<float4 *>(to + 32 * db + 8 * i) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        *reinterpret_cast<float4 *>(to + all * D + 32 * db + 8 * i) = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
      }
    return;
  }
  uint16_t *tk = reinterpret_cast<uint16_t *>(rows_base(dk, k0 + key, h)) + 4 * hf;
  uint16_t *tv = reinterpret_cast<uint16_t *>(rows_base(dv, k0 + key, h)) + 4 * hf;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x16 &x = dka[db], &y = dva[db];
      *reinterpret_cast<uint2 *>(tk + 32 * db + 8 * i) = make_uint2(pack_bf16(x[4 * i] * a.scale, x[4 * i + 1] * a.scale),
                                                                     pack_bf16(x[4 * i + 2] * a.scale, x[4 * i + 3] * a.scale));
      *reinterpret_cast<uint2 *>(tv + 32 * db + 8 * i) = make_uint2(pack_bf16(y[4 * i], y[4 * i + 1]), pack_bf16(y[4 * i + 2], y[4 * i + 3]));
    }
}

template <int D>
hipError_t run(const PackArgs &a, const PackRows &dk, const PackRows &dv, hipStream_t s) {
  const dim3 grid(pack_blocks(a.list.capacity, a.kv_heads, a.splits));
  hipLaunchKernelGGL((packed_keys_kernel<D>), grid, dim3(64 * kWaves), 0, s, a, dk, dv);
  return hipGetLastError();
}

}  // namespace

hipError_t packed_keys(const PackArgs &a, int d, const PackRows &dk, const PackRows &dv, hipStream_t s) {
  return d == 128 ? run<128>(a, dk, dv, s) : run<64>(a, dk, dv, s);
}

}  // namespace scope
