// Attention over packed sequences, fp32 inputs: the forward and dQ by rows, dK and dV
// by keys (packed_plan.hip has the formulas), with fp32 matrix products, so that
// nothing but the results is rounded.  A wave owns 16 rows (query, head of the group)
// or keys, four waves a block; the other side's rows come 32 at a time through LDS.
// The fp32 products run at a sixteenth of the bf16 rate and bound these kernels: 7
// sequences of 356 to 1784 tokens, 4 heads in groups of 2, d = 128, dQ 96 us, dK and dV
// 108 (102 and 116 in the first calls after a pause), fp32 matrix pipe 63 to 66% busy.
#include "attention_tile_f32.h"
#include "packed.h"

namespace scope {

namespace {

static_assert(kPackRowsF32 == kRows, "rows of a block");
static_assert(kPackThreads == kThreads, "threads of a block");

template <int D, bool GRAD>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2))) void packed_queries_f32_kernel(PackArgs a, PackRows out) {
  typedef TileF32<D> T;
  __shared__ __attribute__((aligned(16))) float K0[T::kFloats], K1[T::kFloats], V0[T::kFloats], V1[T::kFloats];
  int h, part, row0;
  int4 sq;
  int2 ends;
  const bool item = pack_item<false, kPackRowsF32>(a, &h, &part, &sq, &row0, &ends);
  if (a.clear && a.splits == 1)
    clear_rows<float, D, kThreads>(out, a.kv_heads * a.group, a.rows_q, ends, GRAD ? nullptr : a.lse);
  if (!item) return;
  const int q0 = sq.x, lq = sq.y, k0 = sq.z, lk = sq.w, rows = lq * a.group;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const T at(l16, g);
  const int own = row0 + 16 * w + l16, row = min(own, rows - 1);
  const bool valid = own < rows, active = row0 + 16 * w < rows;
  const int query = row / a.group, member = row - query * a.group;
  const size_t stat = (static_cast<size_t>(h) * a.rows_q + q0) * a.group + row;
  const int seen = keys_seen(row, a.group, lq, lk, a.causal);
  const int most = __builtin_amdgcn_readlane(seen, 15);
  const int block_most = keys_seen(min(row0 + kRows, rows) - 1, a.group, lq, lk, a.causal);
  float4 qf[D / 16], gf[GRAD ? D / 16 : 1];
  load_row<D>(qf, reinterpret_cast<const float *>(rows_base(a.q, q0, h * a.group) + query * a.q.row + member * a.q.head), valid, g);
  float neg_lse = -INFINITY, delta = 0.0f;
  if constexpr (GRAD) {
    load_row<D>(gf, reinterpret_cast<const float *>(rows_base(a.d_o, q0, h * a.group) + query * a.d_o.row + member * a.d_o.head), valid, g);
    float4 of[D / 16];
    load_row<D>(of, reinterpret_cast<const float *>(rows_base(a.o, q0, h * a.group) + query * a.o.row + member * a.o.head), valid, g);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      delta = fmaf(of[s].x, gf[s].x, delta);
      delta = fmaf(of[s].y, gf[s].y, delta);
      delta = fmaf(of[s].z, gf[s].z, delta);
      delta = fmaf(of[s].w, gf[s].w, delta);
    }
    delta += __shfl_xor(delta, 16);
    delta += __shfl_xor(delta, 32);
    if (valid) {
      const float lse = a.lse[static_cast<size_t>(h * a.group + member) * a.rows_q + q0 + query];
      neg_lse = lse == -INFINITY ? -INFINITY : lse * -1.4426950408889634f;  // no key: no weight
      if (g == 0 && part == 0) {
        a.stats[stat] = neg_lse;
        a.stats[static_cast<size_t>(a.kv_heads) * a.rows_q * a.group + stat] = delta;
      }
    }
  }
  f32x4 acc[D / 16];
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb) acc[cb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;

  // the part's tiles
  const int all = (block_most + kTile - 1) / kTile, per = (all + a.splits - 1) / a.splits;
  const int first = scalar(min(part * per, all)), last = scalar(min(first + per, all));
  const int last_own = scalar(active ? min(last, (most + kTile - 1) / kTile) : 0);
  // rows past the last key repeat it, with no weight; addressed from the tile (a sequence
  // may be longer than 32-bit offsets reach)
  char *const k_base = rows_base(a.k, k0, h), *const v_base = rows_base(a.v, k0, h);
  auto bring = [&](float *kt, float *vt, int index) {
    const int held = min(lk - index * kTile, kTile);
    const __amdgpu_buffer_rsrc_t rk = pack_resource(k_base + static_cast<int64_t>(index) * kTile * a.k.row, span(a.k, held, 1, 4 * D));
    const __amdgpu_buffer_rsrc_t rv = pack_resource(v_base + static_cast<int64_t>(index) * kTile * a.v.row, span(a.v, held, 1, 4 * D));
#pragma unroll
    for (int i = 0; i < T::NG; ++i) {
      const int r0 = (T::RPL * T::NG) * w + T::RPL * i, r = r0 + lane / T::CH;
      const int key = min(r, held - 1), col = 16 * ((lane % T::CH) ^ (r & 15));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, kt + r0 * D, 16, key * static_cast<uint32_t>(a.k.row) + col, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, vt + r0 * D, 16, key * static_cast<uint32_t>(a.v.row) + col, 0, 0, 0);
    }
  };
  auto compute = [&](int index, const float *kt, const float *vt) {
    f32x4 s[2];
    float p[2][4];
    at.scores(kt, qf, s[0], kt + 16 * D, qf, s[1]);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (index * kTile + 16 * b + 4 * g + e >= seen) s[b][e] = -INFINITY;
    if constexpr (!GRAD) {
      float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top * a.scale_log2);
      const float neg = m_new == -INFINITY ? 0.0f : -m_new;
      const float alpha = __builtin_amdgcn_exp2f(m + neg);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int cb = 0; cb < D / 16; ++cb) acc[cb] *= alpha;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], a.scale_log2, neg));
          l += p[b][e];
        }
#pragma unroll
      for (int b = 0; b < 2; ++b) at.accumulate(vt, acc, p[b], b);
    } else {
      f32x4 dp[2];
      at.scores(vt, gf, dp[0], vt + 16 * D, gf, dp[1]);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], a.scale_log2, neg_lse)) * (dp[b][e] - delta);
#pragma unroll
      for (int b = 0; b < 2; ++b) at.accumulate(kt, acc, p[b], b);
    }
  };
  // one step: the next tile brought, this one computed; every wave's loads land before
  // the barrier
  auto step = [&](int index, const float *kc, const float *vc, float *kn, float *vn) {
    if (index + 1 < last) bring(kn, vn, index + 1);
    if (index < last_own) compute(index, kc, vc);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
  };
  if (first < last) bring(K0, V0, first);
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  for (int index = first; index < last; index += 2) {
    step(index, K0, V0, K1, V1);
    if (index + 1 < last) step(index + 1, K1, V1, K0, V0);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (!valid) return;
  if (a.splits > 1) {
    const size_t total = static_cast<size_t>(a.kv_heads) * a.rows_q * a.group, i = part * total + stat;
    store_row<D>(a.parts + i * D, acc, 1.0f, g);
    if (!GRAD && g == 0) reinterpret_cast<float2 *>(a.parts + a.splits * total * D)[i] = make_float2(m, l);
    return;
  }
  float f = a.scale;
  if constexpr (!GRAD) {
    f = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (g == 0)
      a.lse[static_cast<size_t>(h * a.group + member) * a.rows_q + q0 + query] =
          l > 0.0f ? (m + __log2f(l)) * kPackLn2 : l == 0.0f ? -INFINITY : l;
  }
  store_row<D>(reinterpret_cast<float *>(rows_base(out, q0, h * a.group) + query * out.row + member * out.head), acc, f, g);
}

template <int D>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2))) void packed_keys_f32_kernel(PackArgs a, PackRows dk, PackRows dv) {
  typedef TileF32<D> T;
  // Q tiles are followed by their rows' statistics (in the tile's array, as in
  // attention_keys.hip)
  constexpr int kQ = T::kFloats + 2 * 64;
  __shared__ __attribute__((aligned(16))) float Q0[kQ], Q1[kQ], G0[T::kFloats], G1[T::kFloats];
  int h, part, key0;
  int4 sq;
  int2 ends;
  const bool item = pack_item<true, kPackRowsF32>(a, &h, &part, &sq, &key0, &ends);
  if (a.clear && a.splits == 1) {
    clear_rows<float, D, kThreads>(dk, a.kv_heads, a.rows_k, ends, nullptr);
    clear_rows<float, D, kThreads>(dv, a.kv_heads, a.rows_k, ends, nullptr);
  }
  if (!item) return;
  const int q0 = sq.x, lq = sq.y, k0 = sq.z, lk = sq.w, rows = lq * a.group;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const T at(l16, g);
  const int own = key0 + 16 * w + l16, key = min(own, lk - 1);
  const bool valid = own < lk, active = key0 + 16 * w < lk;
  float4 kf[D / 16], vf[D / 16];
  load_row<D>(kf, reinterpret_cast<const float *>(rows_base(a.k, k0 + key, h)), valid, g);
  load_row<D>(vf, reinterpret_cast<const float *>(rows_base(a.v, k0 + key, h)), valid, g);
  // the first row that sees this key
  const int sees = a.causal ? max(key - (lk - lq), 0) * a.group : 0;
  const int sees_least = __builtin_amdgcn_readlane(sees, 0);
  f32x4 dka[D / 16], dva[D / 16];
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb) dka[cb] = dva[cb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const int tiles_all = (rows + kTile - 1) / kTile;
  const int from_tile = min((a.causal ? max(key0 - (lk - lq), 0) * a.group : 0) / kTile, tiles_all);
  const int per = (tiles_all - from_tile + a.splits - 1) / a.splits;
  const int first = scalar(min(from_tile + part * per, tiles_all)), last = scalar(min(first + per, tiles_all));
  const int first_own = scalar(active ? sees_least / kTile : last);
  char *const q_base = rows_base(a.q, q0, h * a.group), *const g_base = rows_base(a.d_o, q0, h * a.group);
  const __amdgpu_buffer_rsrc_t rs = pack_resource(
      a.stats + ((static_cast<size_t>(w & 1) * a.kv_heads + h) * a.rows_q + q0) * a.group, 4u * rows);
  // rows past the last repeat it, with no weight; addressed from the first query that the
  // tile holds a row of
  auto bring = [&](float *q, float *d_o, int index) {
    const int first_query = scalar(index * kTile / a.group), before = index * kTile - first_query * a.group;
    const int held = min(lq - first_query, kTile / a.group + 2);
    const __amdgpu_buffer_rsrc_t rq = pack_resource(q_base + first_query * a.q.row, span(a.q, held, a.group, 4 * D));
    const __amdgpu_buffer_rsrc_t rg = pack_resource(g_base + first_query * a.d_o.row, span(a.d_o, held, a.group, 4 * D));
#pragma unroll
    for (int i = 0; i < T::NG; ++i) {
      const int r0 = (T::RPL * T::NG) * w + T::RPL * i, r = r0 + lane / T::CH;
      const int row = min(before + r, rows - 1 - first_query * a.group);
      const int col = 16 * ((lane % T::CH) ^ (r & 15));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, q + r0 * D, 16, row_offset(row, a.group, a.q) + col, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rg, d_o + r0 * D, 16, row_offset(row, a.group, a.d_o) + col, 0, 0, 0);
    }
    if (w < 2)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, q + T::kFloats + 64 * w, 4, 4u * static_cast<uint32_t>(min(index * kTile + lane, rows - 1)), 0, 0, 0);
  };
  auto compute = [&](const float *qt, const float *gt, int row0) {
    const float *st = qt + T::kFloats + 4 * g;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      if (row0 + 16 * qb >= rows) break;
      f32x4 s, dp;
      at.scores(qt + 16 * qb * D, kf, s, gt + 16 * qb * D, vf, dp);
      float p[4], ds[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 16 * qb + e, row = row0 + 4 * g + i;
        const bool seen = row >= sees && row < rows;
        const float pe = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, st[i]));
        p[e] = seen ? pe : 0.0f;
        ds[e] = seen ? pe * (dp[e] - st[64 + i]) : 0.0f;
      }
      at.accumulate(gt, dva, p, qb);
      at.accumulate(qt, dka, ds, qb);
    }
  };
  auto step = [&](int index, const float *qc, const float *gc, float *qn, float *gn) {
    if (index + 1 < last) bring(qn, gn, index + 1);
    if (index >= first_own) compute(qc, gc, index * kTile);
    __builtin_amdgcn_s_waitcnt(0x0F70);
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
    float *to = a.parts + (2 * static_cast<size_t>(part) * all + static_cast<size_t>(h) * a.rows_k + k0 + key) * D;
    store_row<D>(to, dka, 1.0f, g);
    store_row<D>(to + all * D, dva, 1.0f, g);
  } else {
    store_row<D>(reinterpret_cast<float *>(rows_base(dk, k0 + key, h)), dka, a.scale, g);
    store_row<D>(reinterpret_cast<float *>(rows_base(dv, k0 + key, h)), dva, 1.0f, g);
  }
}

dim3 grid_of(const PackArgs &a) {
  return dim3(pack_blocks(a.list.capacity, a.kv_heads, a.splits));
}

template <int D, bool GRAD>
hipError_t run(const PackArgs &a, const PackRows &out, hipStream_t s) {
  hipLaunchKernelGGL((packed_queries_f32_kernel<D, GRAD>), grid_of(a), dim3(kThreads), 0, s, a, out);
  return hipGetLastError();
}

}  // namespace

hipError_t packed_queries_f32(const PackArgs &a, int d, bool grad, const PackRows &out, hipStream_t s) {
  if (d == 128) return grad ? run<128, true>(a, out, s) : run<128, false>(a, out, s);
  return grad ? run<64, true>(a, out, s) : run<64, false>(a, out, s);
}

hipError_t packed_keys_f32(const PackArgs &a, int d, const PackRows &dk, const PackRows &dv, hipStream_t s) {
  if (d == 128)
    hipLaunchKernelGGL((packed_keys_f32_kernel<128>), grid_of(a), dim3(kThreads), 0, s, a, dk, dv);
  else
    hipLaunchKernelGGL((packed_keys_f32_kernel<64>), grid_of(a), dim3(kThreads), 0, s, a, dk, dv);
  return hipGetLastError();
}

}  // namespace scope
