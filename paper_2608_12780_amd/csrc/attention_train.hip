// Attention over the selected keys for training: the forward with the rows'
// log-sum-exp and dropout, and the gradients (Eq. 11; dense attention, Eq. 1, is
// the one-cluster special case).  With S_c the keys of query i's cluster c,
//   s_ij = <q_i, k_j>, p_ij = exp(scale s_ij - lse_i), m_ij the dropout factor,
//   o_i   = sum_j p_ij m_ij v_j
//   dp_ij = m_ij <do_i, v_j>,  ds_ij = p_ij (dp_ij - <do_i, o_i>)
//   dq_i  = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i,
//   dv_j  = sum_i p_ij m_ij do_i
// The gradients recompute p from lse, so nothing of size n^2 is stored.  dq runs
// over a cluster's gathered keys like the forward, a wave per 32 queries (fp32: 16);
// dk and dv run over the clusters' queries, a wave per 32 keys (fp32: 16), with a
// bit for each (cluster, key), so every sum has one owner and a fixed order: no
// atomics on results, the same bits on every run.  S and dP are computed for either
// side, seven products where five are needed (eight for bf16, whose dq takes ds in two
// terms); one pass for all three would add dq from every block of keys, in an order
// that varies or through memory of its own.
#include <math.h>

#include "attention_slots.h"
#include "attention_tile.h"
#include "attention_tile_f32.h"
#include "common.h"
#include "kernels.h"
#include "mfma.h"
#include "noise.h"

namespace scope {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// fp32 inputs: fp32 matrix products, 16 x 16 results from 4 channels (or rows) per
// instruction, so that inputs, weights and ds are not rounded.  They run at a
// sixteenth of the bf16 rate and need little bandwidth: a wave owns 16 queries
// (or keys), four waves a block, which makes short work items for an even load and
// leaves two blocks a CU (d = 64: four by queries, three by keys) to cover the staging
// of tiles.  Bound by the
// matrix pipe, 73 to 76% busy: 4 heads x 6417 tokens, d = 128, 53% of the keys kept,
// dq 740 to 766 us (88 TFLOP/s of the products that count), dk and dv 1270 to 1300.

// One wave per 16 queries of a cluster, over the cluster's keys: the forward
// (GRAD false) or dq (GRAD true).
template <int D, bool GRAD, bool DROP>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2))) void train_queries_kernel(TrainArgs a, float *out) {
  typedef TileF32<D> T;
  // K tiles are followed by the keys' two dropout words (in the same array for the
  // reason given in attention_keys.hip)
  constexpr int kK = T::kFloats + (DROP ? 2 * 64 : 0);
  __shared__ __attribute__((aligned(16))) float K0[kK], K1[kK], V0[T::kFloats], V1[T::kFloats];
  const int part = static_cast<int>(blockIdx.x) % a.splits, slot = static_cast<int>(blockIdx.x) / a.splits;
  const int4 it = a.items[slot];
  const int h = slot / a.items_per_head;
  const int c = it.x, row0 = it.y, rows = it.z, r = it.w;
  if (rows <= 0) return;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const size_t first = static_cast<size_t>(h) * a.n;
  const T at(l16, g);
  const int ql = 16 * w + l16;
  const bool valid = ql < rows, active = 16 * w < rows;
  int qi = 0;
  if (valid) {
    const int pos = min(max(a.offsets[static_cast<size_t>(h) * (a.c_q + 1) + c] + row0 + ql, 0), a.n - 1);
    qi = min(max(a.perm[first + pos], 0), a.n - 1);
  }
  float4 qf[D / 16], gf[GRAD ? D / 16 : 1];
  load_row<D>(qf, static_cast<const float *>(a.q) + (first + qi) * D, valid, g);
  float neg_lse = -INFINITY, delta = 0.0f;
  if constexpr (GRAD) {
    load_row<D>(gf, static_cast<const float *>(a.d_o) + (first + qi) * D, valid, g);
    if (valid) {
      const float *st = a.stats + 2 * h * static_cast<size_t>(a.n + 1) + qi;
      neg_lse = st[0];
      delta = st[a.n + 1];
    }
  }
  uint2 mine = make_uint2(0, 0);
  if (DROP && valid) {
    const uint32_t *wq = a.words + 4 * first + qi;
    mine = make_uint2(wq[0], wq[a.n]);
  }
  f32x4 acc[D / 16];
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb) acc[cb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;

  // the part's keys, in whole tiles
  const int per = ((r + kTile - 1) / kTile + a.splits - 1) / a.splits * kTile;
  const int from = min(part * per, r), end = min(from + per, r);
  const uint32_t bytes = static_cast<uint32_t>(a.n) * (4 * D);
  const __amdgpu_buffer_rsrc_t rk = resource(static_cast<const float *>(a.k) + first * D, bytes);
  const __amdgpu_buffer_rsrc_t rv = resource(static_cast<const float *>(a.v) + first * D, bytes);
  const __amdgpu_buffer_rsrc_t rs = resource(a.sel_idx + (static_cast<size_t>(h) * a.c_q + c) * a.n, r * 4);
  const __amdgpu_buffer_rsrc_t rw = resource(a.words + 4 * first + (2 + (w & 1)) * static_cast<size_t>(a.n), DROP ? a.n * 4 : 0);
  // rows past the end of the list repeat its last key, with no weight
  struct Idx {
    int row[T::NG], own;
  };
  auto load_idx = [&](int k0, Idx &ix) {
#pragma unroll
    for (int i = 0; i < T::NG; ++i)
      ix.row[i] = __builtin_amdgcn_raw_buffer_load_b32(rs, min(k0 + T::RPL * (T::NG * w + i) + lane / T::CH, r - 1) * 4, 0, 0);
    ix.own = DROP && w < 2 ? __builtin_amdgcn_raw_buffer_load_b32(rs, min(k0 + lane, r - 1) * 4, 0, 0) : 0;
  };
  auto gather = [&](float *k, float *v, const Idx &ix) {
    T::gather(rk, k, ix.row, w, lane);
    T::gather(rv, v, ix.row, w, lane);
    if (DROP && w < 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, k + T::kFloats + 64 * w, 4, ix.own * 4, 0, 0, 0);
  };
  auto compute = [&](int k0, const float *kt, const float *vt) {
    const uint32_t *words = reinterpret_cast<const uint32_t *>(kt + T::kFloats) + 4 * g;
    auto kept = [&](int b, int e) {
      return pair_kept(mine, make_uint2(words[16 * b + e], words[64 + 16 * b + e]), a.drop);
    };
    f32x4 s[2];
    float p[2][4];
    at.scores(kt, qf, s[0], kt + 16 * D, qf, s[1]);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k0 + 16 * b + 4 * g + e >= r) s[b][e] = -INFINITY;
    }
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
          if (DROP && !kept(b, e)) p[b][e] = 0.0f;
        }
#pragma unroll
      for (int b = 0; b < 2; ++b) at.accumulate(vt, acc, p[b], b);
    } else {
      f32x4 dp[2];
      at.scores(vt, gf, dp[0], vt + 16 * D, gf, dp[1]);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = DROP ? (kept(b, e) ? dp[b][e] * a.kept_scale : 0.0f) : dp[b][e];
          p[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], a.scale_log2, neg_lse)) * (x - delta);
        }
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) at.accumulate(kt, acc, p[b], b);
    }
  };
  // one step: indices of the tile after next requested, the next tile gathered, this
  // one computed; every wave's gathers land before the barrier
  Idx now, ahead;
  auto step = [&](int k0, const float *kc, const float *vc, float *kn, float *vn) {
    if (k0 + kTile < end) gather(kn, vn, now);
    load_idx(k0 + 2 * kTile, ahead);
    if (active) compute(k0, kc, vc);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
    now = ahead;
  };
  if (from < end) {
    load_idx(from, ahead);
    load_idx(from + kTile, now);
    gather(K0, V0, ahead);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  for (int k0 = from; k0 < end; k0 += 2 * kTile) {
    step(k0, K0, V0, K1, V1);
    if (k0 + kTile < end) step(k0 + kTile, K1, V1, K0, V0);
  }
  if (a.splits > 1) {
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (!valid) return;
    const size_t at_row = static_cast<size_t>(part) * a.rows + first + qi;
    store_row<D>(a.parts + at_row * D, acc, 1.0f, g);
    if (!GRAD && g == 0) reinterpret_cast<float2 *>(a.parts + a.splits * a.rows * D)[at_row] = make_float2(m, l);
    return;
  }
  float f = a.scale;
  if constexpr (!GRAD) {
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    f = l > 0.0f ? a.kept_scale / l : 0.0f;
    if (valid && g == 0) a.lse[first + qi] = l > 0.0f ? (m + __log2f(l)) * kLn2 : l == 0.0f ? -INFINITY : l;
  }
  if (valid) store_row<D>(out + (first + qi) * D, acc, f, g);
}

// One wave per 16 keys, over the queries of every cluster that keeps any of the
// block's keys: dk and dv, or with several parts their sums over a part's tiles.
template <int D, bool DROP>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2))) void train_keys_kernel(TrainArgs a, float *dk, float *dv) {
  typedef TileF32<D> T;
  constexpr int kList = 1024;  // active tiles listed at a time
  constexpr int kQ = T::kFloats + 4 * 64;
  // Q tiles are followed by their rows' statistics and dropout words
  __shared__ __attribute__((aligned(16))) float Q0[kQ], Q1[kQ], G0[T::kFloats], G1[T::kFloats];
  __shared__ int2 list[kList];
  __shared__ int found[kThreads / 64];
  const int splits = a.splits, blocks = (a.n + kRows - 1) / kRows;
  const int b = static_cast<int>(blockIdx.x) % blocks, part = static_cast<int>(blockIdx.x) / blocks % splits;
  const int h = static_cast<int>(blockIdx.x) / blocks / splits;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const size_t first = static_cast<size_t>(h) * a.n;
  const T at(l16, g);
  const bool by_position = keys_by_position(a.order, h, lane);
  const int place = b * kRows + 16 * w + l16;
  const bool valid = place < a.n;
  const int j = valid && by_position ? a.order.key[first + place] : place;
  const size_t kj = first + (valid ? j : 0);
  float4 kf[D / 16], vf[D / 16];
  load_row<D>(kf, static_cast<const float *>(a.k) + kj * D, valid, g);
  load_row<D>(vf, static_cast<const float *>(a.v) + kj * D, valid, g);
  uint2 mine = make_uint2(0, 0);
  if (DROP) {
    const uint32_t *wk = a.words + 4 * first + 2 * static_cast<size_t>(a.n) + (kj - first);
    mine = make_uint2(wk[0], wk[a.n]);
  }
  f32x4 dka[D / 16], dva[D / 16];
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb) dka[cb] = dva[cb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // the block's two words of each cluster, 16 bits a wave
  constexpr int WORDS = kTrainMaskKeys / 32, SHARE = kTrainMaskKeys / kRows;
  static_assert(kRows == 64, "two words per block");
  const uint32_t *masks = (by_position ? a.order.masks : a.masks) + (static_cast<size_t>(h) * ((a.n + kTrainMaskKeys - 1) / kTrainMaskKeys) + b / SHARE) * a.c_q * WORDS +
                          2 * (b % SHARE);

  const uint32_t bytes = static_cast<uint32_t>(a.n) * (4 * D);
  const __amdgpu_buffer_rsrc_t rq = resource(static_cast<const float *>(a.q) + first * D, bytes);
  const __amdgpu_buffer_rsrc_t rg = resource(static_cast<const float *>(a.d_o) + first * D, bytes);
  const __amdgpu_buffer_rsrc_t rp = resource(a.perm + first, a.n * 4);
  // plane w of the rows' values: statistics, then words
  const __amdgpu_buffer_rsrc_t rs = w < 2 ? resource(a.stats + (2 * static_cast<size_t>(h) + w) * (a.n + 1), (a.n + 1) * 4)
                                          : resource(a.words + (4 * static_cast<size_t>(h) + (w & 1)) * a.n, DROP ? a.n * 4 : 0);
  // rows past a tile's end repeat its last one, with the statistics of row n
  struct Idx {
    int row[T::NG], own, rows;
    uint32_t m;  // the wave's key bits of the tile's cluster
  };
  auto load_idx = [&](int i, int count, Idx &ix) {
    if (i >= count) return;
    const int2 e = list[i];
    const int base = __builtin_amdgcn_readfirstlane(e.x), rows = __builtin_amdgcn_readfirstlane(e.y) & 255;
    const int c = __builtin_amdgcn_readfirstlane(e.y) >> 8;
#pragma unroll
    for (int x = 0; x < T::NG; ++x)
      ix.row[x] = __builtin_amdgcn_raw_buffer_load_b32(rp, (base + min(T::RPL * (T::NG * w + x) + lane / T::CH, rows - 1)) * 4, 0, 0);
    const int own = __builtin_amdgcn_raw_buffer_load_b32(rp, (base + min(lane, rows - 1)) * 4, 0, 0);
    ix.own = lane < rows ? own : a.n;
    ix.rows = rows;
    ix.m = masks[c * WORDS + (w >> 1)] >> (16 * (w & 1)) & 0xFFFFu;
  };
  auto gather = [&](float *q, float *d_o, const Idx &ix) {
    T::gather(rq, q, ix.row, w, lane);
    T::gather(rg, d_o, ix.row, w, lane);
    if (DROP || w < 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, q + T::kFloats + 64 * w, 4, ix.own * 4, 0, 0, 0);
  };
  auto compute = [&](const float *qt, const float *gt, int rows, uint32_t m) {
    const float *st = qt + T::kFloats + 4 * g;
    const bool selected = (m >> l16) & 1u;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      if (16 * qb >= rows) break;
      f32x4 s, dp;
      at.scores(qt + 16 * qb * D, kf, s, gt + 16 * qb * D, vf, dp);
      float p[4], ds[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 16 * qb + e;
        const float pe = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, st[row]));
        float x = dp[e];
        p[e] = selected ? pe : 0.0f;
        if (DROP) {
          const bool kept = pair_kept(make_uint2(__float_as_uint(st[128 + row]), __float_as_uint(st[192 + row])), mine, a.drop);
          x = kept ? x * a.kept_scale : 0.0f;
          if (!kept) p[e] = 0.0f;
        }
        ds[e] = selected ? pe * (x - st[64 + row]) : 0.0f;
      }
      at.accumulate(gt, dva, p, qb);
      at.accumulate(qt, dka, ds, qb);
    }
  };

  const int per = (a.items_per_head + splits - 1) / splits;
  int next = part * per;
  const int end = min(next + per, a.items_per_head);
  const int4 *items = a.items + static_cast<size_t>(h) * a.items_per_head;
  while (next < end) {
    // the tiles whose cluster keeps a key of the block
    int count = 0;
    while (next < end && count + kThreads <= kList) {
      int2 e = make_int2(0, 0);
      bool some = false;
      if (next + t < end) {
        const int4 it = items[next + t];
        if (it.z > 0) {
          some = (masks[it.x * WORDS] | masks[it.x * WORDS + 1]) != 0;
          e = make_int2(a.offsets[static_cast<size_t>(h) * (a.c_q + 1) + it.x] + it.y, it.x << 8 | it.z);
        }
      }
      const unsigned long long votes = __ballot(some);
      if (lane == 0) found[w] = __popcll(votes);
      __syncthreads();
      int slot = count + __popcll(votes & ((1ull << lane) - 1ull));
      for (int i = 0; i < kThreads / 64; ++i) {
        if (i < w) slot += found[i];
        count += found[i];
      }
      if (some) list[slot] = e;
      next += kThreads;
      __syncthreads();
    }
    count = __builtin_amdgcn_readfirstlane(count);
    Idx now{}, ahead{};
    load_idx(0, count, now);
    load_idx(1, count, ahead);
    if (count > 0) gather(Q0, G0, now);
    uint32_t m = now.m;
    int rows = now.rows;
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    auto step = [&](int i, const float *qc, const float *gc, float *qn, float *gn) {
      now = ahead;
      if (i + 1 < count) gather(qn, gn, now);
      load_idx(i + 2, count, ahead);
      if (m) compute(qc, gc, rows, m);
      m = now.m;
      rows = now.rows;
      __builtin_amdgcn_s_waitcnt(0x0F70);
      __syncthreads();
    };
    for (int i = 0; i < count; i += 2) {
      step(i, Q0, G0, Q1, G1);
      if (i + 1 < count) step(i + 1, Q1, G1, Q0, G0);
    }
  }
  if (!valid) return;
  if (splits > 1) {
    float *to = a.parts + 2 * static_cast<size_t>(part) * a.rows * D + kj * D;
    store_row<D>(to, dka, 1.0f, g);
    store_row<D>(to + a.rows * D, dva, 1.0f, g);
  } else {
    store_row<D>(dk + kj * D, dka, a.scale, g);
    store_row<D>(dv + kj * D, dva, a.kept_scale, g);
  }
}

// What the kernels read besides the call's arrays, made by one launch: small calls
// are bound by their launches (2 heads x 256 tokens, d = 64: prepared in four, 13
// us; in one, 4 us).  A block has one of the roles below, in this order.
struct Prepare {
  int heads, n, c_q;
  int list_blocks, mask_blocks, word_blocks;  // the statistics' blocks come last
  const int32_t *offsets, *sel_counts, *sel_idx;
  // lists of work items of rows[i] queries
  int4 *items[2];
  int rows[2], per_head[2], stride[2];  // stride 2: work slots of one chunk
  uint32_t *masks;
  KeyOrder order;  // its costs are cleared
  int32_t *status;
  const uint64_t *rng;
  uint32_t *words;
  const void *o, *d_o;
  const float *lse;
  float *stats;
};

// Work items of `rows` queries of head h: the chunks of every cluster in cluster
// order as (cluster, first row, rows, selected keys), then empty ones.
__device__ void prepare_items(const Prepare &p, int h, int rows, int per_head, int stride, int4 *items) {
  constexpr int PER = kTrainMaxClusters / 256;
  __shared__ int first[kTrainMaxClusters + 1];
  __shared__ int wtot[4];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int32_t *off = p.offsets + static_cast<size_t>(h) * (p.c_q + 1);
  auto count_of = [&](int c) { return min(max(off[c + 1] - off[c], 0), p.n); };
  int k[PER], mine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    k[i] = PER * t + i < p.c_q ? (count_of(PER * t + i) + rows - 1) / rows : 0;
    mine += k[i];
  }
  const int incl = wave_incl_scan(mine);
  if (lane == 63) wtot[w] = incl;
  __syncthreads();
  int at = incl - mine;
  for (int i = 0; i < w; ++i) at += wtot[i];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    first[PER * t + i] = at;  // clusters past c_q: the total
    at += k[i];
  }
  if (t == 255) first[kTrainMaxClusters] = at;
  __syncthreads();
  const int total = first[p.c_q];
  for (int slot = t; slot < per_head; slot += 256) {
    int4 it = make_int4(0, 0, 0, 0);
    if (slot < total) {
      int lo = 0, hi = p.c_q;  // first[lo] <= slot < first[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= slot) lo = mid; else hi = mid;
      }
      const int row0 = (slot - first[lo]) * rows;
      it = make_int4(lo, row0, min(rows, count_of(lo) - row0),
                     min(max(p.sel_counts[static_cast<size_t>(h) * p.c_q + lo], 0), p.n));
    }
    int4 *to = items + (static_cast<size_t>(h) * per_head + slot) * stride;
    to[0] = it;
    if (stride == 2) to[1] = make_int4(0, 0, 0, 0);
  }
}

// Key bits: masks[head][key / 256][cluster][8 words].  A block turns the part of one
// cluster's list with keys in [from, from + 8192) into bits in LDS; a list that is
// not strictly ascending or leaves [0, n) is reported, and its bits are those that
// the search finds.
constexpr int kMaskKeys = 32 * 256;  // a word per thread
__device__ void prepare_masks(const Prepare &p, int h, int c, int from, int segments) {
  __shared__ uint32_t bits[256];
  const int t = threadIdx.x, n = p.n;
  const int r = min(max(p.sel_counts[static_cast<size_t>(h) * p.c_q + c], 0), n);
  const int32_t *sel = p.sel_idx + (static_cast<size_t>(h) * p.c_q + c) * n;
  const int to = min(from + kMaskKeys, n);
  bits[t] = 0;
  auto below = [&](int x) {  // entries below x, 64 places of the list at a time
    int lo = 0, hi = r;
    while (lo < hi) {
      const int step = (hi - lo + 63) / 64, at = lo + step * (t & 63) + step - 1;
      const int less = __popcll(__ballot(at < hi && sel[min(at, hi - 1)] < x));
      lo = min(lo + step * less, hi);
      hi = step == 1 ? lo : min(lo + step - 1, hi);
    }
    return lo;
  };
  const int lo = segments == 1 ? 0 : below(from), hi = segments == 1 ? r : below(to);
  __syncthreads();
  // A bound between two segments is found alike for both, so their ranges cover
  // [below(0), below(n)) whatever the list holds: every entry of a bad list is seen.
  bool bad = lo > 0 && from == 0;
  bad = bad || (hi < r && to == n);
  for (int e0 = lo + 8 * t; e0 < hi; e0 += 8 * 256) {
    // eight neighbours per thread: most fall into one word, set at once
    int before = e0 > 0 ? sel[e0 - 1] : -1, word = 0, j[8];
    uint32_t acc = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) j[i] = sel[min(e0 + i, hi - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (e0 + i >= hi) break;
      const bool here = j[i] >= from && j[i] < to;
      bad = bad || !here || j[i] <= before;
      before = j[i];
      if (!here) continue;
      const int at = (j[i] - from) >> 5;
      if (at != word) {
        if (acc) atomicOr(&bits[word], acc);
        word = at;
        acc = 0;
      }
      acc |= 1u << (j[i] & 31);
    }
    if (acc) atomicOr(&bits[word], acc);
  }
  if (bad && p.status) atomicOr(p.status, kStatusBadSet);
  __syncthreads();
  constexpr int WORDS = kTrainMaskKeys / 32;
  const int blocks = (n + kTrainMaskKeys - 1) / kTrainMaskKeys, b = from / kTrainMaskKeys + t / WORDS;
  if (b < blocks) p.masks[((static_cast<size_t>(h) * blocks + b) * p.c_q + c) * WORDS + t % WORDS] = bits[t];
}

// The rows' statistics for the gradients: (-lse in the exp2 domain, <do, o>).
// A row without keys has lse = -inf: its probabilities are exp2(-inf) = 0.  Row n
// of a head is one of no weight, for the rows that fill up a tile.
template <typename T, int D>
__device__ void prepare_stats(const Prepare &p, size_t block) {
  constexpr int PER = 16 / sizeof(T), LANES = D / PER;
  const T *o = static_cast<const T *>(p.o), *d_o = static_cast<const T *>(p.d_o);
  const size_t i = (block * 256 + threadIdx.x) / LANES, n = p.n;
  const int x = threadIdx.x % LANES;
  if (i >= p.heads * n) return;  // whole groups of LANES
  const uint4 vo = reinterpret_cast<const uint4 *>(o)[i * LANES + x], vg = reinterpret_cast<const uint4 *>(d_o)[i * LANES + x];
  const uint32_t a[4] = {vo.x, vo.y, vo.z, vo.w}, b[4] = {vg.x, vg.y, vg.z, vg.w};
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) {
      s = fmaf(__uint_as_float(a[e] << 16), __uint_as_float(b[e] << 16), s);
      s = fmaf(__uint_as_float(a[e] & 0xFFFF0000u), __uint_as_float(b[e] & 0xFFFF0000u), s);
    } else {
      s = fmaf(__uint_as_float(a[e]), __uint_as_float(b[e]), s);
    }
  }
#pragma unroll
  for (int k = LANES / 2; k > 0; k /= 2) s += __shfl_xor(s, k, LANES);
  if (x) return;
  float *head = p.stats + i / n * 2 * (n + 1);
  head[i % n] = p.lse[i] == -INFINITY ? -INFINITY : -p.lse[i] * kLog2e;
  head[n + 1 + i % n] = s;
  if (i % n == 0) {
    head[n] = -INFINITY;
    head[2 * n + 1] = 0.0f;
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void train_prepare_kernel(Prepare p) {
  int b = static_cast<int>(blockIdx.x);
  if (b < p.list_blocks) {
    const int i = b / p.heads;
    if (i == 0 && p.order.cost) {
      const int h = b % p.heads;
      if (threadIdx.x < 2 * kOrderSlots) p.order.cost[static_cast<size_t>(h) * 2 * kOrderSlots + threadIdx.x] = 0;
    }
    prepare_items(p, b % p.heads, p.rows[i], p.per_head[i], p.stride[i], p.items[i]);
    return;
  }
  b -= p.list_blocks;
  if (b < p.mask_blocks) {
    const int segments = (p.n + kMaskKeys - 1) / kMaskKeys, hc = b / segments;
    prepare_masks(p, hc / p.c_q, hc % p.c_q, b % segments * kMaskKeys, segments);
    return;
  }
  b -= p.mask_blocks;
  if (b < p.word_blocks) {  // dropout's words: of the queries, then of the keys, per head
    const int per = (p.n + 255) / 256, h = b / per / 2, side = b / per % 2, i = b % per * 256 + threadIdx.x;
    if (i >= p.n) return;
    const uint2 x = pair_word(Stream(p.rng), i, h, side);
    uint32_t *at = p.words + (4 * static_cast<size_t>(h) + 2 * side) * p.n + i;
    at[0] = x.x;
    at[p.n] = x.y;
    return;
  }
  prepare_stats<T, D>(p, static_cast<size_t>(b - p.word_blocks));
}

// The parts' sums in part order, scaled and rounded once.
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(size_t count, int splits, float scale_k, float scale_v,
                                                         const float *__restrict__ parts, T *dk, T *dv) {
  const size_t i = 4 * (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x);
  if (i >= count) return;
  const int v = blockIdx.y;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int p = 0; p < splits; ++p) {
    const float4 x = *reinterpret_cast<const float4 *>(parts + (2 * static_cast<size_t>(p) + v) * count + i);
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  const float f = v ? scale_v : scale_k;
  T *at = (v ? dv : dk) + i;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2 *>(at) = make_uint2(pack_bf16(s.x * f, s.y * f), pack_bf16(s.z * f, s.w * f));
  else
    *reinterpret_cast<float4 *>(at) = make_float4(s.x * f, s.y * f, s.z * f, s.w * f);
}

// O and lse, or dQ, from the parts' sums.  A group of D / 4 lanes per query, in the
// clusters' order: queries in no cluster are left as they were.
template <typename T, int D, bool GRAD>
__global__ __launch_bounds__(256) void join_queries_kernel(TrainArgs a, T *out) {
  constexpr int LANES = D / 4;
  const int h = blockIdx.y, pos = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, x = threadIdx.x % LANES;
  const size_t first = static_cast<size_t>(h) * a.n;
  const int32_t *off = a.offsets + static_cast<size_t>(h) * (a.c_q + 1);
  if (pos < off[0] || pos >= min(off[a.c_q], a.n)) return;
  const size_t row = first + min(max(a.perm[first + pos], 0), a.n - 1);
  const float2 *ml = reinterpret_cast<const float2 *>(a.parts + a.splits * a.rows * D);
  float top = 0.0f, l = 0.0f, f = a.scale;
  if constexpr (!GRAD) {
    top = -INFINITY;
    for (int p = 0; p < a.splits; ++p) top = fmaxf(top, ml[p * a.rows + row].x);
    if (top == -INFINITY) top = 0.0f;
    for (int p = 0; p < a.splits; ++p) {
      const float2 s = ml[p * a.rows + row];
      l = fmaf(s.y, __builtin_amdgcn_exp2f(s.x - top), l);
    }
    f = l > 0.0f ? a.kept_scale / l : 0.0f;
    if (x == 0) a.lse[row] = l > 0.0f ? (top + __log2f(l)) * kLn2 : l == 0.0f ? -INFINITY : l;
  }
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int p = 0; p < a.splits; ++p) {
    const float4 v = *reinterpret_cast<const float4 *>(a.parts + (p * a.rows + row) * D + 4 * x);
    const float w = GRAD ? 1.0f : __builtin_amdgcn_exp2f(ml[p * a.rows + row].x - top);
    s.x = fmaf(v.x, w, s.x);
    s.y = fmaf(v.y, w, s.y);
    s.z = fmaf(v.z, w, s.z);
    s.w = fmaf(v.w, w, s.w);
  }
  T *to = out + row * D + 4 * x;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(s.x * f, s.y * f), pack_bf16(s.z * f, s.w * f));
  else
    *reinterpret_cast<float4 *>(to) = make_float4(s.x * f, s.y * f, s.z * f, s.w * f);
}

template <typename K, typename... A>
hipError_t launch(K kernel, dim3 grid, int threads, hipStream_t s, A... args) {
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, args...);
  return hipGetLastError();
}

#define TRAIN_TRY(x)                     \
  do {                                   \
    const hipError_t e_ = (x);           \
    if (e_ != hipSuccess) return e_;     \
  } while (0)

template <typename T>
hipError_t join_parts(size_t count, int splits, float scale_k, float scale_v, const float *parts, T *dk, T *dv, hipStream_t s) {
  return launch(join_parts_kernel<T>, dim3(static_cast<unsigned>((count / 4 + 255) / 256), 2), 256, s, count, splits, scale_k,
                scale_v, parts, dk, dv);
}

// Parts that each block's tiles are cut into, with fp32 sums of their own that a
// second kernel adds: as many, up to 16 of `least` tiles or more, as make the
// launch's rounds shortest; a part costs about 4% of a block more (its start, its
// sums).  `resident`: the blocks that the chip is taken to hold at once.  3 heads x 2185
// tokens, d = 128: dq in parts 43 us and their join 5, dk and dv 47 and 10; calls whose
// blocks fill the chip many times stay whole or take few parts.
int parts_of(long long blocks, long long tiles, int least, int resident) {
  constexpr int kMost = 16;
  int best = 1;
  double shortest = 0.0;
  for (int s = 1; s <= kMost && (s == 1 || s * least <= tiles); ++s) {
    const double rounds = static_cast<double>((blocks * s + resident - 1) / resident) * (1.0 / s + 0.04);
    if (s == 1 || rounds < shortest) {
      shortest = rounds;
      best = s;
    }
  }
  return best;
}
// grad: masks and statistics too.
template <typename T, int D>
hipError_t prepare(const TrainArgs &a, const TrainCall &c, bool grad, hipStream_t s) {
  Prepare p{};
  p.heads = c.heads;
  p.n = a.n;
  p.c_q = a.c_q;
  p.offsets = a.offsets;
  p.sel_counts = a.sel_counts;
  p.sel_idx = a.sel_idx;
  int lists = 0;
  auto list = [&](int4 *items, int rows, int stride) {
    p.items[lists] = items;
    p.rows[lists] = rows;
    p.stride[lists] = stride;
    p.per_head[lists++] = train_items_per_head(a.n, a.c_q, rows);
  };
  if (sizeof(T) == 4) list(c.items, kRows, 1);
  else if (train_lists_slots(c.heads, a.n, a.c_q)) list(c.slots.items, kBM, 2);
  if (grad) list(c.tiles, sizeof(T) == 4 ? kTile : kTrainKeyTile, 1);
  p.list_blocks = lists * c.heads;
  p.word_blocks = a.drop ? 2 * c.heads * ((a.n + 255) / 256) : 0;
  p.rng = c.rng;
  p.words = const_cast<uint32_t *>(a.words);
  size_t stats = 0;
  if (grad) {
    p.mask_blocks = c.heads * a.c_q * ((a.n + kMaskKeys - 1) / kMaskKeys);
    p.masks = const_cast<uint32_t *>(a.masks);
    p.order = a.order;
    p.status = c.status;
    p.o = c.o;
    p.d_o = a.d_o;
    p.lse = a.lse;
    p.stats = const_cast<float *>(a.stats);
    stats = (a.rows * (D * sizeof(T) / 16) + 255) / 256;
  }
  const size_t blocks = p.list_blocks + static_cast<size_t>(p.mask_blocks) + p.word_blocks + stats;
  if (!blocks) return hipSuccess;
  return launch(train_prepare_kernel<T, D>, dim3(static_cast<unsigned>(blocks)), 256, s, p);
}

// The kernels by queries, and where they ran in parts the join.
template <typename T, int D>
hipError_t queries(TrainArgs a, const TrainCall &c, bool grad, T *out, hipStream_t s) {
  a.splits = train_query_parts(c.heads, a.n, D, sizeof(T) == 2, a.c_q);
  if constexpr (sizeof(T) == 2) {
    TRAIN_TRY(train_queries(D, grad, a, c.heads, train_lists_slots(c.heads, a.n, a.c_q), c.slots, out, s));
  } else {
    a.items = c.items;
    a.items_per_head = train_items_per_head(a.n, a.c_q, kRows);
    const dim3 grid(static_cast<unsigned>(c.heads) * a.items_per_head * a.splits);
    if (grad)
      TRAIN_TRY(a.drop ? launch(train_queries_kernel<D, true, true>, grid, kThreads, s, a, out)
                       : launch(train_queries_kernel<D, true, false>, grid, kThreads, s, a, out));
    else
      TRAIN_TRY(a.drop ? launch(train_queries_kernel<D, false, true>, grid, kThreads, s, a, out)
                       : launch(train_queries_kernel<D, false, false>, grid, kThreads, s, a, out));
  }
  if (a.splits == 1) return hipSuccess;
  const dim3 grid((a.n + 1024 / D - 1) / (1024 / D), c.heads);
  return grad ? launch(join_queries_kernel<T, D, true>, grid, 256, s, a, out)
              : launch(join_queries_kernel<T, D, false>, grid, 256, s, a, out);
}

template <typename T, int D>
hipError_t forward(const TrainArgs &a, const TrainCall &c, hipStream_t s) {
  TRAIN_TRY((prepare<T, D>(a, c, false, s)));
  return queries<T, D>(a, c, false, static_cast<T *>(c.o), s);
}

template <typename T, int D>
hipError_t backward(TrainArgs a, const TrainCall &c, hipStream_t s) {
  TRAIN_TRY((prepare<T, D>(a, c, true, s)));
  TRAIN_TRY((queries<T, D>(a, c, true, static_cast<T *>(c.dq), s)));
  T *dk = static_cast<T *>(c.dk), *dv = static_cast<T *>(c.dv);
  a.items = c.tiles;
  a.items_per_head = train_items_per_head(a.n, a.c_q, sizeof(T) == 2 ? kTrainKeyTile : kTile);
  a.splits = train_key_parts(c.heads, a.n, sizeof(T) == 2, a.c_q);
  if (a.order.cost) TRAIN_TRY(train_order(a, c.heads, s));
  if constexpr (sizeof(T) == 2) {
    TRAIN_TRY(train_keys(D, a, c.heads, dk, dv, s));
  } else {
    const dim3 grid(static_cast<unsigned>(c.heads) * a.splits * ((a.n + kRows - 1) / kRows));
    TRAIN_TRY(a.drop ? launch(train_keys_kernel<D, true>, grid, kThreads, s, a, dk, dv)
                     : launch(train_keys_kernel<D, false>, grid, kThreads, s, a, dk, dv));
  }
  return a.splits > 1 ? join_parts(a.rows * D, a.splits, a.scale, a.kept_scale, a.parts, dk, dv, s) : hipSuccess;
}

}  // namespace

// Two blocks a CU.  At d = 64 the chip holds three (bf16 with dropout two), which was
// not measured here.
int train_key_parts(int heads, int n, bool bf16, int c_q) {
  const int keys = bf16 ? kTrainKeyBlock : kRows, tile = bf16 ? kTrainKeyTile : kTile;
  return parts_of(static_cast<long long>(heads) * ((n + keys - 1) / keys), train_items_per_head(n, c_q, tile), 2,
                  512);
}
// The lists are on the device: clusters of a block's queries or fewer are taken to
// fill a block each, larger ones half a block more than their queries do, and every
// key to be selected.  Blocks a CU: bf16 one (d = 64: two, though with dropout the
// chip holds one), fp32 two (though at d = 64 it holds four).
int train_query_parts(int heads, int n, int d, bool bf16, int c_q) {
  const int rows = bf16 ? kBM : kRows, tile = bf16 ? kBN : kTile;
  const long long chunks = n / rows + c_q / 2 > c_q ? n / rows + (c_q + 1) / 2 : c_q;
  const int resident = bf16 && d == 128 ? 256 : 512;
  // a block order of its own fills the chip better, where there are the blocks
  if (bf16 && 2 * heads * chunks > resident && attention_ordered(heads, n, d, c_q)) return 1;
  return parts_of(heads * chunks, n / tile, 4, resident);
}
// Whether the work slots of a bf16 call are listed with the rest: chunks alone, in
// cluster order.  With so few no slots share a block and their order matters little.
bool train_lists_slots(int heads, int n, int c_q) {
  return static_cast<long long>(heads) * attn_items_per_head(n, c_q) <= 256;
}

bool train_launchable(int heads, int n, int d, bool bf16, int c_q) {
  const uint64_t H = heads, chunks = bf16 ? attn_items_per_head(n, c_q) : train_items_per_head(n, c_q, kRows);
  const uint64_t prepared = 2 * H + H * c_q * ((n + kMaskKeys - 1) / kMaskKeys) + 2 * H * ((n + 255) / 256) +
                            (H * n * d * (bf16 ? 2 : 4) / 16 + 255) / 256;
  const uint64_t keys = H * ((n + 63) / 64);
  return prepared * 256 < (1ull << 32) && H * chunks * (bf16 ? 64 * kNW : kThreads) < (1ull << 32) && keys * 256 < (1ull << 32);
}

int train_items_per_head(int n, int c_q, int rows) { return (n + rows - 1) / rows + c_q; }

size_t train_workspace(int heads, int n, int d, bool bf16, int c_q, void *base, TrainArgs *a, TrainCall *c) {
  size_t used = 0;
  auto take = [&](size_t bytes) {
    char *p = base ? static_cast<char *>(base) + used : nullptr;
    used += (bytes + 255) / 256 * 256;
    return p;
  };
  const size_t H = heads;
  const size_t slots = bf16 ? 2 * H * attn_items_per_head(n, c_q) : H * train_items_per_head(n, c_q, kRows);
  char *items = take(slots * sizeof(int4));
  const bool ordered = bf16 && attention_ordered(heads, n, d, c_q);
  char *order = take(ordered ? attention_order_entries(heads, n, d, c_q) * sizeof(int2) : 0);
  char *tiles = take(H * train_items_per_head(n, c_q, bf16 ? kTrainKeyTile : kTile) * sizeof(int4));
  char *words = take(H * n * 4 * sizeof(uint32_t));
  char *stats = take(H * (n + 1) * 2 * sizeof(float));
  const size_t mask_bytes = H * ((n + kTrainMaskKeys - 1) / kTrainMaskKeys) * c_q * (kTrainMaskKeys / 8);
  char *masks = take(mask_bytes);
  const size_t ordered_keys = train_orders_keys(n, c_q) ? 1 : 0;
  char *bin = take(ordered_keys * H * n * sizeof(uint16_t));
  char *start = take(ordered_keys * H * ((n + kOrderKeys - 1) / kOrderKeys) * kOrderBins * sizeof(uint32_t));
  char *key = take(ordered_keys * H * n * sizeof(int32_t));
  char *by_position = take(ordered_keys * mask_bytes);
  char *cost = take(ordered_keys * H * 2 * kOrderSlots * sizeof(unsigned long long));
  const size_t sk = train_key_parts(heads, n, bf16, c_q), sq = train_query_parts(heads, n, d, bf16, c_q);
  const size_t by_keys = sk > 1 ? 2 * sk * d : 0, by_queries = sq > 1 ? sq * (d + 2) : 0;
  char *parts = take(H * n * (by_keys > by_queries ? by_keys : by_queries) * sizeof(float));
  if (a) {
    a->words = reinterpret_cast<uint32_t *>(words);
    a->stats = reinterpret_cast<float *>(stats);
    a->masks = reinterpret_cast<uint32_t *>(masks);
    a->parts = reinterpret_cast<float *>(parts);
    if (ordered_keys)
      a->order = {reinterpret_cast<uint16_t *>(bin), reinterpret_cast<uint32_t *>(start), reinterpret_cast<int32_t *>(key),
                  reinterpret_cast<uint32_t *>(by_position), reinterpret_cast<unsigned long long *>(cost)};
    c->items = c->slots.items = reinterpret_cast<int4 *>(items);
    c->slots.order = ordered ? reinterpret_cast<int2 *>(order) : nullptr;
    c->tiles = reinterpret_cast<int4 *>(tiles);
  }
  return used;
}

hipError_t train_forward(int d, bool bf16, const TrainArgs &a, const TrainCall &c, hipStream_t s) {
  if (bf16) return d == 128 ? forward<uint16_t, 128>(a, c, s) : forward<uint16_t, 64>(a, c, s);
  return d == 128 ? forward<float, 128>(a, c, s) : forward<float, 64>(a, c, s);
}

hipError_t train_backward(int d, bool bf16, const TrainArgs &a, const TrainCall &c, hipStream_t s) {
  if (bf16) return d == 128 ? backward<uint16_t, 128>(a, c, s) : backward<uint16_t, 64>(a, c, s);
  return d == 128 ? backward<float, 128>(a, c, s) : backward<float, 64>(a, c, s);
}

}  // namespace scope
