// Attention over the selected keys for training: the forward with the rows'
// log-sum-exp and dropout, and the gradients (Eq. 11; dense attention, Eq. 1, is
// the one-cluster special case).  With S_c the keys of query i's cluster c,
//   s_ij = <q_i, k_j>, p_ij = exp(scale s_ij - lse_i), m_ij the dropout factor,
//   o_i   = sum_j p_ij m_ij v_j
//   dp_ij = m_ij <do_i, v_j>,  ds_ij = p_ij (dp_ij - <do_i, o_i>)
//   dq_i  = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i,
//   dv_j  = sum_i p_ij m_ij do_i
// The gradients recompute p from lse, so nothing of size n^2 is stored.  dq runs
// over a cluster's gathered keys like the forward, one wave per 32 queries; dk
// and dv run over the clusters' queries, one wave per 32 keys, with a bit for
// each (cluster, key), so every sum has one owner and a fixed order: no atomics,
// the same bits on every run.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "mfma.h"
#include "noise.h"

namespace scope {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kThreads = 256;               // four waves
constexpr int kRows = 32 * kThreads / 64;   // rows (queries or keys) per block
constexpr int kTile = 32;                   // gathered rows per step

// A wave's 32 x 32 matrix product in the tensors' type: bf16 operands of 16
// channels per instruction, or fp32 operands (no rounding) of four times two.
template <typename T>
struct Mma;
template <>
struct Mma<uint16_t> {
  typedef bf16x8 Frag;
  static constexpr int kLane = 8;  // channels per lane and fragment
  static constexpr int kPad = 32;
  static __device__ __forceinline__ void product(f32x16 &acc, Frag a, Frag b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
  }
};
template <>
struct Mma<float> {
  typedef float4 Frag;
  static constexpr int kLane = 4;
  static constexpr int kPad = 4;
  static __device__ __forceinline__ void product(f32x16 &acc, Frag a, Frag b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, b.x, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, b.y, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, b.z, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, b.w, acc, 0, 0, 0);
  }
};

// Tile of kTile rows in LDS, and the two products that read it.
template <typename T, int D>
struct Tile {
  typedef typename Mma<T>::Frag Frag;
  static constexpr int kStride = D + Mma<T>::kPad;
  static constexpr int kSteps = D / (2 * Mma<T>::kLane);
  T x[kTile * kStride];

  // this lane's fragments of a row of a tensor (zeros where there is none)
  static __device__ __forceinline__ void fragments(Frag (&f)[kSteps], const T *row, bool valid, int hf) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      f[s] = valid ? *reinterpret_cast<const Frag *>(row + Mma<T>::kLane * (2 * s + hf)) : Frag{};
  }
  // tile . columns^T: element e of a lane is row 8 (e / 4) + 4 hf + e % 4 of its column
  __device__ __forceinline__ f32x16 scores(const Frag (&f)[kSteps], int l32, int hf) const {
    f32x16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      Mma<T>::product(acc, *reinterpret_cast<const Frag *>(&x[l32 * kStride + Mma<T>::kLane * (2 * s + hf)]), f[s]);
    return acc;
  }
};

// out += tile^T . w, w in the layout of scores()
template <int D>
__device__ __forceinline__ void accumulate_tile(const Tile<uint16_t, D> &t, f32x16 (&out)[D / 32],
                                                const float (&w)[16], int lane) {
  constexpr int S = Tile<uint16_t, D>::kStride;
  // transposing reads, as the forward attention's V: row 4 (lane / 32) +
  // (lane % 16) / 4 of a 16-row step, channels 16 ((lane / 16) % 2) + 4 (lane % 4)
  const int at = (4 * (lane >> 5) + ((lane & 15) >> 2)) * S + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
    const bf16x8 b = as_bf16x8(make_uint4(pack_bf16(w[8 * s2 + 0], w[8 * s2 + 1]), pack_bf16(w[8 * s2 + 2], w[8 * s2 + 3]),
                                          pack_bf16(w[8 * s2 + 4], w[8 * s2 + 5]), pack_bf16(w[8 * s2 + 6], w[8 * s2 + 7])));
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const uint16_t *p = &t.x[16 * s2 * S + 32 * db + at];
      const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(p)));
      const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(p + 8 * S)));
      out[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y)), b, out[db], 0, 0, 0);
    }
  }
}
template <int D>
__device__ __forceinline__ void accumulate_tile(const Tile<float, D> &t, f32x16 (&out)[D / 32],
                                                const float (&w)[16], int lane) {
  const int l32 = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int e = 0; e < 16; ++e)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      out[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(
          t.x[(8 * (e >> 2) + 4 * hf + (e & 3)) * Tile<float, D>::kStride + 32 * db + l32], w[e], out[db], 0, 0, 0);
}

// 16 bytes of a row, `valid` or zeros.
template <typename T>
__device__ __forceinline__ uint4 row_chunk(const T *base, size_t row, int d, int chunk, bool valid) {
  return valid ? *reinterpret_cast<const uint4 *>(base + row * d + chunk * (16 / sizeof(T))) : make_uint4(0, 0, 0, 0);
}

// A lane's 16 rows of D x 32 results times `f`, into the row of its column.
template <typename T, int D>
__device__ __forceinline__ void store_column(T *row, const f32x16 (&acc)[D / 32], float f, int hf) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T *at = row + 32 * db + 8 * i + 4 * hf;
      const float a = acc[db][4 * i] * f, b = acc[db][4 * i + 1] * f, c = acc[db][4 * i + 2] * f, d = acc[db][4 * i + 3] * f;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2 *>(at) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
      else
        *reinterpret_cast<float4 *>(at) = make_float4(a, b, c, d);
    }
}

__device__ __forceinline__ int row_of(int e, int hf) { return 8 * (e >> 2) + 4 * hf + (e & 3); }

// One wave per 32 queries of a cluster, over the cluster's keys: the forward
// (GRAD false) or dq (GRAD true).
template <typename T, int D, bool GRAD, bool DROP>
__global__ __launch_bounds__(kThreads) void train_queries_kernel(TrainArgs a, T *out) {
  typedef Tile<T, D> TileT;
  constexpr int CH = D * sizeof(T) / 16;              // 16-byte chunks of a row
  constexpr int PER = kTile * CH / kThreads;          // of each tile per thread
  static_assert(kTile * CH % kThreads == 0, "tile/threads mismatch");
  __shared__ __attribute__((aligned(16))) TileT K, V;
  __shared__ uint2 words[kTile];
  const int4 it = a.items[blockIdx.x];
  const int h = static_cast<int>(blockIdx.x) / a.items_per_head;
  const int c = it.x, row0 = it.y, rows = it.z, r = it.w;
  if (rows <= 0) return;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, l32 = lane & 31, hf = lane >> 5;
  const size_t first = static_cast<size_t>(h) * a.n;
  const T *k = static_cast<const T *>(a.k) + first * D, *v = static_cast<const T *>(a.v) + first * D;
  const int ql = 32 * w + l32;
  const bool valid = ql < rows;
  size_t qi = first;
  if (valid) {
    const int pos = min(max(a.offsets[static_cast<size_t>(h) * (a.c_q + 1) + c] + row0 + ql, 0), a.n - 1);
    qi += min(max(a.perm[first + pos], 0), a.n - 1);
  }
  typename TileT::Frag qf[TileT::kSteps], gf[GRAD ? TileT::kSteps : 1];
  TileT::fragments(qf, static_cast<const T *>(a.q) + qi * D, valid, hf);
  float neg_lse = -INFINITY, delta = 0.0f;
  if constexpr (GRAD) {
    TileT::fragments(gf, static_cast<const T *>(a.d_o) + qi * D, valid, hf);
    if (valid) {
      const float *st = a.stats + 2 * h * static_cast<size_t>(a.n + 1) + (qi - first);
      neg_lse = st[0];
      delta = st[a.n + 1];
    }
  }
  uint2 mine = make_uint2(0, 0);
  const uint32_t *wq = a.words + 4 * first, *wk = wq + 2 * static_cast<size_t>(a.n);
  if (DROP && valid) mine = make_uint2(wq[qi - first], wq[qi - first + a.n]);
  f32x16 acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  const int32_t *sel = a.sel_idx + (static_cast<size_t>(h) * a.c_q + c) * a.n;
  for (int k0 = 0; k0 < r; k0 += kTile) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = i * kThreads + t, row = at / CH, chunk = at % CH;
      const bool in = k0 + row < r;
      const int j = in ? min(max(sel[k0 + row], 0), a.n - 1) : 0;
      *reinterpret_cast<uint4 *>(&K.x[row * TileT::kStride + chunk * (16 / sizeof(T))]) = row_chunk(k, j, D, chunk, in);
      *reinterpret_cast<uint4 *>(&V.x[row * TileT::kStride + chunk * (16 / sizeof(T))]) = row_chunk(v, j, D, chunk, in);
      if (DROP && chunk == 0) words[row] = make_uint2(wk[j], wk[j + a.n]);
    }
    __syncthreads();
    const f32x16 s = K.scores(qf, l32, hf);
    float p[16];
    if constexpr (!GRAD) {
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = k0 + row_of(e, hf) < r ? s[e] : -INFINITY;
        top = fmaxf(top, p[e]);
      }
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top * a.scale_log2);
      const float neg = m_new == -INFINITY ? 0.0f : -m_new;
      const float alpha = __builtin_amdgcn_exp2f(m + neg);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] *= alpha;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], a.scale_log2, neg));
        l += p[e];
        if (DROP && !pair_kept(mine, words[row_of(e, hf)], a.drop)) p[e] = 0.0f;
      }
      accumulate_tile<D>(V, acc, p, lane);
    } else {
      const f32x16 dp = V.scores(gf, l32, hf);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float g = dp[e];
        if (DROP) g = pair_kept(mine, words[row_of(e, hf)], a.drop) ? g * a.kept_scale : 0.0f;
        const float pe = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, neg_lse));
        p[e] = k0 + row_of(e, hf) < r ? pe * (g - delta) : 0.0f;
      }
      accumulate_tile<D>(K, acc, p, lane);
    }
  }
  if constexpr (!GRAD) {
    l += __shfl_xor(l, 32);
    if (!valid) return;
    store_column<T, D>(out + qi * D, acc, l > 0.0f ? a.kept_scale / l : 0.0f, hf);
    if (hf == 0) a.lse[qi] = l > 0.0f ? (m + __log2f(l)) * kLn2 : l == 0.0f ? -INFINITY : l;
  } else {
    if (!valid) return;
    store_column<T, D>(out + qi * D, acc, a.scale, hf);
  }
}

// One wave per 32 keys, over the queries of every cluster that keeps any of the
// block's keys: dk and dv.
template <typename T, int D, bool DROP>
__global__ __launch_bounds__(kThreads) void train_keys_kernel(TrainArgs a, T *dk, T *dv) {
  typedef Tile<T, D> TileT;
  constexpr int CH = D * sizeof(T) / 16;
  constexpr int PER = kTile * CH / kThreads;
  __shared__ __attribute__((aligned(16))) TileT Q, G;
  __shared__ float2 stats[kTile];
  __shared__ uint2 words[kTile];
  const int blocks = (a.n + kRows - 1) / kRows;
  const int h = static_cast<int>(blockIdx.x) / blocks, b = static_cast<int>(blockIdx.x) % blocks;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, l32 = lane & 31, hf = lane >> 5;
  const size_t first = static_cast<size_t>(h) * a.n;
  const T *q = static_cast<const T *>(a.q), *g = static_cast<const T *>(a.d_o);
  const int j = b * kRows + 32 * w + l32;
  const bool valid = j < a.n;
  const size_t kj = first + (valid ? j : 0);
  typename TileT::Frag kf[TileT::kSteps], vf[TileT::kSteps];
  TileT::fragments(kf, static_cast<const T *>(a.k) + kj * D, valid, hf);
  TileT::fragments(vf, static_cast<const T *>(a.v) + kj * D, valid, hf);
  uint2 mine = make_uint2(0, 0);
  const uint32_t *wq = a.words + 4 * first, *wk = wq + 2 * static_cast<size_t>(a.n);
  if (DROP) mine = make_uint2(wk[kj - first], wk[kj - first + a.n]);
  f32x16 dka[D / 32], dva[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) dka[db][e] = dva[db][e] = 0.0f;
  // the block's four words of each cluster, one per wave
  constexpr int WORDS = kTrainKeyBlock / 32, SHARE = kTrainKeyBlock / kRows;
  const uint32_t *masks = a.masks + (static_cast<size_t>(h) * ((blocks + SHARE - 1) / SHARE) + b / SHARE) * a.c_q * WORDS +
                          kRows / 32 * (b % SHARE);
  for (int i = 0; i < a.items_per_head; ++i) {
    const int4 it = a.items[static_cast<size_t>(h) * a.items_per_head + i];
    const int c = it.x, row0 = it.y, rows = it.z;
    if (rows <= 0) break;
    uint32_t any = 0, own = 0;
    for (int x = 0; x < kRows / 32; ++x) {
      const uint32_t m = masks[c * WORDS + x];
      any |= m;
      if (x == w) own = m;
    }
    if (!any) continue;
    const bool kept = (own >> l32) & 1u;
    const int base = a.offsets[static_cast<size_t>(h) * (a.c_q + 1) + c] + row0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int at = x * kThreads + t, row = at / CH, chunk = at % CH;
      const bool in = row < rows;
      const size_t qi = first + (in ? min(max(a.perm[first + min(max(base + row, 0), a.n - 1)], 0), a.n - 1) : 0);
      *reinterpret_cast<uint4 *>(&Q.x[row * TileT::kStride + chunk * (16 / sizeof(T))]) = row_chunk(q, qi, D, chunk, in);
      *reinterpret_cast<uint4 *>(&G.x[row * TileT::kStride + chunk * (16 / sizeof(T))]) = row_chunk(g, qi, D, chunk, in);
      if (chunk == 0) {
        const float *st = a.stats + 2 * h * static_cast<size_t>(a.n + 1) + (in ? qi - first : a.n);
        stats[row] = make_float2(st[0], st[a.n + 1]);
        if (DROP) words[row] = make_uint2(wq[qi - first], wq[qi - first + a.n]);
      }
    }
    __syncthreads();
    if (!own) continue;
    const f32x16 s = Q.scores(kf, l32, hf), dp = G.scores(vf, l32, hf);
    float p[16], ds[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int row = row_of(e, hf);
      const float2 st = stats[row];
      float pe = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, st.x)), gp = dp[e];
      p[e] = kept ? pe : 0.0f;
      if (DROP) {
        const bool keep = pair_kept(words[row], mine, a.drop);
        gp = keep ? gp * a.kept_scale : 0.0f;
        if (!keep) p[e] = 0.0f;
      }
      ds[e] = kept ? pe * (gp - st.y) : 0.0f;
    }
    accumulate_tile<D>(G, dva, p, lane);
    accumulate_tile<D>(Q, dka, ds, lane);
  }
  if (!valid) return;
  store_column<T, D>(dk + kj * D, dka, a.scale, hf);
  store_column<T, D>(dv + kj * D, dva, a.kept_scale, hf);
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
  int rows[2], per_head[2];
  uint32_t *masks;
  int32_t *status;
  const uint64_t *rng;
  uint32_t *words;
  const void *o, *d_o;
  const float *lse;
  float *stats;
};

// Work items of `rows` queries of head h: the chunks of every cluster in cluster
// order as (cluster, first row, rows, selected keys), then empty ones.
__device__ void prepare_items(const Prepare &p, int h, int rows, int per_head, int4 *items) {
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
    items[static_cast<size_t>(h) * per_head + slot] = it;
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
  auto below = [&](int x) {  // entries below x
    int lo = 0, hi = r;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (sel[mid] < x) lo = mid + 1; else hi = mid;
    }
    return lo;
  };
  const int lo = segments == 1 ? 0 : below(from), hi = segments == 1 ? r : below(to);
  __syncthreads();
  bool bad = false;
  auto check = [&](int e, int j) { bad = bad || j < 0 || j >= n || (e > 0 && sel[e - 1] >= j); };
#pragma unroll 4
  for (int e = lo + t; e < hi; e += 256) {
    const int j = sel[e];
    if (j >= from && j < to) atomicOr(&bits[(j - from) >> 5], 1u << (j & 31));
    if (segments == 1) check(e, j);
  }
  if (segments > 1) {  // entries that no segment's search finds are seen here
#pragma unroll 4
    for (int e = from + t; e < min(to, r); e += 256) check(e, sel[e]);
  }
  if (bad && p.status) atomicOr(p.status, kStatusBadSet);
  __syncthreads();
  constexpr int WORDS = kTrainKeyBlock / 32;
  const int blocks = (n + kTrainKeyBlock - 1) / kTrainKeyBlock, b = from / kTrainKeyBlock + t / WORDS;
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
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < PER; ++e) s = fmaf(load_elem(o, i * D + PER * x + e), load_elem(d_o, i * D + PER * x + e), s);
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
    prepare_items(p, b % p.heads, p.rows[i], p.per_head[i], p.items[i]);
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
  auto list = [&](int4 *items, int rows) {
    p.items[lists] = items;
    p.rows[lists] = rows;
    p.per_head[lists++] = train_items_per_head(a.n, a.c_q, rows);
  };
  if (sizeof(T) == 4) list(c.items, kRows);
  if (grad) list(c.tiles, sizeof(T) == 4 ? kTile : kTrainKeyTile);
  p.list_blocks = lists * c.heads;
  p.word_blocks = a.drop ? 2 * c.heads * ((a.n + 255) / 256) : 0;
  p.rng = c.rng;
  p.words = const_cast<uint32_t *>(a.words);
  size_t stats = 0;
  if (grad) {
    p.mask_blocks = c.heads * a.c_q * ((a.n + kMaskKeys - 1) / kMaskKeys);
    p.masks = const_cast<uint32_t *>(a.masks);
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

template <typename T, int D>
hipError_t forward(TrainArgs a, const TrainCall &c, hipStream_t s) {
  TRAIN_TRY((prepare<T, D>(a, c, false, s)));
  if constexpr (sizeof(T) == 2) {
    return train_queries(D, false, a, c.heads, c.slots, static_cast<T *>(c.o), s);
  } else {
    a.items = c.items;
    a.items_per_head = train_items_per_head(a.n, a.c_q, kRows);
    const dim3 grid(static_cast<unsigned>(c.heads) * a.items_per_head);
    return a.drop ? launch(train_queries_kernel<T, D, false, true>, grid, kThreads, s, a, static_cast<T *>(c.o))
                  : launch(train_queries_kernel<T, D, false, false>, grid, kThreads, s, a, static_cast<T *>(c.o));
  }
}

template <typename T, int D>
hipError_t backward(TrainArgs a, const TrainCall &c, hipStream_t s) {
  TRAIN_TRY((prepare<T, D>(a, c, true, s)));
  T *dq = static_cast<T *>(c.dq), *dk = static_cast<T *>(c.dk), *dv = static_cast<T *>(c.dv);
  if constexpr (sizeof(T) == 2) {
    TRAIN_TRY(train_queries(D, true, a, c.heads, c.slots, dq, s));
    a.items = c.tiles;
    a.items_per_head = train_items_per_head(a.n, a.c_q, kTrainKeyTile);
    return train_keys(D, a, c.heads, train_key_splits(c.heads, a.n, a.c_q), c.parts, dk, dv, s);
  } else {
    a.items = c.items;
    a.items_per_head = train_items_per_head(a.n, a.c_q, kRows);
    const dim3 qgrid(static_cast<unsigned>(c.heads) * a.items_per_head);
    TRAIN_TRY(a.drop ? launch(train_queries_kernel<T, D, true, true>, qgrid, kThreads, s, a, dq)
                     : launch(train_queries_kernel<T, D, true, false>, qgrid, kThreads, s, a, dq));
    a.items = c.tiles;
    a.items_per_head = train_items_per_head(a.n, a.c_q, kTile);
    const dim3 kgrid(static_cast<unsigned>(c.heads) * ((a.n + kRows - 1) / kRows));
    return a.drop ? launch(train_keys_kernel<T, D, true>, kgrid, kThreads, s, a, dk, dv)
                  : launch(train_keys_kernel<T, D, false>, kgrid, kThreads, s, a, dk, dv);
  }
}

}  // namespace

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
  char *masks = take(H * ((n + kTrainKeyBlock - 1) / kTrainKeyBlock) * c_q * (kTrainKeyBlock / 8));
  const int splits = bf16 ? train_key_splits(heads, n, c_q) : 1;
  char *parts = take(splits > 1 ? H * n * d * splits * 2 * sizeof(float) : 0);
  if (a) {
    a->words = reinterpret_cast<uint32_t *>(words);
    a->stats = reinterpret_cast<float *>(stats);
    a->masks = reinterpret_cast<uint32_t *>(masks);
    c->items = c->slots.items = reinterpret_cast<int4 *>(items);
    c->slots.order = ordered ? reinterpret_cast<int2 *>(order) : nullptr;
    c->tiles = reinterpret_cast<int4 *>(tiles);
    c->parts = reinterpret_cast<float *>(parts);
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
