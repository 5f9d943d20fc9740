// The training attention of bf16 inputs by queries: the forward with row statistics
// and dropout, and dQ (attention_train.hip has the formulas, and the kernels for
// fp32).
//
// Work slots and their order, with the costs measured on it, are the inference
// attention's (attention.hip): a block runs up to 256
// queries of a cluster, or of two clusters side by side, a wave 32 of them, over
// the cluster's keys 64 at a time, K and V rows gathered into LDS by the buffer unit
// while the tile before is computed.  The gradient recomputes p from the row's
// log-sum-exp and needs no second pass over the keys:
//   S^T = K_tile . Q^T, dP^T = V_tile . dO^T, ds = p (m dP - D),
//   dQ^T += K_tile^T . ds^T    (ds in two terms, below)
// The forward's normaliser sums the weights in fp32 before they are rounded to bf16
// for the product with V (the inference attention sums the rounded ones): lse is an
// fp32 result, and 2 to 3 keys of weight would leave rounded sums 2^-9 off.
//
// Bound by the matrix pipe and the vector instructions together, 5 heads x 32760,
// 128 clusters, 53% of the keys kept, d = 128: forward 1.56 to 1.84 ms (0.79 to 0.93
// PFLOP/s; matrix pipe 51% busy, vector 51%; the inference attention, which sums the
// rounded weights with the matrix product, 1.54 to 1.57), dQ 2.6 to 2.9 ms (1.0 to
// 1.1 PFLOP/s of its four products; 60% and 49%).  dQ dense, 3 heads x 32760: 2.7 to
// 2.8 ms, 1.2 PFLOP/s.
//
// dQ's ds are two bf16 terms, the second what rounding the first left: a row's ds
// sum to zero, so dQ is a difference of larger sums and keeps more of their rounding
// than dK and dV do.  With one term it was off by 3.2e-3 in the norm where a dQ
// computed in fp32 and rounded once has 1.7e-3; with two it has 1.7e-3.  They take a
// third more matrix products, the whole backward pass 3% (d = 64) to 11% (dense) more
// time.  Taking the rounding's row sum times the mean key out again left 2.8e-3.
#include "attention_slots.h"
#include "attention_tile.h"
#include "common.h"
#include "kernels.h"
#include "noise.h"

namespace scope {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLag = 8.0f;  // the running maximum may lag by 2^8

// Two chunks' tiles; K tiles are followed by the keys' two dropout words (planes of
// kBN), in the same array for the reason given in attention_keys.hip.
template <int D, bool DROP>
struct Tiles {
  static constexpr int kWords = kBN * D;
  static constexpr int kK = kWords + (DROP ? 4 * kBN : 0), kV = kBN * D;
  typedef uint16_t K[2][kK];
  typedef uint16_t V[2][kV];
};

template <int D, bool GRAD, bool DROP, bool PAIRED>
__device__ __forceinline__ void queries_body(const TrainArgs &a, int h, const int4 &ia, const int4 &ib, int part, uint16_t *out,
                                             typename Tiles<D, DROP>::K &K0, typename Tiles<D, DROP>::K &K1,
                                             typename Tiles<D, DROP>::V &V0, typename Tiles<D, DROP>::V &V1) {
  typedef Tiles<D, DROP> T;
  constexpr int CH = D / 8;        // 16-byte chunks per row
  constexpr int RPL = 64 / CH;     // rows per gather load
  constexpr int NG = 8 / RPL;      // gather loads per wave, tile and matrix
  const int t = threadIdx.x, lane = t & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const size_t first = static_cast<size_t>(h) * a.n;
  TileReader<D> at(lane);
  // this wave's chunk: A's ceil(rows / 32) waves first, then B's
  const int wa = (ia.z + 31) >> 5;
  const int g = PAIRED && w >= wa ? 1 : 0;
  const int4 it = g ? ib : ia;
  const int c = it.x, row0 = it.y, rows = it.z, r = it.w;
  const int wl = w - (g ? wa : 0), ql = wl * 32 + l32;
  const bool valid = ql < rows, active = wl * 32 < rows;
  int qi = 0;
  if (valid) {
    const int pos = a.offsets[static_cast<size_t>(h) * (a.c_q + 1) + c] + row0 + ql;
    qi = min(max(a.perm[first + min(max(pos, 0), a.n - 1)], 0), a.n - 1);
  }
  bf16x8 qf[D / 16], gf[GRAD ? D / 16 : 1];
#pragma unroll
  for (int x = 0; x < D / 16; ++x) {
    const size_t from = (first + qi) * D + 16 * x + 8 * hf;
    qf[x] = as_bf16x8(valid ? load8<true>(a.q, from) : make_uint4(0, 0, 0, 0));
    if constexpr (GRAD) gf[x] = as_bf16x8(valid ? load8<true>(a.d_o, from) : make_uint4(0, 0, 0, 0));
  }
  float neg_lse = -INFINITY, delta = 0.0f;
  if (GRAD && valid) {
    const float *st = a.stats + 2 * h * static_cast<size_t>(a.n + 1) + qi;
    neg_lse = st[0];
    delta = st[a.n + 1];
  }
  uint2 mine = make_uint2(0, 0);
  if (DROP && valid) {
    const uint32_t *wq = a.words + 4 * first + qi;
    mine = make_uint2(wq[0], wq[a.n]);
  }

  f32x16 acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.0f;
  float m_run = -INFINITY, l_run = 0.0f;

  // the part's tiles of each chunk's list
  auto tiles_of = [&](int keys) { return ((keys + kBN - 1) / kBN + a.splits - 1) / a.splits; };
  auto begin_of = [&](int keys) { return part * tiles_of(keys); };
  auto count_of = [&](int keys) { return max(min((keys + kBN - 1) / kBN - begin_of(keys), tiles_of(keys)), 0); };
  const int ntA = count_of(ia.w), ntB = PAIRED ? count_of(ib.w) : 0;
  const int ntiles = ntA > ntB ? ntA : ntB, nt_own = count_of(r);
  const int t0A = begin_of(ia.w), t0B = PAIRED ? begin_of(ib.w) : 0, t0_own = begin_of(r);
  auto rsrc = [](const void *p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), static_cast<short>(0), bytes, 0x00020000);
  };
  auto keys_of = [&](const int4 &e) {
    return rsrc(a.sel_idx + (static_cast<size_t>(h) * a.c_q + e.x) * a.n, e.w * 4);
  };
  const __amdgpu_buffer_rsrc_t rselA = keys_of(ia), rselB = PAIRED ? keys_of(ib) : rselA;
  const int nbytes = static_cast<int>(static_cast<uint32_t>(a.n) * (D * 2));
  const __amdgpu_buffer_rsrc_t rk = rsrc(static_cast<const uint16_t *>(a.k) + first * D, nbytes);
  const __amdgpu_buffer_rsrc_t rv = rsrc(static_cast<const uint16_t *>(a.v) + first * D, nbytes);
  // the keys' words: wave 2 chunk + plane brings one plane of a chunk's tile
  const __amdgpu_buffer_rsrc_t rw = rsrc(a.words + 4 * first + (2 + (w & 1)) * static_cast<size_t>(a.n), DROP ? a.n * 4 : 0);

  // gathers: wave w brings rows 8w .. 8w+7 of each chunk's tile, RPL rows (1 KB) per
  // load.  Rows past the end of a key list repeat its last key, with no weight: what
  // no cluster selects is never read.
  struct Idx {
    int a[NG], b[NG], own;
  };
  // one chunk's; a whole tile's rows lie at lane offsets from a scalar one
  auto load_rows = [&](const __amdgpu_buffer_rsrc_t &sel, int count, int tile, int (&rows_of)[NG]) {
    const bool whole = (tile + 1) * kBN <= count;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int row = 8 * w + RPL * i + lane / CH;
      rows_of[i] = whole ? __builtin_amdgcn_raw_buffer_load_b32(sel, row * 4, tile * kBN * 4, 0)
                         : __builtin_amdgcn_raw_buffer_load_b32(sel, min(tile * kBN + row, count - 1) * 4, 0, 0);
    }
  };
  auto load_idx = [&](int tile, Idx &ix) {
    load_rows(rselA, ia.w, t0A + tile, ix.a);
    if constexpr (PAIRED) load_rows(rselB, ib.w, t0B + tile, ix.b);
    ix.own = 0;
    if (DROP && w < (PAIRED ? 4 : 2))
      ix.own = w < 2 ? __builtin_amdgcn_raw_buffer_load_b32(rselA, min((t0A + tile) * kBN + lane, ia.w - 1) * 4, 0, 0)
                     : __builtin_amdgcn_raw_buffer_load_b32(rselB, min((t0B + tile) * kBN + lane, ib.w - 1) * 4, 0, 0);
  };
  auto gather = [&](const __amdgpu_buffer_rsrc_t &rows_of, uint16_t *ta, uint16_t *tb, const Idx &ix) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int r0 = 8 * w + RPL * i, row = r0 + lane / CH;
      const int col = 16 * ((lane % CH) ^ tile_swizzle<D>(row));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rows_of, ta + r0 * D, 16, ix.a[i] * (D * 2) + col, 0, 0, 0);
      if constexpr (PAIRED)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rows_of, tb + r0 * D, 16, ix.b[i] * (D * 2) + col, 0, 0, 0);
    }
  };
  auto gather_k = [&](typename T::K &kn, const Idx &ix) {
    gather(rk, kn[0], kn[1], ix);
    if (DROP && w < (PAIRED ? 4 : 2))
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, kn[w >> 1] + T::kWords + 2 * kBN * (w & 1), 4, ix.own * 4, 0, 0, 0);
  };
  auto gather_v = [&](typename T::V &vn, const Idx &ix) { gather(rv, vn[0], vn[1], ix); };

  // the words of the keys of a lane's elements 4 i .. 4 i + 3 of block kb
  auto key_words = [&](const uint16_t *kt, int kb, int i, uint2 (&x)[4]) {
    const uint32_t *words = reinterpret_cast<const uint32_t *>(kt + T::kWords) + 32 * kb + 8 * i + 4 * hf;
    const uint4 p = *reinterpret_cast<const uint4 *>(words), q = *reinterpret_cast<const uint4 *>(words + kBN);
    x[0] = make_uint2(p.x, q.x);
    x[1] = make_uint2(p.y, q.y);
    x[2] = make_uint2(p.z, q.z);
    x[3] = make_uint2(p.w, q.w);
  };
  // S^T of one block of 32 keys, -inf past the end of the list
  auto scores = [&](const uint16_t *kt, int kb) {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.row(kt + 32 * kb * D, x), qf[x], s, 0, 0, 0);
    return s;
  };
  auto cut = [&](f32x16 &s, int from) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (from + 8 * (e >> 2) + 4 * hf + (e & 3) >= r) s[e] = -INFINITY;
  };
  auto add = [&](const uint16_t *tile, const bf16x8 (&p)[2]) {
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.columns(tile + 16 * s2 * D, db), p[s2], acc[db], 0, 0, 0);
  };
  // of two terms
  auto add2 = [&](const uint16_t *tile, const bf16x8 (&p)[2], const bf16x8 (&rest)[2]) {
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const bf16x8 k = at.columns(tile + 16 * s2 * D, db);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, p[s2], acc[db], 0, 0, 0);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, rest[s2], acc[db], 0, 0, 0);
      }
  };

  auto forward_tile = [&](int tile, const uint16_t *kt, const uint16_t *vt, typename T::K &kn, typename T::V &vn,
                          const Idx &ix) {
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.0f;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.row(kt + 32 * kb * D, x), qf[x], s[kb], 0, 0, 0);
    interleave<D / 8, 1, 0>();
    gather_k(kn, ix);
    if (tile * kBN + kBN > r) {
      cut(s[0], tile * kBN);
      cut(s[1], tile * kBN + 32);
    }
    float mx0 = fmaxf(s[0][0], s[0][1]), mx1 = fmaxf(s[1][0], s[1][1]);
#pragma unroll
    for (int e = 2; e < 16; e += 2) {
      mx0 = fmaxf(fmaxf(mx0, s[0][e]), s[0][e + 1]);
      mx1 = fmaxf(fmaxf(mx1, s[1][e]), s[1][e + 1]);
    }
    float mx = fmaxf(mx0, mx1);
    {
      // the other half-wave holds the query's other keys
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    }
    // a query rescales on its own, where its maximum falls too far behind
    const float mt = mx * a.scale_log2;
    const bool behind = mt > m_run + kLag;
    if (__ballot(behind)) {
      const float m_new = behind ? fmaxf(m_run, mt) : m_run;
      const float alpha = behind ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.0f;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] *= alpha;
      m_run = m_new;
    }
    // no logit above -inf so far: weights of 0, where inf - inf would be NaN
    const float neg_m = m_run == -INFINITY ? 0.0f : -m_run;
    bf16x8 pk[2][2];
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    auto weights = [&](int kb) {
      float p[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint2 kw[4];
        if constexpr (DROP) key_words(kt, kb, i, kw);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 4 * i + j;
          p[e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], a.scale_log2, neg_m));
          sum[j] += p[e];
          if constexpr (DROP) {
            p[e] = pair_kept(mine, kw[j], a.drop) ? p[e] : 0.0f;
            asm("" : "+v"(p[e]));  // or both are rounded and the bits selected
          }
        }
      }
      pk[kb][0] = pack8(p);
      pk[kb][1] = pack8(p + 8);
    };
    weights(0);
    gather_v(vn, ix);
    asm volatile("" : "+v"(pk[0][0]), "+v"(pk[0][1]), "+v"(at.col_at));
    // the second block's weights beside the first's product
    add(vt, pk[0]);
    weights(1);
    interleave<D / 16, 2, D == 128 ? 7 : 14>();
#pragma unroll
    for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(acc[db]));
    asm volatile("" : "+v"(pk[1][0]), "+v"(pk[1][1]), "+v"(at.col_at));
    add(vt + 32 * D, pk[1]);
    interleave<D / 16, 2, 0>();
    l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };

  // In phases, each with matrix products next to the vector work of another block of
  // keys; the empty asm statements end a phase as in attention_keys.hip.
  auto grad_tile = [&](int tile, const uint16_t *kt, const uint16_t *vt) {
    f32x16 s[2], dp[2];
    float p[2][16];
    bf16x8 dsk[2][2], rest[2][2];
    auto weights = [&](int kb) {  // p, negative where dropped, beside dP^T
      f32x16 x;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = 0.0f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.row(vt + 32 * kb * D, i), gf[i], x, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint2 kw[4];
        if constexpr (DROP) key_words(kt, kb, i, kw);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 4 * i + j;
          p[kb][e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], a.scale_log2, neg_lse));
          if constexpr (DROP) p[kb][e] = pair_kept(mine, kw[j], a.drop) ? p[kb][e] : -p[kb][e];
        }
      }
      dp[kb] = x;
      interleave<D / 16, 1, D == 128 ? 4 : 8>();
      asm volatile("" : "+v"(dp[kb]), "+v"(at.row_at), "+v"(at.col_at));
    };
    auto gradient = [&](int kb) {  // ds
      float ds[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = DROP ? (p[kb][e] > 0.0f ? dp[kb][e] * a.kept_scale : 0.0f) : dp[kb][e];
        ds[e] = fabsf(p[kb][e]) * (x - delta);
      }
      dsk[kb][0] = pack8(ds);
      dsk[kb][1] = pack8(ds + 8);
      // what the rounding left
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 u = __builtin_bit_cast(uint4, dsk[kb][i]);
        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ds[8 * i + 2 * j] -= __uint_as_float(x[j] << 16);
          ds[8 * i + 2 * j + 1] -= __uint_as_float(x[j] & 0xFFFF0000u);
        }
      }
      rest[kb][0] = pack8(ds);
      rest[kb][1] = pack8(ds + 8);
    };
    s[0] = scores(kt, 0);
    interleave<D / 16, 1, 0>();
    asm volatile("" : "+v"(s[0]), "+v"(at.row_at));
    if (tile * kBN + 32 > r) cut(s[0], tile * kBN);
    weights(0);
    gradient(0);
    s[1] = scores(kt, 1);
    interleave<D / 16, 1, D == 128 ? 5 : 10>();
    asm volatile("" : "+v"(s[1]), "+v"(dsk[0][0]), "+v"(dsk[0][1]), "+v"(rest[0][0]), "+v"(rest[0][1]), "+v"(at.row_at));
    // d = 64 has registers for one block of keys' ds (kept over the next block's
    // weights they spilled 32 more: dQ of 8 heads x 19721 568 us for 351)
    if constexpr (D == 64) {
      add2(kt, dsk[0], rest[0]);
      interleave<D / 8, 1, 0>();
#pragma unroll
      for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(acc[db]));
    }
    if (tile * kBN + 64 > r) cut(s[1], tile * kBN + 32);
    weights(1);
    gradient(1);
    if constexpr (D == 128) {
      add2(kt, dsk[0], rest[0]);
      interleave<D / 8, 1, 4>();
#pragma unroll
      for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(acc[db]));
    }
    asm volatile("" : "+v"(dsk[1][0]), "+v"(dsk[1][1]), "+v"(rest[1][0]), "+v"(rest[1][1]), "+v"(at.col_at));
    add2(kt + 32 * D, dsk[1], rest[1]);
    interleave<D / 8, 1, 0>();
#pragma unroll
    for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(acc[db]));
    asm volatile("" : "+v"(at.row_at), "+v"(at.col_at));
  };

  // one step: indices of tile T+2 requested, tile T computed while tile T+1 is
  // gathered into the free buffers; every wave's gathers land before the barrier
  Idx now, ahead;
  auto step = [&](int tile, typename T::K &kc, typename T::V &vc, typename T::K &kn, typename T::V &vn) {
    load_idx(tile + 2, ahead);
    const bool mine_too = active && tile < nt_own;
    if (GRAD || !mine_too) {
      gather_k(kn, now);
      gather_v(vn, now);
    }
    if (mine_too) {
      if constexpr (GRAD)
        grad_tile(t0_own + tile, kc[g], vc[g]);
      else
        forward_tile(t0_own + tile, kc[g], vc[g], kn, vn, now);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
    now = ahead;
  };
  if (ntiles > 0) {
    load_idx(0, ahead);
    load_idx(1, now);
    gather_k(K0, ahead);
    gather_v(V0, ahead);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  for (int tile = 0; tile < ntiles; tile += 2) {
    step(tile, K0, V0, K1, V1);
    if (tile + 1 < ntiles) step(tile + 1, K1, V1, K0, V0);
  }

  if (a.splits > 1) {  // the part's sums, and the forward's maximum and normaliser
    float *to = a.parts + (static_cast<size_t>(part) * a.rows + first + qi) * D + 4 * hf;
    const float l = l_run + __shfl_xor(l_run, 32);
    if (!valid) return;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4 *>(to + 32 * db + 8 * i) =
            make_float4(acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]);
    if (!GRAD && hf == 0)
      reinterpret_cast<float2 *>(a.parts + a.splits * a.rows * D)[part * a.rows + first + qi] = make_float2(m_run, l);
    return;
  }
  float f = a.scale;
  if constexpr (!GRAD) {
    // lanes l and l^32 hold the two halves of one query's row sum
    const float l = l_run + __shfl_xor(l_run, 32);
    f = l > 0.0f ? a.kept_scale / l : 0.0f;
    if (valid && hf == 0) a.lse[first + qi] = l > 0.0f ? (m_run + __log2f(l)) * kLn2 : l == 0.0f ? -INFINITY : l;
  }
  if (!valid) return;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2 *>(out + (first + qi) * D + 32 * db + 8 * i + 4 * hf) =
          make_uint2(pack_bf16(acc[db][4 * i] * f, acc[db][4 * i + 1] * f),
                     pack_bf16(acc[db][4 * i + 2] * f, acc[db][4 * i + 3] * f));
}

// d = 128: the tiles' LDS leaves a CU one block.  d = 64: two, within 128 registers (dQ
// spills 9 of them): 8 heads x 19721, 18% kept, 335 to 351 us for 418 with one block.
// Dropout's words would spill far more: 8 x 8000 504 us for 317 (ds in one term).
template <int D, bool GRAD, bool DROP>
__global__ __launch_bounds__(kNW * 64)
__attribute__((amdgpu_waves_per_eu(D == 64 && !DROP ? 4 : 2))) void queries_kernel(TrainArgs a, int total_items,
                                                                         const int4 *__restrict__ items,
                                                                         const int2 *__restrict__ order, uint16_t *out) {
  typedef Tiles<D, DROP> T;
  __shared__ __attribute__((aligned(16))) typename T::K K0;
  __shared__ __attribute__((aligned(16))) typename T::K K1;
  __shared__ __attribute__((aligned(16))) typename T::V V0;
  __shared__ __attribute__((aligned(16))) typename T::V V1;
  int item, half = 0, part = 0;
  if (a.splits > 1) {
    const int b = static_cast<int>(blockIdx.x);
    item = xcd_item(b % total_items, total_items);
    part = b / total_items;
  } else if (order) {
    const int2 e = order[blockIdx.x];  // (slot, 0: all of it, 1 or 2: a half)
    item = e.x;
    half = e.y;
  } else {
    item = xcd_item(static_cast<int>(blockIdx.x), total_items);
  }
  if (item < 0 || item >= total_items) return;
  const int h = item / a.items_per_head;
  int4 ia = items[2 * item], ib = items[2 * item + 1];
  if (half) take_half(&ia, &ib, half);
  if (ia.z <= 0) return;
  if (ib.z > 0)
    queries_body<D, GRAD, DROP, true>(a, h, ia, ib, part, out, K0, K1, V0, V1);
  else
    queries_body<D, GRAD, DROP, false>(a, h, ia, ib, part, out, K0, K1, V0, V1);
}

template <int D, bool GRAD>
hipError_t run(const TrainArgs &a, int total, int blocks, const AttnScratch &w, uint16_t *out, hipStream_t s) {
  const int2 *order = w.order;
  const int4 *items = w.items;
  if (a.drop)
    hipLaunchKernelGGL((queries_kernel<D, GRAD, true>), dim3(blocks), dim3(kNW * 64), 0, s, a, total, items, order, out);
  else
    hipLaunchKernelGGL((queries_kernel<D, GRAD, false>), dim3(blocks), dim3(kNW * 64), 0, s, a, total, items, order, out);
  return hipGetLastError();
}

}  // namespace

hipError_t train_queries(int d, bool grad, const TrainArgs &args, int heads, bool listed, const AttnScratch &scratch,
                         uint16_t *out, hipStream_t s) {
  TrainArgs a = args;
  AttnScratch w = scratch;
  if (a.splits > 1) w.order = nullptr;
  a.items_per_head = attn_items_per_head(a.n, a.c_q);
  const int total = heads * a.items_per_head;
  int blocks = total * a.splits;
  if (!listed) {
    hipError_t e = attention_list(heads, a.n, d, a.c_q, a.c_q > 1, a.offsets, a.sel_counts, w, s);
    if (e != hipSuccess) return e;
    if (a.splits == 1 && (e = attention_plan(heads, a.n, d, a.c_q, w, &blocks, s)) != hipSuccess) return e;
  } else {
    w.order = nullptr;
  }
  if (d == 128) return grad ? run<128, true>(a, total, blocks, w, out, s) : run<128, false>(a, total, blocks, w, out, s);
  return grad ? run<64, true>(a, total, blocks, w, out, s) : run<64, false>(a, total, blocks, w, out, s);
}

}  // namespace scope
