// Attention over packed sequences by rows, bf16 inputs: the forward with row
// statistics, and dQ (packed_plan.hip has the formulas).
//
// A block runs an item's up to 128 rows (query, head of the group) of a key head, a
// wave 32 of them, over the keys that its last row sees, 64 at a time (the forward at
// d = 128: 32): K and V tiles
// are brought into LDS by the buffer unit while the tile before is computed.  A
// wave's tile is
//   S^T = K_tile . Q^T                   keys x rows, a row per lane column
//   online softmax in fp32, exp2 domain; weights rounded to bf16 for
//   O^T += V_tile^T . P^T                (transposing LDS reads of V)
// and for the gradient, p recomputed from the row's log-sum-exp,
//   dP^T = V_tile . dO^T, ds = p (dP - D), dQ^T += K_tile^T . ds^T
// with ds as two bf16 terms, the second what rounding the first left: a row's ds sum
// to zero, so dQ is a difference of larger sums and keeps more of their rounding.
//
// Several blocks share a CU, whose waves drift apart, so that one's matrix products run
// beside another's vector work: two of 128 rows rather than one of 256 (dQ 8% faster,
// single tokens 31 us for 46), and where 32 keys a tile leave registers for it, three (the
// forward at d = 128, 1.05 -> 1.10 PFLOP/s; d = 64 holds four with 64 keys, and five with
// 32 were 4% slower).  S of the next tile beside the weights of this one in a wave was no
// faster.  The kernels fill the matrix pipe until the card lowers its clock.  5 heads x
// 32760, d = 128: forward 2.5 ms, 1.10 PFLOP/s; dQ 4.6 ms, 1.19 PFLOP/s of its four
// products, matrix pipe 67% busy at 1.75 GHz.  d = 64, 10 heads: 2.86 ms, 0.96 PFLOP/s,
// and dQ 5.2 ms, both bound by vector instructions, 80% busy.
#include "attention_tile.h"
#include "packed.h"

namespace scope {

namespace {

constexpr float kLag = 8.0f;  // the running maximum may lag by 2^8
constexpr int kWaves = kPackRows / 32;  // a wave owns 32 rows
static_assert(64 * kWaves == kPackThreads, "threads of a block");

// Wave w's share of a tile of keys' rows, 1 KB per load, through a resource that starts
// at the tile (a sequence may be longer than 32-bit offsets reach); rows past the last
// key repeat it, with no weight.
template <int D, int N, int WAVES>
struct KeyTile {
  static __device__ __forceinline__ void bring(char *base, int64_t stride, uint16_t *tile, int index, int lk, int w, int lane) {
    constexpr int CH = D / 8, RPL = 64 / CH;  // 16-byte chunks per row, rows per load
    const int rows = min(lk - index * N, N);
    const __amdgpu_buffer_rsrc_t from = pack_resource(base + static_cast<int64_t>(index) * N * stride,
                                                      static_cast<uint32_t>(rows - 1) * static_cast<uint32_t>(stride) + 2 * D);
    if (rows == N) {
#pragma unroll
      for (int i = 0; i < N / WAVES / RPL; ++i) {
        const int r0 = N / WAVES * w + RPL * i, r = r0 + lane / CH;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, tile + r0 * D, 16,
                                                 r * static_cast<uint32_t>(stride) + 16 * ((lane % CH) ^ tile_swizzle<D>(r)), 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N / WAVES / RPL; ++i) {
        const int r0 = N / WAVES * w + RPL * i, r = r0 + lane / CH;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, tile + r0 * D, 16,
                                                 min(r, rows - 1) * static_cast<uint32_t>(stride) + 16 * ((lane % CH) ^ tile_swizzle<D>(r)),
                                                 0, 0, 0);
      }
    }
  }
};

template <int D, bool GRAD, bool FEW>
__global__ __launch_bounds__(kWaves * 64)
__attribute__((amdgpu_waves_per_eu(FEW || (GRAD && D == 128) ? 2 : D == 64 ? 4 : 3))) void packed_queries_kernel(PackArgs a, PackRows out) {
  constexpr int KB = GRAD || D == 64 ? 2 : 1, N = 32 * KB;  // blocks of 32 keys in a tile, and its keys
  constexpr int kItem = FEW ? kPackFewRows : kPackRows, kTiles = FEW ? kWaves : 1;  // rows; tiles in LDS
  __shared__ __attribute__((aligned(16))) uint16_t K0[kTiles * N * D], K1[kTiles * N * D], V0[kTiles * N * D], V1[kTiles * N * D];
  int h, part, row0;
  int4 sq;
  int2 ends;
  const bool item = pack_item<false, kItem>(a, &h, &part, &sq, &row0, &ends);
  if (a.clear && a.splits == 1)
    clear_rows<uint16_t, D, kWaves * 64>(out, a.kv_heads * a.group, a.rows_q, ends, GRAD ? nullptr : a.lse);
  if (!item) return;
  const int q0 = sq.x, lq = sq.y, k0 = sq.z, lk = sq.w, rows = lq * a.group;
  const int t = threadIdx.x, lane = t & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  TileReader<D> at(lane);
  const int w_row = row0 + (FEW ? 0 : 32 * w), own = w_row + l32, row = min(own, rows - 1);
  const bool valid = own < rows, active = w_row < rows;
  const int query = row / a.group, member = row - query * a.group;
  const size_t stat = (static_cast<size_t>(h) * a.rows_q + q0) * a.group + row;  // of (key head, row)
  // keys that this row sees, and the wave's fewest and most
  const int seen = keys_seen(row, a.group, lq, lk, a.causal);
  const int fewest = __builtin_amdgcn_readlane(seen, 0), most = __builtin_amdgcn_readlane(seen, 31);
  const int block_most = keys_seen(min(row0 + kItem, rows) - 1, a.group, lq, lk, a.causal);

  bf16x8 qf[D / 16], gf[GRAD ? D / 16 : 1];
  {
    const uint16_t *q = reinterpret_cast<const uint16_t *>(rows_base(a.q, q0, h * a.group) + query * a.q.row + member * a.q.head);
    const uint16_t *g = reinterpret_cast<const uint16_t *>(rows_base(a.d_o, q0, h * a.group) + query * a.d_o.row + member * a.d_o.head);
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      qf[x] = as_bf16x8(valid ? load8<true>(q, 16 * x + 8 * hf) : make_uint4(0, 0, 0, 0));
      if constexpr (GRAD) gf[x] = as_bf16x8(valid ? load8<true>(g, 16 * x + 8 * hf) : make_uint4(0, 0, 0, 0));
    }
  }
  float neg_lse = -INFINITY, delta = 0.0f;
  if constexpr (GRAD) {
    if (valid) {
      const uint16_t *o = reinterpret_cast<const uint16_t *>(rows_base(a.o, q0, h * a.group) + query * a.o.row + member * a.o.head);
#pragma unroll
      for (int x = 0; x < D / 16; ++x) {
        const bf16x8 of = as_bf16x8(load8<true>(o, 16 * x + 8 * hf));
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = fmaf(static_cast<float>(of[j]), static_cast<float>(gf[x][j]), delta);
      }
      const float lse = a.lse[static_cast<size_t>(h * a.group + member) * a.rows_q + q0 + query];
      neg_lse = lse == -INFINITY ? -INFINITY : lse * -1.4426950408889634f;  // no key: no weight
    }
    delta += __shfl_xor(delta, 32);
    if (valid && hf == 0 && part == 0) {
      a.stats[stat] = neg_lse;
      a.stats[static_cast<size_t>(a.kv_heads) * a.rows_q * a.group + stat] = delta;
    }
  }

  f32x16 acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.0f;
  float m_run = -INFINITY, l_run = 0.0f;

  // the part's tiles
  const int all = (block_most + N - 1) / N, per = (all + a.splits - 1) / a.splits;
  const int first = scalar(min(part * per, all)), last = scalar(min(first + per, all));
  const int last_own = scalar(active ? min(last, (most + N - 1) / N) : 0);

  char *const k_base = rows_base(a.k, k0, h), *const v_base = rows_base(a.v, k0, h);
  auto bring_k = [&](uint16_t *tile, int index) { KeyTile<D, N, FEW ? 1 : kWaves>::bring(k_base, a.k.row, tile, index, lk, FEW ? 0 : w, lane); };
  auto bring_v = [&](uint16_t *tile, int index) { KeyTile<D, N, FEW ? 1 : kWaves>::bring(v_base, a.v.row, tile, index, lk, FEW ? 0 : w, lane); };
  auto scores = [&](const uint16_t *kt, int kb) {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.row(kt + 32 * kb * D, x), qf[x], s, 0, 0, 0);
    return s;
  };
  // -inf for the keys from `from` on that the row does not see
  auto cut = [&](f32x16 &s, int from) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (from + 8 * (e >> 2) + 4 * hf + (e & 3) >= seen) s[e] = -INFINITY;
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

  auto forward_tile = [&](int index, const uint16_t *kt, const uint16_t *vt) {
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.0f;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.row(kt + 32 * kb * D, x), qf[x], s[kb], 0, 0, 0);
    interleave<KB * D / 16, 1, 0>();
    if ((index + 1) * N > fewest) {
      cut(s[0], index * N);
      if constexpr (KB == 2) cut(s[KB - 1], index * N + 32);
    }
    auto logit = [&](int i) { return s[i / 16][i % 16]; };
    float mx0 = fmaxf(logit(0), logit(1)), mx1 = fmaxf(logit(8 * KB), logit(8 * KB + 1));
#pragma unroll
    for (int i = 2; i < 8 * KB; i += 2) {
      mx0 = fmaxf(fmaxf(mx0, logit(i)), logit(i + 1));
      mx1 = fmaxf(fmaxf(mx1, logit(8 * KB + i)), logit(8 * KB + i + 1));
    }
    float mx = fmaxf(mx0, mx1);
    {
      // the other half-wave holds the row's other keys
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    }
    // a row rescales on its own, where its maximum falls too far behind
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
    bf16x8 pk[KB][2];
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    auto weights = [&](int kb) {
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], a.scale_log2, neg_m));
        sum[e & 3] += p[e];
      }
      pk[kb][0] = pack8(p);
      pk[kb][1] = pack8(p + 8);
    };
    weights(0);
    asm volatile("" : "+v"(pk[0][0]), "+v"(pk[0][1]), "+v"(at.col_at));
    add(vt, pk[0]);
    if constexpr (KB == 1) {
      interleave<D / 16, 2, 0>();
    } else {
      // the second block's weights beside the first's product
      weights(KB - 1);
      interleave<D / 16, 2, 14>();
#pragma unroll
      for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(acc[db]));
      asm volatile("" : "+v"(pk[KB - 1][0]), "+v"(pk[KB - 1][1]), "+v"(at.col_at));
      add(vt + 32 * D, pk[KB - 1]);
      interleave<D / 16, 2, 0>();
    }
    l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };

  // In phases, each with matrix products next to the vector work of another block of
  // keys; the empty asm statements end a phase as in attention_keys.hip.
  auto grad_tile = [&](int index, const uint16_t *kt, const uint16_t *vt) {
    f32x16 s[2], dp[2];
    float p[2][16];
    bf16x8 dsk[2][2], rest[2][2];
    const bool edge = (index + 1) * N > fewest;
    auto weights = [&](int kb) {  // p beside dP^T
      f32x16 x;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = 0.0f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.row(vt + 32 * kb * D, i), gf[i], x, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 16; ++e) p[kb][e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], a.scale_log2, neg_lse));
      dp[kb] = x;
      interleave<D / 16, 1, D == 128 ? 4 : 8>();
      asm volatile("" : "+v"(dp[kb]), "+v"(at.row_at), "+v"(at.col_at));
    };
    auto gradient = [&](int kb) {  // ds
      float ds[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) ds[e] = p[kb][e] * (dp[kb][e] - delta);
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
    if (edge) cut(s[0], index * N);
    weights(0);
    gradient(0);
    s[1] = scores(kt, 1);
    interleave<D / 16, 1, D == 128 ? 5 : 10>();
    asm volatile("" : "+v"(s[1]), "+v"(dsk[0][0]), "+v"(dsk[0][1]), "+v"(rest[0][0]), "+v"(rest[0][1]), "+v"(at.row_at));
    // d = 64 has registers for one block of keys' ds
    if constexpr (D == 64) {
      add2(kt, dsk[0], rest[0]);
      interleave<D / 8, 1, 0>();
#pragma unroll
      for (int db = 0; db < D / 32; ++db) asm volatile("" : "+v"(acc[db]));
    }
    if (edge) cut(s[1], index * N + 32);
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

  // one step: tile T computed while the next is brought into the free buffers.  Every wave
  // takes all tiles, brought together: its loads land before the barrier.  FEW: a wave
  // takes every kWaves-th tile, which it brings itself, and waits for no other.
  constexpr int kStride = FEW ? kWaves : 1;
  auto land = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    if constexpr (!FEW) __syncthreads();
  };
  auto step = [&](int index, const uint16_t *kc, const uint16_t *vc, uint16_t *kn, uint16_t *vn) {
    if (index + kStride < last) {
      bring_k(kn, index + kStride);
      bring_v(vn, index + kStride);
    }
    if (index < last_own) {
      if constexpr (GRAD)
        grad_tile(index, kc, vc);
      else
        forward_tile(index, kc, vc);
    }
    land();
  };
  const int start = first + (FEW ? w : 0), mine = FEW ? w * N * D : 0;
  if (start < last) {
    bring_k(K0 + mine, start);
    bring_v(V0 + mine, start);
  }
  land();
  for (int index = start; index < last; index += 2 * kStride) {
    step(index, K0 + mine, V0 + mine, K1 + mine, V1 + mine);
    if (index + kStride < last) step(index + kStride, K1 + mine, V1 + mine, K0 + mine, V0 + mine);
  }

  float l = l_run + __shfl_xor(l_run, 32);  // the halves of a row's sum
  if constexpr (FEW) {
    // the waves' sums, in wave order: a wave's share of the channels each
    __shared__ float ms[kWaves][32], ls[kWaves][32];
    // a wave's sums lie where its K tiles were, 16 bytes swizzled by the row
    constexpr int kHalf = N / 2;  // rows in the first tile
    auto sums = [&](int wave, int r, int c) {
      uint16_t *tile = (r < kHalf ? K0 : K1) + wave * N * D;
      return reinterpret_cast<float4 *>(tile) + (r % kHalf) * (D / 4) + ((c / 4) ^ (r & 15));
    };
    if (hf == 0) {
      ms[w][l32] = m_run;
      ls[w][l32] = l;
    }
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *sums(w, l32, 32 * db + 8 * x + 4 * hf) =
            make_float4(acc[db][4 * x], acc[db][4 * x + 1], acc[db][4 * x + 2], acc[db][4 * x + 3]);
    __syncthreads();
    m_run = fmaxf(fmaxf(ms[0][l32], ms[1][l32]), fmaxf(ms[2][l32], ms[3][l32]));
    static_assert(kWaves == 4, "four waves' sums");
    l = 0.0f;
    float f[kWaves];
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      f[i] = __builtin_amdgcn_exp2f(ms[i][l32] - (m_run == -INFINITY ? 0.0f : m_run));
      l = fmaf(ls[i][l32], f[i], l);
    }
    if (!valid) return;
    const size_t total = static_cast<size_t>(a.kv_heads) * a.rows_q * a.group, i = part * total + stat;
    const float scale = a.splits > 1 ? 1.0f : l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (w == 0 && hf == 0) {
      if (a.splits > 1)
        reinterpret_cast<float2 *>(a.parts + a.splits * total * D)[i] = make_float2(m_run, l);
      else
        a.lse[static_cast<size_t>(h * a.group + member) * a.rows_q + q0 + query] =
            l > 0.0f ? (m_run + __log2f(l)) * kPackLn2 : l == 0.0f ? -INFINITY : l;
    }
    uint16_t *to = reinterpret_cast<uint16_t *>(rows_base(out, q0, h * a.group) + query * out.row + member * out.head);
#pragma unroll
    for (int x = 0; x < D / kWaves / 8; ++x) {
      const int c = D / kWaves * w + 8 * x + 4 * hf;
      float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int j = 0; j < kWaves; ++j) {
        const float4 v = *sums(j, l32, c);
        s.x = fmaf(v.x, f[j], s.x);
        s.y = fmaf(v.y, f[j], s.y);
        s.z = fmaf(v.z, f[j], s.z);
        s.w = fmaf(v.w, f[j], s.w);
      }
      if (a.splits > 1)
        *reinterpret_cast<float4 *>(a.parts + i * D + c) = s;
      else
        *reinterpret_cast<uint2 *>(to + c) = make_uint2(pack_bf16(s.x * scale, s.y * scale), pack_bf16(s.z * scale, s.w * scale));
    }
    return;
  }
  if (!valid) return;
  if (a.splits > 1) {  // the part's sums, and the forward's maximum and normaliser
    const size_t total = static_cast<size_t>(a.kv_heads) * a.rows_q * a.group, i = part * total + stat;
    float *to = a.parts + i * D + 4 * hf;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<float4 *>(to + 32 * db + 8 * x) =
            make_float4(acc[db][4 * x], acc[db][4 * x + 1], acc[db][4 * x + 2], acc[db][4 * x + 3]);
    if (!GRAD && hf == 0) reinterpret_cast<float2 *>(a.parts + a.splits * total * D)[i] = make_float2(m_run, l);
    return;
  }
  float f = a.scale;
  if constexpr (!GRAD) {
    f = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (hf == 0)
      a.lse[static_cast<size_t>(h * a.group + member) * a.rows_q + q0 + query] =
          l > 0.0f ? (m_run + __log2f(l)) * kPackLn2 : l == 0.0f ? -INFINITY : l;
  }
  uint16_t *to = reinterpret_cast<uint16_t *>(rows_base(out, q0, h * a.group) + query * out.row + member * out.head) + 4 * hf;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *reinterpret_cast<uint2 *>(to + 32 * db + 8 * x) = make_uint2(pack_bf16(acc[db][4 * x] * f, acc[db][4 * x + 1] * f),
                                                                     pack_bf16(acc[db][4 * x + 2] * f, acc[db][4 * x + 3] * f));
}

template <int D, bool GRAD, bool FEW>
hipError_t run(const PackArgs &a, const PackRows &out, hipStream_t s) {
  const dim3 grid(pack_blocks(a.list.capacity, a.kv_heads, a.splits));
  hipLaunchKernelGGL((packed_queries_kernel<D, GRAD, FEW>), grid, dim3(kWaves * 64), 0, s, a, out);
  return hipGetLastError();
}

}  // namespace

hipError_t packed_queries(const PackArgs &a, int d, bool grad, const PackRows &out, hipStream_t s) {
  if (a.list.rows == kPackFewRows) return d == 128 ? run<128, false, true>(a, out, s) : run<64, false, true>(a, out, s);
  if (d == 128) return grad ? run<128, true, false>(a, out, s) : run<128, false, false>(a, out, s);
  return grad ? run<64, true, false>(a, out, s) : run<64, false, false>(a, out, s);
}

}  // namespace scope
