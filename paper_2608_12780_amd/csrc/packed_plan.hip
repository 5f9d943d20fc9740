// Attention over packed sequences (calls 10 and 11): the work lists of many sequences,
// the joins of parts, and the order of launches.
//
// With n queries and m keys of a sequence, key head h and the query heads of its
// group side by side as rows (query, head):
//   s_ij = <q_i, k_j>, p_ij = exp(scale s_ij - lse_i), j <= i + m - n where causal
//   o_i = sum_j p_ij v_j,  ds_ij = p_ij (<do_i, v_j> - <do_i, o_i>)
//   dq_i = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i, dv_j = sum_i p_ij do_i
// A group's rows share their keys' tiles, and dk and dv sum over them in one place.
// As in the sparse layer's training attention every sum has one owner and a fixed
// order (dq by rows, dk and dv by keys).
//
// Sequence lengths are on the device, so the host launches as many blocks as any
// lengths could need; they find their items, longest first, from the offsets (packed.h),
// or from a list where there are more than 64 sequences.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "mfma.h"
#include "packed.h"

namespace scope {

namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 1024;
constexpr int kMostParts = 16;
constexpr int kFewItems = 32;

struct PackLists {
  PackArgs a;
  PackList lists[2];
  int32_t *header;   // counts, ends
};

// Inclusive scan over the block's threads; `total` receives the last.
template <bool MAX>
__device__ int block_scan(int v, int *wave, int *total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(v, o);
    if (lane >= o) v = MAX ? max(v, t) : v + t;
  }
  __syncthreads();
  if (lane == 63) wave[w] = v;
  __syncthreads();
  int all = wave[0];
  for (int i = 1; i < kThreads / 64; ++i) {
    if (i == w) v = MAX ? max(v, all) : v + all;
    all = MAX ? max(all, wave[i]) : all + wave[i];
  }
  *total = all;
  return v;
}

// Lists of work items for more sequences than a wave has lanes: block 0's by rows, block
// 1's by keys.
__global__ __launch_bounds__(kThreads) void pack_lists_kernel(PackLists p) {
  const int which = static_cast<int>(blockIdx.x);
  const PackArgs &a = p.a;
  const PackList list = p.lists[which];
  __shared__ int wave[kThreads / 64], first[kThreads + 1], hist[kBins];
  __shared__ int4 seq[kThreads];
  const int t = threadIdx.x, S = a.sequences;
  const bool by_keys = which == 1;
  hist[t] = 0;
  // a cost's bin: the longest first; items without work last
  const int most = by_keys ? (a.rows_q * a.group + kCostRows - 1) / kCostRows : (a.rows_k + kCostKeys - 1) / kCostKeys;
  const float per_cost = static_cast<float>(kBins - 2) / max(most, kBins - 2);
  auto bin_of = [&](const int4 &s, int at) {
    int cost;
    if (by_keys) {
      const int from = a.causal ? max(at - (s.w - s.y), 0) : 0;
      cost = (max(s.y - from, 0) * a.group + kCostRows - 1) / kCostRows;
    } else {
      const int last = min(at + list.rows, s.y * a.group) - 1;
      cost = (keys_seen(last, a.group, s.y, s.w, a.causal) + kCostKeys - 1) / kCostKeys;
    }
    return kBins - 1 - min(static_cast<int>(cost * per_cost) + (cost > 0 ? 1 : 0), kBins - 1);
  };
  for (int pass = 0; pass < 2; ++pass) {
    int run_q = 0, run_k = 0;
    bool bad = false;
    for (int base = 0; base < S; base += kThreads) {
      const int s = base + t;
      const int q = s < S ? a.offsets_q[s] : 0, q_next = s < S ? a.offsets_q[s + 1] : 0;
      const int k = s < S ? a.offsets_k[s] : 0, k_next = s < S ? a.offsets_k[s + 1] : 0;
      bad = bad || (s < S && (q < 0 || q_next < q || q_next > a.rows_q || k < 0 || k_next < k || k_next > a.rows_k));
      auto clamped = [](int x, int rows) { return min(max(x, 0), rows); };
      int top_q, top_k;
      const int q1 = max(block_scan<true>(max(clamped(q, a.rows_q), clamped(q_next, a.rows_q)), wave, &top_q), run_q);
      const int k1 = max(block_scan<true>(max(clamped(k, a.rows_k), clamped(k_next, a.rows_k)), wave, &top_k), run_k);
      // a sequence's end is the next one's start
      __syncthreads();
      seq[t] = make_int4(q1, 0, k1, 0);
      __syncthreads();
      int q0, k0;
      if (t > 0) {
        q0 = seq[t - 1].x;
        k0 = seq[t - 1].z;
      } else {
        q0 = base ? run_q : clamped(q, a.rows_q);
        k0 = base ? run_k : clamped(k, a.rows_k);
      }
      __syncthreads();
      int lk = k1 - k0;
      if (a.lengths_k && s < S) {
        const int n = a.lengths_k[s];
        bad = bad || n < 0 || n > lk;
        lk = min(max(n, 0), lk);
      }
      seq[t] = make_int4(q0, q1 - q0, k0, lk);
      if (pass == 0 && which == 0 && base == 0 && t == 0) {
        p.header[2] = q0;
        p.header[4] = k0;
      }
      const int tiles = s < S ? ((by_keys ? lk : (q1 - q0) * a.group) + list.rows - 1) / list.rows : 0;
      int total;
      const int incl = block_scan<false>(tiles, wave, &total);
      first[t] = incl - tiles;
      if (t == 0) first[kThreads] = total;
      __syncthreads();
      for (int slot = t; slot < total; slot += kThreads) {
        int lo = 0, hi = kThreads;  // first[lo] <= slot < first[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (first[mid] <= slot) lo = mid; else hi = mid;
        }
        const int4 sq = seq[lo];
        const int at = (slot - first[lo]) * list.rows;
        const int place = atomicAdd(&hist[bin_of(sq, at)], 1);
        if (pass == 1 && place < list.capacity) {
          list.items[2 * place] = sq;
          list.items[2 * place + 1].x = at;
        }
      }
      run_q = max(run_q, top_q);
      run_k = max(run_k, top_k);
      __syncthreads();
    }
    if (pass == 0) {
      // counts to first places
      __syncthreads();
      const int n = hist[t];
      int total;
      const int incl = block_scan<false>(n, wave, &total);
      hist[t] = incl - n;
      if (t == 0) {
        p.header[which] = min(total, list.capacity);
        if (which == 0) {
          p.header[3] = run_q;
          p.header[5] = run_k;
        }
      }
      if (bad && which == 0 && a.status) atomicOr(a.status, kStatusBadOffsets);
      __syncthreads();
    }
  }
}

// Four channels of an output row.
template <typename T>
__device__ __forceinline__ void store4(T *to, float x, float y, float z, float w) {
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(x, y), pack_bf16(z, w));
  else
    *reinterpret_cast<float4 *>(to) = make_float4(x, y, z, w);
}

// O and lse, or dQ, from the parts' sums.  A group of D / 4 lanes per row.
template <typename T, int D, bool GRAD>
__global__ __launch_bounds__(256) void pack_join_rows_kernel(PackArgs a, PackRows out) {
  constexpr int LANES = D / 4;
  const size_t per = static_cast<size_t>(a.rows_q) * a.group, rows = per * a.kv_heads;
  const size_t row = static_cast<size_t>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  const int x = threadIdx.x % LANES;
  const int2 ends = pack_ends(a, false);
  if (row >= rows) return;
  const int kv = static_cast<int>(row / per), r = static_cast<int>(row % per);
  const int query = r / a.group, head = kv * a.group + r % a.group;
  T *to = reinterpret_cast<T *>(rows_base(out, query, head)) + 4 * x;
  if (query < ends.x || query >= ends.y) {  // in no sequence
    if (!a.clear) return;
    store4(to, 0.0f, 0.0f, 0.0f, 0.0f);
    if (!GRAD && x == 0) a.lse[static_cast<size_t>(head) * a.rows_q + query] = -INFINITY;
    return;
  }
  const float2 *ml = reinterpret_cast<const float2 *>(a.parts + a.splits * rows * D);
  // all parts' maxima and normalisers at once: their loads' latency is most of a small join
  float w[kMostParts], f = a.scale;
  if constexpr (!GRAD) {
    float2 s[kMostParts];
#pragma unroll
    for (int p = 0; p < kMostParts; ++p) s[p] = ml[min(p, a.splits - 1) * rows + row];
    float top = -INFINITY, l = 0.0f;
#pragma unroll
    for (int p = 0; p < kMostParts; ++p) top = fmaxf(top, s[p].x);
    if (top == -INFINITY) top = 0.0f;
#pragma unroll
    for (int p = 0; p < kMostParts; ++p) {
      w[p] = p < a.splits ? __builtin_amdgcn_exp2f(s[p].x - top) : 0.0f;
      l = p < a.splits ? fmaf(s[p].y, w[p], l) : l;
    }
    f = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (x == 0) a.lse[static_cast<size_t>(head) * a.rows_q + query] = l > 0.0f ? (top + __log2f(l)) * kPackLn2 : l == 0.0f ? -INFINITY : l;
  }
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int p = 0; p < kMostParts; ++p) {
    if (p >= a.splits) break;
    const float4 v = *reinterpret_cast<const float4 *>(a.parts + (p * rows + row) * D + 4 * x);
    const float g = GRAD ? 1.0f : w[p];
    s.x = fmaf(v.x, g, s.x);
    s.y = fmaf(v.y, g, s.y);
    s.z = fmaf(v.z, g, s.z);
    s.w = fmaf(v.w, g, s.w);
  }
  store4(to, s.x * f, s.y * f, s.z * f, s.w * f);
}

// dK (blockIdx.y 0) and dV from the parts' sums.
template <typename T, int D>
__global__ __launch_bounds__(256) void pack_join_keys_kernel(PackArgs a, PackRows dk, PackRows dv) {
  constexpr int LANES = D / 4;
  const size_t rows = static_cast<size_t>(a.kv_heads) * a.rows_k;
  const size_t row = static_cast<size_t>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  const int x = threadIdx.x % LANES;
  const int2 ends = pack_ends(a, true);
  if (row >= rows) return;
  const int head = static_cast<int>(row / a.rows_k), key = static_cast<int>(row % a.rows_k);
  const int v = blockIdx.y;
  T *to = reinterpret_cast<T *>(rows_base(v ? dv : dk, key, head)) + 4 * x;
  if (key < ends.x || key >= ends.y) {
    if (a.clear) store4(to, 0.0f, 0.0f, 0.0f, 0.0f);
    return;
  }
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int p = 0; p < a.splits; ++p) {
    const float4 y = *reinterpret_cast<const float4 *>(a.parts + ((2 * static_cast<size_t>(p) + v) * rows + row) * D + 4 * x);
    s.x += y.x;
    s.y += y.y;
    s.z += y.z;
    s.w += y.w;
  }
  const float f = v ? 1.0f : a.scale;
  store4(to, s.x * f, s.y * f, s.z * f, s.w * f);
}

#define PACK_TRY(x)                  \
  do {                               \
    const hipError_t e_ = (x);       \
    if (e_ != hipSuccess) return e_; \
  } while (0)

// Parts that an item's tiles are cut into: as many as make `blocks` of the items, up to
// 16 of `least` tiles or more.  The chip holds 512 to 768 blocks at once; items differ in
// length as sequences do, and causal rows in keys, so that 1024 (dK and dV of bf16 inputs,
// whose longest items take longest: 2048) end more evenly.  A tile of fp32 takes longer and
// its join no longer, so that 2 tiles are enough for a part (6 sequences of 1224 tokens, 9
// heads of 3: the whole backward 152 us for 293 with 4 and 8), where bf16's forward wants 4
// (5 sequences of 1035 tokens, 32 heads of 8: 26 us for 36 with 2).  4 sequences of 512 queries
// behind 5000 to 16000 keys, 16 heads in groups of 4: 276 us with 512, 212 with 1024; 24
// prompts of 22 to 6600 tokens, d = 64, dK and dV: 797 us whole, 571 in two parts, joining
// them included; single tokens of 16 sequences behind up to 8000 keys 43 us with 512, 39
// with 1024 (with up to 64 parts 4 sequences of 16000 keys took 48 us for 38).
int parts_of(long long items, long long tiles, int least, int blocks) {
  long long s = items > 0 ? blocks / items : 1;
  if (s > tiles / least) s = tiles / least;
  return static_cast<int>(s < 1 ? 1 : s > kMostParts ? kMostParts : s);
}

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

hipError_t prepare(const PackArgs &a, const PackCall &c, const PackList &by_rows, int lists, hipStream_t s) {
  if (a.sequences <= 64) return hipSuccess;
  PackLists p{};
  p.a = a;
  p.lists[0] = by_rows;
  p.lists[1] = c.by_keys;
  p.header = c.header;
  hipLaunchKernelGGL(pack_lists_kernel, dim3(lists), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <typename T, int D, bool GRAD>
hipError_t join_rows(const PackArgs &a, const PackRows &out, hipStream_t s) {
  const size_t rows = static_cast<size_t>(a.kv_heads) * a.rows_q * a.group, per = 256 / (D / 4);
  hipLaunchKernelGGL((pack_join_rows_kernel<T, D, GRAD>), dim3(static_cast<unsigned>((rows + per - 1) / per)), dim3(256), 0, s, a, out);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t forward(PackArgs a, const PackCall &c, hipStream_t s) {
  PACK_TRY(prepare(a, c, c.forward, 1, s));
  a.list = c.forward;
  a.count = c.header;
  a.splits = c.splits_forward;
  PACK_TRY(sizeof(T) == 2 ? packed_queries(a, D, false, c.o, s) : packed_queries_f32(a, D, false, c.o, s));
  return a.splits > 1 ? join_rows<T, D, false>(a, c.o, s) : hipSuccess;
}

template <typename T, int D>
hipError_t backward(PackArgs a, const PackCall &c, hipStream_t s) {
  PACK_TRY(prepare(a, c, c.by_rows, 2, s));
  a.list = c.by_rows;
  a.count = c.header;
  a.splits = c.splits_rows;
  PACK_TRY(sizeof(T) == 2 ? packed_queries(a, D, true, c.dq, s) : packed_queries_f32(a, D, true, c.dq, s));
  if (a.splits > 1) PACK_TRY((join_rows<T, D, true>(a, c.dq, s)));
  a.list = c.by_keys;
  a.count = c.header + 1;
  a.splits = c.splits_keys;
  PACK_TRY(sizeof(T) == 2 ? packed_keys(a, D, c.dk, c.dv, s) : packed_keys_f32(a, D, c.dk, c.dv, s));
  if (a.splits > 1) {
    const size_t rows = static_cast<size_t>(a.kv_heads) * a.rows_k, per = 256 / (D / 4);
    hipLaunchKernelGGL((pack_join_keys_kernel<T, D>), dim3(static_cast<unsigned>((rows + per - 1) / per), 2), dim3(256), 0, s, a, c.dk, c.dv);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

size_t packed_workspace(const scope_pack *p, void *base, PackArgs *a, PackCall *c) {
  const bool bf16 = p->dtype == SCOPE_BF16;
  const int group = p->heads / p->kv_heads;
  const long long rows = static_cast<long long>(p->rows_q) * group, keys = p->rows_k;
  char *at = static_cast<char *>(base);
  size_t used = 0;
  auto take = [&](size_t bytes) {
    char *q = at ? at + used : nullptr;
    used = (used + bytes + 255) / 256 * 256;
    return q;
  };
  PackList by_rows{nullptr, bf16 ? kPackRows : kPackRowsF32, 0}, by_keys{nullptr, bf16 ? kPackKeys : kPackRowsF32, 0};
  by_rows.capacity = static_cast<int>(rows / by_rows.rows + p->sequences);
  by_keys.capacity = static_cast<int>(keys / by_keys.rows + p->sequences);
  // items that sequences of one length would give
  auto items_of = [&](long long n, int list_rows) { return p->kv_heads * ceil_div(ceil_div(n, p->sequences), list_rows) * p->sequences; };
  // Few queries of few sequences: items of 32 rows, whose keys a block's four waves share
  // out among them, where parts alone would leave most waves idle.  16 items behind caches
  // of up to 16000 keys 29 us for 38, 8 items 22 for 33, 32 items (8000 keys) 27 for 28, but
  // 48 items 35 for 34 and 64 items 40.5 for 39.5.
  const bool few = bf16 && rows <= static_cast<long long>(kPackFewRows) * p->sequences && items_of(rows, kPackFewRows) <= kFewItems;
  PackList forward = by_rows;
  if (few) forward.rows = kPackFewRows;
  forward.capacity = static_cast<int>(rows / forward.rows + p->sequences);
  int32_t *header = reinterpret_cast<int32_t *>(take(64));
  by_rows.items = forward.items = reinterpret_cast<int4 *>(take(32 * static_cast<size_t>(forward.capacity)));
  by_keys.items = reinterpret_cast<int4 *>(take(32 * static_cast<size_t>(by_keys.capacity)));
  float *stats = reinterpret_cast<float *>(take(8 * static_cast<size_t>(p->kv_heads) * rows));
  const int tile = bf16 ? 64 : 32;
  const long long key_tiles = ceil_div(ceil_div(keys, p->sequences), tile);
  const int splits_rows = parts_of(items_of(rows, by_rows.rows), key_tiles, bf16 ? 4 : 2, 1024);
  // An item of dK and dV writes 2 x 128 fp32 rows a part: short parts (2 tiles) only up to
  // the 512 blocks that the chip holds at once, long ones (8) beyond, to even out the ends.
  // bf16, 24 sequences of 760 tokens in all, 24 heads of 3: the whole backward 42 us for 64
  // with 8 alone; 11 sequences of 4996 tokens, 4 heads of one 134 for 145; but with 4 and
  // 2048 blocks alone 17 sequences of 13527 tokens, 2 heads, took 73 us for 60.
  const long long key_items = items_of(keys, by_keys.rows), row_tiles = ceil_div(ceil_div(rows, p->sequences), 32);
  const int fill = parts_of(key_items, row_tiles, 2, bf16 ? 512 : 1024), even = parts_of(key_items, row_tiles, 8, 2048);
  const int splits_keys = bf16 && even > fill ? even : fill;
  const int splits_forward = few ? parts_of(items_of(rows, kPackFewRows), key_tiles, 4, 256) : splits_rows;
  const int row_splits = splits_forward > splits_rows ? splits_forward : splits_rows;
  const size_t row_parts = row_splits > 1 ? static_cast<size_t>(row_splits) * p->kv_heads * rows * (4 * p->d + 8) : 0;
  const size_t key_parts = splits_keys > 1 ? static_cast<size_t>(splits_keys) * 2 * p->kv_heads * keys * 4 * p->d : 0;
  float *parts = reinterpret_cast<float *>(take(row_parts > key_parts ? row_parts : key_parts));
  if (a) {
    a->stats = stats;
    a->parts = parts;
    a->ends = header ? header + 2 : nullptr;
    c->by_rows = by_rows;
    c->forward = forward;
    c->splits_forward = splits_forward;
    c->by_keys = by_keys;
    c->header = header;
    c->splits_rows = splits_rows;
    c->splits_keys = splits_keys;
  }
  return used;
}

// Fewer than 2^32 threads a launch.  Joins run for at most 1024 items of 128 rows, of 32
// threads a row at most, and need no check.
bool packed_launchable(const scope_pack *p) {
  PackArgs a{};
  PackCall c{};
  packed_workspace(p, nullptr, &a, &c);
  auto fits = [p](long long capacity, int splits) {
    return (capacity * splits + 7) / 8 * 8 * p->kv_heads * kPackThreads < (1LL << 32);
  };
  return fits(c.by_rows.capacity, c.splits_rows) && fits(c.forward.capacity, c.splits_forward) && fits(c.by_keys.capacity, c.splits_keys);
}

hipError_t packed_forward(const PackArgs &a, const PackCall &c, hipStream_t s) {
  if (c.bf16) return c.d == 128 ? forward<uint16_t, 128>(a, c, s) : forward<uint16_t, 64>(a, c, s);
  return c.d == 128 ? forward<float, 128>(a, c, s) : forward<float, 64>(a, c, s);
}
hipError_t packed_backward(const PackArgs &a, const PackCall &c, hipStream_t s) {
  if (c.bf16) return c.d == 128 ? backward<uint16_t, 128>(a, c, s) : backward<uint16_t, 64>(a, c, s);
  return c.d == 128 ? backward<float, 128>(a, c, s) : backward<float, 64>(a, c, s);
}

}  // namespace scope
