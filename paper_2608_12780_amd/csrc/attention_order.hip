// An order of the keys for dK and dV.
//
// The gradient kernels run the 32 keys of a wave (fp32: 16) against every query tile whose cluster
// keeps one of them, so keys in token order waste what their neighbours' sets do not
// share: on the sparse layer's own sets (5 heads x 32760 tokens, 128 clusters) 43%
// of the products at 54% kept keys, 72% at 15% (dK and dV take 5.44 ms for 4.79 in
// the order below, 4.88 for 3.22).  Keys that the same clusters keep
// belong together.  A key's signature are its bits in 12 clusters, spread over the
// list; keys are sorted by it, signatures in the order of the reflected Gray code,
// where neighbours differ in one cluster.  A head uses the order where it leaves
// fewer (wave, tile) pairs, by 3%; where sets follow the token order it does not.
// Finite gradients are the same bit for bit in any order: every key's sums have their
// own column of the matrix products and run over the same tiles, a tile that does
// not keep the key adding zeros.  A NaN or infinity in Q or dO makes NaN of such a
// zero, in the keys that share a wave; so the order is the same on every run as well:
// the sort is stable, keys of one signature ascend.
#include "common.h"
#include "kernels.h"

namespace scope {

namespace {

constexpr int kBits = 12;
static_assert(kOrderBins == 1 << kBits, "a bin per signature");
constexpr int kWords = kTrainMaskKeys / 32;

__device__ __forceinline__ size_t mask_row(const TrainArgs &a, int h, int block, int c) {
  return ((static_cast<size_t>(h) * ((a.n + kTrainMaskKeys - 1) / kTrainMaskKeys) + block) * a.c_q + c) * kWords;
}

// A block counts its keys by signature in LDS; its counts become the places where
// its keys of a signature start.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortKeys = 4;  // keys per thread
static_assert(kOrderKeys == kSortThreads * kSortKeys, "keys of a block");

__device__ __forceinline__ uint32_t *starts_of(const TrainArgs &a, int h, int block, int blocks) {
  return a.order.start + (static_cast<size_t>(h) * blocks + block) * kOrderBins;
}

__global__ __launch_bounds__(kSortThreads) void order_count_kernel(TrainArgs a) {
  __shared__ uint32_t count[kOrderBins];
  const int h = blockIdx.y, t = threadIdx.x;
  for (int i = t; i < kOrderBins; i += kSortThreads) count[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortKeys; ++i) {
    const int key = (blockIdx.x * kSortKeys + i) * kSortThreads + t;
    if (key >= a.n) break;
    uint32_t gray = 0;
#pragma unroll
    for (int x = 0; x < kBits; ++x) {
      const int c = (2 * x + 1) * a.c_q / (2 * kBits);
      const uint32_t w = a.masks[mask_row(a, h, key / kTrainMaskKeys, c) + key % kTrainMaskKeys / 32];
      gray = 2 * gray + (w >> (key & 31) & 1u);
    }
    // the signature's place in the Gray code's sequence
    uint32_t bin = gray;
#pragma unroll
    for (int s = 1; s < kBits; s *= 2) bin ^= bin >> s;
    a.order.bin[static_cast<size_t>(h) * a.n + key] = static_cast<uint16_t>(bin);
    atomicAdd(&count[bin], 1u);
  }
  __syncthreads();
  uint32_t *to = starts_of(a, h, blockIdx.x, gridDim.x);
  for (int i = t; i < kOrderBins; i += kSortThreads) to[i] = count[i];
}

// Counts to first positions: signature by signature, in each block by block.
__global__ __launch_bounds__(1024) void order_scan_kernel(TrainArgs a, int blocks) {
  __shared__ uint32_t wtot[16];
  static_assert(kOrderBins == 4 * 1024, "four signatures per thread");
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  uint4 *start = reinterpret_cast<uint4 *>(starts_of(a, blockIdx.x, 0, blocks)) + t;
  constexpr int STEP = kOrderBins / 4;
  uint4 k = make_uint4(0, 0, 0, 0);
#pragma unroll 8
  for (int b = 0; b < blocks; ++b) {
    const uint4 x = start[static_cast<size_t>(b) * STEP];
    k = make_uint4(k.x + x.x, k.y + x.y, k.z + x.z, k.w + x.w);
  }
  const uint32_t mine = k.x + k.y + k.z + k.w, incl = wave_incl_scan(mine);
  if (lane == 63) wtot[w] = incl;
  __syncthreads();
  uint32_t at = incl - mine;
  for (int i = 0; i < w; ++i) at += wtot[i];
  uint4 next = make_uint4(at, at + k.x, at + k.x + k.y, at + k.x + k.y + k.z);
  // eight loads before their stores, which they may not pass
  for (int b = 0; b < blocks; b += 8) {
    uint4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = start[static_cast<size_t>(min(b + i, blocks - 1)) * STEP];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (b + i >= blocks) break;
      start[static_cast<size_t>(b + i) * STEP] = next;
      next = make_uint4(next.x + x[i].x, next.y + x[i].y, next.z + x[i].z, next.w + x[i].w);
    }
  }
}

// A wave ranks 256 consecutive keys, 64 at a time, among those of their signature:
// after the wave's earlier keys, which its own counters hold, come those of lower
// lanes, which the signature's bits find in 12 votes.  No two waves share a counter,
// so nothing depends on who comes first.  5 heads x 32760: 10 us, and 7 with counters
// that a block's waves shared, in an order that varied.
__global__ __launch_bounds__(kSortThreads) void order_place_kernel(TrainArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t count[kSortWaves][kOrderBins];
  const int h = blockIdx.y, t = threadIdx.x, lane = t & 63, w = t >> 6;
  const size_t first = static_cast<size_t>(h) * a.n;
  const int from = blockIdx.x * kOrderKeys + w * 64 * kSortKeys + lane;
  int bin[kSortKeys], rank[kSortKeys];
#pragma unroll
  for (int i = 0; i < kSortKeys; ++i) bin[i] = from + 64 * i < a.n ? a.order.bin[first + from + 64 * i] : -1;
  for (int i = lane; i < kOrderBins / 8; i += 64) reinterpret_cast<uint4 *>(count[w])[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < kSortKeys; ++i) {
    unsigned long long same = __ballot(bin[i] >= 0);
#pragma unroll
    for (int b = 0; b < kBits; ++b) {
      const bool bit = bin[i] >> b & 1;
      const unsigned long long votes = __ballot(bit);
      same &= bit ? votes : ~votes;
    }
    const int below = __popcll(same & ((1ull << lane) - 1ull));
    // the counters are the wave's own: its LDS accesses keep their order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int before = bin[i] >= 0 ? count[w][bin[i]] : 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (bin[i] >= 0 && below == 0) count[w][bin[i]] = static_cast<uint16_t>(before + __popcll(same));
    rank[i] = before + below;
  }
  __syncthreads();
  // the waves' counts to what the block's earlier waves hold
  for (int i = t; i < kOrderBins; i += kSortThreads) {
    int sum = 0;
#pragma unroll
    for (int x = 0; x < kSortWaves; ++x) {
      const int k = count[x][i];
      count[x][i] = static_cast<uint16_t>(sum);
      sum += k;
    }
  }
  __syncthreads();
  const uint32_t *start = starts_of(a, h, blockIdx.x, gridDim.x);
#pragma unroll
  for (int i = 0; i < kSortKeys; ++i) {
    if (bin[i] < 0) continue;
    const uint32_t at = start[bin[i]] + count[w][bin[i]] + rank[i];
    if (at < static_cast<uint32_t>(a.n)) a.order.key[first + at] = from + 64 * i;
  }
}

// The key bits by position, and what both orders cost: (wave, tile) pairs.
__global__ __launch_bounds__(256) void order_masks_kernel(TrainArgs a) {
  const int b = blockIdx.x, h = blockIdx.y, t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int pos = b * 256 + t;
  const int key = pos < a.n ? a.order.key[static_cast<size_t>(h) * a.n + pos] : 0;
  const uint32_t *from = a.masks + mask_row(a, h, key / kTrainMaskKeys, 0) + key % kTrainMaskKeys / 32;
  const size_t row = mask_row(a, h, b, 0) + 2 * w;
  const int32_t *off = a.offsets + static_cast<size_t>(h) * (a.c_q + 1);
  unsigned long long by_key = 0, by_position = 0;
  const int per = (a.c_q + gridDim.z - 1) / gridDim.z, c0 = blockIdx.z * per;
#pragma unroll 4
  for (int c = c0; c < min(c0 + per, a.c_q); ++c) {
    const unsigned long long votes = __ballot(pos < a.n && (from[c * kWords] >> (key & 31) & 1u));
    const uint32_t lo = static_cast<uint32_t>(votes), hi = static_cast<uint32_t>(votes >> 32);
    if (lane == 0) *reinterpret_cast<uint2 *>(a.order.masks + row + c * kWords) = make_uint2(lo, hi);
    const uint2 old = *reinterpret_cast<const uint2 *>(a.masks + row + c * kWords);
    const unsigned long long tiles = (max(off[c + 1] - off[c], 0) + 31) / 32;
    by_key += tiles * ((old.x != 0) + (old.y != 0));
    by_position += tiles * ((lo != 0) + (hi != 0));
  }
  __shared__ unsigned long long sum[2];
  if (t < 2) sum[t] = 0;
  __syncthreads();
  if (lane == 0) {
    atomicAdd(&sum[0], by_key);
    atomicAdd(&sum[1], by_position);
  }
  __syncthreads();
  // spread over a head's slots: one counter for all blocks was most of the kernel
  if (t < 2) atomicAdd(&a.order.cost[(static_cast<size_t>(h) * kOrderSlots + (b + blockIdx.z) % kOrderSlots) * 2 + t], sum[t]);
}

}  // namespace

// The order takes four launches, 20 to 50 us, which few keys do not earn: the whole
// backward pass with it for the time without, 8 heads, d = 128, 8 to 96 clusters:
//   tokens             2048        4096        8192       16384 (4 heads)
//   sets of whole groups of scattered keys, 20% kept
//                 1.01-1.10   0.84-0.97   0.70-0.84   0.59-0.68
//   each key at random, 50% kept
//                 1.09-1.11   0.99-1.06   0.95-1.02   0.94-1.01
//   sets of runs of 128 tokens, 30% kept (the order is found and not used)
//                 1.13-1.19   1.09-1.12   1.04-1.07   1.03-1.04
// fp32, whose products take longer, 4 heads (up to 2048: 8), 8 to 64 clusters:
//   tokens             1024        2048        4096        8192
//   groups        0.93-1.02   0.75-0.97   0.68-0.91   0.62-0.68
//   random        1.04-1.08   1.00-1.04   1.01-1.02   1.00-1.02
//   runs          1.09-1.10   1.04-1.06   1.04-1.05   1.01-1.02
// so from 4096 tokens on fp32 would gain 9 to 32% with grouped sets and lose up to 5%
// with others; it has bf16's bound.
// Fewer than 8 clusters were not measured: such sets share most blocks of 32 keys.
bool train_orders_keys(int n, int c_q) { return n >= 8192 && c_q >= 8; }

// After the costs have been cleared.
hipError_t train_order(const TrainArgs &a, int heads, hipStream_t s) {
  const dim3 grid((a.n + kOrderKeys - 1) / kOrderKeys, heads);
  hipLaunchKernelGGL(order_count_kernel, grid, dim3(kSortThreads), 0, s, a);
  hipLaunchKernelGGL(order_scan_kernel, dim3(heads), dim3(1024), 0, s, a, static_cast<int>(grid.x));
  hipLaunchKernelGGL(order_place_kernel, grid, dim3(kSortThreads), 0, s, a);
  // the clusters in eighths: its loads are scattered words
  hipLaunchKernelGGL(order_masks_kernel, dim3((a.n + 255) / 256, heads, 8), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace scope
