// Rotary positions: pairs of channels turned by angles that grow with the token's
// position, y_a = f (x_a cos t - x_b sin t), y_b = f (x_a sin t + x_b cos t).
//
// A thread takes the same channels of one token in several heads, so that it forms
// their angles, sines and cosines once: 16 bytes of a row (SCOPE_HALVES: 16 bytes of
// either half) where alignment allows, else one pair.  Angles are fractions of a
// turn in integers: position times frequency modulo 2^64 wraps as the angle does, so
// position 2^24 is as exact as position 1.
//
// Bound by memory.  A 720p layer's queries and keys (24 + 24 heads x 118800 x 128 bf16)
// take 570 us, 5.1 TB/s read and written, where a copy by torch reaches 4.8; gradients of
// 5 + 5 heads x 32760, which leave the caches, 36 us (4.6 TB/s).  With at most 8 heads a
// thread and no loads ahead the gradients took 48, with at most 4 the layer 698: the
// angles cost a thread about as much as 4 heads' rows.
#include "common.h"
#include "kernels.h"
#include "mfma.h"

namespace scope {

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;   // heads loaded together
constexpr int kBlocks = 4;  // blocks of a CU that fill it

// sin and cos of u / 2^32 turns.  The nearest quarter turn is taken off in integers;
// what is left, |x| <= pi / 4, goes through the Taylor series (the first terms left
// out are below 2^-29).
__device__ __forceinline__ void sincos_turn(uint32_t u, float &s, float &c) {
  const uint32_t quarter = (u + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(u - (quarter << 30))) * 0x1.921fb6p-30f;  // 2 pi / 2^32
  const float x2 = x * x;
  float p = 1.0f / 362880.0f;
  p = fmaf(p, x2, -1.0f / 5040.0f);
  p = fmaf(p, x2, 1.0f / 120.0f);
  p = fmaf(p, x2, -1.0f / 6.0f);
  const float sx = fmaf(p * x2, x, x);
  float q = -1.0f / 3628800.0f;
  q = fmaf(q, x2, 1.0f / 40320.0f);
  q = fmaf(q, x2, -1.0f / 720.0f);
  q = fmaf(q, x2, 1.0f / 24.0f);
  q = fmaf(q, x2, -0.5f);
  const float cx = fmaf(q, x2, 1.0f);
  s = quarter & 1 ? cx : sx;
  c = quarter & 1 ? sx : cx;
  if (quarter & 2) s = -s;
  if ((quarter + 1) & 2) c = -c;
}

// The pairs that a thread holds of a row: N values at first, N at second (SCOPE_PAIRS
// with vectors: N / 2 pairs in one run of channels, second unused).
struct Unit {
  int first, second;  // channels; second < 0: none
  int axis, pair;     // of its first pair; axis < 0: copied
};

// The unit of halves or single elements: pairs first, then what is in no range.
template <int W>
__device__ __forceinline__ Unit half_unit(const RotaryArgs &a, int u) {
  int base = 0;
  for (int i = 0; i < a.axes; ++i) {
    const int units = a.len[i] / 2 / W;
    if (u < units) return {a.off[i] + W * u, a.off[i] + a.len[i] / 2 + W * u, i, base + W * u};
    u -= units;
    base += a.len[i] / 2;
  }
  int c = W * u;  // of the channels in no range; ranges come in ascending order of offset
  for (int i = 0; i < a.axes; ++i) {
    const int r = a.by_off[i];
    if (c >= a.off[r]) c += a.len[r];
  }
  return {c, -1, -1, 0};
}

// A vector as it lies in memory, and its values.
template <typename T, int N>
struct Raw {
  uint4 u;
  __device__ __forceinline__ void load(const T *p) { u = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void values(float (&x)[N]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
};
template <typename T>
struct Raw<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T *p) { v = *p; }
  __device__ __forceinline__ void values(float (&x)[1]) const { x[0] = load_elem(&v, 0); }
};
template <typename T, int N>
__device__ __forceinline__ void store_values(T *p, const float (&x)[N]) {
  if constexpr (N == 1) {
    if constexpr (sizeof(T) == 2)
      *p = static_cast<uint16_t>(pack_bf16(x[0], 0.0f));
    else
      *p = x[0];
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
  }
}

// PAIRS, vectors: a unit is the W channels of 16 bytes, whose pairs may lie in different
// ranges.  Otherwise a unit is W values of either half, or W copied ones (W = 1: alignment
// allows no more); pairs
// of single elements are halves one channel apart.
template <typename T, bool PAIRS, int W>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  const long long at = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
  const long long row = at / a.units;
  if (row >= a.rows) return;
  const int u = static_cast<int>(at - row * a.units);
  constexpr int P = PAIRS && W > 1 ? W / 2 : W;  // pairs of a unit
  constexpr bool TWO = !(PAIRS && W > 1);        // a pair's values lie in two places
  Unit unit{W * u, -1, -1, 0};
  if constexpr (PAIRS && W == 1) {
    unit = half_unit<1>(a, u);
    if (unit.axis >= 0) {
      unit.first = 2 * unit.first - a.off[unit.axis];
      unit.second = unit.first + 1;
    }
  } else if constexpr (!PAIRS) {
    unit = half_unit<W>(a, u);
  }
  const bool two = TWO && unit.axis >= 0;

  const int heads = a.heads[0] + a.heads[1];
  const int h0 = static_cast<int>(blockIdx.y) * a.per, h1 = min(h0 + a.per, heads);
  auto place = [&](int h, int &i) {  // the row of a head past the last is the last's
    const int hc = min(h, h1 - 1);
    i = hc >= a.heads[0] ? 1 : 0;
    return hc - (i ? a.heads[0] : 0);
  };
  // The next kAhead heads' loads go out before these are stored (which the compiler
  // cannot know to be elsewhere, or the same thread's), the first before the angles.
  Raw<T, W> raw[2][kAhead], raw2[2][TWO ? kAhead : 1];
  auto load = [&](int set, int hb) {
#pragma unroll
    for (int b = 0; b < kAhead; ++b) {
      int i;
      const int hh = place(hb + b, i);
      const T *x = static_cast<const T *>(a.x[i]) + hh * a.xs[i].head + row * a.xs[i].row;
      raw[set][b].load(x + unit.first);
      if constexpr (TWO)
        if (two) raw2[set][b].load(x + unit.second);
    }
  };
  load(0, h0);

  float cs[P], sn[P];
  bool turned[P];
  auto angle = [&](int axis, int pair, float &s, float &c) {
    const long long p = a.positions[static_cast<size_t>(axis) * a.rows + row];
    const uint64_t t = static_cast<uint64_t>(p) * a.turns[pair];
    sincos_turn(static_cast<uint32_t>(t >> 32), s, c);
    s *= a.inverse ? -a.factor : a.factor;
    c *= a.factor;
  };
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if constexpr (!TWO) {
      const int ch = W * u + 2 * j;
      int axis = -1, pair = 0, base = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        if (i < a.axes && ch >= a.off[i] && ch < a.off[i] + a.len[i]) {
          axis = i;
          pair = base + (ch - a.off[i]) / 2;
        }
        base += a.len[i] / 2;
      }
      turned[j] = axis >= 0;
      if (turned[j]) angle(axis, pair, sn[j], cs[j]);
    } else if (two) {
      angle(unit.axis, unit.pair + j, sn[j], cs[j]);
    }
  }

  auto turn = [&](int set, int hb) {
#pragma unroll
    for (int b = 0; b < kAhead; ++b) {
      if (hb + b >= h1) return;
      int i;
      const int hh = place(hb + b, i);
      T *y = static_cast<T *>(a.y[i]) + hh * a.ys[i].head + row * a.ys[i].row;
      float v[W];
      raw[set][b].values(v);
      if constexpr (!TWO) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const float p = v[2 * j], q = v[2 * j + 1];
          v[2 * j] = turned[j] ? fmaf(p, cs[j], -(q * sn[j])) : p;
          v[2 * j + 1] = turned[j] ? fmaf(p, sn[j], q * cs[j]) : q;
        }
      } else if (two) {
        float z[W];
        raw2[set][b].values(z);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float p = v[j], q = z[j];
          v[j] = fmaf(p, cs[j], -(q * sn[j]));
          z[j] = fmaf(p, sn[j], q * cs[j]);
        }
        store_values<T, W>(y + unit.second, z);
      }
      store_values<T, W>(y + unit.first, v);
    }
  };
  for (int hb = h0; hb < h1; hb += 2 * kAhead) {
    if (hb + kAhead < h1) load(1, hb + kAhead);
    turn(0, hb);
    if (hb + 2 * kAhead < h1) load(0, hb + 2 * kAhead);
    turn(1, hb + kAhead);
  }
}

template <typename T>
hipError_t run(const RotaryArgs &a, bool pairs, bool vectors, dim3 grid, hipStream_t s) {
  constexpr int W = 16 / sizeof(T);
  if (pairs && vectors)
    hipLaunchKernelGGL((rotary_kernel<T, true, W>), grid, dim3(kThreads), 0, s, a);
  else if (pairs)
    hipLaunchKernelGGL((rotary_kernel<T, true, 1>), grid, dim3(kThreads), 0, s, a);
  else if (vectors)
    hipLaunchKernelGGL((rotary_kernel<T, false, W>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((rotary_kernel<T, false, 1>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t rotary_run(const RotaryArgs &args, bool bf16, bool pairs, bool vectors, int d, hipStream_t s) {
  RotaryArgs a = args;
  int turned = 0;
  for (int i = 0; i < a.axes; ++i) turned += a.len[i];
  const int w = !vectors ? 1 : bf16 ? 8 : 4;
  a.units = pairs && vectors ? d / w : turned / 2 / w + (d - turned) / w;
  // Heads of a thread: all of them where the rows alone fill the chip.
  const long long threads = static_cast<long long>(a.rows) * a.units;
  const int heads = a.heads[0] + a.heads[1];
  const long long groups = (256LL * kBlocks * kThreads + threads - 1) / threads;
  a.per = groups < heads ? static_cast<int>((heads + groups - 1) / groups) : 1;
  if (a.per > kAhead) a.per = (a.per + kAhead - 1) / kAhead * kAhead;
  const dim3 grid(static_cast<unsigned>((threads + kThreads - 1) / kThreads), static_cast<unsigned>((heads + a.per - 1) / a.per));
  return bf16 ? run<uint16_t>(a, pairs, vectors, grid, s) : run<float>(a, pairs, vectors, grid, s);
}

}  // namespace scope
