// Dropout of a tensor: y = x / (1 - p) where kept, else 0, plus a residual.
// Eight neighbouring elements share one Philox call (eight 16-bit numbers), so
// nothing but x, the residual and y passes through memory; the gradient is the
// same call on the gradient of y.
//
// Bound by memory: 365 M fp32 values 499 us, 5.9 TB/s read and written (a copy by
// torch 4.8); 21 M bf16 values with a residual, which the last-level cache holds, 20 us.
// One group per thread without a loop of loads: the chip holds enough of them.
#include "common.h"
#include "kernels.h"
#include "mfma.h"
#include "noise.h"

namespace scope {

namespace {

template <typename T>
__device__ __forceinline__ T from_f32(float f) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));
  } else {
    return f;
  }
}

// One thread per group of eight elements.  VEC: every pointer is 16-byte
// aligned, whole groups move as vectors.
template <typename T, bool RES, bool VEC>
__global__ __launch_bounds__(256) void dropout_kernel(int64_t count, const T *x, const T *residual, uint32_t threshold,
                                                      float scale, const uint64_t *__restrict__ rng, T *y) {
  const Stream stream(rng);
  const int64_t groups = (count + 7) / 8;
  for (int64_t g = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; g < groups;
       g += static_cast<int64_t>(gridDim.x) * 256) {
    const uint4 w = philox(make_uint4(static_cast<uint32_t>(g), static_cast<uint32_t>(g >> 32), stream.at.x, stream.at.y),
                           stream.key);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    auto value = [&](int e, float v, float r) {
      const uint32_t number = e & 1 ? u[e >> 1] >> 16 : u[e >> 1] & 0xFFFFu;
      const float kept = number >= threshold ? v * scale : 0.0f;
      return RES ? kept + r : kept;
    };
    const int64_t at = 8 * g;
    if (VEC && at + 8 <= count) {
      __attribute__((aligned(16))) T v[8], r[8];
      constexpr int PARTS = 8 * sizeof(T) / 16;
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        reinterpret_cast<uint4 *>(v)[i] = reinterpret_cast<const uint4 *>(x + at)[i];
        if (RES) reinterpret_cast<uint4 *>(r)[i] = reinterpret_cast<const uint4 *>(residual + at)[i];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = from_f32<T>(value(e, load_elem(v, e), RES ? load_elem(r, e) : 0.0f));
#pragma unroll
      for (int i = 0; i < PARTS; ++i) reinterpret_cast<uint4 *>(y + at)[i] = reinterpret_cast<uint4 *>(v)[i];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < count)
          y[at + e] = from_f32<T>(value(e, load_elem(x, at + e), RES ? load_elem(residual, at + e) : 0.0f));
    }
  }
}

template <typename T, bool RES>
hipError_t run(int64_t count, const void *x, const void *residual, uint32_t threshold, const uint64_t *rng, void *y,
               hipStream_t s) {
  const int64_t blocks = ((count + 7) / 8 + 255) / 256;
  const dim3 grid(static_cast<unsigned>(blocks < (1 << 20) ? blocks : (1 << 20)));
  const float scale = 65536.0f / static_cast<float>(65536 - threshold);
  const bool vec = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(residual) | reinterpret_cast<uintptr_t>(y)) & 15) == 0;
  if (vec)
    hipLaunchKernelGGL((dropout_kernel<T, RES, true>), grid, dim3(256), 0, s, count, static_cast<const T *>(x),
                       static_cast<const T *>(residual), threshold, scale, rng, static_cast<T *>(y));
  else
    hipLaunchKernelGGL((dropout_kernel<T, RES, false>), grid, dim3(256), 0, s, count, static_cast<const T *>(x),
                       static_cast<const T *>(residual), threshold, scale, rng, static_cast<T *>(y));
  return hipGetLastError();
}

}  // namespace

hipError_t dropout_run(bool bf16, int64_t count, const void *x, const void *residual, uint32_t threshold,
                       const uint64_t *rng, void *y, hipStream_t s) {
  if (bf16)
    return residual ? run<uint16_t, true>(count, x, residual, threshold, rng, y, s)
                    : run<uint16_t, false>(count, x, nullptr, threshold, rng, y, s);
  return residual ? run<float, true>(count, x, residual, threshold, rng, y, s)
                  : run<float, false>(count, x, nullptr, threshold, rng, y, s);
}

}  // namespace scope
