// linear_few.hpp - the layer's products over few rows: y and dx.
//
// A block of eight waves makes 32 rows by 32 outputs. The waves share the
// reduction: each takes every eighth step of 32 bytes of k, reads both operands
// straight into the matrix unit's registers, a few steps at a time, and the
// block adds the eight sums in order. With few rows there are few tiles, and a
// call lasts as long as one of them: a handful of memory latencies. Measured: 16 rows,
// 128 + 128 -> 256 in fp32 7.8 us, of which the products are 0.1.
#pragma once

#include "linear_kernels.hpp"

namespace ms {

constexpr int kFewNT = 512;
constexpr int kFewAhead = 4;  // steps whose reads are under way at a time

// k_along() of a column.
template <typename T>
__device__ __forceinline__ u32x4 k_across(const T* column, int64_t stride, int64_t k, int64_t K) {
  constexpr int kV = 16 / sizeof(T);
  cols_t<T, kV> t = (cols_t<T, kV>)(T)0.0f;
  const int skip = K >= kV ? skipped<T>(k, K) : 0;
  const int64_t from = skip ? K - kV : k;
  if (skip < kV) {
#pragma unroll
    for (int q = 0; q < kV; ++q)
      if (q >= skip && from + q < K) t[q] = column[(from + q) * stride];
  }
  return __builtin_bit_cast(u32x4, t);
}

// out(row, column, value) for the rows [r0, r0 + 32) and outputs [n0, n0 + 32)
// that there are.
template <typename T, bool SLOPE, bool ACROSS, int SEGMENTS, typename F>
__device__ __forceinline__ void few_product(const Operand<T> (&x)[SEGMENTS], const Weights<T> (&w)[SEGMENTS], int64_t r0, int64_t rows, int n0, int n, F out) {
  constexpr int kV = 16 / sizeof(T);
  __shared__ __align__(16) float sums[kFewNT / MS_WAVE][32 * 32];
  const int lane = lane_id(), half = lane / 32;
  const int wave = wave_uniform((int32_t)wave_id());
  const int64_t row = min(r0 + lane % 32, rows - 1);  // rows and outputs that are not there repeat the last one
  const int64_t col = min(n0 + lane % 32, n - 1);
  f32x16 acc = {};
#pragma unroll 1
  for (int g = 0; g < SEGMENTS; ++g) {
    const Operand<T>& o = x[g];
    const int64_t steps = (o.K + 2 * kV - 1) / (2 * kV);
    const T *xr = o.p + row * o.stride, *zr = SLOPE ? o.pre + row * o.pre_stride : nullptr;
    const T* wr = w[g].p + (ACROSS ? col : col * w[g].stride);
#pragma unroll 1
    for (int64_t s0 = wave; s0 < steps; s0 += kFewAhead * (kFewNT / MS_WAVE)) {
      u32x4 a[kFewAhead], z[SLOPE ? kFewAhead : 1], b[kFewAhead];
#pragma unroll
      for (int u = 0; u < kFewAhead; ++u) {
        const int64_t k = ((s0 + u * (kFewNT / MS_WAVE)) * 2 + half) * kV;  // steps behind the last one are zeros
        a[u] = k_along(xr, k, o.K);
        if constexpr (SLOPE) z[u] = k_along(zr, k, o.K);
        b[u] = ACROSS ? k_across(wr, w[g].stride, k, o.K) : k_along(wr, k, o.K);
      }
#pragma unroll
      for (int u = 0; u < kFewAhead; ++u) {
        if constexpr (SLOPE) {
          cols_t<T, kV> d = __builtin_bit_cast(cols_t<T, kV>, a[u]);
          act_grads<T, kV>(d, __builtin_bit_cast(cols_t<T, kV>, z[u]), o.act, [](int, float) {});
          a[u] = __builtin_bit_cast(u32x4, d);
        }
        if constexpr (sizeof(T) == 2) {
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[u]), __builtin_bit_cast(bf16x8, b[u]), acc, 0, 0, 0);
        } else {
          const f32x4 fa = __builtin_bit_cast(f32x4, a[u]), fb = __builtin_bit_cast(f32x4, b[u]);
#pragma unroll
          for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[q], fb[q], acc, 0, 0, 0);
        }
      }
    }
  }
  // (accumulator register g of a lane is row 8 (g / 4) + 4 (lane / 32) + g % 4, column lane % 32)
#pragma unroll
  for (int g = 0; g < 16; ++g) sums[wave][(8 * (g / 4) + 4 * half + g % 4) * 32 + lane % 32] = acc[g];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 1024 / kFewNT; ++i) {
    const int at = threadIdx.x + i * kFewNT;
    float t = 0.0f;
#pragma unroll
    for (int v = 0; v < kFewNT / MS_WAVE; ++v) t += sums[v][at];
    if (r0 + at / 32 < rows && n0 + at % 32 < n) out(r0 + at / 32, n0 + at % 32, t);
  }
}

template <typename T>
__global__ __launch_bounds__(kFewNT) void k_linear_few(LinearForward<T> a, int tiles_n) {
  few_product<T, false, false, 2>(a.x, a.w, (int64_t)(blockIdx.x / tiles_n) * 32, a.rows, (int)(blockIdx.x % tiles_n) * 32, a.n,
                               [&](int64_t row, int col, float z) { linear_finish(a, row, col, a.bias ? z + (float)a.bias[col] : z); });
}

template <typename T, bool SLOPE>
__global__ __launch_bounds__(kFewNT) void k_linear_dx_few(LinearDx<T> a, int tiles_n) {
  const Operand<T> dz[1] = {a.dz};
  const Weights<T> w[1] = {a.w};
  few_product<T, SLOPE, true, 1>(dz, w, (int64_t)(blockIdx.x / tiles_n) * 32, a.rows, (int)(blockIdx.x % tiles_n) * 32, a.cols,
                                 [&](int64_t row, int col, float v) { linear_dx_store(a, row, col, v); });
}

}  // namespace ms
