// linear_kernels.hpp - what the kernels of a layer and of its gradients share.
//
//   forward  y = act([x | x2] w^T + bias) + residual
//   dx       dz w              dz = dy * act'(pre), taken as it is read
//   dw       dz^T [x | x2], dbias = sum of dz over the rows
//
// with the matrix unit's 32x32 products (bf16: 16 k at a time; fp32: 2), fp32
// accumulators: linear_few.hpp has y and dx over few rows, linear_stream.hpp
// over many, linear_weights.hpp dw.
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

constexpr int kLinNT = 256;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// ------------------------------------------------------------- activations
// gelu by the tail q = 1 - Phi(s), s = |z|: z q below 0 and z - z q above, so
// that small results are products and no differences.
//   q = exp(-s^2 / 2) t P(t), t = 1 / (1 + 0.34 s),
// P a polynomial of degree 6 with the least largest |error| / (q + 1e-5) for s
// up to 14 (fitted in 64 bits): 7.7e-8. Exponentials and reciprocals are the
// hardware's, one unit in the last place. Over 300K normal values in fp32 the
// root of the mean squared error is 2.2e-8 for gelu and 3.7e-8 for its slope
// (2.5e-8 and 2.6e-8 for the formulas with erf, each operation rounded to
// fp32), and down to z = -6 both are 3e-6 of their size off. The slope shares
// the exponential and is ~20 instructions, where the compiler's erfcf and expf
// made a wide layer's gradients in fp32 half as slow again as the matrix unit
// is.
constexpr float kTailP = 0.34f;
constexpr float kLog2e = 1.44269504f;

// P(t)
__device__ __forceinline__ float tail_poly(float t) {
  return 0.13619301f + t * (0.128087512f + t * (0.163103034f + t * (-0.0440031517f + t * (0.278884839f + t * (-0.209133778f + t * 0.0468685945f)))));
}
// exp(-z^2 / 2) and 1 / (1 + exp(-z))
__device__ __forceinline__ float bell(float z) { return __builtin_amdgcn_exp2f(z * (z * (-0.5f * kLog2e))); }
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z)); }

__device__ __forceinline__ float act_value(float z, int act) {
  if (act == kActRelu) return z <= 0.0f ? 0.0f : z;  // a NaN stays one
  if (act == kActGelu) {
    const float t = __builtin_amdgcn_rcpf(1.0f + kTailP * fabsf(z));
    const float q = bell(z) * (t * tail_poly(t));
    return z < 0.0f ? z * q : z - fminf(z, 40.0f) * q;  // (infinity times a q of 0 would be a NaN)
  }
  return act == kActSilu ? z * logistic(z) : z;
}

// g * act'(z). A slope's products with z are taken with z held within bounds
// beyond which the other factor is 0, so that infinities have their limits'
// slopes; a NaN stays one by the exponential.
__device__ __forceinline__ float act_grad(float g, float z, int act) {
  if (act == kActRelu) return z > 0.0f ? g : 0.0f;
  if (act == kActGelu) {
    // Phi(z) + z phi(z) is r below 0 and 1 - r above, r = (1 - Phi(s)) - s phi(s)
    const float s = fminf(fabsf(z), 40.0f);
    const float t = __builtin_amdgcn_rcpf(1.0f + kTailP * s);
    const float r = bell(z) * (t * tail_poly(t) - 0.39894228f * s);
    return g * (z < 0.0f ? r : 1.0f - r);
  }
  const float s = fminf(fmaxf(z, -100.0f), 100.0f), q = logistic(z);
  return g * (q + q * (s - s * q));
}

// The same for several values: the activation is the same for all of them.
__device__ __forceinline__ void act_values(float (&z)[8], int act) {
  if (act == kActNone) return;
  if (act == kActRelu) {
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] = act_value(z[q], kActRelu);
  } else if (act == kActGelu) {
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] = act_value(z[q], kActGelu);
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] = act_value(z[q], kActSilu);
  }
}
// g becomes dz, rounded to T as the matrix unit takes it; exact(q, value) gets it in fp32.
// In bf16 this is a rounding of its own (exact for the identity and relu): it puts
// the gradients' error at 0.0023 of them, where the results' own rounding leaves
// 0.0017. The 8 bits that it drops, in products of their own, would halve the
// matrix unit's rate, and 0 times an infinity there is a NaN in place of it.
template <typename T, int Q, typename Keep>
__device__ __forceinline__ void act_grads(cols_t<T, Q>& g, const cols_t<T, Q>& z, int act, Keep exact) {
  auto each = [&](int of) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const float v = act_grad((float)g[q], (float)z[q], of);
      exact(q, v);
      g[q] = (T)v;
    }
  };
  if (act == kActRelu) each(kActRelu);
  else if (act == kActGelu) each(kActGelu);
  else each(kActSilu);
}

// ---------------------------------------------------------------- operands
// One operand of a product: element (r, k), r below R, k below K, is at
// p[r * stride + k]; with pre, it is p's times the activation's slope at
// pre's.
template <typename T>
struct Operand {
  const T* p;
  const T* pre;
  int64_t stride, pre_stride;
  int64_t R, K;
  int act;
};

// The weights of a segment of the reduction: those of output n and column k are
// at p[n * stride + k] (along k) or p[k * stride + n] (across k).
template <typename T>
struct Weights {
  const T* p;
  int64_t stride;
};

// A lane of the matrix unit takes 16 bytes of neighbouring k: those from k on
// where they are all there; the segment's last 16 bytes, of which only those
// from k on count, at its end; none behind it. skipped() is the number of
// elements left out (16 bytes' worth for none), without() clears them, and both
// operands of a product are read this way. A segment of under 16 bytes is read
// value by value.
template <typename T>
__device__ __forceinline__ int skipped(int64_t k, int64_t K) {
  constexpr int kV = 16 / sizeof(T);
  return k + kV <= K ? 0 : k < K ? (int)(k + kV - K) : kV;
}
template <typename T>
__device__ __forceinline__ u32x4 without(u32x4 v, int skip) {
  constexpr int kPer = 4 / sizeof(T);  // elements per word
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int left = skip - q * kPer;  // elements of this word to clear
    v[q] = left >= kPer ? 0u : left == 1 && kPer == 2 ? v[q] & 0xFFFF0000u : v[q];
  }
  return v;
}

// The 16 bytes of k that begin at k of a row that runs along k.
template <typename T>
__device__ __forceinline__ u32x4 k_along(const T* row, int64_t k, int64_t K) {
  constexpr int kV = 16 / sizeof(T);
  u32x4 v = (u32x4)0u;
  if (K >= kV) {
    const int skip = skipped<T>(k, K);
    if (skip < kV) v = without<T>(__builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(row + (skip ? K - kV : k))), skip);
  } else {
    cols_t<T, kV> t;
#pragma unroll
    for (int q = 0; q < kV; ++q) t[q] = k + q < K ? row[k + q] : (T)0.0f;
    v = __builtin_bit_cast(u32x4, t);
  }
  return v;
}
// Blocks are dealt to the eight XCDs in turn; consecutive tiles (which share
// rows of A) go to one XCD, whose L2 then serves them.
__device__ __forceinline__ int64_t tile_of_block(int64_t b, int64_t blocks) {
  constexpr int64_t kXcds = 8;
  const int64_t per = blocks / kXcds, rest = blocks % kXcds, x = b % kXcds;
  return x * per + min(x, rest) + b / kXcds;
}

// ----------------------------------------------------------------- forward
template <typename T>
struct LinearForward {
  Operand<T> x[2];
  Weights<T> w[2];  // of each input's columns, along k
  const T *bias, *residual;
  T *y, *pre;
  int64_t residual_stride, y_stride, pre_stride;
  int64_t rows;
  int n, act;
};

// The epilogue of one output, z its product with the bias added.
template <typename T>
__device__ __forceinline__ void linear_finish(const LinearForward<T>& a, int64_t row, int col, float z) {
  if (a.pre) a.pre[row * a.pre_stride + col] = (T)z;
  z = act_value(z, a.act);
  if (a.residual) z += (float)a.residual[row * a.residual_stride + col];
  a.y[row * a.y_stride + col] = (T)z;
}

// ---------------------------------------------------------------------- dx
// The columns asked for, of the first input and then of the second, as one row.
template <typename T>
struct LinearDx {
  Operand<T> dz;
  Weights<T> w;  // of those columns, across k
  T* dx[2];
  int64_t dx_stride[2];
  int64_t rows;
  int cols, split;  // column split is the second input's first
};

template <typename T>
__device__ __forceinline__ void linear_dx_store(const LinearDx<T>& a, int64_t row, int col, float v) {
  const int s = col >= a.split ? 1 : 0;
  a.dx[s][row * a.dx_stride[s] + col - (s ? a.split : 0)] = (T)v;
}
// Eight of them, all there.
template <typename T>
__device__ __forceinline__ void linear_dx_store(const LinearDx<T>& a, int64_t row, int col, const float (&v)[8]) {
  if (col < a.split && col + 8 > a.split) {
#pragma unroll
    for (int q = 0; q < 8; ++q) linear_dx_store(a, row, col + q, v[q]);
    return;
  }
  const int s = col >= a.split ? 1 : 0;
  store_cols<T, 8, false>(a.dx[s] + row * a.dx_stride[s] + col - (s ? a.split : 0), 8, v);
}

// -------------------------------------------------------------------- join
// Adds the parts, of dw (rows of `cols` values) and of dbias: four threads a
// value, each over a quarter of the parts.
constexpr int kJoinWays = 4;
template <typename T>
__global__ __launch_bounds__(kLinNT) void k_linear_join(const float* __restrict__ dw_parts, const float* __restrict__ bias_parts,
                                                        int64_t parts, int n, int cols, T* __restrict__ dw, int64_t dw_stride,
                                                        T* __restrict__ dbias) {
  constexpr int kValues = kLinNT / kJoinWays;
  __shared__ float sums[kJoinWays][kValues];
  const int way = threadIdx.x / kValues;
  const int64_t in_dw = dw_parts ? (int64_t)n * cols : 0, all = in_dw + (bias_parts ? n : 0);
  const int64_t i = (int64_t)blockIdx.x * kValues + threadIdx.x % kValues;
  const bool bias = i >= in_dw;
  const float* p = bias ? bias_parts + (i - in_dw) : dw_parts + i;
  const int64_t step = bias ? n : in_dw, per = (parts + kJoinWays - 1) / kJoinWays;
  float t = 0.0f;
  if (i < all) {
#pragma unroll 8
    for (int64_t q = way * per; q < min(parts, (way + 1) * per); ++q) t += p[q * step];
  }
  sums[way][threadIdx.x % kValues] = t;
  __syncthreads();
  if (way || i >= all) return;
#pragma unroll
  for (int w = 1; w < kJoinWays; ++w) t += sums[w][threadIdx.x];
  if (bias) dbias[i - in_dw] = (T)t;
  else dw[i / cols * dw_stride + i % cols] = (T)t;
}

}  // namespace ms
