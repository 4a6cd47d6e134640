// dropout_kernels.hpp - residual + dropout(x), the mask drawn where it is used.
//
//   y[i][j] = residual[i][j] + (word >= p 2^32 ? x[i][j] / (1 - p) : 0)
//
// word j % 4 of Philox4x32-10 at the counter (j / 4, i, draw, 0) under the
// call's seed: a column's fate hangs on its place alone, not on strides, types
// or the launch, so the gradient draws the same mask again and nothing of it is
// stored. A block of the generator serves four columns of a row.
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

constexpr int kDropNT = 256;
constexpr int kDropAhead = 2;  // rows of a team that are on their way together

template <typename T>
struct Dropout {
  const T *x, *residual;
  T* y;
  const uint64_t* seed_at;  // where the seed is, or null: `seed`
  uint64_t seed;
  int64_t rows, x_stride, residual_stride, y_stride;
  uint32_t draw, below;  // words under `below` drop their column
  int32_t d;
  bool all;  // every column drops
  float scale;
};

// Philox4x32-10: ten rounds over four words, the key raised between them.
__device__ __forceinline__ uint4 philox_block(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ (k0 + r * 0x9E3779B9u);
    c2 = (uint32_t)(a >> 32) ^ c3 ^ (k1 + r * 0xBB67AE85u);
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
  }
  return make_uint4(c0, c1, c2, c3);
}

template <typename T, int T_LANES>
__global__ __launch_bounds__(kDropNT) void k_dropout(Dropout<T> a) {
  constexpr int Q = 16 / sizeof(T), kTeams = kDropNT / T_LANES;
  const int lane = threadIdx.x % T_LANES;
  const uint64_t seed = a.seed_at ? *a.seed_at : a.seed;
  const uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  const int64_t step = (int64_t)gridDim.x * kTeams;
  for (int64_t i0 = (int64_t)blockIdx.x * kTeams + threadIdx.x / T_LANES; i0 < a.rows; i0 += kDropAhead * step) {
    for (int c = lane * Q; c < a.d; c += T_LANES * Q) {
      float x[kDropAhead][Q], res[kDropAhead][Q];
#pragma unroll
      for (int u = 0; u < kDropAhead; ++u) {
        const int64_t i = i0 + u * step;
        if (i >= a.rows) continue;
        load_cols<T, Q>(a.x + i * a.x_stride + c, a.d - c, x[u]);
        if (a.residual) load_cols<T, Q>(a.residual + i * a.residual_stride + c, a.d - c, res[u]);
      }
#pragma unroll
      for (int u = 0; u < kDropAhead; ++u) {
        const int64_t i = i0 + u * step;
        if (i >= a.rows) continue;
        float y[Q];
#pragma unroll
        for (int q = 0; q < Q; q += 4) {
          const uint4 w = philox_block((uint32_t)(c + q) / 4, (uint32_t)i, a.draw, 0, k0, k1);
          const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) y[q + e] = words[e] < a.below || a.all ? 0.0f : x[u][q + e] * a.scale;
        }
        if (a.residual) {
#pragma unroll
          for (int q = 0; q < Q; ++q) y[q] += res[u][q];
        }
        store_cols<T, Q>(a.y + i * a.y_stride + c, a.d - c, y);
      }
    }
  }
}

}  // namespace ms
