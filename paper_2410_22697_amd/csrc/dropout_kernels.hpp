// dropout_kernels.hpp - residual + dropout(x), the mask drawn where it is used.
//
//   y[i][j] = residual[i][j] + (word >= p 2^32 ? x[i][j] / (1 - p) : 0)
//
// word j % 4 of Philox4x32-10 at the counter (j / 4, i, draw, 0) under the
// call's seed: a column's fate hangs on its place alone, not on strides, types
// or the launch, so the gradient draws the same mask again and nothing of it is
// stored. A block of the generator serves four columns of a row.
//
// Bound by memory, in bf16 without a residual by the generator's ten rounds (20
// products of 32 by 32 bits a block: about 1.2 T words/s over the chip).
// Measured: 242K x 256 bf16 53 to 58 us (4.3 to 4.7 TB/s), with the residual 66
// (5.6); 110K x 1024 fp32 143 (6.3); 854K x 100 bf16 94 to 102 (147 with a team of
// lanes a row, three in sixteen of them idle).
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

constexpr int kDropNT = 256;
constexpr int kDropAhead = 2;  // units of a thread that are on their way together
constexpr int kDropChunk = kDropNT * kDropAhead;

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

// Threads take units of Q columns (a multiple of 4, or 4) one after the other
// through the rows, so that no lane draws for columns that are not there but at a
// row's end. A block finds the row of its first unit, and a thread's lies so many
// units on: by a multiplication where a row has less units than the block takes
// (exact: both factors are below 2^11), else the next row at most.
template <typename T, int Q>
__global__ __launch_bounds__(kDropNT) void k_dropout(Dropout<T> a, uint32_t units, uint32_t inverse, int64_t all) {
  const uint64_t seed = a.seed_at ? *a.seed_at : a.seed;
  const uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  for (int64_t first = (int64_t)blockIdx.x * kDropChunk; first < all; first += (int64_t)gridDim.x * kDropChunk) {
    const int64_t row0 = all >> 32 ? first / units : (int64_t)((uint32_t)first / units);
    const uint32_t at0 = (uint32_t)(first - row0 * units);
    float x[kDropAhead][Q], res[kDropAhead][Q];
    int64_t row[kDropAhead];
    int col[kDropAhead];
#pragma unroll
    for (int u = 0; u < kDropAhead; ++u) {
      const uint32_t at = at0 + threadIdx.x + u * kDropNT, over = units == 1 ? at : units < kDropChunk ? __umulhi(at, inverse) : at >= units;
      row[u] = row0 + over;
      col[u] = (int)(at - over * units) * Q;
      if (row[u] >= a.rows) continue;
      load_row<T, Q>(a.x + row[u] * a.x_stride + col[u], a.d - col[u], x[u]);
      if (a.residual) load_row<T, Q>(a.residual + row[u] * a.residual_stride + col[u], a.d - col[u], res[u]);
    }
#pragma unroll
    for (int u = 0; u < kDropAhead; ++u) {
      if (row[u] >= a.rows) continue;
      float y[Q];
#pragma unroll
      for (int q = 0; q < Q; q += 4) {
        const uint4 w = philox_block((uint32_t)(col[u] + q) / 4, (uint32_t)row[u], a.draw, 0, k0, k1);
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) y[q + e] = words[e] < a.below || a.all ? 0.0f : x[u][q + e] * a.scale;
      }
      if (a.residual) {
#pragma unroll
        for (int q = 0; q < Q; ++q) y[q] += res[u][q];
      }
      store_row<T, Q>(a.y + row[u] * a.y_stride + col[u], a.d - col[u], y);
    }
  }
}

}  // namespace ms
