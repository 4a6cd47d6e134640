// linear_weights.hpp - the gradient of a layer's weights: dw = dz^T x, dbias.
//
// The reduction runs over the rows, of which there are many, and the result is
// small: the rows are split into parts, a block sums one tile of dw over one
// part and writes it as fp32, and k_linear_join adds the parts in order. dz and
// x are read once a tile row by row, as they lie in memory, two steps of rows
// ahead in registers (dz gets its slope there), then go through LDS in two
// buffers with one barrier a step. The matrix unit wants neighbouring rows of
// one column in a lane: for bf16, LDS's transposing read gives four of them (16
// lanes read 4 rows of 16 columns, and each gets a column), for fp32 a value is
// a read of its own. Bound by memory (bf16) or by the matrix unit (fp32).
//
// Measured: 110K x 1024 by 128 in bf16 with gelu's slope 130 us (3.7 TB/s, 220
// TFLOP/s), about half of it vector instructions of the slope; 16K x 47 by 512
// in fp32 26 us; their joins 5 to 7 us.
#pragma once

#include "linear_kernels.hpp"

namespace ms {

constexpr int kDwNT = 512;

template <typename T>
struct LinearDw {
  Operand<T> dz, x[2];  // R rows (the reduction), K columns
  float *dw, *dbias;    // [parts][n][k0 + k1] and [parts][n], null where not asked for
  int64_t rows, part;   // rows of a part, a multiple of a step's
  int n, k[2], second;  // second: the position of the second input's first column
  int tiles_n, tiles_k;
};

// Columns are read in vectors of 16 bytes, the last one of an input ending with
// its row: position `at` holds column dw_column(at), or nothing (-1; also the
// columns that the last vector repeats). The second input's positions begin at
// a whole vector behind the first one's.
template <typename T>
__device__ __forceinline__ int dw_column(int at, int columns) {
  constexpr int kV = 16 / sizeof(T);
  const int c = at / kV * kV;
  if (c + kV <= columns || columns < kV) return at < columns ? at : -1;
  const int col = columns - kV + (at - c);
  return c < columns && col >= c ? col : -1;
}

template <typename T>
__device__ __forceinline__ u32x4 dw_load(const T* row, int c, int columns) {
  constexpr int kV = 16 / sizeof(T);
  if (columns >= kV) return __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(row + min(c, columns - kV)));
  cols_t<T, kV> v;
#pragma unroll
  for (int q = 0; q < kV; ++q) v[q] = c + q < columns ? row[c + q] : (T)0.0f;
  return __builtin_bit_cast(u32x4, v);
}

// Rows of `COLS` columns in LDS, 32 bytes apart beyond their length, so that
// four rows' 32 bytes (what 16 lanes read transposed) meet in distinct banks.
template <typename T, int COLS>
constexpr int dw_pitch() {
  return COLS * sizeof(T) + 32;
}

// The four (or eight, in bf16) neighbouring rows that a lane takes of column
// c0 + lane % 32 in a step's k-th part: rows 16 k + 8 (lane / 32) on in bf16,
// 8 k + 4 (lane / 32) on in fp32.
template <typename T, int COLS>
__device__ __forceinline__ u32x4 dw_fragment(const char* lds, int c0, int k) {
  const int lane = lane_id();
  constexpr int pitch = dw_pitch<T, COLS>();
  if constexpr (sizeof(T) == 2) {
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4v* lds_ptr;
    const int group = lane / 16, i = lane % 16;
    const char* p = lds + (16 * k + 8 * (group / 2) + i / 4) * pitch + (c0 + 16 * (group % 2) + 4 * (i % 4)) * 2;
    const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p));
    const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * pitch)));
    return u32x4{a.x, a.y, b.x, b.y};
  } else {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(lds + (8 * k + 4 * (lane / 32)) * pitch) + c0 + lane % 32;
    return u32x4{p[0], p[pitch / 4], p[2 * pitch / 4], p[3 * pitch / 4]};
  }
}

// DW: dw, and dbias if it is asked for; else dbias alone, by one block for each
// TN outputs and part, which reads no x.
template <typename T, bool SLOPE, int TN, int TK, bool DW>
__global__ __launch_bounds__(kDwNT) void k_linear_dw(LinearDw<T> a, int64_t blocks) {
  constexpr int kV = 16 / sizeof(T), kRows = 64 / sizeof(T);  // rows of a step
  constexpr int kVn = TN / kV, kVk = TK / kV;                 // vectors of a row
  constexpr int kPn = (kRows * kVn + kDwNT - 1) / kDwNT, kPk = (kRows * kVk + kDwNT - 1) / kDwNT;
  constexpr int kWn = TN / 64, kWk = 8 / kWn, kI = 2, kJ = TK / kWk / 32;  // waves, and 32x32 squares of a wave
  constexpr int kTileN = kRows * dw_pitch<T, TN>(), kTileK = DW ? kRows * dw_pitch<T, TK>() : 0;
  __shared__ __align__(16) char lds[2 * (kTileN + kTileK)];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t part = tile / (a.tiles_k * a.tiles_n);
  const int in = (int)(tile % (a.tiles_k * a.tiles_n));
  const int n0 = in / a.tiles_k * TN, k0 = in % a.tiles_k * TK;
  const bool bias = a.dbias && k0 == 0;
  const int64_t first = part * a.part, end = min(a.rows, first + a.part);
  const int steps = (int)((end - first + kRows - 1) / kRows);
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int wn = wave % kWn * 64, wk = wave / kWn * (kJ * 32);

  u32x4 dy[2][kPn], z[2][SLOPE ? kPn : 1], xs[2][kPk];
  float sums[kV] = {};
  auto load = [&](auto set, int step) {
    constexpr int S = set();
#pragma unroll
    for (int i = 0; i < kPn; ++i) {
      const int id = threadIdx.x + i * kDwNT;
      const int64_t r = first + (int64_t)step * kRows + id / kVn;
      const int c = n0 + id % kVn * kV;
      dy[S][i] = (u32x4)0u;
      if constexpr (SLOPE) z[S][i] = (u32x4)0u;
      if (id < kRows * kVn && r < end && c < a.n) {
        dy[S][i] = dw_load(a.dz.p + r * a.dz.stride, c, a.n);
        if constexpr (SLOPE) z[S][i] = dw_load(a.dz.pre + r * a.dz.pre_stride, c, a.n);
      }
    }
    if constexpr (!DW) return;
#pragma unroll
    for (int i = 0; i < kPk; ++i) {
      const int id = threadIdx.x + i * kDwNT;
      const int64_t r = first + (int64_t)step * kRows + id / kVk;
      const int at = k0 + id % kVk * kV, seg = at >= a.second ? 1 : 0, c = at - (seg ? a.second : 0);
      const T* x = seg ? a.x[1].p + r * a.x[1].stride : a.x[0].p + r * a.x[0].stride;
      const int columns = seg ? a.k[1] : a.k[0];
      xs[S][i] = (u32x4)0u;
      if (id < kRows * kVk && r < end && c < columns) xs[S][i] = dw_load(x, c, columns);
    }
  };
  auto put = [&](auto set) {
    constexpr int S = set();
    char* to = lds + S * (kTileN + kTileK);
#pragma unroll
    for (int i = 0; i < kPn; ++i) {
      const int id = threadIdx.x + i * kDwNT;
      cols_t<T, kV> g = __builtin_bit_cast(cols_t<T, kV>, dy[S][i]);
      if constexpr (SLOPE) {
        act_grads<T, kV>(g, __builtin_bit_cast(cols_t<T, kV>, z[S][i]), a.dz.act, [&](int q, float v) { sums[q] += v; });
      } else if (bias) {
#pragma unroll
        for (int q = 0; q < kV; ++q) sums[q] += (float)g[q];
      }
      if (DW && id < kRows * kVn) *reinterpret_cast<u32x4*>(to + id / kVn * dw_pitch<T, TN>() + id % kVn * 16) = __builtin_bit_cast(u32x4, g);
    }
    if constexpr (!DW) return;
#pragma unroll
    for (int i = 0; i < kPk; ++i) {
      const int id = threadIdx.x + i * kDwNT;
      if (id < kRows * kVk) *reinterpret_cast<u32x4*>(to + kTileN + id / kVk * dw_pitch<T, TK>() + id % kVk * 16) = xs[S][i];
    }
  };
  f32x16 acc[kI][kJ] = {};
  auto multiply = [&](auto set) {
    if constexpr (!DW) return;
    const char* from = lds + set() * (kTileN + kTileK);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      u32x4 fn[kI], fk[kJ];
#pragma unroll
      for (int i = 0; i < kI; ++i) fn[i] = dw_fragment<T, TN>(from, wn + 32 * i, k);
#pragma unroll
      for (int j = 0; j < kJ; ++j) fk[j] = dw_fragment<T, TK>(from + kTileN, wk + 32 * j, k);
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          if constexpr (sizeof(T) == 2) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fn[i]), __builtin_bit_cast(bf16x8, fk[j]), acc[i][j], 0, 0, 0);
          } else {
            const f32x4 u = __builtin_bit_cast(f32x4, fn[i]), v = __builtin_bit_cast(f32x4, fk[j]);
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(u[q], v[q], acc[i][j], 0, 0, 0);
          }
        }
    }
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  load(even, 0);
  load(odd, 1);
  put(even);
  for (int s = 0; s < steps; s += 2) {
    __syncthreads();
    load(even, s + 2);
    multiply(even);
    put(odd);
    __syncthreads();
    load(odd, s + 3);
    multiply(odd);  // of zeros behind the last step
    put(even);
  }
  __syncthreads();
  if (bias) {
    // the threads that share columns add up in order
    constexpr int kGroups = (kRows * kVn < kDwNT ? kRows * kVn : kDwNT) / kVn;
    float* turn = reinterpret_cast<float*>(lds);
    if ((int)threadIdx.x < kGroups * kVn) {
#pragma unroll
      for (int q = 0; q < kV; ++q) turn[threadIdx.x / kVn * TN + threadIdx.x % kVn * kV + q] = sums[q];
    }
    __syncthreads();
    const int col = (int)threadIdx.x < TN ? dw_column<T>(n0 + threadIdx.x, a.n) : -1;
    if (col >= 0) {
      float t = 0.0f;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) t += turn[g * TN + threadIdx.x];
      a.dbias[part * a.n + col] = t;
    }
  }
  if constexpr (!DW) return;
  const int all = a.k[0] + a.k[1];
  float* dw = a.dw + part * a.n * (int64_t)all;
#pragma unroll
  for (int j = 0; j < kJ; ++j) {
    const int at = k0 + wk + 32 * j + lane % 32, seg = at >= a.second ? 1 : 0;
    int ck = dw_column<T>(at - (seg ? a.second : 0), a.k[seg]);
    if (ck < 0) continue;
    ck += seg ? a.k[0] : 0;
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int g = 0; g < 16; ++g) {
        const int cn = dw_column<T>(n0 + wn + 32 * i + 8 * (g / 4) + 4 * (lane / 32) + g % 4, a.n);
        if (cn >= 0) dw[(int64_t)cn * all + ck] = acc[i][j][g];
      }
  }
}

}  // namespace ms
