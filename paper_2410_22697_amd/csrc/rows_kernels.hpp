// rows_kernels.hpp - rows written to a table in 8 or 4 bits, and read back.
//
// Both kernels give a row to a team of T lanes, T the power of two that covers
// it (64 lanes take a longer row in turns), so rows of a frontier's width share
// a wave. They move each value once and are bound by memory: a value costs ~6
// instructions. Both read what a row's address hangs on and, where it does not,
// the row itself at once, and take two rows at a time (one: 78 us instead of 73
// for the first two figures' call; four: 210 instead of 156 for the last two's).
//
// Measured: 110K rows of 256 bf16 written in 8 bits 30 us (2.8 TB/s of rows read
// and codes written), 242K read back 43 us (4.4 TB/s); 86K rows of 100 floats
// in 4 bits 18 us, 854K read back 139 us (2.9 TB/s: rows of 84 bytes lie at any
// place, and a line of 128 comes for each).
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

constexpr int kRowsNT = 256;
constexpr int kRowsQ = 8;  // columns per lane of a written row: 8 bytes of 8-bit codes, 4 of 4-bit ones
constexpr int kRowsAhead = 2;  // rows of a team that are on their way together

// Largest (or least) over aligned runs of `width` lanes, a power of two. Within
// 16 lanes the partners come by data-parallel moves: the neighbour, the other
// pair, and, since equal groups hold equal values by then, the mirror images.
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}
template <typename F, typename V>
__device__ __forceinline__ V team_reduce(V x, int width, F pick) {
  if (width > 1) x = pick(x, moved<0xB1>(x));   // quad_perm 1 0 3 2
  if (width > 2) x = pick(x, moved<0x4E>(x));   // quad_perm 2 3 0 1
  if (width > 4) x = pick(x, moved<0x141>(x));  // row_half_mirror
  if (width > 8) x = pick(x, moved<0x140>(x));  // row_mirror
  if (width > 16) x = pick(x, __shfl_xor(x, 16, MS_WAVE));
  if (width > 32) x = pick(x, __shfl_xor(x, 32, MS_WAVE));
  return x;
}

// What a group's values have in common: the largest magnitude's bits (which
// order as the magnitudes do, with infinities and NaN above all finite ones,
// where a float maximum would lose a NaN) and, for 4 bits, both ends.
template <int BITS>
struct GroupEnds {
  uint32_t mag = 0;
  float lo = __builtin_inff(), hi = -__builtin_inff();

  __device__ __forceinline__ void add(const float* x, int valid) {
#pragma unroll
    for (int q = 0; q < kRowsQ; ++q)
      if (q < valid) {
        mag = max(mag, __float_as_uint(x[q]) & 0x7FFFFFFFu);
        if constexpr (BITS == 4) {
          lo = fminf(lo, x[q]);
          hi = fmaxf(hi, x[q]);
        }
      }
  }
  __device__ __forceinline__ void join(int width) {
    mag = team_reduce(mag, width, [](uint32_t a, uint32_t b) { return max(a, b); });
    if constexpr (BITS == 4) {
      lo = team_reduce(lo, width, [](float a, float b) { return fminf(a, b); });
      hi = team_reduce(hi, width, [](float a, float b) { return fmaxf(a, b); });
    }
  }
  // step and its reciprocal (0 where every code is 0)
  __device__ __forceinline__ void scale(float& step, float& inv) {
    const float range = BITS == 8 ? __uint_as_float(mag) : hi - lo;
    step = range * (BITS == 8 ? 1.0f / 127 : 1.0f / 15);
    inv = 1.0f / step;
    if (!(range >= 0x1p-119f)) step = inv = 0.0f;
    if (mag >= 0x7F800000u || range == __builtin_inff()) {
      step = lo = __builtin_nanf("");
      inv = 0.0f;
    }
    if (BITS == 8) lo = 0.0f;
  }
};

template <int BITS>
__device__ __forceinline__ void store_codes(uint8_t* row, int c, int d, const float* x, int valid, float lo, float inv) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int q = 0; q < kRowsQ; ++q) {
    // a code of a group without a step is 0, also where x is not finite
    const float r = inv != 0.0f && q < valid ? rintf((x[q] - lo) * inv) : 0.0f;
    if constexpr (BITS == 8)
      w[q / 4] |= ((uint32_t)(int)fminf(fmaxf(r, -127.0f), 127.0f) & 0xFFu) << (8 * (q % 4));
    else
      w[0] |= (uint32_t)fminf(fmaxf(r, 0.0f), 15.0f) << (4 * q);
  }
  uint32_t* p = reinterpret_cast<uint32_t*>(row + (int64_t)c * BITS / 8);
  p[0] = w[0];
  if (BITS == 8 && c + 4 < d) p[1] = w[1];
}

template <typename S, int BITS, int T>
__global__ __launch_bounds__(kRowsNT) void k_pack_rows(const S* __restrict__ src, int64_t stride, int64_t n,
                                                       const int32_t* __restrict__ slots, uint8_t* __restrict__ table,
                                                       int64_t rows, PackedRows f) {
  const int lane = threadIdx.x % T;
  const int d = f.d;
  const bool whole = f.group_log2 == 31;
  const int width = whole ? T : 1 << (f.group_log2 - 3);  // lanes that share a group
  const int64_t step = (int64_t)gridDim.x * (kRowsNT / T);
  for (int64_t i0 = (int64_t)blockIdx.x * (kRowsNT / T) + threadIdx.x / T; i0 < n; i0 += kRowsAhead * step) {
    const int c1 = lane * kRowsQ;
    int64_t slot[kRowsAhead];
    float head[kRowsAhead][kRowsQ];  // the lane's first columns
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const int64_t i = i0 + u * step;
      slot[u] = -1;
      if (i < n) {
        slot[u] = slots ? (int64_t)slots[i] : i;
        if (c1 < d) load_cols<S, kRowsQ>(src + i * stride + c1, d - c1, head[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      if (slot[u] < 0 || slot[u] >= rows) continue;  // the same for the whole team
      const S* x = src + (i0 + u * step) * stride;
      uint8_t* row = table + slot[u] * f.row_bytes;
      float* floats = reinterpret_cast<float*>(row + f.floats_at);
      float step_size, inv;
      if (whole && d > T * kRowsQ) {
        // one group longer than the team: a sweep for its ends, one for the codes
        GroupEnds<BITS> e;
        float v[kRowsQ];
        e.add(head[u], d - c1);
        for (int c = c1 + T * kRowsQ; c < d; c += T * kRowsQ) {
          load_cols<S, kRowsQ>(x + c, d - c, v);
          e.add(v, d - c);
        }
        e.join(T);
        e.scale(step_size, inv);
        for (int c = c1; c < d; c += T * kRowsQ) {
          load_cols<S, kRowsQ>(x + c, d - c, v);
          store_codes<BITS>(row, c, d, v, d - c, e.lo, inv);
        }
        if (lane == 0) {
          if (BITS == 4) floats[0] = e.lo;
          floats[BITS == 4 ? 1 : 0] = step_size;
        }
        continue;
      }
      for (int c0 = 0; c0 < d; c0 += T * kRowsQ) {  // groups end with the team's turn or inside it
        const int c = c0 + c1;
        GroupEnds<BITS> e;
        float v[kRowsQ];
        if (c0 == 0) {
#pragma unroll
          for (int q = 0; q < kRowsQ; ++q) v[q] = head[u][q];
        } else if (c < d) {
          load_cols<S, kRowsQ>(x + c, d - c, v);
        }
        if (c < d) e.add(v, d - c);
        e.join(width);
        e.scale(step_size, inv);
        if (c < d) {
          store_codes<BITS>(row, c, d, v, d - c, e.lo, inv);
          if (lane % width == 0) {
            const int g = c >> f.group_log2;
            if (BITS == 4) floats[2 * g] = e.lo;
            floats[BITS == 4 ? 2 * g + 1 : g] = step_size;
          }
        }
      }
    }
  }
}

// 16 bytes of output a lane.
template <typename O, int BITS, int T>
__global__ __launch_bounds__(kRowsNT) void k_unpack_rows(const uint8_t* __restrict__ table, int64_t rows,
                                                         const int32_t* __restrict__ index, int64_t n, O* __restrict__ out,
                                                         int64_t stride, PackedRows f) {
  constexpr int Q = 16 / sizeof(O);
  const int lane = threadIdx.x % T;
  const int64_t step = (int64_t)gridDim.x * (kRowsNT / T);
  for (int64_t i0 = (int64_t)blockIdx.x * (kRowsNT / T) + threadIdx.x / T; i0 < n; i0 += kRowsAhead * step) {
    int64_t at[kRowsAhead];
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const int64_t i = i0 + u * step;
      at[u] = i < n ? (index ? (int64_t)index[i] : i) : -1;
    }
    for (int c = lane * Q; c < f.d; c += T * Q) {
      PackedCols<BITS, Q> p[kRowsAhead];
#pragma unroll
      for (int u = 0; u < kRowsAhead; ++u)
        if (at[u] >= 0 && at[u] < rows) p[u].load(table + at[u] * f.row_bytes, f, c);
#pragma unroll
      for (int u = 0; u < kRowsAhead; ++u) {
        const int64_t i = i0 + u * step;
        float v[Q];
        p[u].values(v);
        if (i < n) store_cols<O, Q>(out + i * stride + c, f.d - c, v);
      }
    }
  }
}

}  // namespace ms
