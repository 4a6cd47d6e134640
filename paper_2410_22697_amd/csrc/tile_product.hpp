// tile_product.hpp - products of two tall operands, both through LDS.
//
// A block of four waves makes 64 NB by 128 results: a wave 32 NB by 64, 2 NB
// squares of the matrix unit's 32 x 32. The operands come in steps of 64 bytes
// of k: the next step's are on their way in registers while the matrix unit
// takes this one's from LDS, in two buffers with one barrier a step. An operand
// lies along k (a row of k for each of its columns in the product) or across it
// (a row of columns for each k, which LDS's transposing reads turn).
//
// The second operand's columns become the lanes, the first's the registers: a
// lane ends up with four neighbours of the first at a time, for one of the
// second.
//
// Measured: rows along k, 110K by 2048 outputs in bf16, 130 us for each 256 of k
// (890 TFLOP/s) beside what the epilogue takes.
#pragma once

#include "linear_kernels.hpp"
#include "linear_weights.hpp"

namespace ms {

constexpr int kTileNT = 256;
constexpr int kTileSecond = 128;  // columns of the second operand
constexpr int kTileStepBytes = 64;

// k of a step: four units of 16 bytes, two products.
template <typename T>
constexpr int tile_step() {
  return kTileStepBytes / sizeof(T);
}

// An operand along k, COLS columns of it: column c's row of k begins at
// where(c). In LDS the units of a column change places, so that eight columns'
// same units lie in distinct banks.
template <typename T, int COLS>
struct TileAlong {
  static constexpr int kV = 16 / sizeof(T), kPer = COLS * 4 / kTileNT, kBytes = COLS * kTileStepBytes;
  const T* p[kPer];
  u32x4 v[kPer];

  static __device__ __forceinline__ int place(int c, int u) { return (c * 4 + (u ^ ((c >> 1) & 3))) * 16; }
  template <typename F>
  __device__ __forceinline__ void begin(F where) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) p[i] = where((int)threadIdx.x / 4 + i * (kTileNT / 4));
  }
  // k0: the step's first k, of K
  __device__ __forceinline__ void load(int64_t k0, int64_t K) {
    const int64_t k = k0 + threadIdx.x % 4 * kV;
    if (k0 + tile_step<T>() <= K) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(p[i] + k));
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = k_along(p[i], k, K);
    }
  }
  __device__ __forceinline__ void put(char* to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) *reinterpret_cast<u32x4*>(to + place(threadIdx.x / 4 + i * (kTileNT / 4), threadIdx.x % 4)) = v[i];
  }
  // the columns c0 to c0 + 31 in the step's half s
  static __device__ __forceinline__ u32x4 fragment(const char* from, int c0, int s) {
    const int lane = lane_id();
    return *reinterpret_cast<const u32x4*>(from + place(c0 + lane % 32, 2 * s + lane / 32));
  }
};

// An operand across k: the columns of a unit begin at where(c, columns), which
// also says how many of them and those after them there are (none: where() is
// not followed).
template <typename T, int COLS>
struct TileAcross {
  static constexpr int kV = 16 / sizeof(T), kPer = COLS * 4 / kTileNT, kColUnits = COLS / kV;
  static constexpr int kBytes = tile_step<T>() * dw_pitch<T, COLS>();
  const T* p[kPer];
  int64_t stride[kPer];
  int columns[kPer];
  u32x4 v[kPer];

  template <typename F>
  __device__ __forceinline__ void begin(F where) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int id = threadIdx.x + i * kTileNT;
      p[i] = where(id % kColUnits * kV, columns[i], stride[i]) + (int64_t)(id / kColUnits) * stride[i];
    }
  }
  __device__ __forceinline__ void load(int64_t k0, int64_t K) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      // (a ragged end is read as k_along() reads it: the last kV of k, those before k left out)
      const int r = ((int)threadIdx.x + i * kTileNT) / kColUnits, in = r % kV;
      const int64_t unit = k0 + (r - in);
      const int skip = K >= kV ? skipped<T>(unit, K) : (unit + in < K ? 0 : kV);
      const T* from = p[i] + (skip && K >= kV ? K - kV - (r - in) : k0) * stride[i];
      v[i] = (u32x4)0u;
      if (columns[i] > 0 && in >= skip) {
        if (columns[i] >= kV) {
          v[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(from));
        } else {
          cols_t<T, kV> t;
#pragma unroll
          for (int q = 0; q < kV; ++q) t[q] = q < columns[i] ? from[q] : (T)0.0f;
          v[i] = __builtin_bit_cast(u32x4, t);
        }
      }
    }
  }
  __device__ __forceinline__ void put(char* to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int id = threadIdx.x + i * kTileNT;
      *reinterpret_cast<u32x4*>(to + id / kColUnits * dw_pitch<T, COLS>() + id % kColUnits * 16) = v[i];
    }
  }
  static __device__ __forceinline__ u32x4 fragment(const char* from, int c0, int s) { return dw_fragment<T, COLS>(from, c0, s); }
};

template <typename A, typename B>
constexpr int tile_lds() {
  return 2 * (A::kBytes + B::kBytes);
}

// acc[i][j] += the products of the first operand's columns wave % 2 * 32 NB + 32 i
// on and the second's wave / 2 * 64 + 32 j on, over `steps` steps; load(step)
// asks for both operands' part of a step.
template <typename T, int NB, typename A, typename B, typename L>
__device__ __forceinline__ void tile_product(A& first, B& second, int steps, L load, char* lds, f32x16 (&acc)[NB][2]) {
  constexpr int kBuffer = A::kBytes + B::kBytes;
  const int wave = wave_uniform((int32_t)wave_id());
  auto put = [&](int buffer) {
    first.put(lds + buffer * kBuffer);
    second.put(lds + buffer * kBuffer + A::kBytes);
  };
  auto multiply = [&](int buffer) {
    const char *fa = lds + buffer * kBuffer, *fb = fa + A::kBytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 a[NB], b[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) b[j] = B::fragment(fb, wave / 2 * 64 + 32 * j, s);
#pragma unroll
      for (int i = 0; i < NB; ++i) a[i] = A::fragment(fa, wave % 2 * (32 * NB) + 32 * i, s);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if constexpr (sizeof(T) == 2) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, b[j]), acc[i][j], 0, 0, 0);
          } else {
            const f32x4 u = __builtin_bit_cast(f32x4, a[i]), v = __builtin_bit_cast(f32x4, b[j]);
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(u[q], v[q], acc[i][j], 0, 0, 0);
          }
        }
    }
  };
  if (steps > 0) {
    load(0);
    put(0);
  }
  __syncthreads();
  for (int s = 0; s < steps; ++s) {
    if (s + 1 < steps) load(s + 1);
    multiply(s % 2);
    if (s + 1 < steps) put((s + 1) % 2);
    __syncthreads();
  }
}

// A wave's way out: 32 of the second operand's columns, OUT of the first's for
// each, as T. The lanes give four neighbours at a time to LDS, and whole rows of
// OUT leave it.
template <typename T, int OUT>
struct TileTurn {
  static constexpr int kV = 16 / sizeof(T), kPitch = OUT * sizeof(T) + 16, kBytes = 32 * kPitch;
  char* lds;

  // those from 8 q + 4 (lane / 32) on of the square at `at`
  __device__ __forceinline__ void in(int at, int q, const float (&v)[4]) const {
    const int lane = lane_id();
    typedef T four __attribute__((ext_vector_type(4)));
    *reinterpret_cast<four*>(lds + lane % 32 * kPitch + (at + 8 * q + 4 * (lane / 32)) * sizeof(T)) = four{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  }
  // f(row of the 32, first column, values) for whole units
  template <typename F>
  __device__ __forceinline__ void units(F f) const {
    constexpr int kLanes = OUT / kV, kAtOnce = MS_WAVE / kLanes;
    const int lane = lane_id();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < 32 / kAtOnce; ++i) {
      const int r = i * kAtOnce + lane / kLanes;
      f(r, lane % kLanes * kV, __builtin_bit_cast(cols_t<T, kV>, *reinterpret_cast<const u32x4*>(lds + r * kPitch + lane % kLanes * 16)));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // to rows r0 on of `rows` and columns c0 on of `cols`
  __device__ __forceinline__ void out(T* to, int64_t stride, int64_t r0, int64_t rows, int c0, int cols) const {
    units([&](int r, int c, cols_t<T, kV> v) {
      T* p = to + (r0 + r) * stride + c0 + c;
      if (r0 + r >= rows) return;
      if (c0 + c + kV <= cols) {
        *reinterpret_cast<cols_t<T, kV>*>(p) = v;
      } else {
#pragma unroll
        for (int q = 0; q < kV; ++q)
          if (c0 + c + q < cols) p[q] = v[q];
      }
    });
  }
};

}  // namespace ms
