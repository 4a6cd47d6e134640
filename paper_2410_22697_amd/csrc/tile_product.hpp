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

// Both kinds of operand hold what a thread takes of a step: whole() asks for it
// where the step's k are all there, and ragged() where some lie behind the last
// one (left out as k_along() leaves them out); either goes on to the next step.
// A loop of whole() has no branch that would wait for a load.

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
    for (int i = 0; i < kPer; ++i) p[i] = where((int)threadIdx.x / 4 + i * (kTileNT / 4)) + threadIdx.x % 4 * kV;
  }
  __device__ __forceinline__ void whole() {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      v[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(p[i]));
      p[i] += tile_step<T>();
    }
  }
  // k0: the step's first k, of K
  __device__ __forceinline__ void ragged(int64_t k0, int64_t K) {
    const int64_t k = k0 + threadIdx.x % 4 * kV;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      v[i] = k_along(p[i] - k, k, K);
      p[i] += tile_step<T>();
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

// An operand across k. Its columns are read in units of 16 bytes that are all
// there: the last one ends with the row (tile_column() says which columns it
// holds), one behind it repeats it, and its results go nowhere or are stored
// twice. Rows of less than 16 bytes are read value by value, by ragged() alone.
template <typename T, int COLS>
struct TileAcross {
  static constexpr int kV = 16 / sizeof(T), kPer = COLS * 4 / kTileNT, kColUnits = COLS / kV;
  static constexpr int kBytes = tile_step<T>() * dw_pitch<T, COLS>();
  static constexpr int kRows = kTileNT / kColUnits;  // that the block takes at a time: a thread's columns are the same in all of them
  static_assert(kTileNT % kColUnits == 0, "");
  const T* p;
  int64_t stride;
  int narrow;  // columns, where there are less than a unit's
  u32x4 v[kPer];

  // where(c, first, columns, stride): the row of k = 0, which of its columns position c is, how many there are
  template <typename F>
  __device__ __forceinline__ void begin(F where) {
    int c, columns;
    const T* row = where((int)threadIdx.x % kColUnits * kV, c, columns, stride);
    narrow = columns < kV ? columns : 0;
    p = row + (columns < kV ? 0 : min(c, columns - kV)) + (int64_t)(threadIdx.x / kColUnits) * stride;
  }
  __device__ __forceinline__ void whole() {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      v[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(p));
      p += kRows * stride;
    }
  }
  __device__ __forceinline__ void ragged(int64_t k0, int64_t K) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int r = (int)threadIdx.x / kColUnits + i * kRows, in = r % kV;
      const int64_t unit = k0 + (r - in);
      const int skip = K >= kV ? skipped<T>(unit, K) : (unit + in < K ? 0 : kV);
      const T* from = p + (skip && K >= kV ? K - kV - unit : 0) * stride;
      v[i] = (u32x4)0u;
      if (in >= skip) {
        if (narrow) {
          cols_t<T, kV> t;
#pragma unroll
          for (int q = 0; q < kV; ++q) t[q] = q < narrow ? from[q] : (T)0.0f;
          v[i] = __builtin_bit_cast(u32x4, t);
        } else {
          v[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(from));
        }
      }
      p += kRows * stride;
    }
  }
  __device__ __forceinline__ void put(char* to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      *reinterpret_cast<u32x4*>(to + (threadIdx.x / kColUnits + i * kRows) * dw_pitch<T, COLS>() + threadIdx.x % kColUnits * 16) = v[i];
  }
  static __device__ __forceinline__ u32x4 fragment(const char* from, int c0, int s) { return dw_fragment<T, COLS>(from, c0, s); }
};

// The first column of the V that an operand across k has from column c on (c a
// multiple of a unit's; V columns of a unit at most): c, or less where that unit
// was moved to end with the row.
template <typename T>
__device__ __forceinline__ int tile_column(int c, int columns) {
  constexpr int kV = 16 / sizeof(T);
  const int unit = c / kV * kV;
  return c - (columns >= kV && unit + kV > columns ? unit + kV - columns : 0);
}

template <typename A, typename B>
constexpr int tile_lds() {
  return 2 * (A::kBytes + B::kBytes);
}

// A segment of the reduction: K of it, of which the steps all there are taken by
// whole() if `plain` (by ragged() else).
struct TileSegment {
  int64_t K;
  bool plain;
};

// acc[i][j] += the products of the first operand's columns wave % 2 * 32 NB + 32 i
// on and the second's wave / 2 * 64 + 32 j on, over SEGMENTS segments, none of
// them before the first empty; begin(g) begins segment g of both operands.
template <typename T, int NB, int SEGMENTS, typename A, typename B, typename F>
__device__ __forceinline__ void tile_product(A& first, B& second, const TileSegment (&segments)[SEGMENTS], F begin, char* lds, f32x16 (&acc)[NB][2]) {
  constexpr int kBuffer = A::kBytes + B::kBytes, kStep = tile_step<T>();
  const int wave = wave_uniform((int32_t)wave_id());
  auto put = [&](int buffer) {
    first.put(lds + buffer);
    second.put(lds + buffer + A::kBytes);
  };
  auto multiply = [&](int buffer) {
    const char *fa = lds + buffer, *fb = fa + A::kBytes;
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
  // the step that was asked for is put beside the one before it, which is multiplied meanwhile
  int buffer = 0;
  auto step = [&] {
    __builtin_amdgcn_sched_barrier(0);  // the step's loads stay ahead of the products that they run beside, and its stores behind them
    multiply(buffer);
    __builtin_amdgcn_sched_barrier(0);
    buffer = kBuffer - buffer;
    put(buffer);
    __syncthreads();
  };
  begin(0);
  int64_t k0 = 0;
  if (segments[0].plain && kStep <= segments[0].K) {
    first.whole();
    second.whole();
  } else {
    first.ragged(0, segments[0].K);
    second.ragged(0, segments[0].K);
  }
  put(0);
  __syncthreads();
  k0 = kStep;
#pragma unroll 1
  for (int g = 0; g < SEGMENTS; ++g) {
    if (g > 0) {
      if (segments[SEGMENTS - 1].K <= 0) break;
      begin(g);
      k0 = 0;
    }
    const int64_t K = SEGMENTS > 1 && g ? segments[SEGMENTS - 1].K : segments[0].K;
    if (SEGMENTS > 1 && g ? segments[SEGMENTS - 1].plain : segments[0].plain) {
#pragma unroll 1
      for (; k0 + kStep <= K; k0 += kStep) {
        first.whole();
        second.whole();
        step();
      }
    }
#pragma unroll 1
    for (; k0 < K; k0 += kStep) {
      first.ragged(k0, K);
      second.ragged(k0, K);
      step();
    }
  }
  multiply(buffer);
  __syncthreads();
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
