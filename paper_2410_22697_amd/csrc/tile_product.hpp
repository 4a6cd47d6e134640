// tile_product.hpp - products of many rows with weights, both through LDS.
//
// A block of four waves makes 128 rows by 64 NB outputs: a wave 64 rows by
// 32 NB outputs, 2 NB squares of the matrix unit's 32 x 32. Rows and weights
// come in steps of 64 bytes of k: the next step's are on their way in registers
// while the matrix unit takes this one's from LDS, in two buffers with one
// barrier a step. Weights lie along k (a row of k for each output) or across it
// (a row of outputs for each k, read from LDS transposed).
//
// The weights are the matrix unit's first operand and the rows its second, so
// that a lane ends up with four neighbouring outputs of one row at a time.
#pragma once

#include "linear_kernels.hpp"
#include "linear_weights.hpp"

namespace ms {

constexpr int kTileNT = 256;
constexpr int kTileRows = 128;

template <typename T, int NB, bool ACROSS>
struct TileProduct {
  static constexpr int kV = 16 / sizeof(T);
  static constexpr int kStep = 64 / sizeof(T);  // k of a step: four units of 16 bytes, two products
  static constexpr int kCols = 64 * NB;
  static constexpr int kPitch = kCols * sizeof(T) + 32;  // of a row of weights across k
  static constexpr int kXBytes = kTileRows * 64;
  static constexpr int kWBytes = ACROSS ? kStep * kPitch : kCols * 64;
  static constexpr int kLds = 2 * (kXBytes + kWBytes);
  static constexpr int kColUnits = kCols / kV;

  // The 16 bytes of unit u of row r: units change places within their row, so
  // that eight rows' same units lie in distinct banks.
  static __device__ __forceinline__ int place(int r, int u) { return (r * 4 + (u ^ ((r >> 1) & 3))) * 16; }

  // x[2], w[2]: the segments of the reduction. weight_row(c): the row of w that is output c of the tile (along k).
  // col0: the first output (across k), cols how many there are. acc[b][i]: squares of weights by rows.
  template <typename F>
  static __device__ __forceinline__ void run(const Operand<T> (&x)[2], const Weights<T> (&w)[2], int64_t r0, int64_t rows, int col0, int cols,
                                             F weight_row, char* lds, f32x16 (&acc)[NB][2]) {
    const int tid = threadIdx.x, lane = lane_id();
    const int wave = wave_uniform((int32_t)wave_id());
    const int first = (int)((x[0].K + kStep - 1) / kStep), steps = first + (int)((x[1].K + kStep - 1) / kStep);
    const T *xp[2], *wp[NB];
    auto segment = [&](int g) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t r = min(r0 + tid / 4 + i * 64, rows - 1);  // rows that are not there repeat the last one
        xp[i] = x[g].p + r * x[g].stride;
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int id = tid + i * kTileNT;
        wp[i] = ACROSS ? w[g].p + (int64_t)(id / kColUnits) * w[g].stride + min(col0 + id % kColUnits * kV, cols - 1)
                       : w[g].p + (int64_t)weight_row(id / 4) * w[g].stride;
      }
    };
    u32x4 xv[2], wv[NB];
    auto load = [&](int step) {
      const int g = step < first ? 0 : 1;
      if (step == first) segment(1);
      const int64_t K = x[g].K, k0 = (int64_t)(step - (g ? first : 0)) * kStep;
      const int64_t k = k0 + tid % 4 * kV;
      if (k0 + kStep <= K) {
#pragma unroll
        for (int i = 0; i < 2; ++i) xv[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(xp[i] + k));
        if constexpr (!ACROSS) {
#pragma unroll
          for (int i = 0; i < NB; ++i) wv[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(wp[i] + k));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) xv[i] = k_along(xp[i], k, K);
        if constexpr (!ACROSS) {
#pragma unroll
          for (int i = 0; i < NB; ++i) wv[i] = k_along(wp[i], k, K);
        }
      }
      if constexpr (ACROSS) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int id = tid + i * kTileNT, c = col0 + id % kColUnits * kV;
          const T* p = wp[i] + k0 * w[g].stride;
          wv[i] = (u32x4)0u;
          if (k0 + id / kColUnits < K && c < cols) {
            if (c + kV <= cols) {
              wv[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(p));
            } else {
              cols_t<T, kV> t;
#pragma unroll
              for (int q = 0; q < kV; ++q) t[q] = c + q < cols ? p[q] : (T)0.0f;
              wv[i] = __builtin_bit_cast(u32x4, t);
            }
          }
        }
      }
    };
    auto put = [&](int buffer) {
      char* to = lds + buffer * (kXBytes + kWBytes);
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<u32x4*>(to + place(tid / 4 + i * 64, tid % 4)) = xv[i];
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int id = tid + i * kTileNT;
        *reinterpret_cast<u32x4*>(to + kXBytes + (ACROSS ? id / kColUnits * kPitch + id % kColUnits * 16 : place(id / 4, tid % 4))) = wv[i];
      }
    };
    const int xr = wave / 2 * 64 + lane % 32, wr = wave % 2 * (32 * NB);
    auto multiply = [&](int buffer) {
      const char *fx = lds + buffer * (kXBytes + kWBytes), *fw = fx + kXBytes;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 a[NB], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) b[i] = *reinterpret_cast<const u32x4*>(fx + place(xr + 32 * i, 2 * s + lane / 32));
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          if constexpr (ACROSS) a[i] = dw_fragment<T, kCols>(fw, wr + 32 * i, s);
          else a[i] = *reinterpret_cast<const u32x4*>(fw + place(wr + 32 * i + lane % 32, 2 * s + lane / 32));
        }
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
    segment(0);
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

  // Stores a wave's results of 32 rows and kOut outputs that the lanes gave to
  // `turn` as T (rows of turn_pitch()), from row r0 and output c0 of `cols` on.
  template <int kOut>
  static constexpr int turn_pitch() { return kOut * sizeof(T) + 16; }
  template <int kOut>
  static __device__ __forceinline__ void turn_out(const char* turn, T* out, int64_t stride, int64_t r0, int64_t rows, int c0, int cols) {
    constexpr int kLanes = kOut / kV, kAtOnce = MS_WAVE / kLanes;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int lane = lane_id(), c = c0 + lane % kLanes * kV;
#pragma unroll
    for (int i = 0; i < 32 / kAtOnce; ++i) {
      const int r = i * kAtOnce + lane / kLanes;
      const cols_t<T, kV> v = __builtin_bit_cast(cols_t<T, kV>, *reinterpret_cast<const u32x4*>(turn + r * turn_pitch<kOut>() + lane % kLanes * 16));
      T* p = out + (r0 + r) * stride + c;
      if (r0 + r < rows && c < cols) {
        if (c + kV <= cols) {
          *reinterpret_cast<cols_t<T, kV>*>(p) = v;
        } else {
#pragma unroll
          for (int q = 0; q < kV; ++q)
            if (c + q < cols) p[q] = v[q];
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // Gives four neighbouring outputs of the lane's row to `turn`: those from 8 q + 4 (lane / 32) on of the square at `at`.
  template <int kOut>
  static __device__ __forceinline__ void turn_in(char* turn, int at, int q, const float (&v)[4]) {
    const int lane = lane_id();
    typedef T four __attribute__((ext_vector_type(4)));
    *reinterpret_cast<four*>(turn + lane % 32 * turn_pitch<kOut>() + (at + 8 * q + 4 * (lane / 32)) * sizeof(T)) = four{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  }
};

}  // namespace ms
