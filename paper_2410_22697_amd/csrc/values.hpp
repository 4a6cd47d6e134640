// values.hpp - rows of 32-bit, bf16 or packed values, as the operators' kernels
// read and write them: a few neighbouring columns of one row at a time.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ms {

typedef __bf16 bf16;

// Vectors at the alignment of their elements: rows of any stride are read in
// whole vectors, which global memory takes at any address.
template <typename T, int Q>
struct ColsOf {
  typedef T type __attribute__((ext_vector_type(Q), aligned(sizeof(T))));
};
template <typename T, int Q>
using cols_t = typename ColsOf<T, Q>::type;

// Columns [0, valid) of the Q at p as fp32, `fill` in the others.
template <typename T, int Q>
__device__ __forceinline__ void load_cols(const T* p, int valid, float* x, float fill = 0.0f) {
  if (valid >= Q) {
    const cols_t<T, Q> v = *reinterpret_cast<const cols_t<T, Q>*>(p);
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] = (float)v[q];
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] = q < valid ? (float)p[q] : fill;
  }
}

// Stores Q columns of x, rounded to nearest even: past the caches' own lines
// where `streamed`. Results are larger than the L2 wherever their time counts,
// and rows that do not fill their lines would be read back for the rest of them
// (854K rows of 100 floats in 4 bits read back: 169 us kept, 156 streamed; the
// mean's gradient of 242K x 256 floats 186 and 180). Vectors that straddle lines (rows of odd strides) are better put
// together in the cache: dx of 40K x 323 in bf16 103 us streamed, 90 kept.
// So are the layer's, of which a wave has 64 bytes of a row at a time: 242K x
// 256 in bf16 86 us streamed, 77 kept.
template <typename T, int Q>
__device__ __forceinline__ void store_whole(T* p, const float* x, bool streamed) {
  cols_t<T, Q> v;
#pragma unroll
  for (int q = 0; q < Q; ++q) v[q] = (T)x[q];
  if constexpr (sizeof(v) % 4 == 0) {
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(v) / 4)));
    if (streamed) {
      // (as words: two stores of one type would be made one, and lose their kind)
      __builtin_nontemporal_store(__builtin_bit_cast(words, v), reinterpret_cast<words*>(p));
      return;
    }
  }
  *reinterpret_cast<cols_t<T, Q>*>(p) = v;
}
template <typename T, int Q>
__device__ __forceinline__ bool whole_aligned(const T* p) {
  return reinterpret_cast<uintptr_t>(p) % (Q * sizeof(T) < 16 ? Q * sizeof(T) : 16) == 0;
}

// Stores columns [0, valid) of x.
template <typename T, int Q, bool STREAMED = true>
__device__ __forceinline__ void store_cols(T* p, int valid, const float* x) {
  if (valid >= Q) {
    store_whole<T, Q>(p, x, STREAMED && whole_aligned<T, Q>(p));
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (q < valid) p[q] = (T)x[q];
  }
}

// load_cols() and store_cols() of 8 columns of 16 bits in which a row's end of 4
// to 7 has a vector of 4 (us, without it / with: norm of 854K x 100 bf16 to 8 bits
// 120 / 95, of 854K x 103 169 / 129, gradients 352 / 200, dropout with the
// residual 250 / 167; whole rows of 256 within 2 %, to 4 bits 52 / 55).
template <typename T, int Q>
__device__ __forceinline__ void load_row(const T* p, int valid, float* x) {
  if constexpr (Q == 8 && sizeof(T) == 2) {
    if (valid < 8 && valid >= 4) {
      load_cols<T, 4>(p, 4, x);
      load_cols<T, 4>(p + 4, valid - 4, x + 4);
      return;
    }
  }
  load_cols<T, Q>(p, valid, x);
}
template <typename T, int Q>
__device__ __forceinline__ void store_row(T* p, int valid, const float* x) {
  if constexpr (Q == 8 && sizeof(T) == 2) {
    if (valid < 8 && valid >= 4) {
      store_cols<T, 4>(p, 4, x);
      store_cols<T, 4>(p + 4, valid - 4, x + 4);
      return;
    }
  }
  store_cols<T, Q>(p, valid, x);
}

// The layout of packed rows (massive_row_format): codes from byte 0, the
// groups' floats from floats_at on.
struct PackedRows {
  int32_t d;          // values per row
  int32_t group_log2; // columns per group as a power of two, or 31: one group
  int32_t floats_at;
  int64_t row_bytes;
};

// Q columns of a packed row from column c on (c a multiple of Q): codes and
// their group's floats, and the values that they stand for; zeros until they
// are loaded. A row's floats follow its codes, so that Q codes can be read from
// any column on.
template <int BITS, int Q>
struct PackedCols {
  static constexpr int kBytes = Q * BITS / 8;  // 2, 4 or 8
  typedef uint32_t raw __attribute__((ext_vector_type(kBytes > 4 ? 2 : 1), aligned(4)));
  raw w = (raw)0;
  float step = 0.0f, lo = 0.0f;

  __device__ __forceinline__ void load(const uint8_t* row, const PackedRows& f, int c) {
    const uint8_t* p = row + (int64_t)c * BITS / 8;
    if constexpr (kBytes == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
    else w = *reinterpret_cast<const raw*>(p);
    const float* s = reinterpret_cast<const float*>(row + f.floats_at) + (c >> f.group_log2) * (BITS == 8 ? 1 : 2);
    if constexpr (BITS == 8) {
      step = s[0];
    } else {
      lo = s[0];
      step = s[1];
    }
  }
  __device__ __forceinline__ float value(int q) const {
    if constexpr (BITS == 8) return (float)(int8_t)(w[q / 4] >> (8 * (q % 4))) * step;
    else return lo + (float)((w[q / 8] >> (4 * (q % 8))) & 15u) * step;
  }
  __device__ __forceinline__ void values(float* x) const {
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] = value(q);
  }
};

}  // namespace ms
