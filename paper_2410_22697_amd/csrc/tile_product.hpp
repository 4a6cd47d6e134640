// tile_product.hpp - products of two tall operands, both through LDS.
//
// A block of four waves makes 64 NB by 128 results: a wave 32 NB by 64, 2 NB
// squares of the matrix unit's 32 x 32. The operands come in steps of 64 bytes
// of k. Rows of whole, aligned units go to LDS directly, two steps ahead, in
// three buffers; others come through registers, one step ahead, in two. Either
// way there is one barrier a step. An operand
// lies along k (a row of k for each of its columns in the product) or across it
// (a row of columns for each k, which LDS's transposing reads turn).
//
// The second operand's columns become the lanes, the first's the registers: a
// lane ends up with four neighbours of the first at a time, for one of the
// second.
//
// Measured: rows along k, 110K by 2048 outputs in bf16, us for each 256 of k from
// 512 to 1024, beside what begins and ends a tile: 108 to 117 (1 PFLOP/s; through
// registers 128; fp32 at 137 TFLOP/s). Parts of the loop in turn, on one card
// where the whole was 114: without the LDS reads 94, without the loads 76, the
// products alone 46, the loads alone 87 to 105 (a tile of 256 by 128 reads a byte
// for each 43 products, so that is 13 to 15 TB/s from L2). The loads are the
// longest part and the LDS reads, for which the loop's waves wait too, come on top
// of them: neither alone is what bounds it.
#pragma once

#include "gated_rules.hpp"
#include "linear_kernels.hpp"
#include "linear_weights.hpp"

namespace ms {

constexpr int kTileNT = 256;

// k of a step: four units of 16 bytes, two products.
template <typename T>
constexpr int tile_step() {
  return kTileStepBytes / sizeof(T);
}

// Both kinds of operand hold what a thread takes of a step: whole() asks for it
// where the step's k are all there, and ragged() where some lie behind the last
// one (left out as k_along() leaves them out); either goes on to the next step,
// and put() gives it to LDS. direct() is whole() and put() without the registers
// between, for rows whose units are aligned. A thread's units lie in LDS at
// 16 bytes times its number, for that reason; what is where is settled by which
// units it reads.
typedef __attribute__((address_space(1))) const void global_void;
typedef __attribute__((address_space(3))) void lds_void;
__device__ __forceinline__ void tile_direct(const void* from, char* to) {
  __builtin_amdgcn_global_load_lds((global_void*)from, (lds_void*)(to + threadIdx.x / MS_WAVE * (MS_WAVE * 16)), 16, 0, 0);
}

// Four rows' 16-bit values of a column, for 16 lanes: their own 4 columns of 16,
// row by row. (The qualifier is what tells the compiler that the read need not
// wait for what direct() has on its way; tile_arrived() has waited for what counts.)
__device__ __forceinline__ uint2 tile_turned(const char* __restrict__ p) {
  typedef short short4v __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) short4v* lds_ptr;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p));
}

// An operand along k, COLS columns of it: column c's row of k begins at
// where(c). In LDS the units of a column change places, so that eight columns'
// same units lie in distinct banks.
template <typename T, int COLS>
struct TileAlong {
  static constexpr int kV = 16 / sizeof(T), kPer = COLS * 4 / kTileNT, kBytes = COLS * kTileStepBytes;
  const T* p[kPer];
  u32x4 v[kPer];

  static __device__ __forceinline__ int unit() { return (threadIdx.x % 4) ^ (threadIdx.x / 8 % 4); }
  template <typename F>
  __device__ __forceinline__ void begin(F where) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) p[i] = where((int)threadIdx.x / 4 + i * (kTileNT / 4)) + unit() * kV;
  }
  __device__ __forceinline__ void direct(char* to) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      tile_direct(p[i], to + i * (kTileNT * 16));
      p[i] += tile_step<T>();
    }
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
    const int64_t k = k0 + unit() * kV;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      v[i] = k_along(p[i] - k, k, K);
      p[i] += tile_step<T>();
    }
  }
  __device__ __forceinline__ void put(char* to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) *reinterpret_cast<u32x4*>(to + (threadIdx.x + i * kTileNT) * 16) = v[i];
  }
  // the columns c0 to c0 + 31 in the step's half s
  static __device__ __forceinline__ u32x4 fragment(const char* from, int c0, int s) {
    const int lane = lane_id(), c = c0 + lane % 32, u = 2 * s + lane / 32;
    return *reinterpret_cast<const u32x4*>(from + (c * 4 + (u ^ ((c >> 1) & 3))) * 16);
  }
};

// An operand across k. Its columns are read in units of 16 bytes that are all
// there: the last one ends with the row (tile_column() says which columns it
// holds), one behind it repeats it, and its results go nowhere or are stored
// twice. Rows of less than 16 bytes are read value by value, by ragged() alone.
// In LDS 32 bytes change places within their row, so that four rows' same ones
// (what 16 lanes read transposed) lie in distinct banks.
template <typename T, int COLS>
struct TileAcross {
  static constexpr int kV = 16 / sizeof(T), kPer = COLS * 4 / kTileNT, kColUnits = COLS / kV, kPitch = COLS * sizeof(T);
  static constexpr int kBytes = tile_step<T>() * kPitch;
  static constexpr int kRows = kTileNT / kColUnits;  // that the block takes at a time: a thread's columns are the same in all of them
  static_assert(kTileNT % kColUnits == 0 && kRows % 4 == 0, "");
  const T* p;
  int64_t stride;
  int narrow;  // columns, where there are less than a unit's
  u32x4 v[kPer];

  // where(c, first, columns, stride): the row of k = 0, which of its columns position c is, how many there are
  template <typename F>
  __device__ __forceinline__ void begin(F where) {
    int c, columns;
    const T* row = where((((int)threadIdx.x % kColUnits) ^ ((int)threadIdx.x / kColUnits % 4 * 2)) * kV, c, columns, stride);
    narrow = columns < kV ? columns : 0;
    p = row + (columns < kV ? 0 : min(c, columns - kV)) + (int64_t)(threadIdx.x / kColUnits) * stride;
  }
  __device__ __forceinline__ void direct(char* to) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      tile_direct(p, to + i * (kTileNT * 16));
      p += kRows * stride;
    }
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
    for (int i = 0; i < kPer; ++i) *reinterpret_cast<u32x4*>(to + (threadIdx.x + i * kTileNT) * 16) = v[i];
  }
  // the columns c0 to c0 + 31 in the step's half s
  static __device__ __forceinline__ u32x4 fragment(const char* from, int c0, int s) {
    const int lane = lane_id();
    if constexpr (sizeof(T) == 2) {
      const int group = lane / 16, i = lane % 16, r = 16 * s + 8 * (group / 2) + i / 4, chunk = c0 / 16 + group % 2;
      const char* p = from + r * kPitch + (chunk ^ (i / 4)) * 32 + i % 4 * 8;
      const uint2 a = tile_turned(p), b = tile_turned(p + 4 * kPitch);
      return u32x4{a.x, a.y, b.x, b.y};
    } else {
      const int c = c0 + lane % 32;
      const char* p = from + (8 * s + 4 * (lane / 32)) * kPitch + c % 8 * 4;
      u32x4 v;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = *reinterpret_cast<const uint32_t*>(p + q * kPitch + (c / 8 ^ q) * 32);
      return v;
    }
  }
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

constexpr int kTileBuffers[2] = {2, 3};  // of the two ways through registers and direct
template <typename A, typename B>
constexpr int tile_lds(bool direct) {
  return kTileBuffers[direct] * (A::kBytes + B::kBytes);
}

// A segment of the reduction: K of it, of which the steps all there are taken by
// whole() if `plain` (by ragged() else; direct() is for plain ones).
struct TileSegment {
  int64_t K;
  bool plain;
};

// acc[i][j] += the products of the first operand's columns wave % 2 * 32 NB + 32 i
// on and the second's wave / 2 * 64 + 32 j on, in the step that both have in LDS.
template <typename T, int NB, typename A, typename B>
__device__ __forceinline__ void tile_multiply(const char* first, const char* second, f32x16 (&acc)[NB][2]) {
  const int wave = wave_uniform((int32_t)wave_id());
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    u32x4 a[NB], b[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) b[j] = B::fragment(second, wave / 2 * 64 + 32 * j, s);
#pragma unroll
    for (int i = 0; i < NB; ++i) a[i] = A::fragment(first, wave % 2 * (32 * NB) + 32 * i, s);
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
}

// acc += the products over SEGMENTS segments, the first of them not empty;
// begin(g) begins segment g of both operands. Through registers: a step is on its
// way in them while the one before it is multiplied.
template <typename T, int NB, int SEGMENTS, typename A, typename B, typename F>
__device__ __forceinline__ void tile_product(A& first, B& second, const TileSegment (&segments)[SEGMENTS], F begin, char* lds, f32x16 (&acc)[NB][2]) {
  constexpr int kBuffer = A::kBytes + B::kBytes, kStep = tile_step<T>();
  int buffer = 0;
  auto put = [&] {
    first.put(lds + buffer);
    second.put(lds + buffer + A::kBytes);
    __syncthreads();
  };
  auto step = [&] {
    __builtin_amdgcn_sched_barrier(0);  // the step's loads stay ahead of the products that they run beside, and its stores behind them
    tile_multiply<T, NB, A, B>(lds + buffer, lds + buffer + A::kBytes, acc);
    __builtin_amdgcn_sched_barrier(0);
    buffer = kBuffer - buffer;
    put();
  };
  begin(0);
  if (segments[0].plain && kStep <= segments[0].K) {
    first.whole();
    second.whole();
  } else {
    first.ragged(0, segments[0].K);
    second.ragged(0, segments[0].K);
  }
  put();
  int64_t k0 = kStep;
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
  tile_multiply<T, NB, A, B>(lds + buffer, lds + buffer + A::kBytes, acc);
  __syncthreads();
}

// Waits until this wave's memory reads but the last LEFT have arrived.
template <int LEFT>
__device__ __forceinline__ void tile_arrived() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4 | 15 << 8);
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
// Waits until this wave's LDS accesses are done, and for the block's other waves
// to come here.
__device__ __forceinline__ void tile_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// The same with direct(), in three buffers: two steps are on their way while the
// one before them is multiplied. A step goes to the buffer that was multiplied
// before the barrier, and is read behind a barrier that every wave comes to once
// its own part has arrived: reads arrive in order, so what is left then is the
// step asked for last.
template <typename T, int NB, int SEGMENTS, typename A, typename B, typename F>
__device__ __forceinline__ void tile_product_direct(A& first, B& second, const TileSegment (&segments)[SEGMENTS], F begin, char* lds, f32x16 (&acc)[NB][2]) {
  constexpr int kBuffer = A::kBytes + B::kBytes, kStep = tile_step<T>(), kAsked = A::kPer + B::kPer;
  int64_t k0 = 0, K = segments[0].K;
  int left = (int)((K + kStep - 1) / kStep + (SEGMENTS > 1 ? (segments[SEGMENTS - 1].K + kStep - 1) / kStep : 0));
  int to = 0, from = 0;
  bool direct = false;  // how the step asked for last comes
  auto after = [&](int buffer) { return buffer == 2 * kBuffer ? 0 : buffer + kBuffer; };
  auto ask_direct = [&] {
    first.direct(lds + to);
    second.direct(lds + to + A::kBytes);
    to = after(to);
    k0 += kStep;
    --left;
  };
  auto ask = [&] {
    if (SEGMENTS > 1 && k0 >= K) {
      begin(1);
      k0 = 0;
      K = segments[SEGMENTS - 1].K;
    }
    direct = k0 + kStep <= K;
    if (direct) {
      ask_direct();
    } else {
      first.ragged(k0, K);
      second.ragged(k0, K);
      first.put(lds + to);
      second.put(lds + to + A::kBytes);
      to = after(to);
      k0 += kStep;
      --left;
    }
  };
  auto multiply = [&] {
    __builtin_amdgcn_sched_barrier(0);
    tile_multiply<T, NB, A, B>(lds + from, lds + from + A::kBytes, acc);
    __builtin_amdgcn_sched_barrier(0);
    from = after(from);
  };
  auto sync = [&] {
    if (direct) tile_arrived<kAsked>();
    else tile_arrived<0>();
    tile_barrier();
  };
  begin(0);
  const int steps = left;
  ask();
  if (left > 0) ask();
#pragma unroll 1
  while (left > 0) {
    if (direct) {
#pragma unroll 1
      while (k0 + kStep <= K) {
        tile_arrived<kAsked>();
        tile_barrier();
        ask_direct();
        multiply();
      }
    }
    if (left == 0) break;
    sync();
    ask();
    multiply();
  }
  if (steps > 1) {
    sync();
    multiply();
  }
  tile_arrived<0>();
  tile_barrier();
  multiply();
  __syncthreads();
}

// Keeps a wave's memory reads and writes before it and behind it on their sides
// (other instructions may pass: with none passing, silu's gradients in bf16 spill
// three registers).
__device__ __forceinline__ void tile_in_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(1);
}

// The same for a second operand that the threads compute as they put it. The
// first's steps come directly, two ahead; the second's through registers, three
// ahead, in two sets, and a thread puts its part of a step a step ahead. What a
// wave asks for arrives in the order of asking, a step's part of the first
// before the next but one's of the second: so much may be left when a step is
// multiplied (kLeft) and when the next is put (kLeftPut). Both counts hang on
// that order of asking, which is why it is not left to the compiler
// (tile_in_order()): a read for the second that overtook the first's would leave
// a buffer on its way when it is multiplied. (What put() stores is in the queue
// too, ahead of what is asked for behind it, and makes a wait longer at most.)
template <typename T, int NB, typename A, typename B>
constexpr int tile_made_lds() {
  return 3 * A::kBytes + 2 * B::kBytes;
}
template <typename T, int NB, typename A, typename B>
__device__ __forceinline__ void tile_product_made(A& first, B& second, int64_t K, char* lds, f32x16 (&acc)[NB][2]) {
  constexpr int kStep = tile_step<T>(), kLeftPut = A::kPer + B::kAsked, kLeft = B::kAsked + kLeftPut;
  const int steps = (int)((K + kStep - 1) / kStep);
  const bool whole = K % kStep == 0;  // the last step too
  int to = 0, from = 0;
  auto after = [&](int buffer) { return buffer == 2 * A::kBytes ? 0 : buffer + A::kBytes; };
  auto ask_first = [&](int s) {
    if (s + 1 < steps || whole) {
      first.direct(lds + to);
    } else {
      first.ragged((int64_t)s * kStep, K);
      first.put(lds + to);
    }
    to = after(to);
  };
  auto ask_second = [&](int s, auto set) {
    if (s + 1 < steps || whole) second.template whole<set()>();
    else second.template ragged<set()>((int64_t)s * kStep, K);
  };
  auto put = [&](auto set, auto all) { second.template put<set(), all()>(lds + 3 * A::kBytes + set() * B::kBytes); };
  auto multiply = [&](auto set) {
    __builtin_amdgcn_sched_barrier(0);
    tile_multiply<T, NB, A, B>(lds + from, lds + 3 * A::kBytes + set() * B::kBytes, acc);
    __builtin_amdgcn_sched_barrier(0);
    from = after(from);
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  auto step = [&](int s, auto now, auto next) {  // any step: waits for all, so no count hangs on its order
    tile_arrived<0>();
    tile_barrier();
    if (s + 1 < steps) put(next, std::false_type());
    if (s + 2 < steps) ask_first(s + 2);
    if (s + 3 < steps) ask_second(s + 3, next);
    multiply(now);
  };
  auto step_between = [&](auto now, auto next) {  // the steps asked for are whole
    tile_arrived<kLeft>();
    tile_barrier();
    tile_arrived<kLeftPut>();
    put(next, std::true_type());
    first.direct(lds + to);
    to = after(to);
    tile_in_order();
    second.template whole<next()>();
    multiply(now);
  };
  ask_first(0);
  ask_second(0, even);
  tile_arrived<0>();
  put(even, std::false_type());
  if (steps > 1) ask_first(1);
  if (steps > 1) ask_second(1, odd);
  if (steps > 2) ask_second(2, even);
  int s = 0;
  step(s++, even, odd);
  if (s < steps) step(s++, odd, even);
  tile_arrived<0>();  // (whichever way the steps so far came: the compiler's own count of what is on its way begins anew)
#pragma unroll 1
  for (; s + 5 < steps; s += 2) {
    step_between(even, odd);
    step_between(odd, even);
  }
#pragma unroll 1
  for (; s < steps; s += 2) {
    step(s, even, odd);
    if (s + 1 < steps) step(s + 1, odd, even);
  }
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
