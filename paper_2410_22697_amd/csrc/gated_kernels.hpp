// gated_kernels.hpp - a gated layer and what its gradients need.
//
//   g = [x | x2] Wg^T + bg      u = [x | x2] Wu^T + bu      y = act(g) u
//   dg = dy u act'(g)           du = dy act(g)
//   dx = [dg | du] [Wg; Wu]     dW = [dg | du]^T [x | x2]   db = sums over the rows
//
// Both products of an output are made by the same lane, so that the activation
// and the product need no other pass over memory.
#pragma once

#include "gated_rules.hpp"
#include "linear_few.hpp"
#include "linear_kernels.hpp"
#include "tile_product.hpp"

namespace ms {

template <typename T>
struct Gated {
  Operand<T> x[2];
  Weights<T> w[2];  // of each input's columns, along k: n rows of the gate, then n of the other half
  const T* bias;    // [2 n]
  T *y, *pre;       // pre [rows][2 n]
  int64_t y_stride, pre_stride, rows;
  int n, act;
};

template <int V>
__device__ __forceinline__ int round_up_to(int x) {
  return (x + V - 1) / V * V;
}

// Calls f(act) with the activation as a type.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  if (act == kActSilu) f(std::integral_constant<int, kActSilu>());
  else if (act == kActGelu) f(std::integral_constant<int, kActGelu>());
  else if (act == kActRelu) f(std::integral_constant<int, kActRelu>());
  else f(std::integral_constant<int, kActNone>());
}

// Many rows: 128 rows by 32 NB outputs of both halves a block; a wave has 16 NB
// outputs of the gate and the same of the other half.
// 110K x 256 -> 1024 bf16 171 us (680 TFLOP/s): by the slope in k, 90 to 117 are the
// loop (tile_product.hpp says what of), the others the begin and the end of tiles,
// beside which a block neither loads nor multiplies; with pre, whose end stores
// three times as much, 286. 16391 x 100 + 100 -> 323 fp32 70 (60 TFLOP/s of what is
// asked for: 323 outputs take 384, two inputs of 100 take 224 of k, and 774 tiles
// are a few more than the chip holds at a time).
template <typename T, int NB, bool DIRECT>
__global__ __launch_bounds__(kTileNT, 2) void k_gated_tile(Gated<T> a, int tiles_n, int64_t blocks) {
  typedef TileAlong<T, 64 * NB> A;
  typedef TileAlong<T, kTileSecond> B;
  typedef TileTurn<T, 16 * NB> Turn;
  constexpr int kOut = 16 * NB;
  constexpr int kLds = tile_lds<A, B>(DIRECT) > 4 * Turn::kBytes ? tile_lds<A, B>(DIRECT) : 4 * Turn::kBytes;
  // (all in one array: between two, the compiler would have LDS reads wait for whatever is on its way to the other)
  __shared__ __align__(16) char lds[kLds + 64 * NB * sizeof(float)];
  float(*bias)[32 * NB] = reinterpret_cast<float(*)[32 * NB]>(lds + kLds);
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t r0 = tile / tiles_n * kTileSecond;
  const int n0 = (int)(tile % tiles_n) * (32 * NB);
  if ((int)threadIdx.x < 64 * NB) {
    const int h = threadIdx.x / (32 * NB), c = n0 + threadIdx.x % (32 * NB);
    bias[h][threadIdx.x % (32 * NB)] = a.bias && c < a.n ? (float)a.bias[h * a.n + c] : 0.0f;
  }
  A weights;
  B rows;
  f32x16 acc[NB][2] = {};
  const TileSegment segments[2] = {{a.x[0].K, true}, {a.x[1].K, true}};
  auto begin = [&](int g) {
    const T *xp = g ? a.x[1].p : a.x[0].p, *wp = g ? a.w[1].p : a.w[0].p;
    const int64_t x_stride = g ? a.x[1].stride : a.x[0].stride;
    weights.begin([&](int c) {
      const int square = c / 32 % NB, out = n0 + c / (32 * NB) * kOut + square % (NB / 2) * 32 + c % 32;
      return wp + (int64_t)((square >= NB / 2 ? a.n : 0) + min(out, a.n - 1)) * a.w[0].stride;
    });
    rows.begin([&](int r) { return xp + min(r0 + r, a.rows - 1) * x_stride; });  // those that are not there repeat the last one
  };
  if constexpr (DIRECT) tile_product_direct<T, NB>(weights, rows, segments, begin, lds, acc);
  else tile_product<T, NB>(weights, rows, segments, begin, lds, acc);
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const Turn turn = {lds + wave * Turn::kBytes};
  const int c0 = wave % 2 * kOut;
  // f(gate, other half) for every output, to out
  auto each = [&](T* out, int64_t stride, auto f) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int i = 0; i < NB / 2; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = c0 + 32 * i + 8 * q + 4 * (lane / 32);
          const f32x4 bg = *reinterpret_cast<const f32x4*>(&bias[0][c]), bu = *reinterpret_cast<const f32x4*>(&bias[1][c]);
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = f(acc[i][j][4 * q + e] + bg[e], acc[i + NB / 2][j][4 * q + e] + bu[e]);
          turn.in(32 * i, q, v);
        }
      turn.out(out, stride, r0 + wave / 2 * 64 + 32 * j, a.rows, n0 + c0, a.n);
    }
  };
  if (a.pre) {
    each(a.pre, a.pre_stride, [](float g, float) { return g; });
    each(a.pre + a.n, a.pre_stride, [](float, float u) { return u; });
  }
  with_act(a.act, [&](auto act) { each(a.y, a.y_stride, [&](float g, float u) { return act_value(g, act()) * u; }); });
}

// Few rows: 32 rows by 32 outputs of both halves a block, its eight waves share
// the reduction. Bound by the trips to memory that follow each other: a wave makes
// an eighth of those that a tile makes. 250 x 256 -> 1024 fp32 12.1 us where
// narrow tiles take 22.7.
template <typename T>
__global__ __launch_bounds__(kFewNT) void k_gated_few(Gated<T> a, int tiles_n) {
  __shared__ float halves[2][32 * 32];
  const int64_t r0 = (int64_t)(blockIdx.x / tiles_n) * 32;
  const int n0 = (int)(blockIdx.x % tiles_n) * 32;
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    const Weights<T> w[2] = {{a.w[0].p + (int64_t)h * a.n * a.w[0].stride, a.w[0].stride}, {a.w[1].p + (int64_t)h * a.n * a.w[1].stride, a.w[1].stride}};
    few_product<T, false, false, 2>(a.x, w, r0, a.rows, n0, a.n, [&](int64_t row, int col, float z) {
      if (a.bias) z += (float)a.bias[h * a.n + col];
      halves[h][(row - r0) * 32 + col - n0] = z;
      if (a.pre) a.pre[row * a.pre_stride + h * a.n + col] = (T)z;
    });
    __syncthreads();
  }
  for (int at = threadIdx.x; at < 1024; at += kFewNT)
    if (r0 + at / 32 < a.rows && n0 + at % 32 < a.n)
      a.y[(r0 + at / 32) * a.y_stride + n0 + at % 32] = (T)(act_value(halves[0][at], a.act) * halves[1][at]);
}

// ------------------------------------------------------------------ gradients

template <typename T>
struct GatedDz {
  const T *dy, *pre;
  T* dz;         // [rows][2 n], or null
  float* parts;  // [parts][2 n] of db, or null
  int64_t rows, part, dy_stride, pre_stride;
  int n, act, groups;
};

// dz = [dg | du], and the sums of each part of the rows, of dz before it is
// rounded. Bound by memory: 110K x 1024 bf16 212 us (5.3 TB/s).
template <typename T>
__global__ __launch_bounds__(kGateNT) void k_gated_dz(GatedDz<T> a) {
  constexpr int kV = 16 / sizeof(T), kAhead = 2;
  __shared__ float joined[kGateWays][2][kGateUnits * kV];
  const int unit = threadIdx.x % kGateUnits, way = threadIdx.x / kGateUnits;
  const int c = (int)(blockIdx.x % a.groups) * (kGateUnits * kV) + unit * kV, valid = a.n - c;
  const int64_t first = (int64_t)(blockIdx.x / a.groups) * a.part, end = min(a.rows, first + a.part);
  float sums[2][kV] = {};
  with_act(a.act, [&](auto act) {
    if (valid <= 0) return;
    for (int64_t i0 = first + way; i0 < end; i0 += kAhead * kGateWays) {
      float dy[kAhead][kV], g[kAhead][kV], u[kAhead][kV];
#pragma unroll
      for (int v = 0; v < kAhead; ++v) {
        const int64_t i = i0 + v * kGateWays;
        if (i >= end) continue;
        load_row<T, kV>(a.dy + i * a.dy_stride + c, valid, dy[v]);
        load_row<T, kV>(a.pre + i * a.pre_stride + c, valid, g[v]);
        load_row<T, kV>(a.pre + i * a.pre_stride + a.n + c, valid, u[v]);
      }
#pragma unroll
      for (int v = 0; v < kAhead; ++v) {
        const int64_t i = i0 + v * kGateWays;
        if (i >= end) continue;
        float dg[kV], du[kV];
#pragma unroll
        for (int q = 0; q < kV; ++q) {
          dg[q] = act() == kActNone ? dy[v][q] * u[v][q] : act_grad(dy[v][q] * u[v][q], g[v][q], act());
          du[q] = dy[v][q] * act_value(g[v][q], act());
          if (q < valid) {
            sums[0][q] += dg[q];
            sums[1][q] += du[q];
          }
        }
        if (!a.dz) continue;
        store_cols<T, kV, false>(a.dz + i * (2 * (int64_t)a.n) + c, valid, dg);
        store_cols<T, kV, false>(a.dz + i * (2 * (int64_t)a.n) + a.n + c, valid, du);
      }
    }
  });
  if (!a.parts) return;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int q = 0; q < kV; ++q) joined[way][h][unit * kV + q] = sums[h][q];
  __syncthreads();
  for (int at = threadIdx.x; at < 2 * kGateUnits * kV; at += kGateNT) {
    const int h = at / (kGateUnits * kV), j = at % (kGateUnits * kV), col = (int)(blockIdx.x % a.groups) * (kGateUnits * kV) + j;
    float t = 0.0f;
#pragma unroll
    for (int v = 0; v < kGateWays; ++v) t += joined[v][h][j];
    if (col < a.n) a.parts[(int64_t)(blockIdx.x / a.groups) * 2 * a.n + h * a.n + col] = t;
  }
}

// dx = dz w: 128 rows by 64 NB columns a block, and of dz's columns as many as a
// part has. parts: [parts][rows][cols] if there are several, else null; of wide
// tiles there are always enough for one part.
// 110K x 256 -> 1024 bf16 168 to 180 us (690 TFLOP/s; 860 tiles where the chip
// holds 512 at a time are two rounds), fp32 16391 x 200 -> 323 80 with the parts'
// sum 11 more (95 in one part).
template <typename T, int NB, bool DIRECT>
__global__ __launch_bounds__(kTileNT, 2) void k_gated_dx(LinearDx<T> a, float* parts, int64_t part, int tiles_n, int64_t tiles, int64_t blocks) {
  typedef TileAcross<T, 64 * NB> A;
  typedef TileAlong<T, kTileSecond> B;
  typedef TileTurn<T, 32 * NB> Turn;
  typedef TileTurn<float, 32 * NB> WideTurn;
  constexpr int kTurns = 4 * (NB == 2 ? WideTurn::kBytes : Turn::kBytes), kLds = tile_lds<A, B>(DIRECT) > kTurns ? tile_lds<A, B>(DIRECT) : kTurns;
  __shared__ __align__(16) char lds[kLds];
  const int64_t block = tile_of_block(blockIdx.x, blocks), tile = block % tiles, p = block / tiles, from = p * part;
  const int64_t r0 = tile / tiles_n * kTileSecond;
  const int n0 = (int)(tile % tiles_n) * (64 * NB);
  A weights;
  B rows;
  f32x16 acc[NB][2] = {};
  const TileSegment segments[1] = {{min(part, a.dz.K - from), a.cols >= 16 / (int)sizeof(T)}};
  auto begin = [&](int) {
    weights.begin([&](int c, int& at, int& columns, int64_t& stride) {
      at = n0 + c;
      columns = a.cols;
      stride = a.w.stride;
      return a.w.p + from * stride;
    });
    rows.begin([&](int r) { return a.dz.p + from + min(r0 + r, a.rows - 1) * a.dz.stride; });
  };
  if constexpr (DIRECT) tile_product_direct<T, NB>(weights, rows, segments, begin, lds, acc);
  else tile_product<T, NB>(weights, rows, segments, begin, lds, acc);
  const int wave = wave_uniform((int32_t)wave_id());
  const int c0 = n0 + wave % 2 * (32 * NB);
  if constexpr (NB == 2) {
    if (parts) {
      const WideTurn turn = {lds + wave * WideTurn::kBytes};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            turn.in(32 * i, q, v);
          }
        const int64_t at = r0 + wave / 2 * 64 + 32 * j;
        turn.units([&](int r, int c, cols_t<float, 4> v) {
          if (at + r >= a.rows || c0 + c >= round_up_to<16 / (int)sizeof(T)>(a.cols)) return;
          const int col = tile_column<T>(c0 + c, a.cols);
          const float four[4] = {v[0], v[1], v[2], v[3]};
          store_cols<float, 4, false>(parts + (p * a.rows + at + r) * a.cols + col, a.cols - col, four);
        });
      }
      return;
    }
  }
  const Turn turn = {lds + wave * Turn::kBytes};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        turn.in(32 * i, q, v);
      }
    const int64_t at = r0 + wave / 2 * 64 + 32 * j;
    constexpr int kV = 16 / sizeof(T);
    turn.units([&](int r, int c, cols_t<T, kV> v) {
      const int64_t row = at + r;
      if (row >= a.rows || c0 + c >= a.cols) return;
      const int col = tile_column<T>(c0 + c, a.cols), s = col >= a.split ? 1 : 0;
      if (col + kV <= (s ? a.cols : a.split)) {
        *reinterpret_cast<cols_t<T, kV>*>(a.dx[s] + row * a.dx_stride[s] + col - (s ? a.split : 0)) = v;
      } else {
#pragma unroll
        for (int e = 0; e < kV; ++e)
          if (col + e < a.cols) linear_dx_store(a, row, col + e, (float)v[e]);
      }
    });
  }
}

// dw = dz^T [x | x2] and db by parts of the rows, or as they are if one part has
// all rows (`parts` and `sums` null).
template <typename T>
struct GatedDw {
  Operand<T> dz, x[2];
  float *parts, *sums;  // [parts][n][k0 + k1], [parts][n]
  T *dw, *db;           // db null: not asked for
  int64_t dw_stride, rows, part;
  int n, k[2], second;  // n: outputs of both halves; second: the position of the second input's first column
  int tiles_n, tiles_k;
};

// A block's part of dw: row(p) is the output at position p of its 128 (a.n: none).
template <typename T, int NB, typename F>
__device__ __forceinline__ void dw_out(const GatedDw<T>& a, char* lds, const f32x16 (&acc)[NB][2], int64_t part, int k0, F row_at) {
  constexpr int kV = 16 / sizeof(T);
  typedef TileTurn<float, 32 * NB> Turn;
  const int wave = wave_uniform((int32_t)wave_id());
  const Turn turn = {lds + wave * Turn::kBytes};
  const int all = a.k[0] + a.k[1], c0 = k0 + wave % 2 * (32 * NB);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        turn.in(32 * i, q, v);
      }
    turn.units([&](int r, int c, cols_t<float, 4> v) {
      const int at = c0 + c, s = at >= a.second ? 1 : 0, c1 = at - (s ? a.second : 0), columns = s ? a.k[1] : a.k[0];
      const int row = row_at(wave / 2 * 64 + 32 * j + r);
      if (row >= a.n || c1 >= round_up_to<kV>(columns)) return;
      const int col = tile_column<T>(c1, columns), to = (s ? a.k[0] : 0) + col;
      const float four[4] = {v[0], v[1], v[2], v[3]};
      if (a.parts) store_cols<float, 4, false>(a.parts + (part * a.n + row) * (int64_t)all + to, columns - col, four);
      else store_cols<T, 4, false>(a.dw + row * a.dw_stride + to, columns - col, four);
    });
  }
}

// dw = dz^T [x | x2], one part of the rows a block: 128 outputs by 64 NB columns.
// Columns are placed in whole units, the second input's from `second` on.
template <typename T, int NB, bool DIRECT>
__global__ __launch_bounds__(kTileNT, 2) void k_gated_dw(GatedDw<T> a, int64_t blocks) {
  typedef TileAcross<T, 64 * NB> A;
  typedef TileAcross<T, kTileSecond> B;
  typedef TileTurn<float, 32 * NB> Turn;
  constexpr int kLds = tile_lds<A, B>(DIRECT) > 4 * Turn::kBytes ? tile_lds<A, B>(DIRECT) : 4 * Turn::kBytes;
  __shared__ __align__(16) char lds[kLds];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t part = tile / (a.tiles_n * a.tiles_k);
  const int in = (int)(tile % (a.tiles_n * a.tiles_k));
  const int n0 = in / a.tiles_k * kTileSecond, k0 = in % a.tiles_k * (64 * NB);
  const int64_t from = part * a.part, rows = min(a.part, a.rows - from);
  A xs;
  B dzs;
  f32x16 acc[NB][2] = {};
  constexpr int kV = 16 / sizeof(T);
  const TileSegment segments[1] = {{rows, a.n >= kV && a.k[0] >= kV && (a.k[1] == 0 || a.k[1] >= kV)}};
  auto begin = [&](int) {
    xs.begin([&](int c, int& at, int& columns, int64_t& stride) {
      const int s = k0 + c >= a.second && a.k[1] > 0 ? 1 : 0;
      at = k0 + c - (s ? a.second : 0);
      columns = s ? a.k[1] : a.k[0];
      stride = s ? a.x[1].stride : a.x[0].stride;
      return (s ? a.x[1].p : a.x[0].p) + from * stride;
    });
    dzs.begin([&](int c, int& at, int& columns, int64_t& stride) {
      at = n0 + c;
      columns = a.n;
      stride = a.dz.stride;
      return a.dz.p + from * stride;
    });
  };
  if constexpr (DIRECT) tile_product_direct<T, NB>(xs, dzs, segments, begin, lds, acc);
  else tile_product<T, NB>(xs, dzs, segments, begin, lds, acc);
  const int kLast = round_up_to<kV>(a.n);
  dw_out<T, NB>(a, lds, acc, part, k0, [&](int p) { return n0 + p < kLast ? tile_column<T>(n0 + p, a.n) : a.n; });
}

// [dg | du] as an operand across k, made from dy and pre on its way to LDS: COLS
// columns of dg and the same of du, a unit (or W of its columns) of both a thread
// and step. It can leave dz behind, and each thread adds up its columns before
// they are rounded. In bf16 dg and du are rounded to it, as the matrix unit takes
// them: that puts dx's and dw's error at 0.0023 of their size, where the results' own
// rounding leaves 0.0017 (0.0017 too against products of the rounded dz, at 110K x
// 256 -> 1024). The bits that it drops would be a second product each.
template <typename T, int ACT, int COLS = 64, int W = 16 / sizeof(T)>
struct TileGates {
  static constexpr int kCols = COLS, kV = 16 / sizeof(T), kUnits = COLS / W, kNT = kUnits * tile_step<T>(), kPitch = 2 * COLS * sizeof(T), kBytes = tile_step<T>() * kPitch;
  typedef cols_t<T, W> unit_t;
  const T *dy, *pre;
  T* dz;
  int64_t dy_stride, pre_stride;
  int n;
  // two sets of what a thread has asked for: units of dy and of both halves, whether the step has the thread's row, and
  // how far that lies from the place that the step has for it
  static constexpr int kAsked = 3;
  bool live[2];
  int64_t at[2];
  typedef uint32_t raw __attribute__((ext_vector_type(W * sizeof(T) / 4)));
  raw vd[2], vg[2], vu[2];
  float sums[2][W] = {};

  static __device__ __forceinline__ raw read(const T* p) { return __builtin_bit_cast(raw, *reinterpret_cast<const unit_t*>(p)); }
  // rows from `row` on, columns from n0 on (as TileAcross has them)
  __device__ __forceinline__ void begin(const GatedDz<T>& a, int64_t row, int n0) {
    const int s = threadIdx.x % kUnits * W, c = min(n0 + s / kV * kV, a.n - kV) + s % kV;
    row += threadIdx.x / kUnits;
    n = a.n;
    dy_stride = a.dy_stride;
    pre_stride = a.pre_stride;
    dy = a.dy + row * dy_stride + c;
    pre = a.pre + row * pre_stride + c;
    dz = a.dz ? a.dz + row * (2 * (int64_t)n) + c : nullptr;
  }
  template <int SET>
  __device__ __forceinline__ void ask(int64_t ahead) {
    vd[SET] = read(dy + ahead * dy_stride);
    vg[SET] = read(pre + ahead * pre_stride);
    vu[SET] = read(pre + ahead * pre_stride + n);
    at[SET] = ahead;
  }
  __device__ __forceinline__ void go_on() {
    dy += tile_step<T>() * dy_stride;
    pre += tile_step<T>() * pre_stride;
  }
  template <int SET>
  __device__ __forceinline__ void whole() {
    live[SET] = true;
    ask<SET>(0);
    go_on();
  }
  template <int SET>
  __device__ __forceinline__ void ragged(int64_t k0, int64_t K) {
    const int r = threadIdx.x / kUnits, in = r % kV;
    const int64_t unit = k0 + (r - in);
    const int skip = K >= kV ? skipped<T>(unit, K) : (unit + in < K ? 0 : kV);
    live[SET] = in >= skip;
    vd[SET] = vg[SET] = vu[SET] = (raw)0u;
    if (live[SET]) ask<SET>(skip && K >= kV ? K - kV - unit : 0);
    go_on();
  }
  // (an addition of its own, never one with the product that v may be: the kernels that sum have the same bits)
  static __device__ __forceinline__ void add(float& sum, float v) {
#pragma clang fp contract(off)
    sum += v;
  }
  // a step's dg and du, which join the sums
  template <int SET>
  __device__ __forceinline__ void make(unit_t (&z)[2]) {
    const unit_t d = __builtin_bit_cast(unit_t, vd[SET]), g = __builtin_bit_cast(unit_t, vg[SET]), u = __builtin_bit_cast(unit_t, vu[SET]);
#pragma unroll
    for (int q = 0; q < W; ++q) {
      const float dy_u = (float)d[q] * (float)u[q];
      const float dg = ACT == kActNone ? dy_u : act_grad(dy_u, (float)g[q], ACT), du = (float)d[q] * act_value((float)g[q], ACT);
      add(sums[0][q], dg);  // (of zeros where the step has no row)
      add(sums[1][q], du);
      z[0][q] = (T)dg;
      z[1][q] = (T)du;
    }
  }
  // leaves them behind; WHOLE: the step has all rows
  template <int SET, bool WHOLE>
  __device__ __forceinline__ void leave(const unit_t (&z)[2]) {
    if (!dz) return;
    if (WHOLE || live[SET]) {
      T* p = WHOLE ? dz : dz + at[SET] * (2 * (int64_t)n);
      *reinterpret_cast<unit_t*>(p) = z[0];
      *reinterpret_cast<unit_t*>(p + n) = z[1];
    }
    dz += tile_step<T>() * (2 * (int64_t)n);
  }
  template <int SET, bool WHOLE>
  __device__ __forceinline__ void put(char* to) {
    static_assert(W == kV && kNT == kTileNT, "");
    unit_t z[2];
    make<SET>(z);
    const int r = threadIdx.x / kUnits, s = threadIdx.x % kUnits;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int place = h * kUnits + s;
      *reinterpret_cast<u32x4*>(to + r * kPitch + ((place / 2 ^ r % 4) * 2 + place % 2) * 16) = __builtin_bit_cast(u32x4, z[h]);
    }
    leave<SET, WHOLE>(z);
  }
  static __device__ __forceinline__ u32x4 fragment(const char* from, int c0, int s) { return TileAcross<T, 2 * COLS>::fragment(from, c0, s); }
};

// The output at each position of a block's COLS of both halves, from column n0 on
// (2 n: none).
template <typename T, int COLS>
__device__ __forceinline__ auto gates_rows(int n0, int n) {
  const int last = round_up_to<16 / (int)sizeof(T)>(n);
  return [=](int p) {
    const int c = n0 + p % COLS;
    return c < last ? p / COLS * n + tile_column<T>(c, n) : 2 * n;
  };
}
// db's sums of a part of the rows, or db if there is one: the threads that share
// columns add up in order. `lds` holds tile_step() rows of 2 COLS floats.
template <typename T, typename B, typename F>
__device__ __forceinline__ void gates_sums(const B& dzs, const GatedDw<T>& a, char* lds, int64_t part, F row_at) {
  float* joined = reinterpret_cast<float*>(lds);
  constexpr int kCols = B::kCols, kW = kCols / B::kUnits;
  const int r = threadIdx.x / B::kUnits, c = threadIdx.x % B::kUnits * kW;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int q = 0; q < kW; ++q) joined[(r * 2 + h) * kCols + c + q] = dzs.sums[h][q];
  __syncthreads();
  const int row = (int)threadIdx.x < 2 * kCols ? row_at(threadIdx.x) : a.n;
  if (row < a.n) {
    float t = 0.0f;
#pragma unroll
    for (int g = 0; g < tile_step<T>(); ++g) t += joined[g * (2 * kCols) + threadIdx.x];
    if (a.sums) a.sums[part * a.n + row] = t;
    else a.db[row] = (T)t;
  }
  __syncthreads();
}

// dw and the sums for db, of dz as TileGates makes it: one launch that reads dy
// and pre once, for inputs of whole units in one tile of columns. Bound by the
// activation's slope and by memory, which have to share a wave's turns with the
// products: 110K x 256 -> 1024 bf16 295 us and the parts' sum 17 (k_gated_dz, 212,
// and k_gated_dw, 160, each at its own bound, take 60 more).
template <typename T, int NB, int ACT>
__global__ __launch_bounds__(kTileNT, 2) void k_gated_dw_made(GatedDw<T> a, GatedDz<T> z, int64_t blocks) {
  typedef TileAcross<T, 64 * NB> A;
  typedef TileGates<T, ACT> B;
  typedef TileTurn<float, 32 * NB> Turn;
  constexpr int kMade = tile_made_lds<T, NB, A, B>(), kLds = kMade > 4 * Turn::kBytes ? kMade : 4 * Turn::kBytes;
  static_assert(kLds >= tile_step<T>() * 128 * (int)sizeof(float), "");
  __shared__ __align__(16) char lds[kLds];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t part = tile / a.tiles_n;
  const int n0 = (int)(tile % a.tiles_n) * 64;
  const int64_t from = part * a.part, rows = min(a.part, a.rows - from);
  A xs;
  B dzs;
  f32x16 acc[NB][2] = {};
  xs.begin([&](int c, int& at, int& columns, int64_t& stride) {
    const int s = c >= a.second && a.k[1] > 0 ? 1 : 0;
    at = c - (s ? a.second : 0);
    columns = s ? a.k[1] : a.k[0];
    stride = s ? a.x[1].stride : a.x[0].stride;
    return (s ? a.x[1].p : a.x[0].p) + from * stride;
  });
  dzs.begin(z, from, n0);
  tile_product_made<T, NB>(xs, dzs, rows, lds, acc);
  const auto row_at = gates_rows<T, 64>(n0, z.n);
  if (a.db) gates_sums(dzs, a, lds, part, row_at);
  dw_out<T, NB>(a, lds, acc, part, 0, row_at);
}

// dz and the sums for db alone, as k_gated_dw_made has them, for its sizes where
// it is not taken (dw is not asked for, or x lies where it cannot go to LDS
// directly): db then has the same bits whichever of the two makes it. Half a unit
// a thread, so that twice the waves share a CU: slopes take as long as memory.
// Whole lines of 256 bytes a block's row (of 128, 40 us more at the first size).
// us, this / k_gated_dz and its join: db alone, 110K x 1024 bf16 127 / 141; with
// dx, 110K x 256 -> 1024 404 / 383, 110K x 64 -> 512 172 / 172; 40K x 128 -> 64 all
// gradients 36 / 51; 27.5K x 128 -> 1024 fp32 404 / 402.
constexpr int kSumsCols = 128, kSumsNT = 1024;
template <typename T, int ACT>
__global__ __launch_bounds__(kSumsNT) void k_gated_sums(GatedDw<T> a, GatedDz<T> z, int groups, int64_t blocks) {
  constexpr int kStep = tile_step<T>();
  typedef TileGates<T, ACT, kSumsCols, 8 / sizeof(T)> B;
  static_assert(B::kNT == kSumsNT, "");
  __shared__ __align__(16) char lds[kStep * 2 * kSumsCols * sizeof(float)];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t part = tile / groups;
  const int n0 = (int)(tile % groups) * kSumsCols;
  const int64_t from = part * a.part, rows = min(a.part, a.rows - from);
  B dzs;
  dzs.begin(z, from, n0);
  const int64_t whole = rows / kStep, steps = whole + (rows % kStep ? 1 : 0);
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  auto ask = [&](int64_t s, auto set) {
    if (s < whole) dzs.template whole<set()>();
    else if (s < steps) dzs.template ragged<set()>(s * kStep, rows);
  };
  auto make = [&](auto set, auto all) {
    typename B::unit_t made[2];
    dzs.template make<set()>(made);
    dzs.template leave<set(), all()>(made);
  };
  ask(0, even);
  ask(1, odd);
  int64_t s = 0;
#pragma unroll 1
  for (; s + 3 < whole; s += 2) {
    make(even, std::true_type());
    dzs.template whole<even()>();
    make(odd, std::true_type());
    dzs.template whole<odd()>();
  }
#pragma unroll 1
  for (; s < steps; s += 2) {
    make(even, std::false_type());
    ask(s + 2, even);
    if (s + 1 < steps) make(odd, std::false_type());
    ask(s + 3, odd);
  }
  gates_sums(dzs, a, lds, part, gates_rows<T, kSumsCols>(n0, z.n));
}

// Adds parts of arrays of rows, four values a thread, WAYS threads a value, each
// over every WAYS-th part, then in order: for dw and db, or dx. (As many threads a
// value as keep the chip busy: 646 x 200 of 79 parts 11.8 us.)
template <typename T>
struct GatedJoin {
  const float* parts[2];
  T* to[2];
  int64_t values[2], stride[2], count;
  int cols[2], split;  // column split of the first's rows is another array's
  T* beyond;
  int64_t beyond_stride;
};
template <typename T, int WAYS>
__global__ __launch_bounds__(kGateNT) void k_gated_join(GatedJoin<T> a) {
  constexpr int kValues = kGateNT / WAYS * 4;
  __shared__ __align__(16) float sums[WAYS][kValues];
  const int64_t blocks = (a.values[0] + kValues - 1) / kValues;
  const bool other = blockIdx.x >= blocks;
  const float* parts = other ? a.parts[1] : a.parts[0];
  const int64_t values = other ? a.values[1] : a.values[0];
  const int way = threadIdx.x / (kGateNT / WAYS), at = threadIdx.x % (kGateNT / WAYS) * 4;
  const int64_t i = (int64_t)(blockIdx.x - (other ? blocks : 0)) * kValues + at;
  const int valid = (int)min(values - i, (int64_t)4);
  float sum[4] = {};
  if (valid > 0) {
#pragma unroll 4
    for (int64_t p = way; p < a.count; p += WAYS) {
      float v[4];
      load_cols<float, 4>(parts + p * values + i, valid, v);
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[q] += v[q];
    }
  }
  if constexpr (WAYS > 1) {
    *reinterpret_cast<f32x4*>(&sums[way][at]) = f32x4{sum[0], sum[1], sum[2], sum[3]};
    __syncthreads();
    if (way) return;
#pragma unroll
    for (int w = 1; w < WAYS; ++w)
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[q] += sums[w][at + q];
  }
  const int cols = other ? a.cols[1] : a.cols[0];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < valid) {
      const int64_t row = (i + q) / cols;
      const int col = (int)((i + q) % cols);
      if (other) a.to[1][row * a.stride[1] + col] = (T)sum[q];
      else if (col < a.split) a.to[0][row * a.stride[0] + col] = (T)sum[q];
      else a.beyond[row * a.beyond_stride + col - a.split] = (T)sum[q];
    }
}

}  // namespace ms
