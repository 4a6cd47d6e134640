// gated_kernels.hpp - a gated layer and what its gradients need.
//
//   g = [x | x2] Wg^T + bg      u = [x | x2] Wu^T + bu      y = act(g) u
//   dg = dy u act'(g)           du = dy act(g)
//   dx = [dg | du] [Wg; Wu]     dW = [dg | du]^T [x | x2]   db = sums over the rows
//
// Both products of an output are made by the same lane, so that the activation
// and the product need no other pass over memory.
#pragma once

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
// the reduction.
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
constexpr int kGateNT = 256;
constexpr int kGateUnits = 32;  // units of 16 bytes of a row that a block takes
constexpr int kGateWays = kGateNT / kGateUnits;

template <typename T>
struct GatedDz {
  const T *dy, *pre;
  T* dz;         // [rows][2 n]
  float* parts;  // [parts][2 n] of db, or null
  int64_t rows, part, dy_stride, pre_stride, dz_stride;
  int n, act, groups;
};

// dz = [dg | du], and the sums of each part of the rows, of dz before it is
// rounded.
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
        load_cols<T, kV>(a.dy + i * a.dy_stride + c, valid, dy[v]);
        load_cols<T, kV>(a.pre + i * a.pre_stride + c, valid, g[v]);
        load_cols<T, kV>(a.pre + i * a.pre_stride + a.n + c, valid, u[v]);
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
        store_cols<T, kV, false>(a.dz + i * a.dz_stride + c, valid, dg);
        store_cols<T, kV, false>(a.dz + i * a.dz_stride + a.n + c, valid, du);
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

// dx = dz w over many rows: 128 rows by 64 NB columns a block.
template <typename T, int NB, bool DIRECT>
__global__ __launch_bounds__(kTileNT, 2) void k_gated_dx(LinearDx<T> a, int tiles_n, int64_t blocks) {
  typedef TileAcross<T, 64 * NB> A;
  typedef TileAlong<T, kTileSecond> B;
  typedef TileTurn<T, 32 * NB> Turn;
  constexpr int kLds = tile_lds<A, B>(DIRECT) > 4 * Turn::kBytes ? tile_lds<A, B>(DIRECT) : 4 * Turn::kBytes;
  __shared__ __align__(16) char lds[kLds];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t r0 = tile / tiles_n * kTileSecond;
  const int n0 = (int)(tile % tiles_n) * (64 * NB);
  A weights;
  B rows;
  f32x16 acc[NB][2] = {};
  const TileSegment segments[1] = {{a.dz.K, a.cols >= 16 / (int)sizeof(T)}};
  auto begin = [&](int) {
        weights.begin([&](int c, int& at, int& columns, int64_t& stride) {
          at = n0 + c;
          columns = a.cols;
          stride = a.w.stride;
          return a.w.p;
        });
        rows.begin([&](int r) { return a.dz.p + min(r0 + r, a.rows - 1) * a.dz.stride; });
  };
  if constexpr (DIRECT) tile_product_direct<T, NB>(weights, rows, segments, begin, lds, acc);
  else tile_product<T, NB>(weights, rows, segments, begin, lds, acc);
  const int wave = wave_uniform((int32_t)wave_id());
  const Turn turn = {lds + wave * Turn::kBytes};
  const int c0 = n0 + wave % 2 * (32 * NB);
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

// dw = dz^T [x | x2], one part of the rows a block: 128 outputs by 64 NB columns.
// Columns are placed in whole units, the second input's from `second` on.
template <typename T, int NB, bool DIRECT>
__global__ __launch_bounds__(kTileNT, 2) void k_gated_dw(LinearDw<T> a, int64_t blocks) {
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
  const int wave = wave_uniform((int32_t)wave_id());
  const Turn turn = {lds + wave * Turn::kBytes};
  const int all = a.k[0] + a.k[1], c0 = k0 + wave % 2 * (32 * NB);
  float* dw = a.dw + part * a.n * (int64_t)all;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        turn.in(32 * i, q, v);
      }
    const int out = n0 + wave / 2 * 64 + 32 * j;
    turn.units([&](int r, int c, cols_t<float, 4> v) {
      const int at = c0 + c, s = at >= a.second ? 1 : 0, c1 = at - (s ? a.second : 0), columns = s ? a.k[1] : a.k[0];
      if (out + r >= round_up_to<kV>(a.n) || c1 >= round_up_to<kV>(columns)) return;
      const int row = tile_column<T>(out + r, a.n), col = tile_column<T>(c1, columns);
      if (row >= a.n) return;
      float* p = dw + (int64_t)row * all + (s ? a.k[0] : 0) + col;
      if (col + 4 <= columns) {
        *reinterpret_cast<cols_t<float, 4>*>(p) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col + e < columns) p[e] = v[e];
      }
    });
  }
}

// Adds the parts of dw, four values a thread.
template <typename T>
__global__ __launch_bounds__(kGateNT) void k_gated_join(const float* __restrict__ parts, int64_t count, int64_t values, int cols, T* __restrict__ dw, int64_t stride) {
  const int64_t i = ((int64_t)blockIdx.x * kGateNT + threadIdx.x) * 4;
  if (i >= values) return;
  const int valid = (int)min(values - i, (int64_t)4);
  float sum[4] = {};
#pragma unroll 8
  for (int64_t p = 0; p < count; ++p) {
    float v[4];
    load_cols<float, 4>(parts + p * values + i, valid, v);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] += v[q];
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < valid) dw[(i + q) / cols * stride + (i + q) % cols] = (T)sum[q];
}

}  // namespace ms
