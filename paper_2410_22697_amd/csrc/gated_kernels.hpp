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

// Calls f(act) with the activation as a type.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  if (act == kActSilu) f(std::integral_constant<int, kActSilu>());
  else if (act == kActGelu) f(std::integral_constant<int, kActGelu>());
  else if (act == kActRelu) f(std::integral_constant<int, kActRelu>());
  else f(std::integral_constant<int, kActNone>());
}

// Many rows: 128 rows by 32 NB outputs of both halves a block.
template <typename T, int NB>
__global__ __launch_bounds__(kTileNT, 2) void k_gated_tile(Gated<T> a, int tiles_n, int64_t blocks) {
  using P = TileProduct<T, NB, false>;
  constexpr int kOut = 16 * NB;  // outputs of a wave
  constexpr int kTurns = 4 * 32 * P::template turn_pitch<kOut>();
  __shared__ __align__(16) char lds[P::kLds > kTurns ? P::kLds : kTurns];
  __shared__ __align__(16) float bias[2][32 * NB];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t r0 = tile / tiles_n * kTileRows;
  const int n0 = (int)(tile % tiles_n) * (32 * NB);
  if ((int)threadIdx.x < 64 * NB) {
    const int h = threadIdx.x / (32 * NB), c = n0 + threadIdx.x % (32 * NB);
    bias[h][threadIdx.x % (32 * NB)] = a.bias && c < a.n ? (float)a.bias[h * a.n + c] : 0.0f;
  }
  f32x16 acc[NB][2] = {};
  // a wave's squares: NB / 2 of the gate, and those of the other half
  P::run(a.x, a.w, r0, a.rows, 0, 0,
         [&](int c) {
           const int square = c / 32 % NB, out = n0 + c / (32 * NB) * kOut + square % (NB / 2) * 32 + c % 32;
           return (square >= NB / 2 ? a.n : 0) + min(out, a.n - 1);
         },
         lds, acc);
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  char* turn = lds + wave * 32 * P::template turn_pitch<kOut>();
  const int c0 = wave % 2 * kOut;
  // f(gate, other half, results) for four outputs at a time, all of which then go to out
  auto each = [&](T* out, int64_t stride, int at, auto f) {
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
          P::template turn_in<kOut>(turn, 32 * i, q, v);
        }
      P::template turn_out<kOut>(turn, out + at, stride, r0 + wave / 2 * 64 + 32 * j, a.rows, n0 + c0, a.n);
    }
  };
  if (a.pre) {
    each(a.pre, a.pre_stride, 0, [](float g, float) { return g; });
    each(a.pre, a.pre_stride, a.n, [](float, float u) { return u; });
  }
  with_act(a.act, [&](auto act) { each(a.y, a.y_stride, 0, [&](float g, float u) { return act_value(g, act()) * u; }); });
}

// Few rows: 32 rows by 32 outputs of both halves a block, its eight waves share
// the reduction.
template <typename T>
__global__ __launch_bounds__(kFewNT) void k_gated_few(Gated<T> a, int tiles_n) {
  __shared__ float halves[2][32 * 32];
  const int64_t r0 = (int64_t)(blockIdx.x / tiles_n) * 32;
  const int n0 = (int)(blockIdx.x % tiles_n) * 32;
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

}  // namespace ms
