// norm_kernels.hpp - the root-mean-square norm of x + residual, and its gradients.
//
//   s = x + residual          r = 1 / sqrt(mean(s^2) + eps)      y = s r w
//   n = s r, g = dy w:        dx = r (g - n mean(g n)) + ds      dw = sum over the rows of dy n
//
// A row belongs to a team of lanes that holds it in registers (of long rows
// the first columns, the others are read again), so that it is read once, and
// y may leave as the codes of a packed row. Bound by memory: each value is read
// and written once. The gradient's blocks keep their sums for dw in registers over
// all their rows and leave a part each.
//
// Measured: 242K x 256 bf16 41 us (6.0 TB/s of x and y), with the residual and the
// sum 77 (6.4), the same to 8 bits 76 (5.7); gradients 71 (5.2), 93 with ds; 854K x
// 100 fp32 120 (5.7), bf16 75 (4.6).
// Packed rows that are read and written in less are bound by the vector unit, which
// their codes keep busy all the time (36 instructions a value: the normed values are
// made once for their ends and once for the codes): 242K x 256 to 4 bits 56, 854K x
// 100 to 8 bits 91 (units of 8 columns, of which such a row leaves a lane's half
// and three lanes of sixteen empty).
// A long row keeps a block waiting, of which a CU holds one or two, with nothing of
// the next row asked for: 30K x 5000 bf16 166 (3.6; waves wait for three quarters
// of their time, the vector unit is busy for a third of it), gradients 312 to 327
// (2.8). The gradients of columns beyond the registers (8192 in bf16) also read,
// add to and write their part of dw in memory for every row.
#pragma once

#include "common.hpp"
#include "rows_kernels.hpp"
#include "values.hpp"

namespace ms {

constexpr int kNormNT = 256;     // threads of a block of teams
constexpr int kNormLong = 512;   // threads of a block that has one row at a time (the gradients' longest rows: twice as many)

template <typename T>
struct Norm {
  const T *x, *residual, *weight;
  T *sum, *y;
  uint8_t* table;  // packed rows in y's place
  const int32_t* slots;
  int64_t rows, x_stride, residual_stride, sum_stride, y_stride, table_rows;
  PackedRows f;
  int32_t d;
  float inv_d, eps;
};

template <typename T>
struct NormGrads {
  const T *dy, *s, *weight, *ds;
  T* dx;
  float* parts;  // [blocks][d] of dw, or null
  int64_t rows, dy_stride, s_stride, ds_stride, dx_stride;
  int32_t d;
  float inv_d, eps;
};

// A reduction over a team: aligned lanes of a wave, or the whole block.
template <int TEAM, typename V, typename F>
__device__ __forceinline__ V norm_reduce(V x, F pick) {
  if constexpr (TEAM <= MS_WAVE) {
    return team_reduce(x, TEAM, pick);
  } else {
    __shared__ V of_wave[TEAM / MS_WAVE];
    x = team_reduce(x, MS_WAVE, pick);
    __syncthreads();
    if (lane_id() == 0) of_wave[wave_id()] = x;
    __syncthreads();
    x = of_wave[0];
#pragma unroll
    for (int w = 1; w < TEAM / MS_WAVE; ++w) x = pick(x, of_wave[w]);
    return x;
  }
}
template <int TEAM>
__device__ __forceinline__ float norm_sum(float x) {
  return norm_reduce<TEAM>(x, [](float a, float b) { return a + b; });
}
template <int TEAM>
__device__ __forceinline__ uint32_t norm_max(uint32_t x) {
  return norm_reduce<TEAM>(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// 1 / sqrt(mean + eps) is r 2^-e, and a row's values are taken times 2^-e before
// they are multiplied by r. e is 0, and of() not asked, unless the squares leave fp32's range.
struct NormScale {
  float r;
  int e;
  __device__ __forceinline__ float of(float s) const { return ldexpf(s, -e); }
};

// The scale of a row: each(f) gives f every column's value that this lane has,
// the same for all lanes of the team to take part in reductions after it.
template <int TEAM, typename E>
__device__ __forceinline__ NormScale norm_scale(E each, float inv_d, float eps) {
  float sum = 0.0f;
  each([&](float s) { sum += s * s; });
  const float t = norm_sum<TEAM>(sum) * inv_d + eps;
  if (t > 0x1p-96f && t < 0x1p96f) return {__builtin_amdgcn_rsqf(t), 0};
  // squares too large or too small for fp32, or not finite: again, by the largest magnitude's power of two
  uint32_t bits = 0;
  each([&](float s) { bits = max(bits, __float_as_uint(s) & 0x7FFFFFFFu); });
  const float largest = __uint_as_float(norm_max<TEAM>(bits));  // (a NaN's bits are above all others)
  if (!(largest < __builtin_inff())) return {largest == __builtin_inff() ? 0.0f : __builtin_nanf(""), 0};
  const float most = fmaxf(largest, sqrtf(eps));
  if (most == 0.0f) return {__builtin_inff(), 0};
  int e;
  frexpf(most, &e);
  sum = 0.0f;
  each([&](float s) {
    s = ldexpf(s, -e);
    sum += s * s;
  });
  return {__builtin_amdgcn_rsqf(norm_sum<TEAM>(sum) * inv_d + ldexpf(eps, -2 * e)), e};
}

template <typename T, int TEAM, int V, int Q, int BITS>
__global__ __launch_bounds__(TEAM > MS_WAVE ? TEAM : kNormNT) void k_rms_norm(Norm<T> a) {
  constexpr int kTeams = TEAM > MS_WAVE ? 1 : kNormNT / TEAM, kTurn = TEAM * Q;
  constexpr bool kLong = TEAM > MS_WAVE;  // columns may lie beyond the registers
  const int lane = threadIdx.x % TEAM, d = a.d;
  float w[V][Q];
#pragma unroll
  for (int t = 0; t < V; ++t) {
    const int c = t * kTurn + lane * Q;
#pragma unroll
    for (int q = 0; q < Q; ++q) w[t][q] = 1.0f;
    if (a.weight && c < d) load_cols<T, Q>(a.weight + c, d - c, w[t], 0.0f);
  }
  const int64_t step = (int64_t)gridDim.x * kTeams;
  int64_t i = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM;
  // (the rows' places go on by sums: a product for each would cost short rows much of their instructions)
  const T *x = a.x + i * a.x_stride, *res = a.residual ? a.residual + i * a.residual_stride : nullptr;
  T *sum = a.sum ? a.sum + i * a.sum_stride : nullptr, *out = BITS == 0 ? a.y + i * a.y_stride : nullptr;
  const int64_t x_on = step * a.x_stride, res_on = res ? step * a.residual_stride : 0, sum_on = sum ? step * a.sum_stride : 0, out_on = BITS == 0 ? step * a.y_stride : 0;
  for (; i < a.rows; i += step, x += x_on, res += res_on, sum += sum_on, out += out_on) {
    auto load = [&](int c, float (&s)[Q]) {
      load_row<T, Q>(x + c, d - c, s);
      if (res) {
        float r[Q];
        load_row<T, Q>(res + c, d - c, r);
#pragma unroll
        for (int q = 0; q < Q; ++q) s[q] += r[q];
      }
    };
    float s[V][Q];
#pragma unroll
    for (int t = 0; t < V; ++t) {
      const int c = t * kTurn + lane * Q;
#pragma unroll
      for (int q = 0; q < Q; ++q) s[t][q] = 0.0f;
      if (c < d) load(c, s[t]);
    }
    NormScale scale = {0.0f, 0};
    // f(first column, values, weights), zeros where columns are missing; all lanes take part. The values are the row's
    // until there is a scale, which may take a power of two out of them
    auto turns = [&](auto f) {
#pragma unroll
      for (int t = 0; t < V; ++t) f(t * kTurn + lane * Q, s[t], w[t]);
      if constexpr (kLong) {
        for (int c0 = V * kTurn; c0 < d; c0 += kTurn) {
          const int c = c0 + lane * Q;
          float u[Q] = {}, v[Q];
#pragma unroll
          for (int q = 0; q < Q; ++q) v[q] = 1.0f;
          if (c < d) {
            load(c, u);
            if (a.weight) load_cols<T, Q>(a.weight + c, d - c, v, 0.0f);
            if (scale.e) {
#pragma unroll
              for (int q = 0; q < Q; ++q) u[q] = scale.of(u[q]);
            }
          }
          f(c, u, v);
        }
      }
    };
    if (a.sum)
      turns([&](int c, const float (&v)[Q], const float (&)[Q]) {
        if (c < d) store_row<T, Q>(sum + c, d - c, v);
      });
    scale = norm_scale<TEAM>(
        [&](auto f) {
          turns([&](int, const float (&v)[Q], const float (&)[Q]) {
#pragma unroll
            for (int q = 0; q < Q; ++q) f(v[q]);
          });
        },
        a.inv_d, a.eps);
    if (scale.e) {
#pragma unroll
      for (int t = 0; t < V; ++t)
#pragma unroll
        for (int q = 0; q < Q; ++q) s[t][q] = scale.of(s[t][q]);
    }
    // (a product of its own also where a difference follows, so that codes are those of the value that would be stored)
    auto normed = [&](const float (&v)[Q], const float (&wv)[Q], float (&y)[Q]) {
#pragma clang fp contract(off)
#pragma unroll
      for (int q = 0; q < Q; ++q) y[q] = v[q] * scale.r * wv[q];
    };
    if constexpr (BITS == 0) {
      turns([&](int c, const float (&v)[Q], const float (&wv)[Q]) {
        float y[Q];
        normed(v, wv, y);
        if (c < d) store_row<T, Q>(out + c, d - c, y);
      });
    } else {
      const int64_t slot = a.slots ? (int64_t)a.slots[i] : i;
      if (slot < 0 || slot >= a.table_rows) continue;  // the same for the whole team
      uint8_t* row = a.table + slot * a.f.row_bytes;
      float* floats = reinterpret_cast<float*>(row + a.f.floats_at);
      float size, inv;
      if (a.f.group_log2 == 31) {
        GroupEnds<BITS> ends;
        turns([&](int c, const float (&v)[Q], const float (&wv)[Q]) {
          float y[Q];
          normed(v, wv, y);
          ends.add(y, d - c);
        });
        ends.mag = norm_max<TEAM>(ends.mag);
        if constexpr (BITS == 4) {
          ends.lo = norm_reduce<TEAM>(ends.lo, [](float p, float q) { return fminf(p, q); });
          ends.hi = norm_reduce<TEAM>(ends.hi, [](float p, float q) { return fmaxf(p, q); });
        }
        ends.scale(size, inv);
        turns([&](int c, const float (&v)[Q], const float (&wv)[Q]) {
          float y[Q];
          normed(v, wv, y);
          if (c < d) store_codes<BITS>(row, c, d, y, d - c, ends.lo, inv);
        });
        if (lane == 0) {
          if (BITS == 4) floats[0] = ends.lo;
          floats[BITS == 4 ? 1 : 0] = size;
        }
      } else {
        const int width = 1 << (a.f.group_log2 - 3);  // lanes that share a group: never more than a turn's of a wave
        turns([&](int c, const float (&v)[Q], const float (&wv)[Q]) {
          float y[Q];
          normed(v, wv, y);
          GroupEnds<BITS> ends;
          ends.add(y, d - c);
          ends.join(width);
          ends.scale(size, inv);
          if (c < d) {
            store_codes<BITS>(row, c, d, y, d - c, ends.lo, inv);
            if (lane % width == 0) {
              const int g = c >> a.f.group_log2;
              if (BITS == 4) floats[2 * g] = ends.lo;
              floats[BITS == 4 ? 2 * g + 1 : g] = size;
            }
          }
        });
      }
    }
  }
}

template <typename T, int TEAM, int V, int Q>
__global__ __launch_bounds__(TEAM > MS_WAVE ? TEAM : kNormNT) void k_rms_norm_backward(NormGrads<T> a) {
  constexpr int kTeams = TEAM > MS_WAVE ? 1 : kNormNT / TEAM, kTurn = TEAM * Q;
  constexpr bool kLong = TEAM > MS_WAVE;
  __shared__ float joined[kLong ? 1 : kNormNT * Q];
  const int lane = threadIdx.x % TEAM, d = a.d;
  float* part = a.parts ? a.parts + (int64_t)blockIdx.x * d : nullptr;
  float w[V][Q], dw[V][Q];
#pragma unroll
  for (int t = 0; t < V; ++t) {
    const int c = t * kTurn + lane * Q;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      w[t][q] = 1.0f;
      dw[t][q] = 0.0f;
    }
    if (a.weight && c < d) load_cols<T, Q>(a.weight + c, d - c, w[t], 0.0f);
  }
  if (kLong && part)  // the columns beyond the registers are summed where they end up, by the lane that owns them
    for (int c0 = V * kTurn; c0 < d; c0 += kTurn)
      for (int q = 0; q < Q; ++q)
        if (c0 + lane * Q + q < d) part[c0 + lane * Q + q] = 0.0f;
  const int64_t step = (int64_t)gridDim.x * kTeams;
  constexpr int kAhead = TEAM <= 16 ? 2 : 1;  // rows of a team that are on their way together
  int64_t i0 = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM;
  // (the rows' places go on by sums: a product for each would cost a short row a third of its instructions)
  const T *s_at = a.s + i0 * a.s_stride, *dy_at = a.dy + i0 * a.dy_stride, *ds_at = a.ds ? a.ds + i0 * a.ds_stride : nullptr;
  T* dx_at = a.dx ? a.dx + i0 * a.dx_stride : nullptr;
  const int64_t s_on = step * a.s_stride, dy_on = step * a.dy_stride, ds_on = a.ds ? step * a.ds_stride : 0, dx_on = a.dx ? step * a.dx_stride : 0;
  for (; i0 < a.rows; i0 += kAhead * step, s_at += kAhead * s_on, dy_at += kAhead * dy_on, ds_at += kAhead * ds_on, dx_at += kAhead * dx_on) {
    float s_of[kAhead][V][Q], dy_of[kAhead][V][Q], ds_of[kAhead][V][Q];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t i = i0 + u * step;
#pragma unroll
      for (int t = 0; t < V; ++t) {
        const int c = t * kTurn + lane * Q;
#pragma unroll
        for (int q = 0; q < Q; ++q) s_of[u][t][q] = dy_of[u][t][q] = ds_of[u][t][q] = 0.0f;
        if (i < a.rows && c < d) {
          load_row<T, Q>(s_at + u * s_on + c, d - c, s_of[u][t]);
          load_row<T, Q>(dy_at + u * dy_on + c, d - c, dy_of[u][t]);
          if (a.ds) load_row<T, Q>(ds_at + u * ds_on + c, d - c, ds_of[u][t]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t i = i0 + u * step;
      if (i >= a.rows) break;  // the same for the whole team
      float (&s)[V][Q] = s_of[u], (&dy)[V][Q] = dy_of[u], (&ds)[V][Q] = ds_of[u];
      const T *dyr = dy_at + u * dy_on, *sr = s_at + u * s_on, *dsr = a.ds ? ds_at + u * ds_on : nullptr;
      const NormScale scale = norm_scale<TEAM>(
          [&](auto f) {
#pragma unroll
            for (int t = 0; t < V; ++t)
#pragma unroll
              for (int q = 0; q < Q; ++q) f(s[t][q]);
            if constexpr (kLong)
              for (int c = V * kTurn + lane * Q; c < d; c += kTurn) {
                float u[Q];
                load_cols<T, Q>(sr + c, d - c, u);
#pragma unroll
                for (int q = 0; q < Q; ++q) f(u[q]);
              }
          },
          a.inv_d, a.eps);
      if (scale.e) {
#pragma unroll
        for (int t = 0; t < V; ++t)
#pragma unroll
          for (int q = 0; q < Q; ++q) s[t][q] = scale.of(s[t][q]);
      }
      float dot = 0.0f;
#pragma unroll
      for (int t = 0; t < V; ++t)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          s[t][q] *= scale.r;
          dw[t][q] += dy[t][q] * s[t][q];
          dy[t][q] *= w[t][q];
          dot += dy[t][q] * s[t][q];
        }
      // the columns beyond the registers: f(column, normed value, dy, weight)
      auto beyond = [&](auto f) {
        for (int c = V * kTurn + lane * Q; c < d; c += kTurn) {
          float u[Q], g[Q], v[Q];
          load_cols<T, Q>(sr + c, d - c, u);
          load_cols<T, Q>(dyr + c, d - c, g);
#pragma unroll
          for (int q = 0; q < Q; ++q) v[q] = 1.0f;
          if (a.weight) load_cols<T, Q>(a.weight + c, d - c, v);
#pragma unroll
          for (int q = 0; q < Q; ++q) u[q] = (scale.e ? scale.of(u[q]) : u[q]) * scale.r;
          f(c, u, g, v);
        }
      };
      if constexpr (kLong)
        beyond([&](int c, const float (&n)[Q], const float (&g)[Q], const float (&v)[Q]) {
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            dot += g[q] * v[q] * n[q];
            if (part && c + q < d) part[c + q] += g[q] * n[q];
          }
        });
      const float mean = norm_sum<TEAM>(dot) * a.inv_d;
      // the gradients of g's and n's columns, to which `add` is added
      auto back = [&](const float (&g)[Q], const float (&n)[Q], const float (&add)[Q], float (&v)[Q]) {
#pragma unroll
        for (int q = 0; q < Q; ++q) v[q] = scale.r * (g[q] - n[q] * mean);
        if (scale.e) {
#pragma unroll
          for (int q = 0; q < Q; ++q) v[q] = scale.of(v[q]);
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) v[q] += add[q];
      };
      T* dxr = dx_at + u * dx_on;
      if (a.dx) {
#pragma unroll
        for (int t = 0; t < V; ++t) {
          const int c = t * kTurn + lane * Q;
          float v[Q];
          back(dy[t], s[t], ds[t], v);
          if (c < d) store_row<T, Q>(dxr + c, d - c, v);
        }
        if constexpr (kLong)
          beyond([&](int c, const float (&n)[Q], const float (&g)[Q], const float (&v)[Q]) {
            float add[Q] = {}, u[Q], gv[Q];
            if (dsr) load_cols<T, Q>(dsr + c, d - c, add);
#pragma unroll
            for (int q = 0; q < Q; ++q) gv[q] = g[q] * v[q];
            back(gv, n, add, u);
            store_cols<T, Q>(dxr + c, d - c, u);
          });
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int t = 0; t < V; ++t) {
    const int c = t * kTurn + lane * Q;
    if constexpr (kLong) {
#pragma unroll
      for (int q = 0; q < Q; ++q)
        if (c + q < d) part[c + q] = dw[t][q];
    } else {
      // the block's teams add up in order
      __syncthreads();
#pragma unroll
      for (int q = 0; q < Q; ++q) joined[(threadIdx.x / TEAM) * kTurn + lane * Q + q] = dw[t][q];
      __syncthreads();
      for (int j = threadIdx.x; j < kTurn && t * kTurn + j < d; j += kNormNT) {
        float sum = 0.0f;
#pragma unroll 8
        for (int team = 0; team < kTeams; ++team) sum += joined[team * kTurn + j];
        part[t * kTurn + j] = sum;
      }
    }
  }
}

// Adds the blocks' parts of dw: sixteen threads a column, each over every
// sixteenth part, then in order.
constexpr int kNormJoinWays = 16;
template <typename T>
__global__ __launch_bounds__(kNormNT) void k_rms_norm_join(const float* __restrict__ parts, int64_t count, int32_t d, T* __restrict__ dw) {
  constexpr int kCols = kNormNT / kNormJoinWays;
  __shared__ float sums[kNormJoinWays][kCols];
  const int way = threadIdx.x / kCols, at = threadIdx.x % kCols;
  const int64_t c = (int64_t)blockIdx.x * kCols + at;
  float t = 0.0f;
  if (c < d) {
#pragma unroll 8
    for (int64_t p = way; p < count; p += kNormJoinWays) t += parts[p * d + c];
  }
  sums[way][at] = t;
  __syncthreads();
  if (way || c >= d) return;
#pragma unroll
  for (int w = 1; w < kNormJoinWays; ++w) t += sums[w][at];
  dw[c] = (T)t;
}

}  // namespace ms
