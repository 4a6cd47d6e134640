// linear_stream.hpp - the layer's products over many rows: y and dx.
//
// With thousands of rows and a few hundred columns these products are bound by
// the rows' way through memory (bf16) or by the matrix unit (fp32), so nothing
// else may stand in the rows' way. Each wave takes 32 rows at a time and reads
// them straight into the registers from which the matrix unit takes them: 16
// bytes a lane, the next 256 bytes of the row asked for as soon as a register
// is free, with no barrier and no LDS in between. The weights lie in LDS in
// the order in which the waves read them, all of them for the whole call where
// they fit (kStreamLds), else a chunk of 256 bytes of k at a time, in two
// buffers.
//
// Measured: y of 242K rows, 128 + 128 -> 256, in bf16 80 us (3.1 TB/s, 395
// TFLOP/s); dx of 110K x 1024 by 128 in bf16 with gelu's slope 151 us (3.2 TB/s),
// about half of it vector instructions of the slope; dx of 16K x 47 by 512 in fp32
// 28 us.
#pragma once

#include "linear_kernels.hpp"

namespace ms {

constexpr int kStreamNT = 512;              // 8 waves of 32 rows
constexpr int kStreamRows = 256;
constexpr int kStreamSteps = 8;             // 32 bytes of a row each: a chunk of 256 bytes
constexpr int kStreamTurn = 2048;           // LDS of a wave to turn 16 x 32 results
constexpr int kStreamLds = 128 << 10;       // LDS for weights
constexpr int kStreamBlockBytes = 32 * 256; // weights of 32 outputs and a chunk

// A segment of the reduction: rows of the streamed operand (with its slope's
// argument) and the weights that go with its columns.
template <typename T>
struct StreamSegment {
  Operand<T> x;  // R rows, K columns, along k
  Weights<T> w;
  int chunks;    // of K
};

// The units of 16 bytes of k by kV outputs in which a thread moves weights.
template <typename T, bool ACROSS, int NB>
struct StreamWeights {
  static constexpr int kV = 16 / sizeof(T);
  static constexpr int kUnits = NB * (32 / kV) * kStreamSteps * 2;  // of a chunk
  static constexpr int kPer = (kUnits + kStreamNT - 1) / kStreamNT;
  u32x4 v[kPer][kV];

  // unit: outputs kV * (unit % (NB * 32 / kV)) on, step and half above it
  __device__ __forceinline__ void load(const StreamSegment<T>& s, int chunk, int n0, int n) {
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const int unit = threadIdx.x + p * kStreamNT;
      const int r = n0 + (unit % (NB * 32 / kV)) * kV, at = unit / (NB * 32 / kV);
      const int64_t k = (int64_t)chunk * kStreamSteps * 2 * kV + at * kV;
      const int skip = s.x.K < kV ? (k ? kV : 0) : skipped<T>(k, s.x.K);
#pragma unroll
      for (int q = 0; q < kV; ++q) v[p][q] = (u32x4)0u;
      if (unit >= kUnits || skip == kV) continue;
      const int64_t from = skip ? s.x.K - kV : k;
      if constexpr (ACROSS) {
        // kV rows of k, kV outputs of each, turned by store()
#pragma unroll
        for (int q = 0; q < kV; ++q) {
          if (q < skip || from + q >= s.x.K) continue;
          const T* p0 = s.w.p + (from + q) * s.w.stride + r;
          if (r + kV <= n) {
            v[p][q] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(p0));
          } else {
            cols_t<T, kV> t;
#pragma unroll
            for (int i = 0; i < kV; ++i) t[i] = r + i < n ? p0[i] : (T)0.0f;
            v[p][q] = __builtin_bit_cast(u32x4, t);
          }
        }
      } else {
#pragma unroll
        for (int q = 0; q < kV; ++q)
          if (r + q < n && s.x.K < kV)
            v[p][q] = k_along(s.w.p + (int64_t)(r + q) * s.w.stride, k, s.x.K);
          else if (r + q < n)
            v[p][q] = without<T>(__builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(s.w.p + (int64_t)(r + q) * s.w.stride + from)), skip);
      }
    }
  }
  // to [block of 32 outputs][step][half][output % 32] of 16 bytes
  __device__ __forceinline__ void store(char* lds) {
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const int unit = threadIdx.x + p * kStreamNT;
      if (unit >= kUnits) continue;
      const int r = (unit % (NB * 32 / kV)) * kV, at = unit / (NB * 32 / kV);
      char* to = lds + (r / 32) * kStreamBlockBytes + at * 512 + (r % 32) * 16;
#pragma unroll
      for (int q = 0; q < kV; ++q) {
        if constexpr (ACROSS) {
          cols_t<T, kV> t;
#pragma unroll
          for (int i = 0; i < kV; ++i) t[i] = __builtin_bit_cast(cols_t<T, kV>, v[p][i])[q];
          *reinterpret_cast<u32x4*>(to + q * 16) = __builtin_bit_cast(u32x4, t);
        } else {
          *reinterpret_cast<u32x4*>(to + q * 16) = v[p][q];
        }
      }
    }
  }
};

// The products of this block's rows and the outputs [n0, n0 + 32 NB) of n:
// out(first row, first column, turn) gets 16 x 32 of them at a time, in LDS.
// segs: two segments, the second one's chunks may be none. lds: the weights'
// part, then the waves' turns.
template <typename T, bool SLOPE, bool ACROSS, int NB, bool RESIDENT, typename F>
__device__ __forceinline__ void stream_product(const StreamSegment<T> (&segs)[2], int64_t rows, int n0, int n, int64_t tile, int64_t tiles,
                                               int64_t tile_step, char* lds, int lds_weights, F out) {
  constexpr int kV = 16 / sizeof(T);
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int half = lane / 32;
  const int chunks = segs[0].chunks + segs[1].chunks;
  auto seg_of = [&](int c) -> const StreamSegment<T>& { return segs[c < segs[0].chunks ? 0 : 1]; };
  auto in_seg = [&](int c) { return c < segs[0].chunks ? c : c - segs[0].chunks; };
  u32x4 x[kStreamSteps], z[SLOPE ? kStreamSteps : 1];
  // one step of (tile, chunk) to its registers
  auto fetch = [&](int s, const StreamSegment<T>& g, int c, int64_t row) {
    const int64_t k = ((int64_t)c * kStreamSteps + s) * 2 * kV + half * kV;
    if (g.x.K < kV) {  // one step has it all
      x[s] = (u32x4)0u;
      if constexpr (SLOPE) z[s] = (u32x4)0u;
      if (s == 0) {
        x[s] = k_along(g.x.p + row * g.x.stride, k, g.x.K);
        if constexpr (SLOPE) z[s] = k_along(g.x.pre + row * g.x.pre_stride, k, g.x.K);
      }
      return;
    }
    const int64_t from = min(k, g.x.K - kV);  // masked when it is used
    x[s] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(g.x.p + row * g.x.stride + from));
    if constexpr (SLOPE)
      z[s] = __builtin_bit_cast(u32x4, *reinterpret_cast<const cols_t<T, kV>*>(g.x.pre + row * g.x.pre_stride + from));
  };
  auto row_of = [&](int64_t t) { return min(t * kStreamRows + wave * 32 + lane % 32, rows - 1); };
  // the first rows are on their way while the weights are laid out
  if (tile < tiles) {
#pragma unroll
    for (int s = 0; s < kStreamSteps; ++s) fetch(s, segs[0], 0, row_of(tile));
  }
  StreamWeights<T, ACROSS, NB> w;
  constexpr int kChunkBytes = NB * kStreamBlockBytes;
  if constexpr (RESIDENT) {
    for (int c = 0; c < chunks; ++c) {
      w.load(seg_of(c), in_seg(c), n0, n);
      w.store(lds + c * kChunkBytes);
    }
    __syncthreads();
  } else if (tile < tiles) {
    w.load(seg_of(0), 0, n0, n);
    w.store(lds);
    __syncthreads();
  }

  int buffer = 0;
  for (; tile < tiles; tile += tile_step) {
    f32x16 acc[NB] = {};
    for (int c = 0; c < chunks; ++c) {
      const StreamSegment<T>& g = seg_of(c);
      const int cs = in_seg(c);
      // what comes after this chunk: the next one, or the next tile's first
      const bool wrap = c + 1 == chunks;
      const int64_t next_tile = wrap ? (tile + tile_step < tiles ? tile + tile_step : tile) : tile;
      const int next_c = wrap ? 0 : c + 1;
      const StreamSegment<T>& next = seg_of(next_c);
      const int64_t next_row = row_of(next_tile);
      const char* wl = lds + (RESIDENT ? c : buffer) * kChunkBytes + lane * 16;
      const bool more = !RESIDENT && (!wrap || tile + tile_step < tiles);
      if (more) w.load(next, in_seg(next_c), n0, n);
      if (((int64_t)cs + 1) * kStreamSteps * 2 * kV > g.x.K && g.x.K >= kV) {  // the segment's end lies in this chunk
#pragma unroll
        for (int q = 0; q < kStreamSteps; ++q) {
          const int skip = skipped<T>(((int64_t)cs * kStreamSteps + q) * 2 * kV + half * kV, g.x.K);
          x[q] = without<T>(x[q], skip);
          if constexpr (SLOPE) z[q] = without<T>(z[q], skip);
        }
      }
      // the weights of a few blocks of outputs at a time, the reads of the next
      // under way meanwhile
      constexpr int kGroup = NB < 4 ? NB : 4, kGroups = kStreamSteps * NB / kGroup;
      u32x4 v[2][kGroup];
      auto weights = [&](int at) {
        const int s = at * kGroup / NB, b0 = at * kGroup % NB;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) v[at % 2][i] = *reinterpret_cast<const u32x4*>(wl + (b0 + i) * kStreamBlockBytes + s * 1024);
      };
      weights(0);
      // fp32 leaves out the steps behind a segment's end (100 + 100 -> 256: 158 to
      // 141 us); in bf16 they cost less than asking
      const int live = sizeof(T) == 2 ? kStreamSteps
                                      : (int)min((int64_t)kStreamSteps, (g.x.K - (int64_t)cs * kStreamSteps * 2 * kV + 2 * kV - 1) / (2 * kV));
      u32x4 a;
#pragma unroll
      for (int at = 0; at < kGroups; ++at) {
        const int s = at * kGroup / NB, b0 = at * kGroup % NB;
        const bool counts = sizeof(T) == 2 || s < live;
        if (b0 == 0) {
          a = x[s];
          if (SLOPE && counts) {
            cols_t<T, kV> d = __builtin_bit_cast(cols_t<T, kV>, a), p = __builtin_bit_cast(cols_t<T, kV>, z[SLOPE ? s : 0]);
            act_grads<T, kV>(d, p, g.x.act, [](int, float) {});
            a = __builtin_bit_cast(u32x4, d);
          }
          fetch(s, next, in_seg(next_c), next_row);
        }
        if (at + 1 < kGroups) weights(at + 1);
        __builtin_amdgcn_sched_barrier(0);  // loads stay ahead of the products that they run beside
        if (!counts) continue;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
          f32x16& c16 = acc[b0 + i];
          if constexpr (sizeof(T) == 2) {
            c16 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, v[at % 2][i]), c16, 0, 0, 0);
          } else {
            const f32x4 fa = __builtin_bit_cast(f32x4, a), fv = __builtin_bit_cast(f32x4, v[at % 2][i]);
#pragma unroll
            for (int q = 0; q < 4; ++q) c16 = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[q], fv[q], c16, 0, 0, 0);
          }
        }
      }
      if constexpr (!RESIDENT) {
        buffer ^= 1;
        if (more) w.store(lds + buffer * kChunkBytes);
        __syncthreads();
      }
    }
    // (accumulator register g of a lane is row 8 (g / 4) + 4 (lane / 32) + g % 4, column lane % 32)
    float* turn = reinterpret_cast<float*>(lds + lds_weights + wave * kStreamTurn);
    const int64_t r0 = tile * kStreamRows + wave * 32;  // may lie behind the last row
#pragma unroll 1
    for (int b = 0; b < NB; ++b) {
      // (registers have no index: each block of accumulators has its own way to LDS)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
          if (i == b) {
#pragma unroll
            for (int g = 0; g < 8; ++g) turn[(8 * (g / 4) + 4 * half + g % 4) * 32 + lane % 32] = acc[i][8 * u + g];
          }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        out(r0 + 16 * u, n0 + b * 32, turn);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
  }
}

// Gives a wave's 16 x 32 results in `turn`, of which the first `rows` rows and
// `cols` columns count, to f(row, column, values, 8 of them) or, where columns
// are missing, to f1(row, column, value).
template <typename F, typename F1>
__device__ __forceinline__ void stream_out(const float* turn, int rows, int cols, F f, F1 f1) {
  const int lane = lane_id();
  if (cols >= 32) {
    const int r = lane / 4, run = lane % 4 * 8;
    float y[8];
    const f32x4 lo = *reinterpret_cast<const f32x4*>(turn + r * 32 + run), hi = *reinterpret_cast<const f32x4*>(turn + r * 32 + run + 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      y[q] = lo[q];
      y[q + 4] = hi[q];
    }
    if (r < rows) f(r, run, y);
  } else {
#pragma unroll 1
    for (int r = lane / 32; r < rows; r += 2)
      if (lane % 32 < cols) f1(r, lane % 32, turn[r * 32 + lane % 32]);
  }
}

// Blocks of a tile's groups of outputs share an XCD, so that its L2 serves the
// rows to all but the first of them.
__device__ __forceinline__ void stream_place(int groups, int64_t& tile, int64_t& step, int& group) {
  constexpr int kXcds = 8;
  const int64_t local = blockIdx.x / kXcds;
  group = (int)(local % groups);
  tile = local / groups * kXcds + blockIdx.x % kXcds;
  step = gridDim.x / groups;
}

template <typename T, int NB, bool RESIDENT>
__global__ __launch_bounds__(kStreamNT) void k_linear_stream(LinearForward<T> a, int groups, int lds_weights) {
  extern __shared__ __align__(16) char stream_lds[];
  int64_t tile, step;
  int group;
  stream_place(groups, tile, step, group);
  const StreamSegment<T> segs[2] = {{a.x[0], a.w[0], (int)((a.x[0].K * sizeof(T) + 255) / 256)},
                                    {a.x[1], a.w[1], (int)((a.x[1].K * sizeof(T) + 255) / 256)}};
  // the group's bias as fp32, beside the turns: read with LDS's own waits, not behind the rows on their way
  float* bias = reinterpret_cast<float*>(stream_lds + lds_weights + kStreamNT / MS_WAVE * kStreamTurn);
  const int n0 = group * NB * 32;
  if ((int)threadIdx.x < NB * 32) bias[threadIdx.x] = a.bias && n0 + (int)threadIdx.x < a.n ? (float)a.bias[n0 + threadIdx.x] : 0.0f;
  stream_product<T, false, false, NB, RESIDENT>(
      segs, a.rows, n0, a.n, tile, (a.rows + kStreamRows - 1) / kStreamRows, step, stream_lds, lds_weights,
      [&](int64_t r0, int c0, const float* turn) {
        stream_out(
            turn, (int)min(a.rows - r0, (int64_t)16), a.n - c0,
            [&](int r, int c, float (&z)[8]) {
              const int64_t row = r0 + r;
              const f32x4 lo = *reinterpret_cast<const f32x4*>(bias + c0 - n0 + c), hi = *reinterpret_cast<const f32x4*>(bias + c0 - n0 + c + 4);
#pragma unroll
              for (int q = 0; q < 8; ++q) z[q] += q < 4 ? lo[q % 4] : hi[q % 4];
              // (64 bytes of a row at a time: the cache puts its lines together)
              if (a.pre) store_cols<T, 8, false>(a.pre + row * a.pre_stride + c0 + c, 8, z);
              act_values(z, a.act);
              if (a.residual) {
                float t[8];
                load_cols<T, 8>(a.residual + row * a.residual_stride + c0 + c, 8, t);
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] += t[q];
              }
              store_cols<T, 8, false>(a.y + row * a.y_stride + c0 + c, 8, z);
            },
            [&](int r, int c, float z) {
              linear_finish(a, r0 + r, c0 + c, z + bias[c0 - n0 + c]);
            });
      });
}

template <typename T, bool SLOPE, int NB, bool RESIDENT>
__global__ __launch_bounds__(kStreamNT) void k_linear_dx_stream(LinearDx<T> a, int groups, int lds_weights) {
  extern __shared__ __align__(16) char stream_lds[];
  int64_t tile, step;
  int group;
  stream_place(groups, tile, step, group);
  const StreamSegment<T> segs[2] = {{a.dz, a.w, (int)((a.dz.K * sizeof(T) + 255) / 256)}, {a.dz, a.w, 0}};
  stream_product<T, SLOPE, true, NB, RESIDENT>(
      segs, a.rows, group * NB * 32, a.cols, tile, (a.rows + kStreamRows - 1) / kStreamRows, step, stream_lds, lds_weights,
      [&](int64_t r0, int c0, const float* turn) {
        stream_out(
            turn, (int)min(a.rows - r0, (int64_t)16), a.cols - c0,
            [&](int r, int c, const float (&v)[8]) { linear_dx_store(a, r0 + r, c0 + c, v); },
            [&](int r, int c, float v) { linear_dx_store(a, r0 + r, c0 + c, v); });
      });
}

}  // namespace ms
