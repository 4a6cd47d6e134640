// block_kernels.hpp - the mean over a sampled block, and its gradient.
//
// Forward: a team of T lanes per row of the block; its list is read ahead
// kMeanAhead entries at a time, so that many source rows are in flight.
// Backward: dx[j] sums over the rows that list j. The edges are sorted by
// source first (stable radix sort), then each source row is summed from the
// sorted list in the order of the block's rows: no atomics on values, so a
// result does not depend on the order of the device's work.
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

// What block_mean reads its rows from: BITS 0 for rows of S, else packed rows.
template <typename S, int BITS, int Q>
struct SourceCols {
  PackedCols<BITS, Q> p;
  __device__ __forceinline__ void load(const void* x, int64_t rows, int64_t j, int64_t, const PackedRows& f, int c, int) {
    const uint8_t* row = packed_row((const uint8_t*)x, rows, j, f.row_bytes);
    if (row)
      p.load(row, f, c);
    else
      p.none();
  }
  __device__ __forceinline__ void values(float* v) const { p.values(v); }
};
template <typename S, int Q>
struct SourceCols<S, 0, Q> {
  cols_t<S, Q> r;
  __device__ __forceinline__ void load(const void* x, int64_t rows, int64_t j, int64_t stride, const PackedRows&, int c,
                                       int valid) {
    if (j < 0 || j >= rows) {
#pragma unroll
      for (int q = 0; q < Q; ++q) r[q] = (S)0.0f;
      return;
    }
    const S* p = (const S*)x + j * stride + c;
    if (valid >= Q) {
      r = *reinterpret_cast<const cols_t<S, Q>*>(p);
    } else {
#pragma unroll
      for (int q = 0; q < Q; ++q) r[q] = q < valid ? p[q] : (S)0.0f;
    }
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int q = 0; q < Q; ++q) v[q] = (float)r[q];
  }
};

constexpr int kMeanNT = 256;
constexpr int kMeanAhead = 8;

// Row i's entries, cut to the room in indices.
__device__ __forceinline__ void row_span(const int32_t* indptr, int64_t i, int64_t edges, int64_t& b, int64_t& e) {
  b = max((int64_t)indptr[i], (int64_t)0);
  e = min((int64_t)indptr[i + 1], edges);
}

template <typename S, int BITS, typename O, int Q, int T>
__global__ __launch_bounds__(kMeanNT) void k_block_mean(const int32_t* __restrict__ indptr,
                                                        const int32_t* __restrict__ indices, int64_t n, int64_t edges,
                                                        const void* __restrict__ x, int64_t rows, int64_t x_stride,
                                                        PackedRows f, O* __restrict__ out, int64_t out_stride) {
  const int lane = threadIdx.x % T;
  for (int64_t i = (int64_t)blockIdx.x * (kMeanNT / T) + threadIdx.x / T; i < n; i += (int64_t)gridDim.x * (kMeanNT / T)) {
    int64_t b, e;
    row_span(indptr, i, edges, b, e);
    const float share = e > b ? 1.0f / (float)(e - b) : 0.0f;
    for (int c = lane * Q; c < f.d; c += T * Q) {
      float sum[Q] = {};
      for (int64_t at = b; at < e; at += kMeanAhead) {
        SourceCols<S, BITS, Q> r[kMeanAhead];
        int32_t j[kMeanAhead];
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u) j[u] = at + u < e ? indices[at + u] : -1;
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u) r[u].load(x, rows, j[u], x_stride, f, c, f.d - c);
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u) {
          float v[Q];
          r[u].values(v);
#pragma unroll
          for (int q = 0; q < Q; ++q) sum[q] += v[q];
        }
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) sum[q] *= share;
      store_cols<O, Q>(out + i * out_stride + c, f.d - c, sum);
    }
  }
}

// ------------------------------------------------------------------ transpose
// The edges as (source, row) pairs in a stable order of their sources: an LSD
// radix sort over the bits that hold `rows`, at most kDigitBits a pass. Its
// unit is a wave with a chunk of consecutive edges and counters of its own in
// LDS, so ranks need no barrier: a wave counts its chunk's digits (k_edges for
// the first digit, k_digits), a block per 64 digits turns the counts of all
// chunks into first places (k_places), and the wave moves its pairs, 64 at a
// time, each group of equal digits ranked by ballots (k_move).
constexpr int kDigitBits = 11;
constexpr int kSortWaves = 4;     // waves per block of the counting and moving kernels
constexpr int kChunkLeast = 512;  // edges of a chunk at least
constexpr int kChunksMost = 1024; // chunks at most

// the last row that starts at or before edge e
__device__ __forceinline__ int64_t row_of_edge(const int32_t* indptr, int64_t lo, int64_t hi, int64_t e) {
  while (lo < hi) {
    const int64_t mid = (lo + hi + 1) >> 1;
    if ((int64_t)indptr[mid] <= e) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Pairs of the edges, the first digit's counts, and the spans cleared. An edge
// that belongs to no row or has no source gets the key `rows`, which is sorted
// behind the others and summed by nobody.
__global__ __launch_bounds__(kSortWaves* MS_WAVE) void k_edges(const int32_t* __restrict__ indptr,
                                                               const int32_t* __restrict__ indices, int64_t n, int64_t edges,
                                                               int64_t rows, int64_t chunk, int chunks, int bits,
                                                               uint32_t* __restrict__ keys, int32_t* __restrict__ vals,
                                                               int32_t* __restrict__ counts, int2* __restrict__ spans) {
  extern __shared__ int32_t lds[];
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int w = blockIdx.x * kSortWaves + wave;
  for (int64_t j = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; j < rows; j += (int64_t)gridDim.x * blockDim.x)
    spans[j] = make_int2(0, 0);
  const int digits = 1 << bits;
  int32_t* own = lds + wave * digits;
  for (int g = lane; g < digits; g += MS_WAVE) own[g] = 0;
  __syncthreads();
  if (w < chunks) {
    const int64_t b = w * chunk, e = min(edges, b + chunk);
    const int64_t first = row_of_edge(indptr, 0, n - 1, b);
    const int64_t last = row_of_edge(indptr, first, n - 1, e - 1);
    for (int64_t at = b + lane; at < e; at += MS_WAVE) {
      const int64_t i = row_of_edge(indptr, first, last, at);
      const int32_t j = indices[at];
      const bool real = at >= (int64_t)indptr[i] && at < (int64_t)indptr[i + 1] && j >= 0 && j < rows;
      const uint32_t key = real ? (uint32_t)j : (uint32_t)rows;
      keys[at] = key;
      vals[at] = (int32_t)i;
      atomicAdd(&own[key & (digits - 1)], 1);
    }
  }
  __syncthreads();
  if (w < chunks)
    for (int g = lane; g < digits; g += MS_WAVE) counts[(int64_t)w * digits + g] = own[g];
}

__global__ __launch_bounds__(kSortWaves* MS_WAVE) void k_digits(const uint32_t* __restrict__ keys, int64_t edges, int64_t chunk,
                                                                int chunks, int shift, int bits, int32_t* __restrict__ counts) {
  extern __shared__ int32_t lds[];
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int w = blockIdx.x * kSortWaves + wave;
  const int digits = 1 << bits;
  int32_t* own = lds + wave * digits;
  for (int g = lane; g < digits; g += MS_WAVE) own[g] = 0;
  __syncthreads();
  if (w < chunks) {
    const int64_t b = w * chunk, e = min(edges, b + chunk);
    for (int64_t at = b + lane; at < e; at += MS_WAVE) atomicAdd(&own[(keys[at] >> shift) & (digits - 1)], 1);
  }
  __syncthreads();
  if (w < chunks)
    for (int g = lane; g < digits; g += MS_WAVE) counts[(int64_t)w * digits + g] = own[g];
}

// counts[chunk][digit] to the number of equal digits in the chunks before, and
// totals[digit]. 64 digits per block, the chunks split over its 16 waves.
constexpr int kPlacesWaves = 16;
__global__ __launch_bounds__(kPlacesWaves* MS_WAVE) void k_places(int32_t* __restrict__ counts, int chunks, int bits,
                                                                  int32_t* __restrict__ totals) {
  __shared__ int32_t part[kPlacesWaves][MS_WAVE];
  const int lane = lane_id(), wave = wave_id();
  const int digits = 1 << bits;
  const int g = blockIdx.x * MS_WAVE + lane;
  const int per = (chunks + kPlacesWaves - 1) / kPlacesWaves;
  const int b = min(chunks, wave * per), e = min(chunks, b + per);
  int32_t sum = 0;
  if (g < digits) {
#pragma unroll 8
    for (int w = b; w < e; ++w) sum += counts[(int64_t)w * digits + g];
  }
  part[wave][lane] = sum;
  __syncthreads();
  int32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kPlacesWaves; ++w) {
    if (w < wave) before += part[w][lane];
    total += part[w][lane];
  }
  if (g >= digits) return;
  if (wave == 0) totals[g] = total;
  for (int w0 = b; w0 < e; w0 += 8) {
    int32_t v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = w0 + u < e ? counts[(int64_t)(w0 + u) * digits + g] : 0;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (w0 + u < e) {
        counts[(int64_t)(w0 + u) * digits + g] = before;
        before += v[u];
      }
  }
}

__global__ __launch_bounds__(kSortWaves* MS_WAVE) void k_move(const uint32_t* __restrict__ keys, const int32_t* __restrict__ vals,
                                                              int64_t edges, int64_t chunk, int chunks, int shift, int bits,
                                                              const int32_t* __restrict__ counts,
                                                              const int32_t* __restrict__ totals,
                                                              uint32_t* __restrict__ keys_out, int32_t* __restrict__ vals_out) {
  extern __shared__ int32_t lds[];
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int w = blockIdx.x * kSortWaves + wave;
  const int digits = 1 << bits;
  int32_t* first = lds;                       // first place of each digit
  int32_t* own = lds + (1 + wave) * digits;   // the next place of each digit in this wave's chunk
  if (wave == 0) {
    int32_t run = 0;
    for (int g0 = 0; g0 < digits; g0 += MS_WAVE) {
      const int32_t t = g0 + lane < digits ? totals[g0 + lane] : 0;
      const int32_t s = wave_inclusive_scan(t);
      if (g0 + lane < digits) first[g0 + lane] = run + s - t;
      run += __builtin_amdgcn_readlane(s, MS_WAVE - 1);
    }
  }
  __syncthreads();
  if (w >= chunks) return;
  for (int g = lane; g < digits; g += MS_WAVE) own[g] = first[g] + counts[(int64_t)w * digits + g];
  const int64_t b = w * chunk, e = min(edges, b + chunk);
  uint32_t key = b + lane < e ? keys[b + lane] : 0u;
  int32_t val = b + lane < e ? vals[b + lane] : 0;
  for (int64_t at = b; at < e; at += MS_WAVE) {
    const bool in = at + lane < e;
    const int64_t next = at + MS_WAVE + lane;
    const uint32_t next_key = next < e ? keys[next] : 0u;
    const int32_t next_val = next < e ? vals[next] : 0;
    const uint32_t g = (key >> shift) & (digits - 1);
    uint64_t same = ballot(in);
    for (int q = 0; q < bits; ++q) {
      const uint64_t m = ballot((g >> q) & 1u);
      same &= ((g >> q) & 1u) ? m : ~m;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int64_t place = 0;
    if (in) place = (int64_t)own[g] + lanes_below(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && lanes_below(same) == 0) own[g] += (int32_t)__popcll(same);
    if (in) {
      keys_out[place] = key;
      vals_out[place] = val;
    }
    key = next_key;
    val = next_val;
  }
}

// Where each source's entries lie in the sorted list.
__global__ __launch_bounds__(kMeanNT) void k_spans(const uint32_t* __restrict__ keys, int64_t edges, int64_t rows,
                                                   int2* __restrict__ spans) {
  for (int64_t p = (int64_t)blockIdx.x * kMeanNT + threadIdx.x; p < edges; p += (int64_t)gridDim.x * kMeanNT) {
    const uint32_t k = keys[p];
    if (k >= (uint64_t)rows) continue;
    if (p == 0 || keys[p - 1] != k) spans[k].x = (int32_t)p;
    if (p == edges - 1 || keys[p + 1] != k) spans[k].y = (int32_t)(p + 1);
  }
}

// dx: a team per source row.
template <typename D, int Q, int T>
__global__ __launch_bounds__(kMeanNT) void k_block_mean_backward(const int2* __restrict__ spans,
                                                                 const int32_t* __restrict__ vals,
                                                                 const int32_t* __restrict__ indptr, int64_t edges,
                                                                 int64_t rows, const D* __restrict__ dout,
                                                                 int64_t dout_stride, int d, const D* __restrict__ add,
                                                                 int64_t add_stride, int64_t add_rows, D* __restrict__ dx,
                                                                 int64_t dx_stride) {
  const int lane = threadIdx.x % T;
  for (int64_t j = (int64_t)blockIdx.x * (kMeanNT / T) + threadIdx.x / T; j < rows; j += (int64_t)gridDim.x * (kMeanNT / T)) {
    const int2 span = spans[j];
    for (int c = lane * Q; c < d; c += T * Q) {
      float sum[Q] = {};
      if (j < add_rows) load_cols<D, Q>(add + j * add_stride + c, d - c, sum);
      for (int at = span.x; at < span.y; at += kMeanAhead) {
        float v[kMeanAhead][Q], share[kMeanAhead];
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u) {
          share[u] = 0.0f;
          if (at + u < span.y) {
            const int64_t i = vals[at + u];
            int64_t b, e;
            row_span(indptr, i, edges, b, e);
            share[u] = 1.0f / (float)(e - b);
            load_cols<D, Q>(dout + i * dout_stride + c, d - c, v[u]);
          }
        }
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u)
          if (at + u < span.y) {
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] += v[u][q] * share[u];
          }
      }
      store_cols<D, Q>(dx + j * dx_stride + c, d - c, sum);
    }
  }
}

}  // namespace ms
