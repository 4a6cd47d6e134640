// block_kernels.hpp - the mean over a sampled block, and its gradient.
//
// Forward: a team of T lanes per row of the block; its list is read ahead
// kMeanAhead entries at a time, so that many source rows are in flight. Bound by
// the sources' lines: 110K rows of up to 5 of 242K 8-bit rows of 128 24 us, 3.7
// TB/s of the sources and results counted once.
// Backward: dx[j] sums over the rows that list j. The edges are sorted by
// source first (stable radix sort), then each source's entries are summed from
// the sorted list in the order of the block's rows: no atomics on values, so a
// result does not depend on the order of the device's work. 242K sources of 256
// floats from 110K rows and 399K entries: the sort 59 us in six launches, the
// sums 109 (3.3 TB/s of dout and dx counted once; dout's rows are read 3.6 times
// each, most of them from the caches), the joins 7.
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

// The columns that a lane takes at c: its own Q, or, at the end of a row of at
// least Q, the last Q (the lane before computes some of them too, and both
// store the same bits). A row of fewer is taken one column a lane (Q = 1).
template <int Q>
__device__ __forceinline__ int last_cols(int c, int d) {
  return min(c, d - Q);
}

// What block_mean reads its rows from: BITS 0 for rows of S, else packed rows.
// A source is loaded into registers under its own condition; one that is not
// there stays zero.
template <typename S, int BITS, int Q>
struct Source {
  PackedCols<BITS, Q> p;
  __device__ __forceinline__ void load(const void* x, int64_t j, int64_t, const PackedRows& f, int c) {
    p.load((const uint8_t*)x + j * f.row_bytes, f, c);
  }
  __device__ __forceinline__ float value(int q) const { return p.value(q); }
};
template <typename S, int Q>
struct Source<S, 0, Q> {
  cols_t<S, Q> w = (cols_t<S, Q>)(S)0.0f;
  __device__ __forceinline__ void load(const void* x, int64_t j, int64_t stride, const PackedRows&, int c) {
    w = *reinterpret_cast<const cols_t<S, Q>*>((const S*)x + j * stride + c);
  }
  __device__ __forceinline__ float value(int q) const { return (float)w[q]; }
};

constexpr int kMeanNT = 256;
constexpr int kMeanAhead = 8;

// Row i's entries, cut to the room in indices.
__device__ __forceinline__ void row_span(const int32_t* indptr, int64_t i, int32_t edges, int32_t& b, int32_t& e) {
  b = max(indptr[i], 0);
  e = min(indptr[i + 1], edges);
}
__device__ __forceinline__ float share_of(int32_t b, int32_t e) { return e > b ? 1.0f / (float)(e - b) : 0.0f; }

template <typename S, int BITS, typename O, int Q, int T>
__global__ __launch_bounds__(kMeanNT) void k_block_mean(const int32_t* __restrict__ indptr,
                                                        const int32_t* __restrict__ indices, int64_t n, int32_t edges,
                                                        const void* __restrict__ x, int32_t rows, int64_t x_stride,
                                                        PackedRows f, O* __restrict__ out, int64_t out_stride) {
  const int lane = threadIdx.x % T;
  for (int64_t i = (int64_t)blockIdx.x * (kMeanNT / T) + threadIdx.x / T; i < n; i += (int64_t)gridDim.x * (kMeanNT / T)) {
    int32_t b, e;
    row_span(indptr, i, edges, b, e);
    const float share = share_of(b, e);
    for (int c0 = lane * Q; c0 < f.d; c0 += T * Q) {
      const int c = BITS ? c0 : last_cols<Q>(c0, f.d);
      float sum[Q] = {};
      for (int32_t at = b; at < e; at += kMeanAhead) {
        Source<S, BITS, Q> r[kMeanAhead];
        int32_t j[kMeanAhead];
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u) j[u] = at + u < e ? indices[at + u] : -1;
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u)
          if (j[u] >= 0 && j[u] < rows) r[u].load(x, j[u], x_stride, f, c);
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u)
#pragma unroll
          for (int q = 0; q < Q; ++q) sum[q] += r[u].value(q);
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
// the first digit, k_digits), k_places turns the counts of all chunks into
// first places, and the wave moves its pairs, 64 at a time, each group of equal
// digits ranked by ballots (k_move; the last pass also writes each entry's
// share and marks the sources that are listed at all).
constexpr int kDigitBits = 11;
constexpr int kSortWaves = 4;     // waves per block of the counting and moving kernels
constexpr int kChunksMost = 1024; // chunks at most; a chunk is a multiple of 64 edges
constexpr int kEdgeTile = 256;    // edges whose rows k_edges finds at a time

// The last row that starts at or before edge e, or 0: the wave narrows the
// range 64-fold a step.
__device__ __forceinline__ int32_t row_of_edge(const int32_t* indptr, int32_t n, int32_t e) {
  int64_t lo = 0, hi = n;  // the answer is in [lo, hi)
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + MS_WAVE - 1) / MS_WAVE;
    const int64_t at = lo + lane_id() * step;
    const uint64_t below = ballot(at < hi && indptr[min(at, hi - 1)] <= e);
    const int last = below ? 63 - __builtin_clzll(below) : 0;
    lo += last * step;
    hi = min(hi, lo + step);
  }
  return (int32_t)lo;
}

// Pairs of the edges, the first digit's counts, and the marks cleared. An edge
// that belongs to no row or has no source gets the key `rows`, which is sorted
// behind the others and summed by nobody.
__global__ __launch_bounds__(kSortWaves* MS_WAVE) void k_edges(const int32_t* __restrict__ indptr,
                                                               const int32_t* __restrict__ indices, int32_t n, int32_t edges,
                                                               int32_t rows, int32_t chunk, int chunks, int bits,
                                                               uint32_t* __restrict__ keys, int32_t* __restrict__ vals,
                                                               int32_t* __restrict__ counts, uint32_t* __restrict__ marks) {
  extern __shared__ int32_t lds[];
  __shared__ int32_t starts[kSortWaves][kEdgeTile];
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int w = blockIdx.x * kSortWaves + wave;
  for (int64_t j = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; j < ((int64_t)rows + 3) / 4; j += (int64_t)gridDim.x * blockDim.x)
    marks[j] = 0;
  const int digits = 1 << bits;
  int32_t* own = lds + wave * digits;
  for (int g = lane; g < digits; g += MS_WAVE) own[g] = 0;
  if (w >= chunks) return;
  const int32_t b = w * chunk, e = min(edges, b + chunk);
  const int32_t first_edge = indptr[0], last_edge = indptr[n];
  int32_t row = row_of_edge(indptr, n, b);
  for (int32_t t0 = b; t0 < e; t0 += kEdgeTile) {
    const int32_t t1 = min(e, t0 + kEdgeTile);
    // the rows that start in this tile mark their first edge; of several the last one, the others are empty
    for (int q = lane; q < kEdgeTile; q += MS_WAVE) starts[wave][q] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int32_t i = row + 1;
    for (bool more = true; more;) {
      const int32_t at = (int64_t)i + lane < n ? indptr[i + lane] : t1;
      const uint64_t here = ballot(at < t1);
      if (at < t1) atomicMax(&starts[wave][at > t0 ? at - t0 : 0], i + lane);
      i += __popcll(here);
      more = here == ~0ull;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int q = 0; q < kEdgeTile / MS_WAVE; ++q) {
      const int32_t at = t0 + q * MS_WAVE + lane;
      // the running maximum of the starts is each edge's row
      int32_t r = max(starts[wave][q * MS_WAVE + lane], row);
      for (int o = 1; o < MS_WAVE; o <<= 1) {
        const int32_t y = __shfl_up(r, o, MS_WAVE);
        if (lane >= o) r = max(r, y);
      }
      row = __builtin_amdgcn_readlane(r, MS_WAVE - 1);
      if (at < t1) {
        const int32_t j = indices[at];
        const bool real = at >= first_edge && at < last_edge && j >= 0 && j < rows;
        const uint32_t key = real ? (uint32_t)j : (uint32_t)rows;
        keys[at] = key;
        vals[at] = r;
        atomicAdd(&own[key & (digits - 1)], 1);
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int g = lane; g < digits; g += MS_WAVE) counts[(int64_t)w * digits + g] = own[g];
}

__global__ __launch_bounds__(kSortWaves* MS_WAVE) void k_digits(const uint32_t* __restrict__ keys, int32_t edges, int32_t chunk,
                                                                int chunks, int shift, int bits, int32_t* __restrict__ counts) {
  extern __shared__ int32_t lds[];
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int w = blockIdx.x * kSortWaves + wave;
  const int digits = 1 << bits;
  if (w >= chunks) return;
  int32_t* own = lds + wave * digits;
  for (int g = lane; g < digits; g += MS_WAVE) own[g] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const int32_t b = w * chunk, e = min(edges, b + chunk);
#pragma unroll 4
  for (int32_t at = b + lane; at < e; at += MS_WAVE) atomicAdd(&own[(keys[at] >> shift) & (digits - 1)], 1);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int g = lane; g < digits; g += MS_WAVE) counts[(int64_t)w * digits + g] = own[g];
}

// counts[chunk][digit] to the number of equal digits in the chunks before, and
// totals[digit]. A block takes 16 digits (64 bytes of a chunk's counts), its 64
// groups of 16 threads take the chunks in 64 runs, whose counts they keep in
// registers until the places of the runs are known.
constexpr int kPlacesDigits = 16, kPlacesRuns = 64, kPlacesRun = kChunksMost / kPlacesRuns;
__global__ __launch_bounds__(kPlacesDigits* kPlacesRuns) void k_places(int32_t* __restrict__ counts, int chunks, int bits,
                                                                       int32_t* __restrict__ totals) {
  __shared__ int32_t part[kPlacesRuns][kPlacesDigits];
  const int g0 = threadIdx.x % kPlacesDigits, run = threadIdx.x / kPlacesDigits;
  const int digits = 1 << bits;
  const int g = blockIdx.x * kPlacesDigits + g0;
  const int per = (chunks + kPlacesRuns - 1) / kPlacesRuns;  // at most kPlacesRun
  const int b = run * per;
  int32_t v[kPlacesRun], sum = 0;
#pragma unroll
  for (int u = 0; u < kPlacesRun; ++u) v[u] = u < per && b + u < chunks && g < digits ? counts[(int64_t)(b + u) * digits + g] : 0;
#pragma unroll
  for (int u = 0; u < kPlacesRun; ++u) sum += v[u];
  part[run][g0] = sum;
  __syncthreads();
  if (run == 0) {
    int32_t before = 0;
#pragma unroll 16
    for (int w = 0; w < kPlacesRuns; ++w) {
      const int32_t t = part[w][g0];
      part[w][g0] = before;
      before += t;
    }
    if (g < digits) totals[g] = before;
  }
  __syncthreads();
  int32_t before = part[run][g0];
#pragma unroll
  for (int u = 0; u < kPlacesRun; ++u) {
    if (u < per && b + u < chunks && g < digits) counts[(int64_t)(b + u) * digits + g] = before;
    before += v[u];
  }
}

template <bool LAST>
__global__ __launch_bounds__(kSortWaves* MS_WAVE) void k_move(const uint32_t* __restrict__ keys, const int32_t* __restrict__ vals,
                                                              int32_t edges, int32_t chunk, int chunks, int shift, int bits,
                                                              const int32_t* __restrict__ counts,
                                                              const int32_t* __restrict__ totals,
                                                              uint32_t* __restrict__ keys_out, int32_t* __restrict__ vals_out,
                                                              const int32_t* __restrict__ indptr, int32_t rows,
                                                              float* __restrict__ shares, uint8_t* __restrict__ marks) {
  extern __shared__ int32_t lds[];
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  const int w = blockIdx.x * kSortWaves + wave;
  const int digits = 1 << bits;
  int32_t* first = lds;                       // first place of each digit
  int32_t* own = lds + (1 + wave) * digits;   // the next place of each digit in this wave's chunk
  // the digits' totals to first places: each thread scans a few neighbours
  __shared__ int32_t scan[kSortWaves + 1];
  const int per = (digits + kSortWaves * MS_WAVE - 1) / (kSortWaves * MS_WAVE);  // at most 8
  int32_t t[(1 << kDigitBits) / (kSortWaves * MS_WAVE)], sum = 0, total;
#pragma unroll
  for (int u = 0; u < (int)(sizeof t / sizeof t[0]); ++u) {
    const int g = threadIdx.x * per + u;
    t[u] = u < per && g < digits ? totals[g] : 0;
    sum += t[u];
  }
  if (w < chunks)
#pragma unroll 4
    for (int g = lane; g < digits; g += MS_WAVE) own[g] = counts[(int64_t)w * digits + g];
  int32_t run = block_exclusive_scan<kSortWaves * MS_WAVE>(sum, scan, &total);
#pragma unroll
  for (int u = 0; u < (int)(sizeof t / sizeof t[0]); ++u) {
    const int g = threadIdx.x * per + u;
    if (u < per && g < digits) first[g] = run;
    run += t[u];
  }
  __syncthreads();
  if (w >= chunks) return;
#pragma unroll 4
  for (int g = lane; g < digits; g += MS_WAVE) own[g] += first[g];
  const int32_t b = w * chunk, e = min(edges, b + chunk);
  uint32_t key = b + lane < e ? keys[b + lane] : 0u;
  int32_t val = b + lane < e ? vals[b + lane] : 0;
  for (int32_t at = b; at < e; at += MS_WAVE) {
    const bool in = at + lane < e;
    const int32_t next = at + MS_WAVE + lane;
    const uint32_t next_key = next < e ? keys[next] : 0u;
    const int32_t next_val = next < e ? vals[next] : 0;
    const uint32_t g = (key >> shift) & (digits - 1);
    uint64_t same = ballot(in);
    for (int q = 0; q < bits; ++q) {
      const uint64_t m = ballot((g >> q) & 1u);
      same &= ((g >> q) & 1u) ? m : ~m;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int32_t place = 0;
    if (in) place = own[g] + lanes_below(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && lanes_below(same) == 0) own[g] += (int32_t)__popcll(same);
    if (in) {
      keys_out[place] = key;
      vals_out[place] = val;
      if (LAST && key < (uint32_t)rows) {
        int32_t rb, re;
        row_span(indptr, val, edges, rb, re);
        shares[place] = share_of(rb, re);
        marks[key] = 1;  // by every entry of the source alike
      }
    }
    key = next_key;
    val = next_val;
  }
}

// ------------------------------------------------------------------ gradient
// dx from the sorted entries, evenly split whatever the sources' counts: a team
// of T lanes takes `span` consecutive entries and sums the run of each source. A
// run that lies in the span is a row of dx; a run that goes on beyond an end of
// it is a partial sum (the run that begins here in place 1 of the span, one
// that came in from the left in place 0), which k_block_mean_join adds up. The
// blocks after the spans' write the rows that no entry lists.
//
// (Four waves a SIMD, 128 registers: with 136, which it would take, three, and
// 11 us more for 110K rows of 256 floats and 399K entries.)
template <typename D, int Q, int T, bool ADD>
__global__ __launch_bounds__(kMeanNT, ADD ? 3 : 4) void k_block_mean_backward(const uint32_t* __restrict__ keys,
                                                                 const int32_t* __restrict__ vals,
                                                                 const float* __restrict__ shares,
                                                                 const uint8_t* __restrict__ marks, int32_t edges, int32_t rows,
                                                                 const D* __restrict__ dout, int64_t dout_stride, int d,
                                                                 const D* __restrict__ add, int64_t add_stride, int32_t add_rows,
                                                                 D* __restrict__ dx, int64_t dx_stride,
                                                                 float* __restrict__ partial, int span, int span_blocks) {
  constexpr int kTeams = kMeanNT / T;
  const int lane = threadIdx.x % T;
  if ((int)blockIdx.x >= span_blocks) {
    const int64_t step = (int64_t)(gridDim.x - span_blocks) * kTeams;
    for (int64_t j = (int64_t)(blockIdx.x - span_blocks) * kTeams + threadIdx.x / T; j < rows; j += step) {
      if (marks[j]) continue;
      for (int c0 = lane * Q; c0 < d; c0 += T * Q) {
        const int c = last_cols<Q>(c0, d);
        float v[Q] = {};
        if (ADD && j < add_rows) load_cols<D, Q>(add + j * add_stride + c, Q, v);
        store_cols<D, Q>(dx + j * dx_stride + c, Q, v);
      }
    }
    return;
  }
  const int64_t spans = ((int64_t)edges + span - 1) / span;
  for (int64_t s = (int64_t)blockIdx.x * kTeams + threadIdx.x / T; s < spans; s += (int64_t)span_blocks * kTeams) {
    const int32_t b = (int32_t)(s * span), e = (int32_t)min((int64_t)edges, (int64_t)b + span);
    const uint32_t none = 0xFFFFFFFFu;
    const uint32_t before = b > 0 ? keys[b - 1] : none, after = e < edges ? keys[e] : none;
    for (int c0 = lane * Q; c0 < d; c0 += T * Q) {
      const int c = last_cols<Q>(c0, d);
      const bool streamed = whole_aligned<D, Q>(dx + c) && dx_stride * sizeof(D) % 16 == 0;
      uint32_t cur = none;
      bool left = false;  // the run came in from the span before
      float sum[Q] = {};
      auto close = [&](bool right) {
        if (cur >= (uint32_t)rows) return;
        if (!left && !right) {
          store_whole<D, Q>(dx + (int64_t)cur * dx_stride + c, sum, streamed);
        } else {
          store_whole<float, Q>(partial + (2 * s + (left ? 0 : 1)) * d + c, sum, false);
        }
      };
      for (int32_t at = b; at < e; at += kMeanAhead) {
        uint32_t k[kMeanAhead];
        int32_t i[kMeanAhead];
        float share[kMeanAhead];
        // (the arrays have room behind their last entry for whole vectors)
#pragma unroll
        for (int u = 0; u < kMeanAhead; u += 4) {
          *reinterpret_cast<uint4*>(k + u) = *reinterpret_cast<const uint4*>(keys + at + u);
          *reinterpret_cast<int4*>(i + u) = *reinterpret_cast<const int4*>(vals + at + u);
          *reinterpret_cast<float4*>(share + u) = *reinterpret_cast<const float4*>(shares + at + u);
        }
        cols_t<D, Q> r[kMeanAhead], a[ADD ? kMeanAhead : 1];
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u) {
          if (at + u >= e) k[u] = none;
          const uint32_t prev = u > 0 ? k[u - 1] : (at == b ? before : cur);
          r[u] = (cols_t<D, Q>)(D)0.0f;
          if (k[u] < (uint32_t)rows) r[u] = *reinterpret_cast<const cols_t<D, Q>*>(dout + i[u] * dout_stride + c);
          if constexpr (ADD) {
            a[u] = (cols_t<D, Q>)(D)0.0f;
            if (k[u] != prev && k[u] < (uint32_t)add_rows)
              a[u] = *reinterpret_cast<const cols_t<D, Q>*>(add + (int64_t)k[u] * add_stride + c);
          }
        }
#pragma unroll
        for (int u = 0; u < kMeanAhead; ++u) {
          if (k[u] != cur && at + u < e) {
            if (at + u > b) close(false);
            left = at + u == b && k[u] == before;
            cur = k[u];
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] = ADD ? (float)a[ADD ? u : 0][q] : 0.0f;
          }
          if (k[u] < (uint32_t)rows) {
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] += (float)r[u][q] * share[u];
          }
        }
      }
      close(after == cur);
    }
  }
}

// The rows whose runs cross from span to span: the team of a run's first
// crossing adds its partial sums in order, kJoinAhead of them on their way.
constexpr int kJoinAhead = 8;
template <typename D, int Q, int T>
__global__ __launch_bounds__(kMeanNT) void k_block_mean_join(const uint32_t* __restrict__ keys, int32_t edges, int32_t rows, int d, int span,
                                                             const float* __restrict__ partial, D* __restrict__ dx,
                                                             int64_t dx_stride) {
  constexpr int kTeams = kMeanNT / T;
  const int lane = threadIdx.x % T;
  const int64_t spans = ((int64_t)edges + span - 1) / span;
  for (int64_t s = 1 + (int64_t)blockIdx.x * kTeams + threadIdx.x / T; s < spans; s += (int64_t)gridDim.x * kTeams) {
    const int64_t at = s * span;
    const uint32_t k = keys[at];
    if (k >= (uint32_t)rows || keys[at - 1] != k || (s > 1 && keys[at - span - 1] == k)) continue;
    for (int c0 = lane * Q; c0 < d; c0 += T * Q) {
      const int c = last_cols<Q>(c0, d);
      float sum[Q];
      load_cols<float, Q>(partial + (2 * (s - 1) + 1) * d + c, Q, sum);
      bool on = true;
      for (int64_t t = s; on; t += kJoinAhead) {
        float v[kJoinAhead][Q];
        uint32_t at_end[kJoinAhead];
        // (read whether they belong to the row or not: a sum's load need not wait for its key's)
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
          const int64_t to = min(t + u, spans - 1);
          at_end[u] = keys[to * span];
          load_cols<float, Q>(partial + 2 * to * d + c, Q, v[u]);
        }
        bool in[kJoinAhead];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
          in[u] = t + u < spans && at_end[u] == k;
          if (in[u]) {
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] += v[u][q];
          }
        }
        on = in[kJoinAhead - 1];
      }
      store_cols<D, Q>(dx + (int64_t)k * dx_stride + c, Q, sum);
    }
  }
}

// The gradient of a block of few edges, in one launch: a wave per source row
// reads all indices and lists, in LDS and in order, the rows that list its
// source; the block has found each edge's row before. It is bound by its latency,
// of which a source that many rows list has most: with 128 floats, 300 edges
// 8.8 us a call, 2000 edges over 500, 2000 and 8192 sources 19, 13 and 16, where
// the sort's launches take 20, and 20, 26 and 30. A source reads all indices, so
// more edges or sources go to the sort (2000 edges over 16K sources 26 and 30
// us, over 32K 44 and 30), and so do long lists.
constexpr int kFewEdges = 2048, kFewRows = 2048;  // of the block
constexpr int kFewSources = 8192;

template <typename D, int Q, bool ADD>
__global__ __launch_bounds__(kMeanNT) void k_block_mean_backward_few(const int32_t* __restrict__ indptr,
                                                                     const int32_t* __restrict__ indices, int32_t n,
                                                                     int32_t edges, int32_t rows, const D* __restrict__ dout,
                                                                     int64_t dout_stride, int d, const D* __restrict__ add,
                                                                     int64_t add_stride, int32_t add_rows, D* __restrict__ dx,
                                                                     int64_t dx_stride) {
  __shared__ int16_t row_of[kFewEdges];
  __shared__ int16_t lists[kMeanNT / MS_WAVE][kFewEdges];
  __shared__ float shares[kFewRows];
  const int lane = lane_id();
  const int wave = wave_uniform((int32_t)wave_id());
  for (int e = threadIdx.x; e < edges; e += kMeanNT) row_of[e] = -1;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kMeanNT) {
    int32_t b, e;
    row_span(indptr, i, edges, b, e);
    shares[i] = share_of(b, e);
    for (int32_t at = b; at < e; ++at) row_of[at] = (int16_t)i;
  }
  __syncthreads();
  const int64_t j = (int64_t)blockIdx.x * (kMeanNT / MS_WAVE) + wave;
  if (j >= rows) return;
  int16_t* list = lists[wave];
  int count = 0;
  for (int e0 = 0; e0 < edges; e0 += MS_WAVE) {
    const int e = e0 + lane;
    const bool here = e < edges && indices[e] == (int32_t)j && row_of[e] >= 0;
    const uint64_t m = ballot(here);
    if (here) list[count + lanes_below(m)] = row_of[e];
    count += __popcll(m);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int c0 = lane * Q; c0 < d; c0 += MS_WAVE * Q) {
    const int c = last_cols<Q>(c0, d);
    float sum[Q] = {};
    if (ADD && j < add_rows) load_cols<D, Q>(add + j * add_stride + c, Q, sum);
    for (int at = 0; at < count; at += kMeanAhead) {
      cols_t<D, Q> r[kMeanAhead];
      float share[kMeanAhead];
#pragma unroll
      for (int u = 0; u < kMeanAhead; ++u) {
        r[u] = (cols_t<D, Q>)(D)0.0f;
        share[u] = 0.0f;
        if (at + u < count) {
          const int i = list[at + u];
          share[u] = shares[i];
          r[u] = *reinterpret_cast<const cols_t<D, Q>*>(dout + (int64_t)i * dout_stride + c);
        }
      }
#pragma unroll
      for (int u = 0; u < kMeanAhead; ++u)
#pragma unroll
        for (int q = 0; q < Q; ++q) sum[q] += (float)r[u][q] * share[u];
    }
    store_cols<D, Q>(dx + j * dx_stride + c, Q, sum);
  }
}

}  // namespace ms
