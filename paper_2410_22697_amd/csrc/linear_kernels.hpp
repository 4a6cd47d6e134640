// linear_kernels.hpp - a layer's product with its epilogue, and its gradients.
//
//   forward  y = act([x | x2] w^T + bias) + residual
//   dx       dz w              dz = dy * act'(pre), taken as it is read
//   dw       dz^T [x | x2], dbias = sum of dz over the rows
//
// All three are C = A B^T over a reduction index k, with the matrix unit's
// 32x32 products (bf16: 16 k at a time; fp32: 2). Here are the forms of y and
// dx for few rows (linear_stream.hpp has those for many, and
// linear_weights.hpp dw): tiles of BM x BN by a block of four waves. An operand
// is read along k (its rows are k-contiguous: x, w in the forward pass, dz for
// dx) or across k (its columns are: w for dx), through LDS, the next tile's
// loads in flight meanwhile.
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

constexpr int kLinNT = 256;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// ------------------------------------------------------------- activations
// Phi(z) and exp(-z^2 / 2): erf by Abramowitz and Stegun's 7.1.26 (an error of
// 1.5e-7 at most) where the result is rounded to bf16 anyway, since it shares
// the exponential that the slope needs; by the library's erff for fp32.
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  e = __expf(-0.5f * z * z);
  if constexpr (sizeof(T) == 2) {
    const float x = fabsf(z) * 0.70710678f;
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    const float poly = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    const float tail = 0.5f * poly * e;  // 1 - Phi(|z|)
    return z < 0.0f ? tail : 1.0f - tail;
  } else {
    e = expf(-0.5f * z * z);
    return 0.5f * erfcf(-z * 0.70710678f);
  }
}

template <typename T>
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == kActRelu) return z <= 0.0f ? 0.0f : z;  // a NaN stays one
  if (act == kActGelu) {
    float e;
    return z * normal_cdf<T>(z, e);
  }
  if (act == kActSilu) return z / (1.0f + (sizeof(T) == 2 ? __expf(-z) : expf(-z)));
  return z;
}

// g * act'(z). Where z is so large that a factor vanishes, the product with it
// is taken as 0 rather than as infinity times 0.
template <typename T>
__device__ __forceinline__ float act_grad(float g, float z, int act) {
  if (act == kActRelu) return z > 0.0f ? g : 0.0f;
  if (act == kActGelu) {
    float e;
    const float p = normal_cdf<T>(z, e);
    return g * (p + (e > 0.0f ? z * e * 0.39894228f : 0.0f));
  }
  const float q = 1.0f / (1.0f + (sizeof(T) == 2 ? __expf(-z) : expf(-z)));
  const float s = q * (1.0f - q);
  return g * (q + (s > 0.0f ? z * s : 0.0f));
}

// The same for several values: the activation is the same for all of them.
template <typename T>
__device__ __forceinline__ void act_values(float (&z)[8], int act) {
  if (act == kActNone) return;
  if (act == kActRelu) {
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] = act_value<T>(z[q], kActRelu);
  } else if (act == kActGelu) {
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] = act_value<T>(z[q], kActGelu);
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] = act_value<T>(z[q], kActSilu);
  }
}
template <typename T, int Q>
__device__ __forceinline__ void act_grads(cols_t<T, Q>& g, const cols_t<T, Q>& z, int act) {
  if (act == kActRelu) {
#pragma unroll
    for (int q = 0; q < Q; ++q) g[q] = (T)act_grad<T>((float)g[q], (float)z[q], kActRelu);
  } else if (act == kActGelu) {
#pragma unroll
    for (int q = 0; q < Q; ++q) g[q] = (T)act_grad<T>((float)g[q], (float)z[q], kActGelu);
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q) g[q] = (T)act_grad<T>((float)g[q], (float)z[q], kActSilu);
  }
}

// ---------------------------------------------------------------- operands
// One operand of a product: element (r, k), r below R, k below K, is at
// p[r * stride + k] (along k) or p[k * stride + r] (across k); with pre, the
// element is p's times the activation's slope at pre's.
template <typename T>
struct Operand {
  const T* p;
  const T* pre;
  int64_t stride, pre_stride;
  int64_t R, K;
  int act;
};

// A tile of BR rows and 128 bytes of k (64 bf16 or 32 fp32) in LDS, in 16-byte
// chunks of neighbouring k: chunk c of row r lies at place c ^ swizzle(r) of
// its row, so that eight rows at one chunk (a fragment read) and eight chunks
// at one row or every fourth row (the two ways of writing) meet in distinct
// banks.
__device__ __forceinline__ int swizzle(int r) { return (r ^ (r >> 3)) & 7; }
__device__ __forceinline__ int chunk_at(int r, int c) { return r * 128 + ((c ^ swizzle(r)) << 4); }

template <typename T>
struct Tile {
  static constexpr int kK = 128 / sizeof(T);  // k per tile
  static constexpr int kV = 16 / sizeof(T);   // elements per chunk
};

// The way of one tile from global memory to LDS: load() starts the loads,
// put() writes the tile.
template <typename T, bool ALONG, bool SLOPE, int BR>
struct Staged;

template <typename T, bool SLOPE, int BR>
struct Staged<T, true, SLOPE, BR> {  // along k: a thread takes chunk t % 8 of rows t / 8 + 32 i
  static constexpr int kV = Tile<T>::kV, kN = BR / 32;
  cols_t<T, kV> v[kN], z[SLOPE ? kN : 1];

  __device__ __forceinline__ static void one(const T* p, int64_t left, cols_t<T, kV>& v) {
    if (left >= kV) {
      v = *reinterpret_cast<const cols_t<T, kV>*>(p);
    } else {
#pragma unroll
      for (int q = 0; q < kV; ++q) v[q] = q < left ? p[q] : (T)0.0f;
    }
  }
  __device__ __forceinline__ void load(const Operand<T>& o, int64_t r0, int64_t k0) {
    const int64_t k = k0 + (threadIdx.x % 8) * kV;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int64_t r = r0 + threadIdx.x / 8 + 32 * i;
      const int64_t left = r < o.R ? o.K - k : 0;
      one(o.p + r * o.stride + k, left, v[i]);
      if constexpr (SLOPE) one(o.pre + r * o.pre_stride + k, left, z[i]);
    }
  }
  __device__ __forceinline__ void put(char* lds, const Operand<T>& o) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int r = threadIdx.x / 8 + 32 * i;
      if constexpr (SLOPE) act_grads<T, kV>(v[i], z[i], o.act);
      *reinterpret_cast<u32x4*>(lds + chunk_at(r, threadIdx.x % 8)) = __builtin_bit_cast(u32x4, v[i]);
    }
  }
  // fp32: k = 4 * (lane / 32) + j of an 8-k step, j = 0..3
  __device__ __forceinline__ static f32x4 fragment_f32(const char* lds, int r, int step, int half) {
    return *reinterpret_cast<const f32x4*>(lds + chunk_at(r, 2 * step + half));
  }
};

template <int BR>
struct Staged<bf16, false, false, BR> {  // across k: a thread takes 8 k by 4 r, and turns them
  typedef cols_t<bf16, 4> quad;
  quad v[8];
  static constexpr int kRB = BR / 4;  // threads along r

  __device__ __forceinline__ static void one(const bf16* p, int64_t left, quad& v) {
    if (left >= 4) {
      v = *reinterpret_cast<const quad*>(p);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = q < left ? p[q] : (bf16)0.0f;
    }
  }
  __device__ __forceinline__ static bool mine() { return (int)threadIdx.x < kRB * 8; }
  __device__ __forceinline__ void load(const Operand<bf16>& o, int64_t r0, int64_t k0) {
    if (!mine()) return;
    const int64_t r = r0 + (threadIdx.x % kRB) * 4, k1 = k0 + (threadIdx.x / kRB) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t left = k1 + j < o.K ? o.R - r : 0;
      one(o.p + (k1 + j) * o.stride + r, left, v[j]);
    }
  }
  __device__ __forceinline__ void put(char* lds, const Operand<bf16>&) {
    if (!mine()) return;
    const int r = (threadIdx.x % kRB) * 4, c = threadIdx.x / kRB;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x8 w;
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = v[j][q];
      *reinterpret_cast<bf16x8*>(lds + chunk_at(r + q, c)) = w;
    }
  }
};

template <int BR>
struct Staged<float, false, false, BR> {  // across k in fp32: LDS keeps [k][r], a thread takes 4 r of every 8th k
  static constexpr int kRB = BR / 4, kKT = kLinNT / kRB, kN = 32 / kKT;
  typedef cols_t<float, 4> quad;
  quad v[kN];

  __device__ __forceinline__ static void one(const float* p, int64_t left, quad& v) {
    if (left >= 4) {
      v = *reinterpret_cast<const quad*>(p);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = q < left ? p[q] : 0.0f;
    }
  }
  __device__ __forceinline__ void load(const Operand<float>& o, int64_t r0, int64_t k0) {
    const int64_t r = r0 + (threadIdx.x % kRB) * 4;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int64_t k = k0 + threadIdx.x / kRB + kKT * i;
      const int64_t left = k < o.K ? o.R - r : 0;
      one(o.p + k * o.stride + r, left, v[i]);
    }
  }
  __device__ __forceinline__ void put(char* lds, const Operand<float>&) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int k = threadIdx.x / kRB + kKT * i, r = (threadIdx.x % kRB) * 4;
      *reinterpret_cast<f32x4*>(lds + (k * BR + r) * 4) = v[i];
    }
  }
  __device__ __forceinline__ static f32x4 fragment_f32(const char* lds, int r, int step, int half) {
    const float* p = reinterpret_cast<const float*>(lds) + (step * 8 + half * 4) * BR + r;
    return f32x4{p[0], p[BR], p[2 * BR], p[3 * BR]};
  }
};

// ------------------------------------------------------------------- tiles
// Blocks are dealt to the eight XCDs in turn; consecutive tiles (which share
// rows of A) go to one XCD, whose L2 then serves them.
__device__ __forceinline__ int64_t tile_of_block(int64_t b, int64_t blocks) {
  constexpr int64_t kXcds = 8;
  const int64_t per = blocks / kXcds, rest = blocks % kXcds, x = b % kXcds;
  return x * per + min(x, rest) + b / kXcds;
}

// The accumulators of a block's BM x BN tile: four waves as 2 x 2, each
// (BM / 2) x (BN / 2) in squares of 32.
template <typename T, int BM, int BN>
struct Acc {
  static constexpr int kI = BM / 64, kJ = BN / 64;
  f32x16 c[kI][kJ] = {};

  // adds one tile of k: a, b in LDS
  template <typename SA, typename SB>
  __device__ __forceinline__ void multiply(const char* a, const char* b) {
    const int lane = lane_id(), wave = wave_id();
    const int half = lane / 32;
    const int ra = (wave / 2) * (BM / 2) + lane % 32, rb = (wave % 2) * (BN / 2) + lane % 32;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        bf16x8 fa[kI], fb[kJ];
#pragma unroll
        for (int i = 0; i < kI; ++i) fa[i] = *reinterpret_cast<const bf16x8*>(a + chunk_at(ra + 32 * i, 2 * s + half));
#pragma unroll
        for (int j = 0; j < kJ; ++j) fb[j] = *reinterpret_cast<const bf16x8*>(b + chunk_at(rb + 32 * j, 2 * s + half));
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int j = 0; j < kJ; ++j) c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], c[i][j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        f32x4 fa[kI], fb[kJ];
#pragma unroll
        for (int i = 0; i < kI; ++i) fa[i] = SA::fragment_f32(a, ra + 32 * i, s, half);
#pragma unroll
        for (int j = 0; j < kJ; ++j) fb[j] = SB::fragment_f32(b, rb + 32 * j, s, half);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int j = 0; j < kJ; ++j)
              c[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i][q], fb[j][q], c[i][j], 0, 0, 0);
      }
    }
  }

  // Gives the tile to out(row, column, values, 8) in runs of eight columns of a
  // row. Each wave turns its part, 32 rows at a time, through LDS of its own
  // (accumulator register g of a lane is row 8 (g / 4) + 4 (lane / 32) + g % 4,
  // column lane % 32). The block has passed a barrier since the tile's last use.
  static constexpr int kPitch = BN / 2 + 4;
  static constexpr int kTurnBytes = 4 * 32 * kPitch * 4;
  template <typename F>
  __device__ __forceinline__ void emit(char* lds, F out) {
    const int lane = lane_id(), wave = wave_id();
    float* turn = reinterpret_cast<float*>(lds) + wave * 32 * kPitch;
    constexpr int kRuns = BN / 16;  // runs of eight columns in a wave's rows
#pragma unroll
    for (int i = 0; i < kI; ++i) {
#pragma unroll
      for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int g = 0; g < 16; ++g)
          turn[(8 * (g / 4) + 4 * (lane / 32) + g % 4) * kPitch + 32 * j + lane % 32] = c[i][j][g];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int u = 0; u < 32 * kRuns / MS_WAVE; ++u) {
        const int at = u * MS_WAVE + lane, r = at / kRuns, run = at % kRuns;
        float x[8];
        const f32x4 lo = *reinterpret_cast<const f32x4*>(turn + r * kPitch + run * 8);
        const f32x4 hi = *reinterpret_cast<const f32x4*>(turn + r * kPitch + run * 8 + 4);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          x[q] = lo[q];
          x[q + 4] = hi[q];
        }
        out((wave / 2) * (BM / 2) + 32 * i + r, (wave % 2) * (BN / 2) + run * 8, x);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
};

template <typename T, int BM, int BN>
constexpr int lin_lds_bytes() {
  return (BM + BN) * 128 > Acc<T, BM, BN>::kTurnBytes ? (BM + BN) * 128 : Acc<T, BM, BN>::kTurnBytes;
}

// c += A B^T over k in [k0, k1): the loads of a tile fly while the one before
// is multiplied.
template <typename T, bool A_ALONG, bool A_SLOPE, bool B_ALONG, int BM, int BN>
__device__ __forceinline__ void product(Acc<T, BM, BN>& c, char* lds, const Operand<T>& a, int64_t ra, const Operand<T>& b,
                                        int64_t rb, int64_t k0, int64_t k1) {
  typedef Staged<T, A_ALONG, A_SLOPE, BM> SA;
  typedef Staged<T, B_ALONG, false, BN> SB;
  char *la = lds, *lb = lds + BM * 128;
  SA sa;
  SB sb;
  if (k0 < k1) {
    sa.load(a, ra, k0);
    sb.load(b, rb, k0);
  }
  for (int64_t k = k0; k < k1; k += Tile<T>::kK) {
    __syncthreads();
    sa.put(la, a);
    sb.put(lb, b);
    __syncthreads();
    if (k + Tile<T>::kK < k1) {
      sa.load(a, ra, k + Tile<T>::kK);
      sb.load(b, rb, k + Tile<T>::kK);
    }
    c.template multiply<SA, SB>(la, lb);
  }
}

// ----------------------------------------------------------------- forward
template <typename T>
struct LinearForward {
  Operand<T> x[2], w[2];  // the inputs and their columns of w
  const T *bias, *residual;
  T *y, *pre;
  int64_t residual_stride, y_stride, pre_stride;
  int64_t rows;
  int n, act;
};

// The epilogue of eight neighbouring outputs of a row: z holds their products.
template <typename T>
__device__ __forceinline__ void linear_finish(const LinearForward<T>& a, int64_t row, int col, float (&z)[8]) {
  const int left = a.n - col;
  if (left <= 0) return;
  float t[8];
  if (a.bias) {
    load_cols<T, 8>(a.bias + col, left, t);
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] += t[q];
  }
  if (a.pre) store_cols<T, 8>(a.pre + row * a.pre_stride + col, left, z);
  act_values<T>(z, a.act);
  if (a.residual) {
    load_cols<T, 8>(a.residual + row * a.residual_stride + col, left, t);
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] += t[q];
  }
  store_cols<T, 8>(a.y + row * a.y_stride + col, left, z);
}

template <typename T, int BM, int BN>
__global__ __launch_bounds__(kLinNT) void k_linear(LinearForward<T> a, int tiles_n, int64_t blocks) {
  __shared__ __align__(16) char lds[lin_lds_bytes<T, BM, BN>()];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t r0 = tile / tiles_n * BM;
  const int n0 = (int)(tile % tiles_n) * BN;
  Acc<T, BM, BN> c;
#pragma unroll 1
  for (int s = 0; s < 2; ++s)
    product<T, true, false, true, BM, BN>(c, lds, a.x[s], r0, a.w[s], n0, 0, a.x[s].K);
  __syncthreads();
  c.emit(lds, [&](int r, int col, float (&z)[8]) {
    if (r0 + r < a.rows) linear_finish(a, r0 + r, n0 + col, z);
  });
}

// ---------------------------------------------------------------------- dx
template <typename T>
struct LinearDx {
  Operand<T> dz, w[2];
  T* dx[2];
  int64_t dx_stride[2];
  int64_t rows;
  int k[2], tiles[2];  // columns of each input, and their tiles (0 where its gradient is not asked for)
};

template <typename T, bool SLOPE, int BM, int BN>
__global__ __launch_bounds__(kLinNT) void k_linear_dx(LinearDx<T> a, int64_t blocks) {
  __shared__ __align__(16) char lds[lin_lds_bytes<T, BM, BN>()];
  const int tiles = a.tiles[0] + a.tiles[1];
  const int64_t tile = tile_of_block(blockIdx.x, blocks);
  const int64_t r0 = tile / tiles * BM;
  int at = (int)(tile % tiles);
  const int s = at >= a.tiles[0] ? 1 : 0;
  at -= s ? a.tiles[0] : 0;
  const int n0 = at * BN;
  Acc<T, BM, BN> c;
  product<T, true, SLOPE, false, BM, BN>(c, lds, a.dz, r0, a.w[s], n0, 0, a.dz.K);
  __syncthreads();
  T* dx = a.dx[s];
  const int64_t stride = a.dx_stride[s];
  const int k = a.k[s];
  c.emit(lds, [&](int r, int col, float* v) {
    const int64_t row = r0 + r;
    const int left = k - n0 - col;
    if (row < a.rows && left > 0) store_cols<T, 8>(dx + row * stride + n0 + col, left, v);
  });
}

// Adds the parts, of dw (rows of `cols` values) and of dbias.
template <typename T>
__global__ __launch_bounds__(kLinNT) void k_linear_join(const float* __restrict__ dw_parts, const float* __restrict__ bias_parts,
                                                        int64_t parts, int n, int cols, T* __restrict__ dw, int64_t dw_stride,
                                                        T* __restrict__ dbias) {
  const int64_t all = (dw_parts ? (int64_t)n * cols : 0) + (bias_parts ? n : 0);
  for (int64_t i = (int64_t)blockIdx.x * kLinNT + threadIdx.x; i < all; i += (int64_t)gridDim.x * kLinNT) {
    const int64_t in_dw = dw_parts ? (int64_t)n * cols : 0;
    const bool bias = i >= in_dw;
    const float* p = bias ? bias_parts + (i - in_dw) : dw_parts + i;
    const int64_t step = bias ? n : (int64_t)n * cols;
    float t = 0.0f;
#pragma unroll 8
    for (int64_t q = 0; q < parts; ++q) t += p[q * step];
    if (bias) dbias[i - in_dw] = (T)t;
    else dw[i / cols * dw_stride + i % cols] = (T)t;
  }
}

}  // namespace ms
