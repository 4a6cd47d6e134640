// adamw_kernels.hpp - one AdamW step over many tensors, states in 32 or 8 bits.
//
// The tensors' pointers travel in the launch's arguments, so a step is one
// launch per kAdamwTensors tensors and nothing is copied or kept. A block
// takes kAdamwBlock consecutive values of one tensor, a wave 256 of them at a
// time, which is also the block of values that share a scale in 8 bits: its
// largest magnitude is a reduction within the wave. Each value is read and
// written once; the kernel is bound by memory.
//
// Measured: 160M values, states in 8 bits 480 us (2.6 GB, 5.3 TB/s), the states
// read back as floats 275 us; nine weights of 131072 in all 7.0 us.
#pragma once

#include "common.hpp"
#include "values.hpp"

namespace ms {

constexpr int kAdamwNT = 256;
constexpr int kAdamwQ = 4;                     // values per lane: 256 per wave
constexpr int kAdamwShare = MS_WAVE * kAdamwQ; // values that share a scale
constexpr int kAdamwBlock = 16 * kAdamwShare;  // values per block: 4 turns of its waves
constexpr int kAdamwTensors = 48;

struct AdamwTensor {
  void* param;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  bf16* copy;
  int64_t n;
};
struct AdamwLaunch {
  AdamwTensor t[kAdamwTensors];
  int32_t first[kAdamwTensors + 1];  // first block of each tensor, then the number of blocks
  int32_t count;
  float decay, b1, b1c, b2, b2c, lr, v_factor, eps;
};
static_assert(sizeof(AdamwLaunch) <= 4000, "the launch's arguments hold the list");

// 8-bit codes of a value of m (a signed square law) and of v (a fourth power),
// and back. The products are taken in exactly this order, without fused
// multiply-adds, so that a state is the nearest code of its 32-bit value as
// the formula's own roundings give it. The roots of `fast` are the hardware's,
// a unit or two in the last place off: enough unless they lie so near the
// middle between two codes (unsure()) that the rounding could go the other way.
#pragma clang fp contract(off)
__device__ __forceinline__ float root_m(float t, bool fast) { return fast ? __builtin_amdgcn_sqrtf(t) : sqrtf(t); }
__device__ __forceinline__ float root_v(float t, bool fast) {
  return fast ? __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(t)) : sqrtf(sqrtf(t));
}
__device__ __forceinline__ bool unsure(float root) { return fabsf(root - (floorf(root) + 0.5f)) < 0x1p-12f; }
__device__ __forceinline__ int code_m(float m, float root) {
  const float c = fminf(rintf(root), 127.0f);
  return m < 0.0f ? -(int)c : (int)c;
}
__device__ __forceinline__ uint32_t code_v(float t, float root) {
  return t > 0.0f ? (uint32_t)fminf(fmaxf(rintf(root), 1.0f), 255.0f) : 0u;
}
__device__ __forceinline__ float value_m(int c, float scale) { return (float)(c * (c < 0 ? -c : c)) * scale; }
__device__ __forceinline__ float value_v(uint32_t c, float scale) {
  const float s = (float)(c * c);
  return (s * s) * scale;
}

// sqrt(v) to a unit or two in its last place, also where v is a denormal, which
// the hardware's root takes as 0.
__device__ __forceinline__ float root_of_moment(float v) {
  const bool small = v < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? 0x1p-32f : 1.0f);
}

// A block's scale from the bits of its largest magnitude, and the reciprocal
// (0 where every code is 0): NaN if a value is not finite.
__device__ __forceinline__ void state_scale(uint32_t mag, float top, float least, float& scale, float& inv) {
  const float a = __uint_as_float(mag);
  scale = a * top;
  inv = 1.0f / scale;
  if (!(a >= least)) scale = inv = 0.0f;
  if (mag >= 0x7F800000u) {
    scale = __builtin_nanf("");
    inv = 0.0f;
  }
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  for (int o = MS_WAVE / 2; o > 0; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o, MS_WAVE));
  return x;
}

template <typename P, typename G, int BITS>
__global__ __launch_bounds__(kAdamwNT) void k_adamw(AdamwLaunch a) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= (int)blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamwTensor t = a.t[lo];
  const int64_t begin = (int64_t)((int)blockIdx.x - a.first[lo]) * kAdamwBlock;
  const int lane = lane_id(), wave = wave_id();
  for (int64_t at = begin + wave * kAdamwShare; at < min(t.n, begin + kAdamwBlock); at += kAdamwNT * kAdamwQ) {
    const int64_t i = at + lane * kAdamwQ;
    const int valid = (int)min(t.n - i, (int64_t)kAdamwQ);  // may be negative
    float p[kAdamwQ] = {}, g[kAdamwQ] = {}, m[kAdamwQ] = {}, v[kAdamwQ] = {};
    if (valid > 0) {
      load_cols<P, kAdamwQ>((const P*)t.param + i, valid, p);
      load_cols<G, kAdamwQ>((const G*)t.grad + i, valid, g);
      if constexpr (BITS == 32) {
        load_cols<float, kAdamwQ>((const float*)t.m + i, valid, m);
        load_cols<float, kAdamwQ>((const float*)t.v + i, valid, v);
      } else {
        const float sm = t.m_scale[at / kAdamwShare], sv = t.v_scale[at / kAdamwShare];
        const int8_t* cm = (const int8_t*)t.m + i;
        const uint8_t* cv = (const uint8_t*)t.v + i;
        if (valid >= kAdamwQ) {
          const cols_t<int8_t, kAdamwQ> wm = *reinterpret_cast<const cols_t<int8_t, kAdamwQ>*>(cm);
          const cols_t<uint8_t, kAdamwQ> wv = *reinterpret_cast<const cols_t<uint8_t, kAdamwQ>*>(cv);
#pragma unroll
          for (int q = 0; q < kAdamwQ; ++q) {
            m[q] = value_m(wm[q], sm);
            v[q] = value_v(wv[q], sv);
          }
        } else {
#pragma unroll
          for (int q = 0; q < kAdamwQ; ++q)
            if (q < valid) {
              m[q] = value_m(cm[q], sm);
              v[q] = value_v(cv[q], sv);
            }
        }
      }
    }
    uint32_t mag_m = 0, mag_v = 0;
#pragma unroll
    for (int q = 0; q < kAdamwQ; ++q) {
      m[q] = m[q] * a.b1 + g[q] * a.b1c;
      v[q] = v[q] * a.b2 + (g[q] * g[q]) * a.b2c;
      p[q] = p[q] * a.decay;
      // (the quotient to a few units in its last place: it is small beside p. Its
      // divisor is 0, or a normal number)
      p[q] = p[q] - (m[q] * a.lr) * __builtin_amdgcn_rcpf(root_of_moment(v[q]) * a.v_factor + a.eps);
      mag_m = max(mag_m, __float_as_uint(m[q]) & 0x7FFFFFFFu);
      mag_v = max(mag_v, __float_as_uint(v[q]) & 0x7FFFFFFFu);
    }
    if (valid > 0) {
      store_cols<P, kAdamwQ>((P*)t.param + i, valid, p);
      if (t.copy) store_cols<bf16, kAdamwQ>(t.copy + i, valid, p);
    }
    if constexpr (BITS == 32) {
      if (valid > 0) {
        store_cols<float, kAdamwQ>((float*)t.m + i, valid, m);
        store_cols<float, kAdamwQ>((float*)t.v + i, valid, v);
      }
    } else {
      float sm, sv, im, iv;
      state_scale(wave_max(mag_m), 1.0f / (127.0f * 127.0f), 0x1p-112f, sm, im);
      state_scale(wave_max(mag_v), (float)(1.0 / (255.0 * 255.0 * 255.0 * 255.0)), 0x1p-94f, sv, iv);
      if (lane == 0) {
        t.m_scale[at / kAdamwShare] = sm;
        t.v_scale[at / kAdamwShare] = sv;
      }
      if (valid > 0) {
        float tv[kAdamwQ], rm[kAdamwQ], rv[kAdamwQ];
        bool again = false;
#pragma unroll
        for (int q = 0; q < kAdamwQ; ++q) {
          tv[q] = v[q] * iv;
          rm[q] = root_m(fabsf(m[q]) * im, true);
          rv[q] = root_v(tv[q], true);
          again |= unsure(rm[q]) || unsure(rv[q]);
        }
        if (again) {
#pragma unroll
          for (int q = 0; q < kAdamwQ; ++q) {
            rm[q] = root_m(fabsf(m[q]) * im, false);
            rv[q] = root_v(tv[q], false);
          }
        }
        cols_t<int8_t, kAdamwQ> wm;
        cols_t<uint8_t, kAdamwQ> wv;
#pragma unroll
        for (int q = 0; q < kAdamwQ; ++q) {
          wm[q] = (int8_t)(im != 0.0f ? code_m(m[q], rm[q]) : 0);
          wv[q] = (uint8_t)(iv != 0.0f ? code_v(tv[q], rv[q]) : 0u);
        }
        int8_t* cm = (int8_t*)t.m + i;
        uint8_t* cv = (uint8_t*)t.v + i;
        if (valid >= kAdamwQ) {
          *reinterpret_cast<cols_t<int8_t, kAdamwQ>*>(cm) = wm;
          *reinterpret_cast<cols_t<uint8_t, kAdamwQ>*>(cv) = wv;
        } else {
#pragma unroll
          for (int q = 0; q < kAdamwQ; ++q)
            if (q < valid) {
              cm[q] = wm[q];
              cv[q] = wv[q];
            }
        }
      }
    }
  }
}

// What 8-bit states stand for.
__global__ __launch_bounds__(kAdamwNT) void k_adamw_states(const int8_t* __restrict__ cm, const uint8_t* __restrict__ cv,
                                                           const float* __restrict__ sm, const float* __restrict__ sv,
                                                           int64_t n, float* __restrict__ m, float* __restrict__ v) {
  for (int64_t i = ((int64_t)blockIdx.x * kAdamwNT + threadIdx.x) * kAdamwQ; i < n; i += (int64_t)gridDim.x * kAdamwNT * kAdamwQ) {
    const float a = sm[i / kAdamwShare], b = sv[i / kAdamwShare];
    const int valid = (int)min(n - i, (int64_t)kAdamwQ);
    float x[kAdamwQ] = {}, y[kAdamwQ] = {};
    if (valid >= kAdamwQ) {
      const cols_t<int8_t, kAdamwQ> wm = *reinterpret_cast<const cols_t<int8_t, kAdamwQ>*>(cm + i);
      const cols_t<uint8_t, kAdamwQ> wv = *reinterpret_cast<const cols_t<uint8_t, kAdamwQ>*>(cv + i);
#pragma unroll
      for (int q = 0; q < kAdamwQ; ++q) {
        x[q] = value_m(wm[q], a);
        y[q] = value_v(wv[q], b);
      }
    } else {
#pragma unroll
      for (int q = 0; q < kAdamwQ; ++q)
        if (q < valid) {
          x[q] = value_m(cm[i + q], a);
          y[q] = value_v(cv[i + q], b);
        }
    }
    store_cols<float, kAdamwQ>(m + i, valid, x);
    store_cols<float, kAdamwQ>(v + i, valid, y);
  }
}
#pragma clang fp contract(fast)

}  // namespace ms
