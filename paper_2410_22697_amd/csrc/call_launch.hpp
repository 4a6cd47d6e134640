// call_launch.hpp - what the operators' C entry points share on the host:
// refusals, launches, and the choice of a kernel by type and size.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/massive.h"
#include "call_error.hpp"
#include "common.hpp"
#include "launch_rules.hpp"
#include "values.hpp"

namespace ms {

constexpr int64_t kMostBlocks = 1 << 23;  // of a launch: 256 threads each stay below 2^32 in all


#define REFUSE(...) return ms::call_error(MASSIVE_EINVAL, __VA_ARGS__)

// Enqueues a kernel and returns its own status (an error that some earlier call
// left behind is neither reported nor cleared).
template <typename... P, typename... A>
int launch(const char* what, void (*kernel)(P...), int64_t blocks, int threads, size_t lds, void* stream, A... args) {
  std::tuple<P...> held(static_cast<P>(args)...);  // the arguments in the kernel's own types
  const hipError_t e = std::apply(
      [&](P&... a) {
        void* ptrs[] = {(void*)&a...};
        return hipLaunchKernel((const void*)kernel, dim3((unsigned)blocks), dim3((unsigned)threads), ptrs, lds, (hipStream_t)stream);
      },
      held);
  return e == hipSuccess ? MASSIVE_OK : call_error(MASSIVE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool is_type(int32_t t) { return t == MASSIVE_F32 || t == MASSIVE_BF16; }
inline int size_of(int32_t t) { return t == MASSIVE_F32 ? 4 : 2; }
inline bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Lanes that share a row of d columns, q a lane: the power of two that covers
// it, at most a wave.
inline int team_of(int64_t d, int q) {
  int t = 1;
  while (t < MS_WAVE && (int64_t)t * q < d) t *= 2;
  return t;
}

template <typename F>
int with_team(int team, F f) {
  switch (team) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    case 32: return f(std::integral_constant<int, 32>());
    default: return f(std::integral_constant<int, 64>());
  }
}
template <typename F>
int with_type(int32_t type, F f) {
  return type == MASSIVE_F32 ? f((float*)nullptr) : f((bf16*)nullptr);
}
// Columns that a lane takes at a time: 16 bytes, or one where a row is shorter.
template <typename T, typename F>
int with_cols(T*, int64_t d, F f) {
  constexpr int q = 16 / sizeof(T);
  return d >= q ? f(std::integral_constant<int, q>()) : f(std::integral_constant<int, 1>());
}
template <typename F>
int with_bits(int bits, F f) {
  return bits == 8 ? f(std::integral_constant<int, 8>()) : f(std::integral_constant<int, 4>());
}

// Checks a row format; the layout that the kernels take, and the least bytes of
// a row.
__attribute__((visibility("hidden"))) int check_format(const massive_row_format* f, PackedRows* out, int64_t* least);

}  // namespace ms
