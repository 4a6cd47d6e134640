// layers.hip - the C ABI's operators between and beside a training step's
// layers: dropout, the root-mean-square norm, the gated layer. Argument checks
// and launches, as in operators.hip: a call only enqueues.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "../../include/massive.h"
#include "call_launch.hpp"
#include "dropout_kernels.hpp"
#include "norm_kernels.hpp"

namespace {

using namespace ms;

constexpr int64_t kMostRows = int64_t(1) << 29;
constexpr int64_t kMostCols = 1 << 20;

// ------------------------------------------------------------------- dropout
template <typename T>
int dropout(const massive_dropout_args* a, uint64_t below, void* stream) {
  Dropout<T> f;
  f.x = (const T*)a->x;
  f.residual = (const T*)a->residual;
  f.y = (T*)a->y;
  f.seed_at = a->seed_at;
  f.seed = a->seed;
  f.rows = a->rows;
  f.x_stride = a->x_stride;
  f.residual_stride = a->residual_stride;
  f.y_stride = a->y_stride;
  f.draw = a->draw;
  f.below = (uint32_t)below;
  f.all = below >> 32;
  f.d = a->d;
  f.scale = f.all ? 0.0f : (float)(1.0 / (1.0 - a->p));
  const int team = team_of(a->d, 16 / sizeof(T));
  const int64_t blocks = std::min(cdiv(a->rows, kDropAhead * (kDropNT / team)), kMostBlocks);
  return with_team(team, [&](auto t) { return launch("massive_dropout", k_dropout<T, t()>, blocks, kDropNT, 0, stream, f); });
}

// ---------------------------------------------------------------------- norm
// f(team, turns that a team holds in registers): a wave or a part of one for
// rows of up to 32 values a lane, else a block.
template <int Q, typename F>
int with_norm(int64_t d, F f) {
  using std::integral_constant;
  const integral_constant<int, 1> one;
  const integral_constant<int, 2> two;
  if (d <= MS_WAVE * Q) return with_team(team_of(d, Q), [&](auto team) { return f(team, one); });
  const integral_constant<int, MS_WAVE> wave;
  if (d <= 2 * MS_WAVE * Q) return f(wave, two);
  if (d <= 4 * MS_WAVE * Q) return f(wave, integral_constant<int, 4>());
  if constexpr (Q == 4)
    if (d <= 8 * MS_WAVE * Q) return f(wave, integral_constant<int, 8>());
  const integral_constant<int, kNormLong> block;
  return d <= kNormLong * Q ? f(block, one) : f(block, two);
}

constexpr int64_t kNormBlocks = 8192;      // a block takes several rows: it reads the weights once
constexpr int64_t kNormGradBlocks = 1024;  // and leaves one part of dw

template <typename T>
int rms_norm(const massive_norm_args* a, const PackedRows& packed, void* stream) {
  Norm<T> n;
  n.x = (const T*)a->x;
  n.residual = (const T*)a->residual;
  n.weight = (const T*)a->weight;
  n.sum = (T*)a->sum;
  n.y = a->fmt ? nullptr : (T*)a->y;
  n.table = a->fmt ? (uint8_t*)a->y : nullptr;
  n.slots = a->slots;
  n.rows = a->rows;
  n.x_stride = a->x_stride;
  n.residual_stride = a->residual_stride;
  n.sum_stride = a->sum_stride;
  n.y_stride = a->y_stride;
  n.table_rows = a->table_rows;
  n.f = packed;
  n.d = a->d;
  n.inv_d = 1.0f / a->d;
  n.eps = a->eps > 0 ? std::max((float)a->eps, std::numeric_limits<float>::min()) : 0.0f;
  auto go = [&](auto bits, auto q) {
    return with_norm<q()>(a->d, [&](auto team, auto turns) {
      constexpr int kNT = team() > MS_WAVE ? team() : kNormNT, kTeams = kNT / team();
      return launch("massive_rms_norm", k_rms_norm<T, team(), turns(), q(), bits()>, std::min(cdiv(a->rows, kTeams), kNormBlocks), kNT, 0, stream, n);
    });
  };
  using std::integral_constant;
  if (!a->fmt) return go(integral_constant<int, 0>(), integral_constant<int, 16 / sizeof(T)>());
  return with_bits(a->fmt->bits, [&](auto bits) { return go(bits, integral_constant<int, kRowsQ>()); });
}

// Blocks of the gradient's kernel, which are also the parts of dw.
int64_t norm_blocks(const massive_norm_grads* a) {
  const int q = 16 / size_of(a->type);
  int64_t blocks = 0;
  auto of = [&](auto team, auto) {
    constexpr int kTeams = team() > MS_WAVE ? 1 : kNormNT / team();
    // long rows' parts are kept to 256 MB
    blocks = std::min(cdiv(a->rows, kTeams), team() > MS_WAVE ? std::max<int64_t>(1, std::min<int64_t>(512, (int64_t(1) << 26) / a->d)) : kNormGradBlocks);
    return 0;
  };
  if (q == 4) with_norm<4>(a->d, of);
  else with_norm<8>(a->d, of);
  return blocks;
}

int check_norm(const massive_norm_grads* a) {
  if (!a) REFUSE("args is NULL");
  if (!is_type(a->type)) REFUSE("type must be MASSIVE_F32 or MASSIVE_BF16");
  if (a->rows < 0 || a->rows > kMostRows) REFUSE("rows must be in 0..2^29");
  if (a->d < 1 || a->d > kMostCols) REFUSE("d must be in 1..2^20");
  return MASSIVE_OK;
}

template <typename T>
int rms_norm_backward(const massive_norm_grads* a, void* workspace, void* stream) {
  const char* what = "massive_rms_norm_backward";
  NormGrads<T> n;
  n.dy = (const T*)a->dy;
  n.s = (const T*)a->s;
  n.weight = (const T*)a->weight;
  n.ds = a->dx ? (const T*)a->ds : nullptr;
  n.dx = (T*)a->dx;
  n.parts = a->dweight ? (float*)workspace : nullptr;
  n.rows = a->rows;
  n.dy_stride = a->dy_stride;
  n.s_stride = a->s_stride;
  n.ds_stride = a->ds_stride;
  n.dx_stride = a->dx_stride;
  n.d = a->d;
  n.inv_d = 1.0f / a->d;
  n.eps = a->eps > 0 ? std::max((float)a->eps, std::numeric_limits<float>::min()) : 0.0f;
  const int64_t blocks = norm_blocks(a);
  if (a->rows > 0) {
    const int rc = with_norm<16 / sizeof(T)>(a->d, [&](auto team, auto turns) {
      return launch(what, k_rms_norm_backward<T, team(), turns(), 16 / sizeof(T)>, blocks, team() > MS_WAVE ? team() : kNormNT, 0, stream, n);
    });
    if (rc) return rc;
  }
  if (!a->dweight) return MASSIVE_OK;
  return launch(what, k_rms_norm_join<T>, cdiv(a->d, kNormNT / kNormJoinWays), kNormNT, 0, stream, (const float*)workspace, blocks, a->d, (T*)a->dweight);
}

}  // namespace

extern "C" {

int massive_dropout(const massive_dropout_args* a, void* stream) {
  if (!a) REFUSE("args is NULL");
  if (!is_type(a->type)) REFUSE("type must be MASSIVE_F32 or MASSIVE_BF16");
  if (a->rows < 0 || a->rows > kMostRows) REFUSE("rows must be in 0..2^29");
  if (a->d < 1 || a->d > kMostCols) REFUSE("d must be in 1..2^20");
  if (!(a->p >= 0 && a->p <= 1)) REFUSE("p must be in [0, 1]");
  if (a->rows == 0) return MASSIVE_OK;
  if (!a->x || !a->y) REFUSE("x / y are NULL");
  if (a->x_stride < a->d || a->y_stride < a->d || (a->residual && a->residual_stride < a->d)) REFUSE("a stride is below d");
  const int size = size_of(a->type);
  if (!aligned(a->x, size) || !aligned(a->residual, size) || !aligned(a->y, size) || !aligned(a->seed_at, 8)) REFUSE("an array is not aligned");
  const uint64_t below = (uint64_t)std::nearbyint(a->p * 4294967296.0);  // whole numbers to 2^32
  return a->type == MASSIVE_F32 ? dropout<float>(a, below, stream) : dropout<bf16>(a, below, stream);
}

int massive_rms_norm(const massive_norm_args* a, void* stream) {
  if (!a) REFUSE("args is NULL");
  if (!is_type(a->type)) REFUSE("type must be MASSIVE_F32 or MASSIVE_BF16");
  if (a->rows < 0 || a->rows > kMostRows) REFUSE("rows must be in 0..2^29");
  if (a->d < 1 || a->d > kMostCols) REFUSE("d must be in 1..2^20");
  if (!(a->eps >= 0) || !std::isfinite((float)a->eps)) REFUSE("eps must be finite and not negative");
  PackedRows packed = {};
  if (a->fmt) {
    int64_t least;
    if (int rc = check_format(a->fmt, &packed, &least)) return rc;
    if (a->fmt->d != a->d) REFUSE("d is %d, the row format's %d", a->d, a->fmt->d);
    if (a->table_rows < 0) REFUSE("table_rows must not be negative");
  } else if (a->slots) {
    REFUSE("slots without a row format");
  }
  if (a->rows == 0) return MASSIVE_OK;
  if (!a->x || (!a->y && !(a->fmt && a->table_rows == 0))) REFUSE("x / y are NULL");
  if (a->x_stride < a->d || (!a->fmt && a->y_stride < a->d) || (a->residual && a->residual_stride < a->d) || (a->sum && a->sum_stride < a->d))
    REFUSE("a stride is below d");
  const int size = size_of(a->type);
  for (const void* p : {a->x, a->residual, a->weight, (const void*)a->sum, a->fmt ? nullptr : (const void*)a->y})
    if (!aligned(p, size)) REFUSE("an array is not aligned");
  if ((a->fmt && !aligned(a->y, 4)) || !aligned(a->slots, 4)) REFUSE("the table or slots is not aligned");
  return a->type == MASSIVE_F32 ? rms_norm<float>(a, packed, stream) : rms_norm<bf16>(a, packed, stream);
}

int massive_rms_norm_workspace(const massive_norm_grads* a, int64_t* bytes) {
  if (!bytes) REFUSE("bytes is NULL");
  if (int rc = check_norm(a)) return rc;
  *bytes = a->dweight ? norm_blocks(a) * a->d * 4 : 0;
  return MASSIVE_OK;
}

int massive_rms_norm_backward(const massive_norm_grads* a, void* workspace, int64_t workspace_bytes, void* stream) {
  if (int rc = check_norm(a)) return rc;
  if (!(a->eps >= 0) || !std::isfinite((float)a->eps)) REFUSE("eps must be finite and not negative");
  if (!a->dx && !a->dweight) return MASSIVE_OK;
  if (a->rows > 0) {
    if (!a->dy || !a->s) REFUSE("dy / s are NULL");
    if (a->dy_stride < a->d || a->s_stride < a->d || (a->ds && a->ds_stride < a->d) || (a->dx && a->dx_stride < a->d))
      REFUSE("a stride is below d");
  }
  const int size = size_of(a->type);
  for (const void* p : {a->dy, a->s, a->weight, a->ds, (const void*)a->dx, (const void*)a->dweight})
    if (!aligned(p, size)) REFUSE("an array is not aligned");
  const int64_t need = a->dweight ? norm_blocks(a) * a->d * 4 : 0;
  if (need > 0) {
    if (!workspace || workspace_bytes < need)
      return call_error(MASSIVE_ECAPACITY, "workspace of %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0), (long long)need);
    if (!aligned(workspace, 16)) REFUSE("workspace is not 16-byte aligned");
  }
  return a->type == MASSIVE_F32 ? rms_norm_backward<float>(a, workspace, stream) : rms_norm_backward<bf16>(a, workspace, stream);
}

}  // extern "C"
