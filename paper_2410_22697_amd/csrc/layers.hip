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
#include "gated_kernels.hpp"
#include "gated_rules.hpp"
#include "norm_kernels.hpp"

namespace {

using namespace ms;

constexpr int64_t kMostRows = int64_t(1) << 29;
constexpr int64_t kMostCols = 1 << 20;

// Columns a lane takes of rows of d columns: 16 bytes, but 8 where rows are whole
// in units of 8 bytes and not in units of 16, as those of 100 columns in bf16
// are: a lane's 16 bytes would straddle lines and the row's end be read value by
// value (854K such rows, us, 16 bytes / 8: norm 122 / 75, with the residual 243 /
// 137, gradients 235 / 178). By d alone, so that results
// do not hang on where the arrays lie.
template <typename T, typename F>
int with_unit(int64_t d, F f) {
  if constexpr (sizeof(T) == 2)
    if (d % 8 == 4) return f(std::integral_constant<int, 4>());
  return f(std::integral_constant<int, 16 / sizeof(T)>());
}

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
  return with_unit<T>(a->d, [&](auto q) {
    const int64_t units = cdiv(a->d, q()), all = a->rows * units;
    // rounded up: at * inverse / 2^32 is at / units for all at and units below kDropChunk + units
    const uint32_t inverse = units > 1 ? (uint32_t)(((uint64_t(1) << 32) + units - 1) / units) : 0;
    return launch("massive_dropout", k_dropout<T, q()>, std::min(cdiv(all, kDropChunk), kMostBlocks), kDropNT, 0, stream, f, (uint32_t)units, inverse, all);
  });
}

// ---------------------------------------------------------------------- norm
// f(team, turns that a team holds in registers): a wave or a part of one for
// rows of up to 32 values a lane, else a block. The gradients' rows of more than
// one turn of 16-byte units in bf16 take a block of twice the threads: with two
// turns in registers a CU would hold one block of half the waves (us, two turns /
// twice the threads: 30K x 5000 418 / 312, 20K x 8192 316 / 239, 8000 x 20000 698 /
// 608; in units of four values, and forward, two turns are as fast or faster).
template <int Q, bool GRADS, typename F>
int with_norm(int64_t d, F f) {
  using std::integral_constant;
  const integral_constant<int, 1> one;
  const integral_constant<int, 2> two;
  if (d <= MS_WAVE * Q) return with_team(team_of(d, Q), [&](auto team) { return f(team, one); });
  const integral_constant<int, MS_WAVE> wave;
  if (d <= 2 * MS_WAVE * Q) return f(wave, two);
  if (d <= 4 * MS_WAVE * Q) return f(wave, integral_constant<int, 4>());
  const integral_constant<int, kNormLong> block;
  if constexpr (Q == 4) {
    static_assert(kNormLong <= 8 * MS_WAVE, "a block's first turn has no columns that a wave's eight have not");
    if (d <= 8 * MS_WAVE * Q) return f(wave, integral_constant<int, 8>());
    return f(block, two);
  } else {
    if (d <= kNormLong * Q) return f(block, one);
    if constexpr (GRADS) return f(integral_constant<int, 2 * kNormLong>(), one);
    else return f(block, two);
  }
}

constexpr int64_t kNormBlocks = 8192;      // a block takes several rows: it reads the weights once
// The gradient's blocks leave a part of dw each: 1024 of them, and 2048 where a
// team would have over 64 rows one after the other (us, 1024 / 2048: 854K x 100
// bf16, 104 rows a team, 178 / 117; 242K x 256, 30 rows, 71 / 80).
constexpr int64_t kNormGradBlocks = 1024, kNormGradRows = 64;

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
    return with_norm<q(), false>(a->d, [&](auto team, auto turns) {
      constexpr int kNT = team() > MS_WAVE ? team() : kNormNT, kTeams = kNT / team();
      return launch("massive_rms_norm", k_rms_norm<T, team(), turns(), q(), bits()>, std::min(cdiv(a->rows, kTeams), kNormBlocks), kNT, 0, stream, n);
    });
  };
  using std::integral_constant;
  if (!a->fmt) return with_unit<T>(a->d, [&](auto q) { return go(integral_constant<int, 0>(), q); });
  return with_bits(a->fmt->bits, [&](auto bits) { return go(bits, integral_constant<int, kRowsQ>()); });
}

// Blocks of the gradient's kernel, which are also the parts of dw.
int64_t norm_blocks(const massive_norm_grads* a) {
  return with_type(a->type, [&](auto* t) -> int {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_unit<T>(a->d, [&](auto q) {
      return with_norm<q(), true>(a->d, [&](auto team, auto) {
        constexpr int kTeams = team() > MS_WAVE ? 1 : kNormNT / team();
        // long rows' parts are kept to 256 MB
        const int64_t all = cdiv(a->rows, kTeams);
        if (team() > MS_WAVE) return (int)std::min(all, std::max<int64_t>(1, std::min<int64_t>(512, (int64_t(1) << 26) / a->d)));
        return (int)std::min(all, all > kNormGradRows * kNormGradBlocks ? 2 * kNormGradBlocks : kNormGradBlocks);
      });
    });
  });
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
    const int rc = with_unit<T>(a->d, [&](auto q) {
      return with_norm<q(), true>(a->d, [&](auto team, auto turns) {
        return launch(what, k_rms_norm_backward<T, team(), turns(), q()>, blocks, team() > MS_WAVE ? team() : kNormNT, 0, stream, n);
      });
    });
    if (rc) return rc;
  }
  if (!a->dweight) return MASSIVE_OK;
  return launch(what, k_rms_norm_join<T>, cdiv(a->d, kNormNT / kNormJoinWays), kNormNT, 0, stream, (const float*)workspace, blocks, a->d, (T*)a->dweight);
}

// --------------------------------------------------------------- gated layer
int check_gated(int64_t rows, int32_t n, int32_t k, int32_t k_second, int32_t type, int32_t act, const void* x_second) {
  if (!is_type(type)) REFUSE("type must be MASSIVE_F32 or MASSIVE_BF16");
  if (act < MASSIVE_ACT_NONE || act > MASSIVE_ACT_SILU) REFUSE("act is not one of MASSIVE_ACT_*");
  if (rows < 0 || rows > kMostRows) REFUSE("rows must be in 0..2^29");
  if (n < 1 || k < 1 || k_second < 0 || n > (1 << 19) || k > kMostCols || k_second > kMostCols)
    REFUSE("n must be in 1..2^19, k in 1..2^20, k_second in 0..2^20");
  if ((k_second > 0) != (x_second != nullptr) && rows > 0) REFUSE("k_second columns and x_second go together");
  return MASSIVE_OK;
}

template <typename T>
Operand<T> rows_of(const void* p, int64_t stride, int64_t rows, int64_t k) {
  return Operand<T>{(const T*)p, nullptr, stride, 0, rows, k, MASSIVE_ACT_NONE};
}

template <typename T>
int gated(const massive_gated_args* a, void* stream) {
  const char* what = "massive_gated";
  Gated<T> f;
  f.x[0] = rows_of<T>(a->x, a->x_stride, a->rows, a->k);
  f.x[1] = rows_of<T>(a->x_second, a->x_second_stride, a->rows, a->k_second);
  f.w[0] = {(const T*)a->w, a->w_stride};
  f.w[1] = {(const T*)a->w + a->k, a->w_stride};
  f.bias = (const T*)a->bias;
  f.y = (T*)a->y;
  f.pre = (T*)a->pre;
  f.y_stride = a->y_stride;
  f.pre_stride = a->pre_stride;
  f.rows = a->rows;
  f.n = a->n;
  f.act = a->act;
  if (!gated_few(a)) {
    const bool direct = gated_direct(a);
    auto tile = [&](auto nb) {
      const int64_t tiles_n = cdiv(a->n, 32 * nb()), blocks = cdiv(a->rows, kTileSecond) * tiles_n;
      if (blocks > kMostBlocks) REFUSE("too many rows and columns for one call");
      return launch(what, direct ? k_gated_tile<T, nb(), true> : k_gated_tile<T, nb(), false>, blocks, kTileNT, 0, stream, f, (int)tiles_n, blocks);
    };
    return gated_narrow(a) ? tile(std::integral_constant<int, 2>()) : tile(std::integral_constant<int, 4>());
  }
  const int tiles_n = (int)cdiv(a->n, 32);
  return launch(what, k_gated_few<T>, cdiv(a->rows, 32) * tiles_n, kFewNT, 0, stream, f, tiles_n);
}

template <typename T>
GatedDz<T> gates_of(const massive_gated_grads* a, char* dz) {
  GatedDz<T> f = {};
  f.dy = (const T*)a->dy;
  f.pre = (const T*)a->pre;
  f.dz = (T*)dz;
  f.rows = a->rows;
  f.dy_stride = a->dy_stride;
  f.pre_stride = a->pre_stride;
  f.n = a->n;
  f.act = a->act;
  return f;
}

template <typename F>
int with_act_of(int act, F f) {
  switch (act) {
    case MASSIVE_ACT_RELU: return f(std::integral_constant<int, kActRelu>());
    case MASSIVE_ACT_GELU: return f(std::integral_constant<int, kActGelu>());
    case MASSIVE_ACT_SILU: return f(std::integral_constant<int, kActSilu>());
    default: return f(std::integral_constant<int, kActNone>());
  }
}

// Adds up parts, of which the sizes say that there are `values`.
template <typename T>
int gated_join(const GatedJoin<T>& j, int64_t values, void* stream) {
  auto ways = [&](auto w) {
    constexpr int kValues = kGateNT / w() * 4;
    return launch("massive_gated_backward", k_gated_join<T, w()>, cdiv(j.values[0], kValues) + cdiv(j.values[1], kValues), kGateNT, 0, stream, j);
  };
  switch (gated_ways(j.count, values)) {
    case 1: return ways(std::integral_constant<int, 1>());
    case 4: return ways(std::integral_constant<int, 4>());
    default: return ways(std::integral_constant<int, 16>());
  }
}

// dz and db by themselves.
template <typename T>
int gated_dz(const massive_gated_grads* a, const GatedPlan& p, char* workspace, void* stream) {
  const char* what = "massive_gated_backward";
  GatedDz<T> f = gates_of<T>(a, a->dx || a->dx_second || a->dw ? workspace : nullptr);
  f.parts = a->dbias ? (float*)(workspace + p.sums_at) : nullptr;
  f.part = p.part;
  f.groups = (int)p.groups;
  if (int rc = launch(what, k_gated_dz<T>, p.groups * p.parts, kGateNT, 0, stream, f)) return rc;
  if (!a->dbias) return MASSIVE_OK;
  return launch(what, k_rms_norm_join<T>, cdiv(2 * a->n, kNormNT / kNormJoinWays), kNormNT, 0, stream, (const float*)f.parts, p.parts, 2 * a->n, (T*)a->dbias);
}

template <typename T>
int gated_dx(const massive_gated_grads* a, const GatedPlan& p, char* workspace, void* stream) {
  const GatedDxPlan& d = p.dx;
  const int n = 2 * a->n;
  LinearDx<T> f;
  f.dz = rows_of<T>(workspace, n, a->rows, n);
  const int k0 = a->dx ? a->k : 0, k1 = a->dx_second ? a->k_second : 0;
  f.w = {(const T*)a->w + (a->dx ? 0 : a->k), a->w_stride};
  f.dx[0] = (T*)a->dx;
  f.dx[1] = (T*)a->dx_second;
  f.dx_stride[0] = a->dx_stride;
  f.dx_stride[1] = a->dx_second_stride;
  f.rows = a->rows;
  f.cols = k0 + k1;
  f.split = k0;
  float* parts = d.parts > 1 ? (float*)(workspace + p.dw_at) : nullptr;
  const bool direct = gated_dx_direct(a);
  auto tile = [&](auto nb) {
    return launch("massive_gated_backward", direct ? k_gated_dx<T, nb(), true> : k_gated_dx<T, nb(), false>, d.tiles * d.parts, kTileNT, 0, stream, f, parts, d.part,
                  (int)d.tiles_n, d.tiles, d.tiles * d.parts);
  };
  if (int rc = d.nb == 2 ? tile(std::integral_constant<int, 2>()) : tile(std::integral_constant<int, 4>())) return rc;
  if (!parts) return MASSIVE_OK;
  GatedJoin<T> j = {};
  j.parts[0] = parts;
  j.to[0] = f.dx[0];
  j.values[0] = a->rows * f.cols;
  j.stride[0] = a->dx_stride;
  j.count = d.parts;
  j.cols[0] = f.cols;
  j.split = k0;
  j.beyond = f.dx[1];
  j.beyond_stride = a->dx_second_stride;
  return gated_join(j, j.values[0], stream);
}

// The joins of dw and db, each if there are any.
template <typename T>
int dw_join(const massive_gated_grads* a, const float* dw, const float* db, int64_t parts, void* stream) {
  GatedJoin<T> j = {};
  const int cols = a->k + a->k_second, n = 2 * a->n;
  j.parts[0] = dw;
  j.parts[1] = db;
  j.to[0] = (T*)a->dw;
  j.to[1] = (T*)a->dbias;
  j.values[0] = dw ? (int64_t)n * cols : 0;
  j.values[1] = db ? n : 0;
  j.stride[0] = a->dw_stride;
  j.count = parts;
  j.cols[0] = j.split = cols;
  j.cols[1] = n;
  return gated_join(j, (int64_t)n * cols, stream);  // (db's order does not hang on whether dw is there)
}

template <typename T>
int gated_backward(const massive_gated_grads* a, const GatedPlan& p, char* workspace, void* stream) {
  const char* what = "massive_gated_backward";
  const bool dx = a->dx || a->dx_second;
  const bool made = gated_dw_made(a, p), sums = !made && a->dbias && p.in_units;
  const GatedDwPlan& d = p.dw;
  const bool several = d.parts > 1;
  const int n = 2 * a->n;
  GatedDw<T> f;
  f.dz = rows_of<T>(workspace, n, a->rows, n);
  f.x[0] = rows_of<T>(a->x, a->x_stride, a->rows, a->k);
  f.x[1] = rows_of<T>(a->x_second, a->x_second_stride, a->rows, a->k_second);
  f.parts = several && a->dw ? (float*)(workspace + p.dw_at) : nullptr;
  f.sums = several && a->dbias && p.in_units ? (float*)(workspace + p.sums_at) : nullptr;
  f.dw = (T*)a->dw;
  f.db = (T*)a->dbias;
  f.dw_stride = a->dw_stride;
  f.rows = a->rows;
  f.part = d.part;
  f.n = n;
  f.k[0] = a->k;
  f.k[1] = a->k_second;
  f.second = d.second;
  f.tiles_n = (int)d.tiles_n;
  f.tiles_k = (int)d.tiles_k;
  if (sums) {
    const int64_t groups = cdiv(a->n, kSumsCols), blocks = d.parts * groups;
    const int rc = with_act_of(a->act, [&](auto act) {
      return launch(what, k_gated_sums<T, act()>, blocks, kSumsNT, 0, stream, f, gates_of<T>(a, dx || a->dw ? workspace : nullptr), (int)groups, blocks);
    });
    if (rc) return rc;
  } else if (!made) {
    if (int rc = gated_dz<T>(a, p, workspace, stream)) return rc;
  }
  if (a->dw) {
    const int64_t blocks = d.parts * d.tiles_n * d.tiles_k;
    auto tile = [&](auto nb) {
      if (made)
        return with_act_of(a->act, [&](auto act) {
          return launch(what, k_gated_dw_made<T, nb(), act()>, blocks, kTileNT, 0, stream, f, gates_of<T>(a, dx ? workspace : nullptr), blocks);
        });
      return launch(what, gated_dw_direct(a) ? k_gated_dw<T, nb(), true> : k_gated_dw<T, nb(), false>, blocks, kTileNT, 0, stream, f, blocks);
    };
    if (int rc = d.nb == 2 ? tile(std::integral_constant<int, 2>()) : tile(std::integral_constant<int, 4>())) return rc;
  }
  if (f.parts || f.sums)
    if (int rc = dw_join<T>(a, f.parts, f.sums, d.parts, stream)) return rc;
  return dx ? gated_dx<T>(a, p, workspace, stream) : MASSIVE_OK;
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

int massive_gated(const massive_gated_args* a, void* stream) {
  if (!a) REFUSE("args is NULL");
  if (int rc = check_gated(a->rows, a->n, a->k, a->k_second, a->type, a->act, a->x_second)) return rc;
  if (a->rows == 0) return MASSIVE_OK;
  if (!a->x || !a->w || !a->y) REFUSE("x / w / y are NULL");
  if (a->x_stride < a->k || (a->x_second && a->x_second_stride < a->k_second) || a->w_stride < (int64_t)a->k + a->k_second ||
      a->y_stride < a->n || (a->pre && a->pre_stride < 2 * (int64_t)a->n))
    REFUSE("a stride is below its rows' length");
  const int size = size_of(a->type);
  for (const void* p : {a->x, a->x_second, a->w, a->bias, (const void*)a->y, (const void*)a->pre})
    if (!aligned(p, size)) REFUSE("an array is not aligned");
  return a->type == MASSIVE_F32 ? gated<float>(a, stream) : gated<bf16>(a, stream);
}

int massive_gated_workspace(const massive_gated_grads* a, int64_t* bytes) {
  if (!bytes) REFUSE("bytes is NULL");
  if (!a) REFUSE("args is NULL");
  if (int rc = check_gated(a->rows, a->n, a->k, a->k_second, a->type, a->act, a->x_second)) return rc;
  *bytes = a->rows > 0 ? gated_plan(a).bytes : 0;
  return MASSIVE_OK;
}

int massive_gated_backward(const massive_gated_grads* a, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!a) REFUSE("args is NULL");
  if (int rc = check_gated(a->rows, a->n, a->k, a->k_second, a->type, a->act, a->x_second)) return rc;
  if (!a->dx && !a->dx_second && !a->dw && !a->dbias) return MASSIVE_OK;
  if (a->dx_second && !a->k_second) REFUSE("dx_second without a second input");
  const int64_t k = (int64_t)a->k + a->k_second;
  if (a->dw && a->dw_stride < k) REFUSE("a stride is below its rows' length");
  if (a->rows > 0) {
    if (!a->dy || !a->pre) REFUSE("dy / pre are NULL");
    if ((a->dx || a->dx_second) && !a->w) REFUSE("w is NULL");
    if (a->dw && !a->x) REFUSE("x is NULL");
    if (a->dy_stride < a->n || a->pre_stride < 2 * (int64_t)a->n || (a->x && a->x_stride < a->k) ||
        (a->x_second && a->x_second_stride < a->k_second) || (a->w && a->w_stride < k) || (a->dx && a->dx_stride < a->k) ||
        (a->dx_second && a->dx_second_stride < a->k_second))
      REFUSE("a stride is below its rows' length");
  }
  const int size = size_of(a->type);
  for (const void* p : {a->dy, a->pre, a->x, a->x_second, a->w, (const void*)a->dx, (const void*)a->dx_second, (const void*)a->dw, (const void*)a->dbias})
    if (!aligned(p, size)) REFUSE("an array is not aligned");
  const GatedPlan p = gated_plan(a);
  const int64_t dw_blocks = p.dw.parts * p.dw.tiles_n * p.dw.tiles_k;
  if (p.groups * p.parts > kMostBlocks || (a->dw && (dw_blocks > kMostBlocks || cdiv(2 * a->n * k, 4 * kGateNT) + (1 << 15) > kMostBlocks)) ||
      cdiv(a->rows, kTileSecond) * cdiv(k, 128) > kMostBlocks)
    REFUSE("too many rows and columns for one call");
  if (a->rows == 0) {  // sums over no rows
    if (!a->dw && !a->dbias) return MASSIVE_OK;
    // the pointers only say which of the two are asked for: with no parts nothing is read
    const float *dw = (const float*)a->dw, *db = (const float*)a->dbias;
    return a->type == MASSIVE_F32 ? dw_join<float>(a, dw, db, 0, stream) : dw_join<bf16>(a, dw, db, 0, stream);
  }
  if (!workspace || workspace_bytes < p.bytes)
    return call_error(MASSIVE_ECAPACITY, "workspace of %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0), (long long)p.bytes);
  if (!aligned(workspace, 16)) REFUSE("workspace is not 16-byte aligned");
  return a->type == MASSIVE_F32 ? gated_backward<float>(a, p, (char*)workspace, stream) : gated_backward<bf16>(a, p, (char*)workspace, stream);
}

}  // extern "C"
