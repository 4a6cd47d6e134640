// gated_rules.hpp - which kernel a gated layer's call takes, its tiles, its parts
// and its workspace, in plain C++ so that the rules are also built and checked
// without a GPU.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/massive.h"
#include "launch_rules.hpp"

namespace ms {

// A block of the products makes 64 NB by kTileSecond results, in steps of
// kTileStepBytes of the reduction.
constexpr int kTileSecond = 128, kTileStepBytes = 64;
constexpr int kGateNT = 256;
constexpr int kGateUnits = 32;  // units of 16 bytes of a row that a block of dz takes
constexpr int kGateWays = kGateNT / kGateUnits;

inline int gated_size(int32_t type) { return type == MASSIVE_F32 ? 4 : 2; }

// Whether rows begin at multiples of 16 bytes (NULL counts as such).
inline bool in_units(const void* p, int64_t stride, int32_t type) {
  return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * gated_size(type) % 16 == 0);
}

// ------------------------------------------------------------------- forward
// Whether a call takes the form in which a block's waves share the reduction: for
// few results, and in bf16 for a reduction long enough that one block's steps
// last longer than that. us in a graph, few / tiles: bf16, 16 rows -> 1024 by k:
// 256 7.3 / 6.2, 448 8.3 / 8.2, 512 8.7 / 8.9, 1024 12.9 / 14.6, 2048 21 / 26 (250 rows
// 8.3 / 6.5, 9.5 / 8.5, 9.7 / 9.3, 13.9 / 15.1, 22 / 26; the rule's worst, 1000 rows
// of 2048 -> 256, 36 / 26); fp32, k 128 8.7 / 12.3, 256
// 9.9 / 21, 2048 50 / 144. At the limit of results, 250 rows of 256 -> 1024 fp32 11 / 22,
// beyond it 1000 33 / 24 and 4000 of 128 -> 256 27 / 14.5.
inline bool gated_few(const massive_gated_args* a) {
  return a->rows * round_up(a->n, 32) <= int64_t(1) << 18 && (a->type == MASSIVE_F32 || a->k + a->k_second > 448);
}

// Narrow tiles (64 outputs of both halves, not 128) until there are two rounds of
// wide ones for the chip (256 -> 1024 in bf16: 4000 rows 11.8 us wide, 10.8 narrow,
// 16000 30.3 and 30.1, 110K 171 and 183).
inline bool gated_narrow(const massive_gated_args* a) { return cdiv(a->rows, kTileSecond) * cdiv(a->n, 128) < 1024; }

// Whether the rows of x, x2 and both parts of w can go to LDS directly.
inline bool gated_direct(const massive_gated_args* a) {
  return in_units(a->x, a->x_stride, a->type) && in_units(a->x_second, a->x_second_stride, a->type) && in_units(a->w, a->w_stride, a->type) &&
         (!a->x_second || a->k * gated_size(a->type) % 16 == 0);
}

// ----------------------------------------------------------------- gradients
// dw's tiles (128 outputs of both halves; made on the way, 64 of each) and the
// parts of its rows: as many blocks as the chip holds at a time, none of less
// than eight steps of rows (four in fp32, whose steps last longer) where there
// are more. us of all gradients but dx. Narrow tiles / wide ones, 110K rows -> 1024
// bf16: 96 columns 160 / 196, 128 166 / 199, 160 381 / 205 (dz can no longer be made on
// its way); 2000 rows 20 / 26, 21 / 26, 31 / 28; fp32 27.5K 146 / 248, 151 / 250, 350 / 252.
// Least steps 2, 4, 8, 16: bf16 1000 x 256 -> 1024 33, 28, 27, 31, 4000 36, 35, 32,
// 35, 2000 x 128 -> 128 14, 14, 17, 22; fp32 1000 x 256 -> 1024 38, 35, 41, 53, 2000 x
// 128 -> 128 18, 17, 22, 31.
struct GatedDwPlan {
  int nb, second;
  int64_t tiles_n, tiles_k, part, parts, floats;  // floats: of the parts, none of a single one
};
inline GatedDwPlan gated_dw_plan(const massive_gated_grads* a) {
  GatedDwPlan p;
  const int vector = 16 / gated_size(a->type), step = kTileStepBytes / gated_size(a->type);
  p.second = (int)round_up(a->k, vector);
  const int64_t cols = p.second + a->k_second, n = 2 * (int64_t)a->n;
  p.nb = cols <= 128 ? 2 : 4;
  p.tiles_n = cdiv(n, kTileSecond);
  p.tiles_k = cdiv(cols, 64 * p.nb);
  const int64_t most = std::max<int64_t>(1, cdiv(a->rows, (a->type == MASSIVE_F32 ? 4 : 8) * step));
  p.part = std::max<int64_t>(1, round_up(cdiv(a->rows, std::min(most, std::max<int64_t>(1, 512 / (p.tiles_n * p.tiles_k)))), step));
  p.parts = cdiv(a->rows, p.part);
  p.floats = a->dw && p.parts > 1 ? p.parts * n * ((int64_t)a->k + a->k_second) : 0;
  return p;
}

// dx's tiles, narrow ones where wide ones are less than a round for the chip (us of
// dz and dx, narrow / wide, -> 1024 in bf16 and 512 in fp32: 256 columns, 16K rows
// 58 / 69, 48K 176 / 177, 64K 231 / 218, 110K 372 / 362; 512 columns, 32K 148 / 137, 110K
// 490 / 458; 128 columns, 110K 343 / 357; fp32 256, 32K 196 / 198, 64K 396 / 384), and
// the parts of its reduction over dz's columns where there are few tiles. A step
// takes a block about 0.4 us (bf16; fp32 1), and a part's values 8 bytes written
// and read at ~4 TB/s; with the join's launch, 4 us, that says how many parts pay
// (us of all gradients in bf16, parts / none: 16 rows of 256 -> 1024 20 / 42,
// 1000 rows 50 / 56; with four parts wherever tiles leave room, 16K rows of 128 ->
// 256 65, with none 36), up to 768 blocks (at most 512, 768, 1024: fp32 4000 x 512 ->
// 2048 174, 179, 201, 16391 x 200 -> 323 112, 104, 104).
struct GatedDxPlan {
  int nb;
  int64_t tiles_n, tiles, part, parts, floats;
};
inline GatedDxPlan gated_dx_plan(const massive_gated_grads* a) {
  GatedDxPlan p;
  const int64_t cols = (a->dx ? a->k : 0) + (a->dx_second ? a->k_second : 0), n = 2 * (int64_t)a->n, step = kTileStepBytes / gated_size(a->type);
  const int64_t row_tiles = cdiv(a->rows, kTileSecond), steps = cdiv(n, step);
  p.nb = cols <= 128 || row_tiles * cdiv(cols, 256) < 512 ? 2 : 4;
  p.tiles_n = std::max<int64_t>(1, cdiv(cols, 64 * p.nb));
  p.tiles = row_tiles * p.tiles_n;
  const double all = steps * (a->type == MASSIVE_F32 ? 1.0 : 0.4), each = 2e-6 * a->rows * cols;
  int64_t parts = p.nb == 4 ? 1 : (int64_t)std::min(std::sqrt(all / std::max(each, 1e-9)), 768.0 / std::max<int64_t>(1, p.tiles));
  parts = std::max<int64_t>(1, std::min(parts, steps / 4));
  if (all * (1 - 1.0 / parts) < 4 + parts * each) parts = 1;
  p.part = round_up(cdiv(n, parts), step);
  p.parts = cdiv(n, p.part);
  p.floats = p.parts > 1 ? p.parts * a->rows * cols : 0;
  return p;
}

// The backward pass's workspace: dz, the parts of db, those of dw or, later, of
// dx. It has room for dz also where dw is all that is asked for and dz may never
// be written: that hangs on where x lies, which its size does not.
struct GatedPlan {
  int64_t groups, part, parts, sums_at, dw_at, bytes;
  bool in_units;  // sizes for which dz can be made on its way into dw; db is summed in that way's order then, by any way
  GatedDwPlan dw;
  GatedDxPlan dx;
};
inline GatedPlan gated_plan(const massive_gated_grads* a) {
  GatedPlan p;
  const int size = gated_size(a->type), vector = 16 / size;
  p.groups = cdiv(a->n, kGateUnits * vector);
  p.part = std::max<int64_t>(1, cdiv(a->rows, std::max<int64_t>(1, std::min(cdiv(a->rows, 4 * kGateWays), 2048 / std::min<int64_t>(2048, p.groups)))));
  p.parts = cdiv(a->rows, p.part);
  p.dw = gated_dw_plan(a);
  p.in_units = a->k % vector == 0 && a->k_second % vector == 0 && a->n >= vector && p.dw.tiles_k == 1;
  p.sums_at = a->dx || a->dx_second || a->dw ? round_up(a->rows * 2 * a->n * size, 16) : 0;
  p.dw_at = p.sums_at + (a->dbias ? round_up((p.in_units ? p.dw.parts : p.parts) * 2 * a->n * 4, 16) : 0);
  p.dx = gated_dx_plan(a);
  p.bytes = p.dw_at + std::max(p.dw.floats, p.dx.floats) * 4;
  return p;
}

// Whether x's rows go to LDS directly, as those of dw's product.
inline bool gated_x_in_units(const massive_gated_grads* a) {
  const int vector = 16 / gated_size(a->type);
  return a->k % vector == 0 && a->k_second % vector == 0 && in_units(a->x, a->x_stride, a->type) && in_units(a->x_second, a->x_second_stride, a->type);
}
inline bool gated_dw_made(const massive_gated_grads* a, const GatedPlan& p) { return a->dw && p.in_units && gated_x_in_units(a); }
inline bool gated_dw_direct(const massive_gated_grads* a) { return gated_x_in_units(a) && 2 * (int64_t)a->n * gated_size(a->type) % 16 == 0; }
inline bool gated_dx_direct(const massive_gated_grads* a) {
  const int vector = 16 / gated_size(a->type);
  const char* w = (const char*)a->w + (a->dx ? 0 : (int64_t)a->k * gated_size(a->type));
  return 2 * (int64_t)a->n % vector == 0 && ((a->dx ? a->k : 0) + (a->dx_second ? a->k_second : 0)) % vector == 0 && in_units(w, a->w_stride, a->type);
}

// Threads a value that add up `count` parts, as many as fill the chip where there
// are `values` of them (us, one / sixteen: 33 parts of 524K values 14-18 / 19; all
// gradients with 250 parts of 8K 90 / 34; one / four / sixteen, all but dx in bf16:
// 110K x 64 -> 512, 65K values 95 / 87 / 85, x 128, 131K 102 / 94 / 94, x 256, 262K 127 / 122 /
// 124, 20K x 160, 164K 48 / 39 / 41, 4000 x 256 -> 1024, 524K 32 / 32 / 33).
inline int gated_ways(int64_t count, int64_t values) { return count <= 2 || values >= 1 << 19 ? 1 : values >= 1 << 17 ? 4 : 16; }

}  // namespace ms
