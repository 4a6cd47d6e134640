// operators.hip - the C ABI's operators of a training step: packed rows, the
// mean over a sampled block, a layer's product, the AdamW step. Argument checks
// and launches; the kernels are in the headers included here. A call only
// enqueues: it allocates nothing, waits for nothing and keeps nothing.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/massive.h"
#include "adamw_kernels.hpp"
#include "block_kernels.hpp"
#include "call_error.hpp"
#include "linear_few.hpp"
#include "linear_kernels.hpp"
#include "linear_stream.hpp"
#include "linear_weights.hpp"
#include "rows_kernels.hpp"

namespace {

using ms::bf16;
using ms::call_error;

constexpr int64_t kMostBlocks = 1 << 23;  // of a launch: 256 threads each stay below 2^32 in all

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return cdiv(a, b) * b; }

#define REFUSE(...) return call_error(MASSIVE_EINVAL, __VA_ARGS__)

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

bool is_type(int32_t t) { return t == MASSIVE_F32 || t == MASSIVE_BF16; }
int size_of(int32_t t) { return t == MASSIVE_F32 ? 4 : 2; }
bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// -------------------------------------------------------------- packed rows
int check_format(const massive_row_format* f, ms::PackedRows* out, int64_t* least) {
  if (!f) REFUSE("the row format is NULL");
  if (f->d < 1 || f->d > (1 << 20)) REFUSE("d must be in 1..1048576");
  if (f->bits != 8 && f->bits != 4) REFUSE("bits must be 8 or 4");
  if (f->group != 0 && (f->group < 16 || f->group > 512 || (f->group & (f->group - 1))))
    REFUSE("group must be 0 or a power of two from 16 to 512");
  if (f->reserved != 0) REFUSE("reserved must be 0");
  const bool whole = f->group == 0 || f->group >= f->d;
  const int64_t groups = whole ? 1 : cdiv(f->d, f->group);
  out->d = f->d;
  out->group_log2 = whole ? 31 : __builtin_ctz((unsigned)f->group);
  out->floats_at = (int32_t)(4 * cdiv((int64_t)f->d * f->bits, 32));
  *least = out->floats_at + 4 * groups * (f->bits == 8 ? 1 : 2);
  out->row_bytes = f->row_bytes ? f->row_bytes : *least;
  if (out->row_bytes < *least || out->row_bytes % 4)
    REFUSE("row_bytes must be 0 or a multiple of 4 that is at least %lld", (long long)*least);
  return MASSIVE_OK;
}

// Lanes that share a row of d columns, q a lane: the power of two that covers
// it, at most a wave.
int team_of(int64_t d, int q) {
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

int pack_rows(const massive_row_format* fmt, const void* src, int32_t src_type, int64_t src_stride, int64_t n,
              const int32_t* slots, void* table, int64_t table_rows, void* stream) {
  ms::PackedRows f;
  int64_t least;
  if (int rc = check_format(fmt, &f, &least)) return rc;
  if (!is_type(src_type)) REFUSE("src_type must be MASSIVE_F32 or MASSIVE_BF16");
  if (n < 0 || table_rows < 0) REFUSE("n and table_rows must not be negative");
  if (n == 0 || table_rows == 0) return MASSIVE_OK;
  if (!src || !table) REFUSE("src / table are NULL");
  if (src_stride < f.d) REFUSE("src_stride is below d");
  if (!aligned(src, size_of(src_type)) || !aligned(slots, 4) || !aligned(table, 4)) REFUSE("src, slots or table is not aligned");
  const int team = team_of(f.d, ms::kRowsQ);
  const int64_t blocks = std::min(cdiv(n, ms::kRowsAhead * (ms::kRowsNT / team)), kMostBlocks);
  return with_type(src_type, [&](auto* s) {
    using S = std::remove_pointer_t<decltype(s)>;
    return with_bits(fmt->bits, [&](auto bits) {
      return with_team(team, [&](auto t) {
        return launch("massive_pack_rows", ms::k_pack_rows<S, bits(), t()>, blocks, ms::kRowsNT, 0, stream, (const S*)src,
                      src_stride, n, slots, (uint8_t*)table, table_rows, f);
      });
    });
  });
}

int unpack_rows(const massive_row_format* fmt, const void* table, int64_t table_rows, const int32_t* index, int64_t n,
                void* out, int32_t out_type, int64_t out_stride, void* stream) {
  ms::PackedRows f;
  int64_t least;
  if (int rc = check_format(fmt, &f, &least)) return rc;
  if (!is_type(out_type)) REFUSE("out_type must be MASSIVE_F32 or MASSIVE_BF16");
  if (n < 0 || table_rows < 0) REFUSE("n and table_rows must not be negative");
  if (n == 0) return MASSIVE_OK;
  if (!out || (table_rows > 0 && !table)) REFUSE("table / out are NULL");
  if (out_stride < f.d) REFUSE("out_stride is below d");
  if (!aligned(out, size_of(out_type)) || !aligned(index, 4) || !aligned(table, 4)) REFUSE("table, index or out is not aligned");
  const int team = team_of(f.d, 16 / size_of(out_type));
  const int64_t blocks = std::min(cdiv(n, ms::kRowsAhead * (ms::kRowsNT / team)), kMostBlocks);
  return with_type(out_type, [&](auto* o) {
    using O = std::remove_pointer_t<decltype(o)>;
    return with_bits(fmt->bits, [&](auto bits) {
      return with_team(team, [&](auto t) {
        return launch("massive_unpack_rows", ms::k_unpack_rows<O, bits(), t()>, blocks, ms::kRowsNT, 0, stream,
                      (const uint8_t*)table, table_rows, index, n, (O*)out, out_stride, f);
      });
    });
  });
}

// --------------------------------------------------------------- block mean
constexpr int64_t kMostIds = int64_t(1) << 30;  // rows and edges are counted in int32, some of them a step ahead

int check_block(const massive_block* b) {
  if (!b) REFUSE("the block is NULL");
  if (b->n < 0 || b->edges < 0 || b->rows < 0) REFUSE("n, edges and rows must not be negative");
  if (b->n > kMostIds || b->edges > kMostIds || b->rows > kMostIds) REFUSE("n, edges and rows must be at most 2^30");
  if (b->n > 0 && !b->indptr) REFUSE("indptr is NULL");
  if (b->edges > 0 && !b->indices) REFUSE("indices is NULL");
  if (!aligned(b->indptr, 4) || !aligned(b->indices, 4)) REFUSE("indptr or indices is not aligned");
  return MASSIVE_OK;
}

int block_mean(const massive_block* b, const void* x, int32_t x_type, int64_t x_stride, const massive_row_format* fmt,
               int32_t d, void* out, int32_t out_type, int64_t out_stride, void* stream) {
  if (int rc = check_block(b)) return rc;
  if (!is_type(out_type)) REFUSE("out_type must be MASSIVE_F32 or MASSIVE_BF16");
  if (!is_type(x_type) && x_type != MASSIVE_PACKED) REFUSE("x_type must be MASSIVE_F32, MASSIVE_BF16 or MASSIVE_PACKED");
  if (d < 1) REFUSE("d must be at least 1");
  ms::PackedRows f = {};
  f.d = d;
  if (x_type == MASSIVE_PACKED) {
    int64_t least;
    if (int rc = check_format(fmt, &f, &least)) return rc;
    if (fmt->d != d) REFUSE("d is %d, the row format's %d", d, fmt->d);
  } else {
    if (fmt) REFUSE("a row format is given, and x_type is not MASSIVE_PACKED");
    if (x_stride < d) REFUSE("x_stride is below d");
  }
  if (b->n == 0) return MASSIVE_OK;
  if (!out || (b->rows > 0 && !x)) REFUSE("x / out are NULL");
  if (out_stride < d) REFUSE("out_stride is below d");
  if (!aligned(out, size_of(out_type)) || !aligned(x, x_type == MASSIVE_PACKED ? 4 : size_of(x_type)))
    REFUSE("x or out is not aligned");
  auto go = [&](auto* s, auto* o, auto bits, auto q) {
    using S = std::remove_pointer_t<decltype(s)>;
    using O = std::remove_pointer_t<decltype(o)>;
    const int team = team_of(d, q());
    return with_team(team, [&](auto t) {
      return launch("massive_block_mean", ms::k_block_mean<S, bits(), O, q(), t()>,
                    std::min(cdiv(b->n, ms::kMeanNT / team), kMostBlocks), ms::kMeanNT, 0, stream, b->indptr, b->indices, b->n,
                    (int32_t)b->edges, x, (int32_t)b->rows, x_stride, f, (O*)out, out_stride);
    });
  };
  return with_type(out_type, [&](auto* o) {
    if (x_type == MASSIVE_PACKED)
      return with_bits(fmt->bits, [&](auto bits) { return go((float*)nullptr, o, bits, std::integral_constant<int, 8>()); });
    return with_type(x_type, [&](auto* s) {
      return with_cols(s, d, [&](auto q) { return go(s, o, std::integral_constant<int, 0>(), q); });
    });
  });
}

// The backward pass's workspace: two lists of pairs, the entries' shares, the
// chunks' counts, the digits' totals, the sources' marks, the spans' partial
// sums.
struct MeanPlan {
  int passes, bits;        // digits of the sort
  int chunks;
  int span;
  int64_t chunk, spans;
  int64_t keys[2], vals[2], shares, counts, totals, marks, partial, bytes;
};
MeanPlan mean_plan(const massive_block* b, int64_t d) {
  MeanPlan p = {};
  int need = 1;
  while ((int64_t(1) << need) <= b->rows) ++need;  // keys go up to rows
  p.passes = (int)cdiv(need, ms::kDigitBits);
  p.bits = (int)cdiv(need, p.passes);
  p.chunk = std::max<int64_t>(MS_WAVE, round_up(cdiv(b->edges, ms::kChunksMost), MS_WAVE));
  p.chunks = (int)cdiv(b->edges, p.chunk);
  // shorter spans fill the chip, longer ones leave fewer sums to join. 128 floats,
  // sources listed in proportion to their degrees, us of a call with 16 / 32 / 64:
  // 24K edges 37 / 40 / 48, 90K 50 / 51 / 57, 200K 71 / 66 / 69, 300K 93 / 92 / 83,
  // 550K 153 / 146 / 147, 800K 209 / 196 / 185 (256 floats 305 / 286 / 277). 128 of
  // bf16 change over later: 300K 86 / 81 / 87, 800K 169 / 153 / 146
  p.span = b->edges <= (1 << 16) ? 16 : b->edges <= (1 << 18) ? 32 : 64;
  p.spans = cdiv(b->edges, p.span);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += round_up(bytes, 16);
    return here;
  };
  const int64_t list = 4 * round_up(b->edges, ms::kMeanAhead);  // read in whole steps
  for (int i = 0; i < 2; ++i) p.keys[i] = take(list);
  for (int i = 0; i < 2; ++i) p.vals[i] = take(list);
  p.shares = take(list);
  p.counts = take(4 * (int64_t)p.chunks << p.bits);
  p.totals = take(int64_t(4) << p.bits);
  p.marks = take(b->rows);
  p.partial = take(p.spans * 2 * d * 4);
  p.bytes = at;
  return p;
}

// Whether the gradient takes the one-launch form, which reads every index for
// each source, and in which a source adds up its list by itself: 0.1 us an
// entry. Where sources are listed in proportion to their degrees the longest
// list has about edges / sqrt(rows) entries, of which 128 take as long as the
// sort's launches. One launch / sort, us with 128 floats: 1000 edges over 256
// sources 12 / 20, 64 19 / 20, 16 32 / 20, 1 107 / 26; 296 over 16 11 / 20, 4
// 19 / 20, 1 33 / 20.
bool few(const massive_block* b) {
  return b->edges <= ms::kFewEdges && b->n <= ms::kFewRows && b->rows <= ms::kFewSources && b->edges * b->edges <= (b->rows << 14);
}

int block_mean_backward(const massive_block* b, const void* dout, int32_t type, int64_t dout_stride, int32_t d,
                        const void* add, int64_t add_stride, int64_t add_rows, void* dx, int64_t dx_stride, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  if (int rc = check_block(b)) return rc;
  if (!is_type(type)) REFUSE("type must be MASSIVE_F32 or MASSIVE_BF16");
  if (d < 1) REFUSE("d must be at least 1");
  if (add_rows < 0 || add_rows > b->rows) REFUSE("add_rows must be in 0..rows");
  if (!add) add_rows = 0;
  if (add_rows > 0 && add_stride < d) REFUSE("add_stride is below d");
  if (b->rows == 0) return MASSIVE_OK;
  if (!dx || (b->n > 0 && !dout)) REFUSE("dout / dx are NULL");
  if (dx_stride < d || (b->n > 0 && dout_stride < d)) REFUSE("dout_stride or dx_stride is below d");
  const int size = size_of(type);
  if (!aligned(dout, size) || !aligned(add, size) || !aligned(dx, size)) REFUSE("dout, add or dx is not aligned");
  if (few(b))
    return with_type(type, [&](auto* t) {
      using D = std::remove_pointer_t<decltype(t)>;
      return with_cols(t, d, [&](auto q) {
        return launch("massive_block_mean_backward",
                      add_rows > 0 ? ms::k_block_mean_backward_few<D, q(), true> : ms::k_block_mean_backward_few<D, q(), false>,
                      cdiv(b->rows, ms::kMeanNT / MS_WAVE), ms::kMeanNT, 0, stream, b->indptr, b->indices, (int32_t)b->n,
                      (int32_t)(b->n > 0 ? b->edges : 0), (int32_t)b->rows, (const D*)dout, dout_stride, d, (const D*)add, add_stride,
                      (int32_t)add_rows, (D*)dx, dx_stride);
      });
    });
  const MeanPlan p = mean_plan(b, d);
  if (!workspace || workspace_bytes < p.bytes)
    return call_error(MASSIVE_ECAPACITY, "workspace of %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0),
                      (long long)p.bytes);
  if (!aligned(workspace, 16)) REFUSE("workspace is not 16-byte aligned");
  char* w = (char*)workspace;
  uint32_t* keys[2] = {(uint32_t*)(w + p.keys[0]), (uint32_t*)(w + p.keys[1])};
  int32_t* vals[2] = {(int32_t*)(w + p.vals[0]), (int32_t*)(w + p.vals[1])};
  float *shares = (float*)(w + p.shares), *partial = (float*)(w + p.partial);
  int32_t *counts = (int32_t*)(w + p.counts), *totals = (int32_t*)(w + p.totals);
  uint8_t* marks = (uint8_t*)(w + p.marks);
  const char* what = "massive_block_mean_backward";
  const int nt = ms::kSortWaves * MS_WAVE;
  // without a row no edge belongs to one
  const int chunks = b->n > 0 ? p.chunks : 0;
  const int32_t edges = chunks > 0 ? (int32_t)b->edges : 0, rows = (int32_t)b->rows, chunk = (int32_t)p.chunk;
  const int64_t sort_blocks = cdiv(std::max(chunks, 1), ms::kSortWaves);
  const size_t digits = sizeof(int32_t) << p.bits;
  if (int rc = launch(what, ms::k_edges, std::max(sort_blocks, std::min<int64_t>(cdiv(b->rows, 4 * nt), 512)), nt,
                      ms::kSortWaves * digits, stream, b->indptr, b->indices, (int32_t)b->n, edges, rows, chunk, chunks, p.bits,
                      keys[0], vals[0], counts, (uint32_t*)marks))
    return rc;
  int at = 0;
  for (int pass = 0; chunks > 0 && pass < p.passes; ++pass) {
    const int shift = pass * p.bits;
    if (pass > 0)
      if (int rc = launch(what, ms::k_digits, sort_blocks, nt, ms::kSortWaves * digits, stream, keys[at], edges, chunk, chunks, shift,
                          p.bits, counts))
        return rc;
    if (int rc = launch(what, ms::k_places, cdiv(1 << p.bits, ms::kPlacesDigits), ms::kPlacesDigits * ms::kPlacesRuns, 0, stream,
                        counts, chunks, p.bits, totals))
      return rc;
    const bool last = pass == p.passes - 1;
    if (int rc = launch(what, last ? ms::k_move<true> : ms::k_move<false>, sort_blocks, nt, (1 + ms::kSortWaves) * digits, stream,
                        keys[at], vals[at], edges, chunk, chunks, shift, p.bits, counts, totals, keys[1 - at], vals[1 - at],
                        b->indptr, rows, shares, marks))
      return rc;
    at = 1 - at;
  }
  return with_type(type, [&](auto* t) {
    using D = std::remove_pointer_t<decltype(t)>;
    return with_cols(t, d, [&](auto q) {
      const int team = team_of(d, q());
      return with_team(team, [&](auto lanes) {
        const int teams = ms::kMeanNT / team;
        const int span_blocks = edges > 0 ? (int)cdiv(p.spans, teams) : 0;
        // rows that nobody lists: a few turns a block
        const int64_t blocks = span_blocks + std::min<int64_t>(cdiv(b->rows, 4 * teams), 8192);
        const int rc = launch(what, add_rows > 0 ? ms::k_block_mean_backward<D, q(), lanes(), true> : ms::k_block_mean_backward<D, q(), lanes(), false>,
                              blocks, ms::kMeanNT, 0, stream, keys[at], vals[at], shares, marks, edges, rows, (const D*)dout, dout_stride, d,
                              (const D*)add, add_stride, (int32_t)add_rows, (D*)dx, dx_stride, partial, p.span, span_blocks);
        if (rc || edges <= p.span) return rc;
        return launch(what, ms::k_block_mean_join<D, q(), lanes()>, cdiv(p.spans, teams), ms::kMeanNT, 0, stream, keys[at],
                      edges, rows, d, p.span, partial, (D*)dx, dx_stride);
      });
    });
  });
}

// ------------------------------------------------------------------- linear
constexpr int64_t kMostRows = int64_t(1) << 29;

template <typename T>
ms::Operand<T> operand(const void* p, int64_t stride, int64_t R, int64_t K, const void* pre = nullptr, int64_t pre_stride = 0,
                       int act = MASSIVE_ACT_NONE) {
  return ms::Operand<T>{(const T*)p, (const T*)pre, stride, pre_stride, R, K, act};
}

int check_layer(int64_t rows, int32_t n, int32_t k, int32_t k_second, int32_t type, int32_t act, const void* x_second) {
  if (!is_type(type)) REFUSE("type must be MASSIVE_F32 or MASSIVE_BF16");
  if (act < MASSIVE_ACT_NONE || act > MASSIVE_ACT_SILU) REFUSE("act is not one of MASSIVE_ACT_*");
  if (rows < 0 || rows > kMostRows) REFUSE("rows must be in 0..2^29");
  if (n < 1 || k < 1 || k_second < 0 || n > (1 << 20) || k > (1 << 20) || k_second > (1 << 20))
    REFUSE("n and k must be in 1..2^20, k_second in 0..2^20");
  if ((k_second > 0) != (x_second != nullptr) && rows > 0) REFUSE("k_second columns and x_second go together");
  return MASSIVE_OK;
}

// The streaming form's shape for n outputs from `chunks` chunks of k: blocks of
// 32 outputs that a wave accumulates, and whether their weights stay in LDS. As
// many as there are outputs, unless fewer give more of the chip's 256 CUs work;
// eight (WIDE) only in bf16 without a slope, where the accumulators and the rows
// on their way fit the registers and the matrix unit does not set the pace (240K
// rows, 64 + 64 -> 256 in bf16: 64 us with eight, 72 with four).
struct StreamPlan {
  int nb;
  bool resident;
  int lds_weights, lds;
};
template <bool WIDE>
StreamPlan stream_plan(int64_t rows, int64_t n, int64_t chunks) {
  StreamPlan p;
  auto bytes = [&](int nb) { return chunks * nb * ms::kStreamBlockBytes; };
  p.nb = n <= 32 ? 1 : n <= 64 ? 2 : n <= 128 || !WIDE || bytes(8) > ms::kStreamLds ? 4 : 8;
  while (p.nb > 2 && cdiv(rows, ms::kStreamRows) * cdiv(n, p.nb * 32) < 256) p.nb /= 2;
  p.resident = bytes(p.nb) <= ms::kStreamLds;
  p.lds_weights = (int)(p.resident ? bytes(p.nb) : 2 * p.nb * ms::kStreamBlockBytes);
  p.lds = p.lds_weights + ms::kStreamNT / MS_WAVE * ms::kStreamTurn + p.nb * 32 * 4;  // weights, turns, bias
  return p;
}
// Blocks: every CU's share once, in whole rounds of the output groups on the
// eight XCDs.
int64_t stream_blocks(const StreamPlan& p, int64_t rows, int groups) {
  const int64_t per_cu = p.lds <= (80 << 10) ? 2 : 1;
  const int64_t most = std::max<int64_t>(1, 256 * per_cu / 8 / groups) * groups * 8;
  return std::min(most, round_up(cdiv(rows, ms::kStreamRows), 8) * groups);
}

// f(blocks of 32 outputs, whether they stay), both as types.
template <bool WIDE, typename F>
int with_stream(const StreamPlan& p, F f) {
  using std::integral_constant;
  if constexpr (WIDE)
    if (p.nb == 8) return f(integral_constant<int, 8>(), std::true_type());
  if (p.nb == 4) return p.resident ? f(integral_constant<int, 4>(), std::true_type()) : f(integral_constant<int, 4>(), std::false_type());
  if (p.nb == 2) return p.resident ? f(integral_constant<int, 2>(), std::true_type()) : f(integral_constant<int, 2>(), std::false_type());
  return p.resident ? f(integral_constant<int, 1>(), std::true_type()) : f(integral_constant<int, 1>(), std::false_type());
}

// Whether a product of rows x cols results streams its rows: from about 2^21
// results on (dx in bf16: 2^20). Below, both forms take about as long as a
// launch, and the form for few rows has more blocks; above, it reads its
// operands too often. Measured, us, few rows' form / streaming, 256 -> 256: bf16
// 4000 rows 11 / 20, 8000 21 / 20, 16000 41 / 21; fp32 8000 39 / 44, 16000
// 75 / 46. dx in bf16, whose few rows read weights across: 2000 rows 9.8 / 10.1,
// 4000 15 / 10, 8000 22 / 11, and with gelu's slope 16 / 21, 27 / 21, 47 / 22.
bool streams(int64_t rows, int64_t cols, int log2_least) { return rows * round_up(cols, 32) >= int64_t(1) << log2_least; }

template <typename T>
int linear(const massive_linear_args* a, void* stream) {
  ms::LinearForward<T> f;
  const int64_t k = a->k;
  f.x[0] = operand<T>(a->x, a->x_stride, a->rows, k);
  f.x[1] = operand<T>(a->x_second, a->x_second_stride, a->rows, a->k_second);
  f.w[0] = {(const T*)a->w, a->w_stride};
  f.w[1] = {(const T*)a->w + k, a->w_stride};
  f.bias = (const T*)a->bias;
  f.residual = (const T*)a->residual;
  f.y = (T*)a->y;
  f.pre = (T*)a->pre;
  f.residual_stride = a->residual_stride;
  f.y_stride = a->y_stride;
  f.pre_stride = a->pre_stride;
  f.rows = a->rows;
  f.n = a->n;
  f.act = a->act;
  if (streams(a->rows, a->n, 21)) {
    constexpr bool kWide = sizeof(T) == 2;
    const StreamPlan p = stream_plan<kWide>(a->rows, a->n, cdiv(a->k * sizeof(T), 256) + cdiv(a->k_second * sizeof(T), 256));
    const int groups = (int)cdiv(a->n, p.nb * 32);
    return with_stream<kWide>(p, [&](auto nb, auto resident) {
      return launch("massive_linear", ms::k_linear_stream<T, nb(), resident()>, stream_blocks(p, a->rows, groups), ms::kStreamNT, p.lds,
                    stream, f, groups, p.lds_weights);
    });
  }
  const int tiles_n = (int)cdiv(a->n, 32);
  const int64_t blocks = cdiv(a->rows, 32) * tiles_n;  // under 2^16: more are streamed
  return launch("massive_linear", ms::k_linear_few<T>, blocks, ms::kFewNT, 0, stream, f, tiles_n);
}

// dw's tiles, outputs by columns of both inputs (each input's in whole vectors),
// and the parts into which its rows are split. The tile is the one that
// multiplies the fewest zeros; of equal ones the square one, which reads least.
// (256 by 128 read x fewer times and left room for half the waves: the dw of
// 110K x 1024 by 128 with gelu's slope 165 us with it, 145 with 128 by 128.)
// Enough parts for the chip, none of less than four steps of rows where there
// are more. dbias alone is tiles of 128 outputs, without columns.
struct DwPlan {
  int bn, bk, second;
  int64_t tiles_n, tiles_k, part, parts, dw_floats, bytes;
  int64_t blocks, join_blocks;
};
DwPlan dw_plan(const massive_linear_grads* a) {
  DwPlan p = {};
  const int vector = 16 / size_of(a->type), step = 64 / size_of(a->type);
  p.second = (int)round_up(a->k, vector);
  const int64_t cols = p.second + a->k_second;
  int64_t least = 0;
  for (const auto& t : {std::pair<int, int>(128, 128), std::pair<int, int>(64, 256)}) {
    const int64_t area = round_up(a->n, t.first) * round_up(cols, t.second);
    if (!p.bn || area < least) {
      least = area;
      p.bn = t.first;
      p.bk = t.second;
    }
  }
  p.tiles_n = cdiv(a->n, p.bn);
  p.tiles_k = cdiv(cols, p.bk);
  if (!a->dw) {
    p.bn = p.bk = 128;
    p.tiles_n = cdiv(a->n, p.bn);
    p.tiles_k = 1;
  }
  const int64_t most = std::max<int64_t>(1, cdiv(a->rows, 4 * step));
  p.part = round_up(cdiv(a->rows, std::min(most, std::max<int64_t>(1, 512 / (p.tiles_n * p.tiles_k)))), step);
  p.parts = cdiv(a->rows, p.part);
  p.dw_floats = a->dw ? p.parts * a->n * ((int64_t)a->k + a->k_second) : 0;
  p.bytes = 4 * (round_up(p.dw_floats, 4) + (a->dbias ? p.parts * a->n : 0));
  p.blocks = p.parts * p.tiles_n * p.tiles_k;
  const int64_t values = (int64_t)a->n * ((a->dw ? (int64_t)a->k + a->k_second : 0) + (a->dbias ? 1 : 0));
  p.join_blocks = cdiv(values, ms::kLinNT / ms::kJoinWays);
  return p;
}

int check_grads(const massive_linear_grads* a) {
  if (!a) REFUSE("args is NULL");
  return check_layer(a->rows, a->n, a->k, a->k_second, a->type, a->act, a->x_second);
}

template <typename T>
int linear_backward(const massive_linear_grads* a, void* workspace, void* stream) {
  const bool slope = a->act != MASSIVE_ACT_NONE;
  const int64_t k[2] = {a->k, a->k_second};
  if (a->dx || a->dx_second) {
    ms::LinearDx<T> f;
    f.dz = operand<T>(a->dy, a->dy_stride, a->rows, a->n, a->pre, a->pre_stride, a->act);
    const int k0 = a->dx ? a->k : 0, k1 = a->dx_second ? a->k_second : 0;
    f.w = {(const T*)a->w + (a->dx ? 0 : k[0]), a->w_stride};
    f.dx[0] = (T*)a->dx;
    f.dx[1] = (T*)a->dx_second;
    f.dx_stride[0] = a->dx_stride;
    f.dx_stride[1] = a->dx_second_stride;
    f.rows = a->rows;
    f.cols = k0 + k1;
    f.split = k0;
    int rc;
    if (streams(a->rows, f.cols, sizeof(T) == 2 ? 20 : 21)) {
      auto stream_with = [&](auto with_slope) {
        constexpr bool kWide = sizeof(T) == 2 && !with_slope();
        const StreamPlan p = stream_plan<kWide>(a->rows, f.cols, cdiv(a->n * sizeof(T), 256));
        const int groups = (int)cdiv(f.cols, p.nb * 32);
        return with_stream<kWide>(p, [&](auto nb, auto resident) {
          return launch("massive_linear_backward", ms::k_linear_dx_stream<T, with_slope(), nb(), resident()>, stream_blocks(p, a->rows, groups),
                        ms::kStreamNT, p.lds, stream, f, groups, p.lds_weights);
        });
      };
      rc = slope ? stream_with(std::true_type()) : stream_with(std::false_type());
    } else {
      const int tiles_n = (int)cdiv(f.cols, 32);
      const int64_t blocks = cdiv(a->rows, 32) * tiles_n;  // under 2^16: more are streamed
      rc = launch("massive_linear_backward", slope ? ms::k_linear_dx_few<T, true> : ms::k_linear_dx_few<T, false>, blocks, ms::kFewNT, 0, stream, f, tiles_n);
    }
    if (rc) return rc;
  }
  if (!a->dw && !a->dbias) return MASSIVE_OK;
  const DwPlan p = dw_plan(a);
  ms::LinearDw<T> f;
  f.dz = operand<T>(a->dy, a->dy_stride, a->rows, a->n, a->pre, a->pre_stride, a->act);
  f.x[0] = operand<T>(a->x, a->x_stride, a->rows, k[0]);
  f.x[1] = operand<T>(a->x_second, a->x_second_stride, a->rows, k[1]);
  f.dw = a->dw ? (float*)workspace : nullptr;
  f.dbias = a->dbias ? (float*)workspace + round_up(p.dw_floats, 4) : nullptr;
  f.rows = a->rows;
  f.part = p.part;
  f.n = a->n;
  f.k[0] = a->k;
  f.k[1] = a->k_second;
  f.second = p.second;
  f.tiles_n = (int)p.tiles_n;
  f.tiles_k = (int)p.tiles_k;
  auto go = [&](auto bn, auto bk, auto dw) {
    return launch("massive_linear_backward", slope ? ms::k_linear_dw<T, true, bn(), bk(), dw()> : ms::k_linear_dw<T, false, bn(), bk(), dw()>, p.blocks,
                  ms::kDwNT, 0, stream, f, p.blocks);
  };
  using std::integral_constant;
  const int rc = !a->dw        ? go(integral_constant<int, 128>(), integral_constant<int, 128>(), std::false_type())
                 : p.bn == 128 ? go(integral_constant<int, 128>(), integral_constant<int, 128>(), std::true_type())
                               : go(integral_constant<int, 64>(), integral_constant<int, 256>(), std::true_type());
  if (rc) return rc;
  return launch("massive_linear_backward", ms::k_linear_join<T>, p.join_blocks, ms::kLinNT, 0,
                stream, (const float*)f.dw, (const float*)f.dbias, p.parts, a->n, (int)(k[0] + k[1]), (T*)a->dw, a->dw_stride,
                (T*)a->dbias);
}

// -------------------------------------------------------------------- AdamW
int adamw(const massive_adamw_tensor* tensors, int64_t count, const massive_adamw_args* a, void* stream) {
  if (!a) REFUSE("args is NULL");
  if (count < 0 || (count > 0 && !tensors)) REFUSE("tensors is NULL or count negative");
  if (a->state_bits != 32 && a->state_bits != 8) REFUSE("state_bits must be 32 or 8");
  if (!is_type(a->param_type) || !is_type(a->grad_type)) REFUSE("param_type and grad_type must be MASSIVE_F32 or MASSIVE_BF16");
  if (a->t < 1) REFUSE("t counts steps from 1");
  if (a->reserved != 0) REFUSE("reserved must be 0");
  if (!(a->beta_first >= 0 && a->beta_first < 1 && a->beta_second >= 0 && a->beta_second < 1))
    REFUSE("the betas must be in [0, 1)");
  if (!(a->lr >= 0 && a->eps >= 0 && a->weight_decay >= 0) || !std::isfinite(a->lr) || !std::isfinite(a->eps) ||
      !std::isfinite(a->weight_decay))
    REFUSE("lr, eps and weight_decay must be finite and not negative");
  const bool eight = a->state_bits == 8;
  for (int64_t i = 0; i < count; ++i) {
    const massive_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > kMostBlocks * ms::kAdamwBlock / 2) REFUSE("tensor %lld: n must be in 0..2^34", (long long)i);
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v) REFUSE("tensor %lld: param, grad, m or v is NULL", (long long)i);
    if (eight != (t.m_scale && t.v_scale) || (!eight && (t.m_scale || t.v_scale)))
      REFUSE("tensor %lld: states of 8 bits have scales, of 32 bits none", (long long)i);
    if (!aligned(t.param, size_of(a->param_type)) || !aligned(t.grad, size_of(a->grad_type)) || !aligned(t.copy, 2) ||
        !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4) || (!eight && (!aligned(t.m, 4) || !aligned(t.v, 4))))
      REFUSE("tensor %lld: an array is not aligned", (long long)i);
  }
  ms::AdamwLaunch l;
  l.decay = (float)(1.0 - a->lr * a->weight_decay);
  l.b1 = (float)a->beta_first;
  l.b1c = (float)(1.0 - a->beta_first);
  l.b2 = (float)a->beta_second;
  l.b2c = (float)(1.0 - a->beta_second);
  l.lr = (float)(a->lr / (1.0 - std::pow(a->beta_first, (double)a->t)));
  l.v_factor = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta_second, (double)a->t)));
  // the least normal number stands for all below it: the device divides by
  // normal numbers, and beside the root of any v that fp32 holds neither counts
  l.eps = a->eps > 0 ? std::max((float)a->eps, std::numeric_limits<float>::min()) : 0.0f;
  for (int64_t i = 0; i < count;) {
    l.count = 0;
    int64_t blocks = 0;
    for (; i < count && l.count < ms::kAdamwTensors; ++i) {
      const massive_adamw_tensor& t = tensors[i];
      if (t.n == 0) continue;
      const int64_t more = cdiv(t.n, ms::kAdamwBlock);
      if (l.count > 0 && blocks + more > kMostBlocks) break;
      l.t[l.count] = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, (bf16*)t.copy, t.n};
      l.first[l.count++] = (int32_t)blocks;
      blocks += more;
    }
    if (l.count == 0) break;
    l.first[l.count] = (int32_t)blocks;
    const int rc = with_type(a->param_type, [&](auto* p) {
      using P = std::remove_pointer_t<decltype(p)>;
      return with_type(a->grad_type, [&](auto* g) {
        using G = std::remove_pointer_t<decltype(g)>;
        return eight ? launch("massive_adamw", ms::k_adamw<P, G, 8>, blocks, ms::kAdamwNT, 0, stream, l)
                     : launch("massive_adamw", ms::k_adamw<P, G, 32>, blocks, ms::kAdamwNT, 0, stream, l);
      });
    });
    if (rc) return rc;
  }
  return MASSIVE_OK;
}

}  // namespace

extern "C" {

int massive_row_layout(const massive_row_format* fmt, int64_t* row_bytes, int64_t* floats_at) {
  ms::PackedRows f;
  int64_t least;
  if (int rc = check_format(fmt, &f, &least)) return rc;
  if (row_bytes) *row_bytes = least;
  if (floats_at) *floats_at = f.floats_at;
  return MASSIVE_OK;
}

int massive_pack_rows(const massive_row_format* fmt, const void* src, int32_t src_type, int64_t src_stride, int64_t n,
                      const int32_t* slots, void* table, int64_t table_rows, void* stream) {
  return pack_rows(fmt, src, src_type, src_stride, n, slots, table, table_rows, stream);
}

int massive_unpack_rows(const massive_row_format* fmt, const void* table, int64_t table_rows, const int32_t* index, int64_t n,
                        void* out, int32_t out_type, int64_t out_stride, void* stream) {
  return unpack_rows(fmt, table, table_rows, index, n, out, out_type, out_stride, stream);
}

int massive_block_mean(const massive_block* block, const void* x, int32_t x_type, int64_t x_stride,
                       const massive_row_format* fmt, int32_t d, void* out, int32_t out_type, int64_t out_stride, void* stream) {
  return block_mean(block, x, x_type, x_stride, fmt, d, out, out_type, out_stride, stream);
}

int massive_block_mean_workspace(const massive_block* block, int32_t d, int64_t* bytes) {
  if (!bytes) REFUSE("bytes is NULL");
  if (int rc = check_block(block)) return rc;
  if (d < 1) REFUSE("d must be at least 1");
  *bytes = few(block) ? 0 : mean_plan(block, d).bytes;
  return MASSIVE_OK;
}

int massive_block_mean_backward(const massive_block* block, const void* dout, int32_t type, int64_t dout_stride, int32_t d,
                                const void* add, int64_t add_stride, int64_t add_rows, void* dx, int64_t dx_stride,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  return block_mean_backward(block, dout, type, dout_stride, d, add, add_stride, add_rows, dx, dx_stride, workspace,
                             workspace_bytes, stream);
}

int massive_linear(const massive_linear_args* a, void* stream) {
  if (!a) REFUSE("args is NULL");
  if (int rc = check_layer(a->rows, a->n, a->k, a->k_second, a->type, a->act, a->x_second)) return rc;
  if (a->rows == 0) return MASSIVE_OK;
  if (!a->x || !a->w || !a->y) REFUSE("x / w / y are NULL");
  if (a->x_stride < a->k || (a->x_second && a->x_second_stride < a->k_second) ||
      a->w_stride < (int64_t)a->k + a->k_second || a->y_stride < a->n || (a->residual && a->residual_stride < a->n) ||
      (a->pre && a->pre_stride < a->n))
    REFUSE("a stride is below its rows' length");
  const int size = size_of(a->type);
  for (const void* p : {a->x, a->x_second, a->w, a->bias, a->residual, (const void*)a->y, (const void*)a->pre})
    if (!aligned(p, size)) REFUSE("an array is not aligned");
  return a->type == MASSIVE_F32 ? linear<float>(a, stream) : linear<bf16>(a, stream);
}

int massive_linear_workspace(const massive_linear_grads* a, int64_t* bytes) {
  if (!bytes) REFUSE("bytes is NULL");
  if (int rc = check_grads(a)) return rc;
  *bytes = a->rows == 0 || (!a->dw && !a->dbias) ? 0 : dw_plan(a).bytes;
  return MASSIVE_OK;
}

int massive_linear_backward(const massive_linear_grads* a, void* workspace, int64_t workspace_bytes, void* stream) {
  if (int rc = check_grads(a)) return rc;
  const bool dz = a->dx || a->dx_second || a->dw || a->dbias;
  if (!dz) return MASSIVE_OK;
  if (a->dx_second && !a->k_second) REFUSE("dx_second without a second input");
  const int64_t k = (int64_t)a->k + a->k_second;
  if (a->dw && a->dw_stride < k) REFUSE("a stride is below its rows' length");
  if (a->rows > 0) {
    if (!a->dy || (a->act != MASSIVE_ACT_NONE && !a->pre)) REFUSE("dy / pre are NULL");
    if ((a->dx || a->dx_second) && !a->w) REFUSE("w is NULL");
    if (a->dw && !a->x) REFUSE("x is NULL");
    if (a->dy_stride < a->n || (a->act != MASSIVE_ACT_NONE && a->pre_stride < a->n) || (a->x && a->x_stride < a->k) ||
        (a->x_second && a->x_second_stride < a->k_second) || (a->w && a->w_stride < k) || (a->dx && a->dx_stride < a->k) ||
        (a->dx_second && a->dx_second_stride < a->k_second))
      REFUSE("a stride is below its rows' length");
  }
  const int size = size_of(a->type);
  for (const void* p : {a->dy, a->pre, a->x, a->x_second, a->w, (const void*)a->dx, (const void*)a->dx_second,
                        (const void*)a->dw, (const void*)a->dbias})
    if (!aligned(p, size)) REFUSE("an array is not aligned");
  if (a->rows == 0) {  // sums over no rows
    const int64_t values = (int64_t)a->n * ((a->dw ? k : 0) + (a->dbias ? 1 : 0));
    if (values == 0) return MASSIVE_OK;
    const int64_t blocks = cdiv(values, ms::kLinNT / ms::kJoinWays);
    if (blocks > kMostBlocks) REFUSE("too many columns for one call");
    // the pointers only say which of the two are asked for: with no parts nothing is read
    const float *dw = (const float*)a->dw, *db = (const float*)a->dbias;
    return a->type == MASSIVE_F32
               ? launch("massive_linear_backward", ms::k_linear_join<float>, blocks, ms::kLinNT, 0, stream, dw, db, int64_t(0),
                        a->n, (int)k, (float*)a->dw, a->dw_stride, (float*)a->dbias)
               : launch("massive_linear_backward", ms::k_linear_join<bf16>, blocks, ms::kLinNT, 0, stream, dw, db, int64_t(0),
                        a->n, (int)k, (bf16*)a->dw, a->dw_stride, (bf16*)a->dbias);
  }
  if (a->dw || a->dbias) {
    const DwPlan p = dw_plan(a);
    if (p.blocks > kMostBlocks / 2 || p.join_blocks > kMostBlocks) REFUSE("too many rows and columns for one call");
    if (!workspace || workspace_bytes < p.bytes)
      return call_error(MASSIVE_ECAPACITY, "workspace of %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0),
                        (long long)p.bytes);
    if (!aligned(workspace, 16)) REFUSE("workspace is not 16-byte aligned");
  }
  return a->type == MASSIVE_F32 ? linear_backward<float>(a, workspace, stream) : linear_backward<bf16>(a, workspace, stream);
}

int massive_adamw(const massive_adamw_tensor* tensors, int64_t count, const massive_adamw_args* args, void* stream) {
  return adamw(tensors, count, args, stream);
}

int massive_adamw_states(const void* m, const void* v, const float* m_scale, const float* v_scale, int64_t n, float* m_out,
                         float* v_out, void* stream) {
  if (n < 0) REFUSE("n must not be negative");
  if (n == 0) return MASSIVE_OK;
  if (!m || !v || !m_scale || !v_scale || !m_out || !v_out) REFUSE("an array is NULL");
  if (!aligned(m_scale, 4) || !aligned(v_scale, 4) || !aligned(m_out, 4) || !aligned(v_out, 4)) REFUSE("an array is not aligned");
  return launch("massive_adamw_states", ms::k_adamw_states, std::min(cdiv(n, ms::kAdamwNT * ms::kAdamwQ), kMostBlocks),
                ms::kAdamwNT, 0, stream, (const int8_t*)m, (const uint8_t*)v, m_scale, v_scale, n, m_out, v_out);
}

}  // extern "C"
