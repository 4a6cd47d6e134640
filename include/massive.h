/*
 * massive.h - C ABI of libmassive: one graph partition's per-minibatch
 * sampling + halo prefetch buffer + feature gather, after MassiveGNN
 * (Sarkar, Ghosh, Tallent, Jannesari, arXiv 2410.22697), on one MI355X.
 *
 * The three calls follow the paper's procedures:
 *   massive_init        INITIALIZE_PREFETCHER (Algorithm 1)
 *   massive_sample      PREFETCH_WITH_EVICTION up to the eviction check
 *                       (Algorithm 2: NeighborSampler, hit/miss split, S_E
 *                       decay, local/buffer copies, miss fetch, S_A update)
 *   massive_evict_step  the periodic round of Algorithm 2 (EVICT_AND_REPLACE
 *                       with the score swap of Section IV-B, threshold Eq. 1)
 *
 * Ids. The partition's nodes carry partition-local ids: local (owned)
 * nodes [0, L), halo (remote) nodes [L, L+H). The prefetcher's state and the
 * eviction outputs use halo indices h = id - L in [0, H).
 *
 * Semantics (readings of the paper, fixed so that results are exact):
 *   - The sampler walks G_p, the CSR of the subgraph induced on local + halo
 *     nodes. Fanouts are hop-first. Hop k (1-based) samples for every node
 *     of frontier F_{k-1}; new nodes are appended in ascending id, so F_k is
 *     a prefix of F_{k+1} and the seeds come first.
 *   - For a row v of length d at global step t, hop k: if d <= fanout every
 *     position is kept; otherwise the fanout positions j with the smallest
 *     (key_j, j), where key_j is word (j mod 4) of Philox4x32-10 (Salmon et
 *     al., SC'11) with counter (j/4, v, t, k) and key (seed_lo, seed_hi).
 *     Sampled neighbours are emitted in ascending j.
 *   - Halo rank orders halo nodes by (degree desc, global id asc); the
 *     buffer starts with the cap = floor(H * buffer_pct / 100) best ranked.
 *   - Hits/misses use the buffer as it stood at the start of the step.
 *     Every step: S_E *= gamma (fp32, one product per step) for each
 *     buffered node not sampled; S_A += 1 for each miss.
 *   - t counts steps across epochs from 0. After step t, if t > 0 and
 *     t mod delta == 0, the round evicts the slots with S_E < alpha, where
 *     alpha is gamma multiplied delta times in fp32, and replaces them with
 *     the unbuffered halo nodes of highest (S_A, then rank); evicted slots
 *     in ascending order are paired with replacements in that order. If
 *     there are fewer candidates k' than evictions, the k' slots with the
 *     smallest (S_E, rank) are evicted. Swap: evicted node's S_A := its last
 *     S_E, slot's S_E := the replacement's last S_A, replacement's S_A := -1.
 *
 * Threading: calls on one context must not overlap. Different contexts are
 * independent. A context in MASSIVE_LINK_STAGED mode runs host threads of
 * its own, which end in massive_destroy. Every call returns a status;
 * nothing throws across the ABI.
 */
#ifndef MASSIVE_H
#define MASSIVE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* status codes */
#define MASSIVE_OK 0
#define MASSIVE_EINVAL (-1)    /* bad argument (message in massive_last_error) */
#define MASSIVE_ECAPACITY (-2) /* an output buffer is smaller than the bound  */
#define MASSIVE_ENOMEM (-3)    /* device or host allocation failed            */
#define MASSIVE_EHIP (-4)      /* HIP runtime error; from a step or a round, the
                                  context then takes no further work         */
#define MASSIVE_ESTATE (-5)    /* call out of order (see massive_sample)      */

#define MASSIVE_MAX_HOPS 8

/* S_A layouts (massive_init_args.score_layout), the two the paper weighs in
 * Section IV-B: an array over the halo only, or one over every global id */
#define MASSIVE_SCORES_BY_RANK 0 /* S_A over the H halo nodes, in rank order */
#define MASSIVE_SCORES_BY_GID 1  /* S_A over all n_global global ids, indexed by id */
#define MASSIVE_MAX_INFLIGHT 3 /* batches enqueued and not yet waited for */

/* How rows cross the host link (massive_init_args.link_mode): the misses,
 * hits on slots still refilling, and the replacement rows of Algorithm 2's
 * merged fetch. Both modes give the same results. */
#define MASSIVE_LINK_LOADS 0  /* kernels read the mapped pinned store */
#define MASSIVE_LINK_STAGED 1 /* host threads gather the rows into pinned
                                 staging memory, the DMA engines copy them to
                                 the device and a kernel scatters them; no
                                 kernel reads host memory, so kernels running
                                 beside the path (a trainer) are not slowed */

typedef struct massive_ctx massive_ctx;

/* Inputs of massive_init. Every host array is read during the call only,
 * except halo_store, which the context borrows until massive_destroy. */
typedef struct {
  int32_t L;                  /* local nodes, ids [0, L)                      */
  int32_t H;                  /* halo nodes, ids [L, L+H)                      */
  const int64_t* indptr;      /* host [L+H+1], G_p row offsets (int64)        */
  const int32_t* indices;     /* host [indptr[L+H]], partition-local ids      */
  const int32_t* halo_gid;    /* host [H], global id of halo h (rank ties)    */
  const int64_t* halo_degree; /* host [H], degree used to rank halo nodes     */
  const void* local_feat;     /* host [L * row_bytes], copied into HBM        */
  const void* halo_store;     /* PINNED host [H * row_bytes] (hipHostMalloc'd,
                                 e.g. a torch pin_memory tensor): the remote
                                 features; read by the GPU over the host link */
  int64_t row_bytes;          /* bytes per feature row, multiple of 4, <= 1 MiB */
  int32_t K;                  /* hops, 1..MASSIVE_MAX_HOPS                     */
  int32_t fanout[MASSIVE_MAX_HOPS]; /* hop-first fanouts, each >= 1           */
  int32_t buffer_pct;         /* f_p^h as an integer percent, 0..100          */
  float gamma;                /* decay factor, 0 < gamma <= 1                 */
  int32_t delta;              /* eviction interval, >= 1                      */
  uint64_t seed;              /* Philox key                                   */
  void* stream;               /* hipStream_t for all work (NULL: default)     */
  int32_t score_layout;       /* MASSIVE_SCORES_BY_RANK (0, the default) or
                                 MASSIVE_SCORES_BY_GID: S_A (and a rank per
                                 id) over every global id, 8 B per id; the
                                 eviction round then selects over all ids  */
  int64_t n_global;           /* MASSIVE_SCORES_BY_GID: the global id space,
                                 every halo_gid in [0, n_global) and distinct,
                                 n_global <= 2^31; ignored otherwise         */
  int32_t link_mode;          /* MASSIVE_LINK_LOADS (0, the default) or
                                 MASSIVE_LINK_STAGED                          */
  int32_t link_threads;       /* MASSIVE_LINK_STAGED: host threads gathering
                                 rows, 1..64 (0: 8); the context starts them
                                 and one more that feeds the copies          */
} massive_init_args;

/* Creates a context: uploads G_p and local features to HBM, ranks the halo,
 * fills the HBM buffer with the cap best-ranked halo rows from halo_store,
 * and sets S_E = 1, S_A = -1 / 0. Both score layouts give the same results
 * (states, eviction and replacement sets); they differ in memory and in the
 * eviction round's time. MASSIVE_EINVAL for a halo_gid outside [0, n_global)
 * or repeated (BY_GID). On failure *out is NULL and the message is in
 * massive_last_error(NULL). */
int massive_init(const massive_init_args* args, massive_ctx** out);

/* Upper bounds on the output sizes of a batch of n_seeds seeds:
 * n_bound[0..K] frontier sizes, e_bound[0..K-1] sampled edges per hop. */
int massive_output_bounds(const massive_ctx* ctx, int32_t n_seeds, int64_t* n_bound,
                          int64_t* e_bound);

/* Caller-owned device buffers of one batch, plus the sizes written back.
 * Capacities are in elements; each must be at least the bound above. */
typedef struct {
  int32_t* nodes;                          /* [nodes_cap] F_K; F_k = nodes[0:n[k]] */
  uint8_t* mask;                           /* [nodes_cap] 0 local, 1 hit, 2 miss   */
  void* feat;                              /* [nodes_cap * row_bytes], row i is the
                                              feature row of nodes[i]             */
  int64_t nodes_cap;
  /* entry k (0-based) is the block of hop k+1, which samples for the n[k]
   * rows of F_k: indptr[k] has n[k]+1 offsets into indices[k], and
   * indices[k] holds e[k] sampled neighbours as positions in nodes */
  int32_t* indptr[MASSIVE_MAX_HOPS];
  int32_t* indices[MASSIVE_MAX_HOPS];
  int64_t indptr_cap[MASSIVE_MAX_HOPS];
  int64_t indices_cap[MASSIVE_MAX_HOPS];
  /* written by massive_sample */
  int64_t n[MASSIVE_MAX_HOPS + 1];         /* frontier sizes n_0..n_K              */
  int64_t e[MASSIVE_MAX_HOPS];             /* sampled edges per hop                */
  int64_t local, hits, misses;             /* input rows by class (unique nodes)   */
  int64_t host_rows;                       /* rows read over the host link: the
                                              misses, plus hits on slots whose
                                              refill had not landed yet        */
} massive_batch;

/* One minibatch at the context's current step t: samples K hops from the
 * n_seeds device seeds (distinct local ids), classifies every frontier node
 * against the buffer, updates the scores and gathers all feature rows (HBM
 * rows from the local slab and the buffer, misses from halo_store). Returns
 * after the batch is complete on the device (massive_sample_async followed by
 * massive_batch_wait); t advances by one.
 * MASSIVE_ESTATE if the previous step's massive_evict_step was not called.
 * MASSIVE_EINVAL (no state change) if a seed is out of [0, L) or repeated. */
int massive_sample(massive_ctx* ctx, const int32_t* seeds, int32_t n_seeds, massive_batch* io);

/* massive_sample for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same step and the same results, but its per-step scratch (sizes, gather
 * lists, scan flags) lives in one static device array per GPU, of fixed size,
 * instead of the context's per-slot buffers, and the call itself allocates
 * nothing (no hipMalloc, no event creation; timing is off for it). Limit:
 * frontier bound n_bound[K] <= 1,310,720 rows; a larger bound is refused with
 * MASSIVE_ECAPACITY. Synchronous, and refused (MASSIVE_ESTATE) while a batch
 * of this context is in flight. Calls that overlap on one GPU, from any
 * contexts, race on that array: serialise them. */
int massive_sample_noalloc(massive_ctx* ctx, const int32_t* seeds, int32_t n_seeds, massive_batch* io);

/* The asynchronous form of massive_sample, for look-ahead (Algorithm 1
 * prepares the next minibatch while the current one is consumed): enqueues
 * the step and returns at once. The batch's buffers must not be read or
 * reused, and its sizes are not written, until massive_batch_wait returns for
 * it. At most MASSIVE_MAX_INFLIGHT batches are in flight: the next steps can
 * be enqueued (each after its predecessor's massive_evict_step) while earlier
 * ones still read misses over the host link; a further one is refused with
 * MASSIVE_ESTATE. Argument errors are returned here; seed errors
 * are returned by massive_batch_wait (if a later step was already issued the
 * context then refuses further work with MASSIVE_ESTATE). */
int massive_sample_async(massive_ctx* ctx, const int32_t* seeds, int32_t n_seeds, massive_batch* io);

/* Waits for the batch enqueued with io and writes its sizes and counters.
 * MASSIVE_EINVAL for a seed out of [0, L) or repeated (the step is taken
 * back if no later step was issued); MASSIVE_EHIP, and the context refuses
 * further work, if the sampler's threshold search found no acceptable
 * candidate count or a single-pass scan waited past its bound (neither is
 * expected), or if an eviction round produced inconsistent indices.
 * MASSIVE_ESTATE for a batch issued after a step that failed in any of these
 * ways (whichever of the two is waited for first): it was sampled against the
 * failed step's leftover state, so its outputs are not valid. */
int massive_batch_wait(massive_ctx* ctx, massive_batch* io);

/* The eviction round owed by the step just sampled; must be called once after
 * every massive_sample / massive_sample_async. Runs the round iff that step t
 * has t > 0 and t mod delta == 0. The round is decided on the device, on the
 * library's copy stream, beside the next step's sampling (that step's lookup
 * waits for it): with k_out == NULL the call only enqueues it; otherwise it
 * waits for the round and writes k' (0 when no round is due). Optional device
 * outputs, each with room for cap entries: evicted halo ids, the slots they
 * held (ascending), and their replacements (entries [0, k')); they are
 * complete when the call returns with k_out, or once the next step's
 * massive_batch_wait has returned. The replacement rows are copied from
 * halo_store on the copy stream; until they have landed, the next steps read
 * hits on those slots from halo_store (the same bytes) and write them into
 * their slots, so that no row crosses the host link twice. */
int massive_evict_step(massive_ctx* ctx, int32_t* evicted, int32_t* slots, int32_t* replaced,
                       int64_t* k_out);

/* Totals since init (each pointer may be NULL): rounds that evicted at least
 * one slot, slots evicted, and rows the refill copied over the host link
 * (including the initial fill of the buffer; a replacement whose row a miss
 * gather already wrote into its slot is not copied again). Waits for the
 * refill chunks launched so far. */
int massive_get_counters(massive_ctx* ctx, int64_t* rounds, int64_t* evicted, int64_t* refilled);

/* Host copies of the prefetcher state (each pointer may be NULL):
 * slot_id[cap] halo id per slot, S_E[cap], S_A[H], steps sampled so far. */
int massive_get_state(massive_ctx* ctx, int32_t* slot_id, float* S_E, float* S_A, int64_t* t);

/* Host copy of the HBM buffer's rows, [cap * row_bytes]. */
int massive_get_buffer_rows(massive_ctx* ctx, void* host_out);

/* cap (buffer slots) and alpha (each pointer may be NULL). */
int massive_info(const massive_ctx* ctx, int64_t* cap, float* alpha);

/* Per-kernel-group timing with HIP events recorded on the stream each group
 * runs on (the groups of massive_get_timing). groups is a bit mask, bit i for
 * group i (MASSIVE_TIMING_ALL: every group, 0: off); it clears the totals.
 * Each timed group adds event packets to its streams, and the two gathers run
 * in one launch unless group 2 or 3 is on (then one after the other, each
 * alone on its resource), so a run that must not be slowed times only what it
 * needs. MASSIVE_EINVAL for bits outside the
 * mask. */
#define MASSIVE_TIMING_ALL 0x7F
int massive_set_timing(massive_ctx* ctx, int groups);
/* Totals since enabled: out_ms[i] summed milliseconds and out_calls[i]
 * launches for i = 0 sample+dedup, 1 classify and relabel, 2 gather_hbm, 3 gather_miss,
 * 4 eviction round, 5 refill, 6 the last hop's sampler kernel alone (a part
 * of group 0). out_ms and out_calls have room for 7 entries each.
 * Synchronises the context's streams. */
int massive_get_timing(massive_ctx* ctx, double* out_ms, int64_t* out_calls);

/* ------------------------------------------------------------------------
 * Operators of a training step on what massive_sample gathers: rows held in
 * few bits, the mean over a sampled block, a layer's product, a gated layer,
 * the norm and the dropout between them and the step on the weights, with
 * their gradients.
 *
 * They take no context. Every call checks its arguments on the host, enqueues
 * its kernels on `stream` and returns without waiting; it allocates nothing
 * and keeps nothing. Pointers are device memory of the current device unless
 * said otherwise, and a table of packed rows that is read may also be pinned
 * host memory, to be kept as it is until the stream has passed the call.
 * What a call reads and writes must not overlap, except where an argument is
 * documented as updated in place. Arrays hold 32-bit or bf16 values
 * (MASSIVE_F32, MASSIVE_BF16) at their natural alignment; strides are in
 * elements. Sums, products' accumulators and statistics are fp32; a result is
 * rounded to nearest even where it is stored, and nothing before it is rounded
 * to fewer bits, but for dz in massive_linear_grads and massive_gated_grads. Results do not depend on
 * the order in which the device runs a call's blocks: the same call on the
 * same inputs gives the same bits. An empty extent (no rows, no tensors) is
 * MASSIVE_OK and does nothing. On failure the message is in
 * massive_last_error(NULL).
 *
 * A call may be captured into a HIP graph. Its replays read and write the same
 * addresses, and keep the arguments that the call had on the host, among them
 * massive_dropout's seed (but not what it reads at seed_at) and massive_adamw's
 * lr and t: every replay repeats the captured step's bias
 * corrections. That is right only once both are 1; until then the step belongs
 * outside the graph.
 */
#define MASSIVE_F32 0
#define MASSIVE_BF16 1
#define MASSIVE_PACKED 2 /* rows of massive_row_format (massive_block_mean) */

/* Rows of d values held in 8 or 4 bits. The columns form groups of `group`
 * (a power of two from 16 to 512; 0 for one group of the whole row, which is
 * also what a group of d columns or more is); the last may be short. A row is
 * its codes, padded with zeros to four bytes, then each group's floats:
 *   8 bits: int8 codes c in [-127, 127] and step = max|x| / 127; stands for
 *     c * step;
 *   4 bits: codes c in [0, 15], even columns in the low nibbles, and the
 *     group's least value lo and step = (max - lo) / 15; stands for
 *     lo + c * step.
 * c is the nearest code, ties to the even one. A group whose max|x| (8 bits)
 * or max - lo (4 bits) is under 2^-119 has step 0. A group that holds a value
 * that is not finite, or whose max - lo is not, has a step of NaN: all of it
 * reads as NaN. Rows are a multiple of four bytes, so massive_init takes them
 * as feature rows. */
typedef struct {
  int32_t d;         /* values per row, 1..1048576                              */
  int32_t bits;      /* 8 or 4                                                  */
  int32_t group;     /* columns per group, or 0                                 */
  int32_t reserved;  /* 0                                                       */
  int64_t row_bytes; /* bytes from row to row: 0 for the least, or a multiple of
                        four that is at least that                              */
} massive_row_format;

/* Checks a format and writes its least row size, and the offset of the first
 * group's floats in a row (each pointer may be NULL). */
int massive_row_layout(const massive_row_format* fmt, int64_t* row_bytes, int64_t* floats_at);

/* Writes n rows to a table of table_rows rows: row i of src (row i starting at
 * src + i * src_stride) to row slots[i], or to row i if slots is NULL. A slot
 * outside [0, table_rows) is left out. The others must be distinct: a row that
 * two sources share holds neither. Padding bytes between rows are not
 * written. */
int massive_pack_rows(const massive_row_format* fmt, const void* src, int32_t src_type, int64_t src_stride, int64_t n,
                      const int32_t* slots, void* table, int64_t table_rows, void* stream);

/* Reads n rows of a table: row index[i], or row i if index is NULL, to row i
 * of out. An index outside [0, table_rows) reads as a row of zeros. */
int massive_unpack_rows(const massive_row_format* fmt, const void* table, int64_t table_rows, const int32_t* index,
                        int64_t n, void* out, int32_t out_type, int64_t out_stride, void* stream);

/* One sampled block (a hop of massive_batch) or any CSR of its kind: row i of
 * n lists indices[indptr[i] .. indptr[i+1]), source rows in [0, rows); edges
 * is the room in indices, and offsets beyond it are cut to it. An index
 * outside [0, rows) stands for a row of zeros (it counts in the mean). */
typedef struct {
  const int32_t* indptr;  /* [n + 1] */
  const int32_t* indices; /* [edges] */
  int64_t n, edges, rows; /* each at most 2^30 */
} massive_block;

/* out[i] = mean of x[j] over row i's list, d columns; zeros for an empty list.
 * x_type MASSIVE_PACKED: x holds rows of fmt (fmt->d = d; x_stride ignored),
 * otherwise fmt is NULL. */
int massive_block_mean(const massive_block* block, const void* x, int32_t x_type, int64_t x_stride,
                       const massive_row_format* fmt, int32_t d, void* out, int32_t out_type, int64_t out_stride,
                       void* stream);

/* Bytes of workspace of massive_block_mean_backward on rows of d columns. */
int massive_block_mean_workspace(const massive_block* block, int32_t d, int64_t* bytes);

/* The gradient: dx[j] = sum over the entries of j, in the order of the rows
 * that list it, of dout[i] / (length of row i); plus add[j] for j < add_rows
 * (the gradient that the block's own rows, the first of its sources, get from
 * elsewhere; add may be NULL). All arrays have one type; dx is [rows, d].
 * workspace: massive_block_mean_workspace's bytes, 16-byte aligned. */
int massive_block_mean_backward(const massive_block* block, const void* dout, int32_t type, int64_t dout_stride,
                                int32_t d, const void* add, int64_t add_stride, int64_t add_rows, void* dx,
                                int64_t dx_stride, void* workspace, int64_t workspace_bytes, void* stream);

/* Activations of massive_linear: the identity, max(z, 0), z * Phi(z) with the
 * normal distribution's Phi, z / (1 + exp(-z)) */
#define MASSIVE_ACT_NONE 0
#define MASSIVE_ACT_RELU 1
#define MASSIVE_ACT_GELU 2
#define MASSIVE_ACT_SILU 3

/* A layer: z = [x | x2] w^T + bias, y = act(z) + residual, over `rows` rows.
 * x2 (k2 columns; NULL and 0 for none), bias and residual are optional, and
 * so is pre, which receives z for the backward pass. All arrays have one
 * type. A pointer may not be both read and written. */
typedef struct {
  const void* x;        /* [rows, k]                                          */
  const void* x_second; /* [rows, k_second] or NULL                           */
  const void* w;        /* [n, k + k_second], each output's weights in a row  */
  const void* bias;     /* [n] or NULL                                        */
  const void* residual; /* [rows, n] or NULL                                  */
  void* y;              /* [rows, n]                                          */
  void* pre;            /* [rows, n] or NULL                                  */
  int64_t rows;
  int64_t x_stride, x_second_stride, w_stride, residual_stride, y_stride, pre_stride;
  int32_t n, k, k_second;
  int32_t type, act;
} massive_linear_args;

int massive_linear(const massive_linear_args* args, void* stream);

/* The layer's gradients: dz = dy * act'(pre), dx = dz w (columns of x and x2
 * apart), dw = dz^T [x | x2], dbias = sum of dz over the rows. dx, dx_second,
 * dw and dbias may each be NULL; the residual's gradient is dy. w is read for
 * dx and dx_second, x and x_second for dw. pre is z as massive_linear wrote it
 * (for relu, y without a residual serves as well), and NULL for
 * MASSIVE_ACT_NONE. With MASSIVE_BF16, dz is rounded to bf16 before the
 * products dx and dw, whose factors are bf16 (dz is one already for the identity
 * and relu; for gelu and silu a gradient of normal values is 0.0023 of its size
 * off, where its own rounding leaves 0.0017). dbias sums it unrounded. */
typedef struct {
  const void *dy, *pre, *x, *x_second, *w;
  void *dx, *dx_second, *dw, *dbias;
  int64_t rows;
  int64_t dy_stride, pre_stride, x_stride, x_second_stride, w_stride, dx_stride, dx_second_stride, dw_stride;
  int32_t n, k, k_second;
  int32_t type, act;
} massive_linear_grads;

/* Bytes of workspace of massive_linear_backward (0 if neither dw nor dbias is
 * asked for). */
int massive_linear_workspace(const massive_linear_grads* args, int64_t* bytes);
int massive_linear_backward(const massive_linear_grads* args, void* workspace, int64_t workspace_bytes, void* stream);

/* Dropout: y = residual + (x kept ? x / (1 - p) : 0), over rows of d columns;
 * residual may be NULL. The mask is drawn where it is used and not stored:
 * column j of row i is kept if word j % 4 of Philox4x32-10 at the counter
 * (j / 4, i, draw, 0), under the seed (its low word first), is at least p 2^32,
 * rounded to a whole number. It hangs on the column's place alone, so the
 * gradient of x is the same call on y's, without a residual. Draws of one seed
 * (a step's layers, say) have masks of their own. With seed_at, the seed is
 * read there when the stream comes to the call, so that replays of a captured
 * call can each have another. A column that is not kept gives 0 whatever it
 * held. */
typedef struct {
  const void* x;           /* [rows, d]                                       */
  const void* residual;    /* [rows, d] or NULL                               */
  void* y;                 /* [rows, d]                                       */
  const uint64_t* seed_at; /* device memory, or NULL: `seed`                  */
  int64_t rows;
  int64_t x_stride, residual_stride, y_stride;
  uint64_t seed;
  double p;                /* in [0, 1]                                       */
  uint32_t draw;
  int32_t d, type;
} massive_dropout_args;

int massive_dropout(const massive_dropout_args* args, void* stream);

/* The root-mean-square norm of rows of d columns: s = x + residual (which may
 * be NULL), y = s / sqrt(mean(s^2) + eps) * weight (NULL for ones). sum, if not
 * NULL, receives s; y is computed from s before that is rounded. With fmt
 * (fmt->d = d), y is a table of table_rows packed rows as massive_pack_rows
 * writes them, row i of the norm going to row slots[i], or to row i if slots is
 * NULL; y_stride is ignored. An eps between 0 and 2^-126 counts as 2^-126. Rows
 * whose squares leave fp32's range are normed all the same; a row with a NaN is
 * NaN, as a row of zeros with an eps of 0 is, and in a row with an infinity the
 * finite values give 0 and the infinities NaN. */
typedef struct {
  const void* x;        /* [rows, d]                                          */
  const void* residual; /* [rows, d] or NULL                                  */
  const void* weight;   /* [d] or NULL                                        */
  void* sum;            /* [rows, d] or NULL                                  */
  void* y;              /* [rows, d], or a table                              */
  const massive_row_format* fmt;
  const int32_t* slots;
  int64_t table_rows;
  int64_t rows;
  int64_t x_stride, residual_stride, sum_stride, y_stride;
  double eps;
  int32_t d, type;
} massive_norm_args;

int massive_rms_norm(const massive_norm_args* args, void* stream);

/* Its gradients. With r = 1 / sqrt(mean(s^2) + eps), n = s r and g = dy weight:
 * dx = r (g - n mean(g n)) + ds, which is x's gradient and residual's, and
 * dweight = sum of dy n over the rows. s is massive_rms_norm's sum (without a
 * residual, x); ds, which may be NULL, is the gradient that s gets from
 * elsewhere. dx and dweight may each be NULL. */
typedef struct {
  const void *dy, *s, *weight, *ds;
  void *dx, *dweight;
  int64_t rows;
  int64_t dy_stride, s_stride, ds_stride, dx_stride;
  double eps;
  int32_t d, type;
} massive_norm_grads;

/* Bytes of workspace of massive_rms_norm_backward (0 if dweight is not asked for). */
int massive_rms_norm_workspace(const massive_norm_grads* args, int64_t* bytes);
int massive_rms_norm_backward(const massive_norm_grads* args, void* workspace, int64_t workspace_bytes, void* stream);

/* A gated layer: with [g | u] = [x | x2] w^T + bias, whose weights' first n rows
 * are the gate's and the others u's, y = act(g) * u, over `rows` rows. x2,
 * bias and pre are optional; pre receives [g | u] for the backward pass. All
 * arrays have one type. */
typedef struct {
  const void* x;        /* [rows, k]                                          */
  const void* x_second; /* [rows, k_second] or NULL                           */
  const void* w;        /* [2 n, k + k_second]                                */
  const void* bias;     /* [2 n] or NULL                                      */
  void* y;              /* [rows, n]                                          */
  void* pre;            /* [rows, 2 n] or NULL                                */
  int64_t rows;
  int64_t x_stride, x_second_stride, w_stride, y_stride, pre_stride;
  int32_t n, k, k_second; /* n at most 2^19                                   */
  int32_t type, act;
} massive_gated_args;

int massive_gated(const massive_gated_args* args, void* stream);

/* Its gradients: dg = dy * u * act'(g), du = dy * act(g), dx = [dg | du] w
 * (columns of x and x2 apart), dw = [dg | du]^T [x | x2], dbias = sum of
 * [dg | du] over the rows. dx, dx_second, dw and dbias may each be NULL. With
 * MASSIVE_BF16, dg and du are rounded to bf16 before the products dx and dw,
 * as massive_linear_backward rounds dz; dbias sums them unrounded. The order of
 * the sums goes by the sizes, that of dx's also by which of dx and dx_second are
 * asked for, and not by where the arrays lie. */
typedef struct {
  const void *dy, *pre, *x, *x_second, *w;
  void *dx, *dx_second, *dw, *dbias;
  int64_t rows;
  int64_t dy_stride, pre_stride, x_stride, x_second_stride, w_stride, dx_stride, dx_second_stride, dw_stride;
  int32_t n, k, k_second;
  int32_t type, act;
} massive_gated_grads;

/* Bytes of workspace of massive_gated_backward: [dg | du] and the sums' parts. */
int massive_gated_workspace(const massive_gated_grads* args, int64_t* bytes);
int massive_gated_backward(const massive_gated_grads* args, void* workspace, int64_t workspace_bytes, void* stream);

/* One tensor of an AdamW step, n values. Everything but grad is updated in
 * place. With state_bits 32, m and v are float[n] and the scales are NULL.
 * With state_bits 8, m is int8[n] and v uint8[n], and each 256 values share a
 * scale, m_scale and v_scale being float[ceil(n / 256)]:
 *   m = c |c| s with c = round(sqrt(|m| / s)) and the sign of m, s = max|m| / 127^2;
 *   v = c^4 s with c = round((v / s)^(1/4)), at least 1 where v > 0,
 *   s = max v / 255^4.
 * A block whose max|m| is under 2^-112 (max v under 2^-94) holds zeros, and
 * one that holds a value that is not finite reads as NaN. States start as
 * zeros. copy, if not NULL, receives the new values as bf16. */
typedef struct {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  int64_t n;
} massive_adamw_tensor;

typedef struct {
  double lr, beta_first, beta_second, eps, weight_decay;
  int64_t t;          /* the step's number, from 1: tensors that have taken
                         different numbers of steps go in calls of their own */
  int32_t state_bits; /* 32 or 8 */
  int32_t param_type, grad_type;
  int32_t reserved;   /* 0 */
} massive_adamw_args;

/* A step on all tensors of a host array:
 *   p *= 1 - lr * weight_decay
 *   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
 *   p -= lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
 * with the new m and v in 32 bits, before they are held in 8, denormals among
 * them. An eps between 0 and 2^-126 counts as 2^-126. With an eps of 0 a value
 * whose new v is 0 is divided by 0: NaN where m is 0 too, infinite where 8-bit
 * states have kept m and not v. The array is read during the call only. */
int massive_adamw(const massive_adamw_tensor* tensors, int64_t count, const massive_adamw_args* args, void* stream);

/* What 8-bit states stand for, as floats: n codes of m and of v with their
 * scales, to m_out and v_out. */
int massive_adamw_states(const void* m, const void* v, const float* m_scale, const float* v_scale, int64_t n,
                         float* m_out, float* v_out, void* stream);

/* Frees every device and host resource of the context; NULL is a no-op.
 * Always MASSIVE_OK. */
int massive_destroy(massive_ctx* ctx);

/* Message of the last failure on this context (ctx == NULL: of the last
 * failed massive_init or operator call on this thread). Never NULL. */
const char* massive_last_error(const massive_ctx* ctx);

#ifdef __cplusplus
}
#endif

#endif /* MASSIVE_H */
