/*
 * dadam - the per-iteration decentralized Adam step on one MI355X (gfx950).
 *
 * One call of dadam_gossip_step performs, for every updated replica ("row") i and every
 * element e of the packed parameter vector, iteration t of the paper's Algorithm 3
 * (appendix "Decentralized accumulated Adam"; Algorithm 1 of section 4 is its case s = 1):
 *
 *     t_hat = ceil(t / s)                                                   line 4
 *     m     = beta1 * m_hat_i[e] + (1 - beta1) * g_i[e]                      line 6
 *     v     = beta2 * v_hat_i[e] + (1 - beta2) * g_i[e]^2                    line 7
 *     x_dst_i[e] = sum_k w[k] * x_src[col[k]][e]                             line 8, mixing term
 *                  - lr * (m / (1 - beta1^t_hat)) / (sqrt(v / (1 - beta2^t_hat)) + eps)       (eq. (2), section 2)
 *     b_i[e] += g_i[e] / s                                                   line 9
 *     if t mod s == 0:  m_hat_i[e] = beta1 * m_hat_i[e] + (1 - beta1) * b_i[e]               lines 10-13
 *                       v_hat_i[e] = beta_vhat * v_hat_i[e] + (1 - beta_vhat) * b_i[e]^2
 *                       b_i[e] = 0
 *
 * A tensor with weight_decay lambda > 0 uses the AdamW-style variant the appendix mentions without
 * writing it out; the reading taken is decoupled decay of the replica's OWN previous parameters
 * inside the search direction (which, as the paper stresses, depends on the worker's own quantities
 * only):   x_dst_i[e] = mixing term - lr * (direction + lambda * x_src[i][e]),  at every iteration.
 * Source buffer i must then be row i's own previous parameters (n_rows <= n_cols).
 *
 * k runs over row i of a CSR neighbour list (row_ptr, col, w); the replica itself is an ordinary
 * entry of its row.  The sum is taken in the order the row lists its entries, a product and then fused
 * multiply-adds, except where many rows list the same sources with the same weights (an All-Reduce loop): such
 * rows may share one sum, taken in another fixed order.  Every row reads the previous iterate x^(t-1) (the sources), never a value
 * written by the same call.  m and v are temporaries and are not stored.
 *
 * General rules of this interface
 *   - All entry points are extern "C", take plain pointers and sizes, return an int status
 *     (0 = DADAM_OK, negative = error) and never throw or abort.  The text of the last error of a
 *     handle is available from dadam_last_error().
 *   - "host" / "device" says where a pointer must point.  Large buffers (parameters, gradients,
 *     moments, accumulator) are DEVICE memory owned by the caller; the library never allocates,
 *     frees or copies them and never synchronises a stream.  The library owns only metadata on host and
 *     device: the segment table, the CSR slots and, for layouts of many short tensors with at most seven
 *     elements between two of them, a byte of device memory for every four elements of one buffer, up
 *     to 64 MB (d of 2^28); for handles that call what is described under "Around the step", what that needs, and the tables of
 *     dadam_set_matrices.  (One set-up call is the exception and says so: dadam_place_by_timing
 *     overwrites the empty arena it is given and returns when its measurements are done.)
 *   - Launching entry points enqueue work on the given HIP stream (a hipStream_t passed as
 *     void*; NULL = the default stream) and return at once.  The caller keeps every buffer alive
 *     and unmodified until that work has finished.
 *   - All validation happens on the host before anything is launched; a failed call launches
 *     nothing.
 *   - At most DADAM_MAX_ROWS rows and DADAM_MAX_ROWS source buffers per handle (tile mode needs 1 KB of
 *     LDS per source buffer: 160 KB for 160).  Up to 64 of each, every launch carries its own copy of the
 *     pointer tables.  Beyond that the tables of the bound buffers live in device memory, one immutable
 *     copy per dadam_bind; the library keeps the last DADAM_BINDINGS_KEPT of them, so work launched under
 *     a binding must have finished before that many further dadam_bind calls are made, and dadam_bind
 *     then copies to the device (it may wait for work in flight; not for use under stream capture).
 *   - A handle is not thread-safe: calls on one handle must come from one thread at a time.  Launches
 *     on different streams may be in flight together (every launch carries its own copy of the pointer
 *     tables and scalars), except dadam_mix_consensus, whose calls share scratch memory of the handle.
 */
#ifndef DADAM_H_
#define DADAM_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DADAM_ABI_VERSION 2u
#define DADAM_MAX_ROWS 160u
#define DADAM_MAX_SLOTS 16u
#define DADAM_BINDINGS_KEPT 8u
#define DADAM_DEVICE_NONE (-1) /* host-only handle: validation and planning work, launches fail */

/* element types of parameters and gradients; m_hat, v_hat and b are always float32 */
#define DADAM_F32 0u
#define DADAM_BF16 1u

/* status codes */
#define DADAM_OK 0
#define DADAM_EINVAL (-1) /* null pointer, zero size, bad enum, value out of range            */
#define DADAM_EALIGN (-2) /* a device buffer is not 16-byte aligned                            */
#define DADAM_ETOPO (-3)  /* malformed neighbour list                                          */
#define DADAM_EALIAS (-4) /* buffers overlap in a way that would let a row read a new value     */
#define DADAM_ESTATE (-5) /* call order: no buffers bound, slot not set, host-only handle, ...  */
#define DADAM_EHIP (-6)   /* a HIP runtime call failed                                         */

/* flags of dadam_gossip_step.  Without a FORCE flag the library chooses: tile mode when some source is read
 * by two or more rows and the tile fits in LDS (also when an in-place row needs it), direct mode otherwise -
 * and also, where measured faster, for rows of at most two sources on more than 16 sources and for rows of at
 * most eight sources when a CU would hold only one workgroup of the tile (see dadam_get_row_order).
 * dadam_slot_uses_tile_mode reports the choice.  Three kinds of launch are then given to other kernels where that was
 * measured faster: rows that share whole neighbour lists (one sum for all of them), launches of few tiles and very
 * large ones (a wavefront per row in place of the tile, or the other way round; the same sums in the same order). */
#define DADAM_FUSE_ACCUM 1u   /* also do lines 9-13 (accumulate and fold) in the same pass         */
#define DADAM_FORCE_DIRECT 2u /* every row streams its sources from global memory                  */
#define DADAM_FORCE_TILE 4u   /* stage each source tile once in LDS and update all rows from it    */

/* flags reported by dadam_set_topology through *warn */
#define DADAM_WARN_NOT_COLUMN_STOCHASTIC 1u /* square W whose columns do not sum to 1             */

typedef struct dadam_handle dadam_handle; /* opaque, owned by the library */

/* One tensor of the packed layout: elements [offset_elems, offset_elems + numel) of every
 * per-replica buffer.  Tensors must be listed in increasing offset order and must not overlap;
 * elements between tensors (padding) are never written, and what they hold is never used (loads may take them along: up to
 * three at the edge of a tensor, all that lie between tensors at most seven apart).  weight_decay >= 0 is the decoupled
 * weight decay of this tensor (0 = plain Adam; e.g. 3e-5 on all but the normalisation parameters in
 * the paper's ResNet-50 recipe).  flags is reserved and must be 0. */
typedef struct {
  uint64_t offset_elems;
  uint64_t numel;
  float weight_decay;
  uint32_t flags;
} dadam_tensor_desc;

typedef struct {
  uint32_t abi_version; /* DADAM_ABI_VERSION */
  uint32_t n_rows;      /* R: replicas updated by a step                                          */
  uint32_t n_cols;      /* number of source buffers holding x^(t-1) (R for a full simulation;     */
                        /* own parameters + neighbours' receive buffers for one node's share)     */
  uint64_t d;           /* elements per buffer (packed length, padding included)                  */
  uint32_t n_tensors;
  const dadam_tensor_desc* tensors; /* host, copied */
  uint32_t param_dtype;             /* DADAM_F32 | DADAM_BF16: type of x_src and x_dst            */
  uint32_t grad_dtype;              /* DADAM_F32 | DADAM_BF16: type of the gradients              */
  float lr, beta1, beta2, eps;      /* Algorithm 1 / 3 hyper-parameters                           */
  uint32_t accum_s;                 /* s >= 1, iterations per accumulation loop; 1 = Algorithm 1  */
  float beta_vhat; /* decay of v_hat in the fold (line 12).  The listing prints beta_1 there; that is
                      taken as a misprint and the default, selected by a negative value or NaN, is
                      beta2.  Any value in [0, 1) selects it explicitly. */
  int32_t device;  /* HIP device ordinal, or DADAM_DEVICE_NONE */
  uint32_t lds_limit_bytes; /* LDS one workgroup may use.  0: what the device reports (a host-only handle
                               assumes 65536).  A non-zero value plans for that much instead (e.g. to keep
                               room for other kernels' LDS); on a device handle it must not exceed what the
                               device reports.  Large steps of a single row reserve up to 154 KB of every
                               compute unit's LDS without using it, to bound how many of their wavefronts
                               are in flight (5 % faster): a kernel on another stream that needs more than is
                               left waits for them.  A limit below the device's turns that off. */
  uint32_t n_xcds;          /* accelerator complex dies (each with its own L2) that consecutive workgroup
                               ids are dealt over.  0: what the device reports (host-only handle: 8). */
} dadam_config;

/* Arrays (host) of DEVICE pointers, caller-owned; the arrays themselves are copied.
 * Every buffer holds cfg.d elements and is 16-byte aligned.
 * x_dst[i] may be the very same buffer as one x_src[c] (update in place); any other overlap
 * between two different buffers is rejected with DADAM_EALIAS.  In-place update is legal when the
 * step runs in tile mode, or when source c is read by row i only (a step over tensors with weight decay
 * also reads source k for every row k). */
typedef struct {
  const void* const* x_src; /* [n_cols] x^(t-1) */
  void* const* x_dst;       /* [n_rows] x^(t)   */
  float* const* m_hat;      /* [n_rows] */
  float* const* v_hat;      /* [n_rows] */
  float* const* acc;        /* [n_rows] the accumulator b; may be NULL when accum_s == 1 */
} dadam_buffers;

/* What the planner decided, for tests and tuning. */
typedef struct {
  uint32_t n_segments;      /* maximal runs of contiguous tensors                               */
  uint32_t tile_elems;      /* elements of one tile in tile mode                                */
  uint32_t direct_elems;    /* elements of one work item in direct mode                         */
  uint64_t n_tiles_tile;    /* work items (workgroups) of a full step in tile mode that goes by segments: a tile
                               that several of them touch counts for each.  Layouts of short segments side by
                               side mostly go by one grid over the vector, with each tile once */
  uint64_t n_tiles_direct;  /* the same per row in direct mode (work items = this * n_rows)     */
  uint32_t lds_bytes_tile;  /* LDS per workgroup in tile mode                                   */
  uint32_t tile_mode_possible; /* 1 if the source tile fits in LDS                              */
  uint32_t lds_limit_bytes; /* LDS per workgroup the plan was made for                          */
  uint32_t n_xcds;          /* dies the tile order is laid out for                              */
  uint32_t mix_tile_elems;  /* elements of one tile of the mixing-only launch (tile mode)       */
  uint32_t lds_bytes_mix;   /* LDS per workgroup of the mixing-only launch                      */
  uint64_t n_tiles_mix;     /* the same of a mixing-only launch in tile mode                    */
  uint32_t tile_waves, tile_vectors; /* shape of the fused step's tile kernel: wavefronts per workgroup,
                                        16-byte vectors per lane and row                          */
  uint32_t mix_waves, mix_vectors;   /* the same for the mixing-only launch                       */
  uint32_t streaming;       /* 1 if accesses carry the non-temporal hint (large working sets).  Where this is
                               0, steps of up to three rows (not mixing or accumulation) carry it all the same
                               if the sources that the slot's rows list, outputs that are not updated in place,
                               gradients and state add up to more than 344 MB (2^20) */
} dadam_plan_info;

/* Create a handle.  Validates the configuration, builds the segment table from the tensor list
 * and (unless device == DADAM_DEVICE_NONE) uploads it.  *out is set only on success.
 * Errors: DADAM_EINVAL (null, n_rows/n_cols 0 or above DADAM_MAX_ROWS, d == 0, s == 0, dtype,
 * tensors unordered / overlapping / beyond d / negative weight decay / non-zero flags / weight decay with
 * n_rows > n_cols, hyper-parameters out of
 * range: lr finite, 0 <= beta < 1, eps >= 0), DADAM_EHIP. */
int dadam_init(const dadam_config* cfg, dadam_handle** out);

/* Register rows of the mixing matrix W (section 2, eq. (2); Assumption 3 lists the properties the
 * analysis wants) in slot `slot` (< DADAM_MAX_SLOTS); time-varying topologies use one slot per
 * distinct matrix.  row_ptr[n_rows + 1], col_idx[nnz], w[nnz] are HOST arrays and are copied.
 * Checked: row_ptr[0] == 0, non-decreasing, every row non-empty; 0 <= col < n_cols; no column
 * twice in a row; w finite and > 0; |sum of a row - 1| <= 1e-5.  Else DADAM_ETOPO.
 * If n_rows == n_cols and some column sum is off by more than 1e-5, the call still succeeds and
 * sets DADAM_WARN_NOT_COLUMN_STOCHASTIC in *warn (warn may be NULL).
 * A slot may be overwritten only while no launched work still uses it. */
int dadam_set_topology(dadam_handle* h, uint32_t slot, const int32_t* row_ptr,
                       const int32_t* col_idx, const float* w, uint32_t* warn);

/* Bind the device buffers.  May be called again at any time (e.g. to exchange x_src and x_dst);
 * work already launched keeps the pointers it was launched with.
 * Errors: DADAM_EINVAL (null), DADAM_EALIGN, DADAM_EALIAS. */
int dadam_bind(dadam_handle* h, const dadam_buffers* bufs);

/* Exchange the roles of x_src and x_dst (needs n_rows == n_cols): what a ping-pong caller does
 * between two iterations. */
int dadam_swap_x(dadam_handle* h);

/* Iteration t (1-based) of Algorithm 3 as written at the top of this file, using the neighbour
 * list in `slot` and grads[n_rows] (HOST array of DEVICE pointers, each cfg.d elements of
 * grad_dtype, 16-byte aligned, not overlapping any output).  With DADAM_FUSE_ACCUM lines 4-13 are
 * done in one pass; without it only lines 4-8 (x_dst) and the caller follows with
 * dadam_accumulate(grads, t) - never both for one t.  On the first iteration of a loop
 * ((t-1) mod s == 0) the accumulator is taken to be zero and is not read.
 * Errors: DADAM_ESTATE (nothing bound, slot empty, host-only handle), DADAM_EINVAL (t == 0, null,
 * both FORCE flags), DADAM_EALIGN, DADAM_EALIAS (in-place rows that the chosen mode cannot do, or
 * DADAM_FORCE_TILE when the source tile does not fit in LDS -> DADAM_EINVAL), DADAM_EHIP. */
int dadam_gossip_step(dadam_handle* h, uint32_t slot, const void* const* grads, uint64_t t,
                      uint32_t flags, void* hip_stream);

/* The same restricted to tensors [tensor_begin, tensor_end) of the layout (a "bucket" in the
 * sense of section 2.1, where parameters are updated and communicated bucket by bucket).
 * Disjoint ranges of one iteration touch disjoint elements, also where two ranges meet inside one
 * tile and when parameters are updated in place, so they may run on different streams at the same
 * time (issued from one host thread); a range of iteration t + 1 must be ordered after the same
 * range of iteration t.  An empty range is a successful no-op. */
int dadam_gossip_step_range(dadam_handle* h, uint32_t slot, const void* const* grads, uint64_t t,
                            uint32_t flags, uint32_t tensor_begin, uint32_t tensor_end,
                            void* hip_stream);

/* Lines 9-13 of Algorithm 3 alone: b += g / s and, when t mod s == 0, the fold into m_hat and
 * v_hat followed by b = 0. */
int dadam_accumulate(dadam_handle* h, const void* const* grads, uint64_t t, void* hip_stream);

/* x_dst = W x_src: eq. (2) with a zero search direction (pure gossip averaging).  flags: 0 or one
 * of DADAM_FORCE_DIRECT / DADAM_FORCE_TILE. */
int dadam_mix(dadam_handle* h, uint32_t slot, uint32_t flags, void* hip_stream);

/* The gossip round of dadam_mix and, at no extra HBM traffic, the consensus error of the SOURCES,
 *     *consensus_out = sum over source buffers c and elements e of (x_src[c][e] - mean_c x_src[.][e])^2,
 * the squared distance of the replicas from their average whose decay per gossip round the paper
 * plots to compare topologies (section "Important aspects ...", heterogeneous communication; the
 * consensus lemma bounds the same quantity).  consensus_out is a DEVICE pointer to one double,
 * written by work enqueued on the stream; per-element arithmetic is float32, the sum double.
 * Available in tile mode only (the sources of a tile are then on chip together); DADAM_ESTATE
 * otherwise.  x_dst has dadam_mix's bits except where dadam_mix lets many rows share one sum (All-Reduce loops, see the top
 * of this file): this call always sums in the order the row lists, and the two differ there by the rounding of a float32
 * sum.  Calls on one handle must not overlap in time: they share the handle's partial sums. */
int dadam_mix_consensus(dadam_handle* h, uint32_t slot, uint32_t flags, double* consensus_out,
                        void* hip_stream);

/* dadam_mix_consensus for callers that cannot allocate device memory or tolerate a library that does:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments,
 * same results; the partial sums of the consensus error live in an array of DADAM_STATIC_SCRATCH_BYTES
 * bytes inside the library's own device image (every GPU holds its copy from the moment the library is
 * loaded until the process ends) instead of the handle's allocated buffer.  The call itself allocates and
 * frees nothing and clears the array with a kernel before use (it keeps the previous call's contents).
 * ALL handles and calls on one GPU share that one array: two such calls must not overlap in time on a
 * GPU, whatever their streams or handles.  A pass that needed more partial sums than the array holds
 * would be refused with DADAM_EINVAL (today every pass needs exactly DADAM_STATIC_SCRATCH_BYTES / 8).
 * Other errors as dadam_mix_consensus. */
#define DADAM_STATIC_SCRATCH_BYTES 8192u
int dadam_mix_consensus_static(dadam_handle* h, uint32_t slot, uint32_t flags, double* consensus_out,
                               void* hip_stream);

/* Change the step size used by later calls (learning-rate schedules). */
int dadam_set_lr(dadam_handle* h, float lr);

/* Planner facts for this handle. */
int dadam_get_plan_info(const dadam_handle* h, dadam_plan_info* out);

/* The choice between tile and direct mode for a step with this slot when no FORCE flag is given, as described at the
 * flags above: 1 tile, 0 direct, negative status on error.  Launches of rows that share whole neighbour lists, launches
 * of few tiles and very large ones may then run in other kernels all the same. */
int dadam_slot_uses_tile_mode(const dadam_handle* h, uint32_t slot);

/* The order in which direct mode takes the rows of this slot (order_out: n_rows entries, a permutation of
 * 0 .. n_rows-1).  When rows share sources (and the device has more than one die), rows that
 * share sources are neighbours in this order and run on one die at about the same time - all rows of a piece of the
 * vector, or one contiguous group of the order per die, by size - so that a
 * source two rows read comes from memory once and from that die's L2 the second time (one-peer graph on 64
 * replicas, mixing only: 0.54-0.61 of peak with rows as numbered when the two readers sit on different dies,
 * 0.76 when they share one).  The order changes nothing in what is computed.  Returns 1 if such an order is
 * in use, 0 if rows are taken as numbered (order_out is then the identity), negative status on error. */
int dadam_get_row_order(const dadam_handle* h, uint32_t slot, int32_t* order_out);

/* Offsets of a packed layout: tensor k starts at the next multiple of align_elems elements after
 * tensor k-1 ends.  numel[n] in, offsets[n] out (both host); returns the packed length through
 * *d_out. */
int dadam_pack_offsets(const uint64_t* numel, uint32_t n, uint32_t align_elems, uint64_t* offsets,
                       uint64_t* d_out);

/* Layout advice for HBM, part 1: equal distances.  Places n buffers of nbytes[k] bytes in a range of
 * arena_bytes bytes, in the given order, each at a multiple of 2 MiB, with equal gaps between
 * consecutive buffers so that the first starts at 0 and the last ends near the end of the range.
 * nbytes[n] in, offsets[n] out (host).
 * Errors: DADAM_EINVAL if a pointer is null, n == 0, or the buffers do not fit. */
int dadam_spread_offsets(const uint64_t* nbytes, uint32_t n, uint64_t arena_bytes, uint64_t* offsets);

/* Layout advice for HBM, part 2: where to put the buffers.  Measured on MI355X: a pass whose wavefronts read and
 * write contiguous kilobytes sustains 0.62-0.66 of peak bandwidth when the buffers it streams together all lie
 * inside one third (96 GiB) of the device's physical memory - which is where a fresh process's
 * allocations land - and 0.78-0.79 when every group of buffers that is streamed together lies half
 * in one third and half in another.  The library's own streaming kernels have their lanes apart (two places 32 or 64 KB
 * from each other) and depend on it little: placed / ordinary allocations 0.795 / 0.806 (16 float32 replicas of 124
 * million elements), 0.795 / 0.815 (one row of 355 million), 0.813 / 0.833 (64 replicas of 26 million), 0.801 / 0.780 (8
 * bfloat16 replicas of 774 million); the first after 100, 160, 200 GiB of other allocations 0.792 / 0.781, 0.796 / 0.779,
 * 0.801 / 0.778.  Placement is for the last kind and for such cards, and for a caller's own passes over the same buffers.  Nobody outside the driver sees physical addresses, and where the
 * driver puts one allocation relative to another is not predictable (measured: an arena pushed into
 * place by an allocation made before it, or placed by the amount of memory in use, lands elsewhere and
 * runs at 0.64-0.72).  What does hold is that ONE allocation of nearly the whole device (within 16 GiB of
 * device_total_bytes) covers the physical memory in order, so that offsets inside it are physical
 * positions to within what it leaves out.  For such an arena this helper deals the buffers alternately
 * over two regions, one ending 2 GiB below and one starting 2 GiB above the boundary between the first
 * two thirds: buffers 0, 2, 4, ... below, 1, 3, 5, ... above, spread over each region (64 GiB wide, wider
 * when the buffers need it) and staggered inside their gaps by a fixed pseudo-random number of 2 MiB
 * steps, so that the bases do not form an arithmetic progression (for some distances between bases that
 * costs 3-4 %).  Any run of consecutive buffers - all sources, all outputs, one kind of state - is then
 * split evenly.  nbytes[n] in, offsets[n] out (host), every offset a multiple of 2 MiB.  regions_out (may
 * be null) receives lo0, hi0, lo1, hi1 of the two regions, or 0, arena_bytes, 0, 0 for the fall-back.
 * *advice_out (may be null) says what was done:
 *   DADAM_PLACE_TWO_REGIONS     the rule above was applied;
 *   DADAM_PLACE_ARENA_ELSEWHERE the arena does not cover the device: offsets in it say nothing about
 *                               physical positions, and the buffers are placed at equal distances over
 *                               the whole arena instead (0.774 measured for an arena of 235 GiB; with contiguous
 *                               lanes 0.70-0.77, the packed level if the arena happens to lie inside one third);
 *   DADAM_PLACE_TOO_LARGE       half of the buffers do not fit below the boundary or the other half
 *                               between it and the next one: equal distances over the whole arena.
 * The caller hands `arena + offsets[k]` to dadam_bind and may use the space between the buffers for
 * anything else.
 * Errors: DADAM_EINVAL if a pointer is null, n == 0, or the buffers do not fit the arena at all. */
#define DADAM_PLACE_TWO_REGIONS 1u
#define DADAM_PLACE_ARENA_ELSEWHERE 2u
#define DADAM_PLACE_TOO_LARGE 4u
int dadam_place_offsets(const uint64_t* nbytes, uint32_t n, uint64_t arena_bytes, uint64_t device_total_bytes,
                        uint64_t* offsets, uint64_t* regions_out, uint32_t* advice_out);

/* Layout advice for HBM, part 3: the dealing itself, for a caller that knows two
 * regions [lo0, hi0) and [lo1, hi1) of one arena to lie in different thirds of the physical memory - e.g.
 * because it has timed a streaming probe over pairs of chunks of its arena, which tells same third from
 * different third reliably (paper_2410_11998_amd/arena.py does that).  dadam_deal_offsets places every
 * `every`-th buffer (numbers every-1, 2*every-1, ...) in the second region and the others in the first, spread
 * over each region and staggered as described under dadam_place_offsets.  every = 2 deals alternately (the
 * layout measured at 0.79 of peak); every = 4 puts a quarter of the buffers in the second region, for a second
 * region with little room (a 16-source mixing pass dealt 3:1 still ran at 0.79).  2 <= every <= 8.  Region
 * bounds are multiples of 2 MiB and the regions do not overlap.
 * Errors: DADAM_EINVAL (null, n == 0, every out of range, bounds unaligned or overlapping, a side's buffers do
 * not fit). */
int dadam_deal_offsets(const uint64_t* nbytes, uint32_t n, uint64_t lo0, uint64_t hi0, uint64_t lo1, uint64_t hi1,
                       uint32_t every, uint64_t* offsets);

/* Layout advice for HBM, part 4: finding the thirds by measurement.
 *
 * Where the thirds of the physical memory begin inside a caller's allocation cannot be computed (a large
 * allocation is pieced together from whatever is free: made first, its bytes [0, 96 GiB) lie in one third; made
 * after 100 GiB of other allocations, the second boundary was seen at 160 GiB), but it can be measured: a copy of
 * sixteen 64 MiB sources to sixteen outputs by contiguous kilobytes runs at 0.80-0.82 of peak when half of
 * its buffers sit in one third and half in another, and at 0.61-0.75 when all sit in one.
 *
 * dadam_find_stretches: the bookkeeping.  `rate(off_a, off_b, ctx)` is the fraction of peak a streaming pass
 * sustains with half of its buffers in the DADAM_PROBE_CHUNK_BYTES at arena offset off_a and half in those at
 * off_b (negative: failure, reported as DADAM_EHIP).  One chunk every DADAM_PROBE_STEP_BYTES is compared with a
 * reference chunk; those that run fast with it (>= 0.95 of the fastest pairing, which must itself reach 0.75)
 * lie in another third; a second reference among them tells the other two thirds apart.  out receives at most
 * DADAM_MAX_STRETCHES stretches [lo, hi) with the id (0, 1, 2) of their third, in address order; the same third
 * may come back later in the arena.  More stretches than that is noise: the timing is repeated once, then
 * *n_out = 0.  An arena too small for three chunks also gives *n_out = 0.  Host only.
 *
 * dadam_regions_from_stretches: the two regions (regions_out[4] = lo0, hi0, lo1, hi1) to deal the buffers
 * over with dadam_deal_offsets and its `every`: alternately (every = 2) over the two stretches of different
 * thirds with the most room if half of the buffers fit each, otherwise every 3rd, 4th, 6th or 8th buffer in
 * the smaller stretch (160 / 200 GiB allocated before the arena: 0.75 / 0.73 of peak against 0.60 / 0.64 at
 * equal distances).  Returns 1 if found, 0 if no two stretches of different thirds hold the buffers.
 *
 * dadam_place_by_timing: the whole procedure on a device.  `arena` is DEVICE memory (2 MiB aligned,
 * arena_bytes long, contents are overwritten: call it before anything is stored there).  The library times
 * such a pass over the arena (about half a second, some hundreds of short launches on the null stream, no
 * memory besides the arena), finds the stretches, chooses the regions, confirms them with one more pass
 * across the two regions and one inside each, and deals the buffers; if that yields nothing it falls back to
 * dadam_place_offsets (device_total_bytes is passed on).  offsets[n] and *report say what was done.  Synchronous.
 * Errors: DADAM_EINVAL, DADAM_EALIGN, DADAM_EHIP. */
#define DADAM_PROBE_CHUNK_BYTES 1073741824ull
#define DADAM_PROBE_STEP_BYTES 4294967296ull
#define DADAM_MAX_STRETCHES 6u
#define DADAM_POLICY_TIMED_REGIONS 1u  /* two regions found by timing, dealt with report.every             */
#define DADAM_POLICY_RULE_REGIONS 2u   /* dadam_place_offsets' two regions (arena covers the device)        */
#define DADAM_POLICY_EQUAL_DISTANCES 3u
#define DADAM_NOTE_NO_PROBE 1u         /* arena too small for the probe, or one buffer only                   */
#define DADAM_NOTE_NO_PICTURE 2u       /* the timings gave no consistent picture of the thirds              */
#define DADAM_NOTE_NO_ROOM 3u          /* no two stretches of different thirds hold the buffers             */
#define DADAM_NOTE_NOT_CONFIRMED 4u    /* the confirming passes disagreed with the stretches                */
typedef double (*dadam_pair_rate_fn)(uint64_t off_a, uint64_t off_b, void* ctx);
typedef struct {
  uint32_t third;    /* 0, 1, 2: stretches with the same id share a third */
  uint32_t reserved; /* 0 */
  uint64_t lo, hi;   /* arena offsets */
} dadam_stretch;
typedef struct {
  uint32_t policy;         /* DADAM_POLICY_* */
  uint32_t advice;         /* DADAM_PLACE_* as dadam_place_offsets reports it */
  uint32_t every;          /* DADAM_POLICY_TIMED_REGIONS: every `every`-th buffer lies in the second region */
  uint32_t note;           /* 0, or why the timing was not used: DADAM_NOTE_* */
  uint32_t n_stretches;
  uint32_t probe_launches; /* passes the probe launched */
  dadam_stretch stretches[DADAM_MAX_STRETCHES];
  uint64_t regions[4];     /* lo0, hi0, lo1, hi1 (lo1 = hi1 = 0: one region) */
  float rate_across;       /* fraction of peak of the confirming pass across the regions, 0 if none ran */
  float rate_inside[2];    /* ... and inside each region */
  uint32_t reserved;
} dadam_placement;
int dadam_find_stretches(uint64_t arena_bytes, dadam_pair_rate_fn rate, void* ctx, dadam_stretch* out,
                         uint32_t* n_out);
int dadam_regions_from_stretches(const dadam_stretch* stretches, uint32_t n_stretches, const uint64_t* nbytes,
                                 uint32_t n, uint64_t* regions_out, uint32_t* every_out);
int dadam_place_by_timing(void* arena, uint64_t arena_bytes, int32_t device, const uint64_t* nbytes, uint32_t n,
                          uint64_t device_total_bytes, uint64_t* offsets, dadam_placement* report);

/* ------------------------------------------------------------------------------------------------------------
 * Around the step: gradient clipping before it, 4-bit gossip behind it
 *
 * All of these take their buffers in the call: HOST arrays of n_rows (messages that are read: n_cols) DEVICE pointers,
 * caller-owned, 16-byte aligned and below address 2^52; nothing has to be bound.  Buffers of parameters have cfg.d elements of param_dtype,
 * gradients cfg.d of grad_dtype, copies and sums cfg.d float32, messages dadam_mx4_info.bytes bytes.  What a call writes must not
 * overlap anything else it reads or writes, but where "in place" is named.  Padding between tensors takes no part: it is
 * neither used nor written.  The first such call on a handle allocates and uploads what tells padding from elements (4 bytes for every 512
 * elements, 64 more where padding lies among them; nothing for one tensor of a multiple of 512), the scratch of the norms and the lists of the slots
 * as these calls read them (from then on dadam_set_topology does that); it may wait for the device and is refused while
 * hip_stream is being captured, later calls allocate nothing and may be recorded into a graph.
 * Errors of all: DADAM_EINVAL (null, address too high, value out of range, d above 2^36), DADAM_EALIGN, DADAM_EALIAS, DADAM_ESTATE (slot empty,
 * host-only handle, first call under capture, n_rows != n_cols where named), DADAM_EHIP. */

/* The global norm of every row's gradient over all tensors of the layout,
 *     norms[i] = sqrt(sum_e grads[i][e]^2),
 * to norms[n_rows], DEVICE memory, float32.  Squares and sums are taken in 64 bits, in an order that depends on the layout,
 * n_rows and the entry point only: the same call gives the same bits, and no square overflows or vanishes.  A NaN makes the norm NaN,
 * an infinity (without a NaN) makes it infinite; a norm above float32's range is infinite too.  Calls of dadam_grad_norm and dadam_clip_grads on one handle must not
 * overlap in time: they share the handle's partial sums. */
int dadam_grad_norm(dadam_handle* h, const void* const* grads, float* norms, void* hip_stream);

/* Clipping by the global norm, as recipes for language models have it before Adam: the norms as above, and
 *     out[i][e] = grads[i][e]                             if norms[i] <= max_norm (the same bits),
 *                 grads[i][e] * (max_norm / norms[i])     otherwise,
 * the quotient and the product in float32, rounded once to grad_dtype.  An infinite norm makes the factor 0 (finite elements
 * become 0, infinite ones NaN), a NaN norm makes all elements NaN: a caller who would rather skip such a step looks at norms.
 * out[i] may be grads[i] (in place; a row that needs no scaling is then not written).  max_norm is finite and >= 0. */
int dadam_clip_grads(dadam_handle* h, const void* const* grads, void* const* out, float max_norm, float* norms,
                     void* hip_stream);

/* Messages: a vector in microscaled 4-bit floating point.  Block k is elements [32 k, 32 k + 32) of the packed vector, whatever
 * tensors they belong to (pack with align_elems = 32 for blocks that no two tensors share).  Bytes 16 k .. 16 k + 15 of a message
 * hold its codes, element 32 k + 2 j in the low half of byte j and 32 k + 2 j + 1 in the high half: a sign (8) and a magnitude
 * 0, 1/2, 1, 3/2, 2, 3, 4, 6 (0 to 7).  Byte scale_offset + k holds the block's power of two: b stands for 2^(b - 127), 255 makes
 * the whole block NaN.  (E2M1 elements and E8M0 scales of the OCP microscaling formats, blocks of 32.)  Codes of padding are 0. */
#define DADAM_MX4_BLOCK 32u
typedef struct {
  uint64_t n_blocks;     /* ceil(d / 32) */
  uint64_t scale_offset; /* 16 n_blocks */
  uint64_t bytes;        /* 17 n_blocks, rounded up to 16 */
} dadam_mx4_info;
int dadam_mx4_get_info(const dadam_handle* h, dadam_mx4_info* out);

/* What a worker sends.  For every row i, with u = x[i] - copy_in[i] in float32 (u = x[i] where copy_in is null) and, in every
 * block, a = max |u| over its elements:
 *     scale 2^e, e = max(floor(log2 a) - 2, -126);   q = u / 2^e to the nearest magnitude above, ties to the even code, at most 6
 *     msg[i] = the codes and scales;   copy_out[i] = copy_in[i] + q 2^e   (q 2^e where copy_in is null)
 * A block with an infinite or NaN u is sent as NaN (scale 255, codes 0).  copy_out may be null; copy_out[i] may be copy_in[i] (in place).
 * Sending differences against a copy that sender and receivers move alike (start it at x^(0), or at 0) is what makes so coarse a
 * message enough: what one round loses stays in the next round's difference. */
int dadam_mx4_encode(dadam_handle* h, const void* const* x, const float* const* copy_in, float* const* copy_out,
                     void* const* msg, void* hip_stream);

/* out[i] = sum_k w[k] * value(msg[col[k]]) over row i of the slot's neighbour list, or out[i] += that with DADAM_MX4_ADD: the rows of W
 * times vectors held in 4 bits.  msg has n_cols entries; those that no row lists are not read.  float32 sums in the order the row lists;
 * rows that list the same sources with the same weights share one sum, in order of the sources.
 * The identity matrix decodes. */
#define DADAM_MX4_ADD 1u
int dadam_mx4_product(dadam_handle* h, uint32_t slot, const void* const* msg, float* const* out, uint32_t flags,
                      void* hip_stream);

/* The gossip update of a worker that keeps ONE vector for all its neighbours, sum[i] = sum_k w[k] copy[col[k]]:
 *     sum[i] += sum_k w[k] * value(msg[col[k]]);      x_dst[i] = x_src[i] + gamma * (sum[i] - copy[i])
 * with copy[i] the worker's own public copy, already moved by its own message (dadam_mx4_encode), and that message among msg.
 * With a doubly stochastic W the replicas' mean does not move; 0 < gamma <= 1 (smaller for sparser graphs and coarser messages).  x_dst[i] may be x_src[i] (in place).
 * float32, one rounding of x_dst to param_dtype.
 * A sum belongs to one matrix, which no call can check.  It has to be sum_k w[k] copy[col[k]] before the first round (copies and sums all 0, or all the
 * x^(0) that the replicas have in common; replicas that start apart start from 0, or from copies that the sums are made of), and it stays that only if it takes
 * every round's messages with that matrix.  A program whose slots change from round to round therefore keeps a sum for every slot, and adds each
 * round's messages to all of them: dadam_mx4_gossip with the round's slot on that slot's sum, dadam_mx4_product with DADAM_MX4_ADD and the other slots on
 * theirs (a worker has to receive the messages of its neighbours in every slot, every round). */
int dadam_mx4_gossip(dadam_handle* h, uint32_t slot, const void* const* msg, float* const* sum, const float* const* copy,
                     const void* const* x_src, void* const* x_dst, float gamma, void* hip_stream);

/* One whole round where the handle holds every replica (n_rows == n_cols): dadam_mx4_encode of x_src against copy (in place) and
 * dadam_mx4_gossip of the messages, in one pass and with the same bits, the messages never leaving the chip.  x_dst[i] may be x_src[i].
 * The sums are those of dadam_mx4_gossip, of this slot's matrix from the first round on; the messages are not kept, so a program whose slots
 * change makes the two calls.
 * The messages of a piece of every row lie in LDS: 272 bytes a row up to 64 rows, 136 beyond (21760 at most).  DADAM_EINVAL if that is above
 * the handle's lds_limit_bytes: dadam_mx4_encode and dadam_mx4_gossip do the same there. */
int dadam_mx4_round(dadam_handle* h, uint32_t slot, const void* const* x_src, void* const* x_dst, float* const* copy,
                    float* const* sum, float gamma, void* hip_stream);

/* ------------------------------------------------------------------------------------------------------------
 * The ends of an iteration: the loss of a language model's head, and the step of its matrices along an orthogonalised direction
 *
 * These calls take a workspace: DEVICE memory, caller-owned, 256-byte aligned, that a call may overwrite throughout and that holds nothing between
 * calls.  Calls that may overlap in time need one each, and so do graphs that are replayed side by side.  The calls themselves allocate nothing, and may be
 * recorded into a graph.  With less workspace than `bytes` of the information calls (but `least_bytes`) they go in more, smaller launches: orthogonalised matrices
 * are the same bits then, losses and their gradients differ within what is said below.  Every call on the same inputs and as much workspace gives the same bits.
 * What a call writes must not overlap anything else that it reads or writes, but where "in place" is named.
 * Errors of all: DADAM_EINVAL (null, value out of range, workspace too small), DADAM_EALIGN, DADAM_EALIAS, DADAM_ESTATE, DADAM_EHIP. */

/* The output matrix of a language model: tensor `tensor` of the layout, vocab rows (one a word) of width elements, and the words' bias, another tensor, of
 * vocab elements, or DADAM_HEAD_NO_BIAS.  vocab is 1 to 2^24, width 1 to 65536. */
#define DADAM_HEAD_NO_BIAS 0xffffffffu
typedef struct {
  uint32_t tensor, bias_tensor;
  uint32_t vocab, width;
} dadam_head;

typedef struct {
  uint64_t least_bytes; /* the workspace without which a call is refused: one replica and 128 words at a time */
  uint64_t bytes;       /* what a call makes good use of */
} dadam_head_info;
/* The workspace of dadam_head_loss for n_tokens tokens a row, with (gradient != 0) or without gradients. */
int dadam_head_get_info(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens, uint32_t gradient, dadam_head_info* out);

/* Softmax cross entropy of every row's hidden vectors against its own head: with W and bias in
 * params[i], h_t the t-th of hidden[i]'s n_tokens vectors of width elements, y_t = targets[i][t]
 *     z = W h_t + bias;    nll[i][t] = log sum_v exp z[v] - z[y_t];    losses[i] = s * sum_t nll[i][t]
 *     dz_t = s (softmax z - e[y_t]);    dhidden[i][t] = W^T dz_t;    in grads[i]: dW = sum_t dz_t h_t^T, dbias = sum_t dz_t
 * s is scale, with DADAM_HEAD_MEAN divided by the number of row i's tokens that have a target.  A token whose target is negative or vocab and above has none: it takes no
 * part (nll 0, dhidden 0), whatever its hidden vector holds.  With DADAM_HEAD_ADD dW and dbias are added to what grads holds (a head that
 * is the embedding too, or gradients of several calls), otherwise written; other elements of grads are not touched.
 * params: n_rows packed vectors of param_dtype; hidden and dhidden: n_rows times n_tokens x width of param_dtype; targets: int32; losses (n_rows, DEVICE) and nll: float32;
 * grads: n_rows packed vectors of grad_dtype.  nll, dhidden and grads may be null; without the last two only the loss is formed.  Of all these only params and grads
 * have to be 16-byte aligned, the others by their elements.  n_tokens is 0 to 2^20;
 * buffers of no tokens are not looked at (a table of nulls will do).
 * The logits are kept for up to 64 tokens (4 bytes each).  Of more tokens only softmax is, 2 bytes a logit with bfloat16 parameters and gradients and 4 otherwise, and
 * only where a replica's is at most 2 GiB and the workspace has room for it; elsewhere they are formed twice, a piece of the vocabulary at a time.
 * Sums are float32 (the loss 64 bits).  With bfloat16 parameters and gradients softmax - e[y] is rounded to bfloat16 before the gradients' products (where it is kept, to half
 * precision before that: 2^-11 of itself or 2^-40 of the largest of its 64 or 128 words); otherwise operands have 22 bits, or 2^-39 of the largest magnitude of the head,
 * of the hidden vectors or (softmax) of 1.  An infinity or NaN in W, or in a hidden vector that takes part, leaves its own replica's loss and gradients without
 * meaning, and no other's; a bias of minus infinity takes its word out. */
#define DADAM_HEAD_MEAN 1u
#define DADAM_HEAD_ADD 2u
int dadam_head_loss(dadam_handle* h, const dadam_head* head, const void* const* params, const void* const* hidden,
                    const int32_t* const* targets, uint32_t n_tokens, float scale, uint32_t flags, float* losses, float* const* nll,
                    void* const* dhidden, void* const* grads, void* workspace, uint64_t workspace_bytes, void* hip_stream);

/* A matrix of the packed layout: element (r, c) is element first + r * ld + c of the tensor.  Several may share a tensor (projections that are
 * fused side by side) but no element, and columns do not run on into the next row: first % ld + cols <= ld.  scale multiplies the orthogonalised direction
 * (for instance sqrt(max(1, rows / cols)), or 0.2 sqrt(max(rows, cols)) for updates of Adam's size).  flags must be 0. */
typedef struct {
  uint32_t tensor;
  uint32_t rows, cols; /* 1 to 65536 */
  uint32_t ld;         /* >= cols */
  uint64_t first;
  float scale;
  uint32_t flags;
} dadam_matrix_desc;

/* Register the matrices that the two calls below are about, in place of those registered before; n may be 0.  matrices[n] is a HOST array and is
 * copied.  Allocates and uploads 144 bytes a matrix and up to 16 bytes for every 128 x 128 elements, and may wait for the device: not for use under stream capture, and
 * only while no launched work still uses the old ones. */
int dadam_set_matrices(dadam_handle* h, const dadam_matrix_desc* matrices, uint32_t n);

/* The iterations that orthogonalise: coefficients[3 k ...] (HOST) are a, b, c of iteration k.  The default is five times 3.4445, -4.7750, 2.0315, which takes
 * singular values from about 0.01 on to between 0.7 and 1.2.  DADAM_EINVAL where a singular value of up to 1 would go beyond 1024 on the way. */
#define DADAM_ORTHO_MAX_STEPS 16u
int dadam_set_ortho_schedule(dadam_handle* h, uint32_t n_steps, const float* coefficients);

typedef struct {
  uint32_t n_matrices, reserved;
  uint64_t least_bytes; /* the workspace without which a call is refused: that of one replica's largest matrix; 0 where every
                           matrix fits a compute unit (for instance 128 x 160 or 64 x 416 at most), and workspace may be null */
  uint64_t bytes;       /* what a call makes good use of */
} dadam_ortho_info;
int dadam_ortho_get_info(const dadam_handle* h, dadam_ortho_info* out);

/* Every registered matrix M of every row i brought near its orthogonal polar factor by Newton-Schulz iterations:
 *     X = M / (|M| + 1e-7)   (Frobenius norm, summed in 64 bits);   every iteration:  A = X X^T,  X = a X + (b A + c A A) X
 * (of a matrix with more rows than columns, its transpose's).  in and out: n_rows buffers of cfg.d elements of grad_dtype; out[i] may be in[i] (in place).
 * Elements outside the matrices are neither used nor written.  A matrix of zeros stays one; a NaN or an infinity makes its own matrix NaN and no other.
 * float32 results come from operands of 22 bits, bfloat16 results from operands of 11 bits (X itself of 22), sums are float32: the error is about 3e-6 and 2e-3 of
 * the result (2-norms). */
int dadam_orthogonalize(dadam_handle* h, const void* const* in, void* const* out, void* workspace, uint64_t workspace_bytes, void* hip_stream);

/* The step of the registered matrices along the orthogonalised first moment, in iteration t of Algorithm 3 and on the bound buffers: with
 *     m = beta1 * m_hat_i + (1 - beta1) * g_i                               line 6
 *     u = m,  or  beta1 * m + (1 - beta1) * g_i  with DADAM_ORTHO_NESTEROV
 *     x_dst_i = sum_k w[k] * x_src[col[k]] - lr * (scale * O(u) + weight_decay * x_src[i])       O: dadam_orthogonalize of the matrix
 * and with DADAM_FUSE_ACCUM lines 9 to 13 for m_hat and b (v_hat takes no part).  O does not depend on the length of u, so there is no bias correction.  Elements outside
 * the matrices are left to dadam_gossip_step_range over the other tensors.  Arguments as there, and the same rules for updates in place: x_dst[i] may be a source that no
 * other row reads.  Precision of O by param_dtype; sums over neighbours and the step in float32, one rounding to param_dtype. */
#define DADAM_ORTHO_NESTEROV 8u
int dadam_ortho_step(dadam_handle* h, uint32_t slot, const void* const* grads, uint64_t t, uint32_t flags, void* workspace,
                     uint64_t workspace_bytes, void* hip_stream);

/* Text of the last error recorded on this handle ("" if none).  With h == NULL: the text of the
 * last dadam_init failure of the calling thread.  The pointer stays valid until the next call on
 * the same handle (thread). */
const char* dadam_last_error(const dadam_handle* h);

/* Free the handle and its metadata.  The caller makes sure launched work has finished. */
void dadam_destroy(dadam_handle* h);

#ifdef __cplusplus
}
#endif
#endif /* DADAM_H_ */
