/*
 * moe_cache.h - C ABI of the batch-1 MoE decode path with cache-conditional routing.
 *
 * One MoE layer step for one token is
 *   z = W_gate x, w = softmax(z)                                  (paper Eq. 3)
 *   z' = z + lambda * Delta_avg * m~_t, select top-K of z'          (Sec. 3.3, Eq. 9, Eq. 10)
 *   hits/misses against the cache as it stood before the token     (Sec. 2.2, Eq. 4)
 *   LRU update of the expert cache                                 (Sec. 4.2)
 *   y = sum_k w_k E_k(x) (+ shared expert), E = SwiGLU             (Eq. 1)
 * The paper's DRAM tier is a pool of `capacity` expert slots per layer in device memory,
 * its Flash tier is pinned host memory holding every expert; a miss is filled by an
 * asynchronous host-to-device copy on `copy_stream`.
 *
 * Conventions
 *  - Every function returns MOE_OK or a negative moe_status; nothing throws or aborts.
 *    moe_last_error() gives a message for the calling thread's last failure.
 *  - "device" pointers are HIP device memory, "host" pointers ordinary host memory, "pinned"
 *    is page-locked host memory.  All buffers handed in are BORROWED: the caller allocates them,
 *    keeps them alive until moe_cache_destroy and frees them afterwards.  The library allocates
 *    only its own small tables (state, route records, partial sums).
 *  - Streams are hipStream_t passed as void*; both are borrowed.  Calls on one context must come
 *    from one thread at a time.
 *  - Expert ids are 0..n_experts-1, slots 0..capacity-1.  n_experts <= 64, top_k <= 8.
 *  - Environment variables read by moe_cache_init (all optional):
 *      MOE_HOST_SYNC=event     the host waits for a routing decision on a stream event instead of polling the
 *                              words the router stores into mapped host memory
 *      MOE_FUSE_BOUNDARY=0|1   overrides the rule that decides whether a non-blocking moe_stack_route_step runs
 *                              inside the layer's expert launch (see moe_cache_plan)
 *      MOE_ROUTE_EVERYWHERE=0|1 overrides the rule that decides whether, where it does not, the routing is left to every
 *                              workgroup of the expert launch (hidden 512, 1024, 2048, 4096; 256 with fp32)
 *      MOE_POISON_FILLS=1      debugging aid: a slot is overwritten with 0xff bytes (NaNs in every format's
 *                              scales or weights) on the copy stream right before its fill, so that anything
 *                              computed from a slot before its fill has landed shows up as NaN in the output
 *      MOE_TAG_SPINS=n         polls before a workgroup stops waiting for the first workgroup of its own launch
 *                              (a test lowers it to reach the error path described at moe_stack_route_step)
 */
#ifndef MOE_CACHE_H
#define MOE_CACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MOE_MAX_EXPERTS 64
#define MOE_MAX_TOPK 8
/* the operators on many rows: experts and width at most; rows, and tokens times top_k, fewer than */
#define MOE_ROWS_MAX_EXPERTS 512
#define MOE_ROWS_MAX_HIDDEN 8192
#define MOE_ROWS_LIMIT (1 << 26)
/* attention: the width of a head, heads and sequences at most */
#define MOE_ATTEND_MAX_DIM 128
#define MOE_ATTEND_MAX_HEADS 256
#define MOE_ATTEND_MAX_SEQS 16384

typedef struct moe_cache moe_cache_t; /* opaque, owned by the library */

enum moe_status { MOE_OK = 0, MOE_EINVAL = -1, MOE_ENOMEM = -2, MOE_EHIP = -3, MOE_ESTATE = -4 };
enum moe_weight_fmt { MOE_W_FP32 = 0, MOE_W_BF16 = 1, MOE_W_INT8_PC = 2, MOE_W_INT4_G128 = 3 };
enum moe_act_fmt { MOE_A_FP32 = 0, MOE_A_BF16 = 1 };
/* elements of rows (the row operators below); 8-bit codes stand for code * scale of their row */
enum moe_row_fmt { MOE_R_FP32 = 0, MOE_R_BF16 = 1, MOE_R_INT8 = 2 };
/* The logit range Delta that scales the prior (Eq. 9-10; App. D on the choice of the estimate): the running mean
 * over the tokens seen since the last reset (the paper's method), a fixed value given by the caller (e.g. from a
 * calibration set), or the current token's own range max z - min z. */
enum moe_delta_mode { MOE_DELTA_RUNNING_MEAN = 0, MOE_DELTA_FIXED = 1, MOE_DELTA_TOKEN = 2 };
/* How the ranking vector is altered before the top-K cut.  CACHE_PRIOR is the paper's method
 * (Sec. 3.3); MAX_RANK (Sec. 3.1, Eq. 6-7) and CUMSUM (Sec. 3.2, Eq. 8) are its two baselines. */
enum moe_route_mode { MOE_ROUTE_CACHE_PRIOR = 0, MOE_ROUTE_MAX_RANK = 1, MOE_ROUTE_CUMSUM = 2 };

typedef struct moe_cache_config {
  int32_t n_layers;
  int32_t hidden;       /* d; a multiple of 64 * (16 / bytes per weight) */
  int32_t n_experts;    /* N <= 64 */
  int32_t inter;        /* I, SwiGLU intermediate of a routed expert */
  int32_t shared_inter; /* intermediate of the always-on shared expert, 0 = none */
  int32_t top_k;        /* K <= 8 */
  int32_t top_j;        /* router's own top-J always selected (Sec. 3.3), 0..top_k */
  int32_t capacity;     /* expert slots per layer, top_k <= capacity <= n_experts */
  int32_t weight_fmt;   /* moe_weight_fmt of expert blobs */
  int32_t act_fmt;      /* moe_act_fmt of x, y and the router matrix */
  int32_t renormalize;  /* 1: divide the K weights by their sum (Sec. 2.1) */
  int32_t delta_mode;   /* moe_delta_mode */
  int32_t route_mode;   /* moe_route_mode */
  int32_t max_rank;     /* M of Eq. 6 (MOE_ROUTE_MAX_RANK) */
  float lambda;         /* >= 0, strength of the cache prior (Eq. 9) */
  float delta_fixed;    /* Delta_avg when delta_mode == MOE_DELTA_FIXED */
  float cumsum_p;       /* p of Eq. 8 (MOE_ROUTE_CUMSUM) */
  int32_t reserved;
  void *compute_stream; /* hipStream_t for kernels */
  void *copy_stream;    /* hipStream_t for miss fills; must differ from compute_stream */
} moe_cache_config_t;

typedef struct moe_cache_buffers {
  const void *const *host_expert_blob; /* [n_layers*n_experts] pinned host, packed blobs (moe_pack_expert) */
  void *const *slot_pool;              /* [n_layers] device, capacity*moe_slot_bytes(cfg) each, 256-byte aligned */
  const void *const *gate_w;           /* [n_layers] device, router matrix [N,d] row-major, act_fmt */
  const void *const *shared_blob;      /* [n_layers] device packed blob of the shared expert, or NULL */
  const int32_t *initial_resident;     /* host [n_layers*n_initial] experts preloaded into slots 0.., or NULL */
  int32_t n_initial;                   /* 0..capacity (App. G: empty or random initial cache) */
} moe_cache_buffers_t;

/* What one routing step decided; entries 0..top_k-1 are valid, ranked by the altered logits. */
typedef struct moe_route_out {
  int32_t sel_expert[MOE_MAX_TOPK];
  int32_t sel_slot[MOE_MAX_TOPK];   /* slot each selected expert occupies after the step */
  float sel_weight[MOE_MAX_TOPK];   /* softmax of the UNMODIFIED logits (Sec. 3.3), renormalised if asked */
  int32_t miss[MOE_MAX_TOPK];       /* 1 if the expert was not resident before the step (Eq. 4) */
  int32_t evicted[MOE_MAX_TOPK];    /* expert that lost its slot to this one, or -1 */
  int32_t n_miss;
  int32_t token;                    /* index of this step within the layer, from 0 */
  float delta;                      /* Delta_avg used (Eq. 10) */
  float margin;                     /* gap between the K-th and (K+1)-th altered logit */
  float logits[MOE_MAX_EXPERTS];    /* z, as used */
  uint32_t opaque[4];               /* the library's own compact copy of the decision (read by its expert kernels);
                                     * not part of the interface: do not interpret, do not rely on */
} moe_route_out_t;

typedef struct moe_cache_stats {
  int64_t tokens, selections, hits, misses, cold_misses, evictions, bytes_filled;
  int64_t lifetime_sum; /* over the evictions: tokens between an expert's load and its eviction; divided by
                         * `evictions` it is the average cache lifetime of Sec. 4.6 / Table 2 */
} moe_cache_stats_t;

/* Per-layer tables, for checking against a reference (host struct). */
typedef struct moe_cache_tables {
  int32_t expert_slot[MOE_MAX_EXPERTS]; /* expert -> slot or -1 */
  int32_t slot_expert[MOE_MAX_EXPERTS]; /* slot -> expert or -1 */
  int64_t stamp[MOE_MAX_EXPERTS];       /* recency stamp of resident experts: token*K + position */
  float delta_sum;                      /* running sum of max(z)-min(z) (Eq. 10) */
  int32_t count;                        /* tokens seen */
} moe_cache_tables_t;

/* Bytes of one packed expert with intermediate size `inter` (0 on invalid arguments).  A slot and a
 * host blob are moe_blob_bytes(fmt, hidden, cfg.inter); the shared blob uses cfg.shared_inter. */
size_t moe_blob_bytes(int32_t weight_fmt, int32_t hidden, int32_t inter);
/* Bytes of one expert slot of the fast tier for this configuration (Sec. 2.2: the cache holds whole experts), so
 * that the caller can size slot_pool (capacity * moe_slot_bytes per layer) and the host blobs.  Only weight_fmt,
 * hidden and inter are read.  0 on NULL or an unsupported shape. */
size_t moe_slot_bytes(const moe_cache_config_t *cfg);

/* Pack one expert from canonical row-major weights into the blob layout the kernels stream
 * (record i = gate row i | up row i | column i of down).  All pointers are device memory:
 *  fp32/bf16: gate,up [I,d], down [d,I] of that type; scale pointers NULL.
 *  int8: int8 values as above, fp16 scales gate_s,up_s [I], down_s [d] (one per output row).
 *  int4: bytes [I,d/2], [I,d/2], [d,I/2] (nibble = q+8, even column low), fp16 scales
 *        [I,d/128], [I,d/128], [d,I/128] (Sec. 4.5 names 4- and 8-bit weights; the format is ours).
 * Runs asynchronously on `stream`.  MOE_EINVAL on bad shapes/NULLs, MOE_EHIP on launch failure. */
int moe_pack_expert(int32_t weight_fmt, int32_t hidden, int32_t inter, const void *gate, const void *up,
                    const void *down, const void *gate_s, const void *up_s, const void *down_s, void *blob_dev,
                    void *stream);

/* Create a context (problem statement of Sec. 2.1-2.2 and 3.3).  Validates everything before touching
 * the GPU (MOE_EINVAL), preloads initial residents synchronously, leaves the cache otherwise empty. */
int moe_cache_init(const moe_cache_config_t *cfg, const moe_cache_buffers_t *bufs, moe_cache_t **out);
void moe_cache_destroy(moe_cache_t *ctx);

/* Routing step of one layer for one token (Eq. 3, Eq. 9-10, Eq. 4, Sec. 4.2): exactly one of x_dev
 * (device [d], act_fmt: the router GEMV is computed) and logits_dev (device [N] fp32: used as z) is
 * non-NULL.  logits_dev must stay unchanged until this call (out_host given) or the layer's moe_expert_forward has
 * returned.  x_dev is read by kernels of both calls and must stay unchanged until compute_stream has run them.
 * With out_host non-NULL the call returns once the decision is known on the host (written to *out_host)
 * and the copies filling missed experts' slots are enqueued on copy_stream.  With out_host NULL the call
 * only enqueues the router kernel or, with x_dev and where the rule for MOE_BOUNDARY_ROUTED_EVERYWHERE holds (any size from
 * d = 1024 on, below that 10 MB a layer-token; Cumsum-Threshold with int4 later), the gate logits alone: the expert launch
 * then routes by itself.  moe_expert_forward takes care of the fills (see there).
 * MOE_ESTATE if the layer's previous step has not been followed by moe_expert_forward. */
int moe_route_step(moe_cache_t *ctx, int32_t layer, const void *x_dev, const float *logits_dev,
                   moe_route_out_t *out_host);

/* Eq. 1 for the layer's last routing step: y = sum_k w_k E_k(x) + shared(x); x_dev (the vector given to
 * moe_route_step), y_dev device [d] in act_fmt.  The kernels are asynchronous on compute_stream.
 * After a routing step that was waited for, a first launch covers the shared expert and the experts that were
 * resident, a second one (behind the fills) the experts that were missing.
 * After one that was not (out_host NULL), one launch covers everything: it reads the experts that miss from the host
 * blobs itself, computes with them and puts them into their slots on the way; the call returns at once (after a step
 * on given logits: once these have been read).  Whatever its kernels read - x_dev, h_dev and a_dev of a
 * moe_stack_route_step, the host blobs - then has to stay valid and unchanged until compute_stream has run them, not only
 * until the call returns.  That needs all host blobs in pinned memory that the device can read; where some are not (or with
 * MOE_DEVICE_FILLS=0 in the environment at moe_cache_init) the call waits for the decision, enqueues the fills on
 * copy_stream and proceeds as above.
 * A step cannot be captured into a graph (MOE_EHIP).  MOE_ESTATE without a preceding moe_route_step.
 * y_dev may be NULL: the output then stays inside the library as fp32 partial sums and is finished by the next
 * moe_stack_route_step (of any layer), which must follow before another moe_expert_forward. */
int moe_expert_forward(moe_cache_t *ctx, int32_t layer, const void *x_dev, void *y_dev);

/* Prompt phase: n_tokens (1..128) tokens of one layer in one call.  The paper applies its routing during generation and
 * leaves prompt processing to batched kernels (Sec. 4.5; App. F varies the prompt length); here a batch is routed as
 * its tokens one after the other - the cache bitmask m_t of Sec. 3.3 is the state after token t-1, also inside a batch -
 * so decisions, slots, evictions, Delta_avg (Eq. 10) and the miss counts of Eq. 4 are exactly those of n_tokens calls of
 * moe_route_step in the same order; only the arithmetic is batched (matrix cores).
 * moe_route_batch: exactly one of x_dev (device [n_tokens, d], act_fmt: the gate logits are computed) and logits_dev
 *   (device [n_tokens, N] fp32) is non-NULL.  Returns once all decisions are on the host; out_host (may be NULL)
 *   receives n_tokens records.  x_dev must stay unchanged until moe_expert_forward_batch: with x_dev the expert kernels of a
 *   batch that nothing misses in are enqueued behind the routing by this call already, and the other only adds the sum.
 * moe_expert_forward_batch: y[t] = sum_k w_k E_k(x[t]) + shared(x[t]) (Eq. 1) for every token of the batch routed
 *   last; x_dev as given to moe_route_batch, y_dev device [n_tokens, d] in act_fmt.  Tokens are grouped per expert;
 *   where a slot is refilled inside the batch after an earlier token has read it, the batch is cut there and the
 *   parts run one after the other; within a part the experts that are resident (and the shared expert) are computed
 *   while the part's fills stream, the filled ones behind them.  The partial results are added in a fixed order (y
 *   is reproducible bit for bit).  Returns when y is complete.
 * Shapes: bf16 weights and activations, hidden 1024 or 2048, intermediate sizes that are multiples of 16;
 * MOE_EINVAL otherwise.  MOE_ESTATE if a single-token step of the layer or an expert output is pending, or if
 * moe_expert_forward_batch does not follow a moe_route_batch of the same layer and size. */
int moe_route_batch(moe_cache_t *ctx, int32_t layer, const void *x_dev, const float *logits_dev, int32_t n_tokens,
                    moe_route_out_t *out_host);
int moe_expert_forward_batch(moe_cache_t *ctx, int32_t layer, const void *x_dev, void *y_dev, int32_t n_tokens);

/* moe_expert_forward for callers that cannot allocate device memory or hold a context: code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation.  Computes y = sum_k w_k E_k(x) + shared(x) for experts that are
 * all in their slots, with the kernels moe_expert_forward uses.  The call allocates nothing (no hipMalloc / hipFree, no
 * memset): the selection travels in the launch's arguments, and the fp32 partial rows live in a fixed 4 MiB device array
 * inside the library, one per GPU, held until the process ends.  Hence the limits: hidden <= 4096, at most 256
 * workgroups; larger shapes are refused with MOE_EINVAL.  Every call on a GPU shares that GPU's array: calls that
 * overlap in time on one GPU (different streams, different threads) race; calls on one stream are ordered.
 *   slot_pool_dev   device, n_slots slots of moe_blob_bytes(weight_fmt, hidden, inter) each, 256-byte aligned
 *   shared_blob_dev device packed shared expert (shared_inter > 0) or NULL
 *   sel_slot_host, sel_weight_host   HOST arrays [top_k]: the slot of each selected expert and its weight (read
 *                   before the call returns; slots are checked against n_slots)
 *   x_dev, y_dev    device [hidden] in act_fmt; y is complete when `stream` reaches the end of the two kernels
 *                   this call enqueues.  The device of `stream` must be current. */
int moe_expert_forward_static(int32_t weight_fmt, int32_t act_fmt, int32_t hidden, int32_t inter, int32_t shared_inter,
                              int32_t top_k, const void *slot_pool_dev, int32_t n_slots, const void *shared_blob_dev,
                              const int32_t *sel_slot_host, const float *sel_weight_host, const void *x_dev,
                              void *y_dev, void *stream);

/* Layer boundary of a multi-layer stack (workload glue fused with the router kernel: Eq. 3, 9, 10, 4, Sec. 4.2):
 *   y  = the expert output left pending by moe_expert_forward(..., y_dev = NULL), if any
 *   h  = carry ? h + y + perturb * a : perturb * a  (a may be NULL; carry = 0 starts a new token)
 *   x  = h / sqrt(mean(h^2) + 1e-6), rounded to act_fmt, written to x_dev
 *   then the routing step of `layer` on x, exactly as moe_route_step(ctx, layer, x_dev, NULL, out_host).
 * h_dev: device fp32 [d] in/out; a_dev: device fp32 [d] or NULL; x_dev: device act_fmt [d] (pass it to the
 * layer's moe_expert_forward); y_dev: device act_fmt [d] or NULL, receives the finished pending output.
 * hidden must be at most 8192.  Same blocking rule and errors as moe_route_step.
 * With out_host NULL the library may defer x and the routing into the layer's expert launch (its first workgroup
 * does them while the others already stream the shared expert; see moe_cache_plan), or the routing alone (every
 * workgroup then works the decision out from the logits): x_dev and the routing record may then be written by the kernels
 * moe_expert_forward enqueues, not by this call's, so nothing but moe_expert_forward(ctx, layer, x_dev, ...) and
 * further calls of moe_stack_route_step may use h_dev and x_dev in between (a_dev is read by a kernel that this call
 * enqueues and must stay unchanged until compute_stream has run it), and that call must be given the same x_dev
 * (another one is refused with MOE_EINVAL where the shape has the first form and a third of a layer's records or more are
 * the shared expert's).  Counters, tables and snapshots taken in between include the step.
 * The other workgroups' wait for the first one is bounded; should it ever run out, they finish without the routed
 * experts, and every later call that names a layer returns MOE_EHIP until moe_cache_reset. */
int moe_stack_route_step(moe_cache_t *ctx, int32_t layer, float *h_dev, const float *a_dev, float perturb,
                         int32_t carry, void *x_dev, void *y_dev, moe_route_out_t *out_host);

/* The last routing decision of a layer that has reached the host (after a blocking moe_route_step, or after
 * the moe_expert_forward that followed a non-blocking one).  MOE_ESTATE if a decision is still pending. */
int moe_cache_last_route(moe_cache_t *ctx, int32_t layer, moe_route_out_t *out_host);

/* Counters of one layer, or summed over layers with layer = -1 (Eq. 4 numerators/denominators).
 * Synchronises compute_stream.  MOE_EHIP after an abandoned hand-over (see moe_stack_route_step), like every
 * other call on a context in that state. */
int moe_cache_stats(moe_cache_t *ctx, int32_t layer, moe_cache_stats_t *out_host);
/* Slot table, stamps and Delta accumulator of one layer.  Synchronises compute_stream. */
int moe_cache_tables(moe_cache_t *ctx, int32_t layer, moe_cache_tables_t *out_host);
/* Save / restore the cache state of one layer (slot tables, stamps, Delta_avg accumulator of Eq. 10, counters of
 * Eq. 4) as an opaque host blob, e.g. to resume a decode or to start a comparison from a recorded state.
 * moe_cache_snapshot: *bytes holds the size of buf_host on entry and the size of the blob on return; with
 * buf_host NULL only the size is returned.  MOE_EINVAL if the buffer is too small.  Synchronises compute_stream.
 * moe_cache_restore: checks that the blob was taken from a context of the same n_experts / capacity / top_k and
 * that its tables are consistent (MOE_EINVAL otherwise, nothing changed), then installs it and copies every
 * resident expert's blob from the host tier into its slot, synchronously.  MOE_ESTATE while a routing step of
 * the layer or an expert output is pending. */
int moe_cache_snapshot(moe_cache_t *ctx, int32_t layer, void *buf_host, size_t *bytes);
int moe_cache_restore(moe_cache_t *ctx, int32_t layer, const void *buf_host, size_t bytes);
/* Change the strength lambda of the cache prior (Eq. 9: z' = z + lambda * Delta_avg * m~_t; Sec. 3.3 sweeps it as
 * the knob between the original routing, lambda = 0, and fully cache-driven routing) from the next routing step on.
 * Finite and >= 0, else MOE_EINVAL.  Does not touch the cache or Delta_avg. */
int moe_cache_set_lambda(moe_cache_t *ctx, float lambda);
/* Switch between the paper's method and its two list-based baselines (Sec. 3.1-3.2) and set M of Eq. 6 / p of Eq. 8. */
int moe_cache_set_baseline(moe_cache_t *ctx, int32_t route_mode, int32_t max_rank, float cumsum_p);
/* Start a new evaluation: empty every layer's cache (then preload the initial residents again, App. G), restart
 * the running mean Delta_avg of Eq. 10 (sum and token count to zero) and the hit/miss counters of Eq. 4; drops
 * pending steps and outputs and clears the error state described at moe_stack_route_step.  Synchronises both
 * streams. */
int moe_cache_reset(moe_cache_t *ctx);

/* Workload glue for multi-layer synthetic stacks (not part of the paper's method):
 * h = (carry ? h : 0) + y + perturb * a (y, a may be NULL); x = h / sqrt(mean(h^2) + 1e-6) rounded to act_fmt.
 * h: device fp32 [d] in/out; y: device act_fmt [d] or NULL; a: device fp32 [d] or NULL; x: device act_fmt [d].
 * carry = 0 starts a new token (h is overwritten). */
int moe_residual_rmsnorm(float *h_dev, const void *y_dev, const float *a_dev, float perturb, int32_t carry,
                         void *x_dev, int32_t hidden, int32_t act_fmt, void *stream);

/* Offline analysis of a recorded selection trace; host memory only, no GPU work, no context.
 * trace[t*top_k + k]: the experts one layer selected at token t (distinct, each in 0..n_experts-1), in the order
 * the cache touches them (descending router weight, Sec. 4.2).  Misses are counted per token against the cache
 * before the token (Eq. 4), starting from `initial` (n_initial experts, may be NULL/0).
 *   MOE_POLICY_LRU       least-recently-used eviction as in Sec. 4.2; any capacity in 1..n_experts (below top_k
 *                        only the most recently touched experts of a token stay: the cache-size sweep of Sec. 4.8)
 *   MOE_POLICY_FARTHEST  evict the resident expert, not needed by the current token, whose next use is farthest
 *                        (never again first, ties to the lowest id): the optimal-eviction bound of Sec. 4.8;
 *                        needs capacity >= top_k
 * Outputs: *misses; optionally (may be NULL) *lifetime_sum and *evictions as in moe_cache_stats_t.
 * MOE_EINVAL on NULL/out-of-range arguments or a token with repeated experts. */
enum { MOE_POLICY_LRU = 0, MOE_POLICY_FARTHEST = 1 };
int moe_trace_misses(const int32_t *trace, int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t capacity,
                     int32_t policy, const int32_t *initial, int32_t n_initial, int64_t *misses,
                     int64_t *lifetime_sum, int64_t *evictions);

/* The launch shape the context chose for the expert kernels, and whether a moe_stack_route_step without out_host
 * runs x and its routing in the first workgroup of the layer's expert launch (bf16 activations, a supported shape, and,
 * other than int4, a shared expert of at least a third of the layer's records and 20 KB of them per hidden column;
 * MOE_FUSE_BOUNDARY=0 or 1 in the environment at moe_cache_init overrides the last condition). */
typedef struct moe_cache_plan {
  int32_t grid, wavefronts, depth, packed_bf16_dot, boundary_in_expert_launch;
} moe_cache_plan_t;
int moe_cache_plan(moe_cache_t *ctx, moe_cache_plan_t *out_host);
/* How a moe_stack_route_step without out_host is run: all of it by launches of its own, x and the routing in the first
 * workgroup of the layer's expert launch (boundary_in_expert_launch above), or the routing in every workgroup of it. */
enum { MOE_BOUNDARY_OWN_LAUNCH = 0, MOE_BOUNDARY_IN_FIRST_WORKGROUP = 1, MOE_BOUNDARY_ROUTED_EVERYWHERE = 2 };
int moe_cache_boundary_form(moe_cache_t *ctx, int32_t *out_host);
/* Who brings in the experts that miss in a step that nobody waits for (see moe_expert_forward): the host, with copies that
 * it enqueues once it knows the decision, or the expert launch. */
enum { MOE_FILLS_BY_HOST = 0, MOE_FILLS_IN_EXPERT_LAUNCH = 1 };
int moe_cache_fill_form(moe_cache_t *ctx, int32_t *out_host);

/* Average duration in microseconds of the timed expert-GEMV launches that covered a whole layer (no expert missing)
 * since the last call with reset != 0, and their count; measured with start/stop events attached to the launches
 * on compute_stream.  enable = 0 switches the timing off, enable = n > 0 times every n-th first-pass launch from
 * this call on (1 = all of them; events on every launch slow the host down to where the device idles between
 * launches, a stride co-prime to the layer count samples every layer without that); at most 32768 launches are
 * timed between two resets, later ones run untimed.  Each timed launch is preceded by a 50 us hold of the stream,
 * so that the kernel is already queued behind its start marker when the device reaches the marker. */
int moe_cache_profile(moe_cache_t *ctx, int32_t enable, int32_t reset, double *avg_us, int64_t *launches);

/* ---- Many rows at once: a layer of a long prompt or of a training batch whose experts are all in device memory ----
 *
 * The calls below need no context, allocate nothing and wait for nothing: they check their arguments (MOE_EINVAL), enqueue
 * their kernels on `stream` (whose device must be current) and return; all pointers are device memory.  They may be captured
 * into a graph.  Rows are dense (row i at i * hidden elements) where no stride is given; strides count elements.
 * hidden <= MOE_ROWS_MAX_HIDDEN, n_rows and n_tokens * top_k < MOE_ROWS_LIMIT, experts <= MOE_ROWS_MAX_EXPERTS, top_k <=
 * MOE_MAX_TOPK: other sizes are refused before a pointer is looked at.  Elements are aligned to their type (the experts' rows to 16
 * bytes).  n_rows or n_tokens 0 is no error.
 * Sums and statistics are held in 32 bits; results are the same bit for bit from call to call.
 *
 * moe_norm_rows: h_out = h + y (rounded to h_fmt), x = h_out * rstd * gain, rstd = 1 / sqrt(mean(h_out^2) + eps).
 *   y_dev NULL: h_out = h, h_out_dev may then be NULL.  gain_dev (fp32 [hidden]) NULL: ones.  h_fmt, y_fmt: fp32 or bf16.
 *   h_out_dev may be h_dev itself where h_stride is hidden.  rstd_dev (fp32 [n_rows]) may be NULL; the backward needs it.
 *   x_fmt MOE_R_INT8: with v = h_out * gain and top the largest |v| of the row, code = round(v * (127 * (1 / top))) (32-bit steps, to even) and
 *   scale_dev[row] = top / 127 * rstd, so that code * scale stands for x.  A row with top < 1e-30 has codes and scale 0, one
 *   that holds an infinity or NaN codes 0 and scale NaN.  Other formats: scale_dev is NULL.
 * moe_norm_rows_backward: gradients of h (and of y) and of gain, from those of x and of h_out:
 *   n = h_out * rstd, dh = dh_out + rstd (dx gain - n mean(dx gain n)), dgain = sum over the rows of dx n (fp32 [hidden]).
 *   h_out_dev, rstd_dev: as moe_norm_rows left them.  dx_dev: x_fmt fp32 or bf16.  dh_in_dev (h_fmt, the gradient of h_out) may
 *   be NULL, and so may dgain_dev.  dh_dev: h_fmt, may be dh_in_dev.  With dgain_dev a workspace of
 *   moe_norm_rows_backward_bytes(n_rows, hidden) bytes, 16-byte aligned, is needed. */
int moe_norm_rows(const void *h_dev, int32_t h_fmt, int64_t h_stride, const void *y_dev, int32_t y_fmt, int64_t y_stride,
                  const float *gain_dev, float eps, int32_t n_rows, int32_t hidden, void *h_out_dev, void *x_dev, int32_t x_fmt,
                  float *scale_dev, float *rstd_dev, void *stream);
size_t moe_norm_rows_backward_bytes(int32_t n_rows, int32_t hidden);
int moe_norm_rows_backward(const void *h_out_dev, int32_t h_fmt, const float *gain_dev, const float *rstd_dev, const void *dx_dev,
                           int32_t x_fmt, const void *dh_in_dev, int32_t n_rows, int32_t hidden, void *dh_dev, float *dgain_dev,
                           void *workspace_dev, size_t workspace_bytes, void *stream);

/* Tokens sorted by expert.  ids_dev [n_tokens, top_k]: the expert of each place (token, k); an id outside 0..n_experts-1 (-1)
 * is a place without an expert.  An expert's rows are its places in the order of the tokens:
 *   offsets_dev [n_experts + 1]       expert e has rows offsets[e] .. offsets[e + 1] - 1
 *   row_of_dev  [n_tokens, top_k]     row of each place, -1: none
 *   entry_of_dev [n_tokens * top_k]   place (token * top_k + k) of each row, -1: a row of nobody (those come last)
 * The workspace: moe_sort_tokens_bytes bytes, 4-byte aligned (0: none needed).
 * moe_gather_rows: xs[row_of[t, k]] = x[t] for elements of any moe_row_fmt, scale_dev [n_tokens] -> xs_scale_dev likewise
 *   (both NULL: none); rows of nobody are zeros.  xs_dev: [n_tokens * top_k, hidden].  Its gradient is moe_combine_rows of the
 *   gradients of xs with weight_dev NULL.
 * moe_combine_rows: y[t] = base[t] + sum over k of weight[t, k] * ys[row_of[t, k]], the places without a row left out whatever
 *   their weight is.  weight_dev (fp32) NULL: ones; base_dev (y_fmt, may be y_dev) NULL: zeros.  Formats: fp32 or bf16.
 * moe_combine_rows_backward: dys[row_of[t, k]] = weight[t, k] * dy[t] (rows of nobody: zeros) and
 *   dweight[t, k] = <dy[t], ys[row_of[t, k]]> (places without a row: 0; dweight_dev and ys_dev NULL: not wanted).  The gradient
 *   of base is dy itself. */
size_t moe_sort_tokens_bytes(int32_t n_tokens, int32_t top_k, int32_t n_experts);
int moe_sort_tokens(const int32_t *ids_dev, int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t *offsets_dev,
                    int32_t *row_of_dev, int32_t *entry_of_dev, void *workspace_dev, size_t workspace_bytes, void *stream);
int moe_gather_rows(const void *x_dev, int32_t fmt, int64_t x_stride, const float *scale_dev, const int32_t *row_of_dev,
                    const int32_t *offsets_dev, int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t hidden, void *xs_dev,
                    float *xs_scale_dev, void *stream);
int moe_combine_rows(const void *ys_dev, int32_t ys_fmt, const int32_t *row_of_dev, const float *weight_dev, const void *base_dev,
                     int32_t n_tokens, int32_t top_k, int32_t hidden, void *y_dev, int32_t y_fmt, void *stream);
int moe_combine_rows_backward(const void *dy_dev, int32_t dy_fmt, const void *ys_dev, int32_t ys_fmt, const int32_t *row_of_dev,
                              const int32_t *offsets_dev, const float *weight_dev, int32_t n_tokens, int32_t top_k,
                              int32_t n_experts, int32_t hidden, void *dys_dev, float *dweight_dev, void *stream);

/* The SwiGLU experts on sorted rows (Eq. 1 without the weighted sum): ys[r] = E_e(xs[r]) for offsets[e] <= r < offsets[e + 1],
 * zeros for the rows of nobody (those ahead of offsets[0], too: a part of the offsets with its blobs is a part of the experts).
 * blobs_dev: packed experts (moe_pack_expert), expert e at e * blob_stride bytes, 16-byte aligned.  hidden and inter as moe_blob_bytes
 * takes them, one blob smaller than 0xf0000000 bytes.
 *   MOE_W_BF16     xs_dev bf16, scale_dev NULL
 *   MOE_W_INT8_PC  xs_dev 8-bit codes with a scale for each row (moe_norm_rows, moe_gather_rows).  The sums of the first product
 *                  are whole numbers and exact; h is bf16.
 * Other formats are refused.  ys_dev: bf16.  xs_dev and ys_dev 16-byte aligned.
 * h_dev: bf16 [n_rows, pitch], pitch = inter rounded up to a multiple of 64: the products silu(g) * u as the down projection reads
 * them.  gu_dev: fp32 [n_rows, 2, pitch]: g and u, for the backward, or NULL.  Both 16-byte aligned; the caller keeps them for the
 * backward or throws them away.
 * moe_experts_rows_backward (MOE_W_BF16): from dys the gradients of xs and, in the layout of the blobs, of the weights (zeros
 * for an expert without rows; what lies between blobs is left as it is).  h_dev, gu_dev: as the forward left them; dgu_dev:
 * workspace, bf16 [n_rows, 2, pitch], 16-byte aligned.  dxs_dev or dblobs_dev NULL: not wanted.  Rows of nobody: dxs is zero. */
int moe_experts_rows(int32_t weight_fmt, int32_t hidden, int32_t inter, int32_t n_experts, const void *blobs_dev, int64_t blob_stride,
                     const void *xs_dev, const float *scale_dev, const int32_t *offsets_dev, int32_t n_rows, void *h_dev, float *gu_dev,
                     void *ys_dev, void *stream);
int moe_experts_rows_backward(int32_t weight_fmt, int32_t hidden, int32_t inter, int32_t n_experts, const void *blobs_dev,
                              int64_t blob_stride, const void *xs_dev, const int32_t *offsets_dev, int32_t n_rows, const void *h_dev,
                              const float *gu_dev, const void *dys_dev, void *dgu_dev, void *dxs_dev, void *dblobs_dev, void *stream);

/* ---- Attention beside the experts: of the rows of a prompt or a training batch, and of new tokens over a cache of pages ----
 *
 * As the calls above: no context, nothing allocated, nothing waited for, sizes refused before a pointer is looked at, graphs
 * possible, the same results from call to call.  Rows are bf16; a row of q has n_heads heads of head_dim values, one of k and v has
 * n_kv_heads; query head h reads head h / (n_heads / n_kv_heads).  head_dim is a multiple of 8 up to MOE_ATTEND_MAX_DIM, n_heads a multiple of
 * n_kv_heads up to MOE_ATTEND_MAX_HEADS, n_seqs <= MOE_ATTEND_MAX_SEQS.  Strides count elements, from token to token and from head to
 * head; the values of a head are dense.  Pointers and strides of bf16 rows that are read are multiples of 16 bytes.
 *   A query at position p sees key j if j <= p and (window 0, or j > p - window, or j < sinks).
 *   z_j = softmax_scale <q, k_j>, y = sum_j exp(z_j - lse) v_j, lse = log sum_j exp(z_j), over the keys that it sees; y is 0 (lse
 *   -infinity) if there are none, or if all z_j are -infinity.  Sums are held in 32 bits.  What a query does not see may hold anything;
 *   a z_j that is NaN makes its y and lse NaN, infinities and NaN in values that it sees go into y.
 *
 * A cache has n_pages pages of `page` tokens (a power of two, 16 to 1024), page_stride elements from page to page:
 *   k_pages, v_pages [n_pages][n_kv_heads][page][head_dim]; page * n_pages < 2^31
 *   MOE_R_BF16  k_scale, v_scale NULL
 *   MOE_R_INT8  codes c that stand for c * scale; k_scale, v_scale fp32 [n_pages][n_kv_heads][page], dense
 * both 16-byte aligned, as are their pages.  table_dev [n_seqs, table_pages]: token t of sequence i is in page table[i, t / page]; ids outside
 * 0..n_pages-1 (-1) are no page, and what would be there is seen by nobody.
 *
 * moe_plan_pages: pages and places for the tokens that the sequences bring.  Sequence i has have[i] tokens in the cache and brings more[i]
 *   (negative: 0).  Entries ceil(have / page) .. ceil((have + more) / page) - 1 of its row of the table, as far as the row goes, are
 *   taken from free_dev [n_free] in the order of the sequences, from element *used_dev on (used_dev NULL: 0); behind the end of free_dev
 *   they become -1.  All other entries are read or left alone.
 *     offsets_dev [n_seqs + 1]     the tokens of sequence i are rows offsets[i] .. offsets[i + 1] - 1
 *     slots_dev, positions_dev [n_tokens]  of each row: page * `page` + place in it, -1 if there is no page; position in the sequence.
 *                                  Rows behind the last sequence: -1 and -1
 *     lengths_dev [n_seqs]         have + more
 *     used_out_dev [1]             *used_dev + the entries that were to be taken; more than n_free: there were too few pages
 *   Numbers that pass 2^31 - 1 stay there.  No result may overlap what is read, nor two rows of the table each other.
 * moe_store_pages: rows of k and v (fmt fp32 or bf16) to their slots; a slot outside 0..n_pages*page-1 takes nothing.  Slots have to
 *   differ.  cache_fmt bf16: rounded.  int8: with top the largest |v| of a token's head, code = round(127 v / top) (to even, as if
 *   computed exactly), scale = top / 127; top < 1e-30: codes and scale 0; with an infinity or NaN: codes 0, scale NaN.
 * moe_attend_pages: one new token per sequence, the last of its lengths_dev[i] tokens.  Length 0 (or less): y is 0.  Every sequence is
 *   split over the GPU by what the lengths say; the workspace holds the parts' sums: moe_attend_pages_bytes(n_seqs, n_heads,
 *   n_kv_heads, head_dim) bytes, 16-byte aligned, of this call alone until it is done.
 * moe_attend_rows: packed sequences.  Sequence i has the rows offsets[i] .. offsets[i + 1] - 1 of q and y, and k_offsets[i] ..
 *   k_offsets[i + 1] - 1 of k and v (k_offsets_dev NULL: the same); its queries are its last rows, so that query r of nq is at position
 *   nk - nq + r (one ahead of the first key sees nothing).  y_dev dense [n_rows, n_heads, head_dim].  For the backward, or NULL:
 *   y_low_dev (as y_dev): bf16 of what the rounding of y leaves; lse_dev fp32 [n_heads, n_rows].  Rows of no sequence: y is 0, the
 *   others are left alone.  Few queries of many keys are split over the GPU: the workspace holds what the shares have,
 *   moe_attend_rows_bytes bytes, 16-byte aligned, of this call alone until it is done (0: none is needed, it may be NULL).
 * moe_attend_rows_backward: from dy the gradients of q, k and v, dense, bf16 (rows of no sequence: 0).  y, y_low, lse: as the forward left
 *   them (y_low_dev NULL: y is taken as it is rounded, and dq and dk are less exact).  P = exp(z - lse), dv = sum P dy, dz = P (<dy, v>
 *   - <dy, y>), dq = softmax_scale sum dz k, dk = softmax_scale sum dz q, sums over the heads of a group and over all queries in a fixed
 *   order.  For the matrix cores P and dz are rounded to bf16, dz for dq to two of them.  Infinities and NaN in a sequence may make NaN
 *   of any of its gradients (of no other sequence's).  y and dy dense.  The workspace: moe_attend_rows_backward_bytes bytes, 16-byte aligned, of this call alone until it is done. */
int moe_plan_pages(const int32_t *have_dev, const int32_t *more_dev, int32_t n_seqs, int32_t page, const int32_t *free_dev, int32_t n_free,
                   const int32_t *used_dev, int32_t *table_dev, int32_t table_pages, int32_t *offsets_dev, int32_t *slots_dev,
                   int32_t *positions_dev, int32_t n_tokens, int32_t *lengths_dev, int32_t *used_out_dev, void *stream);
int moe_store_pages(const void *k_dev, const void *v_dev, int32_t fmt, int64_t k_stride, int64_t k_head_stride, int64_t v_stride,
                    int64_t v_head_stride, const int32_t *slots_dev, int32_t n_rows, int32_t n_kv_heads, int32_t head_dim, void *k_pages_dev,
                    void *v_pages_dev, int32_t cache_fmt, int64_t page_stride, int32_t n_pages, int32_t page, float *k_scale_dev,
                    float *v_scale_dev, void *stream);
size_t moe_attend_pages_bytes(int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);
int moe_attend_pages(const void *q_dev, int64_t q_stride, int64_t q_head_stride, const void *k_pages_dev, const void *v_pages_dev,
                     int32_t cache_fmt, int64_t page_stride, int32_t n_pages, int32_t page, const float *k_scale_dev,
                     const float *v_scale_dev, const int32_t *table_dev, int32_t table_pages, const int32_t *lengths_dev, int32_t n_seqs,
                     int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float softmax_scale, int32_t window, int32_t sinks, void *y_dev,
                     void *workspace_dev, size_t workspace_bytes, void *stream);
size_t moe_attend_rows_bytes(int32_t n_rows, int32_t n_k_rows, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);
int moe_attend_rows(const void *q_dev, int64_t q_stride, int64_t q_head_stride, const void *k_dev, int64_t k_stride, int64_t k_head_stride,
                    const void *v_dev, int64_t v_stride, int64_t v_head_stride, const int32_t *offsets_dev, const int32_t *k_offsets_dev,
                    int32_t n_seqs, int32_t n_rows, int32_t n_k_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                    float softmax_scale, int32_t window, int32_t sinks, void *y_dev, void *y_low_dev, float *lse_dev, void *workspace_dev,
                    size_t workspace_bytes, void *stream);
size_t moe_attend_rows_backward_bytes(int32_t n_rows, int32_t n_k_rows, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);
int moe_attend_rows_backward(const void *q_dev, int64_t q_stride, int64_t q_head_stride, const void *k_dev, int64_t k_stride,
                             int64_t k_head_stride, const void *v_dev, int64_t v_stride, int64_t v_head_stride, const int32_t *offsets_dev,
                             const int32_t *k_offsets_dev, int32_t n_seqs, int32_t n_rows, int32_t n_k_rows, int32_t n_heads,
                             int32_t n_kv_heads, int32_t head_dim, float softmax_scale, int32_t window, int32_t sinks, const void *y_dev,
                             const void *y_low_dev, const float *lse_dev, const void *dy_dev, void *dq_dev, void *dk_dev, void *dv_dev, void *workspace_dev,
                             size_t workspace_bytes, void *stream);

const char *moe_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* MOE_CACHE_H */
