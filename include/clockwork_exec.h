/*
 * clockwork_exec.h -- C ABI of the MI355X worker hot path: the steps of an INFER
 * action on one GPU (INPUT -> EXEC -> OUTPUT) plus LOAD / UNLOAD of weights and a
 * measured EXEC-latency profile per (model, batch size).
 *
 * The call set follows the action model of the paper (section 4.4 "Predictable DNN
 * Worker", section 5.1 "Models", section 5.2 "DNN Workers"):
 *   - a model is weights + kernels per batch size + static memory metadata + a
 *     seed latency profile (section 5.1);
 *   - all device memory is allocated once and split into a workspace for
 *     intermediates, an IO cache for inputs/outputs and a pool for weights
 *     (section 5.2, "Managing model weights in memory");
 *   - INFER = INPUT, EXEC, OUTPUT; EXEC checks that weights and input are present
 *     and runs the kernels; one EXEC at a time per GPU (sections 4.4, 5.2);
 *   - every action reports a status and its on-device duration (section 5.2,
 *     "Results").
 *
 * Conventions
 *   - Every call returns an int32_t status: CW_OK (0) or a negative CW_ERR_*.
 *     No exception crosses this boundary.  cw_strerror() names a status;
 *     cw_last_error() gives detail for the last failing call on a context.
 *   - Pointers marked [host] are host memory owned by the caller; the library owns
 *     all device memory.  The device pools (workspace, IO cache, weight pool, LOAD
 *     staging) are allocated once, by cw_create(), and nothing is taken from or returned
 *     to the device allocator afterwards.  Host-side runtime objects are still created
 *     later: one event per model in cw_model_define(), and one recorded HIP graph per
 *     (model, batch size) in cw_load_weights() (recording executes nothing).
 *   - `stream` is a raw hipStream_t (passed as void*; NULL = the default stream).
 *     Calls that take a stream only enqueue work; the caller must keep [host]
 *     buffers alive and unmodified until that stream has been synchronised.  Host
 *     buffers should be pinned for the copies to be asynchronous.
 *   - A context is bound to one GPU and is not thread safe: serialise calls on
 *     one context (the paper's executors are one thread per action type; here the
 *     caller provides that discipline).
 *   - Storage type of weights and activations: fp16 or bf16 (per model);
 *     accumulation is always fp32; biases, logits and probabilities are fp32.
 */
#ifndef CLOCKWORK_EXEC_H
#define CLOCKWORK_EXEC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cw_ctx cw_ctx; /* one per GPU: the paper's "worker-GPU" */

enum {
    CW_OK = 0,
    CW_ERR_INVALID = -1,        /* bad argument (null pointer, unknown id, bad size) */
    CW_ERR_HIP = -2,            /* a HIP runtime call failed; see cw_last_error() */
    CW_ERR_NO_MEMORY = -3,      /* a pre-allocated pool cannot hold the request */
    CW_ERR_NOT_LOADED = -4,     /* EXEC on a model whose weights are not resident */
    CW_ERR_ALREADY_LOADED = -5, /* LOAD of a model that is resident */
    CW_ERR_NO_INPUT = -6,       /* EXEC/OUTPUT on a slot that holds no input / no result */
    CW_ERR_BAD_BATCH = -7,      /* batch size the model has no plan for */
    CW_ERR_BUSY = -8,           /* an EXEC is still in flight on another stream */
    CW_ERR_UNSUPPORTED = -9,    /* topology the kernels cannot run (see cw_model_define) */
    CW_ERR_NO_SLOT = -10,       /* every IO slot is in use */
    CW_ERR_TOO_LATE = -11,      /* an action's executor reached it after its `latest`: not executed */
    CW_ERR_TIMEOUT = -12        /* cw_worker_next_result: no result within the time given */
};

enum { CW_OP_CONV = 0, CW_OP_MAXPOOL = 1, CW_OP_GAVGPOOL = 2, CW_OP_FC = 3, CW_OP_SOFTMAX = 4, CW_OP_CONCAT = 5, CW_OP_FC4 = 6 };
enum { CW_ACT_NONE = 0, CW_ACT_RELU = 1, CW_ACT_HSWISH = 2 };   /* values of cw_op.relu */
enum { CW_DTYPE_FP16 = 0, CW_DTYPE_BF16 = 1, CW_DTYPE_FP32 = 2, CW_DTYPE_E4M3 = 3 };   /* a model's storage type is one of the first two; the last is for a cache's pages */

/* One operator of a model.  Ops form a DAG over earlier ops' outputs.
 * CONV:     cross-correlation, kh x kw, `stride`, zero padding, + bias[cout], then (if
 *           residual_from >= 0) + output of that op, then the activation `relu` (CW_ACT_*: none,
 *           ReLU, or hard swish x * min(max(x + 3, 0), 6) / 6).  A square filter is padded by
 *           `pad` on every side; a rectangular one (kh != kw, e.g. 1x7 and 7x1) by `pad` rows and
 *           `pad_w` columns.  groups <= 1: dense; groups == cin == cout: depthwise (one kh x kw
 *           filter per channel, weights W[cout][1][kh][kw]).
 * MAXPOOL:  kh x kw window, `stride`, `pad`; padded taps are ignored.
 * GAVGPOOL: mean over all spatial positions.
 * FC:       cin -> cout, + bias; its fp32 output is the model's logits.
 * SOFTMAX:  over the cout values of each sample; its output is the probabilities.
 * CONCAT:   the channels of op input_from followed by those of op residual_from (same spatial
 *           size; cin = channels of the first, cout = of both).  Where the producers allow it
 *           they write straight into their channel range of the result and nothing is copied.
 * FC4:      FC over 4-bit weights (see cw_fc4) in the place of FC; `groups` inputs share a scale and a zero
 *           point (a multiple of 32).  A quarter of the bytes to LOAD and to keep.
 * The operators beyond the ResNet set serve the other model families of the paper's Table 1
 * (DenseNet: concatenation; Inception v3: rectangular filters; MobileNet: depthwise, hard swish). */
typedef struct {
    int32_t op;            /* CW_OP_* */
    int32_t cin, cout;     /* channels in / out (MAXPOOL, GAVGPOOL, SOFTMAX: cin == cout) */
    int32_t kh, kw;        /* filter or window size (0 where unused) */
    int32_t stride, pad;
    int32_t relu;          /* CONV only: CW_ACT_* */
    int32_t residual_from; /* CONV: -1 or index of an earlier op to add; CONCAT: the second source */
    int32_t input_from;    /* -1 = the network input, else index of an earlier op */
    int32_t pad_w;         /* CONV with kh != kw: padding in width (`pad` is then the padding in height) */
    int32_t groups;        /* CONV: 0 or 1 = dense, cin = depthwise; FC4: inputs of a group */
} cw_op;

typedef struct {
    int32_t device;             /* HIP device ordinal */
    size_t workspace_bytes;     /* intermediates of the one EXEC in flight (paper: 512 MB) */
    size_t io_bytes;            /* IO cache: inputs and outputs of in-flight INFERs (paper: 512 MB) */
    size_t weight_pool_bytes;   /* packed weights of all resident models, handed out in pages */
    size_t load_staging_bytes;  /* device landing zone of one canonical blob during LOAD;
                                   must be >= the largest blob that will be loaded */
    size_t weight_page_bytes;   /* page size of the weight pool; 0 = 16 MiB (the paper's, section 5.1);
                                   a multiple of 256, and no weight tensor may be larger */
} cw_config;

/* Section 5.2, "Managing model weights in memory": a worker takes all the device memory it
 * will use when it starts and manages it itself, so that no allocation happens on the path of
 * an action.  cw_create makes one allocation per region of cw_config (+ the streams and events
 * the context needs); cfg [host].  CW_ERR_NO_MEMORY when the device cannot give a region,
 * CW_ERR_UNSUPPORTED on a GPU other than gfx950, CW_ERR_INVALID for a bad ordinal or page
 * size.  device == -1 makes a planning-only context: models and plans can be defined and
 * inspected, every call that would touch a GPU returns CW_ERR_INVALID. */
int32_t cw_create(cw_ctx **out, const cw_config *cfg);
/* The worker shuts down: waits for all work the context enqueued, then frees every region,
 * graph, stream and event.  The handle is invalid afterwards. */
int32_t cw_destroy(cw_ctx *ctx);

/* ---- models (section 5.1: kernels per batch size + memory metadata) ----------
 * Defines a topology and compiles one fixed launch plan per batch size: kernel
 * variant, grid, split-K factor and workspace offsets are functions of (ops, input
 * size, batch) only.  Nothing is tuned or chosen at run time.
 * ops, batch_sizes: [host], copied.  The first op must read the network input
 * (in_c x in_h x in_w, NCHW fp32 at the boundary); the list must end FC, SOFTMAX or FC4, SOFTMAX.
 * Supported: CONV with cin % 32 == 0, cout % 32 == 0 and kh == kw <= 5 anywhere,
 * plus a first CONV with cin <= 4 and kh == kw <= 8; GAVGPOOL over a multiple of 64
 * channels; FC with cin % 256 == 0, or FC4, reading the GAVGPOOL.  Returns CW_ERR_UNSUPPORTED otherwise,
 * CW_ERR_NO_MEMORY if a plan's workspace exceeds workspace_bytes. */
int32_t cw_model_define(cw_ctx *ctx, const cw_op *ops, int32_t n_ops,
                        int32_t in_c, int32_t in_h, int32_t in_w,
                        const int32_t *batch_sizes, int32_t n_batch,
                        int32_t dtype, int32_t *model_id);
/* ResNet-18 / 50 / 152 (depth) with batch sizes 1,2,4,8,16 (section 5.1 default). */
int32_t cw_model_define_resnet(cw_ctx *ctx, int32_t depth, int32_t in_h, int32_t in_w,
                               int32_t dtype, int32_t *model_id);
/* Copies the model's op list to ops_out[0..cap) [host]; *n_ops = its length. */
int32_t cw_model_get_ops(cw_ctx *ctx, int32_t model_id, cw_op *ops_out, int32_t cap,
                         int32_t *n_ops);
/* Size in bytes of the canonical weight blob LOAD expects (0 for a bad id). */
size_t cw_model_weight_bytes(cw_ctx *ctx, int32_t model_id);
/* Workspace bytes the plan for (model, batch) uses (0 for a bad id / batch). */
size_t cw_model_workspace_bytes(cw_ctx *ctx, int32_t model_id, int32_t batch);

/* ---- LOAD / UNLOAD (section 5.2) ----------------------------------------------
 * Canonical blob [host]: for every op that owns weights (CONV, FC), in op order,
 * W[cout][cin][kh][kw] in the model's storage type, back to back; zero padding to
 * a multiple of 4 bytes; then every bias[cout] as fp32 in the same op order.
 * In W's place an FC4 has its weights q[cout][ceil(cin/2)] (bytes, the even input in the low four bits),
 * the scales[cout][ceil(cin/groups)] in the storage type and the zero points [cout][ceil(cin/groups)]
 * (bytes), each of the three padded with zeros to a multiple of 2 bytes.
 * The weight pool is a set of equal pages (section 5.1; cw_config.weight_page_bytes).  A
 * model's packed tensors were given places in cw_model_weight_pages() pages of its own when it
 * was defined, none straddling a page boundary; LOAD takes that many free pages of the pool,
 * whichever they are (lowest-numbered first; CW_ERR_NO_MEMORY when fewer are free: the
 * paper's LOAD aborts when no pages are free), copies the blob to the device on `stream`
 * and re-lays it out there, tensor by tensor, for the MFMA kernels, which receive each
 * tensor's address as a kernel argument.  The same packed weights serve every batch size.
 * `bytes` must equal cw_model_weight_bytes(). */
int32_t cw_load_weights(cw_ctx *ctx, int32_t model_id, const void *host_blob,
                        size_t bytes, void *stream);
/* The same LOAD in steps, for a caller whose threads share one context under a lock of their
 * own (the worker's executors, section 5.2: LOAD runs beside EXEC), so that the lock is held
 * only while work is enqueued:
 *   cw_load_weights_begin    takes the pages and enqueues the copy and the re-layout on `stream`;
 *                            the model counts as resident from here on (an EXEC waits for the
 *                            copy on its own stream) and runs with plain launches until the end
 *                            step.  Serialise with the other calls on the context.
 *   cw_load_weights_record   records the plans' HIP graphs for the pages taken.  Host work of a few
 *                            milliseconds, nothing executes.  May run while other threads call
 *                            into the same context; only one recording at a time per context.
 *   cw_load_weights_end      installs the recorded graphs (nothing if the model has been unloaded
 *                            meanwhile).  Serialise with the other calls on the context.
 *   cw_load_weights_release  destroys `pending` and the graphs the new ones displaced.  Needs no
 *                            serialisation.  Always call it once for a `pending` that begin returned.
 * cw_load_weights() is these four in a row.  `*pending` is NULL when begin fails. */
typedef struct cw_load_pending cw_load_pending;
int32_t cw_load_weights_begin(cw_ctx *ctx, int32_t model_id, const void *host_blob, size_t bytes,
                              void *stream, cw_load_pending **pending);
int32_t cw_load_weights_record(cw_ctx *ctx, cw_load_pending *pending);
int32_t cw_load_weights_end(cw_ctx *ctx, cw_load_pending *pending);
void    cw_load_weights_release(cw_load_pending *pending);
/* Metadata only; succeeds whether or not the model is resident (section 5.2).  The pages go
 * back to the free list at once; an EXEC of the model that is still queued or running keeps
 * reading them safely, because the next LOAD that takes one of them makes its stream wait for
 * that EXEC's end before it writes. */
int32_t cw_unload_weights(cw_ctx *ctx, int32_t model_id);
/* Free pages of the weight pool: the only memory state a controller needs (section 5.1);
 * in bytes (free pages x page size), and as a count.  cw_model_weight_pages: the pages one
 * LOAD of the model takes (negative: unknown id). */
size_t cw_weight_pool_free(cw_ctx *ctx);
int32_t cw_weight_pages_free(cw_ctx *ctx);
int32_t cw_model_weight_pages(cw_ctx *ctx, int32_t model_id);

/* ---- INFER = INPUT, EXEC, OUTPUT (section 5.2) --------------------------------
 * INPUT: takes an IO slot and copies host_nchw [host], fp32 [batch][in_c][in_h][in_w],
 * to it on `stream`.  *slot receives the slot id.  CW_ERR_NO_SLOT / CW_ERR_NO_MEMORY
 * when the IO cache is full, CW_ERR_BAD_BATCH for a batch without a plan. */
int32_t cw_input(cw_ctx *ctx, int32_t model_id, int32_t batch, const float *host_nchw,
                 int32_t *slot, void *stream);
/* EXEC: checks that the model's weights are resident (else CW_ERR_NOT_LOADED) and
 * that `slot` holds an input of this (model, batch) (else CW_ERR_NO_INPUT /
 * CW_ERR_BAD_BATCH), then enqueues the plan's kernels on `stream`, bracketed by
 * two events.  The stream is made to wait for the slot's INPUT copy and the
 * model's LOAD, so they may have been issued on other streams.  A second EXEC
 * issued on a different stream while one is in flight returns CW_ERR_BUSY; on
 * the same stream EXECs simply run back to back.  EXEC may be repeated on a slot. */
int32_t cw_exec(cw_ctx *ctx, int32_t model_id, int32_t batch, int32_t slot, void *stream);
/* EXEC for callers that cannot allocate: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same plan, same kernels and same results as cw_exec, but
 *   - the input, the logits and the probabilities are the caller's own device buffers:
 *     dev_input_nchw [device] fp32 [batch][in_c][in_h][in_w], dev_logits and dev_probs [device]
 *     fp32 [batch][classes]; the caller orders their producers and consumers on `stream`;
 *   - the intermediates (activations, split-K partial sums and arrival counters) live in an array
 *     built into the library, cw_exec_static_capacity() bytes (80 MiB) per GPU, instead of the
 *     context's workspace: a plan whose intermediates need more returns CW_ERR_NO_MEMORY (see
 *     cw_model_workspace_bytes; ResNet-50 and ResNet-152 at 224x224 fit up to batch 16);
 *   - the call allocates nothing, creates no event or graph and records nothing but kernel
 *     launches (plus one wait for the model's LOAD if that has not finished yet).
 * Every call on a GPU uses that GPU's one array, whatever the context: calls that overlap in time
 * on one GPU (two streams, two contexts) race; on one stream they simply run in order.  The EXEC
 * is not timed and does not take part in cw_exec's one-at-a-time check.
 * CW_ERR_NOT_LOADED / CW_ERR_BAD_BATCH / CW_ERR_INVALID as for cw_exec. */
int32_t cw_exec_static(cw_ctx *ctx, int32_t model_id, int32_t batch, const float *dev_input_nchw,
                       float *dev_logits, float *dev_probs, void *stream);
/* Bytes of intermediates a plan may need to run through cw_exec_static. */
size_t cw_exec_static_capacity(void);
/* OUTPUT: enqueues the copies of the slot's results to host_probs [host]
 * [batch][classes] and, if not NULL, host_logits [host] [batch][classes] on
 * `stream` (after the slot's EXEC), then releases the slot; its memory is reused
 * only after these copies have completed.  CW_ERR_NO_INPUT if no EXEC ran. */
int32_t cw_output(cw_ctx *ctx, int32_t slot, float *host_probs, float *host_logits,
                  void *stream);
/* OUTPUT of the answer instead of the rows of probabilities (see cw_answer for what it holds): computed on
 * `stream` behind the slot's EXEC from its logits and copied to host_answer [host], cw_answer_bytes(batch, top)
 * bytes: logp fp32 [batch], rank int32 [batch], entropy fp32 [batch], top_id int32 [batch][top], top_logp fp32
 * [batch][top], back to back.  host_given [host] int32 [batch] or NULL (nothing given); it is copied on `stream` and, like
 * host_answer, belongs to the call until that copy is over.  Then releases the slot as cw_output does.  CW_ERR_NO_INPUT if no EXEC ran, CW_ERR_INVALID / CW_ERR_UNSUPPORTED for arguments that cw_answer
 * refuses, CW_ERR_NO_MEMORY where the answer is larger than the slot's input and its probabilities; the slot then stays. */
int32_t cw_output_answer(cw_ctx *ctx, int32_t slot, const int32_t *host_given, int32_t top, float scale,
                         void *host_answer, void *stream);
/* Bytes of that answer (0 for batch < 0 or top outside 0..CW_ANSWER_MOST_TOP). */
size_t cw_answer_bytes(int32_t batch, int32_t top);
/* Batch size of the request that holds the slot; CW_ERR_NO_INPUT if none does. */
int32_t cw_slot_batch(cw_ctx *ctx, int32_t slot);
/* Section 5.2, INFER: an action that is rejected after its INPUT (its window passed, its EXEC
 * failed) must give its IO-cache entry back without an OUTPUT.  Releases the slot without
 * copying anything out; the memory is reused only after its INPUT copy and its last EXEC have
 * finished.
 * Succeeds on a slot that is already free. */
int32_t cw_release(cw_ctx *ctx, int32_t slot);
/* On-device duration of the slot's last EXEC (the "timing" field of a result).
 * Blocks until that EXEC has finished. */
int32_t cw_exec_duration_ns(cw_ctx *ctx, int32_t slot, uint64_t *on_device_ns);

/* ---- measured latency profile per (model, batch) (section 5.1 "Profiling data") */
typedef struct {
    uint32_t n;
    float p50_us, p99_us, p999_us, min_us, max_us, mean_us;
    float p9999_us;   /* nearest rank like the others: the maximum for n < 10000 */
} cw_profile;
/* Runs `repeats` EXECs of (model, batch) back to back on an internal stream, each timed on
 * the device, and stores and returns nearest-rank percentiles.  The EXECs read the input held
 * by `slot` (an IO slot of this (model, batch) filled by cw_input; it stays the caller's), or,
 * with slot == -1, a zero-filled input of the library's own.  EXEC time depends slightly on the
 * operand values through power and clocks, so a profile meant to predict real requests should
 * be measured over a representative input.  The EXECs are submitted in bursts of 128; one
 * untimed EXEC leads each burst so that every timed one starts behind queued work.
 * Synchronous.  samples_us [host] may be NULL, else receives the `repeats` individual
 * durations in microseconds. */
int32_t cw_profile_measure(cw_ctx *ctx, int32_t model_id, int32_t batch, int32_t slot,
                           uint32_t repeats, cw_profile *out, float *samples_us);
/* Last measured profile; n == 0 if none was measured. */
int32_t cw_profile_get(cw_ctx *ctx, int32_t model_id, int32_t batch, cw_profile *out);

/* ---- single operators over the caller's device memory ------------------------------------------
 * As cw_exec_static: every buffer is the caller's, on the context's GPU, and stays valid until the work is over; the call
 * allocates nothing, enqueues kernel launches on `stream` and nothing else, and may be captured into a HIP graph.
 * Inputs and outputs must not overlap.  Strides are in elements (bytes for 4-bit weights) from one row to
 * the next; the elements of a row are contiguous.  Input rows may overlap (stride 0: one row for all), output
 * rows not.  CW_ERR_INVALID for a null or misaligned pointer, a bad size, stride or type, CW_ERR_UNSUPPORTED for
 * sizes the kernels do not run; nothing is enqueued then.  No row: CW_OK, nothing to do. */

/* Fully connected layer over 4-bit weights with group scales:
 *   y[m][n] = bias[n] + sum over k < cin of x[m][k] * (q[n][k] - zero[n][k / group]) * scale[n][k / group]
 * q - zero and its products with what stands for x are exact, sums are fp32, and the result is rounded once, to y's type.  fp16 activations stand as they are;
 * bf16 and fp32 ones as fp16 numbers scaled by a power of two for every 128 inputs of a row, fp32 in two parts: an fp32 activation is off by up to 2^-23 of
 * itself and 2^-39 of the largest of these 128, a bf16 one by less than 2^-38 of the largest, and by nothing from 2^-31 of it on.  With them a scale beyond
 * 2^100 may overflow. A NaN or an infinity of x stays in its row and comes out as the formula has it (an infinity times a weight of zero is a NaN),
 * one of scale or bias stays in its column. */
typedef struct {
    const void *x;          /* [rows][cin], x_dtype */
    const uint8_t *q;       /* [cout][ceil(cin / 2)]: k even in the low, k odd in the high four bits */
    const void *scales;     /* [cout][ceil(cin / group)], scale_dtype */
    const uint8_t *zeros;   /* [cout][ceil(cin / group)], 0..15 (of larger values the low four bits), or NULL: 8 everywhere */
    const float *bias;      /* [cout] or NULL */
    void *y;                /* [rows][cout], y_dtype */
    int64_t x_stride, q_stride, scale_stride, zero_stride, y_stride;
    int32_t rows, cin, cout;
    int32_t group;          /* inputs that share a scale: a multiple of 32 (the last group of a row may be short) */
    int32_t x_dtype, scale_dtype, y_dtype;   /* CW_DTYPE_* */
} cw_fc4_args;
int32_t cw_fc4(cw_ctx *ctx, const cw_fc4_args *args, void *stream);

/* The answer of every row of logits.  With d[i] = scale * (x[i] - max x) over the classes i with x[i] > -inf (a masked class
 * has -inf) and S = sum exp d:
 *   logp     d[given] - ln S; 0 for a negative `given` (nothing given), NaN for one >= classes, -inf for a masked class
 *   rank     classes that come before the given one: larger logits, and equal ones of lower index (0: it is the first); -1 for
 *            a `given` outside the classes
 *   entropy  ln S - sum(d exp d) / S, in nats
 *   top_id, top_logp  the `top` likeliest classes, equal ones by index, and d - ln S; behind the last class that is not masked -1
 *            and -inf
 * A row with nothing but -inf: logp -inf, entropy 0, no top classes.  A row with a NaN or +inf: logp, entropy and
 * top_logp NaN, rank and top_id -1 (a negative `given` has logp 0 all the same).  The order is that of the logits as they are stored; sums are
 * fp32 over 32 classes and fp64 beyond, to fp32 at their end, and of two logits whose difference leaves fp32's range the smaller has no probability.
 * With few rows a row is shared by several workgroups, which meet in `workspace`: its first CW_ANSWER_COUNTERS bytes must be
 * zero before the first call and are zero behind every call.  Calls that may overlap in time need a workspace each.
 * Without one (NULL, or smaller than cw_answer_workspace_bytes) a workgroup takes a row; the answers are the same but for
 * the order of the sums. */
#define CW_ANSWER_MOST_TOP 64
#define CW_ANSWER_COUNTERS 1024
typedef struct {
    const void *logits;     /* [rows][classes], dtype */
    const int32_t *given;   /* [rows] or NULL */
    float *logp;            /* [rows] or NULL; with `given` only */
    int32_t *rank;          /* [rows] or NULL; with `given` only */
    float *entropy;         /* [rows] or NULL */
    int32_t *top_id;        /* [rows][top], NULL with top == 0 */
    float *top_logp;        /* [rows][top], NULL with top == 0 */
    void *workspace;        /* 16-byte aligned, or NULL */
    size_t workspace_bytes;
    int64_t stride;
    int32_t rows, classes;
    int32_t top;            /* 0..CW_ANSWER_MOST_TOP */
    int32_t dtype;          /* CW_DTYPE_* */
    float scale;            /* of the logits (1 / temperature): finite, > 0 */
} cw_answer_args;
int32_t cw_answer(cw_ctx *ctx, const cw_answer_args *args, void *stream);
/* Workspace that serves every call (less than 1 MiB). */
size_t cw_answer_workspace_bytes(void);

/* Keys and values of sequences of tokens, in pages of `page` tokens that a program gives out as it likes: row s of a `table` names the pages of sequence s in
 * order, its token t lies at place t % page of page table[s][t / page].  A page number outside 0..pages - 1 stands for a page that is not there: nothing is
 * written to it, what is read of it is 0, attention leaves its tokens out.  The same goes for tokens beyond the table's row.
 * With CW_DTYPE_E4M3 a number is code * 2^(exponent - 127): codes have 8 bits (sign, 4, 3; the largest 448), the exponent is a byte for every token and head, of keys
 * and of values.  Strides are in elements (bytes for codes and exponents), 16 bytes divide the addresses of all keys' and values' rows and head_dim is a multiple
 * of 16. */
typedef struct {
    void *k, *v;                /* [pages][kv_heads][page][head_dim], dtype */
    uint8_t *k_exp, *v_exp;     /* [pages][kv_heads][page] with CW_DTYPE_E4M3, else NULL */
    int64_t page_stride, head_stride, token_stride;               /* of k and of v */
    int64_t exp_page_stride, exp_head_stride, exp_token_stride;   /* of k_exp and of v_exp */
    int32_t pages, kv_heads;
    int32_t page;               /* a power of two, up to CW_CACHE_MOST_PAGE */
    int32_t head_dim;           /* a multiple of 16, up to CW_ATTEND_MOST_DIM */
    int32_t dtype;              /* CW_DTYPE_FP16, BF16 or E4M3 */
} cw_cache;
#define CW_CACHE_MOST_PAGE 4096
#define CW_ATTEND_MOST_DIM 256

/* Writes the newest tokens of sequences to their pages, reads them back.  Sequence s has lengths[s] tokens, these included, and rows first[s]..first[s + 1] - 1 of k and v
 * are its last ones; rows outside first[0]..first[sequences] - 1 are not touched, nor read.  Tokens before a sequence's beginning (more rows than lengths[s]) are not written
 * and read as 0.  A place that is in the table twice must not be written twice in one call.
 * Writing: numbers are rounded to the pages' type; with CW_DTYPE_E4M3 the exponent is the least (from -127 on) with which the largest finite magnitude of a token's head is
 * at most 448 * 2^exponent, codes are the nearest (ties to even) of x / 2^exponent, a NaN or an infinity becomes a NaN.  Reading: code * 2^exponent, rounded once to
 * the rows' type. */
typedef struct {
    const cw_cache *cache;      /* [host] */
    void *k, *v;                /* [tokens][kv_heads][head_dim], dtype: read by cw_cache_write, written by cw_cache_read */
    const int32_t *first;       /* [sequences + 1], not falling; NULL: one row a sequence (tokens == sequences) */
    const int32_t *lengths;     /* [sequences] */
    const int32_t *table;       /* [sequences][table_pages] */
    int64_t k_stride, k_head_stride, v_stride, v_head_stride, table_stride;
    int32_t tokens, sequences, table_pages;
    int32_t dtype;              /* CW_DTYPE_FP16, BF16 or FP32 */
} cw_cache_args;
int32_t cw_cache_write(cw_ctx *ctx, const cw_cache_args *args, void *stream);
int32_t cw_cache_read(cw_ctx *ctx, const cw_cache_args *args, void *stream);

/* Attention of one new token of each sequence over the tokens in its pages (its own among them, written before):
 *   y[s][h] = sum over t of p[t] * v[t][h'],  p = softmax over t of scale * q[s][h] . k[t][h'],  h' = h / (heads / kv_heads)
 * over the tokens t < lengths[s], with `window` > 0 the last `window` of them.  lse is the logarithm of the softmax's denominator, with which results over parts of a
 * sequence can be joined.  A row that sees no token has y 0 and lse -inf.  Products with the numbers as they are stored are exact, sums and the softmax fp32; of
 * fp16, and of E4M3, p goes into the second product in 11 bits, off by 2^-36 of the row's largest at most where that is more (of p times the power of two of its token's value, with E4M3), of bf16 in 15; the
 * result is rounded once.  An infinite value whose p is that small makes the result NaN.  Scores of +inf or NaN make their row NaN; numbers of tokens that
 * are not seen have no effect whatever they are.
 * How a sequence is shared goes by table_pages, `window` and how many sequences there are, as lengths are on the GPU: a table is best as wide as its longest sequence needs (200 sequences of 30 to 150 tokens, 32 heads over 8
 * of 128 bf16, 18 us, with a table for 4096 tokens 29; 64 of up to 8192 202 us, with one for 32768 214).
 * Sequences are shared by several workgroups, which meet in `workspace`: its first CW_ATTEND_COUNTERS bytes must be zero before the first call and are zero behind every call.  Calls
 * that may overlap in time need a workspace each.  Without one (NULL), or with less than cw_attend_one_workspace_bytes(), a sequence's heads are shared less or not at all; the results
 * are the same but for the order of the sums. */
#define CW_ATTEND_COUNTERS 65536
typedef struct {
    const cw_cache *cache;      /* [host] */
    const void *q;              /* [sequences][heads][head_dim], dtype */
    void *y;                    /* the same */
    float *lse;                 /* [sequences][heads] or NULL */
    const int32_t *lengths;     /* [sequences] */
    const int32_t *table;       /* [sequences][table_pages] */
    void *workspace;            /* 16-byte aligned, or NULL */
    size_t workspace_bytes;
    int64_t q_stride, q_head_stride, y_stride, y_head_stride, table_stride;
    int32_t sequences, heads;   /* heads: a multiple of kv_heads */
    int32_t table_pages;        /* also a bound of the lengths, by which sequences are shared */
    int32_t window;             /* 0: all tokens */
    int32_t dtype;              /* CW_DTYPE_FP16 or BF16; that of the cache unless it is E4M3 */
    float scale;                /* finite, 2^127 in magnitude at most */
} cw_attend_one_args;
int32_t cw_attend_one(cw_ctx *ctx, const cw_attend_one_args *args, void *stream);
/* Workspace that serves every call (32 MiB): more changes nothing. */
size_t cw_attend_one_workspace_bytes(void);

/* Attention of whole prompts, or of parts of them behind their histories, packed one behind the other: queries first[s]..first[s + 1] - 1 see keys
 * first_k[s]..first_k[s + 1] - 1 of their sequence.  causal: the last query sees all of the sequence's keys, the one before it all but the last, and so on
 * (query i of n those j <= i + m - n of m keys); with `window` > 0 the last `window` of these.  Else as cw_attend_one, with p in the second product in the values' type, of fp16
 * off by 2^-36 of the row's largest p at most where that is more than half a step.  Rows outside first[0]..first[sequences] - 1 are not touched. */
typedef struct {
    const void *q;              /* [tokens][heads][head_dim], dtype */
    const void *k, *v;          /* [keys][kv_heads][head_dim], dtype; rows at most 2^23 elements apart */
    void *y;                    /* [tokens][heads][head_dim], dtype */
    float *lse;                 /* [tokens][heads] or NULL */
    const int32_t *first;       /* [sequences + 1], not falling */
    const int32_t *first_k;     /* the same of the keys, or NULL: that of the queries */
    int64_t q_stride, q_head_stride, k_stride, k_head_stride, v_stride, v_head_stride, y_stride, y_head_stride;
    int32_t tokens, keys, sequences;
    int32_t heads, kv_heads;    /* heads: a multiple of kv_heads */
    int32_t head_dim;           /* a multiple of 16, up to CW_ATTEND_MOST_DIM */
    int32_t causal;             /* 0 or 1 */
    int32_t window;             /* 0: no bound; else with causal only */
    int32_t dtype;              /* CW_DTYPE_FP16 or BF16 */
    float scale;                /* finite, 2^127 in magnitude at most */
} cw_attend_args;
int32_t cw_attend(cw_ctx *ctx, const cw_attend_args *args, void *stream);

/* Device ordinal the context was created on (-1: planning only). */
int32_t cw_context_device(cw_ctx *ctx);

/* ---- the worker's executors (section 5.2: actions with `earliest` / `latest`, results) ---------
 * A cw_worker runs one executor thread per action type over one context: LOAD, UNLOAD, and for
 * INFER the three steps INPUT (runs on receipt), EXEC (inherits the action's window; one at a
 * time) and OUTPUT (follows EXEC at once), each with a stream of its own (default priority).  An
 * executor takes its actions in order of `earliest` (arrival order among equals), waits until
 * `earliest`, and does not execute an action it reaches after `latest` (CW_ERR_TOO_LATE; an
 * INFER's IO slot is released).  Every action yields exactly one result.  While a worker exists,
 * the context's own calls must not be used from other threads. */
typedef struct cw_worker cw_worker;
enum { CW_ACTION_LOAD = 1, CW_ACTION_UNLOAD = 2, CW_ACTION_INFER = 3 };
typedef struct {
    int64_t id;                 /* the caller's; returned in the result */
    int32_t type;               /* CW_ACTION_* */
    int32_t model_id;
    int32_t batch;              /* INFER */
    uint64_t earliest_ns;       /* the action may begin from this time on ... */
    uint64_t latest_ns;         /* ... and is rejected when it has not begun by this time; both on the
                                   clock of cw_worker_now_ns() */
    const void *host_in;        /* [host] LOAD: canonical blob; INFER: fp32 [batch][in_c][in_h][in_w];
                                   the caller keeps it alive and unchanged until the result arrives */
    size_t host_in_bytes;       /* LOAD: size of the blob */
    float *host_probs;          /* [host] INFER: [batch][classes], written before the result arrives */
    float *host_logits;         /* [host] INFER: same shape, or NULL */
} cw_action;
typedef struct {
    int64_t id;
    int32_t type;
    int32_t status;             /* CW_OK or the error of the step that failed */
    uint64_t begin_ns, end_ns;  /* host clock: the executor began LOAD / UNLOAD / EXEC (or rejected
                                   the action); the action was complete (INFER: outputs on the host) */
    uint64_t device_ns;         /* on-device duration: EXEC of an INFER, copy and packing of a LOAD; else 0 */
} cw_result;
/* cores [host]: NULL, or 5 CPU numbers (-1 = unpinned) for the LOAD, UNLOAD, INPUT, EXEC and
 * OUTPUT executors; the threads also ask for real-time priority (silently kept at normal
 * priority where the process may not). */
int32_t cw_worker_create(cw_ctx *ctx, const int32_t *cores, cw_worker **out);
/* Stops the executors (actions not yet begun yield no result), waits for the GPU work they
 * issued and frees the worker; the context stays. */
int32_t cw_worker_destroy(cw_worker *w);
/* Monotonic clock of the action windows and result times, in nanoseconds. */
uint64_t cw_worker_now_ns(void);
/* Copies the action [host] and queues it; returns at once.  CW_ERR_INVALID for a malformed one. */
int32_t cw_worker_submit(cw_worker *w, const cw_action *action);
/* Next finished action, in order of completion; waits up to timeout_ns (CW_ERR_TIMEOUT). */
int32_t cw_worker_next_result(cw_worker *w, cw_result *out, uint64_t timeout_ns);
/* Action profile (section 5.3): over the last 10 successful actions of (type, model, batch;
 * batch ignored unless INFER), their count, mean and largest duration (device_ns where the
 * action has one, else end - begin). */
int32_t cw_worker_profile(cw_worker *w, int32_t type, int32_t model_id, int32_t batch, uint32_t *n,
                          uint64_t *mean_ns, uint64_t *max_ns);

/* Section 5.2, "Results": a result carries success or an error code.  cw_strerror names a
 * status (static string, never NULL); cw_last_error gives the detail of the last failing call
 * on a context (NULL context: of the last failing cw_create on this thread); the string is
 * owned by the library and valid until the next call on that context. */
const char *cw_strerror(int32_t status);
const char *cw_last_error(cw_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* CLOCKWORK_EXEC_H */
