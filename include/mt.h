/*
 * mt.h - C ABI of the multi-tenant inference worker runtime for one AMD MI355X.
 *
 * The library is the internal model-execution runtime of one worker of the
 * shared inference system the paper proposes: tenants upload a DNN, then send
 * inference requests (paper, section 3); a worker hosts the DNNs of many
 * tenants at once and multiplexes their requests (section 3); models come as a
 * description of structure plus parameters and are built only from a closed set
 * of supported layer types, never from user code (section 3.1); a DNN is a
 * fixed sequence of layers applied in turn, and the answer to a request is a
 * vector of class probabilities (section 1.1).
 *
 * One mt_run serves every pending request of every tenant: requests are grouped
 * by tenant on the device, then each layer index is executed as one grouped
 * launch over all tenants (tenant-specific weights, per-tenant batch sizes), and
 * predictions come back in submission order.
 *
 * Conventions
 *   - Every call returns an mt_status; nothing aborts or throws across the ABI.
 *     mt_last_error() gives a text for the last failing call on a context.
 *   - "HOST" pointers are ordinary process memory; "DEVICE" pointers are HIP
 *     device memory on the context's GPU (e.g. a torch tensor's data_ptr()).
 *   - A context is not thread-safe.  One mt_run may be in flight per context, or
 *     cfg.run_slots of them when they are enqueued on different streams: a run
 *     takes the slot (batch descriptors, activation buffers) that its stream used
 *     last, else a slot not used yet, else the one used longest ago, whose run its
 *     stream then waits for on the device.  Result queries (mt_last_counts) refer
 *     to the run enqueued last.
 *   - Element type of weights, inputs and hidden activations is the context's
 *     dtype: MT_F32 (4 bytes) or MT_BF16 (2 bytes, bfloat16 bit patterns).
 *     Biases, logits and probabilities are always fp32.  With MT_BF16 every
 *     hidden activation is rounded to bfloat16 (nearest even) after bias and
 *     activation; accumulation over the fan-in is fp32 throughout.
 */
#ifndef MT_H
#define MT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct mt_ctx mt_ctx;

typedef enum {
    MT_OK = 0,
    MT_EINVAL = 1,       /* null pointer, zero size, value out of range            */
    MT_ENOMEM = 2,       /* weight arena or a device allocation exhausted          */
    MT_ENOTFOUND = 3,    /* tenant has no registered model                         */
    MT_EEXIST = 4,       /* tenant already has a model                             */
    MT_EUNSUPPORTED = 5, /* layer kind / activation / geometry outside the closed set */
    MT_EFULL = 6,        /* more than max_requests rows pending                    */
    MT_ESTATE = 7,       /* call not valid in this state (e.g. host-only context)  */
    MT_EDEVICE = 8       /* a HIP call failed; text in mt_last_error               */
} mt_status;

typedef enum { MT_FC = 0, MT_CONV2D = 1, MT_GAP = 2, MT_MAXPOOL = 3, MT_ADD = 4 } mt_kind;
typedef enum { MT_ACT_NONE = 0, MT_ACT_RELU = 1, MT_ACT_GELU = 2 } mt_act;
typedef enum { MT_F32 = 0, MT_BF16 = 1,
               MT_MX8 = 2,       /* rows of mt_linear4 only: e4m3 values with an e8m0 scale for every MT_MX_BLOCK of a row */
               MT_KV8 = 3        /* caches (mt_kv_cache) only: e4m3 values with an e8m0 scale for every token and head      */
} mt_dtype;

#define MT_MAX_LAYERS 48
#define MT_SEG_SLOTS 8      /* runs made of several submissions that may be in flight at once */
#define MT_MX_BLOCK 32      /* consecutive values of a row that share a scale in the 8-bit and 4-bit formats */
#define MT_SCORE_MAX_TOP 32     /* most alternatives that mt_score returns for a row */
#define MT_SCORE_MAX_GIVEN 16   /* most given classes of a row                       */

/* One layer of a model (closed set, paper section 3.1; section 1.1: DNNs are built from a few
 * dozen layer types).
 *   MT_FC:      y[n] = act(b[n] + sum_k W[n][k] x[k]); in_features = K, out_features = N.
 *   MT_CONV2D:  kh x kw cross-correlation (kh = kw = 1, 3 or 7) over an NHWC image of
 *               in_h x in_w x in_features, zero padding pad = (kh - 1) / 2, stride 1 or 2,
 *               out_features output channels (a multiple of 8; in_features too, except in a
 *               model's first layer), bias per channel, then act.  Output size
 *               floor((in + 2 pad - kh) / stride) + 1 each way.
 *   MT_GAP:     mean over in_h x in_w of every one of in_features channels
 *               (out_features must equal in_features, act must be MT_ACT_NONE).
 *   MT_MAXPOOL: maximum over a kh x kw window (kh = kw = 2 or 3), stride 1 or 2, pad 0 or 1
 *               (below kh); positions outside the image never win.  out_features = in_features,
 *               act MT_ACT_NONE.
 *   MT_ADD:     act(a + b) elementwise, a residual connection: a and b are the outputs of two
 *               earlier layers of the same shape in_h x in_w x in_features (out_features =
 *               in_features).
 * A layer reads the output of the layer before it (layer 0: the request), unless src says
 * otherwise: src = j + 1 reads the output of layer j (j below this layer's index), src = 0 the
 * previous layer.  MT_ADD takes its second operand from src2 the same way (src2 must be given).
 * Image layers (convolution, max-pool, add) pass NHWC images on; MT_FC reads a vector, so it
 * follows MT_FC or MT_GAP (or is the first layer).  The activation of a model's last layer,
 * which must be MT_FC, must be MT_ACT_NONE: its outputs are the logits.  At most four layer
 * outputs may be alive at once (a chain needs two; a residual block with a projection three). */
typedef struct {
    uint32_t kind, act;
    uint32_t in_features, out_features;
    uint32_t in_h, in_w, kh, kw, stride, pad;
    uint32_t src, src2;
} mt_layer_spec;

typedef struct {
    uint32_t max_tenants;   /* tenant ids are 0 .. max_tenants-1                         */
    uint32_t max_requests;  /* most rows that may be pending for one mt_run              */
    uint32_t max_width;     /* most elements any request occupies at any layer boundary  */
    uint32_t max_classes;   /* most outputs of any model's last layer                    */
    uint64_t arena_bytes;   /* size of the packed weight arena in device memory          */
    uint32_t dtype;         /* mt_dtype of weights / inputs / hidden activations         */
    int32_t  device;        /* HIP device ordinal; -1 = host-only context: registration,
                               validation and accounting work, mt_run returns MT_ESTATE  */
    uint32_t run_slots;     /* runs that may be in flight at once, each on a stream of its
                               own (batch interleaving, footnote of paper section 1.3): 0
                               or 1 = one; at most 4.  Every slot has its own batch
                               descriptors and activation buffers; the weights are shared */
    uint32_t cache;         /* 1: the arena is a cache of the registered models (paper
                               section 3.3): every model's packed weights stay in pinned
                               host memory, registering or prefetching a model when the
                               arena is full evicts the models used least recently, and
                               evicted models are reloaded on demand (mt_prefetch).
                               0: every registered model stays resident; a full arena
                               is MT_ENOMEM                                              */
} mt_config;

/* Where mt_run writes predictions.  All DEVICE memory owned by the caller, valid
 * until the stream work of that mt_run has completed.  Row i belongs to the i-th
 * submitted row.  logits and probs have row_stride floats per row; columns at and
 * past n_classes[i] are written as 0.  A row whose tenant id was out of range or
 * had no model gets label -1, n_classes 0 and zero rows.  logits, probs and
 * n_classes may each be NULL to skip that output. */
typedef struct {
    int32_t*  labels;      /* [capacity]                                  */
    float*    probs;       /* [capacity * row_stride]                     */
    float*    logits;      /* [capacity * row_stride]                     */
    int32_t*  n_classes;   /* [capacity]                                  */
    uint32_t  capacity;    /* rows the buffers can hold, >= pending rows  */
    uint32_t  row_stride;  /* floats per row, >= max_classes              */
} mt_outputs;

typedef struct {
    uint32_t n_tenants;          /* models registered                                  */
    uint64_t arena_used;         /* bytes of the arena in use (padded layouts)         */
    uint64_t arena_bytes;
    uint32_t last_run_rows;      /* rows consumed by the last mt_run                   */
    uint32_t last_run_launches;  /* kernels the last mt_run enqueued                   */
} mt_stats;

/* Create a worker context (paper section 3: a worker is a long-lived process that hosts the
 * DNNs of many tenants at once; section 3.3: their weights stay in device memory): allocates
 * the weight arena, the tenant table, and per run slot the batch descriptors and two
 * activation buffers of max_requests * max_width elements on cfg->device.  Serving calls
 * (submit, run, prefetch) allocate no device memory; registering a model with skip connections
 * adds the third or fourth activation buffer its layer graph needs.
 * Errors: MT_EINVAL (null / zero sizes), MT_ENOMEM, MT_EDEVICE. */
mt_status mt_create(mt_ctx** out, const mt_config* cfg);

/* Free everything the context owns (synchronises the device first). */
mt_status mt_destroy(mt_ctx* ctx);

/* Upload a tenant's DNN (paper section 3: a tenant hands over its model before it sends requests).
 *   specs[n_layers]: layer chain; out length of layer l must equal in length of l+1.
 *   weights[l]: HOST, context dtype; FC [N][K] row-major, CONV [C_out][C_in][kh][kw];
 *               ignored (may be NULL) for the kinds without parameters.
 *   biases[l]:  HOST fp32 [N] or [C_out]; NULL means zeros.
 * Weights are copied and repacked into the arena before the call returns; the caller
 * keeps ownership of its buffers.  Nothing is allocated when the call fails.
 * A run serves the models registered when mt_run is called; rows of one registered since, while
 * the run is still queued, are answered like those of a tenant without a model (label -1).  A run
 * that was captured in a graph goes on, when it is replayed, to serve models registered since that
 * its launches cover: those with the layers of one that was registered at the capture (and finite
 * weights, like it), so a tenant's model can be replaced by one with other weights.
 * Errors: MT_EINVAL, MT_EEXIST, MT_EUNSUPPORTED (kind/act/geometry outside the closed
 * set, dims that do not chain, more than MT_MAX_LAYERS layers, widths beyond
 * max_width / max_classes), MT_ENOMEM (arena full), MT_EDEVICE. */
mt_status mt_register_model(mt_ctx* ctx, uint32_t tenant, const mt_layer_spec* specs, uint32_t n_layers,
                            const void* const* weights, const void* const* biases);

/* mt_register_model for models whose convolutions are followed by batch normalisation, which the
 * library folds into the convolution (the models of paper section 1.1 are built that way; the
 * runtime executes the folded form).  bn[l]: HOST fp32 [4][C_out] = gamma, beta, running mean,
 * running variance of the normalisation behind convolution l, or NULL for none (must be NULL for
 * other kinds); bn itself may be NULL.  With s = gamma / sqrt(var + bn_eps) per output channel the
 * layer becomes W' = round(W * s), b' = float((b - mean) * s + beta), computed in double
 * precision from the given values and rounded once, W' to the context's element type (nearest
 * even) and b' to fp32; the layer's act applies after it.  Errors: as mt_register_model, and
 * MT_EINVAL for a variance + eps that is not positive. */
mt_status mt_register_model_bn(mt_ctx* ctx, uint32_t tenant, const mt_layer_spec* specs, uint32_t n_layers,
                               const void* const* weights, const void* const* biases, const float* const* bn, float bn_eps);

/* Remove a tenant's model and return its arena slice.  Must not be called while an
 * mt_run that may serve the tenant is still executing.  Errors: MT_ENOTFOUND. */
mt_status mt_unregister_model(mt_ctx* ctx, uint32_t tenant);

/* Queue n_rows requests of ONE tenant for the next mt_run (paper section 3: once its
 * model is in place a tenant sends inference requests).  inputs: DEVICE, n_rows rows of the model's
 * input length, contiguous, context dtype; borrowed until the next mt_run's stream
 * work has completed.  *first_index (optional) receives the submission index of the
 * first row.  Errors: MT_EINVAL, MT_ENOTFOUND, MT_EFULL. */
mt_status mt_submit(mt_ctx* ctx, uint32_t tenant, const void* inputs, uint32_t n_rows, uint32_t* first_index);

/* Queue n_rows requests of MIXED tenants in arrival order (paper section 3: a worker receives
 * the incoming requests of all the tenants it hosts and multiplexes them), with the tenant id of
 * every row already in device memory (what a request front-end that lands ids and
 * payloads in GPU memory would hand over).  tenant_ids: DEVICE int32 [n_rows];
 * inputs: DEVICE, row i at inputs + i*row_stride elements, each row holding its
 * tenant's input length; row_stride must be at least the longest input of any
 * registered model (else MT_EINVAL), so that no row read can leave the buffer.  Ids are validated on the device: rows of
 * unknown tenants are answered with label -1 and never touch any model's weights.
 * Both buffers are borrowed like in mt_submit.  Errors: MT_EINVAL, MT_EFULL. */
mt_status mt_submit_batch(mt_ctx* ctx, const int32_t* tenant_ids, const void* inputs, uint32_t n_rows,
                          uint32_t row_stride, uint32_t* first_index);

/* Serve everything pending (paper section 3: the worker multiplexes the requests of many
 * models; section 1.1: a model is evaluated by applying its layers in turn, and the answer to
 * a request is a vector of class probabilities): enqueue, on hip_stream (a hipStream_t, NULL =
 * default stream), tenant segmentation, the gather into tenant-contiguous rows, one grouped
 * launch per layer index and kind, and the softmax/argmax head; write predictions to *out in
 * submission order.  Never waits for the GPU and allocates nothing; clears the pending list
 * (also when it fails after part of the run has been enqueued: those rows are lost and their
 * outputs undefined).  *n_rows (optional) receives the number of rows served.  With nothing
 * pending it returns MT_OK and serves 0 rows.  Errors: MT_EINVAL (out too small), MT_ESTATE,
 * MT_EFULL (the run is made of several submissions and the tables of MT_SEG_SLOTS earlier
 * such runs are all still being read by the GPU: nothing was enqueued, the pending list is
 * kept, call again later), MT_EDEVICE. */
mt_status mt_run(mt_ctx* ctx, void* hip_stream, const mt_outputs* out, uint32_t* n_rows);

/* What a model needs of a context, from its description alone (no context, no device): the
 * bytes its packed weights occupy in the arena (padded layouts, what mt_register_model takes
 * from cfg.arena_bytes and what an upload moves: the fixed footprint of paper section 3.3),
 * the max_width and max_classes a context must have to accept it, and the length of one
 * request's input.  dtype: mt_dtype.  Errors: MT_EINVAL (null), MT_EUNSUPPORTED (a chain that
 * mt_register_model would reject for its kinds, activations or geometry). */
typedef struct {
    uint64_t arena_bytes;
    uint32_t min_width;      /* smallest cfg.max_width that accepts the model   */
    uint32_t n_classes;      /* smallest cfg.max_classes that accepts the model */
    uint32_t in_len;         /* elements of one request's input                 */
    uint32_t reserved;
} mt_model_footprint;
mt_status mt_model_footprint_get(const mt_layer_spec* specs, uint32_t n_layers, uint32_t dtype, mt_model_footprint* out);

/* mt_run for callers that may not allocate device memory around the call and want a run that
 * touches no allocation of the context besides its weights and tables: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  It does what mt_run does,
 * with the same kernels, but the run's scratch (batch descriptors, both activation buffers,
 * logits) lives in one array of MT_STATIC_SCRATCH_BYTES that the library holds in device
 * memory for the life of the process (one per GPU).  A run whose scratch does not fit (the
 * need grows with the pending rows, the context's max_width, max_classes and max_tenants) is
 * refused with MT_EINVAL and nothing is enqueued; the pending list is kept, so mt_run can
 * serve it.  The call allocates nothing, on the device or through any allocating routine.
 * Every call on a GPU shares that GPU's array: the descriptors a run starts from are cleared
 * on the stream first, and runs enqueued through this call on different streams (or from
 * different contexts) that overlap on one GPU race; runs of one context are ordered by the
 * library (a later one waits for the earlier one on the device).  Other errors as mt_run. */
#define MT_STATIC_SCRATCH_BYTES (16u << 20)
mt_status mt_run_static(mt_ctx* ctx, void* hip_stream, const mt_outputs* out, uint32_t* n_rows);

/* The per-tenant batch sizes of the last mt_run (paper section 3.2: the cost of a run varies
 * with the batch size of every model in it, which the device-side segmentation computes):
 * copies the counts to HOST counts[max_tenants] after synchronising the stream the run was
 * enqueued on.  For tests and accounting. */
mt_status mt_last_counts(mt_ctx* ctx, uint32_t* counts);

/* Model cache (cfg.cache; paper section 3.3: a worker alternates between many tenants'
 * models, most requests find their model cached, and the cost of a miss is predictable
 * because a model's footprint is fixed).  mt_prefetch makes the n named models resident:
 * models that are not are copied from their pinned host images to the arena on `stream`
 * without waiting, after the least recently used other models have given way (a model
 * named in this call never gives way to another one of it).  The copies queue up behind
 * every run in flight, and a later mt_run on any stream waits for them on the device;
 * nothing blocks the host.  mt_run itself prefetches the tenants of pending mt_submit
 * calls; tenants that appear only in mt_submit_batch id arrays have to be prefetched by the
 * caller (the router knows them), else their rows are answered like rows of a tenant without
 * a model.  "Used" means registered or named in a prefetch.  Outside cache mode the call only
 * checks its arguments.  Errors: MT_EINVAL, MT_ENOTFOUND (a tenant without a model),
 * MT_ENOMEM (the named models do not fit the arena together; those named first may have
 * been brought in), MT_EDEVICE. */
mt_status mt_prefetch(mt_ctx* ctx, const uint32_t* tenants, uint32_t n, void* hip_stream);

typedef struct {
    uint32_t resident_models;
    uint64_t uploads, upload_bytes;   /* models copied to the arena so far (registration included) */
    uint64_t evictions;               /* models that gave way                                       */
} mt_cache_stats;
mt_status mt_cache_stats_get(const mt_ctx* ctx, mt_cache_stats* out);

/* Per-tenant accounting.  A request's cost follows from the model description alone
 * (paper section 3.2: the flops of every layer are known a priori), so billing by work
 * done (section 1.3) needs only a count of the requests served, which the batcher keeps
 * on the device.  flops_per_request = 2 x multiply-accumulates over all layers with the
 * true dimensions (convolutions count all nine taps at every output pixel);
 * weight_bytes = the parameters (true dimensions, the context's element type) and fp32
 * biases; io_bytes_per_request = the request's input, every hidden activation written
 * once and read once, logits, probabilities and label.
 * requests / runs count what every mt_run enqueued so far has served of this tenant and
 * in how many runs it had at least one request (the call synchronises the device; 0 for a
 * host-only context).  Errors: MT_EINVAL, MT_ENOTFOUND (no model), MT_EDEVICE. */
typedef struct {
    uint64_t requests, runs;
    uint64_t flops_per_request, weight_bytes, io_bytes_per_request;
    uint64_t resident;      /* 1: the model is in the device arena now                    */
    uint64_t arena_bytes;   /* bytes it occupies there (padded layouts): what an upload moves */
} mt_tenant_account;
mt_status mt_tenant_account_get(mt_ctx* ctx, uint32_t tenant, mt_tenant_account* out);

/* Predicted cost of one mt_run that serves counts[t] requests of tenant t (HOST array of
 * max_tenants entries; tenants without a model must have 0), from the registered
 * descriptors alone, before anything is enqueued (section 3.2: inference is a fixed
 * sequence of operations, so its cost is predictable; an admission controller picks
 * what enters the next run from this).  flops and hbm_bytes are the algorithmic work
 * (weights of active tenants read once, activations written once and read once);
 * launches is the number of kernels mt_run will enqueue (for the requests as they are pending,
 * or for others in one submission: a run of fully-connected models may take one launch more in
 * several submissions, and one more while its stream is being captured, or two if a model has
 * 33 to 128 classes); device_ms is the predicted
 * time of the run alone on the GPU, from a per-kernel model (fixed cost per launch +
 * bytes through HBM + bytes re-read through L2, or tile rounds for compute-bound
 * launches) whose constants were fitted on one MI355X.  Works on a host-only context.
 * Errors: MT_EINVAL (null, or more rows than max_requests), MT_ENOTFOUND (rows for a
 * tenant without a model). */
typedef struct {
    double flops, hbm_bytes, device_ms;
    uint32_t rows, launches;
    double upload_bytes, upload_ms;   /* models with requests that are not resident now: bytes to
                                         bring in first, and the predicted time of that copy  */
} mt_run_estimate;
mt_status mt_estimate_run(mt_ctx* ctx, const uint32_t* counts, mt_run_estimate* out);

/* Admission (paper section 3.2: because a run's cost is predictable before it runs, the
 * system can decide what to admit so that latency targets hold and no tenant starves the
 * others).  pending[t] = requests of tenant t waiting (HOST, max_tenants entries);
 * budget_ms = the device time the next run may take (uploads of models that are not
 * resident count towards it).  admitted[t] receives a max-min fair share: every tenant gets
 * min(pending[t], level) requests, with the highest level whose predicted run
 * (mt_estimate_run) fits the budget and max_requests; est (optional) receives the prediction
 * for the admitted mix.  A budget that not even one request per waiting tenant fits admits
 * nothing (level 0).  Works on a host-only context.  Errors: MT_EINVAL (null, budget <= 0),
 * MT_ENOTFOUND (requests pending for a tenant without a model). */
mt_status mt_admit(mt_ctx* ctx, const uint32_t* pending, double budget_ms, uint32_t* admitted, mt_run_estimate* est);

mt_status mt_get_stats(const mt_ctx* ctx, mt_stats* out);

/* ---- Answers of language models -------------------------------------------------------------
 * The step behind a language model's layers, for rows of many tenants at once: mt_add_norm adds a
 * layer's output to the residual stream and normalises it, mt_linear4 multiplies the rows of every
 * tenant by that tenant's 4-bit weights (hidden layers, or the last one over a vocabulary), and
 * mt_score says what the resulting logits (or those of mt_run) say about given classes.  Unlike the
 * models of mt_run these are single operators: the caller holds every buffer between them.
 *
 * All pointers in the argument blocks are DEVICE memory of the context's GPU, borrowed until the work
 * enqueued on hip_stream (a hipStream_t, NULL = default stream) has completed; the blocks themselves and
 * group lists are HOST memory that may change as soon as the call returns.  Strides are in
 * elements between consecutive rows (scales: in bytes, masks: in words); pointers and strides need the
 * alignment of one element, nothing more.  The calls allocate nothing, never wait for the GPU, may be
 * captured in a graph, and keep nothing between calls.  0 rows: MT_OK, nothing is enqueued.  Calls on different streams
 * are independent as long as their buffers are (scratch too).
 *
 * 8-bit rows: values e4m3 (1 sign, 4 exponent, 3 mantissa bits, no infinities, 0x7f and 0xff NaN),
 * and for every MT_MX_BLOCK consecutive values of a row, counted from its start, a scale e8m0 (a power of two,
 * 2^(byte - 127); 0xff is NaN); a row's last block may be shorter.  4-bit weights: e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives, the sign is bit 3), with scales of the same kind along the fan-in. */

/* h = x + residual; y = h / sqrt(mean(h^2) + eps) * gain, row by row, in fp32, every output rounded once.  Rows of finite h may have any
 * magnitude, also where h^2 leaves fp32's range.
 *   sum (h), y: in dtype; y8 with y8_scales: 8-bit rows, a block's scale the least power of two (2^-126 at least) at which none
 *   of its values exceeds 448, 1 where all are zero; where one is infinite or NaN the block's scale and values are NaN.
 * sum, y and y8 (with its scales) may each be NULL, not all of them; sum may be x or residual itself (same stride),
 * y may be x or residual where sum is not; other overlaps of outputs with anything are not allowed.
 * gain_ids[i] names row i's gain among n_gains (a tenant's); a row whose id is out of range gets y and y8 of zeros
 * (scales 1) and touches no gain.  gain_ids NULL: every row takes the first; gain NULL: no gain is applied.
 * Errors: MT_EINVAL (null, zero width, a stride below the width, eps negative or not finite, n_gains 0 with a gain),
 * MT_EUNSUPPORTED (dtype other than MT_F32 and MT_BF16, width over 2^24), MT_ESTATE (host-only context), MT_EDEVICE. */
typedef struct {
    const void* x;              /* [rows][x_stride], dtype                     */
    const void* residual;       /* [rows][residual_stride], dtype, or NULL     */
    const float* gain;          /* [n_gains][gain_stride], or NULL             */
    const int32_t* gain_ids;    /* [rows], or NULL                             */
    void* sum;                  /* [rows][sum_stride], dtype, or NULL          */
    void* y;                    /* [rows][y_stride], dtype, or NULL            */
    uint8_t* y8;                /* [rows][y8_stride], or NULL                  */
    uint8_t* y8_scales;         /* [rows][y8_scales_stride]                    */
    uint64_t x_stride, residual_stride, gain_stride, sum_stride, y_stride, y8_stride, y8_scales_stride;
    uint32_t rows, width, n_gains, dtype;
    float eps;
    uint32_t reserved;
} mt_norm_args;
mt_status mt_add_norm(mt_ctx* ctx, void* hip_stream, const mt_norm_args* args);

/* Bring a tenant's 4-bit matrix [out_features][in_features] into the context's arena.
 *   codes: HOST, (in_features + 1) / 2 bytes a row, two e2m1 values to a byte, the even column in the low half;
 *   scales: HOST e8m0, (in_features + 31) / 32 bytes a row, 27 .. 227 (2^-100 .. 2^100);
 *   bias: HOST fp32 [out_features], or NULL for none.
 * *matrix receives its number.  Matrices never give way to models (in a cache context models give way to them); any
 * number of them may be registered beside the tenants' models.  The call is synchronous, like mt_register_model.
 * mt_matrix4_footprint_get gives the bytes of arena it takes.  Errors: MT_EINVAL, MT_EUNSUPPORTED (a scale outside
 * the range, more than 2^24 features), MT_ENOMEM, MT_EDEVICE. */
mt_status mt_register_matrix4(mt_ctx* ctx, uint32_t out_features, uint32_t in_features, const uint8_t* codes, const uint8_t* scales,
                              const float* bias, uint32_t* matrix);
mt_status mt_matrix4_footprint_get(uint32_t out_features, uint32_t in_features, uint64_t* arena_bytes);

/* Take a matrix out of the arena (synchronises the device first); its number may be given out again.  Errors: MT_ENOTFOUND. */
mt_status mt_unregister_matrix4(mt_ctx* ctx, uint32_t matrix);

/* y[i][n] = act(bias[n] + sum_k W[n][k] x[i][k]) for the rows i of each group, W and bias those of the group's
 * matrix: one call serves the rows of many tenants.  Products are exact, sums fp32, y is rounded once.  (Rows are bf16 values on their way: of fp32 rows, and of
 * 8-bit rows with scales below 2^-124, bits below 2^-133 are left out; 8-bit values beyond 255 * 2^120, which take scales above 2^119, count as infinite.)
 * GELU is z Phi(z) of the sum z, in fp32 within 2^-19 + z^2 2^-22 of itself, for MT_BF16 within 2^-16 + z^2 2^-22 before the rounding; of -infinity it is NaN.
 * Columns of y from a matrix's out_features on, and rows in no group, are left as they are.
 * Groups come in the order of their rows and share none; a group of 0 rows is skipped.
 * Errors: MT_EINVAL (null, strides below a matrix's sizes, rows outside 0..rows or out of order), MT_ENOTFOUND (a
 * matrix that is not registered), MT_EUNSUPPORTED (types, activation, a group of outputs beyond 2^23 workgroups of 16 x 16 or
 * more each), MT_ESTATE (host-only context), MT_EDEVICE.  After an error the groups' outputs may be written in part. */
typedef struct { uint32_t matrix, first_row, n_rows; } mt_row_group;
typedef struct {
    const void* x;              /* [rows][x_stride], x_dtype                           */
    const uint8_t* x_scales;    /* [rows][x_scales_stride], with MT_MX8; else NULL     */
    void* y;                    /* [rows][y_stride], y_dtype; may not overlap x        */
    uint64_t x_stride, x_scales_stride, y_stride;
    uint32_t rows;
    uint32_t x_dtype;           /* MT_F32, MT_BF16 or MT_MX8   */
    uint32_t y_dtype;           /* MT_F32 or MT_BF16           */
    uint32_t act;               /* mt_act                      */
} mt_linear4_args;
mt_status mt_linear4(mt_ctx* ctx, void* hip_stream, const mt_linear4_args* args, const mt_row_group* groups, uint32_t n_groups);

/* The same for rows that are narrower than their strides (a slice of columns of a wider buffer): MT_EINVAL, and nothing is touched, where a
 * group with rows has a matrix of more than x_width in_features or y_width out_features. */
mt_status mt_linear4_within(mt_ctx* ctx, void* hip_stream, const mt_linear4_args* args, const mt_row_group* groups, uint32_t n_groups,
                            uint32_t x_width, uint32_t y_width);

/* What rows of logits say, with p = softmax(logits / temperature) over a row's allowed classes: those below
 * n_classes[i] (NULL: all; the n_classes of mt_run fits) whose bit of `allowed` is set (bit c % 32 of word c / 32; NULL: all) and
 * whose logit is not -infinity.  Everything is optional but the logits and one output:
 *   given_logprobs[i][g] = log p of class given[i][g]; given_ranks[i][g] = allowed classes in front of it, in the order
 *     of falling logits, lower numbers first among equals.  A class that is not allowed, or no class: -infinity and -1.
 *   entropy[i] = -sum p log p (natural logarithm), 0 for a row without an allowed class.
 *   top_ids[i][k], top_logprobs[i][k]: the first `top` classes in that order; past the last allowed one -1 and -infinity.
 * A log probability beyond fp32's range is -infinity.
 * A row with a NaN or +infinity among its allowed classes has no distribution: NaN and -1 (entries that are -infinity
 * and -1 for want of a class stay so).  What stands in classes that are not allowed does not matter.
 * scratch: DEVICE memory of mt_score_scratch_get's size for the call's sizes, which few rows of many classes share among
 * workgroups; zero before its first use, left ready for the next call (of any sizes that it is large enough for), and
 * used by one call at a time.  NULL where that size is 0.
 * Errors: MT_EINVAL (null, no classes, a stride below the classes, temperature below 2^-126 or not finite, given without
 * classes, scratch too small, top or n_given beyond their limits), MT_EUNSUPPORTED (dtype), MT_ESTATE, MT_EDEVICE. */
typedef struct {
    const void* logits;             /* [rows][row_stride], dtype                        */
    const int32_t* n_classes;       /* [rows], or NULL; taken into 0 .. classes         */
    const uint32_t* allowed;        /* [rows][allowed_stride], or NULL                  */
    const int32_t* given;           /* [rows][n_given], or NULL with n_given 0          */
    float* given_logprobs;          /* [rows][n_given], or NULL                         */
    int32_t* given_ranks;           /* [rows][n_given], or NULL                         */
    float* entropy;                 /* [rows], or NULL                                  */
    int32_t* top_ids;               /* [rows][top], or NULL                             */
    float* top_logprobs;            /* [rows][top], or NULL                             */
    void* scratch;
    uint64_t scratch_bytes;
    uint64_t row_stride, allowed_stride;
    uint32_t rows, classes, n_given, top;
    uint32_t dtype;                 /* MT_F32 or MT_BF16                                */
    float temperature;
} mt_score_args;
mt_status mt_score(mt_ctx* ctx, void* hip_stream, const mt_score_args* args);
mt_status mt_score_scratch_get(uint32_t rows, uint32_t classes, uint32_t n_given, uint32_t top, uint64_t* bytes);

/* ---- Caches of language models ---------------------------------------------------------------
 * Keys and values of the tokens that tenants' sequences have seen, in pages of a few tokens: mt_kv_write puts new tokens'
 * into their places, mt_attend lets new tokens attend to all of their sequence, the mt_kv_ calls on pages give, share, take back and
 * move them, and mt_sample chooses the token that comes next.  Conventions as above: DEVICE pointers (argument blocks and this struct are HOST memory),
 * nothing is allocated or waited for, every call may be captured, and what it decides from lengths and tables it decides on the device.
 *
 * Sequence s has lengths[s] tokens; its token t is slot t % page_tokens of page table[s][t / page_tokens].  So it holds its table's first
 * ceil(lengths[s] / page_tokens) entries, and only they are looked at.  refs[p] counts the sequences that hold page p: 0 is free.  A cache starts with
 * lengths and refs of 0; whoever prefers books of their own writes tables and lengths and leaves the calls on pages alone.
 * A page that only some sequences have filled is held by one of them: full pages may be shared.  Calls that read or write one cache go on one
 * stream, or are put in order by the caller; calls that only read it (mt_attend) may overlap.
 * Values are held feature by feature, a page's tokens side by side: that is how the products over tokens read them.
 * In MT_KV8 a token's head_dim elements of one head share a scale, the least power of two (2^-126 at least) at which none exceeds 448; 1 where all
 * are zero; infinite or NaN elements make scale and values of that token and head NaN. */
#define MT_KV_MAX_SEQS 16384     /* most sequences of a cache                     */
#define MT_KV_MAX_WIDTH 131072   /* most pages of a sequence                      */
#define MT_KV_MAX_DIM 256        /* largest head_dim                              */
#define MT_SAMPLE_MAX_CLASSES (1u << 20)
typedef struct {
    void* k;                    /* [layers][n_pages][heads][page_tokens][head_dim]; of page_stride, layer_stride elements  */
    void* v;                    /* [layers][n_pages][heads][head_dim][page_tokens]; the same strides                       */
    uint8_t* k_scales;          /* [layers][n_pages][heads][page_tokens], with MT_KV8, else NULL; of scales_..._stride bytes */
    uint8_t* v_scales;          /* the same                                                                                */
    int32_t* table;             /* [seqs][table_stride]                                                                    */
    int32_t* lengths;           /* [seqs]                                                                                  */
    int32_t* refs;              /* [n_pages]; calls on pages only                                                          */
    void* work;                 /* work_bytes of mt_kv_work_get's size, 16-byte boundary; calls on pages only              */
    uint64_t page_stride, layer_stride, scales_page_stride, scales_layer_stride, table_stride, work_bytes;
    uint32_t dtype;             /* MT_F32, MT_BF16 or MT_KV8                                                               */
    uint32_t layers, n_pages, heads;
    uint32_t page_tokens;       /* 16, 32, 64, 128 or 256                                                                  */
    uint32_t head_dim;          /* a multiple of 16 up to MT_KV_MAX_DIM                                                    */
    uint32_t seqs, table_width;
} mt_kv_cache;
/* Errors of a cache in every call: MT_EINVAL (null k, v, table or lengths, scales with other types than MT_KV8 or missing with it, sizes of 0, pages,
 * strides or scales that are not on 16 bytes, strides that make pages or layers overlap, table_stride below table_width), MT_EUNSUPPORTED (dtype,
 * page_tokens, head_dim, more than MT_KV_MAX_SEQS or MT_KV_MAX_WIDTH, 2^31 pages or more). */

/* The rows of a call and whose they are: rows first_row[b] .. first_row[b + 1] - 1 are the last tokens, in their order, of sequence seqs[b], whose length
 * counts them already.  seqs NULL: sequence b.  first_row NULL: row b (rows = n_seqs).  Rows in no sequence are left as they are; a row that first_row would put outside 0 .. rows is
 * none.  max_new: the most rows of a sequence, which the work is cut by; more are served too, but slowly.  No row stands in two sequences. */
typedef struct {
    const int32_t* seqs;        /* [n_seqs], or NULL          */
    const int32_t* first_row;   /* [n_seqs + 1], or NULL      */
    uint32_t rows, n_seqs, max_new;
    uint32_t reserved;
} mt_kv_batch;

/* Keys and values of the batch's rows into the pages of one layer: [heads][head_dim] elements a row, rounded once.  A row without a place (its sequence's
 * number out of range, its token beyond the table's width, its page's number out of range, more rows than tokens) is not written.
 * Errors: MT_EINVAL (null, a stride below heads x head_dim, layer out of range, rows other than n_seqs without first_row, max_new 0), MT_EUNSUPPORTED (rows neither MT_F32 nor MT_BF16, or
 * of another type than a cache that is not MT_KV8; more than 2^20 sequences in a batch, or 2^23 pairs of these and heads), MT_ESTATE (host-only context), MT_EDEVICE. */
typedef struct {
    const void* k;              /* [rows][k_stride], dtype    */
    const void* v;              /* [rows][v_stride], dtype    */
    uint64_t k_stride, v_stride;
    uint32_t dtype, layer;
} mt_kv_write_args;
mt_status mt_kv_write(mt_ctx* ctx, void* hip_stream, const mt_kv_cache* cache, const mt_kv_batch* batch, const mt_kv_write_args* args);

/* out = sum_t p_t v_t with p = softmax(scale * q.k_t) over the tokens t that a row sees, head by head: those up to itself, of these the last `window` (0: all).
 * q_heads is a multiple of the cache's heads; query heads h * q_heads / heads and on share head h of the cache.  lse = log sum_t e^(scale q.k_t), with
 * which results over several caches can be joined.  Products are exact for MT_BF16 and fp32 for MT_F32; sums and statistics are fp32; where rows are MT_BF16 weights
 * are off by up to 2^-16 of themselves on top; out is rounded once.  Sums are divided last and hold weights of up to 2^8 for every token: where those times the values (or these alone) leave fp32's range,
 * out is infinite or NaN.
 * A NaN among a row's products makes out and lse NaN; else one of +infinity (or beyond fp32's range) out NaN and lse +infinity.
 * A row that sees nothing (no tokens, its sequence's number out of range, or all its products -infinity) gets out 0 and lse -infinity.  Tokens in pages whose
 * number is out of range, or beyond the table's width, are not seen.  What stands in tokens that are not seen does not matter.
 * max_length: tokens of the longest sequence, which the work is cut by (0: the table's width); longer ones are served too, but slowly.
 * scratch: as in mt_score, of mt_attend_scratch_get's size for the call's sizes.
 * Errors: MT_EINVAL (null, q_heads no multiple of heads or 0, strides below q_heads x head_dim, layer out of range, scale not finite or beyond 1e38, scratch too small),
 * MT_EUNSUPPORTED (as in mt_kv_write, and more than 65535 query heads), MT_ESTATE, MT_EDEVICE. */
typedef struct {
    const void* q;              /* [rows][q_stride], dtype           */
    void* out;                  /* [rows][out_stride], dtype; may be q itself (same stride)  */
    float* lse;                 /* [rows][q_heads], or NULL          */
    void* scratch;
    uint64_t scratch_bytes;
    uint64_t q_stride, out_stride;
    uint32_t q_heads, dtype, layer, window, max_length;
    float scale;
} mt_attend_args;
mt_status mt_attend(mt_ctx* ctx, void* hip_stream, const mt_kv_cache* cache, const mt_kv_batch* batch, const mt_attend_args* args);
mt_status mt_attend_scratch_get(const mt_kv_cache* cache, const mt_kv_batch* batch, uint32_t q_heads, uint32_t max_length, uint64_t* bytes);

/* Calls on pages.  Lists are DEVICE int32 [n], n at most the cache's seqs.  An entry that names no sequence (out of range) does nothing, nor does one whose
 * sequence an earlier entry of the call has named (of mt_kv_fork: as a child).  granted[i] (or NULL): 1 where entry i was served, 0 where not.
 *
 * mt_kv_grow: room for tokens[i] more tokens of sequence seqs[i] (NULL: i); its length counts them from now on.  Entries take pages in the order of the list, free pages in the order
 *   of their numbers.  An entry that would need more than table_width pages, or whose tokens are negative, takes none; one for whose pages, with all
 *   before it, there are not enough free ones changes nothing; what needs no page is always served.
 * mt_kv_fork: sequence children[i], which has no tokens, becomes a copy of sequence parents[i] as it was before the call: full pages are shared, a last page that is not full is copied into
 *   a free one (all layers), taken as in mt_kv_grow.
 * mt_kv_free: the sequences' pages are let go (table entries -1), their lengths are 0.
 * mt_kv_compact: with n pages held, these are pages 0 .. n - 1 afterwards: the i-th held one from number n on moves into the i-th free one below (all layers), and the
 *   tables follow.  *live (DEVICE, or NULL) receives n.
 * mt_kv_copy: page from[i] is copied over page to[i] (all layers); tables and counts stay.  A pair out of range, or whose target an entry behind it names again, does nothing; a
 *   pair whose page from[i] is another pair's target leaves any mix of what that page held before and after in page to[i]: chains take a call for each link.  n may be any number.
 * Errors: MT_EINVAL (null list, refs or work, work too small, n over seqs), MT_ESTATE, MT_EDEVICE. */
mt_status mt_kv_grow(mt_ctx* ctx, void* hip_stream, const mt_kv_cache* cache, const int32_t* seqs, const int32_t* tokens, uint32_t n, int32_t* granted);
mt_status mt_kv_fork(mt_ctx* ctx, void* hip_stream, const mt_kv_cache* cache, const int32_t* parents, const int32_t* children, uint32_t n, int32_t* granted);
mt_status mt_kv_free(mt_ctx* ctx, void* hip_stream, const mt_kv_cache* cache, const int32_t* seqs, uint32_t n);
mt_status mt_kv_compact(mt_ctx* ctx, void* hip_stream, const mt_kv_cache* cache, int32_t* live);
mt_status mt_kv_copy(mt_ctx* ctx, void* hip_stream, const mt_kv_cache* cache, const int32_t* from, const int32_t* to, uint32_t n);
mt_status mt_kv_work_get(uint32_t n_pages, uint32_t seqs, uint64_t* bytes);

/* One class for every row of logits, drawn with the row's own settings (DEVICE fp32 or int32 [rows]; NULL: the setting that changes nothing).  Allowed classes and
 * their order (falling logits, lower numbers first among equals) are mt_score's; w = e^((x - max) / temperature).  A row keeps
 *   of its allowed classes the first top_k (0 or less: all), of these those with w >= min_p (0 or less: all; more than 1 counts as 1), of these the shortest front part that has top_p of their
 *   weight (1 or more: all; the first always).
 * Drawn is the first kept class, in the order of class numbers, up to which the kept classes have more than uniform[i] of their weight (uniform in [0, 1): a class is drawn with
 * its share of the weight); with uniform of 1 or more the last one of any weight.  temperature 0 (or below 2^-126) keeps the first class alone.
 * Weights and sums of them are off by up to 2^-39 of themselves, in 64 bits and in an order that depends on nothing but the inputs: where a border between classes lies nearer than that to where top_p or the
 * random number falls, a class on its other side may be taken (several, where classes weigh less than that).
 *   ids[i]: the class; logprobs[i] = log of its share of the kept weight; kept[i]: classes kept.  Each may be NULL, not all.
 * A row without an allowed class: -1, -infinity, 0.  A row with a NaN or +infinity among its allowed classes or a setting that is NaN, or with a negative temperature: -1, NaN, -1.
 * scratch: none is needed (mt_sample_scratch_get says 0, NULL will do); what is given stays as it is.
 * Errors: as mt_score, but for the scratch; MT_EUNSUPPORTED for more than MT_SAMPLE_MAX_CLASSES classes too. */
typedef struct {
    const void* logits;             /* [rows][row_stride], dtype                */
    const int32_t* n_classes;       /* [rows], or NULL; taken into 0 .. classes */
    const uint32_t* allowed;        /* [rows][allowed_stride], or NULL          */
    const float* uniform;           /* [rows]                                   */
    const float* temperature;       /* [rows], or NULL: 1                       */
    const int32_t* top_k;           /* [rows], or NULL: all                     */
    const float* top_p;             /* [rows], or NULL: 1                       */
    const float* min_p;             /* [rows], or NULL: 0                       */
    int32_t* ids;                   /* [rows], or NULL                          */
    float* logprobs;                /* [rows], or NULL                          */
    int32_t* kept;                  /* [rows], or NULL                          */
    void* scratch;
    uint64_t scratch_bytes;
    uint64_t row_stride, allowed_stride;
    uint32_t rows, classes, dtype;
    uint32_t reserved;
} mt_sample_args;
mt_status mt_sample(mt_ctx* ctx, void* hip_stream, const mt_sample_args* args);
mt_status mt_sample_scratch_get(uint32_t rows, uint32_t classes, uint64_t* bytes);

/* Text of the last error on this context ("" if none); valid until the next call. */
const char* mt_last_error(const mt_ctx* ctx);

/* Library version string, e.g. "mt 0.1 gfx950". */
const char* mt_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MT_H */
