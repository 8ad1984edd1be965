/*
 * petra.h -- C ABI of the MI355X (gfx950) PETRA reversible-stage library.
 *
 * PETRA trains a network split into stages; each stage keeps one copy of its
 * parameters and, per time step, runs the forward of one micro-batch and the
 * backward of another with the same current parameters, then updates them in
 * place (paper: Sec. 3.3, Eq. 5 and Alg. 1).  For a reversible stage the
 * backward first rebuilds the stage input from its output (Sec. 3.2, Eq. 4),
 * so no activation is kept between the two passes.
 *
 * Conventions shared by every call below
 *  - All tensors are device pointers into memory the caller owns.  The library
 *    owns only the host-side handle and the HIP streams/events it creates for
 *    itself; no call allocates or frees device memory.
 *  - Activations are NHWC.  A stage activation with C channels is passed as two
 *    contiguous half-tensors x1 (channels [0, C/2)) and x2 (channels [C/2, C)),
 *    each [N][H][W][C/2], of the stage's storage type (fp32 or bf16).
 *  - Parameters live in flat fp32 buffers whose layout the library defines and
 *    reports through petra_stage_param_info(): conv weights are KRSC
 *    ([C_out][R][S][C_in]).  Gradient accumulator and momentum buffers use the
 *    same layout.  BN running statistics are two fp32 arrays (mean, variance)
 *    of petra_stage_query()'s n_bn_channels entries.
 *  - `stream` is a hipStream_t (NULL = the null stream).  Compute calls only
 *    enqueue work and return; buffers must stay alive until the stream has
 *    drained them.
 *  - Argument, shape, alignment and state errors are detected on the host
 *    before anything is enqueued and return a non-zero status; nothing is
 *    launched in that case.  An asynchronous HIP error is reported as
 *    PETRA_ERR_HIP by the call that observes it.  petra_last_error() gives
 *    a readable message for the calling thread.  The library never aborts.
 *  - Device pointers must be 16-byte aligned.  A handle must not be used by
 *    two host threads at once.
 */
#ifndef PETRA_H
#define PETRA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PETRA_OK = 0,
  PETRA_ERR_INVALID_ARG = 1, /* null pointer, bad enum, bad hyper-parameter   */
  PETRA_ERR_SHAPE = 2,       /* unsupported or inconsistent sizes             */
  PETRA_ERR_DTYPE = 3,       /* unsupported storage type                      */
  PETRA_ERR_ALIGN = 4,       /* a device pointer is not 16-byte aligned       */
  PETRA_ERR_WORKSPACE = 5,   /* workspace missing or too small                */
  PETRA_ERR_STATE = 6,       /* call out of order (e.g. compute before bind)  */
  PETRA_ERR_HIP = 7,         /* a HIP runtime call failed                     */
  PETRA_ERR_ALIAS = 8        /* two buffers overlap where that is not allowed */
} petra_status;

typedef enum { PETRA_FP32 = 0, PETRA_BF16 = 1 } petra_dtype; /* storage; accumulation is fp32 */

typedef enum {
  PETRA_BLOCK_BASIC = 0,      /* conv3x3-BN-ReLU-conv3x3-BN                        */
  PETRA_BLOCK_BOTTLENECK = 1  /* conv1x1-BN-ReLU-conv3x3-BN-ReLU-conv1x1-BN         */
} petra_block_kind;

typedef enum {
  PETRA_ROLE_CONV_WEIGHT = 0,
  PETRA_ROLE_BN_GAMMA = 1,
  PETRA_ROLE_BN_BETA = 2,
  PETRA_ROLE_FC_WEIGHT = 3,
  PETRA_ROLE_FC_BIAS = 4
} petra_param_role;

/* One reversible stage: num_blocks reversible blocks y1 = x1 + F(x2),
 * y2 = x2 + G(y1) (Sec. 3.2, Fig. 2) at a fixed activation shape.
 * Each block has two residual functions F and G of the given kind, acting on
 * one stream of c_half channels (c_mid = inner width of a bottleneck).
 * BN runs in training mode with batch statistics over N*H*W (eps bn_eps);
 * running statistics use momentum bn_momentum and move only during the
 * backward recompute (Sec. 4.1, "Model adaptations").
 * Limits: c_half and c_mid are 8 times a power of two, at most 512;
 * N*H*W*max(c_half, c_mid)*element size < 2^31 bytes (every tensor is
 * addressed with 32-bit byte offsets); PETRA_ERR_SHAPE otherwise. */
typedef struct {
  int32_t n, h, w;
  int32_t c_half;
  int32_t c_mid;
  int32_t num_blocks;
  int32_t kind;   /* petra_block_kind */
  int32_t dtype;  /* petra_dtype      */
  float bn_eps;
  float bn_momentum;
} petra_stage_desc;

/* SGD with momentum (Nesterov when nesterov != 0) and gradient accumulation
 * over accum_k backward steps with averaging (Sec. 4.1; Alg. 1).  Weight decay
 * applies to conv/FC weights only, never to BN parameters or biases. */
typedef struct {
  float lr;
  float momentum;
  float weight_decay;
  int32_t nesterov;
  int32_t accum_k;
} petra_sgd;

/* Placement of one parameter tensor in the flat fp32 buffers.  Tensors are
 * indexed in canonical order: block b, function F then G, conv l, and for
 * each conv its weight, BN gamma, BN beta. */
typedef struct {
  int64_t offset;        /* element offset into the flat buffers           */
  int64_t numel;
  int32_t role;          /* petra_param_role                                */
  int32_t ndim;
  int32_t shape[4];      /* KRSC for conv weights, [C] for BN parameters    */
  int32_t weight_decay;  /* 1 if weight decay applies                       */
  int32_t bn_index;      /* BN layer index for gamma/beta (and the conv it follows), else -1 */
} petra_param_info;

typedef struct petra_stage petra_stage;

/* Status name, e.g. "PETRA_ERR_SHAPE". */
const char* petra_status_str(petra_status s);
/* Message of the calling thread's last failed call ("" if none). */
const char* petra_last_error(void);

/* Build a handle from a description (host only, no device work). */
petra_status petra_stage_create(const petra_stage_desc* desc, petra_stage** out);
petra_status petra_stage_destroy(petra_stage* st);

/* Sizes the caller must allocate: n_params fp32 elements for each of the
 * parameter, gradient-accumulator and momentum buffers; n_tensors parameter
 * tensors; n_bn_channels fp32 elements for each running-statistics array;
 * workspace_bytes of device scratch (compute copies of the weights, one residual
 * function's intermediates for the forward and two functions' for the backward,
 * partial sums).  Beside the copies it does not grow with num_blocks, but for two
 * kinds of stages, which keep every function's intermediates and four half-width
 * tensors per inner block through a backward: those that this costs at most 32 MiB,
 * and bf16 stages all of whose convs have a kernel for their size (3x3 of 32
 * channels 32 or 56 wide, of multiples of 64 channels 8 or 16 wide; 1x1 of 128 to 32
 * channels and back). */
petra_status petra_stage_query(const petra_stage* st, int64_t* n_params, int32_t* n_tensors,
                               int64_t* n_bn_channels, size_t* workspace_bytes);
petra_status petra_stage_param_info(const petra_stage* st, int32_t index, petra_param_info* out);

/* Attach caller-owned device buffers.  params: fp32 master weights theta;
 * grad_accum: the accumulator Delta; momentum: optimizer state; run_mean /
 * run_var: BN running statistics; workspace: scratch of at least
 * workspace_bytes.  The caller initialises params, zeroes grad_accum and
 * momentum, and sets run_mean = 0, run_var = 1; then calls
 * petra_stage_sync_weights().  workspace = NULL with workspace_bytes = 0 binds
 * a handle for petra_stage_forward_noalloc only. */
petra_status petra_stage_bind(petra_stage* st, float* params, float* grad_accum, float* momentum,
                              float* run_mean, float* run_var, void* workspace,
                              size_t workspace_bytes);

/* Optimizer settings used by petra_stage_update() and the (1/k) gradient
 * scale of petra_stage_reconstruct_backward(). */
petra_status petra_stage_set_optimizer(petra_stage* st, const petra_sgd* opt);

/* Graph replay (default off): each distinct call (kind of call and the device
 * pointers passed) is captured once into a HIP graph and replayed on a private
 * stream ordered with events after prior work on the caller's stream and
 * before later work on it; set_optimizer() drops the cached graphs.
 * enable = 0 launches every kernel directly (on the caller's stream and the
 * stage's side streams). */
petra_status petra_stage_set_graphs(petra_stage* st, int32_t enable);

/* Streams used by one backward call: 1 = every kernel on one stream; 2 = the
 * weight gradients on a second stream; 3 = in addition the recompute of the
 * next residual function on a third stream, overlapped with the input-gradient
 * chain of the current one.  Default: 1 for every block kind (the weight
 * gradients wait for the end of a residual function or of the backward and run
 * grouped, which fills the chip better than per-layer launches beside the
 * chain).  Results are identical in every mode.
 * PETRA_ERR_INVALID_ARG outside [1, 3]. */
petra_status petra_stage_set_streams(petra_stage* st, int32_t n);

/* Refresh the storage-type compute copies of the conv weights from the fp32
 * master (needed once after the caller writes params directly). */
petra_status petra_stage_sync_weights(petra_stage* st, void* stream);

/* Forward of the stage with the current parameters (Eq. 5, first line):
 * blocks 1..B in order.  Reads x1, x2; writes y1, y2.  In place is allowed
 * (x1 == y1 and/or x2 == y2); no other overlap.  BN uses batch statistics and
 * leaves the running statistics untouched. */
petra_status petra_stage_forward(petra_stage* st, const void* x1, const void* x2, void* y1,
                                 void* y2, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): the forward
 * of petra_stage_forward, with the same arguments, aliasing rules and result
 * bits, that needs no workspace.  Its scratch -- the compute copies of the
 * conv weights, refreshed from params on every call, and one residual
 * function's pre-BN tensors and BN partial sums -- lives in a static device
 * array of PETRA_STATIC_SCRATCH_BYTES (and 6 MiB more for partial sums beyond it)
 * that the library holds on each device it runs on until the process ends.  The call allocates nothing and always
 * launches directly (no graph cache, no timing events).  The handle may be
 * bound with workspace = NULL and workspace_bytes = 0 (every other compute
 * call then returns PETRA_ERR_WORKSPACE).  PETRA_ERR_WORKSPACE when the stage's
 * forward needs more scratch than the array holds (about 2 bytes per conv
 * weight plus N*H*W*(sum of one residual function's conv output widths)*element
 * size).  Runs on the current device.  Every call on a device shares that
 * device's array: calls that overlap in time on one device (other streams or
 * threads) race and must be ordered by the caller. */
#define PETRA_STATIC_SCRATCH_BYTES (64u << 20)
petra_status petra_stage_forward_noalloc(petra_stage* st, const void* x1, const void* x2,
                                         void* y1, void* y2, void* stream);

/* Backward of the stage with the current parameters (Eq. 5, lines 2-4;
 * Alg. 1): blocks B..1, each rebuilding its input from its output
 * (x2 = y2 - G(y1), x1 = y1 - F(x2), Eq. 4) while recomputing the graph of G
 * and F, then taking the vector-Jacobian products through them.
 * Inputs: the stage output y1, y2 and its gradient dy1, dy2.
 * Outputs: the reconstructed input x1, x2 and the input gradient dx1, dx2.
 * Adds (1/accum_k) of the parameter gradient to grad_accum and updates the BN
 * running statistics.  In place is allowed for x1 == y1, x2 == y2,
 * dx1 == dy1, dx2 == dy2; no other overlap. */
petra_status petra_stage_reconstruct_backward(petra_stage* st, const void* y1, const void* y2,
                                              const void* dy1, const void* dy2, void* x1,
                                              void* x2, void* dx1, void* dx2, void* stream);

/* Parameter update (Eq. 5, last line; Alg. 1): when the number of backward
 * calls so far is a multiple of accum_k (and no update has run since the last
 * backward), applies the optimizer to params from grad_accum, zeroes
 * grad_accum and refreshes the compute copies.  *updated (nullable) receives
 * 1 if the update ran. */
petra_status petra_stage_update(petra_stage* st, void* stream, int32_t* updated);

/* One PETRA stage step (Eq. 5): the forward of one micro-batch (x -> y) and
 * the backward of another (yb, dyb -> xb, dxb), both reading the current
 * parameters; the update follows both.  They run concurrently, the forward on a
 * library-owned stream, or one after the other on `stream` where the step is so
 * small that the event calls would take longer.  All work is ordered after prior work on `stream`, and later
 * work on `stream` is ordered after it.  Aliasing rules of the two calls
 * apply; the forward and backward buffers must not overlap each other. */
petra_status petra_stage_step(petra_stage* st, const void* x1, const void* x2, void* y1, void* y2,
                              const void* yb1, const void* yb2, const void* dyb1,
                              const void* dyb2, void* xb1, void* xb2, void* dxb1, void* dxb2,
                              void* stream, int32_t* updated);

/* ------------------------------------------------------------------------
 * Multi-stage schedule on one GPU (Alg. 1, Eq. 5; delays of App. B).
 *
 * The network is split into num_stages stages.  Stage 0 opens with a 3x3 conv
 * (pad 1) + BN + ReLU on the images; stage j > 0 opens with a non-reversible
 * 1x1 stride-2 conv + BN on the previous stage's output (both streams taken as
 * one tensor, x1 first); each stage then runs blocks_per_stage reversible basic
 * blocks at width widths[j] (two streams of widths[j]/2 channels); the last
 * stage ends with global average pooling, a linear layer with bias and softmax
 * cross-entropy averaged over the micro-batch (Sec. 4.1, "Model adaptations").
 *
 * petra_net_tick() runs one time step of every stage: stage j (0-based) runs
 * the forward of micro-batch t - j and the backward of micro-batch
 * t - (2 num_stages - 2 - j), both with its current parameters, and then its
 * update, so the delay between a stage's forward and backward of the same
 * micro-batch is 2(num_stages - 1 - j).  Front layers keep their input in a
 * ring of micro-batches and recompute it on the backward (Sec. 3.2,
 * "Non-reversible stages"); the reversible blocks rebuild their input from
 * their output.  All stages of a tick run concurrently on library streams; the
 * tick is ordered after prior work on `stream` and later work on `stream`
 * follows it.
 *
 * Limits: h and w divisible by 2^(num_stages-1); widths[j]/2 is 8 times a
 * power of two, at most 512; c_img <= 8; classes <= 64; num_stages <= 8;
 * every stage's activation below 2^31 bytes (as for a stage).
 * ------------------------------------------------------------------------ */
#define PETRA_MAX_STAGES 8

typedef struct {
  int32_t n, h, w, c_img;              /* micro-batch of images [n][h][w][c_img] */
  int32_t num_stages;
  int32_t widths[PETRA_MAX_STAGES];    /* full width of each stage (both streams) */
  int32_t blocks_per_stage;
  int32_t classes;
  int32_t dtype;                       /* petra_dtype */
  float bn_eps;
  float bn_momentum;
  /* Buffers kept per micro-batch in flight, for the backward variants of
   * Table 4 (petra_net_set_backward) and the gradient probes: the blocks'
   * input (input buffer) and the parameters of the forward (parameter
   * buffer, a weight stash).  0 = PETRA's setting (neither). */
  int32_t input_buffer;
  int32_t param_buffer;
  /* 0: one stage per level (front layer + its blocks).  1: the paper's
   * per-layer split (Table 6, App. B): every front layer (stem, downsampling)
   * and every reversible block is a stage of its own, the last block also
   * owning the head, so num_stages x (1 + blocks_per_stage) stages; a
   * reversible stage below another one rebuilds its input from the
   * reconstruction that stage sends back.  num_stages then counts levels. */
  int32_t split_stages;
} petra_net_desc;

typedef struct petra_net petra_net;

petra_status petra_net_create(const petra_net_desc* desc, petra_net** out);
petra_status petra_net_destroy(petra_net* net);
/* Number of stages of the schedule (num_stages, or the per-layer split's count). */
petra_status petra_net_num_stages(const petra_net* net, int32_t* stages);
/* Sizes as for a stage.  Parameter tensors in canonical order: per stage j,
 * the front conv weight (KRSC, [w_j][3][3][c_img] or [w_j][1][1][w_{j-1}]), its
 * BN gamma and beta, the reversible blocks' tensors in the stage order, and
 * for the last stage the linear weight [classes][w_last] and bias [classes]. */
petra_status petra_net_query(const petra_net* net, int64_t* n_params, int32_t* n_tensors,
                             int64_t* n_bn_channels, size_t* workspace_bytes);
petra_status petra_net_param_info(const petra_net* net, int32_t index, petra_param_info* out);
/* Caller-owned buffers as for petra_stage_bind (workspace 256-byte aligned). */
petra_status petra_net_bind(petra_net* net, float* params, float* grad_accum, float* momentum,
                            float* run_mean, float* run_var, void* workspace,
                            size_t workspace_bytes);
petra_status petra_net_set_optimizer(petra_net* net, const petra_sgd* opt);
petra_status petra_net_sync_weights(petra_net* net, void* stream);
/* One tick.  images: the next micro-batch [n][h][w][c_img] in the storage type
 * and labels: its [n] int32 class ids (device pointers), or both NULL once the
 * input has ended (then only the micro-batches in flight advance; feeding
 * cannot resume).  loss (nullable, device fp32): receives the mean loss of the
 * micro-batch that reached the head in this tick; *loss_written (nullable)
 * tells whether one did. */
petra_status petra_net_tick(petra_net* net, const void* images, const int32_t* labels,
                            float* loss, void* stream, int32_t* loss_written);
/* Drain the pipeline (Alg. 1 once the input has ended): runs ticks without
 * input until no micro-batch is in flight, so every micro-batch fed so far
 * has had its backward in every stage and its updates applied.  Feeding cannot
 * resume afterwards.  losses (nullable, device fp32, at least petra_net_num_stages()
 * entries, 16-byte aligned): entry i receives the mean loss of the i-th
 * micro-batch that reaches the head during the drain; *n_losses (nullable)
 * their count; *ticks_run (nullable) the ticks this call ran (0 if nothing
 * was in flight).  Ordered after prior work on `stream`; later work on
 * `stream` follows every tick. */
petra_status petra_net_drain(petra_net* net, float* losses, void* stream, int32_t* n_losses,
                             int32_t* ticks_run);
/* Ticks run so far, micro-batches fed, and micro-batches still in flight. */
petra_status petra_net_state(const petra_net* net, int64_t* ticks, int64_t* fed,
                             int64_t* in_flight);
/* Backward variants of the ticks (Table 4; App. B): which of the kept buffers
 * the backward of a non-last stage uses.  RECONSTRUCT is PETRA: the blocks'
 * input is rebuilt from their output with the current parameters and the VJP
 * taken there.  INPUT_BUFFER takes the VJP at the stored block input with the
 * current parameters; PARAM_BUFFER at the input reconstructed with the current
 * parameters, with the parameters the forward used (blocks and front layer);
 * DELAYED uses both buffers, the standard delayed gradient.  The last stage
 * has no delay, so every variant is the PETRA backward there. */
typedef enum {
  PETRA_BWD_RECONSTRUCT = 0,
  PETRA_BWD_INPUT_BUFFER = 1,
  PETRA_BWD_PARAM_BUFFER = 2,
  PETRA_BWD_DELAYED = 3
} petra_bwd_mode;
/* Sets the variant of the following ticks (default: the buffers kept).
 * PETRA_ERR_STATE if it needs a buffer the description did not ask for. */
petra_status petra_net_set_backward(petra_net* net, int32_t mode);
/* Stage `stage`'s parameters are elements [*offset, *offset + *numel) of the
 * flat buffers (front layer, blocks, and the head for the last stage). */
petra_status petra_net_stage_params(const petra_net* net, int32_t stage, int64_t* offset,
                                    int64_t* numel);
/* Device memory of stage `stage` by purpose, in bytes (Tables 3 and 6).  The
 * first field counts the caller-owned fp32 buffers (parameters, accumulator,
 * momentum, running statistics); the rest are the stage's parts of the
 * workspace, which sum with the other stages' to petra_net_query()'s
 * workspace_bytes. */
typedef struct {
  int64_t params;             /* fp32 parameters, accumulator, momentum, running stats */
  int64_t weight_copies;      /* compute copies of the conv weights (forward, transposed) */
  int64_t activation_buffer;  /* the front layer's input, one per micro-batch in flight */
  int64_t input_buffer;       /* the blocks' input per micro-batch in flight (if kept) */
  int64_t param_buffer;       /* stashed parameters per micro-batch in flight (if kept) */
  int64_t scratch;            /* one micro-batch's working set, messages, the rest */
  int64_t total;
} petra_net_mem;
petra_status petra_net_memory(const petra_net* net, int32_t stage, petra_net_mem* out);
/* Gradient probes for the gradient-quality diagnostics (App. B); neither
 * changes parameters, accumulators, running statistics, counters or the
 * micro-batches in flight.  grad_out: device fp32 [n_params], 16-byte aligned,
 * zeroed and then filled with unscaled gradients (no 1/accum_k); ordered on
 * `stream` after prior work.
 * petra_net_probe_tick: the gradients the backward passes of the next tick
 * would compute in variant `mode` (stages without a backward then stay zero).
 * petra_net_probe_backprop: the end-to-end gradient of one micro-batch
 * (images, labels as for petra_net_tick) at the current parameters. */
petra_status petra_net_probe_tick(petra_net* net, int32_t mode, float* grad_out, void* stream);
petra_status petra_net_probe_backprop(petra_net* net, const void* images, const int32_t* labels,
                                      float* grad_out, void* stream);
/* Reversible backpropagation baseline (Sec. 4.2 and Table 5, the comparison
 * of iteration times): one micro-batch through the same network and kernels
 * with exact gradients and no overlap.  The forward of every stage in order
 * (front layers keep their output, reversible blocks keep nothing), the loss
 * head, then the backward of every stage from the last to the first, the
 * blocks rebuilding their inputs from their outputs; each stage applies its
 * update (petra_net_set_optimizer; accum_k counts these steps) right after its
 * backward, which the stages below do not read.  All work is ordered on
 * `stream`.  images [n][h][w][c_img] (storage type) and labels [n] int32 are
 * device pointers (16-byte aligned); loss (nullable, device fp32) receives the
 * micro-batch's mean loss.  Does not advance the tick counters.
 * PETRA_ERR_STATE while micro-batches of petra_net_tick are in flight (the
 * step would update parameters they have yet to use in their backward). */
petra_status petra_net_backprop_step(petra_net* net, const void* images, const int32_t* labels,
                                     float* loss, void* stream);

/* ------------------------------------------------------------------------
 * Operators of stages over tokens: attention, the coupling of a residual
 * function to its stream with norms, gate and residual scale, dropout, the norms
 * and rotation of heads, the loss over a vocabulary and the AdamW step.
 *
 * They are stateless: a description, device pointers and a stream a call, no
 * handle.  The conventions above hold (the caller owns all memory, workspaces
 * included; work is ordered on `stream` only; errors are found on the host
 * before anything is enqueued; nothing is allocated, so calls may be captured
 * in a HIP graph).  A workspace holds nothing between calls; calls that
 * overlap in time need one each.  Results do not depend on timing: no sum is
 * taken by atomic additions.
 *
 * Dropout.  `rng` points to two 64-bit device numbers {seed, offset}, read by
 * the kernels.  An element is kept if its 16 bits of Philox-4x32 (7 rounds, key
 * seed, counter (group, offset)) are at least round(65536 p), and then divided
 * by the share kept, 1 - round(65536 p) / 65536.  No mask is stored: a backward
 * (or a recomputed forward) with the same {seed, offset} has the same mask, so a
 * micro-batch in flight keeps 16 bytes; a new call takes a new offset.  Group i
 * of a tensor is its elements 8 i .. 8 i + 7.  rng may be NULL where the
 * dropout probability is 0.
 * ------------------------------------------------------------------------ */

/* Attention.  For query i of head h in batch row b, over the visible keys j of
 * key head h / (heads / kv_heads):
 *   lse_i = log sum_j exp(scale q_i.k_j),  p_ij = exp(scale q_i.k_j - lse_i),
 *   o_i = sum_j m_ij p_ij v_j
 * Visible are the keys j < kv_lens[b], and with `causal` j <= i + kv_lens[b] -
 * q_lens[b] (the last query sees every key).  A query without visible keys, or
 * at or past q_lens[b], has o = 0, lse = -inf and takes no part in any gradient,
 * whatever it and its d_o hold; so has one whose scores are all -inf.  Nothing at
 * or past the lengths is used, whatever it holds; keys that the causal mask alone
 * hides from a query that sees others enter its sums times zero and have to be
 * finite.  A NaN query, or one that sees a NaN key, has o = lse = NaN.  m is
 * dropout's 0 or 1 / (share kept); its groups are, for each row (b, h, i), the keys
 * 16 a + 4 c + {0, 1, 2, 3, 8, 9, 10, 11} for c = 0, 1, in the order (b, h, i, a, c).
 *
 * Scores, statistics and sums are fp32.  With bf16 tensors p and the backward's
 * gradients of the scores are rounded to bf16 as operands of the products that
 * follow, and the backward takes o as stored: results are off by about 1.3 times
 * (gradients 1.4 times) what rounding them alone to bf16 would give.
 *
 * Layout: tensors [batch][q_len or kv_len][heads or kv_heads][head_dim] with the
 * given strides, in elements, of the first three dimensions (all three zero:
 * contiguous); channels are contiguous.  o and d_o have o_stride; a gradient has
 * its tensor's strides.  lse is fp32 [batch][heads][q_len].
 * A written tensor shares no element with another tensor of the call.  Interleaved ones are
 * fine (slices of one tensor, such as the q, k and v of one product); two that are woven into
 * each other with different strides, so that 2^16 pairs of their rows do not tell them apart,
 * are refused.
 * Limits: heads a multiple of kv_heads; head_dim a multiple of 8, at most 128;
 * strides not negative and multiples of 16 bytes, those of written tensors such
 * that no elements share memory, a token stride of k and v of head_dim or more and
 * below 2^22 elements, in the backward 64 token strides and heads / kv_heads head
 * strides of q and of o together below 2^31 bytes, no tensor from end to end 2^47 bytes
 * or more; q_len * heads / kv_heads and kv_len at most 2^30, batch * kv_heads at most
 * 65535; scale > 0. */
typedef struct {
  int32_t batch, q_len, kv_len;
  int32_t heads, kv_heads, head_dim;
  int32_t dtype;    /* petra_dtype */
  int32_t causal;
  float scale;
  float dropout;    /* probability of dropping, 0 <= p < 1 - 2^-17 */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];   /* batch, token, head */
} petra_attn_desc;

/* Workspace of the two calls, in bytes (may be 0). */
petra_status petra_attn_query(const petra_attn_desc* desc, size_t* forward_bytes,
                              size_t* backward_bytes);
/* q_lens, kv_lens: device int32 [batch] (nullable: full lengths; values are
 * taken as if clamped to 0 .. q_len, kv_len).  Writes o and lse. */
petra_status petra_attn_forward(const petra_attn_desc* desc, const void* q, const void* k,
                                const void* v, const int32_t* q_lens, const int32_t* kv_lens,
                                const uint64_t* rng, void* o, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream);
/* o, lse: the forward's, of the same inputs and rng.  Writes dq, dk, dv whole
 * (zeros where nothing is visible); gradients of a shared key head are summed
 * over its query heads. */
petra_status petra_attn_backward(const petra_attn_desc* desc, const void* q, const void* k,
                                 const void* v, const void* o, const float* lse, const void* d_o,
                                 const int32_t* q_lens, const int32_t* kv_lens,
                                 const uint64_t* rng, void* dq, void* dk, void* dv,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* Coupling of a residual function's output f to a stream x, row by row (a row is
 * a token's width channels, contiguous), with the norm before the next function:
 *   y = residual_scale x + gate m n(f; post),   u = n(y as stored; pre)
 * n is a root-mean-square norm (z / sqrt(mean z^2 + eps) gamma) or a layer norm
 * ((z - mean) / sqrt(var + eps) gamma + beta); m is dropout's.  Parameters are fp32
 * [width]; beta is nullable in either norm.  gate is fp32 [rows / rows_per_gate][width]: row r takes
 * gate r / rows_per_gate (0: one gate for all rows).
 * Limits: width a multiple of 8, at most 8192; rows a multiple of
 * rows_per_gate. */
typedef enum { PETRA_NORM_RMS = 0, PETRA_NORM_LAYER = 1 } petra_norm;

typedef struct {
  int64_t rows;
  int64_t rows_per_gate;
  int32_t width;
  int32_t dtype;           /* petra_dtype */
  int32_t norm;            /* petra_norm */
  float eps;               /* > 0 */
  float residual_scale;    /* not 0 */
  float dropout;           /* as in petra_attn_desc */
} petra_coupling_desc;

/* Parameters of one norm, or where their gradients go. */
typedef struct {
  float* gamma;
  float* beta;   /* nullable */
} petra_norm_params;

petra_status petra_coupling_query(const petra_coupling_desc* desc, size_t* backward_bytes);
/* f = NULL (with gate, post and y NULL): only u = n(x; pre), the norm before a
 * stage's first function.  u = NULL (with pre NULL): only y.  y == x is allowed,
 * and u == f; no other overlap. */
petra_status petra_coupling_forward(const petra_coupling_desc* desc, const void* x, const void* f,
                                    const float* gate, const petra_norm_params* post,
                                    const petra_norm_params* pre, const uint64_t* rng, void* y,
                                    void* u, void* stream);
/* From y, f, the gradient dy of y and (nullable, with pre and dpre) du of u:
 *   t = dy + (dn(y; pre)/dy)^T du,  dx = residual_scale t,
 *   df = (dn(f; post)/df)^T (gate m t),  and the gradients of gate, post and pre,
 * and rebuilds x = (y - gate m n(f; post)) / residual_scale (x nullable).  Gradients of
 * parameters are written, not added; d*.beta is written where beta is given.
 * f = NULL (with gate, post, x, df, dgate and dpost NULL): only dx and dpre, the
 * norm before a stage's first function.
 * x == y, dx == dy, df == f and dx == du are allowed; no other overlap. */
petra_status petra_coupling_backward(const petra_coupling_desc* desc, const void* y,
                                     const void* f, const void* dy, const void* du,
                                     const float* gate, const petra_norm_params* post,
                                     const petra_norm_params* pre, const uint64_t* rng, void* x,
                                     void* dx, void* df, float* dgate,
                                     const petra_norm_params* dpost,
                                     const petra_norm_params* dpre, void* workspace,
                                     size_t workspace_bytes, void* stream);

/* y = residual + alpha m x over n elements (residual nullable: 0).  alpha = -1
 * takes the same dropout off again: the inverse of a coupling y = x + m f.  With
 * x a gradient it is the backward.  y == x and y == residual are allowed, no other
 * overlap with them. */
petra_status petra_dropout(int64_t n, int32_t dtype, float p, float alpha, const void* x,
                           const void* residual, const uint64_t* rng, void* y, void* stream);

/* Norms of query and key heads with the rotation by their tokens' positions, between the
 * product that forms them and the attention.  For each head's channels x of a token:
 *   z = n(x; norm),  (y_a, y_b) = (z_a cos t - z_b sin t, z_a sin t + z_b cos t)
 * for its pairs (a, b) of channels, t = freq[i] position[axis[i]] for pair i < pairs; channels in
 * no pair are not rotated.  n is over the head's channels, as in petra_coupling_desc, with one
 * gamma (and beta, nullable) [head_dim] for all query heads and one for all key heads; without
 * (NULL) n(x) = x.  With several axes (time, height and width of images, say) a pair
 * turns by the position on its own.  Angles are within 2^-31 of a turn for every position and finite
 * frequency.
 *
 * Layout: q [batch][len][heads][head_dim], k [batch][len][kv_heads][head_dim] with the given
 * strides as in petra_attn_desc, the results likewise (all three zero: contiguous).  kv_heads = 0:
 * queries only.  positions: device int32 [axes][batch][len], any values (NULL: a token's index in
 * its sequence, on every axis).  Limits: head_dim a multiple of 8, at most 128; pairs a multiple of 4,
 * at most head_dim / 2; batch * len below 2^31; strides not negative and multiples of 16 bytes, those
 * of written tensors such that no elements share memory. */
enum { PETRA_HEAD_AXES = 4, PETRA_HEAD_PAIRS = 64 };

typedef enum {
  PETRA_PAIRS_HALVES = 0,      /* channels (i, i + pairs)   */
  PETRA_PAIRS_NEIGHBOURS = 1   /* channels (2 i, 2 i + 1)   */
} petra_pairs;

typedef struct {
  int32_t batch, len;
  int32_t heads, kv_heads, head_dim;
  int32_t dtype;                     /* petra_dtype */
  int32_t norm;                      /* petra_norm */
  float eps;                         /* > 0 */
  int32_t layout;                    /* petra_pairs */
  int32_t pairs, axes;               /* 1 <= axes <= PETRA_HEAD_AXES */
  int32_t axis[PETRA_HEAD_PAIRS];    /* of each pair, below axes */
  double freq[PETRA_HEAD_PAIRS];     /* of each pair, radians a position */
  int64_t q_stride[3], k_stride[3], yq_stride[3], yk_stride[3];   /* batch, token, head */
} petra_heads_desc;

/* Workspace of the backward, in bytes. */
petra_status petra_heads_query(const petra_heads_desc* desc, size_t* backward_bytes);
/* Writes yq and yk.  yq == q and yk == k with the same strides are allowed; no other overlap. */
petra_status petra_heads_forward(const petra_heads_desc* desc, const void* q, const void* k,
                                 const petra_norm_params* q_norm, const petra_norm_params* k_norm,
                                 const int32_t* positions, void* yq, void* yk, void* stream);
/* From the forward's inputs and the gradients dyq, dyk (laid out like yq, yk): dq, dk (laid out
 * like q, k) and the gradients of the norms' parameters, written, not added.  Without a norm the
 * tensor itself (q, k) is not read.  dq == q, and dq == dyq with the same strides, are allowed
 * (and for k); no other overlap. */
petra_status petra_heads_backward(const petra_heads_desc* desc, const void* q, const void* k,
                                  const petra_norm_params* q_norm,
                                  const petra_norm_params* k_norm, const int32_t* positions,
                                  const void* dyq, const void* dyk, void* dq, void* dk,
                                  const petra_norm_params* dq_norm,
                                  const petra_norm_params* dk_norm, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* The loss of a last stage over a large vocabulary: softmax cross entropy of x W^T and its
 * gradients, without a rows x vocab tensor.  For the rows x_i [width] and their targets t_i:
 *   s_ij = scale x_i . w_j,  lse_i = log sum_j exp s_ij,  loss_i = lse_i - s_it
 *   L = sum_i weight_i loss_i,  dx = dL/dx,  dw = dL/dw (written, not added)
 * A row whose target is not in 0 .. vocab - 1 takes no part, whatever it holds: its loss, lse and
 * dx are 0.  weight: device fp32 [rows]; NULL: the mean, 1 / (the rows that take part).
 *
 * Rows are worked on in pieces (piece_rows at a time; 0: as many as keep a piece's scores within 1 GiB), whose
 * gradients of w are summed in fp32.  Scores, statistics and sums are fp32, and a loss is log(1 + R) of the others'
 * sum R, so that rows whose target has nearly all of the softmax keep theirs.  With bf16 tensors each term of dx is rounded to
 * bf16 once before the sums (2^-8 of it at most) and each of dw twice; once more in rows with a loss of 59 or more.  The
 * targets' terms are not (in dw: unless a piece has more than 16 rows a column, or 65536 rows).  Measured against what
 * rounding the results to bf16 alone gives: dx and the rows of dw whose columns are targets are off by 1.0 to 1.1 times that (over
 * a vocabulary of 2, where the other terms are as large, by 1.2 and 1.5), the other rows of dw, which have only rounded terms,
 * by 1.6 times in the median and 3 at most.
 * x, dx [rows][width] and w, dw [vocab][width] are contiguous, targets int32 [rows].
 * Limits: width a multiple of 8, at most 65536; 1 <= vocab <= 2^20; rows at most 2^30; 0 < scale < 2^127. */
typedef struct {
  int64_t rows;
  int64_t piece_rows;
  int32_t width, vocab;
  int32_t dtype;          /* petra_dtype */
  float scale;
} petra_vocab_desc;

/* Workspace of the two calls, in bytes. */
petra_status petra_vocab_query(const petra_vocab_desc* desc, size_t* loss_bytes,
                               size_t* gradient_bytes);
/* Writes loss and lse (fp32 [rows]) only. */
petra_status petra_vocab_loss(const petra_vocab_desc* desc, const void* x, const void* w,
                              const int32_t* targets, float* loss, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream);
/* Writes loss, lse, dx and dw: forward and backward in one, three products of the scores' size. */
petra_status petra_vocab_gradient(const petra_vocab_desc* desc, const void* x, const void* w,
                                  const int32_t* targets, const float* weight, float* loss,
                                  float* lse, void* dx, void* dw, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* AdamW over many tensors at once, the update of stages over tokens:
 *   g = grad_scale grad,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   theta -= lr (m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay theta)
 * for t = steps + 1, all in fp32 (the corrections in fp64).  Gradients are fp32 or bf16; a bf16
 * copy of theta for the forward is written along where one is given.
 *
 * States are fp32, or with PETRA_E4M3 8 bits: blocks of 64 elements of m, and of r = sqrt(v), as
 * e4m3 numbers (4 exponent and 3 mantissa bits) times the block's scale, the power of two that
 * brings its largest magnitude into [128, 256).  A value is rounded up or down at random to its
 * neighbours in the format, such that m and v are kept on average (v's changes by a step are far
 * smaller than the format's); r of v > 0 stays above 0.  An element's 2 x 16 random bits are Philox's, as
 * for dropout: groups are of 4 elements, element e takes bits 32 e .. 32 e + 15 for m and the 16 above for r;
 * a tensor's groups follow those of the tensor before it, its length rounded up to 64.  A step with the same rng
 * rounds alike; a new step takes a new offset.  An infinite or NaN gradient
 * leaves NaN in its own element.
 *
 * The tensors are laid out once: petra_adamw_layout writes a table, which the caller copies to
 * device memory (16-byte aligned) and keeps, with the tensors, as long as it steps.
 * Limits: n >= 0, count at most 2^20, all chunks of 4096 elements fewer than 2^24. */
enum { PETRA_E4M3 = 2 };   /* state_dtype only */

typedef struct {
  float* theta;
  void* grad;
  void *m, *v;                /* fp32 [n], or bytes [n rounded up to 64] */
  float *m_scale, *v_scale;   /* 8 bits only: [n / 64 rounded up], 4-byte aligned */
  void* copy;                 /* bf16 [n], nullable */
  int64_t n;
  float weight_decay;
} petra_adamw_tensor;

typedef struct {
  double beta1, beta2;        /* in [0, 1) */
  float eps;                  /* at least 2^-126 */
  int32_t grad_dtype;         /* PETRA_FP32 or PETRA_BF16 */
  int32_t state_dtype;        /* PETRA_FP32 or PETRA_E4M3 */
  int32_t zero_grads;         /* gradients are set to 0 as they are read */
} petra_adamw_desc;

/* Bytes of the table of these tensors, its chunks (both for petra_adamw_step) and the step's workspace. */
petra_status petra_adamw_query(const petra_adamw_desc* desc, const petra_adamw_tensor* tensors,
                               int64_t count, size_t* table_bytes, int64_t* chunks,
                               size_t* workspace_bytes);
/* Checks the tensors and writes their table to host memory. */
petra_status petra_adamw_layout(const petra_adamw_desc* desc, const petra_adamw_tensor* tensors,
                                int64_t count, void* table, size_t table_bytes);
/* One step of all tensors.  steps (int64: the steps done, advanced by the call), lr, grad_scale
 * (fp32, nullable: 1) and rng are device memory, so that a captured step may be replayed. */
petra_status petra_adamw_step(const petra_adamw_desc* desc, const void* table, size_t table_bytes,
                              int64_t count, int64_t chunks, int64_t* steps, const float* lr,
                              const float* grad_scale, const uint64_t* rng, void* workspace,
                              size_t workspace_bytes, void* stream);

/* Measurement support (not part of the method).  petra_stage_profile(st, 1)
 * clears the counters and starts bracketing every kernel launch of the stage
 * with HIP events on the stream the kernel is launched on; 0 stops it.
 * petra_stage_profile_read() waits for the recorded events and returns, for
 * kernel class `kernel_class` (0 .. until it returns PETRA_ERR_INVALID_ARG),
 * its name, launch count, summed device time in ms and the summed algorithmic
 * flops and bytes of those launches (compulsory traffic of each launch: every
 * operand read once, every result written once). */
petra_status petra_stage_profile(petra_stage* st, int32_t enable);
petra_status petra_stage_profile_read(petra_stage* st, int32_t kernel_class, const char** name,
                                      int64_t* launches, double* total_ms, double* flops,
                                      double* bytes);
/* The same totals per kernel (template instance) and class, index 0 .. until
 * it returns PETRA_ERR_INVALID_ARG, in order of first launch since the
 * profile was enabled: *name receives the kernel's demangled symbol as the
 * profiler tools print it (valid until the next petra_stage_profile call),
 * *kernel_class its class index for petra_stage_profile_read. */
petra_status petra_stage_profile_kernel(petra_stage* st, int32_t index, const char** name,
                                        int32_t* kernel_class, int64_t* launches,
                                        double* total_ms, double* flops, double* bytes);

#ifdef __cplusplus
}
#endif

#endif /* PETRA_H */
