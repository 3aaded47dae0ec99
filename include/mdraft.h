/*
 * mdraft — conv1d + selective-SSM (S6) + gate for a Mamba drafter, on one B200.
 *
 * C ABI.  Plain pointers and sizes only; no C++ or framework types.  Unless a
 * parameter says HOST, every pointer is a DEVICE pointer owned by the caller;
 * the library allocates nothing and keeps no caller pointer after a call
 * returns.  Its only state between calls is the fixed scratch array of
 * mdraft_conv_scan_prefill_noalloc and that array's cached per-device address
 * (see the sharing rules at its declaration); every other entry point is
 * stateless.  All work is enqueued on `stream` (a cudaStream_t passed as
 * void*; NULL = the default stream) and no entry point synchronises with the
 * host, except where stated.
 *
 * What is computed.  The paper drafts with a Mamba model (Section 3.1) and
 * expands a draft tree by batch generation in which a child needs only its
 * parent's recurrent state (Section 4.1).  The part of the Mamba block this
 * library covers is, per channel d (0..D-1) and state index n (0..N-1):
 *
 *     u_t     = SiLU( conv_b[d] + sum_{k=0..W-1} conv_w[d][k] * x[t-(W-1)+k][d] )
 *     Delta_t = softplus( dt[t][d] + dt_bias[d] )            (MDRAFT_DT_SOFTPLUS)
 *     h_t[n]  = exp(Delta_t * A[d][n]) * h_{t-1}[n] + Delta_t * B[t][n] * u_t
 *     y_t     = sum_n C[t][n] * h_t[n] + D[d] * u_t
 *     out[t][d] = y_t * SiLU(z[t][d])                        (rounded to the activation type)
 *
 * The in/x/dt/out projections of the block are outside these formulas; mdraft_tree_step_proj and mdraft_block_generation include them.
 *
 * State.  Per sequence (or tree node) and layer: the SSM state h (D x N, fp32,
 * n contiguous) and the conv window = the last W-1 RAW inputs x (W-1 rows of D,
 * activation type, oldest row first).  States live in a caller-allocated pool
 * of numbered slots (mdraft_cache); the library only reads and writes slots by
 * index.  This replaces the paper's one-cache-per-batch-size scheme (Section
 * 4.1, "Efficient cache utilization"): forking a node is "read the parent's
 * slot, write the child's slot" inside the update itself, with no copy pass.
 *
 * Layout.  Activations are token-major with channels contiguous; every matrix
 * argument comes with its row stride `ld*` in ELEMENTS so that x/z may be the
 * halves of one projection output and B/C slices of another.
 *
 * Supported shapes: d_state == 16, d_conv == 4, d_inner a multiple of 8,
 * activation type fp32 or bf16; anything else returns MDRAFT_ERR_UNSUPPORTED.
 * Alignment: activation base pointers and row strides must be multiples of 16
 * bytes; pool strides multiples of 16 bytes (else MDRAFT_ERR_MISALIGNED).
 *
 * Errors.  Every entry point returns an mdraft_status (0 = ok, negative =
 * error) and never aborts or throws.  Problems visible on the host (NULL
 * pointers, unsupported shapes, misalignment, workspace too small) are reported
 * before anything is launched.  Problems only visible on the device (a slot
 * index outside [0, n_slots), a cu_seqlens entry outside [0, total_tokens])
 * turn the affected node / sequence into a no-op and OR a bit of
 * mdraft_dev_status into *dev_status (if non-NULL); nothing is read or written
 * out of bounds.
 */
#ifndef MDRAFT_H
#define MDRAFT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MDRAFT_OK              =  0,
    MDRAFT_ERR_INVALID_ARG = -1,  /* NULL where data is required, negative size, bad index   */
    MDRAFT_ERR_UNSUPPORTED = -2,  /* shape or dtype outside the supported set                */
    MDRAFT_ERR_MISALIGNED  = -3,  /* pointer or stride not a multiple of 16 bytes            */
    MDRAFT_ERR_WORKSPACE   = -4,  /* workspace NULL, or smaller than the call can do with    */
    MDRAFT_ERR_CUDA        = -5   /* a CUDA runtime call or launch failed                    */
} mdraft_status;

typedef enum { MDRAFT_F32 = 0, MDRAFT_BF16 = 1 } mdraft_dtype;

/* mdraft_layer.flags */
enum {
    MDRAFT_DT_SOFTPLUS = 1u,  /* Delta = softplus(dt + dt_bias); otherwise Delta = dt + dt_bias as given        */
    MDRAFT_PRECONV     = 2u,  /* x already is u = SiLU(conv(x)): skip the conv, leave conv windows untouched    */
    MDRAFT_CONV_ONLY   = 4u,  /* write u to `out`, advance the conv window, do not run the recurrence           */
    MDRAFT_A_POWERS    = 8u,  /* caller asserts A[d][n] == (n+1)*A[d][0] exactly in fp32 (e.g. the S4D-real
                                 initialisation -(1..N)): decays are then formed from ONE exponential per
                                 token and channel by repeated multiplication.  mdraft_classify_A checks it. */
    MDRAFT_BETA_SIGMOID = 16u /* delta layers: beta = sigmoid of what is passed; otherwise beta as given */
};

/* bits ORed into *dev_status by kernels */
enum {
    MDRAFT_DEV_BAD_SLOT    = 1,  /* a slot index outside [0, n_slots)                  */
    MDRAFT_DEV_BAD_SEQLENS = 2,  /* cu_seqlens not non-decreasing within [0, T]        */
    MDRAFT_DEV_WAIT_EXPIRED = 4  /* a bounded on-chip wait ran out (results invalid)   */
};

/* Per-layer constants.  All arrays fp32, device, read-only, caller-owned.  The context encodes may start while the kernel
 * ahead of them on the stream is finishing, and read these arrays (not their inputs, states or slots) without waiting for
 * it: constants that a kernel has just written need a synchronisation, a copy or another kernel in between. */
typedef struct {
    int32_t d_inner;        /* D */
    int32_t d_state;        /* N, must be 16 */
    int32_t d_conv;         /* W, must be 4  */
    int32_t act;            /* mdraft_dtype of x, z, dt, B, C, out and of the conv windows */
    uint32_t flags;
    uint32_t reserved;
    const float *A;         /* (D, N) row-major, every entry <= 0                           */
    const float *D;         /* (D) skip weight, or NULL for 0                               */
    const float *conv_w;    /* (D, W) row-major; tap W-1 multiplies the current token       */
    const float *conv_b;    /* (D) or NULL for 0                                            */
    const float *dt_bias;   /* (D) or NULL for 0                                            */
} mdraft_layer;

/* State pool for a whole stack of layers.  Slot s of layer l:
 *   ssm  + l*ssm_layer_stride  + s*ssm_slot_stride   -> (D, N) fp32            (strides in floats)
 *   conv + l*conv_layer_stride + s*conv_slot_stride  -> (W-1, D) activation    (strides in elements)  */
typedef struct {
    float  *ssm;
    int64_t ssm_layer_stride, ssm_slot_stride;
    void   *conv;
    int64_t conv_layer_stride, conv_slot_stride;
    int32_t n_layers, n_slots;
} mdraft_cache;

/* Optional tuning and profiling hooks for the prefill; pass NULL for the defaults. */
typedef struct {
    int32_t chunk_len;      /* tokens per scan chunk; 0 = chosen from the problem size; otherwise >= 4   */
    int32_t block_channels; /* channels per thread block: 0 = chosen from the problem size, else 128 or 512 */
    int32_t reserved[2];    /* must be 0 */
    void *event_after_chunk_state;  /* cudaEvent_t or NULL: recorded on `stream` after the chunk-summary kernel  */
    void *event_after_carry_scan;   /* cudaEvent_t or NULL: recorded after the carry scan, before the main scan  */
} mdraft_prefill_opts;

/*
 * Context encode ("prefill"): conv1d+SiLU, Delta activation, S6 scan and gate
 * over packed sequences, in parallel over channels and over chunks of tokens
 * whose (decay, input) summaries are combined by a prefix scan into each chunk's
 * incoming state (the recurrence is first-order linear, so chunks compose
 * associatively).  Paper Section 3.1
 * (drafter encode) and Fig. 1a.
 *
 *   x, z, dt : (T, D) activations, strides ldx, ldz, lddt           [read]
 *   B, C     : (T, N) activations, strides ldb, ldc                 [read]
 *   out      : (T, D) activations, stride ldo                       [written]
 *   cu_seqlens : n_seq+1 int32, tokens of sequence s are rows cu_seqlens[s] .. cu_seqlens[s+1]-1.  May be NULL
 *                when n_seq == 1: the one sequence is then rows 0 .. total_tokens-1, and no kernel has to
 *                fetch offsets from memory before it can start
 *   init_slot  : n_seq int32 or NULL; slot holding each sequence's starting state, -1 / NULL = zero state
 *   final_slot : n_seq int32 or NULL; slot that receives the state after the last token, -1 / NULL = discard.
 *                init_slot[s] == final_slot[s] is allowed (encode a context in pieces).
 *                Hazards (caller's duty): the sequences of a call run side by side, in any order.  No two may have the same
 *                final_slot.  Any number may start from a slot that none of them stores to.  A sequence may start from
 *                another's final_slot only where it is cut, which a chunk length in `opts` guarantees for sequences of more
 *                tokens than that: it then starts from what the slot held before the call
 *   max_seqlen : an upper bound on the longest sequence (HOST value, used to size the launch)
 *   workspace  : device scratch, 256-byte aligned; contents need not be initialised and are garbage afterwards.
 *                mdraft_prefill_workspace_bytes(...) says how much the call would like.  With less it cuts the sequences
 *                into fewer, longer chunks (slower, and another rounding), as long as those give every SM three or four blocks
 *                of 128 channels (one of 512 where the width fills those) or are, for several sequences, at most 256
 *                tokens; less is MDRAFT_ERR_WORKSPACE.  Sequences that the library leaves whole need none, although
 *                the query for a single layer answers as if they were cut.  A chunk length given in `opts` is kept:
 *                it needs all that the query says.  Small problems are encoded in one kernel that uses none of it, or, where several
 *                sequences with both starting and final slots would otherwise be cut, passes their final states through
 *                it; they are refused all the same where the workspace would not serve the other form
 *   dev_status : device int32 or NULL (see mdraft_dev_status bits); never cleared by the library
 */
size_t mdraft_prefill_workspace_bytes(const mdraft_layer *layer, int32_t total_tokens, int32_t n_seq,
                                      int32_t max_seqlen, const mdraft_prefill_opts *opts);

int mdraft_conv_scan_prefill(const mdraft_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                             const void *x, int64_t ldx, const void *z, int64_t ldz, const void *dt, int64_t lddt,
                             const void *B, int64_t ldb, const void *C, int64_t ldc,
                             void *out, int64_t ldo,
                             int32_t total_tokens, int32_t n_seq, int32_t max_seqlen,
                             const int32_t *cu_seqlens, const int32_t *init_slot, const int32_t *final_slot,
                             void *workspace, size_t workspace_bytes, const mdraft_prefill_opts *opts,
                             int32_t *dev_status, void *stream);

/* One layer's activations in a call over several layers; meanings and strides as in mdraft_conv_scan_prefill / mdraft_tree_step. */
typedef struct {
    const void *x, *z, *dt, *B, *C;
    void *out;
    int64_t ldx, ldz, lddt, ldb, ldc, ldo;
} mdraft_io;

/*
 * The same prefill for several layers whose inputs are all there already (HOST arrays of n_layers entries each; layer i reads
 * and writes pool layer layer_index[i]).  Paper Section 3.1: the drafter encodes a context with every layer of its stack.
 * The results are those of one mdraft_conv_scan_prefill per layer up to the rounding of another chunk plan.  Layers that share
 * their flags run in one launch (up to 32), which fills the GPU without cutting sequences into chunks; d_inner and act must
 * agree over all layers (else MDRAFT_ERR_UNSUPPORTED).
 * Hazards (caller's duty): the layers run side by side, so no layer's `out` may overlap another layer's inputs or `out`, and
 * no pool layer may appear twice.
 *   workspace : as above; mdraft_prefill_stack_workspace_bytes answers for layers that share the flags of `layer`.  The
 *               launches of a call share it, so layers with different flags need the largest answer over their groups
 * mdraft_prefill_stack_launches: kernels such a call launches (for accounting), if it is of one sequence or has no init_slot or
 * no final_slot; with both, a batch that would be cut takes two or three also where this says one.
 */
size_t mdraft_prefill_stack_workspace_bytes(const mdraft_layer *layer, int32_t n_layers, int32_t total_tokens, int32_t n_seq,
                                            int32_t max_seqlen, const mdraft_prefill_opts *opts);

int32_t mdraft_prefill_stack_launches(const mdraft_layer *layer, int32_t n_layers, int32_t total_tokens, int32_t n_seq,
                                      int32_t max_seqlen, const mdraft_prefill_opts *opts);

int mdraft_conv_scan_prefill_stack(int32_t n_layers, const mdraft_layer *layers, const mdraft_cache *cache, const int32_t *layer_index,
                                   const mdraft_io *io, int32_t total_tokens, int32_t n_seq, int32_t max_seqlen,
                                   const int32_t *cu_seqlens, const int32_t *init_slot, const int32_t *final_slot,
                                   void *workspace, size_t workspace_bytes, const mdraft_prefill_opts *opts,
                                   int32_t *dev_status, void *stream);

/*
 * The same prefill for callers that cannot allocate device memory.  No counterpart in the paper: this is a
 * deployment variant of mdraft_conv_scan_prefill.  Some hosts of this library must never call cudaMalloc or a
 * framework allocator once they are running: a serving loop whose memory pool was carved up at start-up, code
 * that runs inside someone else's stream capture, a plug-in that is handed pointers but owns no allocator.
 * They have nowhere to get the chunk workspace from, so this entry point brings its own: a fixed array of
 * MDRAFT_NOALLOC_SCRATCH_BYTES inside the library image (every GPU that loads the library holds those bytes
 * until the process exits).  Inputs, outputs and the state pool are still the caller's.
 *
 * Arguments and results are those of mdraft_conv_scan_prefill without `workspace` / `workspace_bytes`; the output
 * is the same, bit for bit, as that call given a workspace of MDRAFT_NOALLOC_SCRATCH_BYTES bytes of its own.
 *   - A problem that such a workspace does not serve (see `workspace` above: not even with the longest chunks) returns
 *     MDRAFT_ERR_WORKSPACE before anything is launched: shorten the call (encode the context in pieces through
 *     init_slot / final_slot) or use the entry point above with your own buffer.
 *   - The first call on each device looks up the array's device address (the device must be current); make that
 *     first call outside any stream capture.  Later calls do no set-up.
 *   - Nothing is allocated or freed, here or in anything this calls.
 *   - All calls on a device share the one array.  It holds whatever the previous call left; the prefill writes
 *     every scratch word before reading it, so nothing needs clearing.  Two calls that may run at the same time
 *     on one GPU (different streams, or different host threads) would overwrite each other's scratch: keep them
 *     on one stream or otherwise ordered.
 */
#define MDRAFT_NOALLOC_SCRATCH_BYTES (8u << 20)

int mdraft_conv_scan_prefill_noalloc(const mdraft_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                                     const void *x, int64_t ldx, const void *z, int64_t ldz, const void *dt, int64_t lddt,
                                     const void *B, int64_t ldb, const void *C, int64_t ldc,
                                     void *out, int64_t ldo,
                                     int32_t total_tokens, int32_t n_seq, int32_t max_seqlen,
                                     const int32_t *cu_seqlens, const int32_t *init_slot, const int32_t *final_slot,
                                     const mdraft_prefill_opts *opts, int32_t *dev_status, void *stream);

/*
 * Draft-tree step: one token for each of n_nodes nodes (of any number of
 * sequences) in one launch per tree level.  Node i reads the conv window and
 * SSM state in slot parent_slot[i], applies one step of the recurrence with its
 * own inputs (row i of x, z, dt, B, C), writes out[i] and stores the resulting
 * state to slot node_slot[i] — the fork is the gather itself; no state is
 * copied first.  Paper Section 4.1 (a child needs only a copy of its parent's
 * state; generation i is a batch of N_1*...*N_i single-token inputs).
 *
 *   parent_slot, node_slot : n_nodes int32 each (device)
 *   level_offsets : HOST array of n_levels+1 ints, or NULL with n_levels <= 1 for a single level.
 *                   Level l = nodes [level_offsets[l], level_offsets[l+1]); levels are launched in
 *                   order on `stream`, so a parent may live in an earlier level of the same call.
 * Hazards (caller's duty): within one level no node_slot may equal another node's parent_slot or
 * node_slot; parent_slot[i] == node_slot[i] (in-place chain decode) is fine.  Within one call the
 * input rows of a node (x, z, dt, B, C) must not be rows that another node of the same call writes
 * (`out` may be the same buffer as `x` as long as node i writes row i only): the levels of a call
 * overlap their set-up, and a level may fetch its input rows before the levels ahead have finished.
 * The result of a node does not depend on where in the level it sits or on how levels are split
 * across calls.
 */
int mdraft_tree_step(const mdraft_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                     const void *x, int64_t ldx, const void *z, int64_t ldz, const void *dt, int64_t lddt,
                     const void *B, int64_t ldb, const void *C, int64_t ldc,
                     void *out, int64_t ldo,
                     int32_t n_nodes, const int32_t *parent_slot, const int32_t *node_slot,
                     int32_t n_levels, const int32_t *level_offsets,
                     int32_t *dev_status, void *stream);

/*
 * The same tree step for several layers whose inputs are all there already: one launch per level takes every layer (up to 32
 * with the same flags), so a round of L layers waits for n_levels dependent launches instead of L * n_levels.  HOST arrays
 * of n_layers entries; layer i works on pool layer layer_index[i]; bit for bit the results of one mdraft_tree_step per layer.
 * Paper Section 4.1.  Hazards: those of mdraft_tree_step, and between layers those of mdraft_conv_scan_prefill_stack.
 */
int mdraft_tree_step_stack(int32_t n_layers, const mdraft_layer *layers, const mdraft_cache *cache, const int32_t *layer_index,
                           const mdraft_io *io, int32_t n_nodes, const int32_t *parent_slot, const int32_t *node_slot,
                           int32_t n_levels, const int32_t *level_offsets, int32_t *dev_status, void *stream);

/*
 * Draft-tree step with the block's own selection projections: like
 * mdraft_tree_step for ONE level, but the step size, B and C of a node are not
 * inputs; the call forms them from the node's conv output u (all d_inner
 * channels) the way the drafter's Mamba block does (paper Section 3.1: the
 * drafter is a Mamba model; Section 4.1: generation i is one batch of the
 * level's nodes, each from its parent's state):
 *
 *     s     = W_x u                       W_x : (dt_rank + 2*d_state) x d_inner, row-major
 *     dt[d] = sum_{r<dt_rank} W_dt[d][r] * s[r]     W_dt: d_inner x dt_rank, row-major
 *     B[n]  = s[dt_rank + n],   C[n] = s[dt_rank + d_state + n]
 *
 * then dt_bias / softplus, the recurrence, the skip term and the gate exactly
 * as in mdraft_tree_step.  u, s and dt are kept in fp32 from the conv to the
 * recurrence (nothing is rounded to the activation dtype in between).  One
 * launch per call; the blocks of a node exchange their shares of s through
 * cluster shared memory, so no workspace is needed.
 *
 *   proj->W_x, proj->W_dt : device, activation dtype of the layer, 16-byte aligned, dense (no padding)
 *   proj->dt_rank         : multiple of 8, 8..256
 *   proj->nodes_per_cluster: tuning only (the result of a node does not depend on it, bit for bit); 0 lets the
 *                           library choose: 1 for narrow levels, 2 or 4 for wide ones
 *   x, z, out             : device, n_nodes rows of d_inner activations (strides ldx, ldz, ldo in elements)
 *   parent_slot, node_slot: device, n_nodes int32 each; same meaning and hazards as mdraft_tree_step
 * layer->flags: MDRAFT_DT_SOFTPLUS and MDRAFT_A_POWERS are honoured; MDRAFT_PRECONV and
 * MDRAFT_CONV_ONLY make no sense here (MDRAFT_ERR_INVALID_ARG).  d_inner above 4096 is
 * MDRAFT_ERR_UNSUPPORTED (the blocks of a node must fit one cluster): use the split mode there.
 * Device-side faults are reported through dev_status as in mdraft_tree_step.
 *
 * Width of a level.  The call is built for the level widths of drafting (the paper's trees have 1 to 18 nodes per
 * level; it is about twice as fast as the split mode there).  Every node's blocks read both matrices again (out of
 * L2), so the cost per node does not fall with the width, while the split mode's matrix products amortise the weights
 * over the level: beyond MDRAFT_PROJ_STEP_MAX_NODES nodes per level the split mode (MDRAFT_CONV_ONLY step, the
 * caller's two matrix products, MDRAFT_PRECONV step) is the faster path and callers should switch to it there, as
 * the package's block stack does.  The call itself accepts any width and stays correct.
 */
#define MDRAFT_PROJ_STEP_MAX_NODES 256
typedef struct mdraft_select_proj {
    const void *W_x;
    const void *W_dt;
    int32_t dt_rank;
    int32_t nodes_per_cluster;   /* 0 = chosen from the level's width; 1, 2 or 4 = that many nodes share one set of weight loads */
} mdraft_select_proj;

int mdraft_tree_step_proj(const mdraft_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                          const mdraft_select_proj *proj,
                          const void *x, int64_t ldx, const void *z, int64_t ldz, void *out, int64_t ldo,
                          int32_t n_nodes, const int32_t *parent_slot, const int32_t *node_slot,
                          int32_t *dev_status, void *stream);

/*
 * One generation of a whole drafter stack (paper Section 4.1: generation i is one batch of the nodes of level i): embedding
 * rows of the nodes' tokens, then per layer
 *     xz = rmsnorm(h) W_in;   y = the projection step above on (x, z) = xz;   h = h + y W_out
 * and logits = rmsnorm(h) W_lm.  bf16 weights and activations, fp32 accumulation; h is rounded to bf16 after every layer; the
 * norm has no weight.  All kernels of a call are chained so that each fetches its weights while the one ahead runs.
 *   W_in[l] (d_model, 2 d_inner), W_out[l] (d_inner, d_model), W_lm (d_model, vocab), embed (vocab, d_model): row-major, dense
 *   W_x[l], W_dt[l]     : as mdraft_select_proj       (the arrays themselves are HOST arrays of n_layers device pointers)
 *   tokens              : n_nodes int64, device; an id outside the vocabulary raises MDRAFT_DEV_BAD_SLOT (its row is zero)
 *   h, xz, y            : device scratch of n_nodes x d_model, x 2 d_inner, x d_inner bf16
 *   logits              : n_nodes rows of vocab bf16, stride ldl (a multiple of 8)
 * Layer l works on pool layer l.  No node_slot may equal another node's parent_slot or node_slot.
 * Supported: n_nodes <= MDRAFT_BLOCK_MAX_NODES, d_model a multiple of 32 up to 1408, d_inner a multiple of 32 up to 2048, vocab
 * a multiple of 8, dt_rank as above; anything else is MDRAFT_ERR_UNSUPPORTED.
 */
#define MDRAFT_BLOCK_MAX_NODES 64
typedef struct {
    int32_t n_layers, d_model, dt_rank, vocab;
    const mdraft_layer *layers;   /* HOST, n_layers */
    const void *const *W_in, *const *W_x, *const *W_dt, *const *W_out;
    const void *embed, *W_lm;
    float eps;                    /* of the norms */
} mdraft_block_stack;

int mdraft_block_generation(const mdraft_block_stack *stack, const mdraft_cache *cache, const int64_t *tokens, int32_t n_nodes,
                            const int32_t *parent_slot, const int32_t *node_slot, void *h, void *xz, void *y,
                            void *logits, int64_t ldl, int32_t *dev_status, void *stream);

/*
 * ---------------------------------------------------------------------------------------------------------
 * Mamba-2 (SSD) drafter layer.  The paper names Mamba-2 as the model whose advances "directly benefit" the approach
 * (Section 1, the paragraph before Related Work) and defines nothing about it; what is computed here is the cited
 * model's recurrence, written like the one at the top of this file with ONE scalar A and ONE step size per head:
 * the D channels form H = D / P heads of P channels (d = j*P + p),
 *
 *     u_t[d]     = SiLU( conv_b[d] + sum_k conv_w[d][k] * x[t-(W-1)+k][d] )
 *     Delta_t[j] = softplus( dt[t][j] + dt_bias[j] )                         (MDRAFT_DT_SOFTPLUS)
 *     h_t[d][n]  = exp(Delta_t[j] * A[j]) * h_{t-1}[d][n] + Delta_t[j] * B[t][n] * u_t[d]
 *     y_t[d]     = sum_n C[t][n] * h_t[d][n] + D[d] * u_t[d]
 *     out[t][d]  = y_t[d] * SiLU(z[t][d])
 *
 * B and C are shared by all heads (one group) and are inputs as given (a block that also convolves them does so
 * before the call).  Supported: headdim P = 64, d_state N = 128, d_conv 4, bf16 activations, d_inner a multiple of
 * 64; anything else is MDRAFT_ERR_UNSUPPORTED.  State slots: (D, 128) fp32 + (3, D) bf16 window, in an mdraft_cache
 * whose strides are sized for N = 128.  flags: MDRAFT_DT_SOFTPLUS only.
 *
 * Precision.  The context encode runs the chunk-local sums on the tensor cores (tcgen05, bf16 operands, fp32
 * accumulation): u * Delta and the masked C.B products are rounded to bf16 on the way into a product, so `out`
 * carries a relative error of a few 2^-9 before its own rounding to bf16; the incoming state of a chunk and the
 * operand of the state product are split into a bf16 value plus a bf16 remainder (two products into one
 * accumulator), so what depends on the state, and the state written to the slot, keep fp32-level accuracy.  The
 * encode's gate uses SiLU(z) = z/2 * (1 + tanh(z/2)) with the hardware's approximate tanh (about 2^-11).
 */
typedef struct {
    int32_t d_inner;        /* D */
    int32_t headdim;        /* P, must be 64 */
    int32_t d_state;        /* N, must be 128 */
    int32_t d_conv;         /* W, must be 4 */
    int32_t act;            /* must be MDRAFT_BF16 */
    uint32_t flags;         /* MDRAFT_DT_SOFTPLUS or 0 */
    const float *A;         /* (H) one scalar per head, <= 0 */
    const float *D;         /* (D) skip weight per channel, or NULL for 0 */
    const float *conv_w;    /* (D, W) row-major; tap W-1 multiplies the current token */
    const float *conv_b;    /* (D) or NULL */
    const float *dt_bias;   /* (H) or NULL */
} mdraft_ssd_layer;

/*
 * Context encode of an SSD layer over packed sequences (paper Section 3.1 for the encode; Section 1 for Mamba-2).
 * Tokens are cut into chunks of 128 that never straddle a sequence; per (head, chunk) the sums inside the chunk are
 * matrix products on the tensor cores, chunk states are chained by a small scan in between.
 *   x, z, out : (T, D) bf16, strides ldx, ldz, ldo          dt : (T, H) bf16, stride lddt (elements; any value >= H)
 *   B, C      : (T, 128) bf16, strides ldb, ldc (multiples of 8 elements, base 16-byte aligned)
 *   cu_seqlens, init_slot, final_slot, dev_status, stream: as in mdraft_conv_scan_prefill (cu_seqlens may be NULL
 *   for one sequence), but no sequence may start from another's final_slot, however long it is
 *   workspace : device scratch of at least mdraft_ssd_prefill_workspace_bytes(...) bytes, 256-byte aligned
 */
size_t mdraft_ssd_prefill_workspace_bytes(const mdraft_ssd_layer *layer, int32_t total_tokens, int32_t n_seq);

int mdraft_ssd_prefill(const mdraft_ssd_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                       const void *x, int64_t ldx, const void *z, int64_t ldz, const void *dt, int64_t lddt,
                       const void *B, int64_t ldb, const void *C, int64_t ldc,
                       void *out, int64_t ldo,
                       int32_t total_tokens, int32_t n_seq,
                       const int32_t *cu_seqlens, const int32_t *init_slot, const int32_t *final_slot,
                       void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream);

/*
 * Draft-tree step of an SSD layer: one token for each node of a level, node i from slot parent_slot[i] into slot
 * node_slot[i] (paper Section 4.1, as mdraft_tree_step).  x, z, out: (M, D); dt: (M, H); B, C: (M, 128).  Levels,
 * hazards (early input rows included) and device-side faults as in mdraft_tree_step.  All arithmetic is
 * fp32 (no tensor cores: one token per node is a memory-bound update of a (D, 128) state).
 */
int mdraft_ssd_tree_step(const mdraft_ssd_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                         const void *x, int64_t ldx, const void *z, int64_t ldz, const void *dt, int64_t lddt,
                         const void *B, int64_t ldb, const void *C, int64_t ldc,
                         void *out, int64_t ldo,
                         int32_t n_nodes, const int32_t *parent_slot, const int32_t *node_slot,
                         int32_t n_levels, const int32_t *level_offsets,
                         int32_t *dev_status, void *stream);

/*
 * ---------------------------------------------------------------------------------------------------------
 * Gated delta rule drafter layer.  Like Mamba-2 a recurrent layer with one decay per head and a state of constant size, so it
 * drafts the way the paper's drafter does (Section 3.1 encode, Section 4.1 tree); what a token writes is the difference between
 * its value and what the state already holds for its key.  Per value head j (key head j / (n_v_heads / n_k_heads)), with the
 * state S a d_v x d_k matrix:
 *
 *     alpha_t = exp( softplus(dt[t][j] + dt_bias[j]) * A[j] )                 (MDRAFT_DT_SOFTPLUS; else exp((dt + dt_bias) A))
 *     beta_t  = sigmoid( beta[t][j] )                                         (MDRAFT_BETA_SIGMOID; else as given)
 *     r       = beta_t * ( v_t - alpha_t * S_{t-1} k_t )
 *     S_t     = alpha_t * S_{t-1} + r k_t^T
 *     o_t     = scale * S_t q_t
 *     out_t   = [ o_t / sqrt(mean(o_t^2) + eps) * norm_w ]  [ * SiLU(z_t) ]      (rounded to the activation type)
 *
 * The bracketed parts are left out where norm_w / z is NULL.  q, k and v are taken as given: a block convolves its q | k | v
 * channels with a MDRAFT_CONV_ONLY call over a layer of that many channels (the same state pool holds the windows) and brings
 * the query and key heads to unit length with mdraft_qk_norm.  Keys have to keep beta * |k|^2 at 2 or less, as unit keys do: with larger ones the
 * recurrence itself grows without bound.  A NaN or infinity among a token's q, k, v, dt or beta stays with its sequence, and there reaches, as in the
 * recurrence, the tokens behind it; a long sequence is encoded 64 tokens at a time, and then it may reach tokens of the same 64 ahead of it as well.
 *
 * Supported: d_k and d_v 64 or 128, n_v_heads a multiple of n_k_heads, fp32 or bf16 activations; anything else is
 * MDRAFT_ERR_UNSUPPORTED.  State slots: (n_v_heads * d_v, d_k) fp32 in an mdraft_cache, whose windows these calls do not touch (cache->conv may
 * be NULL).  flags: MDRAFT_DT_SOFTPLUS, MDRAFT_BETA_SIGMOID.
 */
typedef struct {
    int32_t n_k_heads, n_v_heads, d_k, d_v;
    int32_t act;            /* mdraft_dtype of q, k, v, z, dt, beta, out */
    uint32_t flags;
    float scale;            /* of the outputs, d_k^-1/2 as a rule */
    float eps;              /* of the output norm */
    const float *A;         /* (n_v_heads), <= 0 */
    const float *dt_bias;   /* (n_v_heads) or NULL for 0 */
    const float *norm_w;    /* (d_v) or NULL: no output norm */
} mdraft_gdr_layer;

/*
 * Context encode of a delta layer over packed sequences.
 *   q, k      : (T, n_k_heads * d_k), strides ldq, ldk          v, z, out : (T, n_v_heads * d_v), strides ldv, ldz, ldo; z may be NULL
 *   dt, beta  : (T, n_v_heads), strides lddt, ldbeta (elements; any value >= n_v_heads)
 *   cu_seqlens, init_slot, final_slot, dev_status, stream: as in mdraft_conv_scan_prefill (cu_seqlens may be NULL for one sequence), but
 *   no sequence may start from another's final_slot, however long it is.  init_slot[s] == final_slot[s] is allowed.  Rows that belong to no sequence
 *   are neither read into a result nor written
 *   max_seqlen: an upper bound on the longest sequence (HOST value): with its help the call chooses how it works; the results do not
 *               depend on it beyond rounding: states are as good as fp32 arithmetic makes them, outputs are off by their own rounding and, where a long bf16 sequence's
 *               products cancel, by 2^-14 of the products' sizes
 *   workspace : device scratch of at least mdraft_gdr_prefill_workspace_bytes(...) bytes, 256-byte aligned; NULL where that is 0.  Its contents
 *               need not be initialised; calls that may run at the same time (other streams, graphs replayed side by side) each need their own.
 *               `out` must not overlap an input, and no two sequences may end in one slot
 */
size_t mdraft_gdr_prefill_workspace_bytes(const mdraft_gdr_layer *layer, int32_t total_tokens, int32_t n_seq, int32_t max_seqlen);

int mdraft_gdr_prefill(const mdraft_gdr_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                       const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, const void *z, int64_t ldz,
                       const void *dt, int64_t lddt, const void *beta, int64_t ldbeta, void *out, int64_t ldo,
                       int32_t total_tokens, int32_t n_seq, int32_t max_seqlen,
                       const int32_t *cu_seqlens, const int32_t *init_slot, const int32_t *final_slot,
                       void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream);

/*
 * Draft-tree step of a delta layer: one token for each node of a level, node i from slot parent_slot[i] (-1: the zero state) into slot
 * node_slot[i] (paper Section 4.1, as mdraft_tree_step).  q, k: (M, n_k_heads * d_k); v, z, out: (M, n_v_heads * d_v); dt, beta:
 * (M, n_v_heads).  Levels, hazards (early input rows included) and device-side faults as in mdraft_tree_step.  All arithmetic is fp32.
 */
int mdraft_gdr_tree_step(const mdraft_gdr_layer *layer, const mdraft_cache *cache, int32_t layer_index,
                         const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, const void *z, int64_t ldz,
                         const void *dt, int64_t lddt, const void *beta, int64_t ldbeta, void *out, int64_t ldo,
                         int32_t n_nodes, const int32_t *parent_slot, const int32_t *node_slot,
                         int32_t n_levels, const int32_t *level_offsets, int32_t *dev_status, void *stream);

/*
 * Norm of every query and key head, with the position rotation in the same pass.  Per row and head of d_head values
 *
 *     y = x / sqrt(mean(x^2) + eps) * w      (MDRAFT_NORM_RMS)
 *     y = x / sqrt(sum(x^2) + eps) * w       (MDRAFT_NORM_L2)
 *     y = x                                  (MDRAFT_NORM_NONE)
 *
 * with w = q_w or k_w (NULL: 1), then for i < rot_dim / 2 the pair (a, b) = (y[i], y[i + rot_dim/2]) (MDRAFT_ROT_HALF) or
 * (y[2i], y[2i+1]) (MDRAFT_ROT_PAIRS) becomes
 *
 *     (a cos t - b sin t, b cos t + a sin t) * rot_scale,      t = positions[row] * freqs[i]
 *
 * and the values from rot_dim on stay as the norm left them.  Arithmetic is fp32, rounded once at the end; t is formed and
 * reduced in 64 bits, so far positions lose nothing.  Contexts stretched by other frequencies come with their own `freqs` (and rot_scale).  A
 * tree node's position is its sequence's length plus its depth.
 *   q, q_out : (rows, n_q_heads * d_head), strides ldq, ldqo      k, k_out : (rows, n_k_heads * d_head), strides ldk, ldko
 *              q_out may be q with the same stride, k_out likewise (in place); no other overlap.  One of the head counts may be 0
 *   positions: (rows) int32, may be NULL when rot_dim is 0
 * Supported: d_head a multiple of 8 up to 256; rot_dim even and at most d_head, a multiple of 16 for MDRAFT_ROT_HALF; fp32 or bf16
 * activations, n_rows up to 2^31 - 4097; anything else is MDRAFT_ERR_UNSUPPORTED.  No counterpart in the paper, which does not look inside a layer.
 */
enum { MDRAFT_NORM_NONE = 0, MDRAFT_NORM_L2 = 1, MDRAFT_NORM_RMS = 2 };
enum { MDRAFT_ROT_HALF = 0, MDRAFT_ROT_PAIRS = 1 };

typedef struct {
    int32_t d_head, n_q_heads, n_k_heads;
    int32_t act;            /* mdraft_dtype of q, k and the results */
    int32_t norm;           /* MDRAFT_NORM_* */
    int32_t rot_dim;        /* rotated values of a head, 0 = none */
    int32_t rot_layout;     /* MDRAFT_ROT_* */
    float eps, rot_scale;
    const float *q_w, *k_w; /* (d_head) or NULL */
    const float *freqs;     /* (rot_dim / 2) radians per position */
} mdraft_qk_norm_spec;

int mdraft_qk_norm(const mdraft_qk_norm_spec *spec, const void *q, int64_t ldq, const void *k, int64_t ldk,
                   void *q_out, int64_t ldqo, void *k_out, int64_t ldko, const int32_t *positions, int32_t n_rows, void *stream);

/*
 * Accepted-path commit: for j in [0, n_commit) and every layer of the cache,
 * slot dst_slot[j] <- slot src_slot[j] (SSM state and conv window), bit for
 * bit.  After verification the drafter continues from the state of the last
 * accepted node (paper Section 3, speculative decoding loop; Section 4.1).
 * src == dst is a no-op.  A dst that is also some other pair's src is the
 * caller's hazard.  d_inner / d_state / act describe the slot contents (d_state 16 for the S6 layers above, 128 for
 * SSD layers).
 */
int mdraft_state_commit(const mdraft_cache *cache, int32_t d_inner, int32_t d_state, int32_t d_conv, int32_t act,
                        int32_t n_commit, const int32_t *src_slot, const int32_t *dst_slot,
                        int32_t *dev_status, void *stream);

/*
 * The same for slots whose state and window differ in width, as a delta layer's do: the state is (d_inner, d_state) fp32 with d_state 64
 * or 128, the window (d_conv - 1, conv_channels) activations.  conv_channels 0: the pool has no windows (cache->conv may be NULL).
 */
int mdraft_gdr_state_commit(const mdraft_cache *cache, int32_t d_inner, int32_t d_state, int32_t conv_channels, int32_t d_conv, int32_t act,
                            int32_t n_commit, const int32_t *src_slot, const int32_t *dst_slot, int32_t *dev_status, void *stream);

/*
 * Checks on the device whether A (D x N, fp32) satisfies A[d][n] == (n+1)*A[d][0]
 * bit for bit in fp32 for every d, n, and whether every entry is <= 0.
 * SYNCHRONISES `stream`.  *is_powers (HOST) receives 1 or 0; *is_nonpositive (HOST,
 * may be NULL) likewise.  No counterpart in the paper: set-up helper for MDRAFT_A_POWERS.
 * `scratch` is a device int32[2] owned by the caller.
 */
int mdraft_classify_A(const float *A, int32_t d_inner, int32_t d_state, int32_t *scratch,
                      int32_t *is_powers, int32_t *is_nonpositive, void *stream);

/*
 * Test-time tree search (paper Section 4.2, Eq. 1-2 and Appendix A.4).  Each drafting round is a round of a
 * multi-armed bandit whose K arms are preset tree configurations; the policy is UCB:
 *
 *     k* = argmax_k  mean_k + lambda_ucb * sqrt( 2 ln t / n_k )                                   (Eq. 1)
 *     r  = -( 1 / N_accept + lambda_gamma * gamma / N_accept )    for the arm that was played      (Eq. 2)
 *
 * with t the round about to be played (from 1), n_k how often arm k was played, mean_k = reward_sum[k] / n_k the
 * running mean of its rewards (the paper's "cumulative reward mean"), gamma the draft length (levels) of the played
 * tree and N_accept >= 1 the tokens the round produced.  An arm that was never played is chosen first (lowest
 * index first); ties go to the lowest index.  HOST code and HOST pointers throughout: the caller owns and zero-
 * initialises reward_sum[n_arms], count[n_arms] and round; nothing here touches a GPU.
 * Errors: NULL pointers, n_arms <= 0, arm out of range, draft_len < 1 or n_accept < 1 -> MDRAFT_ERR_INVALID_ARG.
 */
typedef struct {
    int32_t n_arms;
    int32_t reserved;
    int64_t round;          /* rounds played so far */
    double lambda_ucb;      /* exploration weight   */
    double lambda_gamma;    /* drafter / target time per token (weight of the draft-length penalty) */
    double *reward_sum;     /* HOST, n_arms */
    int64_t *count;         /* HOST, n_arms */
} mdraft_ucb;

double mdraft_ucb_reward(double lambda_gamma, int32_t draft_len, int32_t n_accept);
int mdraft_ucb_select(const mdraft_ucb *bandit, int32_t *arm);
int mdraft_ucb_update(mdraft_ucb *bandit, int32_t arm, int32_t draft_len, int32_t n_accept);

const char *mdraft_status_string(int status);

/* Library version: major*10000 + minor*100 + patch. */
int mdraft_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MDRAFT_H */
