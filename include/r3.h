/*
 * r3.h - C ABI of the replayed-routing MoE layer (Rollout Routing Replay, "R3") for NVIDIA B200.
 *
 * The library evaluates one Mixture-of-Experts layer whose expert selection is REPLAYED from a
 * record made by an inference engine, as defined in Section 4.1 of the paper
 * "Stabilizing MoE Reinforcement Learning by Aligning Training and Inference Routers":
 *
 *   s        = x W_r                                            (router logits, first equation)
 *   I        = TopKMask(s, K)                                   (second equation; capture side)
 *   g_i      = I_infer,i exp(s_train,i) / sum_j I_infer,j exp(s_train,j)      (Eq. replay_gate)
 *   y        = sum_i g_i E_i(x_train)                                          (Eq. replay_output)
 *
 * plus the gradient of a loss with respect to s_train through the replayed gate (the mask is a
 * constant; Section 4.1, purpose (b)).  The expert network E_i is a bias-free SwiGLU feed-forward
 * network of width F:  E_i(x) = W_down,i ( silu(W_gate,i x) * (W_up,i x) ).
 *
 * Notation: T tokens, d hidden size, E (= M) experts, K experts per token, R = T*K rows.
 *
 * General rules
 *  - Every pointer is a DEVICE pointer owned by the caller unless the parameter is documented as
 *    "host".  The library never allocates, frees or synchronises (except r3_replay_layer_host,
 *    which synchronises the stream before it returns); each call enqueues its kernels on
 *    `stream` (a cudaStream_t passed as void*; NULL = the legacy default stream) and returns.
 *    r3_replay_layer and the entry points built on it (_host, _blocks, _stack) also use one
 *    internal non-blocking helper stream per device, created at the first such call on that
 *    device and kept until the process exits: the router logits run there beside the
 *    permutation.  The helper is forked from and joined back into `stream` with events, so the
 *    call as a whole is ordered on `stream` exactly as if everything had been enqueued there.
 *    Host threads may call at once: the enqueue of a layer takes a process-wide lock for its
 *    few microseconds, because the helper streams and their events belong to the device.
 *  - Matrices are row-major and dense.  Weights are stored output-major: W_r [E, d],
 *    W_gate/W_up [E, F, d], W_down [E, d, F].
 *  - Activations and expert weights have dtype `act_dtype` (R3_F32 or R3_BF16); W_r has dtype
 *    `router_w_dtype`; logits, gates and their gradients are always float32.  All accumulation is
 *    float32.
 *  - The routing record holds K expert indices per token, `idx_type` R3_IDX_U8 (E <= 256) or
 *    R3_IDX_I16 (E <= 32767), laid out [layer][token][slot].  Replay accepts the K indices of a
 *    token in any order; gates are returned in the same slot order.
 *  - Alignment: all base pointers 16-byte aligned, workspaces 256-byte aligned; d and F
 *    multiples of 8.
 *  - Errors the host can see (null pointer, bad shape, workspace too small, failed launch) are
 *    returned as r3_status and nothing is launched.  Data-dependent problems (index out of range,
 *    duplicate index within a token, an internal wait that ran out) are written to the optional
 *    device word `dev_status` (first error wins; 0 = clean; the caller zeroes it); kernels never
 *    trap, and skip the offending element.
 *  - T = 0 returns R3_OK without launching.  Experts with no rows are legal.
 *  - Results are bit-reproducible from run to run: no floating-point atomics are used anywhere.
 *  - Host threads: the library keeps small host-side caches (encoded tensor maps, per-kernel
 *    attributes, the helper stream).  Calls from several host threads must be serialised by the
 *    caller; one process per GPU with one calling thread is the intended use.
 */
#ifndef R3_H_
#define R3_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    R3_OK = 0,
    R3_ERR_INVALID_ARG = 1,   /* null pointer, non-positive size, K > E, index type too narrow */
    R3_ERR_UNSUPPORTED = 2,   /* a legal shape the library has no kernel for */
    R3_ERR_WORKSPACE = 3,     /* workspace missing, too small or misaligned */
    R3_ERR_CUDA = 4,          /* a CUDA runtime/driver call failed (launch, tensor-map encode) */
    R3_ERR_SCRATCH_LIMIT = 5, /* the problem needs more than the library's fixed on-device scratch */
    R3_ERR_OUT_OF_PAGES = 6   /* r3_pagepool_alloc: fewer free pages than asked for */
} r3_status;

enum { R3_F32 = 0, R3_BF16 = 1 };
enum { R3_IDX_U8 = 1, R3_IDX_I16 = 2 };

/* values written to *dev_status by kernels */
enum { R3_DEV_OK = 0, R3_DEV_BAD_INDEX = 1, R3_DEV_DUP_INDEX = 2, R3_DEV_TIMEOUT = 3 };

typedef struct {
    int32_t T, d, E, K, F;
    int32_t act_dtype;        /* R3_F32 | R3_BF16 : x, dy, xp, h, o, y, expert weights */
    int32_t router_w_dtype;   /* R3_F32 | R3_BF16 : W_r */
    int32_t idx_type;         /* R3_IDX_U8 | R3_IDX_I16 */
} r3_shape;

const char* r3_status_string(r3_status s);

/* Section 4.1, first and second equations: router logits and TopKMask, fused.
 *   s[t,i] = sum_c x[t,c] W_r[i,c];  idx_out[t, 0..K) = the K experts with the largest s[t,.],
 *   slot order = descending logit, exact ties to the lower expert index.
 * x [T,d] act_dtype; w_router [E,d] router_w_dtype; idx_out [T,K] idx_type (may be NULL when only
 * logits are wanted); logits_out [T,E] float32 or NULL.  At least one output must be non-NULL.
 * Used on the inference side to make the record, and on the training side (logits_out set) for
 * s_train.  bf16 activations with bf16 router weights (E a multiple of 16 up to 256, K <= 16)
 * run on the tensor cores; other combinations use a float32 FMA kernel (E <= 512). */
r3_status r3_capture_topk(const r3_shape* shape, const void* x, const void* w_router,
                          void* idx_out, float* logits_out, void* stream);

/* The same for L independent layers in one launch sequence: x [L,T,d], w_router [L,E,d],
 * idx_out [L,T,K], logits_out [L,T,E] or NULL. */
r3_status r3_capture_topk_batched(const r3_shape* shape, int32_t L, const void* x,
                                  const void* w_router, void* idx_out, float* logits_out,
                                  void* stream);

/* The same with caller scratch, which lets float32 router weights use the tensor cores too: the
 * weights are split into three bf16 planes (hi + mid + lo = all 24 mantissa bits) in the
 * workspace and the three products are accumulated in fp32, so the logits keep float32-level
 * accuracy.  workspace: r3_capture_topk_workspace_bytes(shape, L) bytes (0 when none is needed:
 * bf16 router weights, or a shape the tensor-core kernel does not cover).  Without a workspace
 * (or through r3_capture_topk / _batched) float32 router weights take the float32 FMA kernel.
 * Tensor-core kernel: bf16 activations, E a multiple of 16 up to 256, K <= 16. */
size_t r3_capture_topk_workspace_bytes(const r3_shape* shape, int32_t L);
r3_status r3_capture_topk_ws(const r3_shape* shape, int32_t L, const void* x,
                             const void* w_router, void* idx_out, float* logits_out,
                             void* workspace, size_t ws_bytes, void* stream);

/* Eq. (replay_gate): softmax of the TRAINING logits over the K RECORDED experts.
 *   gates[t,j] = exp(s[t,e_j] - m) / sum_j' exp(s[t,e_j'] - m),  e_j = idx[t,j], m = max_j s[t,e_j]
 * logits [T,E] f32; idx [T,K]; gates [T,K] f32 (slot-aligned with idx).
 * dev_status (optional): R3_DEV_BAD_INDEX / R3_DEV_DUP_INDEX if a token's record is invalid; the
 * gates of such a token are written as 0. */
r3_status r3_replay_gate_fwd(const r3_shape* shape, const float* logits, const void* idx,
                             float* gates, int32_t* dev_status, void* stream);

/* Gradient through Eq. (replay_gate) with the mask held constant:
 *   c = sum_j g[t,j] dg[t,j];  dlogits[t,e_j] = g[t,j] (dg[t,j] - c);  dlogits[t,i] = 0 elsewhere.
 * gates, dgates [T,K] f32; idx [T,K]; dlogits [T,E] f32, every element written; a dlogits that is
 * not 16-byte aligned returns R3_ERR_INVALID_ARG. */
r3_status r3_replay_gate_bwd(const r3_shape* shape, const float* gates, const float* dgates,
                             const void* idx, float* dlogits, void* stream);

/* Token dispatch implied by Eq. (replay_output): expert i is evaluated only on tokens whose
 * recorded mask has I_i = 1.  The R (token, slot) pairs are grouped by expert, stably (within an
 * expert, ascending token).
 *   counts[e]        = number of pairs with idx = e                       [E]   int32
 *   offsets          = exclusive scan of counts, offsets[E] = R           [E+1] int32
 *   row_of_slot[t,j] = destination row of pair (t,j)                      [T,K] int32
 *   slot_of_row[r]   = t*K + j of the pair stored in row r                [R]   int32
 *   xp[r]            = x[slot_of_row[r] / K]                              [R,d] act_dtype
 * x / xp may both be NULL to compute the maps only.  Integer outputs are exact and independent of
 * scheduling.  workspace: r3_permute_workspace_bytes(shape) bytes.  Supported: E <= 1024.
 * dev_status (optional): R3_DEV_BAD_INDEX for an index >= E (that pair is dropped). */
size_t r3_permute_workspace_bytes(const r3_shape* shape);
r3_status r3_permute(const r3_shape* shape, const void* idx, const void* x, int32_t* counts,
                     int32_t* offsets, int32_t* row_of_slot, int32_t* slot_of_row, void* xp,
                     void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream);

/* r3_permute without a caller-supplied workspace (the paper has no counterpart; this exists for
 * the integration, not for the method).  Meant for callers that cannot allocate device memory at
 * the point of the call: for example a host process whose whole device-memory budget belongs to
 * another component's pool, where a fresh driver allocation may fail or stall the device, or a
 * step whose memory plan was fixed in advance.  The scratch (per-expert, per-256-token-chunk
 * counters) lives in a fixed array inside the library, 1 MiB on every GPU that loads the library,
 * held until the process exits.  Inputs and outputs are the caller's, exactly as for r3_permute,
 * and the results are identical to r3_permute's.
 *  - Limit: E * ceil(T / 256) <= 262144 (e.g. E = 128 up to T = 524288); beyond it the call
 *    returns R3_ERR_SCRATCH_LIMIT and launches nothing.  E <= 1024 as for r3_permute.
 *  - The call itself allocates and frees nothing, on the host or on the device.
 *  - The first call on each device looks up the array's device address (with that device
 *    current) and caches it; make that first call outside any stream capture.
 *  - Every call uses the same array, and it keeps the previous call's contents (no part of it
 *    has to be cleared: each call overwrites all the counters it later reads).  Calls that may
 *    overlap on the GPU - different streams or host threads - race on it; serialise them. */
r3_status r3_permute_static(const r3_shape* shape, const void* idx, const void* x, int32_t* counts,
                            int32_t* offsets, int32_t* row_of_slot, int32_t* slot_of_row,
                            void* xp, int32_t* dev_status, void* stream);

/* Expert networks E_i on the grouped rows: for expert e and rows r in [offsets[e], offsets[e+1])
 *   h[r] = silu(xp[r] W_gate,e^T) * (xp[r] W_up,e^T);   o[r] = h[r] W_down,e^T.
 * xp [R,d]; offsets [E+1]; w_gate, w_up [E,F,d]; w_down [E,d,F]; o [R,d]; all act_dtype.
 * bf16: tcgen05 tensor-core grouped GEMMs with fp32 accumulation, h and o rounded to bf16.
 * f32:  plain fp32 FMA kernels.
 * workspace: r3_grouped_swiglu_workspace_bytes(shape) bytes (holds h [R,F] and the tile list).
 * dev_status (optional): R3_DEV_TIMEOUT if an internal bounded wait ran out (outputs invalid). */
size_t r3_grouped_swiglu_workspace_bytes(const r3_shape* shape);
r3_status r3_grouped_swiglu(const r3_shape* shape, const void* xp, const int32_t* offsets,
                            const void* w_gate, const void* w_up, const void* w_down, void* o,
                            void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream);

/* r3_grouped_swiglu without the permuted copy of the activations: the token operand of the up
 * projection is read in place from x [T,d], row slot_of_row[r] / K for grouped row r (Eq.
 * (replay_output): expert i sees exactly the tokens whose recorded mask has I_i = 1), so
 * r3_permute can be called with x = xp = NULL and the R x d buffer never exists.  Results are
 * bit-identical to r3_grouped_swiglu on xp[r] = x[slot_of_row[r] / K].  The rows arrive through
 * four-row TMA gather copies, which on B200 run well below the rate of the tiled copies of the
 * permuted form (measured: the up projection takes about 2.8x as long), so this form is for
 * callers short of memory, not of time; r3_replay_layer uses the permuted copy.  bf16 only
 * (R3_ERR_UNSUPPORTED for float32).  slot_of_row [R] and offsets [E+1] as written by r3_permute;
 * workspace and dev_status as for r3_grouped_swiglu. */
r3_status r3_grouped_swiglu_gather(const r3_shape* shape, const void* x, const int32_t* slot_of_row,
                                   const int32_t* offsets, const void* w_gate, const void* w_up,
                                   const void* w_down, void* o, void* workspace, size_t ws_bytes,
                                   int32_t* dev_status, void* stream);

/* The two halves of r3_grouped_swiglu as separate calls (same kernels, same workspace), so that a
 * caller can place other work, or timing events, between them:
 *   r3_expert_up_swiglu : builds the tile list from offsets and writes h = silu(xp Wg^T)*(xp Wu^T)
 *                         into the workspace;
 *   r3_expert_down      : o = h W_down^T, reading h and the tile list that the preceding
 *                         r3_expert_up_swiglu call left in the SAME workspace.
 * Expert network E_i of Eq. (replay_output); argument rules as for r3_grouped_swiglu. */
r3_status r3_expert_up_swiglu(const r3_shape* shape, const void* xp, const int32_t* offsets,
                              const void* w_gate, const void* w_up, void* workspace,
                              size_t ws_bytes, int32_t* dev_status, void* stream);
r3_status r3_expert_down(const r3_shape* shape, const void* w_down, void* o, void* workspace,
                         size_t ws_bytes, int32_t* dev_status, void* stream);

/* Eq. (replay_output): y[t] = sum_{j=0..K-1} gates[t,j] * o[row_of_slot[t,j]], added in slot
 * order in fp32 (no atomics), rounded once to act_dtype.  o [R,d]; y [T,d].
 * r3_combine, r3_combine_residual and r3_combine_bwd_gates take no dev_status word: should one of
 * their internal bounded waits ever run out, the affected token's output is left unwritten without
 * a report.  r3_replay_finish (what the layer runs) computes the same values and reports
 * R3_DEV_TIMEOUT. */
r3_status r3_combine(const r3_shape* shape, const void* o, const int32_t* row_of_slot,
                     const float* gates, void* y, void* stream);

/* The same with a residual: y[t] = residual[t] + sum_j gates[t,j] * o[row_of_slot[t,j]] (the sum is
 * formed first, the residual added last, all in fp32, one rounding).  residual [T,d] act_dtype or
 * NULL (then identical to r3_combine).  Used by r3_replay_stack for x_{l+1} = x_l + y_l. */
r3_status r3_combine_residual(const r3_shape* shape, const void* o, const int32_t* row_of_slot,
                              const float* gates, const void* residual, void* y, void* stream);

/* Chain rule on Eq. (replay_output): dgates[t,j] = sum_c dy[t,c] * o[row_of_slot[t,j], c].
 * dy [T,d] act_dtype; dgates [T,K] f32. */
r3_status r3_combine_bwd_gates(const r3_shape* shape, const void* dy, const void* o,
                               const int32_t* row_of_slot, float* dgates, void* stream);

/* Everything that follows the expert networks, in one pass over the expert outputs: the replay
 * gate of Eq. (replay_gate), the combine of Eq. (replay_output), the gate gradient and the
 * router-logit gradient (Section 4.1, purpose (b): the mask is a constant).  Per token,
 *   g      = softmax of logits[t, idx[t, .]]                       (as r3_replay_gate_fwd)
 *   y[t]   = residual[t] + sum_j g_j o[row_of_slot[t,j]]           (as r3_combine_residual)
 *   dg_j   = <dy[t], o[row_of_slot[t,j]]>                          (as r3_combine_bwd_gates)
 *   dlogits[t, idx[t,j]] = g_j (dg_j - sum_j' g_j' dg_j'), 0 elsewhere   (as r3_replay_gate_bwd)
 * with the same arithmetic and summation orders as those four calls, so y, gates and dlogits are
 * bit-identical to theirs, but each expert-output row is read once instead of twice.
 * logits [T,E] f32; idx [T,K]; o [R,d]; row_of_slot [T,K]; dy [T,d]; residual [T,d] or NULL;
 * outputs y [T,d], gates_out [T,K] f32 or NULL, dlogits [T,E] f32 (every element written).
 * Supported for K <= 8 (R3_ERR_UNSUPPORTED beyond; use the four calls).  dev_status as for
 * r3_replay_gate_fwd. */
r3_status r3_replay_finish(const r3_shape* shape, const float* logits, const void* idx,
                           const void* o, const int32_t* row_of_slot, const void* dy,
                           const void* residual, void* y, float* gates_out, float* dlogits,
                           int32_t* dev_status, void* stream);

/* The whole replayed layer, forward and router-logit backward, enqueued back to back on one
 * stream: logits -> replay gate -> permute -> experts -> combine -> dgates -> dlogits.
 * Inputs x [T,d], w_router [E,d], idx [T,K], expert weights, dy [T,d];
 * outputs y [T,d] act_dtype and dlogits [T,E] f32.  Intermediates live in `workspace`
 * (r3_replay_layer_workspace_bytes).  Optional outputs (may be NULL): gates_out [T,K] f32. */
size_t r3_replay_layer_workspace_bytes(const r3_shape* shape);
r3_status r3_replay_layer(const r3_shape* shape, const void* x, const void* w_router,
                          const void* idx, const void* w_gate, const void* w_up,
                          const void* w_down, const void* dy, void* y, float* dlogits,
                          float* gates_out, void* workspace, size_t ws_bytes,
                          int32_t* dev_status, void* stream);
/* The same layer for another pass over the SAME record: the rollout's record is replayed in the
 * Recompute stage and again in the Update stage (Section 5.1, settings of the method; Section 6.3),
 * so the dispatch (counts, offsets, both maps) and the expert
 * work lists that the preceding r3_replay_layer call left in `workspace` still hold; this call
 * copies the rows of the new x with those maps and skips the dispatch.  `workspace` must be the
 * one that call used, untouched since, with the same shape and the same idx (idx is still read:
 * the gate needs it); x, the weights and dy may differ.  Results are bit-identical to
 * r3_replay_layer on the same arguments.  Passing a workspace that holds no such dispatch gives
 * undefined results (rows are copied to whatever row numbers it holds: call r3_replay_layer
 * first). */
r3_status r3_replay_layer_same_record(const r3_shape* shape, const void* x, const void* w_router,
                          const void* idx, const void* w_gate, const void* w_up,
                          const void* w_down, const void* dy, void* y, float* dlogits,
                          float* gates_out, void* workspace, size_t ws_bytes,
                          int32_t* dev_status, void* stream);

/* L independent replayed MoE blocks enqueued back to back: block l is r3_replay_layer on its own
 * input x[l], record idx[l], weights and upstream gradient dy[l] (a model's MoE blocks with the
 * sublayers between them left out, so that every block's input is given).  All tensors carry a
 * leading layer axis: x, dy, y [L,T,d]; w_router [L,E,d]; idx [L,T,K]; w_gate/w_up [L,E,F,d];
 * w_down [L,E,d,F]; dlogits [L,T,E] f32.  workspace: r3_replay_layer_workspace_bytes(shape). */
r3_status r3_replay_blocks(const r3_shape* shape, int32_t L, const void* x, const void* w_router,
                           const void* idx, const void* w_gate, const void* w_up,
                           const void* w_down, const void* dy, void* y, float* dlogits,
                           void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream);

/* A stack of L replayed MoE blocks (no attention) with residual connections,
 *   x_{l+1} = x_l + y_replay,l(x_l),   l = 0..L-1,
 * each block being Eq. (replay_output) with its own weights and its own record, plus the
 * router-logit gradient of every block for one upstream gradient dy [T,d] shared by all blocks
 * (the gradient that reaches a block's output through the identity path of the later blocks).
 * Per-layer tensors are stacked on a leading layer axis: w_router [L,E,d], idx [L,T,K],
 * w_gate/w_up [L,E,F,d], w_down [L,E,d,F]; x0 [T,d]; outputs x_out [T,d] = x_L and
 * dlogits [L,T,E] f32.  workspace: r3_replay_stack_workspace_bytes(shape) (independent of L). */
size_t r3_replay_stack_workspace_bytes(const r3_shape* shape);
r3_status r3_replay_stack(const r3_shape* shape, int32_t L, const void* x0, const void* w_router,
                          const void* idx, const void* w_gate, const void* w_up,
                          const void* w_down, const void* dy, void* x_out, float* dlogits,
                          void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream);

/* As r3_replay_layer, with the per-step tensors in HOST memory (pinned memory recommended):
 * x_host, idx_host, dy_host are copied to the device, y_host and dlogits_host are copied back,
 * and the stream is synchronised before returning.  Weights stay on the device.  The workspace
 * must hold r3_replay_layer_host_workspace_bytes(shape) bytes (device staging included).
 * From 16384 tokens on the batch goes through in chunks of tokens (r3_replay_layer_host_chunks),
 * each a layer of its own: the copies travel on two library-owned streams beside the kernels on
 * `stream`, which ends behind the last result copy.  Every token's result is what a layer of its
 * chunk alone gives; against one launch over the whole batch it may differ in the last bits (the
 * router kernel sums d in another order for another token count). */
size_t r3_replay_layer_host_workspace_bytes(const r3_shape* shape);
/* How r3_replay_layer_host cuts shape->T tokens: writes starts[0..n] (host memory, room for 17
 * values; starts[0] = 0, starts[n] = T, chunk c holds tokens [starts[c], starts[c+1])) and returns
 * n; 0 for a bad shape or a null pointer.  Equal chunks of at least 8192 tokens, multiples of
 * 256, the last one cut into a half and two quarters (the compute and the result copy of the last
 * chunk are what the call cannot hide under its input copies).  A host-side schedule: the paper
 * has no counterpart. */
int32_t r3_replay_layer_host_chunks(const r3_shape* shape, int64_t* starts);
r3_status r3_replay_layer_host(const r3_shape* shape, const void* x_host, const void* w_router,
                               const void* idx_host, const void* w_gate, const void* w_up,
                               const void* w_down, const void* dy_host, void* y_host,
                               float* dlogits_host, void* workspace, size_t ws_bytes,
                               int32_t* dev_status, void* stream);
/* The same without the final synchronisation: copies in, layer and copies out are enqueued on
 * `stream` and the call returns.  y_host and dlogits_host hold the result once the caller has
 * synchronised the stream; the host buffers and the workspace must stay untouched until then
 * (pageable host memory makes the copies synchronous: use pinned memory).  A caller that feeds a
 * sequence of batches keeps two or more of them in flight, each with its own stream, workspace and
 * host buffers: the copies of one batch then run beside the kernels of another.  Errors as
 * r3_replay_layer_host. */
r3_status r3_replay_layer_host_enqueue(const r3_shape* shape, const void* x_host,
                                       const void* w_router, const void* idx_host,
                                       const void* w_gate, const void* w_up, const void* w_down,
                                       const void* dy_host, void* y_host, float* dlogits_host,
                                       void* workspace, size_t ws_bytes, int32_t* dev_status,
                                       void* stream);

/* ---- Update-stage backward to the layer input (Section 4.1, purpose (b)) ------------------------ */

/* Input gradient of the expert networks on the grouped rows.  With a = xp W_gate,e^T,
 * b = xp W_up,e^T (the forward's pre-activations), h = silu(a) * b, o = h W_down,e^T and a
 * gradient dout = dL/do:
 *   dh  = dout W_down,e ;  da = dh * b * silu'(a) ;  db = dh * silu(a) ;
 *   dxp = da W_gate,e + db W_up,e                                   (= dL/dxp)
 * dout, dxp [R,d]; pre_gate, pre_up [R,F] (as stored by the forward, bf16); weights as in
 * r3_grouped_swiglu (read transposed in place, no transposed copy is made).  bf16 only
 * (R3_ERR_UNSUPPORTED for float32).  dh, da, db are rounded to bf16 once each.
 * workspace: r3_grouped_swiglu_bwd_workspace_bytes(shape). */
size_t r3_grouped_swiglu_bwd_workspace_bytes(const r3_shape* shape);
r3_status r3_grouped_swiglu_bwd_input(const r3_shape* shape, const void* dout, const void* pre_gate,
                                      const void* pre_up, const int32_t* offsets,
                                      const void* w_gate, const void* w_up, const void* w_down,
                                      void* dxp, void* workspace, size_t ws_bytes,
                                      int32_t* dev_status, void* stream);

/* The whole backward of the grouped experts: dxp as r3_grouped_swiglu_bwd_input, and the
 * gradients of the expert weights, for each expert e over its rows [offsets[e], offsets[e+1]):
 *   dW_down[e] = dout_e^T h_e     dW_gate[e] = da_e^T xp_e     dW_up[e] = db_e^T xp_e
 * xp [R,d] are the permuted rows the forward saw.  dw_gate, dw_up [E,F,d] and dw_down [E,d,F] are
 * float32 and are OVERWRITTEN (an expert without rows gets zeros); products of bf16 operands
 * (h, da, db rounded to bf16 once each) accumulate in float32 in a fixed order.  bf16 only.
 * workspace: r3_grouped_swiglu_bwd_workspace_bytes(shape). */
r3_status r3_grouped_swiglu_bwd(const r3_shape* shape, const void* xp, const void* dout,
                                const void* pre_gate, const void* pre_up, const int32_t* offsets,
                                const void* w_gate, const void* w_up, const void* w_down,
                                void* dxp, float* dw_gate, float* dw_up, float* dw_down,
                                void* workspace, size_t ws_bytes, int32_t* dev_status,
                                void* stream);

/* r3_grouped_swiglu that also keeps what its backward needs: besides o it stores the
 * pre-activations pre_gate = xp W_gate,e^T and pre_up = xp W_up,e^T ([R,F] each, rounded to bf16
 * from the float32 accumulator; h is formed from the unrounded values, so o is bit-identical to
 * r3_grouped_swiglu's).  bf16 only (R3_ERR_UNSUPPORTED for float32).  Same workspace. */
r3_status r3_grouped_swiglu_train(const r3_shape* shape, const void* xp, const int32_t* offsets,
                                  const void* w_gate, const void* w_up, const void* w_down,
                                  void* o, void* pre_gate, void* pre_up, void* workspace,
                                  size_t ws_bytes, int32_t* dev_status, void* stream);

/* Gradient of the expert outputs under Eq. (replay_output), y_t = sum_j g[t,j] o[row(t,j)]:
 *   dout[row_of_slot[t,j], :] = gates[t,j] * dy[t, :]
 * dy [T,d], gates [T,K] float32, row_of_slot [T,K], dout [R,d] (every row written once; slots
 * with row_of_slot < 0 are skipped).  No workspace. */
r3_status r3_scale_rows(const r3_shape* shape, const void* dy, const float* gates,
                        const int32_t* row_of_slot, void* dout, void* stream);

/* Last step of the backward to the layer input.  The input x_t reaches the loss through its K
 * experts and through the training logits s = x W_r^T that feed the replay gate (the recorded
 * mask is a constant, Section 4.1):
 *   dx[t,:]        = dx_residual[t,:] + sum_j dxp[row_of_slot[t,j], :]
 *                    + sum_j dlogits[t, e_j] * W_r[e_j, :]
 *   dw_router[e,:] = sum over tokens t whose record holds e of dlogits[t,e] * x[t,:]
 * (the replay gate's dlogits is zero outside the record, so these are the full products dlogits W_r and
 * dlogits^T x; of a gradient that is not, r3_balance_loss's say, only the recorded experts' columns would
 * be used, so it does not go through here.)  dxp [R,d], dlogits [T,E] float32, idx [T,K], x [T,d], w_router [E,d]
 * (router_w_dtype), dx [T,d], dw_router [E,d] float32; dx_residual [T,d] (the gradient that
 * reaches x around the layer, e.g. through a residual connection) or null for none, never the
 * same buffer as dx; row_of_slot / slot_of_row / offsets from
 * r3_permute.  Sums run in float32 in a fixed order (dx: slot order; dw_router: eight interleaved
 * partial sums over the expert's rows, added in order): reproducible.  An
 * expert that appears twice in a token's record contributes its term twice to dx, as the
 * gradient of the gate does.  K <= 64 (R3_ERR_UNSUPPORTED beyond).  No workspace. */
r3_status r3_input_grad_finish(const r3_shape* shape, const void* dxp, const int32_t* row_of_slot,
                               const int32_t* slot_of_row, const int32_t* offsets,
                               const float* dlogits, const void* idx, const void* x,
                               const void* w_router, const void* dx_residual, void* dx,
                               float* dw_router, void* stream);

/* r3_replay_layer followed by its backward to the layer input and to the router weight, one
 * enqueue: y, dlogits as in r3_replay_layer, then dout = g dy, the expert input gradient
 * (r3_grouped_swiglu_bwd) and r3_input_grad_finish.  dx [T,d], dw_router [E,d] float32.
 * dw_gate, dw_up [E,F,d], dw_down [E,d,F] float32 receive the expert-weight gradients
 * (overwritten); pass all three null to skip them.  bf16 only
 * (R3_ERR_UNSUPPORTED for float32; r3_replay_layer_train_workspace_bytes returns 0 then).
 * workspace: r3_replay_layer_train_workspace_bytes(shape), 256-byte aligned. */
size_t r3_replay_layer_train_workspace_bytes(const r3_shape* shape);
r3_status r3_replay_layer_train(const r3_shape* shape, const void* x, const void* w_router,
                                const void* idx, const void* w_gate, const void* w_up,
                                const void* w_down, const void* dy, void* y, float* dlogits,
                                void* dx, float* dw_router, float* dw_gate, float* dw_up,
                                float* dw_down, void* workspace, size_t ws_bytes,
                                int32_t* dev_status, void* stream);

/* L residual blocks x_{l+1} = x_l + y_replay,l(x_l) (as r3_replay_stack), then the exact backward
 * chain of <dy, x_L>:  g_L = dy,  g_l = g_{l+1} + dx_l(g_{l+1}),  where block l's backward is
 * r3_replay_layer_train's at its own input x_l with upstream gradient g_{l+1} and the residual
 * path carries g_{l+1} through unchanged.  Block inputs are kept (L activations of [T,d]); each
 * block's forward is run again in the backward pass instead of keeping its intermediates.
 * Per-block tensors are stacked along a leading L: w_router [L,E,d], idx [L,T,K], w_gate / w_up
 * [L,E,F,d], w_down [L,E,d,F]; dy [T,d] = dL/dx_L.  Outputs: x_out [T,d] = x_L, dlogits [L,T,E]
 * (the exact router-logit gradients), dx0 [T,d] = dL/dx_0 (not the same buffer as dy),
 * dw_router [L,E,d] float32, and dw_gate / dw_up [L,E,F,d], dw_down [L,E,d,F] float32 or all
 * three null.  Activations and the gradients g_l are stored in bf16 between blocks.  bf16 only.
 * workspace: r3_replay_stack_train_workspace_bytes(shape, L). */
size_t r3_replay_stack_train_workspace_bytes(const r3_shape* shape, int32_t L);
r3_status r3_replay_stack_train(const r3_shape* shape, int32_t L, const void* x0,
                                const void* w_router, const void* idx, const void* w_gate,
                                const void* w_up, const void* w_down, const void* dy, void* x_out,
                                float* dlogits, void* dx0, float* dw_router, float* dw_gate,
                                float* dw_up, float* dw_down, void* workspace, size_t ws_bytes,
                                int32_t* dev_status, void* stream);

/* ---- expert parallelism: bookkeeping of the row exchange (an extension; the paper describes
 * no parallelism) ------------------------------------------------------------------------------
 *
 * With the E experts split over N ranks (rank q owns the experts [q E/N, (q+1) E/N)) every rank
 * runs r3_permute on its own tokens with GLOBAL expert numbers; the grouped rows bound for one rank
 * are then a contiguous block, the blocks are exchanged with an all-to-all (the caller's:
 * torch.distributed / NCCL), and the receiver holds [source rank][local expert][row].  The library
 * supplies the reordering into the [local expert][source rank][row] order that r3_grouped_swiglu
 * takes (with T = received rows, K = 1, E = E/N), and its inverse for the way back.
 *
 * r3_ep_regroup_map: recv_counts [n_src, e_local] int32 = rows received from each source for each
 * local expert; rows = their sum (known to the host from the split sizes; a table that does not
 * add up to it sets dev_status and writes nothing).  Writes perm [rows] (position in the new
 * order -> arrival index) and offsets [e_local + 1] (first row of each local expert in the new
 * order).  n_src * e_local <= 4096 (R3_ERR_UNSUPPORTED beyond).
 * r3_ep_move_rows: inverse = 0: dst[j] = src[perm[j]];  inverse = 1: dst[perm[j]] = src[j], for
 * rows of row_bytes bytes (a multiple of 16).  src and dst must not be the same buffer. */
r3_status r3_ep_regroup_map(const int32_t* recv_counts, int32_t n_src, int32_t e_local,
                            int32_t rows, int32_t* perm, int32_t* offsets, int32_t* dev_status,
                            void* stream);
r3_status r3_ep_move_rows(const void* src, void* dst, const int32_t* perm, int32_t rows,
                          size_t row_bytes, int32_t inverse, void* stream);

/* The same exchange without a collective for the rows: every rank writes its rows straight
 * into the owners' buffers (plain stores to memory this GPU can address: its own, or a peer's
 * mapped with peer access / symmetric memory, over NVLink), at the place they have in the owner's
 * [local expert][source][row] order, and later fetches the expert outputs of its rows from the
 * owners' output buffers by address.  No multicast load is involved anywhere.
 *
 * r3_ep_dest_table: counts_all [n_ranks, E] int32 (device; the ranks' `counts` of r3_permute after
 * an all-gather).  Writes dst_base [E] (row, in the owner's buffer, of THIS rank's first row of
 * every expert) and offsets_local [E / n_ranks + 1] (the offsets r3_grouped_swiglu takes for this
 * rank's own experts).  n_ranks <= 64.
 * r3_ep_dispatch_rows: copies x[t] to its K places; idx, row_of_slot and my_offsets (= offsets) are
 * those of this rank's r3_permute (called without x); peer_buffers_host [n_ranks] is a HOST array
 * of device addresses, entry q = base of rank q's receive buffer [capacity_rows, d] (the same
 * capacity on every rank).  A row whose place lies at or beyond capacity_rows is NOT stored and
 * dev_status (optional) receives R3_DEV_BAD_INDEX: a peer's memory is never written out of
 * bounds.  The owners must not read the buffers before every rank's call has completed (a barrier
 * of the job's own).
 * r3_ep_slot_rows: row_ptr [T, K] (device, 64-bit addresses) = where the expert-output row of each
 * (token, slot) pair will stand in the owners' OUTPUT buffers (peer_buffers_host: their bases,
 * capacity_rows as above); 0 for a pair that r3_permute dropped or whose place is beyond the
 * capacity (then dev_status receives R3_DEV_BAD_INDEX).
 * r3_replay_finish_rows: r3_replay_finish with the rows given by address (row_ptr) instead of
 * (o, row_of_slot).  K <= 8 and the rows of one token must fit in shared memory
 * ((K + 2) d elements, else R3_ERR_UNSUPPORTED). */
r3_status r3_ep_dest_table(const int32_t* counts_all, int32_t n_ranks, int32_t E, int32_t rank,
                           int32_t* dst_base, int32_t* offsets_local, void* stream);
r3_status r3_ep_dispatch_rows(const r3_shape* shape, int32_t n_ranks, const void* x,
                              const void* idx, const int32_t* row_of_slot,
                              const int32_t* my_offsets, const int32_t* dst_base,
                              const unsigned long long* peer_buffers_host, int64_t capacity_rows,
                              int32_t* dev_status, void* stream);
r3_status r3_ep_slot_rows(const r3_shape* shape, int32_t n_ranks, const void* idx,
                          const int32_t* row_of_slot, const int32_t* my_offsets,
                          const int32_t* dst_base, const unsigned long long* peer_buffers_host,
                          int64_t capacity_rows, unsigned long long* row_ptr, int32_t* dev_status,
                          void* stream);
r3_status r3_replay_finish_rows(const r3_shape* shape, const float* logits, const void* idx,
                                const unsigned long long* row_ptr, const void* dy,
                                const void* residual, void* y, float* gates_out, float* dlogits,
                                int32_t* dev_status, void* stream);

/* ---- between two blocks: norm, gate, scaled residual, norm (an extension; the paper's model has
 * norms around its blocks and does not discuss them) ---------------------------------------------- */

/* What the gate of a block's output is, and along what it is broadcast over [T, d]. */
enum { R3_GATE_NONE = 0, R3_GATE_CHANNEL = 1, R3_GATE_TOKEN = 2, R3_GATE_FULL = 3 };

/* T rows of d columns (a multiple of 8) of act_dtype; w_dtype is the type of w_post, w_pre and of a
 * CHANNEL gate [d].  A TOKEN gate [T] is float32, a FULL gate [T,d] act_dtype.  eps > 0. */
typedef struct {
    int32_t T, d;
    int32_t act_dtype, w_dtype, gate_kind;
    float eps, residual_scale, branch_scale;
} r3_norm;

/* The step from one residual block to the next, in one pass:
 *   n     = y rsqrt(mean(y^2) + eps) w_post          RMSNorm behind the block (n = y if w_post is NULL)
 *   x_out = residual_scale x + branch_scale gate n
 *   h     = x_out rsqrt(mean(x_out^2) + eps) w_pre   RMSNorm in front of the next block
 * x [T,d] the residual stream, y [T,d] the block's output.  h is formed from the float32 x_out, each
 * output is rounded once.  y NULL (with w_post, gate and x_out NULL): in front of the first block,
 * h = the norm of x.  w_pre and h NULL: behind the last block.  x_out may be x's buffer, and h y's.
 * T up to 2^30; d up to 16384 for bf16 and 8192 for f32 (R3_ERR_UNSUPPORTED beyond).  No workspace. */
r3_status r3_norm_residual(const r3_norm* shape, const void* x, const void* y, const void* w_post,
                           const void* gate, const void* w_pre, void* x_out, void* h, void* stream);

/* Its gradients, from dx_out = dL/dx_out [T,d] (NULL = 0) and dh = dL/dh [T,d]:
 *   g = dx_out + (gradient of the pre-norm at x_out);   dx = residual_scale g;
 *   dy, dw_post, dgate through the branch;   dw_pre = sum_t dh x_out rsqrt(mean(x_out^2) + eps)
 * x_out and y as the forward left them (x_out is x where y is NULL; it is not needed without w_pre).
 * dx, dy [T,d] act_dtype; dw_post, dw_pre [d] float32; dgate float32 [d] (CHANNEL) or [T] (TOKEN),
 * act_dtype [T,d] (FULL).  All are overwritten; the sums over tokens are formed in float32 in an
 * order that depends on the shape alone.  An output is given exactly where its input is.  dx may be
 * dx_out's or dh's buffer, dy may be y's, dh's or dx_out's (dx and dy differ).  workspace:
 * r3_norm_residual_bwd_workspace_bytes(shape), 256-byte aligned. */
size_t r3_norm_residual_bwd_workspace_bytes(const r3_norm* shape);
r3_status r3_norm_residual_bwd(const r3_norm* shape, const void* x_out, const void* y,
                               const void* w_post, const void* gate, const void* w_pre,
                               const void* dx_out, const void* dh, void* dx, void* dy,
                               float* dw_post, void* dgate, float* dw_pre, void* workspace,
                               size_t ws_bytes, void* stream);

/* ---- optimiser step (an extension: what follows the weight gradients of the training calls) ------ */

/* One tensor of a step; the struct lives in HOST memory, its pointers are device pointers (16-byte
 * aligned, the scales 4-byte).  n elements (0: the entry is skipped).
 *   param             n of param_dtype, updated
 *   master            n float32 (with config->master, for bf16 parameters: the step updates them and
 *                     stores their rounding to param, which is not read) or NULL
 *   grad              n of grad_dtype
 *   exp_avg, exp_avg_sq   states: n float32 each; or, with 8-bit states, n e4m3 codes each and one
 *                     float32 scale per 256 elements (ceil(n / 256)) in exp_avg_scale and
 *                     exp_avg_sq_scale.  A value is code * scale; exp_avg_sq then holds the square
 *                     ROOT of the second moment.  All zero bytes are the fresh state in both forms. */
typedef struct {
    void* param;
    float* master;
    const void* grad;
    void* exp_avg;
    void* exp_avg_sq;
    float* exp_avg_scale;
    float* exp_avg_sq_scale;
    int64_t n;
    float weight_decay;
} r3_adamw_tensor;

/* step t counts from 1; master is 0 or 1; state_bits 8 or 32; eps >= 1e-30. */
typedef struct {
    int32_t param_dtype, grad_dtype, master, state_bits;
    int64_t step;
    double lr, beta1, beta2, eps;
} r3_adamw;

/* One AdamW step over n_tensors tensors (a HOST array) in one launch per 400:
 *   g = grad * grad_scale
 *   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2
 *   w = w (1 - lr weight_decay) - lr m / (1 - beta1^t) / ( sqrt(v / (1 - beta2^t)) + eps )
 * in float32, w rounded once to param_dtype.  8-bit states: the scale of a block of 256 elements is
 * the smallest power of two (at least 2^-126) that brings its largest magnitude to 448 or less, a
 * code is the nearest e4m3 value (ties to even), a root above 0 gets at least the smallest code.
 * Every product and sum that forms m, v and the scales is rounded to float32 by itself, and so are the root
 * (of the stored states and of the update) and the update's quotient; only with 8-bit states and bf16
 * parameters without masters the update takes the hardware's approximations of these two (within 2^-21 of
 * it, before the weight's rounding).  The stored states do not depend on the launch or the other tensors.
 *  - grad_scale (device, float32, or NULL = 1): a loss scale's inverse or a clipping factor.  If it
 *    is not finite the whole step is skipped: nothing is written.
 *  - scalars (device, [3] float32, or NULL): {lr, 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)} in place of
 *    config's lr and step, for a captured step that is replayed with new values.
 *  - A gradient element that is not finite makes its own weight NaN and its states NaN, or infinite as the
 *    gradient is (an 8-bit state: the NaN code; the scale is that of the block's finite elements).
 * Buffers that the step writes (params, masters, states, scales; of all entries) and that overlap, each
 * other or a gradient, grad_scale or scalars, are refused.  No workspace. */
r3_status r3_adamw_step(const r3_adamw* config, const r3_adamw_tensor* tensors, int32_t n_tensors,
                        const float* grad_scale, const float* scalars, void* stream);

/* ---- orthogonalised updates (an extension: an optimiser for matrices beside r3_adamw_step) ---------- */

/* batch matrices [rows, cols], dense and row-major, sides up to 16384.  steps 1 to 16; coefs (HOST,
 * [steps][3] = a, b, c of each step) or NULL = (3.4445, -4.7750, 2.0315) for all.  products: 1 = every product
 * from fp16 operands (off by 1.3e-3 to 3e-3 of the result's root mean square, a rounding to bf16 by 1.7e-3; matrices
 * with a side below 16, which would be further off, take 3), 3 = from operands of two fp16 planes (a float32 result).
 * eps >= 0 (below 4e-36 taken as that). */
typedef struct {
    int32_t batch, rows, cols, in_dtype, out_dtype, steps, products;
    double eps;
    const double* coefs;
} r3_orthogonal;

/* Newton-Schulz iteration, per matrix: X = x / (|x|_F + eps), then steps times, with the Gram matrix of the
 * smaller side (here rows <= cols),
 *   A = X X^T;   B = b A + c A^2;   X = a X + B X
 * which brings the singular values near one; out = X.  x of in_dtype, out of out_dtype: the same buffer (of
 * one type) or no memory in common.  All products accumulate in float32, X is carried in 22 bits between the
 * steps (into the last one in 11, where its a is at most 4 and the result is rounded to bf16): so far as an
 * element of X is above 2^-28, below that within 2^-50 (one plane, as the operand of one product: 2^-39).  With
 * coefficients whose iterates pass 3.75 in norm these limits rise, to 16 times that at 60.
 *  - A matrix of zeros gives zeros, one that holds what is not finite gives NaN; the others of a batch are
 *    not touched by it.
 *  - Coefficients whose iterates could pass 16 in norm (or b A + c A^2, with or without a, 60) are refused.
 * workspace: r3_orthogonalize_workspace_bytes(config), 256-byte aligned: up to about 600 MB (or what one matrix
 * needs); larger batches are taken in parts.  Matrices with a side of at most 128 and the other of at most 2048
 * need none to speak of: they are taken in one launch, on the chip. */
size_t r3_orthogonalize_workspace_bytes(const r3_orthogonal* config);
r3_status r3_orthogonalize(const r3_orthogonal* config, const void* x, void* out, void* workspace,
                           size_t ws_bytes, int32_t* dev_status, void* stream);

/* A stack of `batch` matrices [rows, cols] of one parameter (expert weights [E, F, d] are E of them); the struct
 * lives in HOST memory, its pointers are device pointers (16-byte aligned).  momentum float32; master float32
 * (with config->master) or NULL.  scale multiplies the orthogonalised update. */
typedef struct {
    void* param;
    float* master;
    const void* grad;
    float* momentum;
    int32_t batch, rows, cols;
    float weight_decay, scale;
} r3_muon_stack;

/* products, steps, coefs and eps as for r3_orthogonal. */
typedef struct {
    int32_t param_dtype, grad_dtype, master, nesterov, steps, products;
    double lr, momentum, eps;
    const double* coefs;
} r3_muon;

/* One step over n_stacks stacks (a HOST array).  Per matrix, with g = grad * grad_scale:
 *   m = momentum m + g;   u = g + momentum m (nesterov) or m;   o = r3_orthogonalize(u)
 *   w = w (1 - lr weight_decay) - lr scale o
 * w is the master where there is one (param then gets its rounding), else param.  Stacks of one shape are taken
 * together.  grad_scale (device, float32, or NULL = 1): not finite = the whole step is skipped, nothing is
 * written.  lr (device, [1] float32, or NULL): in place of config's, for a captured step.
 *  - A matrix whose u is not finite gets NaN weights; its momentum is what the formula gives.
 *  - Buffers that the step writes and that overlap, each other or one that it reads, are refused.
 * workspace: r3_muon_workspace_bytes(config, stacks, n_stacks). */
size_t r3_muon_workspace_bytes(const r3_muon* config, const r3_muon_stack* stacks, int32_t n_stacks);
r3_status r3_muon_step(const r3_muon* config, const r3_muon_stack* stacks, int32_t n_stacks,
                       const float* grad_scale, const float* lr, void* workspace, size_t ws_bytes,
                       int32_t* dev_status, void* stream);

/* ---- stacks of replayed blocks with norms around every block (an extension) ----------------------- */

/* The norms of L blocks, stacked on a leading layer axis, all of w_dtype and 16-byte aligned:
 *   h_l     = RMSNorm(x_l) w_pre[l]
 *   x_{l+1} = residual_scale x_l + branch_scale gate[l] RMSNorm(y_replay,l(h_l)) w_post[l]
 * w_pre [L,d]; w_post [L,d] or NULL (the block's output is not normalised); gate [L,d] or NULL.
 * dw_pre, dw_post, dgate [L,d] float32: their gradients, overwritten by r3_normed_stack_train, given
 * exactly where their vector is.  The struct lives in HOST memory. */
typedef struct {
    const void *w_pre, *w_post, *gate;
    float *dw_pre, *dw_post, *dgate;
    int32_t w_dtype;
    float eps, residual_scale, branch_scale;
} r3_block_norms;

/* The stack forward: x0 [T,d] -> x_out [T,d] = x_L.  Between two blocks runs one r3_norm_residual; a
 * block's router and experts read h_l.  Layers as in r3_replay_stack.  workspace:
 * r3_normed_stack_workspace_bytes(shape). */
size_t r3_normed_stack_workspace_bytes(const r3_shape* shape);
r3_status r3_normed_stack(const r3_shape* shape, int32_t L, const r3_block_norms* norms,
                          const void* x0, const void* w_router, const void* idx, const void* w_gate,
                          const void* w_up, const void* w_down, void* x_out, void* workspace,
                          size_t ws_bytes, int32_t* dev_status, void* stream);

/* Forward and the exact backward chain of <dy, x_L>: dlogits [L,T,E], dx0 [T,d] = dL/dx_0, dw_router
 * [L,E,d] float32, the norms' gradients, and the expert-weight gradients dw_gate / dw_up [L,E,F,d],
 * dw_down [L,E,d,F] float32 or all three NULL.  x_out is a buffer of its own.  x_l, h_l and y_l are kept,
 * a block's other intermediates are formed again in the backward pass.  bf16 only (R3_ERR_UNSUPPORTED for
 * float32).
 *
 * With adamw (HOST) the expert weights are updated in place, each block's as soon as its gradients are
 * there: dw_gate, dw_up [E,F,d] and dw_down [E,d,F] then hold ONE block's gradients (those of block 0
 * at the end), so that no more than that exists at a time.  expert_states (HOST) has 3 L entries, block
 * by block w_gate, w_up, w_down, as for r3_adamw_step; param must be the block's weights, grad is
 * ignored.  adamw, grad_scale and scalars as for r3_adamw_step, param_dtype R3_BF16, grad_dtype R3_F32.
 * With T = 0 nothing is written and no step taken.  A block takes no step once dev_status is not 0, by an
 * error of this call (with dev_status NULL the call watches for itself) or one that it still holds: an invalid
 * record is found in the forward pass, before any step; a wait that runs out in the backward pass leaves the
 * blocks behind it stepped, and those before it as they were.
 * workspace: r3_normed_stack_train_workspace_bytes(shape, L). */
size_t r3_normed_stack_train_workspace_bytes(const r3_shape* shape, int32_t L);
r3_status r3_normed_stack_train(const r3_shape* shape, int32_t L, const r3_block_norms* norms,
                                const void* x0, const void* w_router, const void* idx, void* w_gate,
                                void* w_up, void* w_down, const void* dy, void* x_out, float* dlogits,
                                void* dx0, float* dw_router, float* dw_gate, float* dw_up,
                                float* dw_down, const r3_adamw* adamw,
                                const r3_adamw_tensor* expert_states, const float* grad_scale,
                                const float* scalars, void* workspace, size_t ws_bytes,
                                int32_t* dev_status, void* stream);

/* ---- token log probabilities (the p_train and p_infer of Sections 3.1 and 3.2) -------------- */

/* A batch of logits: T rows of V values, row t at logits + t * ld elements (ld >= V, so a padded or
 * sliced vocabulary is taken as it lies), dtype R3_F32 or R3_BF16.  token_ids are int32 or int64
 * (id_bytes 4 or 8).  temperature (1e-6 to 1e20) divides the logits. */
typedef struct {
    int32_t T, V;
    int64_t ld;
    int32_t dtype, id_bytes;
    double temperature;
} r3_logits;

/* For every row x, with top = max_v x_v and L = log sum_v exp((x_v - top) / temperature):
 *   logp[t]     = (x_id - top) / temperature - L     log probability of token_ids[t]   [T]    f32
 *   entropy[t]  = - sum_v p_v log p_v                                                  [T]    f32
 *   stats[t]    = (top, L): what r3_token_logprobs_bwd needs                           [T,2]  f32
 *   top_ids[t]  = the n_top most probable tokens, descending, ties to the lower id     [T,n_top] i32
 *   top_logp[t] = their log probabilities                                              [T,n_top] f32
 * Every output may be NULL (at least one is not); n_top <= 32 (R3_ERR_UNSUPPORTED beyond) and
 * <= V.  Logits and outputs need the alignment of their own type only.  One pass over the logits;
 * sums in float32; no workspace.
 *  - A negative token id marks a row that is not a response token (prompt, padding): its logits
 *    are not read, its outputs are 0 (top_ids -1).  An id >= V is treated the same and reported as
 *    R3_DEV_BAD_INDEX.  token_ids may be NULL when logp is: then every row counts.
 *  - Masked logits may be -inf or the type's lowest value.  A row of -inf alone has logp and
 *    top_logp -inf, entropy 0, stats (-inf, 0) and the first n_top ids; a row that holds NaN or
 *    +inf has no distribution: its outputs are NaN and its top_ids -1. */
r3_status r3_token_logprobs(const r3_logits* shape, const void* logits, const void* token_ids,
                            float* logp, float* entropy, float* stats, int32_t n_top,
                            int32_t* top_ids, float* top_logp, int32_t* dev_status, void* stream);

/* Gradient of a loss with dlogp = dL/dlogp [T] f32 (or NULL) and dentropy = dL/dentropy [T] f32 (or
 * NULL; then entropy [T] of the forward is not needed either) with respect to the logits:
 *   dlogits[t,v] = ( dlogp (1[v = id] - p_v) - dentropy p_v (log p_v + entropy) ) / temperature
 * with p from the logits and the forward's stats.  dlogits has the logits' dtype and row stride
 * ld_out >= V; columns from V on are left as they were.  It may be the logits' own buffer (with
 * ld_out = ld).  Every element of the V columns is written: rows with a negative token id (or one
 * >= V, reported) and rows of -inf alone get zeros. */
r3_status r3_token_logprobs_bwd(const r3_logits* shape, const void* logits, const void* token_ids,
                                const float* stats, const float* entropy, const float* dlogp,
                                const float* dentropy, void* dlogits, int64_t ld_out,
                                int32_t* dev_status, void* stream);

/* ---- policy loss (an extension: what stands between r3_token_logprobs and r3_token_logprobs_bwd) -- */

enum { R3_RATIO_TOKEN = 0, R3_RATIO_SEQUENCE = 1 };    /* a ratio per token, or one per sequence */
enum { R3_REDUCE_TOKEN = 0, R3_REDUCE_SEQUENCE = 1 };  /* mean over tokens, or over sequences' means */

/* T packed tokens of S sequences.  advantages are [T] (adv_per_token) or [S].  0 <= clip_low <= 1,
 * clip_high >= 0 (infinite: no border), dual_clip 0 (none) or above 1, infer_cap above 0 (infinite: none).
 * denominator 0: counted by the call. */
typedef struct {
    int32_t T, S;
    int32_t ratio, reduce, adv_per_token;
    double clip_low, clip_high, dual_clip, infer_cap, kl_coef, entropy_coef, denominator;
} r3_policy;

/* Clipped policy loss and its gradients, in one call.  Token t of sequence i, d = logp - logp_old (with
 * R3_RATIO_SEQUENCE the mean of that over the sequence's tokens), rho = exp(d), A the advantage:
 *   w     = min(exp(logp_old - logp_infer), infer_cap)              1 without logp_infer
 *   term  = -w min(rho A, min(max(rho, 1 - clip_low), 1 + clip_high) A);  with a dual clip, for A < 0, at
 *           most -w dual_clip A
 *   kl    = exp(x) - 1 - x,  x = logp_ref - logp                    0 without logp_ref
 *   loss  = sum_t weight_t (term + kl_coef kl - entropy_coef entropy)
 *   weight_t = 1 / D (R3_REDUCE_TOKEN, D = number of tokens) or 1 / (n_i D) (R3_REDUCE_SEQUENCE, n_i = the
 *              sequence's tokens, D = sequences that have any); a denominator > 0 stands in for D (a batch
 *              that is taken in parts, or over several ranks)
 *   dlogp = dloss dL/dlogp,  dentropy = dloss dL/dentropy           dloss: [1] on the device, NULL = 1
 * logp, logp_old [T]; logp_infer, logp_ref, entropy [T] or NULL; all float32.  w, logp_old and the masks are
 * constants.  A token counts where it belongs to a sequence and mask (uint8 [T], NULL = all) is not 0: the
 * others' values are not used, their gradients are 0.  cu_seqlens [S+1] int32 (device), ascending from 0 to at most T:
 * tokens behind its last entry belong to no sequence; NULL with S = 1: one sequence of all tokens.
 * Outputs: loss [1]; dlogp [T] or NULL; dentropy [T] (only with entropy) or NULL; metrics [3] or NULL = the
 * weighted sums of term, kl and entropy; counts [3] int32 or NULL = tokens, tokens beyond a border (that take
 * no policy gradient), tokens whose w is the cap.  dlogp may be logp's buffer, dentropy entropy's.
 *  - Borders are decided on d in 64 bits; on a border a token counts as inside.  Sums run in float64, in an
 *    order that depends on T, S and cu_seqlens alone.
 *  - What is not finite follows the formulas and stays with its token (with R3_RATIO_SEQUENCE: its
 *    sequence) and the loss; an advantage of 0 makes the term 0 whatever the ratio is, and a part with
 *    coefficient 0 is only reported in metrics.
 *  - cu_seqlens that do not ascend or leave [0, T] are reported as R3_DEV_BAD_INDEX (results undefined, nothing is accessed
 *    out of range).  T = 0 or no counting token: the loss is 0.
 * workspace: r3_policy_loss_workspace_bytes(config). */
size_t r3_policy_loss_workspace_bytes(const r3_policy* config);
r3_status r3_policy_loss(const r3_policy* config, const float* logp, const float* logp_old,
                         const float* advantages, const int32_t* cu_seqlens, const uint8_t* mask,
                         const float* logp_infer, const float* logp_ref, const float* entropy,
                         const float* dloss, float* loss, float* dlogp, float* dentropy, float* metrics,
                         int32_t* counts, void* workspace, size_t ws_bytes, int32_t* dev_status,
                         void* stream);

/* ---- balance loss of the routers (an extension; the paper trains without one) ---------------------- */

typedef struct {
    double balance_coef, z_coef;
    int32_t accumulate;       /* 1: the gradient is added to dlogits */
    int32_t counts_given;     /* 1: counts are read (those of a larger batch, say), not formed from idx */
} r3_balance;

/* Balance and z loss of L blocks' routers with their gradient, in one call.  Over the N tokens that count,
 * with p_t the softmax of logits[l,t,.] over all E experts and counts[l,i] = how often the record idx[l,t,.]
 * holds expert i:
 *   f_i = E counts_i / sum_j counts_j
 *   loss[l,0] = sum_i f_i (1/N) sum_t p_ti            1 where all experts are used alike
 *   loss[l,1] = (1/N) sum_t (log sum_i exp logits[l,t,i])^2
 *   dlogits   = balance_coef p_ti (f_i - sum_j f_j p_tj) / N + 2 z_coef (log sum exp) p_ti / N
 * (the gradient of balance_coef loss[l,0] + z_coef loss[l,1]; the counts are constants).
 * This gradient is dense, it has E columns, where the replay gate's has K: what takes it further are the caller's
 * own two products, dw_router += dlogits^T x and dx += dlogits W_r.  r3_input_grad_finish reads the recorded
 * experts' columns alone, and the backward chains (r3_replay_layer_train, r3_replay_stack_train,
 * r3_normed_stack_train) form dx and dw_router from the gate's gradient within the call: added to the dlogits that
 * they return it changes neither.  A chain over several blocks neither returns its inner inputs nor takes a gradient
 * at them, so blocks trained with this loss are chained by the caller, one r3_replay_layer_train each.
 * logits [L,T,E] f32; idx [L,T,K] idx_type (may be NULL with counts_given); mask uint8 [T] or NULL: tokens
 * that do not count have 0 there, and their logits and record are not used; counts [L,E] int32, written, may be NULL (with
 * counts_given: read); loss [L,2] f32; dlogits [L,T,E] f32 or NULL (may be the logits' buffer), every
 * element written (tokens that do not count: 0, or left as they are with accumulate).  Only T, E, K and idx_type of
 * the shape matter.  E <= 1024 and T <= 2^30 (R3_ERR_UNSUPPORTED beyond).  Sums run in an order that depends on the shape
 * alone.  dev_status: R3_DEV_BAD_INDEX for an index >= E (not counted).
 *  - A logit of -inf has p = 0; a token with no other logit counts in N and adds nothing.  A token with NaN or +inf
 *    makes its own gradient and its block's losses NaN.  Any finite logit is one, the type's lowest included (a
 *    token that holds nothing else chooses evenly; its z loss may pass float32's range).
 *  - No token that counts: losses 0.
 * workspace: r3_balance_loss_workspace_bytes(shape, L). */
size_t r3_balance_loss_workspace_bytes(const r3_shape* shape, int32_t L);
r3_status r3_balance_loss(const r3_shape* shape, int32_t L, const r3_balance* config,
                          const float* logits, const void* idx, const uint8_t* mask, int32_t* counts,
                          float* loss, float* dlogits, void* workspace, size_t ws_bytes,
                          int32_t* dev_status, void* stream);

/* ---- training/inference discrepancy measures (Sections 3.1 and 3.2) -------------------------- */

/* Eq. (kl), the k3 estimate of KL(pi_train || pi_infer), and Eq. (etdf), the Extreme Token
 * Distribution Function, over n response tokens:
 *   *kl_out       = (1/n) sum_t [ r_t - 1 - log r_t ],   r_t = p_train[t] / p_infer[t]   (float64)
 *   counts_out[i] = #{ t : max(r_t, 1/r_t) > taus[i] }   (so F(taus[i]) = counts_out[i] / n)
 * p_train, p_infer [n] float32 probabilities of the sampled tokens (positive); taus [n_tau]
 * float32 (device), n_tau <= 16; kl_out [1] float64 and counts_out [n_tau] int64 (device).
 * Each k3 term is formed in float32 by a cancellation-free expression of (p_train - p_infer) /
 * p_infer (relative error below 1e-5, typically 1e-7) and the terms are summed in float64 in a
 * fixed order (reproducible); the threshold decision is taken on float32 ratios.  workspace: r3_prob_discrepancy_workspace_bytes(n). */
size_t r3_prob_discrepancy_workspace_bytes(int64_t n);
r3_status r3_prob_discrepancy(const float* p_train, const float* p_infer, int64_t n,
                              const float* taus, int32_t n_tau, double* kl_out,
                              int64_t* counts_out, void* workspace, size_t ws_bytes, void* stream);

/* Section 3.2, router-level and token-level comparison of two routing records rec_a, rec_b
 * [L, T, K] (shape->T, K, E, idx_type; K <= 32; each (layer, token) holds K distinct experts, in
 * any slot order):
 *   diff[l,t]        = K - |{rec_a[l,t,.]} & {rec_b[l,t,.]}|   differing expert choices of a router
 *   hist[v]          = number of routers (l,t) with diff = v                 [K+1] int64
 *   token_choices[t] = sum_l diff[l,t]                                       [T]   int32
 *   token_routers[t] = number of layers l with diff[l,t] > 0                 [T]   int32
 * diff_out [L,T] uint8 may be NULL.  All outputs are exact integers. */
r3_status r3_record_diff(const r3_shape* shape, int32_t L, const void* rec_a, const void* rec_b,
                         uint8_t* diff_out, int32_t* token_choices, int32_t* token_routers,
                         int64_t* hist, void* stream);

/* Section 3.2, sequence-level comparison: seq_sum[s] = sum of token_routers over the tokens
 * [cu_seqlens[s], cu_seqlens[s+1]) of sequence s; the paper's mean difference per token of a
 * sequence is seq_sum[s] / length.  cu_seqlens [S+1] int32 (device), seq_sum [S] int64. */
r3_status r3_sequence_diff(const int32_t* token_routers, const int32_t* cu_seqlens, int32_t S,
                           int64_t* seq_sum, void* stream);

/* ---- routing-record store (Section 4.2: router masks cached with the prefix KV cache) --------- */

/* Records are kept in pages of `page_tokens` tokens, laid out [page][layer][token in page][slot]
 * (r3_record_page_bytes per page) in a device buffer `pages` of n_pages pages owned by the
 * caller.  A sequence is the list of its page numbers: row b of block_table [B, max_pages] int32
 * (device).  Two sequences that share a prefix list the same pages for it, which is how cached
 * masks are reused without recomputation (Section 4.2).  shape gives K and idx_type.
 *
 * r3_record_append (inference side): rec_new [L, N, K] holds the records of N new tokens, packed
 * sequence after sequence (cu_new [B+1]); the tokens of sequence b go to positions seq_pos0[b],
 * seq_pos0[b]+1, ... of that sequence.  Multi-turn use appends again to the same sequence.
 * r3_record_gather (training side): out [L, T, K] receives the records of positions 0 ..
 * len_b - 1 of every sequence, packed in the order of cu_seqlens [B+1] - the record that
 * r3_replay_layer / r3_replay_blocks take.
 * Both copy bytes (bit-exact).  dev_status (optional): R3_DEV_BAD_INDEX when a position has no
 * page (table entry < 0, >= n_pages, or beyond max_pages); that record is skipped. */
size_t r3_record_page_bytes(const r3_shape* shape, int32_t L, int32_t page_tokens);
r3_status r3_record_append(const r3_shape* shape, int32_t L, int32_t page_tokens, int32_t n_pages,
                           void* pages, const int32_t* block_table, int32_t max_pages,
                           const int32_t* seq_pos0, const int32_t* cu_new, int32_t B,
                           const void* rec_new, int32_t N, int32_t* dev_status, void* stream);
r3_status r3_record_gather(const r3_shape* shape, int32_t L, int32_t page_tokens, int32_t n_pages,
                           const void* pages, const int32_t* block_table, int32_t max_pages,
                           const int32_t* cu_seqlens, int32_t B, void* out, int32_t T,
                           int32_t* dev_status, void* stream);

/* Host-side bookkeeping of the pages (no device work; all pointers are HOST pointers; the pool
 * allocates host memory only, freed by r3_pagepool_destroy).  Not thread-safe.
 *   match   : the pages of the longest already stored whole-page prefix of token_ids (use counts
 *             go up); returns how many pages matched - their records need not be produced again
 *   alloc   : n unused pages (use count 1), R3_ERR_OUT_OF_PAGES if fewer are free
 *   publish : makes every full page of a sequence (token_ids = the n_tokens ids whose records the
 *             table's pages hold) findable by later match calls; a prefix is indexed once
 *   release : use counts go down; a page nobody uses leaves the index and becomes free
 * A page is identified by a chained 64-bit hash of all token ids up to its end, and a match also
 * compares the page's own ids: distinct prefixes are confused only on a hash collision. */
typedef struct r3_pagepool r3_pagepool;
r3_pagepool* r3_pagepool_create(int32_t n_pages, int32_t page_tokens);
void r3_pagepool_destroy(r3_pagepool* pool);
int32_t r3_pagepool_free_pages(const r3_pagepool* pool);
int32_t r3_pagepool_match(r3_pagepool* pool, const int32_t* token_ids, int32_t n_tokens,
                          int32_t* pages_out, int32_t max_pages);
r3_status r3_pagepool_alloc(r3_pagepool* pool, int32_t n, int32_t* pages_out);
r3_status r3_pagepool_publish(r3_pagepool* pool, const int32_t* token_ids, int32_t n_tokens,
                              const int32_t* table, int32_t n_table);
r3_status r3_pagepool_release(r3_pagepool* pool, const int32_t* table, int32_t n);

/* ---- self-test of the error path (the paper has no counterpart) ---------------------------------
 *
 * The tensor-core kernels wait on shared-memory barriers for their copies and MMAs; every such
 * wait is bounded, and a wait that runs out raises an abort flag in its CTA, writes
 * R3_DEV_TIMEOUT to dev_status and lets the kernel drain and return (see "General rules").  In a
 * healthy run that path never executes.  r3_selftest_bounded_wait runs it on purpose in a
 * harmless form: one 32-thread CTA waits, with the library's own wait routine and a limit of
 * `limit_clocks` SM clocks (1 .. 2e9, else R3_ERR_INVALID_ARG), on a barrier of its own that nothing
 * signals - no copy is in flight and no tensor memory is held.  Afterwards dev_status (optional)
 * holds R3_DEV_TIMEOUT and out [4] int32 (device) = {the wait's return value (0 = gave up), the
 * abort flag (1), clocks spent waiting (saturated), the return value of a second wait entered
 * while the CTA was already aborting (0)}.  The context stays usable: the next call is an
 * ordinary one. */
r3_status r3_selftest_bounded_wait(int64_t limit_clocks, int32_t* dev_status, int32_t* out,
                                   void* stream);

#ifdef __cplusplus
}
#endif
#endif /* R3_H_ */
