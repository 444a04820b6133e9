/*
 * hla.h - C ABI of the B200 (sm_100a) Hadamard Linear Attention operator.
 *
 * The operator is the linear-time form of HLA (paper Section 4.2, Lemma 4.1 and
 * Theorem 4.2, the normaliser paragraph after it, Algorithm 1 steps 4-5 and the
 * 2-/3-factor einsum listings of the appendix):
 *
 *     q_i   = phi_q(Q_i),   k^f_j = phi_{k_f}(K_j),  f = 1..F      (Algorithm 1 step 4)
 *     T_k[j] = k^1_j (x) ... (x) k^F_j,   T_q[i] = q_i (x) ... (x) q_i     in R^P, P = d_phi^F
 *     C = sum_j T_k[j] v_j^T  (P x d),    z = sum_j T_k[j]               (state build)
 *     eta_i = T_q[i] . z,    o_i = (T_q[i]^T C) / (eta_i + eps)          (readout + normaliser)
 *
 * which equals row-normalising A = (.)_f phi_q(Q) phi_{k_f}(K)^T (Eq. "hla") and
 * multiplying by V.  The backward entry point returns the gradients of
 * sum(dO * O) with respect to the inputs.
 *
 * General rules
 *   - All tensor pointers are DEVICE pointers, contiguous, innermost dimension
 *     last, 16-byte aligned.  The caller owns every buffer, including the
 *     workspace and the phi weights; the library allocates no device memory and
 *     borrows pointers only for the work it enqueues.
 *   - hla_ctx is host memory owned by the library (hla_create / hla_destroy).
 *   - hla_forward / hla_backward only enqueue work on `cuda_stream` (a
 *     cudaStream_t passed as void*; NULL = default stream) and return without
 *     synchronising.  They never throw, abort or print: every failure is a
 *     return code, and arguments are validated before anything is launched.
 *   - Device-side waits are bounded; a wait that runs out makes the kernel
 *     record a code in the workspace and return.  hla_last_device_status reads it.
 *     Each wait gives up after two seconds, and the warps of a block that depend
 *     on one another give up one after the other, so a launch that has timed out
 *     can take several times two seconds to return.
 *   - One ctx must not be used from two host threads at once.  This holds for the contexts of all
 *     operators below (hla_heads, hla_adamw, hla_scan), and calls that share a workspace, those
 *     of captured graphs too, have to follow one another on the device.
 */
#ifndef HLA_H_
#define HLA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hla_ctx hla_ctx;

typedef enum {
    HLA_OK = 0,
    HLA_ERR_INVALID_ARG = 1,   /* null / misaligned pointer, non-positive size, bad enum   */
    HLA_ERR_UNSUPPORTED = 2,   /* valid request outside the supported set (see hla_config)  */
    HLA_ERR_WORKSPACE = 3,     /* workspace smaller than hla_workspace_bytes()              */
    HLA_ERR_CUDA = 4,          /* a CUDA runtime/driver call failed                        */
    HLA_ERR_DEVICE_TIMEOUT = 5,/* a bounded device-side wait expired (results are invalid)  */
    HLA_ERR_NO_MEMORY = 6      /* host memory for the context could not be obtained          */
} hla_status;

typedef enum { HLA_BF16 = 0, HLA_F32 = 1 } hla_dtype;

typedef enum {
    HLA_PHI_MLP = 0, /* Q, K are raw per-head tensors [B,H,N,d]; the library applies phi_q, phi_k1..F  */
    HLA_PHI_NONE = 1 /* Q is q_phi [B,H,N,d_phi] fp32, K is k_phi [B,H,F,N,d_phi] fp32 (the listings'
                        signature: features are given, must be >= 0 for the normaliser to make sense) */
} hla_phi_mode;

/*
 * Problem statement.  V, O, dO, dV (and Q, K, dQ, dK in HLA_PHI_MLP mode) are
 * [B,H,N,d] in `dtype`.  Features (HLA_PHI_NONE inputs and their gradients) are
 * always fp32.  Supported set: F in {1,2,3,4}, d_phi^F <= 256, d <= 128 and
 * d % 4 == 0.  dtype bf16 with d in {64,128}, (F, d_phi) = (3, 6) or
 * (2, 12) - the paper's two variants - and B*H*N < 2^31 runs on the tensor-core
 * kernels; everything else in the supported set runs on the fp32 SIMT kernels.
 * causal = 1 (Section 4.4 "Causal Attention, Decay Factors and Sequential
 * Updates": token i sees the tokens j <= i, itself included, and the normaliser
 * sums the same entries, o_i = sum_{j<=i} A_ij v_j / (sum_{j<=i} A_ij + eps))
 * is supported for the 3-factor tensor-core set only (bf16, d in {64,128},
 * F = 3, d_phi = 6), forward and backward; any other combination with
 * causal = 1 is HLA_ERR_UNSUPPORTED.  Decay factors (a non-binary mask) are
 * not defined by the paper and not supported.
 */
typedef struct {
    int32_t B, H, N, d;
    int32_t F;        /* number of Hadamard factors; 0 -> 3 (the paper's main model)          */
    int32_t d_phi;    /* feature width; 0 -> 6 if F == 3, 12 if F == 2 (appendix "Defining phi") */
    int32_t phi;      /* hla_phi_mode                                                          */
    int32_t dtype;    /* hla_dtype                                                             */
    float eps;        /* added to the normaliser, o = num / (eta + eps); <= 0 -> 1e-6          */
    int32_t n_splits; /* token splits of the state build per head; 0 -> chosen from the SM count */
    int32_t causal;   /* 0: every token sees every token; 1: token i sees tokens j <= i          */
    int32_t value_mod; /* 1: the workspace also holds the scratch of hla_value_mod_forward / _backward (bf16 with
                          d in {64,128} only; HLA_ERR_UNSUPPORTED otherwise); 0: those calls are refused            */
} hla_config;

/*
 * One feature network (appendix "Defining phi"): feat = ReLU(W2^T GELU(W1^T x + b1) + b2),
 * the erf form of GELU (the tensor-core kernels evaluate its normal CDF with an
 * error below 4e-4 and its derivative with an error below 1.3e-3, both under the bf16
 * rounding of the hidden layer).  Device pointers in the ctx dtype: W1 [d][d] (input index
 * first), b1 [d], W2 [d][d_phi], b2 [d_phi].  One set per map, shared by all
 * batches and heads.
 */
typedef struct {
    const void *W1, *b1, *W2, *b2;
} hla_mlp;

/*
 * One value-modulation network (Section 4.5 "Value Modulation"; appendix "Defining phi"):
 *     phi_v(x) = W2^T GELU(W1^T LN(x) + b1) + b2,   LN(x) = (x - mean) / sqrt(var + 1e-5) * ln_g + ln_b  over the d channels
 * (two Linear layers of width d, no final activation; the paper only says that these maps use a LayerNorm - it is read
 * as acting on the input of the map).  Device pointers in the ctx dtype: ln_g [d], ln_b [d], W1 [d][d] (input index
 * first), b1 [d], W2 [d][d], b2 [d]; W1 and W2 16-byte aligned.
 */
typedef struct {
    const void *ln_g, *ln_b, *W1, *b1, *W2, *b2;
} hla_vmlp;

/*
 * Where hla_backward_weights puts the gradients of one feature network: fp32 device buffers with the shapes of the
 * weights, dW1 [d][d], db1 [d], dW2 [d][d_phi], db2 [d_phi], 16-byte aligned.  The call overwrites them.
 */
typedef struct {
    void *dW1, *db1, *dW2, *db2;
} hla_mlp_grad;

/* Byte offsets of the regions of the workspace that outlive a call (for
 * checking and for callers that want the state).  A region that the
 * configuration does not use has offset (size_t)-1. */
typedef struct {
    size_t status;   /* int32[16]  device status words                                   */
    size_t qf;       /* fp32 [B,H,N,d_phi]     features phi_q(Q)        (HLA_PHI_MLP)   */
    size_t kf;       /* fp32 [B,H,F,N,d_phi]   features phi_kf(K)       (HLA_PHI_MLP)   */
    size_t state;    /* fp32 [B,H,state_rows,state_ld]  columns 0..d-1 = C, column d = z.  state_rows = P = d_phi^F
                        on the SIMT path.  The tensor-core path keeps the state folded over the permutation
                        symmetry of the query tensor q (x) q (x) q: row m = (a <= b <= c) in lexicographic order
                        holds the sum of C over the distinct permutations of (a,b,c); 56 rows for F = 3, d_phi = 6 */
    size_t eta;      /* fp32 [B,H,N]           normaliser before eps                    */
    size_t dstate;   /* fp32 [B,H,state_rows,state_ld]  gradient of the loss w.r.t. that state (after hla_backward) */
    size_t dqf;      /* fp32 [B,H,N,d_phi]     feature gradients        (HLA_PHI_MLP)   */
    size_t dkf;      /* fp32 [B,H,F,N,d_phi]                            (HLA_PHI_MLP)   */
    int32_t state_ld; /* row stride of state / dstate in floats (>= d+1)                */
    int32_t state_rows;
    int32_t n_splits; /* the split count in use                                          */
    int32_t tensor_core; /* 1 if this configuration runs the tcgen05 kernels              */
} hla_ws_layout;

/* Validates the configuration and creates a context.  *out is NULL on failure. */
hla_status hla_create(const hla_config *cfg, hla_ctx **out);

/* HLA_PHI_MLP only: remembers the weight pointers (phi_k points to F entries).
 * The weights must stay valid and unchanged while the ctx is used. */
hla_status hla_set_phi(hla_ctx *ctx, const hla_mlp *phi_q, const hla_mlp *phi_k);

/* Bytes of caller-provided device scratch that forward and backward need. */
size_t hla_workspace_bytes(const hla_ctx *ctx);

hla_status hla_workspace_layout(const hla_ctx *ctx, hla_ws_layout *out);

/*
 * Forward: O = HLA(Q, K, V).  Leaves the features, the state (C, z) and eta in
 * the workspace for a later hla_backward.  With causal = 1 the state left in the
 * workspace is the one after the last token (Eq. "seq.updates": C^N) and eta_i
 * is the masked row sum.  The workspace must be 256-byte
 * aligned and at least hla_workspace_bytes() long.
 */
hla_status hla_forward(hla_ctx *ctx, const void *Q, const void *K, const void *V, void *O,
                       void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Sequential updates (Section 4.4, Eq. "seq.updates": C^i = C^{i-1} + T_{k_i} (x) v_i; the context tensor is the state of
 * the sequence).  Contexts created with causal = 1 only.  With carry = 1 every following hla_forward on a workspace
 * starts from the state (C, z) that the previous hla_forward left in that workspace instead of from zero, and leaves
 * the updated state there: a sequence handed over in chunks of N tokens per call gives the outputs of one causal pass
 * over the concatenation (the state is carried in fp32).  The first chunk of a sequence is run with carry = 0 (or on a
 * workspace whose state region the caller has zeroed; hla_workspace_layout gives its offset and size).  hla_backward is
 * HLA_ERR_UNSUPPORTED while carry = 1.  HLA_ERR_INVALID_ARG for a context without the mask or a value other than 0, 1.
 */
hla_status hla_set_carry(hla_ctx *ctx, int carry);

/*
 * Backward of the forward that last wrote `workspace` (same Q, K, V, O; the
 * workspace untouched in between): dQ, dK, dV = d sum(dO * O) / d(Q, K, V).
 * In HLA_PHI_NONE mode dQ, dK are fp32 feature gradients with the shapes of Q, K.
 * In HLA_PHI_MLP mode on the tensor-core kernels dQ and dK must be 32-byte aligned
 * (their rows leave the kernel as 32-byte stores); anything else is refused with
 * HLA_ERR_INVALID_ARG before a launch.
 * Gradients with respect to the phi weights are not computed by this call.
 * In HLA_PHI_MLP mode dQ may be the buffer of Q, V, O or dO and dK that of K; with
 * features given, dK may be that of K and, without the mask, dQ that of Q.  (Such a call runs
 * its kernels one after the other where they would otherwise run side by side, and
 * hla_backward_weights needs the Q and K that it overwrites.)
 * With causal = 1, O must be the output of that forward (the call reads it for
 * dO_i . o_i; without the mask it is not read) and V, O, dO, dV must be 16-byte
 * aligned like every tensor.
 */
hla_status hla_backward(hla_ctx *ctx, const void *Q, const void *K, const void *V, const void *O,
                        const void *dO, void *dQ, void *dK, void *dV,
                        void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * The two passes in two halves, for a sequence whose N tokens are split over several devices (one context per device,
 * each created with its own share of N).  Theorem 4.2's state C = sum_j T_k[j] v_j^T and the key-side sum z are sums
 * over the tokens, so the shards' states add: between the two halves of a pass the caller adds the state region of the
 * workspaces of all shards (fp32; hla_workspace_layout gives `state` / `dstate`, state_rows and state_ld; one all-reduce
 * of B*H*state_rows*state_ld floats) and leaves the sum in every workspace.
 *   forward:   hla_forward_keys (feature maps of K, state of the shard)  ->  sum of `state` over the shards  ->
 *              hla_forward_queries (feature map of Q, readout against the summed state, O of the shard's tokens)
 *   backward:  hla_backward_queries (query pass: dQ-side gradients, gradient state of the shard)  ->  sum of `dstate`
 *              over the shards  ->  hla_backward_keys (key pass on the summed gradient state, then the phi backward:
 *              dQ, dK, dV of the shard's tokens)
 * Each half takes the arguments of the whole call and uses those it needs (the key half of the forward K and V, the
 * query half Q and O; both halves of the backward the full list).  With a single shard and no sum in between the two
 * halves give the results of hla_forward / hla_backward bit for bit.  Tensor-core set without the mask only:
 * HLA_ERR_UNSUPPORTED on the fp32 SIMT path and for causal = 1 (a causal pass would need an exclusive scan of the
 * shards' states instead of their sum).  The library itself never communicates between devices.
 */
hla_status hla_forward_keys(hla_ctx *ctx, const void *K, const void *V, void *workspace, size_t workspace_bytes, void *cuda_stream);
hla_status hla_forward_queries(hla_ctx *ctx, const void *Q, void *O, void *workspace, size_t workspace_bytes, void *cuda_stream);
hla_status hla_backward_queries(hla_ctx *ctx, const void *Q, const void *K, const void *V, const void *O,
                                const void *dO, void *dQ, void *dK, void *dV,
                                void *workspace, size_t workspace_bytes, void *cuda_stream);
hla_status hla_backward_keys(hla_ctx *ctx, const void *Q, const void *K, const void *V, const void *O,
                             const void *dO, void *dQ, void *dK, void *dV,
                             void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Gradients of sum(dO * O) with respect to the weights of the feature networks (Section 5, "Training Details": the
 * paper trains the phi maps with the rest of the model; Algorithm 1 step 4 defines where they act).  HLA_PHI_MLP
 * contexts on the tensor-core kernels only (HLA_ERR_UNSUPPORTED otherwise).  Call it after hla_backward with the
 * same Q, K and the same workspace: it reads the features the forward kept and the feature gradients the backward
 * left there, recomputes the hidden layer, and sums over all batches, heads and tokens (one weight set per map is
 * shared by all of them).  dphi_q receives the gradients of phi_q, dphi_k points to F entries for phi_k1..F; either
 * may be NULL to skip that side.  The sums are formed in a fixed order: results are bit-reproducible.
 */
hla_status hla_backward_weights(hla_ctx *ctx, const void *Q, const void *K, const hla_mlp_grad *dphi_q, const hla_mlp_grad *dphi_k,
                                void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Value modulation of the attention result (Section 4.5):  Out = T + phi_v1(T) (.) phi_v2(V), with T the output of
 * hla_forward and V its value input, both [B,H,N,d]; one weight set per map, shared by all batches and heads.
 * Contexts created with value_mod = 1 only.  hla_set_phi_v remembers the weight pointers (they must stay valid).
 * The forward keeps nothing for the backward; the backward recomputes both maps and returns
 *     dT = dOut + J1^T (dOut (.) phi_v2(V)),     dV = J2^T (dOut (.) phi_v1(T))      (J: Jacobian of a map w.r.t. its input)
 * the gradients of sum(dOut * Out) with respect to T and V (weights fixed).  With accumulate_dV != 0 the V-side
 * gradient is added to what dV already holds (the dV that hla_backward wrote for the same step), else dV is overwritten.
 * Out, dT, dV must be 32-byte aligned.  Out may not alias T or V; dT may be the buffer of T, and dV that of V, T or dOut.  hla_value_mod_forward clears the device status words
 * like hla_forward does (read hla_last_device_status before it if the record of hla_forward matters); the backward
 * keeps them.  A whole step is then
 *     hla_forward -> hla_value_mod_forward;   hla_value_mod_backward -> hla_backward(dO = dT) with accumulate_dV = 0 and
 *     the two dV added by the caller, or hla_backward first and hla_value_mod_backward with accumulate_dV = 1.
 */
hla_status hla_set_phi_v(hla_ctx *ctx, const hla_vmlp *v1, const hla_vmlp *v2);
hla_status hla_value_mod_forward(hla_ctx *ctx, const void *T, const void *V, void *Out, void *workspace, size_t workspace_bytes,
                                 void *cuda_stream);
hla_status hla_value_mod_backward(hla_ctx *ctx, const void *T, const void *V, const void *dOut, void *dT, void *dV,
                                  int32_t accumulate_dV, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Forward without a caller-provided workspace (no counterpart in the paper: a
 * deployment aid).  Some callers of this library cannot obtain device memory
 * at the time they need the operator: a plug-in running inside a host
 * application that owns the allocator, a real-time loop that forbids
 * allocation after start-up, code that only receives the tensors it is
 * handed.  For them the library carries its own scratch: one array of
 * HLA_STATIC_WS_BYTES bytes that is part of the loaded module, so every GPU
 * that loads the library holds that much memory until the process exits.
 * This call computes exactly what hla_forward computes, with that array as the
 * workspace, and calls no memory-allocating routine.
 *
 *   - Contexts whose hla_workspace_bytes() exceeds HLA_STATIC_WS_BYTES are
 *     refused with HLA_ERR_WORKSPACE before anything is enqueued.  (The split
 *     count that n_splits = 0 stands for is lowered where the workspace would
 *     be too large for speed only.)
 *   - The first call on a device looks up the array's device address (with
 *     that device current) and remembers it; make that first call outside any
 *     stream capture.  Later calls on the same device only enqueue work.
 *   - All contexts and all calls share the one array, and it keeps what the
 *     previous call left in it.  Everything a call reads from it is written
 *     earlier in the same call (the status words are cleared at the start),
 *     so back-to-back calls on one stream are independent; two calls that can
 *     overlap on the GPU (different streams without an ordering between them)
 *     race on it and must not be made.
 *   - If `scratch_out` is not NULL it receives the array's device address:
 *     pass it as `workspace` to hla_last_device_status, to hla_backward (the
 *     state of the forward lives there), or add hla_workspace_layout offsets
 *     to read eta or the state.
 */
#define HLA_STATIC_WS_BYTES (16u * 1024u * 1024u)
hla_status hla_forward_static(hla_ctx *ctx, const void *Q, const void *K, const void *V, void *O,
                              void *cuda_stream, void **scratch_out);

/* Synchronises `cuda_stream`, reads the device status words of `workspace`
 * and returns HLA_OK, HLA_ERR_DEVICE_TIMEOUT or HLA_ERR_CUDA. */
hla_status hla_last_device_status(hla_ctx *ctx, const void *workspace, void *cuda_stream);

/*
 * Self-test of the failure path (no counterpart in the paper).  Every wait inside the kernels is bounded; this
 * call enqueues a one-block kernel that waits, with a 1 ms limit, on a barrier that nothing arrives at.  The wait
 * must run out, the kernel must return normally, and a following hla_last_device_status(ctx, workspace, stream)
 * must report HLA_ERR_DEVICE_TIMEOUT.  The status words are cleared by the next hla_forward.
 */
hla_status hla_selftest_bounded_wait(hla_ctx *ctx, void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Number of kernels the last hla_forward / hla_backward on this ctx launched. */
int32_t hla_last_launch_count(const hla_ctx *ctx);

/*
 * Optional per-kernel timing (no counterpart in the paper: a measurement aid).
 * While enabled, every kernel launch of hla_forward / hla_backward is bracketed
 * by CUDA events on the launching stream.  After the caller has synchronised
 * the stream, hla_timing_collect folds the recorded launches into per-kernel
 * totals (replacing earlier totals) and returns how many distinct kernels
 * there are; hla_timing_get returns entry i: a static name, the summed device
 * time in milliseconds and the number of launches.
 */
hla_status hla_timing_enable(hla_ctx *ctx, int32_t on);
int32_t hla_timing_collect(hla_ctx *ctx);
hla_status hla_timing_get(const hla_ctx *ctx, int32_t i, const char **name, double *total_ms, int64_t *launches);

hla_status hla_destroy(hla_ctx *ctx);

/*
 * Head preparation (Algorithm 1 steps 1-3: reshape to heads, rotary positions, scale), between a projection and
 * hla_forward.  Every row x of d channels (one head of one token) becomes
 *     y = s * R(theta) ( x / sqrt(mean(x^2) + eps) * w )
 * with the RMS norm (norm = 1) and the scale (s = q_scale) on q, the norm on k, and neither norm, rotation nor scale on v.
 * R turns the pairs of channels: pair p by theta = position[axis(p)] * inv_freq[p].  The first axis_width[0] / 2 pairs belong to axis
 * 0 (the time of a video, say), the next axis_width[1] / 2 to axis 1, and so on; channels behind the last axis do not turn.
 * HLA_PAIR_ADJACENT: pair p is the channels (2p, 2p+1).  HLA_PAIR_HALVES: the channels (p, p + R/2), R the sum of the
 * widths.  Where inv_freq is NULL, pair j of an axis of n pairs has inv_freq = theta^(-j/n).  Angles are reduced in 64 bits: positions
 * may be any int32.
 * Positions: with a grid (row-major, its product N), token n is at its place in the grid plus start.  Without one
 * (all of grid 0), or where a call is given `positions` (device int32 [B][N][n_axes], positions_batch_stride elements from one
 * batch to the next, 0 for positions shared by all), they are read.
 * Supported: d <= 128, rows and, for HLA_PAIR_HALVES, R in whole 16-byte pieces (d and R multiples of 8 in bf16, 4 in fp32),
 * B*H <= 65535, B*N <= 2^28.  Sums and rotations are formed in fp32 and rounded once.
 */
typedef struct hla_heads hla_heads;
typedef enum { HLA_PAIR_ADJACENT = 0, HLA_PAIR_HALVES = 1 } hla_pairing;
typedef struct {
    int32_t B, H, N, d;
    int32_t dtype;         /* hla_dtype of all tensors and norm weights                                   */
    int32_t pairing;       /* hla_pairing                                                                 */
    int32_t norm;          /* 1: q and k are RMS-normalised per row                                       */
    int32_t n_axes;        /* 0 (no rotation) to 3                                                        */
    int32_t axis_width[3]; /* channels that turn with each axis: even, their sum <= d                     */
    int32_t grid[3];       /* tokens along each axis, product N; all 0: every call is given positions     */
    int32_t start[3];      /* position of the grid's first token                                          */
    float eps;             /* 0 -> 1e-6                                                                   */
    float q_scale;         /* 0 -> 1                                                                      */
    double theta;          /* 0 -> 10000                                                                  */
    const double *inv_freq; /* HOST array of one value per pair, copied; NULL: from theta                 */
} hla_heads_config;

/* A tensor [B][N][H][d] whose rows of H*d elements are contiguous: strides in elements, in whole 16-byte pieces (a
 * projection [B][N][3][H][d] has token stride 3*H*d).  Rows do not share memory: either batches lie one behind another, or
 * every token's batches behind those of the token before ([N][B][H][d]). */
typedef struct {
    const void *data;
    int64_t batch_stride, token_stride;
} hla_rows;
typedef struct {
    void *data;
    int64_t batch_stride, token_stride;
} hla_rows_out;

hla_status hla_heads_create(const hla_heads_config *cfg, hla_heads **out);

/* Scratch of hla_heads_backward (0 without norm; only needed where it is asked for dwq or dwk). */
size_t hla_heads_workspace_bytes(const hla_heads *ctx);

/* q, k, v -> Q, K, V [B][H][N][d], each may be NULL together with its output.  wq, wk: norm weights [d] (norm = 1 only), NULL for
 * ones.  No output may lie within the memory that an input spans. */
hla_status hla_heads_forward(hla_heads *ctx, const hla_rows *q, const hla_rows *k, const hla_rows *v, const void *wq, const void *wk,
                             const int32_t *positions, int64_t positions_batch_stride, void *Q, void *K, void *V, void *cuda_stream);

/*
 * Gradients of sum(dQ Q + dK K + dV V): dq, dk, dv with strides of their own, and dwq, dwk (fp32 [d], overwritten; NULL: not wanted).
 * dq, dk, dv can be parts of one tensor that the projection's backward reads: of equal strides then, the larger a multiple of the
 * smaller.  dQ, dK, dV may be NULL together with their outputs.  q and k are only read with norm = 1 and are the inputs of the
 * forward.  The sums of dwq and dwk are formed in a fixed order.  dV alone moves a head-major tensor [B][H][N][d] to token-major rows,
 * as an output projection reads them.
 */
hla_status hla_heads_backward(hla_heads *ctx, const void *dQ, const void *dK, const void *dV, const hla_rows *q, const hla_rows *k,
                              const void *wq, const void *wk, const int32_t *positions, int64_t positions_batch_stride,
                              const hla_rows_out *dq, const hla_rows_out *dk, const hla_rows_out *dv, void *dwq, void *dwk,
                              void *workspace, size_t workspace_bytes, void *cuda_stream);
hla_status hla_heads_destroy(hla_heads *ctx);

/*
 * AdamW step over many tensors (the update of a training step: the feature networks whose gradients hla_backward_weights
 * leaves, and whatever else the model trains):
 *     g = grad_scale * min(1, max_norm / (norm + 1e-6)) * grad,      norm = |grad_scale| * || all grads ||_2     (max_norm > 0)
 *     m = beta1 m + (1 - beta1) g,    v = beta2 v + (1 - beta2) g^2
 *     param = param - rate * weight_decay * param - rate * (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps),  rate = lr * lr_mul
 * With max_norm > 0 a step whose norm is not finite changes no tensor; nor does one whose number, read on the device, is below 1.
 * Weights are fp32 or bf16, gradients fp32 or bf16, tensor by tensor.  fp32 weights may have a bf16 `copy`, rounded to nearest, for
 * the kernels that read them; bf16 weights are rounded up or down at random with the probability that keeps the mean.
 * HLA_STATE_F32: m, v fp32.  HLA_STATE_Q8: m, v are e4m3 codes (1 byte an element) with an fp32 scale for every 128
 * elements of a tensor (m_scale, v_scale; the last scale may stand for fewer), scale = max |x| / 448; rounded at random like bf16
 * weights, a positive second moment to a positive code.  A group whose largest entry is below 2^-100 is held as zeros; one with an
 * entry that is not finite has a scale that is no number.  Random numbers are a function of seed, step, and the places of tensor and
 * element: a step can be repeated bit for bit.  Zeros everywhere are the states before the first step.
 */
typedef struct hla_adamw hla_adamw;
typedef enum { HLA_STATE_F32 = 0, HLA_STATE_Q8 = 1 } hla_state_type;
typedef struct {
    void *param, *copy;          /* copy: bf16, with fp32 weights only; may be NULL                    */
    const void *grad;
    void *m, *v;
    void *m_scale, *v_scale;     /* fp32 [(n + 127) / 128], HLA_STATE_Q8 only                          */
    int64_t n;                   /* elements; 0: the tensor is passed over                             */
    float lr_mul;                /* 0 -> 1                                                             */
    float weight_decay;
    int32_t param_dtype, grad_dtype; /* hla_dtype                                                      */
} hla_adamw_tensor;
typedef struct {
    double beta1, beta2, eps;    /* 0 <= beta < 1, eps >= 2^-126 (HLA_STATE_Q8: 2^-50)                    */
    int32_t state;               /* hla_state_type                                                     */
    uint64_t seed;
} hla_adamw_config;
typedef struct {
    double lr;
    int64_t step;                /* the first step is 1                                                */
    const float *lr_device;      /* device scalar that is read instead of lr, or NULL                  */
    const int64_t *step_device;  /* device scalar that is read instead of step, or NULL: a captured step can be replayed with new values */
    float max_norm;              /* 0: no norm is taken; infinity: the norm is taken and nothing is clipped */
    float grad_scale;            /* 0 -> 1                                                             */
    float *norm;                 /* device scalar that receives the norm (max_norm > 0), or NULL; the three scalars and the workspace
                                    lie apart from the tensors of the list                             */
} hla_adamw_step_args;

/* The pointers (16-byte aligned) are remembered; nothing that a step writes may share memory with another tensor of the list. */
hla_status hla_adamw_create(const hla_adamw_config *cfg, const hla_adamw_tensor *tensors, int32_t n, hla_adamw **out);
/* Other gradients (same types and sizes) from the next step on: one pointer per tensor of the list. */
hla_status hla_adamw_set_grads(hla_adamw *ctx, const void *const *grads, int32_t n);
size_t hla_adamw_workspace_bytes(const hla_adamw *ctx);      /* only needed by steps with max_norm > 0 */
hla_status hla_adamw_step(hla_adamw *ctx, const hla_adamw_step_args *args, void *workspace, size_t workspace_bytes, void *cuda_stream);
hla_status hla_adamw_destroy(hla_adamw *ctx);

/*
 * Gated linear recurrence (Section 4.4 "Causal Attention, Decay Factors and Sequential Updates", for a state of one value per
 * channel): over the tokens of every sequence and for every channel
 *     h_t = a_t h_{t-1} + u_t,     a_t = exp(g_t) (HLA_GATE_LOG, g_t <= 0) or 1 / (1 + exp(-g_t)) (HLA_GATE_SIGMOID),
 *     u_t = x_t, or (1 - a_t) x_t with convex = 1.
 * x, g [B][N][C] with strides (x and g may be parts of one projection); h, dh, dx, dg [B][N][C] contiguous and 16-byte aligned; states
 * h0, h_last, dh_last, dh0 are fp32 [B][C] and may be NULL (zeros; not wanted).  A sequence that arrives in pieces is continued by
 * passing the h_last of one call as the h0 of the next, the same buffer if wanted (not a part of it).  The state is carried in fp32, whatever the
 * dtype.  The backward returns the gradients of sum(dh h) + sum(dh_last h_last) with respect to x, g and h0; h is the output of
 * the forward.  x is only read there with convex = 1.  Outputs may not lie over inputs, but for dh0 over h0 or dh_last.
 */
typedef struct hla_scan hla_scan;
typedef enum { HLA_GATE_LOG = 0, HLA_GATE_SIGMOID = 1 } hla_gate;
typedef struct {
    int32_t B, N, C;
    int32_t dtype;                                   /* hla_dtype                              */
    int32_t gate;                                    /* hla_gate                               */
    int32_t convex;
    int64_t x_batch_stride, x_token_stride;          /* elements; 0: contiguous                */
    int64_t g_batch_stride, g_token_stride;
} hla_scan_config;
hla_status hla_scan_create(const hla_scan_config *cfg, hla_scan **out);
/*
 * Scratch of both calls: HLA_SCAN_STATUS_BYTES, and more where a long sequence of few channels runs in parts; only these need it.  A call that
 * needs none can be given none (NULL, 0), or another one of at least HLA_SCAN_STATUS_BYTES, 256-byte aligned, for its record:
 * blocks that share a sequence wait for one another for two seconds at most; where a wait runs out the outputs from there on are not numbers, and
 * the first bytes of the workspace record it.  hla_scan_last_device_status synchronises `cuda_stream`, reads the record, takes it back and returns
 * HLA_OK, HLA_ERR_DEVICE_TIMEOUT (since it was last read) or HLA_ERR_CUDA.  The record is one value that memory does not hold by chance; memory that
 * was the workspace of a call that timed out is zeroed before it is one again.  hla_scan_selftest_bounded_wait enqueues a kernel that
 * waits for a millisecond for what never comes, records it and returns.
 */
#define HLA_SCAN_STATUS_BYTES 256u
size_t hla_scan_workspace_bytes(const hla_scan *ctx);
hla_status hla_scan_forward(hla_scan *ctx, const void *x, const void *g, const void *h0, void *h, void *h_last, void *workspace, size_t workspace_bytes,
                            void *cuda_stream);
hla_status hla_scan_backward(hla_scan *ctx, const void *x, const void *g, const void *h0, const void *h, const void *dh, const void *dh_last,
                             void *dx, void *dg, void *dh0, void *workspace, size_t workspace_bytes, void *cuda_stream);
hla_status hla_scan_last_device_status(hla_scan *ctx, void *workspace, void *cuda_stream);
hla_status hla_scan_selftest_bounded_wait(hla_scan *ctx, void *workspace, size_t workspace_bytes, void *cuda_stream);
hla_status hla_scan_destroy(hla_scan *ctx);

const char *hla_status_string(hla_status s);

#ifdef __cplusplus
}
#endif
#endif /* HLA_H_ */
