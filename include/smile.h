/*
 * libsmile: forward and backward pass of one SMILE bi-level routed
 * Mixture-of-Experts layer on one AMD MI355X (gfx950), as a C-ABI library of
 * hand-written HIP kernels.
 *
 * Method: "SMILE: Scaling Mixture-of-Experts with Efficient Bi-level Routing",
 * arXiv 2212.05191.  A token is routed to one of n groups by an inter router
 * and then to one of the m experts of that group by an intra router
 * (Section 3.2.1); its output is p_i * q_j * E_{i,j}(x) (Eq. 3); the layer
 * adds a two-term load-balancing loss (Eq. 4).  On one GPU the paper's node /
 * GPU hierarchy is a logical two-level grouping: all N = n*m experts are
 * resident and the two All2All stages become one composed row permutation.
 *
 * General rules
 *   - Every tensor pointer is a DEVICE pointer owned by the caller, dense,
 *     row-major, 16-byte aligned.  The library reads/writes it only during the
 *     call's enqueued work and never frees or keeps it.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     All work is enqueued asynchronously on it; no call synchronises, and no
 *     call other than smile_create/smile_destroy allocates or frees memory.
 *   - Every function returns a smile_status; nothing throws or aborts.
 *     Argument checks happen on the host before anything is enqueued, so a
 *     non-OK status means no work was submitted (except SMILE_HIP_ERROR from a
 *     failed launch).
 *   - Notation: T tokens, d = d_model, F = d_ff, n = n_groups, m = m_local,
 *     N = n*m, flat expert id e = group*m + local, C = capacity (rows of each
 *     expert's buffer).  dtype is the storage type of x, router and expert
 *     weights, the expert buffers and y: 0 = fp32, 1 = bfloat16, 2 = IEEE half.
 *     Logits, probabilities, gates and the loss are always fp32; products of
 *     16-bit values accumulate in fp32 on the matrix cores.
 *   - Limits: T, d, F, n, m, C >= 1; d % 8 == 0 and F % 8 == 0 (for the 16-bit
 *     types: d % 64 == 0 and F % 64 == 0); n <= 1024, m <= 1024, N <= 4096;
 *     N*C*max(d,F) < 2^40 elements; N*C and T below 2^31 (T <= 2^30 with a
 *     group capacity).  n = 1 (or m = 1) gives the flat one-level top-1
 *     router of Section 2 (Eq. 1-2, k = 1).
 *   - Floating-point inputs must be finite; NaN/Inf give unspecified results.
 *   - Tuning switches (never needed in normal use; tests and sweeps set them): smile_create and
 *     smile_create_with_workspace read the environment variables SMILE_FFN_TILE (0-9: tile shape of
 *     the forward expert GEMMs; 6 names none: the library's choice), SMILE_TGEMM_TILE (0-4: tile shape of the gradient GEMMs),
 *     SMILE_FFN_PERSIST (0/1: plain or persistent grid of the GEMM kernels that have both) and SMILE_ROUTER_GRAD_MFMA (0: vector-ALU
 *     router-gradient kernels) ONCE and keep the values in the ctx; no other call looks at the
 *     environment.  They change which kernel variant runs, never a result beyond rounding order.
 *     The same two calls ask the runtime for the compute-unit count of the current device, which
 *     sizes the persistent GEMM grids of that ctx.
 */
#ifndef SMILE_H
#define SMILE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum smile_status {
    SMILE_OK = 0,
    SMILE_INVALID_ARG = 1,   /* NULL or misaligned pointer, NULL ctx/desc */
    SMILE_BAD_SHAPE = 2,     /* a size is out of range or violates a divisibility rule */
    SMILE_UNSUPPORTED = 3,   /* unknown dtype / activation, or a shape no kernel covers */
    SMILE_WORKSPACE = 4,     /* caller-supplied workspace too small or misaligned */
    SMILE_HIP_ERROR = 5      /* a HIP runtime call failed (allocation, launch) */
} smile_status;

enum { SMILE_DTYPE_F32 = 0, SMILE_DTYPE_BF16 = 1, SMILE_DTYPE_F16 = 2 };   /* F16: IEEE half, the paper's training precision (Section 4.1) */
enum { SMILE_ACT_RELU = 0, SMILE_ACT_GELU = 1 };   /* GELU is the exact erf form (Section 4.1) */

/* Static description of one layer; copied by smile_create. */
typedef struct smile_layer_desc {
    int32_t T;          /* tokens per call */
    int32_t d_model;
    int32_t d_ff;
    int32_t n_groups;   /* n: fan-out of the inter router (the paper's nodes) */
    int32_t m_local;    /* m: fan-out of the intra router (the paper's GPUs per node) */
    int32_t capacity;   /* C: rows per expert buffer, see smile_capacity */
    int32_t dtype;      /* SMILE_DTYPE_* */
    int32_t act;        /* SMILE_ACT_* */
    float alpha;        /* Eq. 4 coefficients */
    float beta;
    int32_t group_capacity;   /* Cg: rows of each group's first-hop buffer (Section 3.2.3); 0 = no limit */
} smile_layer_desc;

typedef struct smile_ctx smile_ctx;   /* opaque: a validated desc + device workspace */

/* Static string for a status code (never NULL). */
const char *smile_status_string(int32_t status);

/* Library version, e.g. "0.1.0". */
const char *smile_version(void);

/* Switch-style expert capacity for the "capacity factor" of Section 4.2:
 * ceil(cf * T / N), at least 1.  Host helper; returns -1 on invalid input. */
int32_t smile_capacity(int32_t T, int32_t N, double capacity_factor);

/* Host-only check of a desc against the limits above (no GPU needed). */
smile_status smile_validate_desc(const smile_layer_desc *desc);

/* Bytes of device workspace a ctx for `desc` needs (routing histograms and
 * partial sums, and the hidden activation h[N,C,F] between the two expert
 * GEMMs).  Host-only. */
smile_status smile_workspace_bytes(const smile_layer_desc *desc, size_t *bytes);

/* Create a ctx whose workspace the library allocates with hipMalloc on the
 * current device (freed by smile_destroy). */
smile_status smile_create(const smile_layer_desc *desc, smile_ctx **ctx);

/* Create a ctx on caller-owned device memory: `workspace` must be 256-byte
 * aligned, at least smile_workspace_bytes() long and must outlive the ctx.
 * Nothing is allocated on the device.  Calls on one ctx must not overlap. */
smile_status smile_create_with_workspace(const smile_layer_desc *desc, void *workspace, size_t bytes,
                                         smile_ctx **ctx);

/* Release a ctx (and its workspace if the library allocated it).  The caller
 * must have synchronised every stream that used it.  NULL is allowed. */
smile_status smile_destroy(smile_ctx *ctx);

/* Kernel timing, for benchmarks and profiles.  `events` is an array of 2*pairs hipEvent_t handles
 * (passed as void*, created by the caller with timing enabled, owned by the caller and alive until
 * detached).  While attached, every kernel that a later call on this ctx launches takes the next pair
 * (start, stop), which receives the begin and end timestamps of that kernel itself, so that
 * hipEventElapsedTime(start, stop) after synchronisation is the kernel's own duration without launch
 * gaps.  Each call starts again at pair 0; kernels beyond `pairs` (at most 32 are used) run untimed.
 * pairs = 0 detaches.  smile_kernel_timing_count: kernels that took a pair in the most recent call;
 * smile_kernel_timing_name: the kernel's name (a static string, "" out of range).  Results are
 * unchanged.  The array must not be in use by two threads at once. */
smile_status smile_kernel_timing(smile_ctx *ctx, void **events, int32_t pairs);
int32_t smile_kernel_timing_count(const smile_ctx *ctx);
const char *smile_kernel_timing_name(const smile_ctx *ctx, int32_t i);

/* Step 1 -- router logits r(x) = W_r x (Section 2, text before Eq. 1) for the
 * two tied routers of Section 3.2.1, both reading the same token vector:
 *   logits_inter[t,i] = sum_k x[t,k] * w_inter[i,k]      [T,n] fp32
 *   logits_intra[t,j] = sum_k x[t,k] * w_intra[j,k]      [T,m] fp32
 * x[T,d], w_inter[n,d], w_intra[m,d] in the ctx dtype; products accumulate in fp32. */
smile_status smile_gate_logits(smile_ctx *ctx, const void *x, const void *w_inter, const void *w_intra,
                               float *logits_inter, float *logits_intra, void *stream);

/* Steps 2-3 -- bi-level top-1 routing with capacity (Section 3.2.1; Eq. 1
 * read as a softmax; Section 3.2.2 for the statistics; Section 4.2 capacity).
 *   a[t,:] = logits_inter[t,:] + bias_inter            (one fp32 add, bias may be NULL)
 *   group_idx[t] = lowest index of max a[t,:];  p = softmax(a[t,:]);  p_top[t] = p[group_idx[t]]
 *   c[t,:] = logits_intra[t,:] + bias_intra[group_idx[t],:]   (bias_intra[n,m] may be NULL)
 *   local_idx[t] = lowest index of max c[t,:];  q = softmax(c[t,:]);  q_top[t] = q[local_idx[t]]
 *   gate[t] = p_top[t] * q_top[t]                      (Eq. 3)
 *   pos_in_group[t] = number of earlier tokens with the same group       (stage-1 position)
 *   rank = number of earlier tokens with the same (group, local)          (stage-2 position)
 *   slot[t] = rank if rank < C, else -1 (token dropped)
 *   With desc.group_capacity = Cg > 0 the first hop of Section 3.2.3 has a buffer of Cg rows per
 *   group as well: a token with pos_in_group[t] >= Cg is dropped there (slot -1) and is not counted
 *   in `rank` of later tokens; kept_count[e] is then min(tokens of e that passed the first hop, C).
 *   The counts and sums below ignore both kinds of drops.
 *   group_count[n], local_count[m] (summed over all groups), expert_count[N]: top-1 counts of all T
 *   tokens, before drops;  kept_count[e] = min(expert_count[e], C);
 *   p_sum[i] = sum_t p[t,i];  q_sum[j] = sum_t q[t,j]    (fp32)
 * Integer outputs are exact and independent of launch geometry; float sums are
 * accumulated in a fixed order, so repeated calls give identical bits. */
smile_status smile_route_bilevel(smile_ctx *ctx, const float *logits_inter, const float *logits_intra,
                                 const float *bias_inter, const float *bias_intra,
                                 int32_t *group_idx, int32_t *local_idx, int32_t *pos_in_group, int32_t *slot,
                                 float *gate, float *p_top, float *q_top,
                                 int32_t *group_count, int32_t *local_count, int32_t *expert_count,
                                 int32_t *kept_count, float *p_sum, float *q_sum, void *stream);

/* smile_route_bilevel for callers that cannot allocate device memory or create a ctx: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same kernels, same arguments
 * and bit-identical results; instead of a ctx it takes the layer description, and its scratch memory
 * (per-block histograms, partial probability sums, block-local ranks: 8*T bytes and 4*(N+2n+2m) bytes for
 * each block of 16, 32 or 64 tokens while these make at most 2 MB and T <= 65536, otherwise for each block of
 * 256 tokens) is a fixed array of SMILE_STATIC_SCRATCH_BYTES inside the library's device image, which
 * every GPU the library runs on holds until the process ends.  Returns SMILE_WORKSPACE when the shape
 * needs more than that (T = 65536 with 32 x 8 experts needs 1.9 MB, with 64 x 64 experts 5 MB) and enqueues nothing then.  It calls
 * no hipMalloc / hipFree and nothing that allocates; the first call on a device looks up the array's
 * address (make that call outside a graph capture).  All calls on one GPU share the array: calls that
 * overlap there (other streams, other threads) race, calls in stream order do not, and no call
 * depends on what an earlier one left in it. */
#define SMILE_STATIC_SCRATCH_BYTES (4u << 20)
smile_status smile_route_bilevel_static(const smile_layer_desc *desc, const float *logits_inter,
                                        const float *logits_intra, const float *bias_inter,
                                        const float *bias_intra, int32_t *group_idx, int32_t *local_idx,
                                        int32_t *pos_in_group, int32_t *slot, float *gate, float *p_top,
                                        float *q_top, int32_t *group_count, int32_t *local_count,
                                        int32_t *expert_count, int32_t *kept_count, float *p_sum, float *q_sum,
                                        void *stream);

/* Step 3 -- dispatch: xe[e, slot[t], :] = x[t, :] for every kept token, e =
 * group_idx[t]*m + local_idx[t] (the two routing hops of Section 3.2.1 composed
 * into one row move).  xe[N,C,d] in the ctx dtype; rows at or beyond
 * kept_count[e] are not written. */
smile_status smile_dispatch(smile_ctx *ctx, const void *x, const int32_t *group_idx, const int32_t *local_idx,
                            const int32_t *slot, void *xe, void *stream);

/* The same move as the two hops of Section 3.2.3, with the first-hop buffer materialised (what the
 * inter-node All2All delivers): xg[n, group_rows, d] in the ctx dtype.
 *   hop 1: xg[group_idx[t], pos_in_group[t], :] = x[t, :]        for pos_in_group[t] < group_rows
 *   hop 2: xe[e, slot[t], :] = xg[group_idx[t], pos_in_group[t], :]   for slot[t] >= 0
 * group_rows >= 1; with a group capacity it is normally desc.group_capacity, without one any value
 * not below the largest group_count.  hop 2 requires pos_in_group[t] < group_rows for every kept
 * token (true for the outputs of smile_route_bilevel under the rule above) and does not check it on
 * the device beyond skipping such tokens.  Rows that receive nothing are not written. */
smile_status smile_dispatch_hop1(smile_ctx *ctx, const void *x, const int32_t *group_idx,
                                 const int32_t *pos_in_group, int32_t group_rows, void *xg, void *stream);
smile_status smile_dispatch_hop2(smile_ctx *ctx, const void *xg, const int32_t *group_idx,
                                 const int32_t *local_idx, const int32_t *pos_in_group, const int32_t *slot,
                                 int32_t group_rows, void *xe, void *stream);

/* Step 3 -- expert FFN E_e of Eq. 3 (Section 4.1: hidden -> intermediate ->
 * hidden with the activation of the ctx) on rows r < kept_count[e]:
 *   h  = act(xe[e,r,:] . w1[e]^T + b1[e])     w1[N,F,d]  (out-features x in-features), b1[N,F] or NULL
 *   ye[e,r,:] = h . w2[e]^T + b2[e]           w2[N,d,F],                              b2[N,d] or NULL
 * Weights and biases in the ctx dtype; accumulation in fp32; h is rounded to
 * the ctx dtype between the two products.  kept_count is read on the device
 * (no host sync); rows at or beyond kept_count[e] of ye are not written. */
smile_status smile_expert_ffn(smile_ctx *ctx, const void *xe, const int32_t *kept_count,
                              const void *w1, const void *b1, const void *w2, const void *b2,
                              void *ye, void *stream);

/* The two halves of smile_expert_ffn as separate calls (same kernels, same results), for callers
 * that want to time or interleave them: _up computes h = act(xe . w1^T + b1) into the ctx
 * workspace, _down computes ye = h . w2^T + b2 from it.  _down must follow an _up on the same ctx
 * and stream with the same kept_count. */
smile_status smile_expert_ffn_up(smile_ctx *ctx, const void *xe, const int32_t *kept_count,
                                 const void *w1, const void *b1, void *stream);
smile_status smile_expert_ffn_down(smile_ctx *ctx, const int32_t *kept_count, const void *w2, const void *b2,
                                   void *ye, void *stream);

/* smile_expert_ffn_up with kernel timing, for benchmarks: `start_event` and `stop_event` are
 * hipEvent_t handles (passed as void*, created by the caller with timing enabled, both non-NULL).
 * They receive the begin and end timestamps of the up-projection kernel itself, so that
 * hipEventElapsedTime(start, stop) after synchronisation is the kernel's own duration without
 * launch gaps.  Same work and results as smile_expert_ffn_up. */
smile_status smile_expert_ffn_up_timed(smile_ctx *ctx, const void *xe, const int32_t *kept_count,
                                       const void *w1, const void *b1, void *start_event, void *stop_event,
                                       void *stream);

/* Step 4 -- combine (Eq. 3): y[t,:] = gate[t] * ye[e, slot[t], :] for kept
 * tokens, 0 for dropped ones; product in fp32, rounded once to the ctx dtype. */
smile_status smile_combine(smile_ctx *ctx, const void *ye, const int32_t *group_idx, const int32_t *local_idx,
                           const int32_t *slot, const float *gate, void *y, void *stream);

/* Step 4 -- additive load-balancing loss (Eq. 4), from the statistics of
 * smile_route_bilevel:
 *   out3[0] = n * sum_i (group_count[i]/T) * (p_sum[i]/T)
 *   out3[1] = m * sum_j (local_count[j]/T) * (q_sum[j]/T)
 *   out3[2] = alpha*out3[0] + beta*out3[1]
 * out3: 3 fp32 values on the device. */
smile_status smile_aux_loss(smile_ctx *ctx, const int32_t *group_count, const int32_t *local_count,
                            const float *p_sum, const float *q_sum, float *out3, void *stream);

/* All tensors of one forward pass, for smile_layer_forward. */
typedef struct smile_layer_io {
    /* inputs */
    const void *x, *w_inter, *w_intra, *w1, *b1, *w2, *b2;
    const float *bias_inter, *bias_intra;
    /* intermediates and outputs (all caller-allocated) */
    float *logits_inter, *logits_intra;
    int32_t *group_idx, *local_idx, *pos_in_group, *slot;
    float *gate, *p_top, *q_top;
    int32_t *group_count, *local_count, *expert_count, *kept_count;
    float *p_sum, *q_sum;
    void *xe, *ye;   /* expert buffers [N,C,d]: both given, or both NULL (see smile_layer_forward) */
    void *y;
    float *loss3;
    /* optional: hipEvent_t pair (both or neither) receiving the begin / end timestamps of the
     * up-projection kernel, as in smile_expert_ffn_up_timed; NULL = no timing */
    void *prof_up_start, *prof_up_stop;
    /* optional (both or neither), for a backward pass that does not recompute them: the hidden
     * activation h = act(pre) and the pre-activation pre = xe . w1^T + b1, [N,C,F] in the ctx dtype,
     * rows below kept_count[e] only.  When given, h lives there instead of in the ctx workspace. */
    void *h_save, *pre_save;
} smile_layer_io;

/* The whole forward pass in one call: enqueues the six steps above in order on
 * `stream` (gate logits, route, dispatch, expert FFN, combine, loss).  Same checks
 * and bit-identical results as calling them one by one, with fewer launches: the router logits
 * are computed by the kernel that routes them (most shapes), and the last routing kernel evaluates the loss.
 *   - io->xe and io->ye given: the expert buffers are materialised as by
 *     smile_dispatch / smile_expert_ffn; the last routing kernel moves the rows and the down-projection also
 *     writes y;
 *   - io->xe == io->ye == NULL: the permutations are fused into the expert GEMMs --
 *     the up-projection gathers its rows from x through a slot -> token map and the
 *     down-projection returns gate-weighted rows straight to y; rows of dropped
 *     tokens are zeroed by the routing (no [N,C,d] traffic).
 * Launches: three for a batch of at most 64 tokens and 64 KB of x (router of at most some hundred columns; four with expert
 * buffers); otherwise four, one more where a kernel of its own orders the routing blocks (more than 256 of them, or
 * (N + n) * blocks beyond 32768 counts: from about 16384 tokens or 100 experts on), one more (per 128 router columns) where the
 * logits have a kernel of their own (33 to 48 router columns from 8193 tokens on, more than 65536 tokens, routers of
 * several hundred columns); a group capacity adds one or two. */
smile_status smile_layer_forward(smile_ctx *ctx, const smile_layer_io *io, void *stream);

/* ---------------------------------------------------------------------------
 * Backward pass.  The paper trains the layer (Section 4.1) and prints no gradient formulas; these
 * entry points compute the derivative of the forward map defined above (Eq. 3 for y, Eq. 4 for the
 * loss) by the chain rule, for
 *     L = sum_{t,k} dy[t,k] * y[t,k] + dloss * (alpha*inter + beta*intra),
 * with the discrete decisions (top-1 indices, slots, drops) and the fractions f of Eq. 4 held
 * constant, as for the Switch loss of Section 2.  Gradient tensors stored in the ctx dtype (dye,
 * dxe, dx, dw1, dw2) are rounded once from fp32; dgate, dlp, dlq, dw_inter, dw_intra are fp32.
 * Experts with bias vectors are not covered (there is no b1 / b2 argument and no gradient for them).
 * The steps mirror the forward ones in reverse order; the tensors "saved from the forward pass" are
 * the outputs of the forward entry points for the same inputs.
 * ------------------------------------------------------------------------- */

/* Bytes of device scratch memory smile_expert_ffn_backward, smile_gate_weights_backward and
 * smile_layer_backward need: the recomputed h and pre, the gradient at the pre-activation (3 N*C*F
 * elements) and partial sums of the router-weight gradient.  Host-only.  The memory is the caller's,
 * 256-byte aligned, and only used during the call's enqueued work. */
smile_status smile_backward_workspace_bytes(const smile_layer_desc *desc, size_t *bytes);

/* Eq. 3 backwards: for a kept token dye[e, slot[t], :] = gate[t] * dy[t, :] and
 * dgate[t] = sum_k dy[t,k] * ye[e, slot[t], k]; a dropped token gives dgate[t] = 0.
 * dy[T,d], ye[N,C,d], dye[N,C,d] in the ctx dtype; rows of dye no token owns are not written. */
smile_status smile_combine_backward(smile_ctx *ctx, const void *dy, const void *ye, const int32_t *group_idx,
                                    const int32_t *local_idx, const int32_t *slot, const float *gate,
                                    void *dye, float *dgate, void *stream);

/* The two routers backwards (Eq. 1 softmax, Eq. 3 gate, Eq. 4 loss).  With p, q the softmax rows of
 * token t (biases as in smile_route_bilevel), g = group_idx[t], l = local_idx[t]:
 *   u_i = dloss*alpha*n*group_count[i]/T^2 + [i == g] * dgate[t] * q[l],   dlp[t,k] = p_k (u_k - sum_i u_i p_i)
 *   v_j = dloss*beta *m*local_count[j]/T^2 + [j == l] * dgate[t] * p[g],   dlq[t,k] = q_k (v_k - sum_j v_j q_j)
 * dlp[T,n], dlq[T,m] fp32: the gradients with respect to the router logits. */
smile_status smile_route_backward(smile_ctx *ctx, const float *logits_inter, const float *logits_intra,
                                  const float *bias_inter, const float *bias_intra,
                                  const int32_t *group_idx, const int32_t *local_idx, const float *dgate,
                                  const int32_t *group_count, const int32_t *local_count, float dloss,
                                  float *dlp, float *dlq, void *stream);

/* Expert FFN backwards (E_e of Eq. 3, Section 4.1, no bias vectors), rows r < kept_count[e]:
 *   pre = xe[e] . w1[e]^T, h = act(pre)     (both rounded to the ctx dtype; taken from h / pre, the
 *                                            buffers smile_layer_forward saved, or recomputed here
 *                                            when both are NULL)
 *   dpre = (dye[e] . w2[e]) * act'(pre)
 *   dxe[e] = dpre . w1[e]                                              [N,C,d]
 *   dw2[e][c,f] = sum_r dye[e,r,c] * h[r,f]                            [N,d,F]
 *   dw1[e][f,k] = sum_r dpre[r,f] * xe[e,r,k]                          [N,F,d]
 * Rows of dxe at or beyond kept_count[e] are not written; an expert without rows gets zero
 * weight gradients. */
smile_status smile_expert_ffn_backward(smile_ctx *ctx, const void *xe, const int32_t *kept_count,
                                       const void *w1, const void *w2, const void *dye,
                                       const void *h, const void *pre,
                                       void *dxe, void *dw1, void *dw2,
                                       void *workspace, size_t workspace_bytes, void *stream);

/* Dispatch and router logits backwards: dx[t,:] = dxe[e, slot[t], :] (zero for a dropped token)
 *   + sum_i dlp[t,i] * w_inter[i,:] + sum_j dlq[t,j] * w_intra[j,:], rounded once.  dx[T,d]. */
smile_status smile_dispatch_backward(smile_ctx *ctx, const void *dxe, const int32_t *group_idx,
                                     const int32_t *local_idx, const int32_t *slot, const float *dlp,
                                     const float *dlq, const void *w_inter, const void *w_intra, void *dx,
                                     void *stream);

/* Router weights backwards: dw_inter[i,:] = sum_t dlp[t,i] * x[t,:], dw_intra[j,:] = sum_t dlq[t,j] * x[t,:]
 * (fp32 [n,d] and [m,d]); summed in a fixed order, so repeated calls give identical bits. */
smile_status smile_gate_weights_backward(smile_ctx *ctx, const void *x, const float *dlp, const float *dlq,
                                         float *dw_inter, float *dw_intra,
                                         void *workspace, size_t workspace_bytes, void *stream);

/* All tensors of one backward pass, for smile_layer_backward. */
typedef struct smile_backward_io {
    /* inputs of the forward pass */
    const void *x, *w_inter, *w_intra, *w1, *w2;
    const float *bias_inter, *bias_intra;            /* may be NULL */
    /* saved from the forward pass */
    const float *logits_inter, *logits_intra;
    const int32_t *group_idx, *local_idx, *slot;
    const float *gate;
    const int32_t *group_count, *local_count, *kept_count;
    const void *xe, *ye;
    const void *h, *pre;                             /* h_save / pre_save of the forward pass, or both NULL */
    /* upstream gradient of y */
    const void *dy;
    /* intermediates (caller-allocated): dye[N,C,d], dgate[T], dlp[T,n], dlq[T,m], dxe[N,C,d] */
    void *dye;
    float *dgate, *dlp, *dlq;
    void *dxe;
    /* results */
    void *dx;
    float *dw_inter, *dw_intra;
    void *dw1, *dw2;
} smile_backward_io;

/* The five backward steps in one call, in the order combine, route, expert FFN, dispatch, router
 * weights; same results as calling them one by one.  dloss is the upstream gradient of the
 * scalar loss of Eq. 4 (out3[2] of smile_aux_loss). */
smile_status smile_layer_backward(smile_ctx *ctx, const smile_backward_io *io, float dloss,
                                  void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Operators in 8 bits around and inside the layer: the norm in front of it, products of 8-bit operands,
 * and activations kept in 8 bits for the backward pass.  They need no ctx (but smile_fp8_dispatch), allocate
 * nothing and take tensors of any size within the stated limits.
 *
 * 8-bit rows.  A row of K values is cut into blocks of 128 (the last one may be shorter).  A block has a
 * power-of-two scale 2^(b - 127), kept as its byte b, and each value a code in 8-bit floating point (1 sign,
 * 4 exponent, 3 fraction bits, bias 7, no infinity, NaN = 0x7f / 0xff): value = code * 2^(b - 127).
 *   codes  [N][C][smile_fp8_pitch(K)]        bytes; columns K .. pitch - 1 are zero codes
 *   scales [N][ceil(K/128)][smile_fp8_scale_pitch(C)] bytes; entry r of a block's line belongs to row r
 * Packing: b is the least byte >= 1 for which the block's largest magnitude is at most 448 * 2^(b - 127), so
 * a block of zeros has b = 1; value / 2^(b - 127) is rounded to the nearest code, ties to even, with
 * gradual underflow.  Infinities and NaN become NaN codes and do not count for b.  Unlike those of the layer
 * these operators take NaN: it stays in its row and column, through the activations too, and the derivative at a kept NaN is NaN.
 * 8-bit weights w[N][Nout][K] have one scale for each 128 x 128 block:
 *   codes  [N][Nout][smile_fp8_pitch(K)],  scales [N][ceil(K/128)][smile_fp8_scale_pitch(ceil(Nout/128))]
 * and in transposed form the same codes as [N][K][smile_fp8_pitch(Nout)] with scales
 * [N][ceil(Nout/128)][smile_fp8_scale_pitch(ceil(K/128))].
 * Why powers of two: the matrix cores apply them for nothing, scaling rounds nothing, and the values
 * are exact in bfloat16 (from b = 3 on; and in half precision within its range).  Magnitudes above 31/32 * 2^128 round to
 * 2^128, which is infinite in fp32 and bfloat16.
 *
 * `rows`: int32 [N] on the device, valid rows of each group (clamped to 0 .. C), or NULL for all C.  Rows at
 * or beyond it are neither read nor written.
 * Limits: N, C, T, K, Nout, d >= 1; K, Nout, d % 8 == 0; N <= 4096; K, Nout <= 32768, d of the norm <= 16384; N*C, N*Nout and
 * T <= 2^27; elements of any tensor below 2^40, scales of a group below 2^31.
 * ------------------------------------------------------------------------- */

/* Bytes of a row of codes (K up to a multiple of 128) and of a line of scales (rows up to a multiple of 16).  Host helpers. */
int32_t smile_fp8_pitch(int32_t K);
int32_t smile_fp8_scale_pitch(int32_t rows);

/* Root-mean-square norm with the residual's addition, over the d columns of T rows in storage type `dtype`:
 *   s[t,:] = x[t,:] + residual[t,:], rounded to the storage type (residual NULL: s = x)
 *   rstd[t] = (mean_k s[t,k]^2 + eps)^(-1/2);   y[t,k] = s[t,k] * rstd[t] * weight[k]
 * from s as it is rounded, in fp32.  Outputs, each of which may be NULL, but not both y and y8: sum (s; NULL without
 * residual), y in the storage type, y8 with y8_scale (8-bit rows, N = 1, C = T; rounded from fp32, not from y), rstd [T].
 * weight[d] in the storage type; eps > 0.  sum may be x or residual itself, y may be x. */
smile_status smile_rms_norm(int32_t T, int32_t d, int32_t dtype, const void *x, const void *residual, const void *weight,
                            float eps, void *sum, void *y, void *y8, void *y8_scale, float *rstd, void *stream);

/* Its gradients.  s and rstd as smile_rms_norm gave them, dy the gradient of y, dsum that of s from its other uses (NULL: none):
 *   u = s * rstd, g = weight * dy:   ds = dsum + rstd * (g - u * mean_k(g * u)),   dweight[k] = sum_t dy[t,k] * u[t,k]
 * ds (of x and of residual alike) in the storage type; ds may be dy or dsum itself.  dweight fp32 [d], summed in a fixed order:
 * chains of at most T / 768 (rounded up) + 16 additions in fp32, and their sums in 64 bits.  The 8-bit output counts as y itself.  workspace: at least
 * smile_rms_norm_backward_workspace_bytes bytes, 256-byte aligned. */
smile_status smile_rms_norm_backward_workspace_bytes(int32_t T, int32_t d, size_t *bytes);
smile_status smile_rms_norm_backward(int32_t T, int32_t d, int32_t dtype, const void *dy, const void *dsum, const void *s,
                                     const void *weight, const float *rstd, void *ds, float *dweight, void *workspace,
                                     size_t workspace_bytes, void *stream);

/* src[N][C][K] in `dtype` to 8-bit rows, and 8-bit rows to dst[N][C][K] in `dtype` (in half precision what
 * is beyond +-65504 becomes that). */
smile_status smile_fp8_pack_rows(int32_t N, int32_t C, int32_t K, int32_t dtype, const void *src, const int32_t *rows,
                                 void *codes, void *scales, void *stream);
smile_status smile_fp8_unpack_rows(int32_t N, int32_t C, int32_t K, int32_t dtype, const void *codes, const void *scales,
                                   const int32_t *rows, void *dst, void *stream);

/* w[N][Nout][K] in `dtype` to 8-bit weights, and to their transposed form where codes_t and scales_t are given (both or neither). */
smile_status smile_fp8_pack_weights(int32_t N, int32_t Nout, int32_t K, int32_t dtype, const void *w, void *codes, void *scales,
                                    void *codes_t, void *scales_t, void *stream);

/* smile_dispatch for 8-bit rows of the tokens (N = 1, C = T, K = d_model): row t of x8 and its scales to row slot[t] of its
 * expert's buffer in xe8 [N][C][...], xe_scale.  Any dtype of the ctx. */
smile_status smile_fp8_dispatch(smile_ctx *ctx, const void *x8, const void *x_scale, const int32_t *group_idx,
                                const int32_t *local_idx, const int32_t *slot, void *xe8, void *xe_scale, void *stream);

enum { SMILE_ACT_NONE = 2 };   /* smile_fp8_gemm: no activation */

/* Grouped product of 8-bit rows with 8-bit weights, rows r < rows[e] of every group e:
 *   p[r,o] = sum_k x[e,r,k] * w[e,o,k] + bias[e,o]           (fp32)
 *   v = act(p), or, where grad8 is given, p * act'(g) with g the value that grad8 keeps of the pre-activation
 * y: v in the storage type; y8 / y_scale: v as 8-bit rows; pre8 / pre_scale: p as 8-bit rows, the checkpoint that a
 * backward product takes as grad8 (with SMILE_ACT_RELU its codes next to zero come from sums in 64 bits, since the derivative
 * goes by the side of zero; sums that are zero, as of columns of zero weights beside others in a block of 128, count as such, and many of them
 * cost many times the product).  With weights in transposed form it is the gradient of the rows.
 * A sum that overflows is infinite, and so is its activation (that of -infinity is 0): a NaN code in 8 bits.
 * GELU is the erf form with the accuracy of the 16-bit expert FFN whatever y's type: 4e-7 (1 + |p|), in the tail 0.5 % of the value at p = -6.5, 4 %
 * at -13.  Sums are held in fp32.  The matrix cores add the
 * products of 16 neighbouring k at a time to about 2^-16 of the largest of them: normwise 1.5e-5 on normally distributed
 * values, 6e-5 where a block's codes are spread evenly over all exponents.  Of 8-bit results some three codes in ten thousand, next to the
 * middle between two, are therefore one step off those of exact sums. */
typedef struct smile_fp8_gemm_args {
    int32_t N, C, K, Nout;       /* groups, rows of each group's buffer, contraction length, columns of the result */
    int32_t dtype, act;          /* storage type of y and bias; SMILE_ACT_* */
    const void *x8, *x_scale;    /* 8-bit rows [N][C][K] */
    const void *w8, *w_scale;    /* 8-bit weights [N][Nout][K] */
    const void *bias;            /* [N][Nout] or NULL; not with grad8 */
    const int32_t *rows;         /* [N] or NULL */
    void *y;                     /* [N][C][Nout] or NULL */
    void *y8, *y_scale;          /* 8-bit rows [N][C][Nout], or both NULL; y or y8 is given */
    void *pre8, *pre_scale;      /* 8-bit rows [N][C][Nout], or both NULL; not with grad8 */
    const void *grad8, *grad_scale;   /* 8-bit rows [N][C][Nout], or both NULL; needs an activation */
} smile_fp8_gemm_args;
smile_status smile_fp8_gemm(const smile_fp8_gemm_args *args, void *stream);

/* Weight gradient from an operand kept in 8 bits: dw[e,o,k] = sum_{r < rows[e]} dy[e,r,o] * x[e,r,k], dy[N][C][Nout] and
 * dw[N][Nout][K] in `dtype`, x8 / x_scale 8-bit rows [N][C][K].  Products of 16-bit values (K and Nout % 64 == 0) or of fp32 ones,
 * summed in fp32 and rounded once (in half precision the operand counts as what it holds: beyond +-65504 as that, below 2^-14 as
 * its subnormals); a group without rows gets zeros.  workspace: at least smile_fp8_weight_grad_workspace_bytes
 * bytes, 256-byte aligned (the operand in `dtype`). */
smile_status smile_fp8_weight_grad_workspace_bytes(int32_t N, int32_t C, int32_t K, int32_t dtype, size_t *bytes);
smile_status smile_fp8_weight_grad(int32_t N, int32_t C, int32_t Nout, int32_t K, int32_t dtype, const void *dy, const void *x8,
                                   const void *x_scale, const int32_t *rows, void *dw, void *workspace, size_t workspace_bytes,
                                   void *stream);

/* ---------------------------------------------------------------------------
 * Operators of a layer without dropped tokens, and of its optimizer: k experts for a token, the (token, choice) pairs sorted by expert,
 * products of each expert's rows (or of dense rows), the weighted return, the gradients, and an AdamW step.  They need no ctx and
 * allocate nothing.  Workspaces are the caller's, 256-byte aligned, and only used during the call's enqueued work; calls that overlap must not share
 * one.  The functions ending in _bytes, and smile_adamw_plan, work on the host alone.
 * What a call writes must not overlap what it reads or writes besides, but where a tensor may be another: SMILE_INVALID_ARG.
 * Limits: T, rows, N, k, d, K, F >= 1; N <= 4096; k <= N and k <= 64; T*k < 2^26, rows and R <= 2^27; d, K, F % 8 == 0; d <= 16384,
 * K, F <= 32768; elements of any tensor below 2^40; rows * N of a product below 2^36.
 * Indices and row numbers are never followed outside their tensors: a pair whose expert is not in 0 .. N - 1 has no row, a row number that is not in
 * 0 .. R - 1 counts as none, and a first row outside of 0 .. rows counts as its border.  First rows that are not in order lead nowhere else either, but what the products'
 * results then hold is not defined.
 * ------------------------------------------------------------------------- */

/* k experts for each of T tokens.  v[t,e] = logits[t,e] + bias[e] (one fp32 addition; bias NULL: none), -infinity where bias[e] is: such an
 * expert is shut off.  p[t,:] = softmax of v[t,:] (zeros if every v is -infinity).
 *   idx[t,j]     the expert of the j-th largest v, equal ones in the order of their index; -1 where only -infinity is left
 *   weight[t,j]  p of it, divided by the sum over the token's choices if `normalize`; 0 where idx is -1
 *   p_sum[e]     sum over t of p[t,e], in a fixed order (fp32 over the tokens of a workgroup's lane, their sums in 64 bits); may be NULL
 * logits[T,N], bias[N], weight[T,k], p_sum[N] fp32, idx[T,k] int32.  A NaN or +infinity among a token's v makes its weights, and p_sum, NaN.
 * workspace: smile_topk_workspace_bytes bytes; not needed without p_sum. */
smile_status smile_topk_workspace_bytes(int32_t T, int32_t N, size_t *bytes);
smile_status smile_topk(int32_t T, int32_t N, int32_t k, int32_t normalize, const float *logits, const float *bias, int32_t *idx, float *weight,
                        float *p_sum, void *workspace, size_t workspace_bytes, void *stream);

/* Gradient of the logits, for L = sum dweight * weight + coef * sum_e count[e] * p_sum[e] with idx and count held constant.  With u[t,e] =
 * coef * count[e] (count NULL: 0):
 *   not normalize:  u[t,e] += dweight[t,j] for e = idx[t,j];   dlogits = p (u - sum_e p u)
 *   normalize:      the same without dweight, and + w (dweight[t,j] - sum_j w dweight[t,:]) at e = idx[t,j], w the weights
 * idx as smile_topk gave it (a token's experts differ).  coef = alpha * N / (k T^2) makes the second term
 * alpha N sum_e f_e P_e, Eq. 4 of one level with the fractions f_e = count[e] / (k T) and P_e = p_sum[e] / T.
 * dlogits[T,N] fp32, may be logits; the sum of it over t is the gradient of the bias. */
smile_status smile_topk_backward(int32_t T, int32_t N, int32_t k, int32_t normalize, const float *logits, const float *bias, const int32_t *idx,
                                 const float *dweight, const int32_t *count, float coef, float *dlogits, void *stream);

/* The pairs (t, j), numbered t*k + j, sorted by expert idx[t,j] and then by their number:
 *   count[e]   pairs of expert e;   start[e] = sum of count[0 .. e-1], start[N] their number
 *   pos[t,j]   the pair's row in the sorted order, -1 without one;   source[r]  the pair of row r, -1 from start[N] to T*k - 1
 * All int32: idx[T,k], count[N], start[N+1], pos[T,k], source[T*k]. */
smile_status smile_sort_experts_workspace_bytes(int32_t T, int32_t k, int32_t N, size_t *bytes);
smile_status smile_sort_experts(int32_t T, int32_t k, int32_t N, const int32_t *idx, int32_t *count, int32_t *start, int32_t *pos, int32_t *source,
                                void *workspace, size_t workspace_bytes, void *stream);

/* Tokens to their sorted rows: xs[pos[t,j],:] = x[t,:].  x[T,d], xs[R,d] in `dtype`; rows no pair has are left as they were, and no row may have
 * two pairs (here and in smile_sorted_combine_backward: either's could remain). */
smile_status smile_sorted_dispatch(int32_t T, int32_t k, int32_t d, int32_t R, int32_t dtype, const void *x, const int32_t *pos, void *xs, void *stream);

/* And back: y[t,:] = residual[t,:] + sum_j weight[t,j] * ys[pos[t,j],:], in fp32, rounded once.  weight NULL: ones, which makes it the gradient of
 * smile_sorted_dispatch; residual NULL: zeros; y may be residual.  Pairs without a row add nothing.  y[T,d], ys[R,d], residual[T,d] in `dtype`. */
smile_status smile_sorted_combine(int32_t T, int32_t k, int32_t d, int32_t R, int32_t dtype, const void *ys, const int32_t *pos, const float *weight,
                                  const void *residual, void *y, void *stream);

/* Its gradients: dys[pos[t,j],:] = weight[t,j] * dy[t,:], dweight[t,j] = sum_c dy[t,c] * ys[pos[t,j],c] (fp32; 0 for a pair without a row).
 * Rows of dys no pair has are left as they were.  dweight and ys may be NULL together. */
smile_status smile_sorted_combine_backward(int32_t T, int32_t k, int32_t d, int32_t R, int32_t dtype, const void *dy, const void *ys, const int32_t *pos,
                                           const float *weight, void *dys, float *dweight, void *stream);

/* y[r,f] = act(sum_k x[r,k] * w[e,f,k] + bias[e,f]) + residual[r,f] for the rows start[e] <= r < start[e+1] of every group e; start NULL: N = 1 and
 * all rows.  Rows of no group are neither read nor written.  Sums, activation and the residual's addition in fp32, rounded once; `pre`, if
 * given, receives the activation's argument (the form that smile_linear_backward reads).  act: SMILE_ACT_RELU, _GELU (erf form; 16-bit types with
 * an error of 4e-7 (1 + |v|)) or _NONE.  y may be residual.  NaN and infinities stay in their row and column. */
typedef struct smile_linear_args {
    int32_t N, rows, K, F;       /* groups; rows of x, y, residual and pre; columns of x; columns of y */
    int32_t dtype, act;
    const void *x;               /* [rows][K] */
    const void *w;               /* [N][F][K] */
    const void *bias;            /* [N][F] or NULL */
    const void *residual;        /* [rows][F] or NULL */
    const int32_t *start;        /* [N+1] or NULL */
    void *y;                     /* [rows][F] */
    void *pre;                   /* [rows][F] or NULL */
} smile_linear_args;
smile_status smile_linear(const smile_linear_args *args, void *stream);

/* Its gradients (that of the residual is dy).  With g = dy * act'(pre), rounded to the storage type where it enters a product (in half precision infinite above 65504):
 *   dx[r,:] = sum_f g[r,f] * w[e,f,:],   dw[e,f,:] = sum_r g[r,f] * x[r,:],   dbias[e,f] = sum_r g[r,f]   (g before its rounding)
 * summed in fp32 in a fixed order, rounded once.  Each of dx, dw, dbias may be NULL, but not all; w is needed for dx, x for dw, pre for
 * an activation.  Rows of no group are neither read nor written; a group without rows gets zeros. */
typedef struct smile_linear_backward_args {
    int32_t N, rows, K, F;
    int32_t dtype, act;
    const void *dy;              /* [rows][F] */
    const void *x, *w, *pre;
    const int32_t *start;
    void *dx;                    /* [rows][K] or NULL */
    void *dw;                    /* [N][F][K] or NULL */
    void *dbias;                 /* [N][F] or NULL */
} smile_linear_backward_args;
smile_status smile_linear_backward_workspace_bytes(const smile_linear_backward_args *args, size_t *bytes);
smile_status smile_linear_backward(const smile_linear_backward_args *args, void *workspace, size_t workspace_bytes, void *stream);

/* AdamW over any number of tensors in one launch, in place.  t = step[0] + 1, g the gradient, p the master weight where there is one, else the parameter:
 *   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2
 *   p = p - lr (weight_decay p + m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps));   param = p rounded;   step[0] = t
 * in fp32 (the powers in 64 bits; the root and the reciprocal of its sum with eps each to a unit of the last place).  lr[1] fp32 and
 * step[1] int32 (>= 0) are on the device, so that a captured graph follows them.
 * State of 32 bits: m[n], v[n] fp32.  State of 8 bits: blocks of 128 neighbouring elements share a power of two, kept as its byte b:
 *   m: e4m3 codes times 2^(b - 127), b the least byte >= 1 for which the block's largest magnitude is at most 448 * 2^(b - 127)
 *   v: codes c of 5 exponent and 3 fraction bits without a sign, (1 + (c & 7) / 8) * 2^((c >> 3) - 30) * 2^(b - 127), 0 for c = 0; b is the power of two
 *      of the block's largest finite value (at least 1); what is not 0 is at least c = 1, what is finite at most c = 248; c = 255 is infinity (249 to 254 are not used)
 * The stored moments (not those of this step's update) are rounded up or down by 16 random bits R each: up where the part cut off is at least
 * 1 - R / 65536 of a step.  The bits are a hash of (seed, t, tensor, element), so a step gives the same bits wherever it runs.
 * m, v [n up to a multiple of 128], m_scale, v_scale [their blocks]; padding gets zero codes; all zeros is a new state.  A gradient that is not finite makes
 * its parameter and the first moment of an 8-bit state NaN.  Where it is finite and its square is not, v is infinite from then on (unless beta2 is 0), as the formulas have
 * it in fp32, and the element's update 0.  What is not finite does not count for the block's power of two.
 * A state that decayed below fp32's normal range is kept as far as the codes reach.
 * The tensors of a plan share their types; each pointer is 16-byte aligned, the scales' excepted.  The plan is built on the host and copied to the device by the
 * caller (no tensor or state twice in it, and no gradient among them; the device copy 256-byte aligned; the step keeps a counter in it, so steps of one plan must not overlap, and
 * lr and step are not of the plan's tensors, which the call itself does not know). */
typedef struct smile_adamw_tensor {
    void *param;                 /* [n] in `dtype` */
    const void *grad;            /* [n] in `grad_dtype` */
    float *master;               /* [n] or NULL (all tensors of a plan alike); 16-bit parameters only */
    void *m, *v;
    void *m_scale, *v_scale;     /* 8-bit states, else NULL */
    int64_t n;                   /* 1 .. 2^32 */
    float weight_decay;
} smile_adamw_tensor;
typedef struct smile_adamw_args {
    int32_t tensors;
    int32_t dtype, grad_dtype;   /* of the parameters; of the gradients: the same or SMILE_DTYPE_F32 */
    int32_t state_bits;          /* 32 or 8 */
    int32_t has_master;
    int32_t seed;
    double beta1, beta2, eps;    /* 0 <= beta < 1, 2^-126 <= eps <= 1; 1 - beta is taken in 64 bits */
    int64_t chunks;              /* filled in by smile_adamw_plan */
} smile_adamw_args;
smile_status smile_adamw_plan_bytes(const smile_adamw_args *args, const smile_adamw_tensor *tensors, size_t *bytes);
smile_status smile_adamw_plan(smile_adamw_args *args, const smile_adamw_tensor *tensors, void *plan, size_t plan_bytes);
smile_status smile_adamw(const smile_adamw_args *args, void *device_plan, size_t plan_bytes, const float *lr, int32_t *step, void *stream);

/* 8-bit states of n elements (a multiple of 128) as values in `dtype` (fp32 or bfloat16), for checkpoints and inspection. */
smile_status smile_adamw_unpack_states(int64_t n, int32_t dtype, const void *m, const void *m_scale, const void *v, const void *v_scale, void *m_value,
                                       void *v_value, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SMILE_H */
