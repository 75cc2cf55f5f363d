/*
 * clearmoe.h -- C ABI of the GB300 (sm_103a) CLEAR-MoE FFN layer.
 *
 * CLEAR-MoE (arxiv 2606.28516) converts a frozen ViT FFN into a shared fc1, a shared truncated-SVD
 * fc2 basis and per-cluster residual fc2 experts chosen by a top-1 router (Eq. 2, Algorithms 2-3):
 *
 *     z = GELU(W1 x + b1)                       (fc1 shared by every expert, exact-erf GELU)
 *     a = argmax_e (W_g x + b_g)_e              (linear router, lowest index on ties)
 *     y = U_r diag(S_r) Vh_r z + W_a^res z      (shared SVD basis + residual expert of token a)
 *
 * Shapes (row-major, element type "D" = the layer's dtype unless stated):
 *   x [T x d], W1 [H x d], b1 [H], U_r [d x r], S_r [r] (always float32), Vh_r = V_r^T [r x H],
 *   residual_e[e] [d x H] for e < E, W_g [E x d], b_g [E], W2 [d x H], out [T x d].
 *
 * Conventions for every call below:
 *   - Every pointer named as a tensor is a DEVICE pointer owned by the caller, 16-byte aligned,
 *     to a dense row-major array of the stated shape. The library never frees caller memory.
 *   - `stream` is a cudaStream_t (NULL = the legacy default stream). Calls only enqueue work and
 *     return; they never synchronise, except clearmoe_layer_status and clearmoe_layer_destroy.
 *   - One handle may be used by one stream at a time: its workspace holds the hidden states and
 *     routing of the last forward.
 *   - Kernels are launched with programmatic dependent launch: the first kernel of a call may start,
 *     and read the weights (every tensor argument except x), while the kernel enqueued just before it
 *     on the same stream is finishing; x is read only after that kernel has completed. So weights
 *     must not be written by the kernel immediately before the call (any later-enqueued work in
 *     between, or a synchronisation, is enough; of a kernel of the caller's own that work must not
 *     let its successor start before it has waited for its predecessor). clearmoe_route_noalloc reads
 *     nothing early, nor do the calls that take no handle: those on 8-bit and 4-bit blocks, and the norm.
 *   - Arguments are validated on the host first; on a validation error (EINVAL, EUNSUPPORTED)
 *     nothing is enqueued and the outputs are untouched. CLEARMOE_ECUDA can also come from a
 *     launch after earlier kernels of the same call were enqueued; the outputs are then
 *     undefined. Return values are clearmoe_status codes.
 *   - Device-side waits are bounded. A wait that runs out writes CLEARMOE_ETIMEOUT into the
 *     handle's device status word (read by clearmoe_layer_status); the outputs of that call are
 *     then undefined, and the handle stays usable.
 */
#ifndef CLEARMOE_H
#define CLEARMOE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    CLEARMOE_OK = 0,
    CLEARMOE_EINVAL = -1,       /* bad argument: null pointer, size out of range, misalignment */
    CLEARMOE_EUNSUPPORTED = -2, /* valid but not tiled by this build (see clearmoe_layer_create) */
    CLEARMOE_ECUDA = -3,        /* a CUDA runtime/driver call failed */
    CLEARMOE_ENOMEM = -4,       /* workspace allocation failed */
    CLEARMOE_ETIMEOUT = -5      /* a bounded device-side wait ran out */
} clearmoe_status;

typedef enum {
    CLEARMOE_F32 = 0,
    CLEARMOE_BF16 = 1,
    CLEARMOE_FP8 = 2 /* weights of clearmoe_ffn_weights only: 8-bit blocks (clearmoe_fp8) */
} clearmoe_dtype;

/* Capacity of a layer handle. d and hidden are fixed per handle; T, E and r are per call and
 * bounded by max_tokens, max_E and max_r. dtype selects the arithmetic:
 *   CLEARMOE_BF16: bf16 storage, fp32 accumulation on the tcgen05 tensor cores; z, the shared-
 *                  basis coefficients t = diag(S_r) Vh_r z and out are stored in bf16.
 *   CLEARMOE_F32:  fp32 storage; the routing logits in fp32 FMA on the CUDA cores. The GEMMs of
 *                  the forward and of the dense FFN run on the TF32 tensor cores with each fp32
 *                  operand split into a TF32 part and its remainder and three products per term
 *                  (relative error near 2^-21 per product) when d, hidden and r are multiples
 *                  of 16 and the LayerNorm is not folded; otherwise, and in the other fp32 calls,
 *                  in exact fp32 FMA on the CUDA cores.
 * Tiling limits (else CLEARMOE_EUNSUPPORTED): bf16 needs d % 64 == 0, d <= 1024, hidden % 64 == 0
 * and r % 16 == 0 per call; fp32 needs d % 4 == 0, d <= 512, hidden % 4 == 0 and r % 4 == 0.
 * max_E <= 16, max_r <= 256, max_tokens <= 2^30. */
typedef struct {
    int64_t max_tokens;
    int32_t d;
    int32_t hidden;
    int32_t max_E;
    int32_t max_r;
    int32_t dtype; /* clearmoe_dtype */
} clearmoe_layer_desc;

/* Linear router (Phase 4, "Linear": d x E weights and a bias per expert): W [E x d], b [E],
 * both device pointers in the layer's dtype. */
typedef struct {
    const void* W;
    const void* b;
} clearmoe_router;

/* MLP router (Phase 4, "MLP": one hidden layer of d/6 units; the paper does not name its
 * activation, so both are offered): logits = W_out act(W_in x + b_in) + b_out with W_in
 * [hidden x d], b_in [hidden], W_out [E x hidden], b_out [E], device pointers in the layer's dtype.
 * The hidden layer runs on the tensor-core GEMM (fp32 on the fp32 layer) and is kept in fp32; the
 * output layer and the argmax run in fp32 on the routing kernel, so the decision is taken on fp32
 * logits as for the linear router. hidden: a multiple of 16 (bf16) or 4 (fp32), at most H / 2
 * (bf16) or H (fp32): the hidden layer lives in the hidden-state workspace before fc1 runs. */
typedef enum { CLEARMOE_ACT_NONE = -1, CLEARMOE_ACT_RELU = 0, CLEARMOE_ACT_GELU = 1 } clearmoe_act;
typedef struct {
    const void* W_in;
    const void* b_in;
    const void* W_out;
    const void* b_out;
    int32_t hidden;
    int32_t act; /* clearmoe_act */
} clearmoe_mlp_router;

typedef struct clearmoe_layer clearmoe_layer;

/* Allocates the handle and its device workspace on the current device (hidden states
 * [max_tokens x hidden], in bf16 layers no less than the tokens and hidden states in 8-bit blocks,
 * max_tokens (ceil128(d) + ceil128(hidden)) bytes and their scales, nor than 4 hidden bytes for each
 * of up to CLEARMOE_FEW_MAX tokens; basis coefficients [max_tokens x max_r], routing arrays, status word,
 * and for the folded LayerNorm 8 bytes per token of statistics, fp32 row sums [2 hidden + 16] and,
 * in bf16 layers, 128 bytes per token and per hidden unit of fc1's augmentation block).
 * Returns EINVAL for a null/invalid desc, EUNSUPPORTED per the tiling limits above, ENOMEM or
 * ECUDA if allocation fails (nothing is leaked). */
int clearmoe_layer_create(const clearmoe_layer_desc* desc, clearmoe_layer** out);

/* Synchronises the device, frees the workspace and the handle. NULL is accepted. */
int clearmoe_layer_destroy(clearmoe_layer* layer);

/* Routing only (Algorithm 3, steps 3-4): for every token t, a_t = the lowest e maximising
 * the fp32 logit W_g x_t + b_g; counts_e, offsets = exclusive prefix sum of counts (E + 1
 * entries), and perm[slot] = token with the tokens of expert e in slots
 * [offsets_e, offsets_{e+1}) in increasing id order (a stable sort by expert). One fused
 * kernel (logits, argmax, per-range histograms and ranks) and a slot kernel; results stay in
 * the handle (read them with clearmoe_get_routing).
 * 1 <= T <= max_tokens, 1 <= E <= max_E. */
int clearmoe_route(clearmoe_layer* layer, const void* x, int64_t T, const clearmoe_router* router,
                   int32_t E, void* stream);

/* Routing only with the MLP router: its hidden layer (one GEMM launch), then the routing kernel on
 * the fp32 hidden layer with W_out, b_out as the router, then the slot kernel. Same outputs and
 * errors as clearmoe_route; EINVAL for a NULL or misaligned weight, an unknown act or a hidden
 * width outside the limits above. */
int clearmoe_route_mlp(clearmoe_layer* layer, const void* x, int64_t T, const clearmoe_mlp_router* mlp,
                       int32_t E, void* stream);

/* The CLEAR-MoE FFN forward (Eq. 2 with Algorithm 3): routes (as clearmoe_route), computes
 * z = GELU(W1 x + b1) for every token in expert-sorted order (fc1 reads x in token order and its
 * epilogue stores each row at the token's slot), the shared basis through its factors,
 * t = diag(S_r) Vh_r z, and then, per expert sub-batch, out[perm[slot]] = U_r t + residual_e[e] z
 * (the scatter and the sum of the shared and residual terms are folded into the epilogue; each
 * row is written once).
 * residual_e is a HOST array of E device pointers, each to a [d x H] matrix.
 * 1 <= T <= max_tokens, 1 <= E <= max_E, 1 <= r <= min(max_r, d, H). out [T x d] must not
 * alias any input. */
int clearmoe_ffn_forward(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                         const void* b1, const void* U_r, const float* S_r, const void* Vh_r,
                         const void* const* residual_e, const clearmoe_router* router,
                         int32_t E, int32_t r, void* out, void* stream);

/* Deployment options of clearmoe_ffn_forward_ex (zero-initialise, then set the fields used).
 *  b2          fc2's bias [d] in the layer dtype (device), added once to every output row; NULL:
 *              none (Eq. 2 as printed has no fc2 bias; a pretrained ViT layer has one).
 *  cls_stride  > 0: token t with t % cls_stride == 0 is a class token (cls_stride = tokens per
 *              image, 197 for a 224 px ViT at patch 16, the class token first): it skips the router
 *              and takes the dense path out_t = W2 z_t (+ b2), as the dispatch benchmark keeps the
 *              class token out of expert dispatch. The class tokens form group E after the experts:
 *              idx = E, counts[E] = n_cls = ceil(T / cls_stride), slots [T - n_cls, T) in token
 *              order. Requires W2 and E + 1 <= 16 (EUNSUPPORTED otherwise). 0: every token routed.
 *  W2          the layer's dense fc2 [d x H] row-major (device), read for class tokens only.
 *  mlp_router  the MLP router in place of the linear one (see clearmoe_mlp_router).
 *  input_layernorm  non-zero: x is the un-normalised residual stream y of a ViT block, and the
 *              sublayer's input is its per-token LayerNorm without affine, LN(y) = (y - mean) /
 *              sqrt(biased variance + 1e-6), as clearmoe_layer_norm computes it (a pretrained
 *              block's LN affine folds into W1, b1 and the router offline). LN(y) is never
 *              written: one launch forms (mean, rstd) per token and the row sums c = W 1 of W1 and
 *              of the router's first matrix (W_g, or the MLP router's W_in), and the router and fc1
 *              use W LN(y) = rstd (W y - mean c) on their fp32 accumulators. 0: x is the input.
 *  router_in_fc1  non-zero: the linear router's logits (Phase 4 "Linear", Algorithm 3 step 3) are
 *              computed inside fc1 from the token tiles fc1 has already loaded (one more 256 x 32
 *              MMA unit per 256-token tile, W_g as its B operand), so the tokens are read from HBM
 *              once for both; fc1 stores z in token order, a slot kernel forms counts, offsets,
 *              perm and inv from per-128-token-range counts and ranks, the basis factor stores t at
 *              each token's slot, and the grouped GEMM gathers z rows by perm (TMA four-row
 *              gathers). Same results as the default path (expert indices bit-exact outside near
 *              ties, outputs within the tolerance). bf16 layers with the 2-SM kernels only (H a
 *              multiple of 128 and <= 4096, d a multiple of 128), the linear router, and neither
 *              class tokens, the MLP router, input_layernorm nor the materialised basis:
 *              EUNSUPPORTED otherwise. Works with clearmoe_ffn_forward_ex (factorised basis) and
 *              clearmoe_ffn_forward_folded_ex. */
typedef struct {
    const void* b2;
    int64_t cls_stride;
    const void* W2;
    const clearmoe_mlp_router* mlp_router; /* non-NULL: routes with it (router may then be NULL) */
    int32_t input_layernorm;
    int32_t router_in_fc1;
} clearmoe_ffn_options;

/* clearmoe_ffn_forward with deployment options (opt may be NULL: then identical to it). With
 * class tokens the basis step covers the routed slots only and the grouped GEMM has E + 1 groups,
 * the last one z x W2^T alone. EINVAL for cls_stride < 0 or > 2^30, a misaligned b2 or W2, or a
 * NULL W2 with cls_stride > 0. */
int clearmoe_ffn_forward_ex(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                            const void* b1, const void* U_r, const float* S_r, const void* Vh_r,
                            const void* const* residual_e, const clearmoe_router* router,
                            int32_t E, int32_t r, const clearmoe_ffn_options* opt, void* out,
                            void* stream);

/* The shared basis folded into the experts (Eq. 2 regrouped; the paper materialises W_shared in
 * Phase 3): W_comb[e] = U_r diag(S_r) Vh_r + residual_e[e] for e < E, so that the layer output is
 * y_t = W_comb[a_t] GELU(W1 x_t + b1). W_shared is formed in fp32 (products in fp32, summed over
 * k ascending) and each sum is rounded once to the layer dtype. W_comb is a HOST array of E
 * caller-owned device buffers, each [d x H] row-major like residual_e; computed once per weight
 * set, it replaces the basis step of every later forward. Arguments as clearmoe_ffn_forward. */
int clearmoe_fold_basis(clearmoe_layer* layer, const void* U_r, const float* S_r, const void* Vh_r,
                        const void* const* residual_e, int32_t E, int32_t r, void* const* W_comb,
                        void* stream);

/* The CLEAR-MoE FFN forward on folded weights: routing and fc1 as clearmoe_ffn_forward, then per
 * expert sub-batch out[perm[slot]] = W_comb[e] z in one grouped GEMM (no basis step: the dense
 * FFN's arithmetic plus the routing). Same limits and errors as clearmoe_ffn_forward. */
int clearmoe_ffn_forward_folded(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                                const void* b1, const void* const* W_comb,
                                const clearmoe_router* router, int32_t E, void* out, void* stream);

/* clearmoe_ffn_forward_folded with the deployment options of clearmoe_ffn_forward_ex (fc2 bias,
 * class tokens on the dense path W2, the MLP router); opt may be NULL. Same errors as
 * clearmoe_ffn_forward_ex. */
int clearmoe_ffn_forward_folded_ex(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                                   const void* b1, const void* const* W_comb,
                                   const clearmoe_router* router, int32_t E,
                                   const clearmoe_ffn_options* opt, void* out, void* stream);

/* The paper's own form of the shared basis (Phase 3 text: W_shared materialised before
 * inference): W_sh = U_r diag(S_r) Vh_r as one [d x H] row-major matrix in the layer dtype, formed
 * in fp32 (products in fp32, summed over k ascending) and rounded once. W_sh is a caller-owned
 * device buffer. 1 <= r <= min(max_r, d, H). */
int clearmoe_materialize_basis(clearmoe_layer* layer, const void* U_r, const float* S_r, const void* Vh_r,
                               int32_t r, void* W_sh, void* stream);

/* The CLEAR-MoE FFN forward with the materialised basis (Eq. 2 as the paper computes it):
 * routing and fc1 as clearmoe_ffn_forward, then per expert sub-batch out[perm[slot]] =
 * W_sh z + residual_e[e] z in one grouped GEMM whose K chain is [z | z] x [W_e^res | W_sh]
 * (2 d H multiply-adds per token there, against d (H + r) + r H factorised). Same limits and
 * errors as clearmoe_ffn_forward_folded. */
int clearmoe_ffn_forward_materialized(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                                      const void* b1, const void* W_sh, const void* const* residual_e,
                                      const clearmoe_router* router, int32_t E, void* out, void* stream);

/* clearmoe_ffn_forward_materialized with the deployment options of clearmoe_ffn_forward_ex; opt
 * may be NULL. Same errors as clearmoe_ffn_forward_ex. */
int clearmoe_ffn_forward_materialized_ex(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                                         const void* b1, const void* W_sh, const void* const* residual_e,
                                         const clearmoe_router* router, int32_t E,
                                         const clearmoe_ffn_options* opt, void* out, void* stream);

/* The residual structure of Algorithm 2 exploited: its residual experts are scaled copies of one
 * matrix, W_e^res = s_e R with R = W2 - W_shared, so y_t = W_shared z_t + s_{a_t} R z_t =
 * s_{a_t} (U_r t'_t + R z_t) with t'_t = diag(S_r) Vh_r z_t / s_{a_t}. Routing (idx), fc1, the
 * basis factor (column scale S_r and row scale 1 / s_a) and one GEMM with the K chain
 * [z | t'] x [R | U_r] and row scale s_a, all in token order: no sort, no scatter, one residual
 * matrix instead of E. Exact (up to rounding) only for residuals of that form; s_e [E] fp32
 * device, every s_e finite and non-zero (Algorithm 2's are ratios of mean norms, positive), else
 * the rows of that expert are not finite. R [d x H] row-major in the layer dtype. counts, offsets
 * and perm are still produced (after the output) for clearmoe_get_routing. Errors as
 * clearmoe_ffn_forward. */
int clearmoe_ffn_forward_scaled(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                                const void* b1, const void* U_r, const float* S_r, const void* Vh_r,
                                const void* R, const float* s_e, const clearmoe_router* router,
                                int32_t E, int32_t r, void* out, void* stream);

/* The dense FFN the layer was converted from, on the same device: out = W2 GELU(W1 x + b1)
 * (the comparison path; no bias on fc2, as in Eq. 2). 1 <= T <= max_tokens. */
int clearmoe_dense_ffn_forward(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                               const void* b1, const void* W2, void* out, void* stream);

/* The dense FFN with fc2's bias: out = W2 GELU(W1 x + b1) + b2, b2 [d] in the layer dtype
 * (NULL: as clearmoe_dense_ffn_forward). */
int clearmoe_dense_ffn_forward_ex(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                                  const void* b1, const void* W2, const void* b2, void* out,
                                  void* stream);

/* The dense FFN with the options of clearmoe_ffn_forward_ex that apply to it: b2 (as
 * clearmoe_dense_ffn_forward_ex) and input_layernorm (x is y; LN(y) folded into fc1 as there).
 * opt may be NULL. EINVAL for cls_stride != 0 or a non-NULL mlp_router; opt->W2 is not read. */
int clearmoe_dense_ffn_forward_opt(clearmoe_layer* layer, const void* x, int64_t T, const void* W1,
                                   const void* b1, const void* W2, const clearmoe_ffn_options* opt,
                                   void* out, void* stream);

/* Per-token LayerNorm without affine between stacked sublayers: x_out = (y - mean(y)) /
 * sqrt(var(y) + 1e-6), biased variance, fp32 statistics; y and x_out [T x d] in the layer's
 * dtype (they may alias). 1 <= T <= max_tokens. */
int clearmoe_layer_norm(clearmoe_layer* layer, const void* y, int64_t T, void* x_out,
                        void* stream);

/* Copies (device to device, on `stream`) the routing of the last clearmoe_route /
 * clearmoe_ffn_forward on this handle: idx [T], counts [G], offsets [G + 1], perm [T], all
 * int32 device pointers, G = E (E + 1 when that forward had class tokens: group E is theirs);
 * any may be NULL to skip it. EINVAL if no forward has run yet. */
int clearmoe_get_routing(clearmoe_layer* layer, int32_t* idx, int32_t* counts, int32_t* offsets,
                         int32_t* perm, void* stream);

/* Synchronises the device, returns the handle's device status word (CLEARMOE_OK or the first
 * device-side error since the last call, e.g. CLEARMOE_ETIMEOUT) and clears it; after an error it
 * also clears the handle's split-K arrival counters, which a GEMM that gave up may have left
 * part-counted, so that the next calls run on a consistent handle. */
int clearmoe_layer_status(clearmoe_layer* layer);

/* Fault injection for tests of the bounded waits: every device-side wait of the handle's kernels
 * gives up after wait_limit_ns nanoseconds (default 1e9, at least 1,000; the hardware may suspend a
 * wait for some microseconds before the limit is looked at) and, when phantom_arrivals > 0, the
 * bf16 routing withholds the copy of its first stage (the first K blocks of its first 128-row block,
 * in its first CTA), so that the MMA warp's wait for it runs out and the call reports
 * CLEARMOE_ETIMEOUT through clearmoe_layer_status. A kernel that gave up lets its copies in flight
 * land before it exits, and the layer stays usable. phantom_arrivals = 0 restores normal use. */
int clearmoe_debug_set_wait(clearmoe_layer* layer, int64_t wait_limit_ns, int32_t phantom_arrivals);

/* Per-stage timing: when n >= 5, clearmoe_ffn_forward records events[0] before its first kernel
 * and events[i] after its i-th kernel (1 routing, 2 fc1 + GELU, 3 shared-basis factor, 4 grouped
 * residual GEMM); clearmoe_dense_ffn_forward records events[0..2] around its two kernels. The
 * events are cudaEvent_t handles owned by the caller, recorded on the call's stream; n = 0 (or
 * events = NULL) turns recording off. The library never waits on them. */
int clearmoe_set_profile_events(clearmoe_layer* layer, void* const* events, int32_t n);

/* Routing without a handle, for callers that cannot allocate device memory (engines that own
 * every device byte and forbid allocation in their enqueue path, processes held to a fixed
 * memory budget, loops that cannot afford cudaMalloc's implicit device synchronisation). The
 * paper has no counterpart: this is a deployment variant of clearmoe_route, with the same results
 * (idx [T], counts [E], offsets [E + 1], perm [T]: caller-owned int32 device outputs) for tokens
 * x [T x d] of dtype `dtype` and the router W [E x d], b [E] in that dtype.
 *   - It calls no cudaMalloc, cudaFree or other allocating routine. Its scratch (per-CTA expert
 *     histograms and a spare status word) is one static device array of 65,600 bytes that every
 *     GPU loading the library holds until exit; it serves up to 1,024 routing CTAs (two per SM on
 *     GPUs with up to 512 SMs). A launch that would need more returns CLEARMOE_EUNSUPPORTED and
 *     enqueues nothing. Between its two kernels idx holds packed per-token words; the second
 *     kernel leaves the experts there.
 *   - The first call on a device looks up the array's device address (once per device, with that
 *     device current); make that first call before any stream capture.
 *   - Every call shares the array and it keeps the last call's contents; each call clears what
 *     must start at zero (the caller's status word; the histograms are rewritten before they are read).
 *     Calls whose work overlaps on the GPU (other streams, other host threads) race on the
 *     array: serialise them.
 *   - Its first kernel may start while the kernel enqueued just before it on the same stream is
 *     finishing, but reads nothing before that kernel has completed: x, W and b may be its output.
 *   - status (optional int32 device pointer, else NULL) is set to 0 at the start of the call and
 *     receives CLEARMOE_ETIMEOUT if a bounded device-side wait (1 s) runs out, in which case the
 *     outputs are undefined.
 * Limits: 1 <= T <= 2^30, 1 <= E <= 16; bf16: d % 64 == 0, d <= 1024; fp32: d % 4 == 0, d <= 512;
 * x and W 16-byte aligned. Host-side errors return EINVAL / EUNSUPPORTED / ECUDA with nothing
 * enqueued. */
int clearmoe_route_noalloc(const void* x, int64_t T, int32_t d, int32_t dtype,
                           const clearmoe_router* router, int32_t E, int32_t* idx, int32_t* counts,
                           int32_t* offsets, int32_t* perm, int32_t* status, void* stream);

/* ---- 8-bit floating point with one scale per block of 128 ----
 *
 * A matrix [rows x cols] in e4m3 with power-of-two scales: value = e4m3(q) 2^(s - 127).
 *   q      one byte per element, row-major, rows of cols rounded up to a multiple of 128 bytes; the bytes past
 *          cols are zero (the quantising calls write them; in a block that is NaN they may be anything). 32-byte
 *          aligned.
 *   scale  one byte s per block, row-major, rows of 4 ceil(cols / 512) bytes, of which the first
 *          ceil(cols / 128) are used. 4-byte aligned. Blocks are 128 columns wide; those of activations one
 *          row high (rows scale rows), those of weights 128 rows (ceil(rows / 128) scale rows).
 * The quantising calls give each block the least s with max |value| <= 448 2^(s - 127) (448: e4m3's largest
 * value; s = 0 at the least) and round value 2^(127 - s) to nearest even. A block with an infinity or a NaN
 * gets s = 255, which stands for NaN: every value of the block, and every output that depends on it, is NaN.
 * Scales are powers of two so that the tensor cores apply them inside the product, exactly.
 * Both buffers are the caller's. rows <= 2^30, cols <= 2^24. */
typedef struct {
    void* q;
    uint8_t* scale;
    int64_t rows;
    int64_t cols;
} clearmoe_fp8;

/* Activations x [out->rows x out->cols] (dtype CLEARMOE_F32 or CLEARMOE_BF16, rows ld elements apart, ld >=
 * cols, any alignment of the element type) to 1 x 128 blocks. gather (nullable, int32 [out->rows], device): row
 * i is x's row gather[i] instead; every entry must be a row of x, which this call cannot check (the next one does).
 * No handle; stream-ordered; x may be the preceding kernel's output. */
int clearmoe_fp8_quantize_rows(const void* x, int32_t dtype, int64_t ld, const int32_t* gather, const clearmoe_fp8* out,
                               void* stream);

/* The same with the number of x's rows: of an entry of gather outside [0, x_rows) nothing is read, and the row is NaN
 * (s = 255). x_rows >= 1, and at least out->rows without gather. */
int clearmoe_fp8_quantize_gathered(const void* x, int64_t x_rows, int32_t dtype, int64_t ld, const int32_t* gather,
                                   const clearmoe_fp8* out, void* stream);

/* A weight matrix W [out->rows x out->cols] to 128 x 128 blocks; arguments as above. Once per weight set. */
int clearmoe_fp8_quantize_weight(const void* W, int32_t dtype, int64_t ld, const clearmoe_fp8* out, void* stream);

/* The values that a matrix stands for, rounded once to dtype: out [rows x cols], rows ld elements apart.
 * block_rows: 1 for activations, 128 for weights. */
int clearmoe_fp8_dequantize(const clearmoe_fp8* in, int32_t block_rows, void* out, int32_t dtype, int64_t ld, void* stream);

/* What follows the product: + bias[n] (nullable, [N] of bias_dtype F32 or BF16, device), then the activation.
 * status (nullable, int32, device): receives CLEARMOE_ETIMEOUT if a bounded device-side wait (1 s) runs out, in
 * which case the outputs are undefined; the call does not clear it. */
typedef struct {
    const void* bias;
    int32_t bias_dtype;
    int32_t act; /* clearmoe_act */
    int32_t* status;
} clearmoe_fp8_epilogue;

/* out = act(A W^T + bias): A [M x K] activations, W [N x K] weights (A->cols == W->cols), products of e4m3 values
 * and the scales exact, sums in fp32 (the tensor cores cut where fp32 additions would round), the result rounded once to out_dtype (F32 or BF16) and stored at
 * out [M x N], rows ldo elements apart (ldo >= N, any alignment of the element type). epi may be NULL (no bias, no
 * activation). N <= 2^24. No handle and no workspace; stream-ordered; out must not alias an input. */
int clearmoe_fp8_gemm(const clearmoe_fp8* A, const clearmoe_fp8* W, const clearmoe_fp8_epilogue* epi, void* out,
                      int32_t out_dtype, int64_t ldo, void* stream);

/* The same with the fp32 result quantised as clearmoe_fp8_quantize_rows would: out [M x N] in 8-bit blocks, the
 * next product's activations, without its intermediate in memory. */
int clearmoe_fp8_gemm_fp8(const clearmoe_fp8* A, const clearmoe_fp8* W, const clearmoe_fp8_epilogue* epi,
                          const clearmoe_fp8* out, void* stream);

/* Grouped by expert: rows [offsets[e], offsets[e + 1]) of A (offsets: int32 [E + 1], device, ascending from 0 to
 * A->rows; an expert may have none) times W[e]^T (host array of E matrices of the same shape); row i goes to
 * row perm[i] of out (perm: nullable int32 [M], device; a permutation). 1 <= E <= 16. */
int clearmoe_fp8_grouped_gemm(const clearmoe_fp8* A, const clearmoe_fp8* W, int32_t E, const int32_t* offsets,
                              const int32_t* perm, const clearmoe_fp8_epilogue* epi, void* out, int32_t out_dtype,
                              int64_t ldo, void* stream);

/* For tests: every later product of 8-bit blocks that the calling thread asks for takes the tcgen05 kernel of this
 * tile width, on pairs of SMs (pair 1: 256, 192, 128) or single ones (pair 0: 192, 128, 64, 32), or the kernel for few
 * rows (16, 0), where the rows and the output allow it (8-bit outputs: a multiple of 128); (0, 0) restores the choice
 * by size. EINVAL for another kernel. */
int clearmoe_debug_fp8_kernel(int32_t width, int32_t pair);

/* The weights of a folded layer (clearmoe_fold_basis), bound once and passed to each of the two forwards below.
 *  dtype            of W1, W_comb and W2: the layer's own, or CLEARMOE_FP8 (a bf16 layer's weights in 8-bit
 *                   blocks). With the layer's own dtype only the q of each matrix is read, a dense row-major
 *                   matrix (16-byte aligned); rows and cols must say its shape in any case.
 *  W1 [H x d], W_comb[e] [d x H] for e < E; b1 [H] and the linear router in the layer's dtype.
 *  b2, cls_stride, W2 ([d x H], read with cls_stride > 0 only), input_layernorm: as clearmoe_ffn_options. */
typedef struct {
    int32_t dtype;
    int32_t E;
    clearmoe_fp8 W1;
    clearmoe_fp8 W2;
    clearmoe_fp8 W_comb[16];
    const void* b1;
    const void* b2;
    clearmoe_router router;
    int64_t cls_stride;
    int32_t input_layernorm;
} clearmoe_ffn_weights;

/* The whole folded layer for a few tokens, 1 <= T <= CLEARMOE_FEW_MAX: y_t = W_comb[a_t] GELU(W1 x_t + b1)
 * (+ b2), a_t as clearmoe_route's, in two launches: one takes every token through the router and fc1, the other
 * through its expert. Of an expert without a token at most the first columns and the scales are read, asked for
 * before the routing is known, so every matrix has to be readable. The linear router only. Weights of the layer's
 * dtype or 8-bit blocks (bf16 layers; the weights' values times unquantised activations). Sums in fp32; z is stored in
 * the layer's dtype as in the other forwards, of up to 16 tokens of bf16 layers in two bf16 parts (16 bits of
 * significand); fp32 layers use three TF32 products per term (relative error near 2^-21; NaN for an infinity and for a
 * magnitude past TF32's largest value, 3.4e38, whose remainder is not finite). The routing can be read with
 * clearmoe_get_routing. Errors as clearmoe_ffn_forward_folded_ex; EUNSUPPORTED for more tokens, and for 8-bit weights
 * with hidden > 589,824. */
#define CLEARMOE_FEW_MAX 64
int clearmoe_ffn_forward_few(clearmoe_layer* layer, const void* x, int64_t T, const clearmoe_ffn_weights* w, void* out,
                             void* stream);

/* The whole folded layer of a bf16 handle with both products in 8-bit blocks (w->dtype CLEARMOE_FP8): the
 * tokens routed in bf16 as clearmoe_route, x (after the LayerNorm, with input_layernorm) quantised in expert
 * order, z = GELU(W1 x + b1) quantised in fc1's epilogue, out = W_comb[a] z (+ b2) in bf16. 1 <= T <= max_tokens.
 * Errors as clearmoe_ffn_forward_folded_ex; EUNSUPPORTED for fp32 handles and other weight types. */
int clearmoe_ffn_forward_fp8(clearmoe_layer* layer, const void* x, int64_t T, const clearmoe_ffn_weights* w, void* out,
                             void* stream);

/* ---- 4-bit floating point with one scale per 32 columns of a row ----
 *
 * A matrix [rows x cols] in e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with power-of-two scales, activations
 * and weights alike: value = e2m1(q) 2^(s - 127).
 *   q      two codes a byte, the column of even number in the low half, row-major, rows of 32 ceil(cols / 64) bytes; the
 *          codes past cols are zero (the quantising calls write them; in a block that is NaN they may be anything). 32-byte
 *          aligned.
 *   scale  one byte s per block of 32 columns of one row, in tiles of 128 rows x 128 columns: ceil(rows / 128) rows of
 *          ceil(cols / 128) tiles, 512 bytes each, in which the byte of row r and block b (r < 128, b < 4 within the tile)
 *          is byte 16 (r % 32) + 4 (r / 32) + b, as the tensor cores take them. 32-byte aligned. Bytes of rows past the
 *          last and of blocks at or past 2 ceil(cols / 64) are not used and may be anything; that of a block past cols
 *          before there may be any but 255 (the quantising calls write 0).
 * The quantising calls give each block the least s with max |value| <= 6 2^(s - 127) (6: e2m1's largest value; s = 0 at
 * the least) and round value 2^(127 - s) to nearest even. A block with an infinity or a NaN gets s = 255, which stands
 * for NaN: every value of the block, and every output that depends on it, is NaN.
 * Both buffers are the caller's. rows <= 2^30, cols <= 2^24. */
typedef struct {
    void* q;
    uint8_t* scale;
    int64_t rows;
    int64_t cols;
} clearmoe_fp4;

/* x [x_rows x out->cols] (dtype CLEARMOE_F32 or CLEARMOE_BF16, rows ld elements apart, ld >= cols, any alignment of the
 * element type) to 4-bit blocks: activations before a product, weights once per set. gather (nullable, int32
 * [out->rows], device): row i is x's row gather[i] instead; of an entry outside [0, x_rows) nothing is read, and the row
 * is NaN (s = 255). x_rows >= 1, and at least out->rows without gather. No handle; stream-ordered; x may be the preceding
 * kernel's output. */
int clearmoe_fp4_quantize(const void* x, int64_t x_rows, int32_t dtype, int64_t ld, const int32_t* gather,
                          const clearmoe_fp4* out, void* stream);

/* The values that a matrix stands for, rounded once to dtype: out [rows x cols], rows ld elements apart. */
int clearmoe_fp4_dequantize(const clearmoe_fp4* in, void* out, int32_t dtype, int64_t ld, void* stream);

/* out = act(A W^T + bias): A [M x K], W [N x K] (A->cols == W->cols), products of e2m1 values and the scales exact, sums in
 * fp32 (the tensor cores cut where fp32 additions would round), the result rounded once to out_dtype (F32 or BF16) and
 * stored at out [M x N], rows ldo elements apart (ldo >= N, any alignment of the element type). epi may be NULL (no bias,
 * no activation); its status as in the 8-bit products. The GELU is a kind of output's own, the same at every size:
 * before the rounding within 2.5e-7 of the exact one to fp32 and within 3.2e-7 to bf16 and 4-bit blocks, or half a step of
 * fp32 where that is more; NaN and -inf give NaN, as u (1 + erf(u / sqrt 2)) / 2 does, and inf gives inf. N <= 2^24. No
 * handle and no workspace; stream-ordered; out must not alias an input. */
int clearmoe_fp4_gemm(const clearmoe_fp4* A, const clearmoe_fp4* W, const clearmoe_fp8_epilogue* epi, void* out,
                      int32_t out_dtype, int64_t ldo, void* stream);

/* The same with the fp32 result (the GELU as said) quantised as clearmoe_fp4_quantize would: out [M x N] in 4-bit blocks,
 * the next product's activations, without its intermediate in memory. */
int clearmoe_fp4_gemm_fp4(const clearmoe_fp4* A, const clearmoe_fp4* W, const clearmoe_fp8_epilogue* epi,
                          const clearmoe_fp4* out, void* stream);

/* Grouped by expert: rows [offsets[e], offsets[e + 1]) of A (offsets: int32 [E + 1], device, ascending from 0 to
 * A->rows; an expert may have none) times W[e]^T (host array of E matrices of the same shape); row i goes to
 * row perm[i] of out (perm: nullable int32 [M], device; a permutation). 1 <= E <= 16. */
int clearmoe_fp4_grouped_gemm(const clearmoe_fp4* A, const clearmoe_fp4* W, int32_t E, const int32_t* offsets,
                              const int32_t* perm, const clearmoe_fp8_epilogue* epi, void* out, int32_t out_dtype,
                              int64_t ldo, void* stream);

/* For tests: every later product of 4-bit blocks that the calling thread asks for takes the tcgen05 kernel of this tile
 * width on pairs of SMs (pair 1: 256, 128) or single ones (pair 0: 128, 64), or the kernel for up to 128 rows (16, 0)
 * where the product is not grouped; (0, 0) restores the choice by size. EINVAL for another kernel. */
int clearmoe_debug_fp4_kernel(int32_t width, int32_t pair);

/* For tests of the bounded waits: those of the calling thread's later products of 4-bit blocks run out after
 * wait_limit_ns nanoseconds; 0 restores 1 s. EINVAL below 0 and above 1 s. */
int clearmoe_debug_fp4_wait(int64_t wait_limit_ns);

/* ---- a residual's addition and the root-mean-square norm of the sum ----
 *
 * s = x + residual, rounded to dtype, is the stream as it goes on; its norm y = s weight / sqrt(mean(s^2) + eps) feeds the
 * next sublayer. Sums and statistics in fp32, y rounded once. Squares and their sum may leave fp32's range where s and the mean
 * square do not: a row is zero where its mean square is past the range, and with eps 0 NaN where it is all zeros, no others.
 *  x, residual (nullable: s = x), sum (nullable: s is not stored) [rows x cols] of dtype (F32 or BF16), rows ldx, ldr and
 *  lds elements apart; weight (nullable: ones) [cols] of weight_dtype; eps >= 0.
 * Every tensor may start anywhere that its element type allows. sum may be x or residual (with the same pitch), and out
 * may be x or residual (of the same dtype and pitch) where sum is not; they must not overlap otherwise. 1 <= rows <= 2^30,
 * 1 <= cols <= CLEARMOE_NORM_MAX (EUNSUPPORTED above). No handle; stream-ordered; reads nothing before the preceding kernel
 * has completed. */
#define CLEARMOE_NORM_MAX 32768
typedef struct {
    const void* x;
    const void* residual;
    void* sum;
    const void* weight;
    int64_t ldx, ldr, lds;
    int64_t rows, cols;
    int32_t dtype;
    int32_t weight_dtype;
    float eps;
} clearmoe_norm;

/* y to out [rows x cols] of out_dtype, rows ldo elements apart. */
int clearmoe_rms_norm(const clearmoe_norm* n, void* out, int32_t out_dtype, int64_t ldo, void* stream);

/* y to 8-bit blocks of activations, as clearmoe_fp8_quantize_rows would make them of the fp32 y. */
int clearmoe_rms_norm_fp8(const clearmoe_norm* n, const clearmoe_fp8* out, void* stream);

/* y to 4-bit blocks, as clearmoe_fp4_quantize would make them of the fp32 y. */
int clearmoe_rms_norm_fp4(const clearmoe_norm* n, const clearmoe_fp4* out, void* stream);

/* Static string for a status code. */
const char* clearmoe_strerror(int status);

/* Library version as MAJOR * 10000 + MINOR * 100 + PATCH. */
int clearmoe_version(void);

#ifdef __cplusplus
}
#endif

#endif /* CLEARMOE_H */
