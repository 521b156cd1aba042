/*
 * moce.h -- C ABI of the MI355X (gfx950) Mixture of Channel Experts forward
 * pass (arxiv 2608.23794, "Mixture of Channel Experts: Static Sparse Supports
 * with Input-Adaptive Mixing for Pointwise Projections").
 *
 * A MoCE layer replaces a pointwise projection from C input channels to E <= C
 * outputs (Sec. 3.1): E-1 routed experts, each a convex mixture of k input
 * channels on a static support (Sec. 3.2-3.3), plus one residual output that
 * averages the channels outside every support (Sec. 3.4, Eq. 6).
 *
 * Conventions shared by every entry point
 *  - The descriptor and gate structs are host memory; every array argument is
 *    a device pointer (hipMalloc'd or otherwise device-accessible) unless its
 *    name ends in _host.  The caller owns all memory.  The library never
 *    allocates device memory and keeps no pointer after a call returns.
 *  - Every call except moce_support_prepare is asynchronous on `stream`
 *    (0 = the null stream) and returns as soon as its kernels are enqueued.
 *  - Layouts: MOCE_NCHW is x[B][C][H][W] and y[B][E][H][W]; MOCE_NHWC is
 *    x[B][H][W][C] and y[B][H][W][E].  Token inputs x[B][N][C] are MOCE_NHWC
 *    with H = N, W = 1.  y always has the layout and element type of x.
 *  - Element types: x and y are both MOCE_F32 or both MOCE_BF16 (bfloat16 bit
 *    patterns, 2 bytes).  Accumulation is float32 throughout; bf16 outputs are
 *    rounded to nearest, ties to even.  d, tau, alpha and all parameters are
 *    float32; supports are int32 channel indices.
 *  - Output channel E-1 is the residual expert; channels 0..E-2 are the routed
 *    experts in support-row order.
 *  - x and y must be 16-byte aligned.
 *  - Errors are negative moce_status codes.  Every error detectable on the host
 *    is reported before anything is enqueued, and then no output is written.
 *    A failed kernel launch returns MOCE_ERR_DEVICE.  The library holds no
 *    mutable global state; calls on different streams are independent as long
 *    as their output buffers do not overlap.
 */
#ifndef MOCE_H
#define MOCE_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum moce_status {
    MOCE_OK = 0,
    MOCE_ERR_NULL = -1,        /* a required pointer is NULL */
    MOCE_ERR_SHAPE = -2,       /* B, C, H, W < 1; E outside [1, C]; k outside [1, C] */
    MOCE_ERR_DTYPE = -3,       /* unknown element type or x/y types differ */
    MOCE_ERR_LAYOUT = -4,      /* unknown layout code */
    MOCE_ERR_SUPPORT = -5,     /* a support row is invalid (moce_support_prepare) */
    MOCE_ERR_GATE = -6,        /* unknown gate kind, or tau_min/tau_max invalid */
    MOCE_ERR_WORKSPACE = -7,   /* workspace NULL or smaller than required */
    MOCE_ERR_ALIGN = -8,       /* x or y not 16-byte aligned */
    MOCE_ERR_DEVICE = -9,      /* a HIP call or kernel launch failed */
    MOCE_ERR_UNSUPPORTED = -10 /* the shape exceeds a documented size limit */
} moce_status;

enum { MOCE_F32 = 0, MOCE_BF16 = 1 };
enum { MOCE_NCHW = 0, MOCE_NHWC = 1 };

/* Gate kinds.  Both read the k descriptors of an expert's support in
 * canonical order (descending routing logit), so gate position i is the
 * expert's i-th most preferred channel (Sec. 3.3).
 *  MOCE_GATE_SOFTPLUS_LINEAR: tau[b][o] = softplus(c[o] + sum_i a[o][i] d[b][s[o][i]]) + 1e-3,
 *     a per-expert linear gate (a: [E-1][k], c: [E-1]).
 *  MOCE_GATE_MLP_SIGMOID: the paper's gate (Sec. 3.3 Eq. 3): one two-layer MLP
 *     of hidden width k shared by all experts of the layer,
 *     h = ReLU(W1 z + b1), g = w2 . h + b2,
 *     tau = tau_min + (tau_max - tau_min) sigmoid(g)
 *     (W1: [k][k] row-major, row j feeds hidden unit j; b1, w2: [k]). */
enum { MOCE_GATE_SOFTPLUS_LINEAR = 0, MOCE_GATE_MLP_SIGMOID = 1 };

typedef struct moce_desc {
    int64_t B, C, H, W;   /* x is B images of C channels over H*W positions */
    int32_t E;            /* outputs: E-1 routed experts + 1 residual, 1 <= E <= C */
    int32_t k;            /* support size, 1 <= k <= C */
    int32_t x_dtype;      /* MOCE_F32 or MOCE_BF16 */
    int32_t y_dtype;      /* must equal x_dtype */
    int32_t layout;       /* MOCE_NCHW or MOCE_NHWC */
    int32_t reserved;     /* set to 0 */
} moce_desc;

typedef struct moce_gate_params {
    int32_t kind;         /* MOCE_GATE_* */
    int32_t reserved;     /* set to 0 */
    const float* a;       /* softplus-linear: [E-1][k] slopes, canonical positions */
    const float* c;       /* softplus-linear: [E-1] offsets */
    const float* W1;      /* MLP: [k][k] */
    const float* b1;      /* MLP: [k] */
    const float* w2;      /* MLP: [k] */
    float b2;             /* MLP: output bias */
    float tau_min;        /* MLP: lower temperature bound, > 0 */
    float tau_max;        /* MLP: upper temperature bound, >= tau_min */
} moce_gate_params;

/* Static support preparation (Sec. 3.2 Eq. 2: supports fixed at inference;
 * Sec. 3.3: gate input order; Sec. 3.4: the uncovered set U).
 *
 * In:  s[E-1][k] int32 channel indices and w[E-1][k] float32 selected routing
 *      logits, one row per routed expert, in any order.
 * Out: s_out, w_out [E-1][k]: each row sorted by logit descending, equal
 *      logits by ascending channel (the canonical order every other entry
 *      point expects); covered[C] uint8: 1 if the channel is in some support;
 *      U[C] int32: the uncovered channels ascending in U[0..nU-1] (the rest
 *      is left unspecified); info[2] int32 device scratch receiving
 *      {nU, first bad expert or -1}; *nU_host and *bad_expert_host receive the
 *      same two values.
 * A row is invalid if a channel lies outside [0, C), repeats within the row,
 * or its logit is not finite; the call then returns MOCE_ERR_SUPPORT with
 * *bad_expert_host = the lowest invalid expert (outputs other than info and
 * the two host values are unspecified).  s_out/w_out may not alias s/w.
 * This call synchronises `stream` once (it is a once-per-model step).
 * Limits: C <= 2^24, k <= 4096. */
moce_status moce_support_prepare(const moce_desc* desc, const int32_t* s, const float* w,
                                 int32_t* s_out, float* w_out, uint8_t* covered, int32_t* U,
                                 int32_t* info, int32_t* nU_host, int32_t* bad_expert_host,
                                 hipStream_t stream);

/* moce_support_prepare for supports kept in the deployment storage format:
 * s[E-1][k] as 16-bit unsigned channel indices (Sec. 3.5, Storage: a
 * deployed layer keeps its (E-1)k selected logits, their indices in 16 bits
 * and the gate).  Same outputs (int32 prepared rows), checks and errors;
 * MOCE_ERR_UNSUPPORTED when C > 65536.  This call synchronises `stream`
 * once. */
moce_status moce_support_prepare16(const moce_desc* desc, const uint16_t* s, const float* w,
                                   int32_t* s_out, float* w_out, uint8_t* covered, int32_t* U,
                                   int32_t* info, int32_t* nU_host, int32_t* bad_expert_host,
                                   hipStream_t stream);

/* Global average pooling descriptor z = GAP(x) (Sec. 3.3):
 * d[b][c] = (1 / (H W)) sum over positions of x[b][c][.]; d is [B][C] float32. */
moce_status moce_pool(const moce_desc* desc, const void* x, float* d, hipStream_t stream);

/* Temperatures (Sec. 3.3, Eq. 3 or the softplus-linear form) and mixing
 * coefficients (Eq. 4): tau[b][o] and, if alpha != NULL,
 * alpha[b][o][i] = exp(w[o][i] / tau[b][o]) / sum_j exp(w[o][j] / tau[b][o]).
 * d is [B][C]; s, w are prepared rows; tau is [B][E-1]; alpha is [B][E-1][k].
 * Does nothing when E == 1.  Limits for MOCE_GATE_MLP_SIGMOID: k <= 256. */
moce_status moce_gate(const moce_desc* desc, const float* d, const int32_t* s, const float* w,
                      const moce_gate_params* gate, float* tau, float* alpha, hipStream_t stream);

/* Temperatures, coefficients and mixing in one kernel (Secs. 3.3-3.4): the
 * y of moce_gate followed by moce_mix, bit for bit, from the pooled
 * descriptors d [B][C], without writing tau or alpha.  Each workgroup of the
 * mix evaluates the softplus-linear gate for the experts of the images it
 * mixes.  Only where moce_forward_path(desc, gate->kind) is
 * MOCE_PATH_MFMA_GATE (otherwise MOCE_ERR_UNSUPPORTED); s, w: prepared rows;
 * U, nU as for moce_mix; y is fully overwritten. */
moce_status moce_gate_mix(const moce_desc* desc, const void* x, const float* d, const int32_t* s, const float* w,
                          const moce_gate_params* gate, const int32_t* U, int32_t nU, void* y,
                          hipStream_t stream);

/* Routed outputs (Sec. 3.3 Eq. 5) and residual output (Sec. 3.4 Eq. 6):
 * y[b][o][p] = sum_i alpha[b][o][i] x[b][s[o][i]][p] for o < E-1, and
 * y[b][E-1][p] = (1/nU) sum_{c in U} x[b][c][p], or 0 when nU == 0.
 * s: prepared [E-1][k]; alpha: [B][E-1][k]; U: [nU] uncovered channels with
 * 0 <= nU <= C (U may be NULL when nU == 0).  y is fully overwritten. */
moce_status moce_mix(const moce_desc* desc, const void* x, const int32_t* s, const float* alpha,
                     const int32_t* U, int32_t nU, void* y, hipStream_t stream);

/* Bytes of device workspace moce_forward needs for `desc` (0 on an invalid
 * descriptor).  The workspace holds the descriptor d, the temperatures, the
 * softmax statistics and, depending on the path, the coefficients or the
 * support schedule. */
size_t moce_forward_workspace_bytes(const moce_desc* desc);

/* Paths moce_forward can take. */
enum { MOCE_PATH_GENERIC = 0, MOCE_PATH_TILE = 1, MOCE_PATH_MFMA = 2, MOCE_PATH_MFMA_GATE = 3,
       MOCE_PATH_SCHEDULED = 4, MOCE_PATH_GATHER = 5 };

/* The path moce_forward takes for `desc` (moce_mix takes the same kernels,
 * MOCE_PATH_MFMA for MOCE_PATH_MFMA_GATE, MOCE_PATH_GENERIC for
 * MOCE_PATH_SCHEDULED, the gather for MOCE_PATH_GATHER):
 *  MOCE_PATH_GATHER: channels-last bfloat16 with small supports (k <= 16,
 *     C a multiple of 8 up to 4096, E-1 <= 1024, or 512 for k > 8): pooling, the gate's
 *     coefficients, then a gather whose work scales with k (x staged in LDS
 *     transposed, 8 positions per read);
 *  MOCE_PATH_SCHEDULED: channels-last bfloat16 (C a multiple of 64 up to
 *     4096, E a multiple of 8): pooling, the gate's softmax statistics, then
 *     a schedule of the supports by 64-channel step (Sec. 3.2: static
 *     supports) and the routed and residual outputs as a dense bf16 product
 *     on the matrix cores whose coefficient operand is written step by step
 *     from the schedule (coefficients split into two bf16 parts: 16
 *     significant bits);
 *  MOCE_PATH_MFMA_GATE: MOCE_PATH_MFMA with the softplus-linear gate
 *     evaluated inside the mix kernel, as moce_gate_mix (k = 32);
 *  MOCE_PATH_MFMA: the gate kernel, then the routed and residual outputs of an image as one dense
 *     bf16 matrix product on the matrix cores, the coefficients split into
 *     bf16 parts that sum to them exactly (NCHW bfloat16, E-1 >= 1, C a
 *     multiple of 32 up to 256, E <= 64, H*W a multiple of 8);
 *  MOCE_PATH_TILE: the tile gather kernel (NCHW bfloat16, C <= 256, H*W a
 *     multiple of 8);
 *  MOCE_PATH_GENERIC: the layout- and type-generic kernels.
 * All compute the same values up to float32 rounding order; the MFMA path
 * requires distinct channels within each support row, as
 * moce_support_prepare guarantees.  `gate_kind` must be a valid gate kind.
 * A negative moce_status for an invalid descriptor or gate kind. */
int moce_forward_path(const moce_desc* desc, int gate_kind);

/* The whole layer (Secs. 3.3-3.4): pooling, temperatures, mixing
 * coefficients, routed experts and residual, equal to moce_pool + moce_gate +
 * moce_mix.  s, w: prepared rows; U, nU: as returned by moce_support_prepare;
 * ws: device workspace of at least moce_forward_workspace_bytes(desc) bytes,
 * 256-byte aligned, owned by the caller; its contents on entry are ignored and
 * on return unspecified.  Concurrent calls must use distinct workspaces. */
moce_status moce_forward(const moce_desc* desc, const void* x, const int32_t* s, const float* w,
                         const moce_gate_params* gate, const int32_t* U, int32_t nU, void* y,
                         void* ws, size_t ws_bytes, hipStream_t stream);

/* Output epilogue of moce_forward_ex: each output value v of channel o
 * (routed or residual) becomes act(scale[o] v + shift[o]) before it is
 * rounded and stored, act = ReLU when relu != 0 and the identity otherwise.
 * scale, shift: device float32 [E], both given or both NULL (no affine map).
 * The replaced projection is followed by batch normalisation and the block's
 * nonlinearity, which the paper leaves unchanged (Sec. 4.1); at inference the
 * normalisation is this affine map (scale = gamma / sqrt(var + eps),
 * shift = beta - mean scale), and applying it as the output is written avoids
 * a second pass over y, the memory-traffic fusion Sec. 4.7 points to. */
typedef struct moce_epilogue {
    const float* scale;
    const float* shift;
    int32_t relu;
    int32_t reserved;     /* set to 0 */
} moce_epilogue;

/* moce_forward followed by the epilogue `ep` (NULL: none, then identical to
 * moce_forward).  On the matrix-core paths (MOCE_PATH_MFMA, MOCE_PATH_MFMA_GATE,
 * MOCE_PATH_SCHEDULED) and MOCE_PATH_GATHER the mix kernel applies it to the float32 accumulators
 * before rounding; on the others a second kernel applies it to y in place
 * (for bf16 y, to the rounded value).  Errors: those of moce_forward, and
 * MOCE_ERR_NULL when exactly one of scale and shift is NULL. */
moce_status moce_forward_ex(const moce_desc* desc, const void* x, const int32_t* s, const float* w,
                            const moce_gate_params* gate, const int32_t* U, int32_t nU, const moce_epilogue* ep,
                            void* y, void* ws, size_t ws_bytes, hipStream_t stream);

/* Bytes of the device array that moce_forward_static uses as its workspace. */
#define MOCE_STATIC_SCRATCH_BYTES ((size_t)16 << 20)

/* The whole layer, as moce_forward, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid allocation): no workspace argument and no allocation.  The
 * workspace is a fixed array of MOCE_STATIC_SCRATCH_BYTES inside the library,
 * one per GPU, held from the library's load until the process ends; its
 * device address is looked up on the first call on each device.  Same
 * arguments, kernels and results as moce_forward.  Errors: those of
 * moce_forward, and MOCE_ERR_WORKSPACE (before any launch) when
 * moce_forward_workspace_bytes(desc) exceeds MOCE_STATIC_SCRATCH_BYTES;
 * MOCE_ERR_DEVICE if the array's address cannot be obtained.  Every call on
 * one GPU shares that array: calls that overlap on the same device (on
 * different streams or from different host threads) race, and the caller
 * must serialise them. */
moce_status moce_forward_static(const moce_desc* desc, const void* x, const int32_t* s, const float* w,
                                const moce_gate_params* gate, const int32_t* U, int32_t nU, void* y,
                                hipStream_t stream);

/* Router of the input-conditioned support variant (Sec. 4.5 Eq. 11).  From the
 * pooled descriptor z of an example, h = ReLU(Wh z + bh) (d values), and the
 * example's routing logits are L(X)[e][c] = L[e][c] + sum_t q[e][t] h[t] v[c][t]
 * over the full static routing logits L[E-1][C]. */
typedef struct moce_router {
    int32_t d;            /* bottleneck width, 1 <= d <= 64 */
    int32_t reserved;     /* set to 0 */
    const float* Wh;      /* [d][C] */
    const float* bh;      /* [d] */
    const float* v;       /* [C][d] channel embeddings */
    const float* q;       /* [E-1][d] expert embeddings */
} moce_router;

/* Bytes of device workspace moce_forward_dynamic needs (0 on an invalid
 * descriptor or router width). */
size_t moce_forward_dynamic_workspace_bytes(const moce_desc* desc, int32_t d);

/* The layer with input-conditioned supports (Sec. 4.5 Eq. 11), inference path.
 * Per example b: z = GAP(x_b); L(X) as above; S_e(X) = the k channels of
 * largest L(X)[e][.], equal logits by ascending channel, in canonical order
 * (logit descending, then channel ascending); the gate reads z at S_e(X) in
 * that order (gate position i is the i-th channel of S_e(X)); the
 * coefficients are the softmax of L(X)[e][S_e(X)] over the temperature; the
 * residual output E-1 is the mean of x over U(X), the channels in no
 * S_e(X) of that example (0 when U(X) is empty).
 *
 * x, y as for moce_forward (16-byte aligned, y fully overwritten);
 * L: [E-1][C] float32 device; router: host struct of device pointers;
 * gate: as for moce_forward (gate->a indexed by canonical position);
 * S_out: optional device [B][E-1][k] int32 receiving S_e(X) (NULL: not
 * written); ws: device workspace of at least
 * moce_forward_dynamic_workspace_bytes(desc, router->d) bytes, 256-byte
 * aligned, contents on return unspecified.
 * Errors: those of moce_forward; MOCE_ERR_NULL for a missing L, router or
 * router array; MOCE_ERR_UNSUPPORTED when d > 64, k > 512 or C > 4096.
 * Asynchronous on `stream`. */
moce_status moce_forward_dynamic(const moce_desc* desc, const void* x, const float* L, const moce_router* router,
                                 const moce_gate_params* gate, void* y, int32_t* S_out, void* ws, size_t ws_bytes,
                                 hipStream_t stream);

/* Gradient outputs of the gate's parameters (device arrays, float32, fully
 * overwritten); only those of the gate's own kind are read and written.
 *  MOCE_GATE_SOFTPLUS_LINEAR: da [E-1][k] (canonical positions, as a), dc [E-1];
 *  MOCE_GATE_MLP_SIGMOID: dW1 [k][k], db1 [k], dw2 [k], db2 [1]. */
typedef struct moce_gate_grads {
    float* da;
    float* dc;
    float* dW1;
    float* db1;
    float* dw2;
    float* db2;
} moce_gate_grads;

/* Bytes of device workspace moce_backward needs for `desc` with a gate of
 * kind `gate_kind` (0 on an invalid descriptor or kind, or a shape beyond the
 * backward's limits). */
size_t moce_backward_workspace_bytes(const moce_desc* desc, int gate_kind);

/* Gradients of the static layer (Secs. 3.2-3.4) for an upstream gradient dy
 * of y = moce_forward(x).  The supports are fixed (Sec. 3.2: no gradient
 * through the selection); the loss reaches the routing logits only through
 * the selected values w (Eq. 4), the gate through the temperature, and x
 * both through the routed and residual sums (Eqs. 5-6) and through the
 * pooled descriptor that feeds the gate (Sec. 3.3):
 *   dx:  d loss / d x, layout and element type of x, fully overwritten;
 *   dw:  [E-1][k] float32, d loss / d w[e][i] for the prepared rows
 *        (canonical order), fully overwritten;
 *   the gate's parameter gradients into *grads (moce_gate_grads).
 * x, s, w, gate as for moce_forward (prepared rows; the uncovered set is
 * derived from s); dy: the layout and element type of y; x, dy and dx
 * 16-byte aligned; ws: device workspace of at least
 * moce_backward_workspace_bytes(desc, gate->kind) bytes, 256-byte aligned,
 * contents on return unspecified.  Gradients are accumulated in float32.
 * Errors: those of moce_forward; MOCE_ERR_NULL for a missing dy, dx, dw or
 * gradient array of the gate's kind; MOCE_ERR_UNSUPPORTED when k > 1024, or
 * k > 128 with the MLP gate.  Asynchronous on `stream`. */
moce_status moce_backward(const moce_desc* desc, const void* x, const void* dy, const int32_t* s, const float* w,
                          const moce_gate_params* gate, void* dx, float* dw, const moce_gate_grads* grads,
                          void* ws, size_t ws_bytes, hipStream_t stream);

/* Bytes of device workspace moce_logit_backward needs (0 when R < 1 or C is
 * outside [1, 32768]). */
size_t moce_logit_backward_workspace_bytes(int32_t R, int64_t C);

/* The coverage loss over the full routing logits (Sec. 3.4 Eq. 7) and the
 * whole gradient of the routing logits (Sec. 3.2: the task loss reaches the
 * selected entries, the coverage term every entry):
 *   p[e][c] = softmax_c(L[e]), u[c] = (1/R) sum_e p[e][c], ub = mean_c u[c],
 *   loss = sum_c (u[c] - ub)^2 / (ub^2 + eps),
 *   dL[e][c] = lambda d loss / d L[e][c] + (dw[e][i] where c = s[e][i]).
 * L: [R][C] float32 (R = E-1 routed experts); s, dw: prepared rows and the
 * dw of moce_backward, [R][k], or both NULL for the coverage term alone;
 * loss: device float, or NULL; dL: [R][C] float32, fully overwritten;
 * eps >= 0 (the paper leaves it unstated); ws as sized above.
 * Errors: MOCE_ERR_NULL (L, dL, ws; s without dw or dw without s),
 * MOCE_ERR_SHAPE (R < 1, C < 1, k outside [1, C] with dw given),
 * MOCE_ERR_UNSUPPORTED (C > 32768), MOCE_ERR_WORKSPACE, MOCE_ERR_ALIGN
 * (ws not 256-byte aligned); eps < 0 or not finite: MOCE_ERR_SHAPE. */
moce_status moce_logit_backward(int32_t R, int64_t C, int32_t k, const float* L, const int32_t* s, const float* dw,
                                float eps, float lambda, float* loss, float* dL, void* ws, size_t ws_bytes,
                                hipStream_t stream);

/* ---- dense pointwise projections ------------------------------------------
 *
 * The projections of a network that stay dense beside its channel-expert
 * layers: the expansion that closes a bottleneck, the token projections of a
 * transformer block.  With v[o][p] = sum_c weight[o][c] x[c][p] at position p,
 *   z[o][p] = scale[o] v[o][p] + shift[o] + residual[o][p],   y = act(z);
 * scale, shift and residual are optional (NULL: 1, 0, 0). */

/* Activations: z; max(z, 0); z (1 + erf(z / sqrt 2)) / 2; z / (1 + e^-z).
 * A NaN stays one, and infinities give the limits.  In bfloat16 a value of
 * 2^-119 or more is evaluated to within 2^-12 of itself before its rounding. */
enum { MOCE_ACT_NONE = 0, MOCE_ACT_RELU = 1, MOCE_ACT_GELU = 2, MOCE_ACT_SILU = 3 };

typedef struct moce_project_desc {
    int64_t B, C, H, W;   /* x is B images of C channels over H*W positions */
    int64_t O;            /* output channels, any number >= 1 */
    int32_t dtype;        /* of x, weight, residual, y, z and their gradients: MOCE_F32 or MOCE_BF16 */
    int32_t layout;       /* MOCE_NCHW or MOCE_NHWC, of x and y alike */
    int32_t act;          /* MOCE_ACT_* */
    int32_t reserved;     /* set to 0 */
} moce_project_desc;

/* Bytes of device workspace moce_project needs (0: none, or an invalid
 * descriptor).  It holds operands whose lines are not whole 16 bytes, packed
 * into lines that are, and the partial products of shapes with few outputs,
 * whose contraction is divided. */
size_t moce_project_workspace_bytes(const moce_project_desc* desc);

/* The projection.  x, residual, y, z: tensors of the descriptor's layout (C
 * channels for x, O for the others), weight: [O][C] row-major, all of the
 * descriptor's type, contiguous and 16-byte aligned; scale, shift: float32
 * [O].  y is fully overwritten, and so is z where it is given (the
 * pre-activation that moce_project_backward reads, rounded to the type; y
 * itself comes from the unrounded one).  residual may be y or z (in place);
 * y, z, ws and the other inputs may not overlap.  Sums are float32.
 * ws: as sized above, 256-byte aligned, contents on return unspecified; may
 * be NULL where no bytes are needed; calls that can run at the same time need
 * one each, captured calls that are replayed so too.  Rows of channels of any
 * grouping are MOCE_NHWC with B rows and H = W = 1.  Asynchronous on `stream`.
 * Errors: MOCE_ERR_NULL (desc, x, weight, y), MOCE_ERR_SHAPE (a size below 1,
 * an unknown act, memory that overlaps), MOCE_ERR_DTYPE, MOCE_ERR_LAYOUT, MOCE_ERR_ALIGN,
 * MOCE_ERR_WORKSPACE, MOCE_ERR_DEVICE; MOCE_ERR_UNSUPPORTED when C or O
 * exceeds 2^20, C O 2^35, B H W 2^29, C H W or O H W 2^31 - 1, or B C H W or
 * B O H W 2^33. */
moce_status moce_project(const moce_project_desc* desc, const void* x, const void* weight, const float* scale,
                         const float* shift, const void* residual, void* y, void* z, void* ws, size_t ws_bytes,
                         hipStream_t stream);

/* Gradients of moce_project, each optional (NULL: not computed) and fully
 * overwritten:
 *   dz = act'(z) dy;                      dresidual = dz;
 *   dshift[o] = sum_p dz[o][p];           G[o][c] = sum_p dz[o][p] x[c][p];
 *   dweight[o][c] = scale[o] G[o][c];     dscale[o] = sum_c weight[o][c] G[o][c];
 *   dx[c][p] = sum_o scale[o] weight[o][c] dz[o][p]. */
typedef struct moce_project_grads {
    void* dx;             /* layout and type of x */
    void* dweight;        /* [O][C], type of weight */
    float* dscale;        /* [O]; needs scale; MOCE_ACT_NONE and MOCE_ACT_RELU (the others: with
                           * dresidual of one call as dy of another with MOCE_ACT_NONE) */
    float* dshift;        /* [O] */
    void* dresidual;      /* layout and type of y */
} moce_project_grads;

/* Bytes of device workspace moce_project_backward needs (0 on an invalid
 * descriptor). */
size_t moce_project_backward_workspace_bytes(const moce_project_desc* desc);

/* The gradients of moce_project for an upstream gradient dy of y (layout and
 * type of y).  x, weight, scale as in the forward; z: the pre-activation that
 * the forward wrote (for MOCE_ACT_RELU its y serves as well; not read for
 * MOCE_ACT_NONE).  act' of ReLU is 0 where z <= 0.  All tensors contiguous
 * and 16-byte aligned; dresidual may be dy (in place), no other output,
 * and not ws, may overlap an input or another output.  For bfloat16, dz enters the products
 * rounded to its type (exact for MOCE_ACT_NONE and MOCE_ACT_RELU), and so does
 * the scaled weight of dx; sums are float32.  ws as sized above, 256-byte
 * aligned.  Errors: those of moce_project; MOCE_ERR_NULL for a missing dy or
 * z, or dscale without scale; MOCE_ERR_UNSUPPORTED for dscale with
 * MOCE_ACT_GELU or MOCE_ACT_SILU.  Asynchronous on `stream`. */
moce_status moce_project_backward(const moce_project_desc* desc, const void* x, const void* weight,
                                  const float* scale, const void* z, const void* dy,
                                  const moce_project_grads* grads, void* ws, size_t ws_bytes, hipStream_t stream);

/* How one of the products of this descriptor is cut, for tests and timing (the
 * results do not depend on it but for the order of float32 sums). */
enum { MOCE_PRODUCT_FORWARD = 0, MOCE_PRODUCT_DX = 1, MOCE_PRODUCT_DWEIGHT = 2 };

typedef struct moce_project_cut {
    int32_t rows, columns; /* a tile of the product; 0: the forward of up to 32 rows, which has none */
    int32_t stages;        /* of the contraction in LDS */
    int32_t splits;        /* parts of the contraction, joined by another kernel (1: none) */
    int32_t a_along;       /* whether the rows' operand runs along the contraction in memory */
    int32_t b_along;       /* and the columns' */
    int32_t images;        /* whether lines along the contraction pass from image to image */
    int32_t reserved;
} moce_project_cut;

/* A query on the host.  Errors: MOCE_ERR_NULL (desc, cut), MOCE_ERR_SHAPE for
 * an unknown product, and those of moce_project for the descriptor. */
moce_status moce_project_path(const moce_project_desc* desc, int32_t product, moce_project_cut* cut);

/* ---- group norm with an activation -------------------------------------------
 *
 * x holds B images of C channels over H*W positions; the channels form G groups
 * of C / G neighbours.  Per image b and group g, over the n = (C / G) H W
 * elements of the group:
 *   mean = sum x / n,   rstd = 1 / sqrt(sum (x - mean)^2 / n + eps),
 *   h = (x - mean) rstd,   z = scale[c] h + shift[c],   y = act(z)
 * (scale and shift optional: NULL is 1 and 0).  G = 1 takes all channels of an
 * image together, G = C each by itself. */
typedef struct moce_group_norm_desc {
    int64_t B, C, H, W;
    int64_t G;            /* groups, a divisor of C */
    int32_t dtype;        /* of x, y and their gradients: MOCE_F32 or MOCE_BF16 */
    int32_t layout;       /* MOCE_NCHW or MOCE_NHWC (tokens: H of them, W = 1) */
    int32_t act;          /* MOCE_ACT_* */
    float eps;            /* finite, >= 0 */
} moce_group_norm_desc;

/* Bytes of device workspace moce_group_norm needs (0 on an invalid descriptor). */
size_t moce_group_norm_workspace_bytes(const moce_group_norm_desc* desc);

/* The normalisation.  x, y: contiguous, 16-byte aligned; scale, shift: float32
 * [C]; stats (optional): float32 [2][B][G], the means, then the rstd, which the
 * backward reads.  y is fully overwritten and may be x (in place); nothing else
 * may overlap.  Sums are float32, squares of deviations from a value of the
 * group or its mean, so that a mean that is large against the deviation costs no
 * digits of it (a sum of a group's values, or a square, past float32's range is
 * infinite); their order depends on the descriptor alone.  A NaN or infinity
 * makes its group NaN, and no other.  ws: as sized above, 256-byte aligned;
 * calls that can run at the same time need one each, captured calls that are
 * replayed so too.  Asynchronous on
 * `stream`.  Errors: MOCE_ERR_NULL (desc, x, y), MOCE_ERR_SHAPE (a size below
 * 1, C not a multiple of G, an unknown act, eps, memory that overlaps),
 * MOCE_ERR_DTYPE, MOCE_ERR_LAYOUT, MOCE_ERR_ALIGN, MOCE_ERR_WORKSPACE,
 * MOCE_ERR_DEVICE; MOCE_ERR_UNSUPPORTED when C exceeds 2^20, C H W 2^31 - 1, B
 * 2^29 or B C H W 2^38. */
moce_status moce_group_norm(const moce_group_norm_desc* desc, const void* x, const float* scale, const float* shift,
                            void* y, float* stats, void* ws, size_t ws_bytes, hipStream_t stream);

/* Gradients of moce_group_norm, each optional (NULL: not computed) and fully
 * overwritten; t = scale dz, means over the group:
 *   dz = act'(z) dy;   dshift[c] = sum dz;   dscale[c] = sum dz h;
 *   dx = rstd (t - mean(t) - h mean(t h)). */
typedef struct moce_group_norm_grads {
    void* dx;             /* layout and type of x */
    float* dscale;        /* [C] */
    float* dshift;        /* [C] */
} moce_group_norm_grads;

/* Bytes of device workspace moce_group_norm_backward needs (0 on an invalid
 * descriptor). */
size_t moce_group_norm_backward_workspace_bytes(const moce_group_norm_desc* desc);

/* The gradients for an upstream gradient dy of y (layout and type of y); x,
 * scale and shift as in the forward, stats as it wrote them (h and z are formed
 * again).  act' of ReLU is 0 where z <= 0.  dx may be dy or x (in place); no
 * other output, and not ws, may overlap an input or another output.  Sums are
 * float32 (of dscale and dshift over the images float64), their order depends on
 * the descriptor alone.  ws as sized above, 256-byte aligned.  Errors: those of
 * moce_group_norm; MOCE_ERR_NULL for a missing dy, stats or grads.
 * Asynchronous on `stream`. */
moce_status moce_group_norm_backward(const moce_group_norm_desc* desc, const void* x, const float* scale,
                                     const float* shift, const float* stats, const void* dy,
                                     const moce_group_norm_grads* grads, void* ws, size_t ws_bytes, hipStream_t stream);

/* ---- the losses of a classification head ----------------------------------------
 *
 * A head projects P rows of C features to V classes, z[p][v] = sum_c x[p][c]
 * weight[v][c] + shift[v] (moce_project gives the logits z themselves).  The
 * calls here take the loss of the logits and its gradients without keeping the
 * logits: the forward leaves the softmax statistics of a row, the backward
 * forms the logits again, in pieces of the classes.  Both keep at most 256 MB of
 * logits or their gradient in the workspace, or 256 classes of all rows.
 *
 * Cross entropy with a label t[p], smoothed by e:
 *   loss[p] = lse - (1 - e) z[p][t] - e mean_v z[p][v],   lse = log sum_v e^z[p][v].
 * Distillation from K entries of a teacher's logits, classes i[p][k] and logits
 * l[p][k], at temperature T: q = softmax(l[p] / T) over the entries, those of
 * one class added up; with s = z / T,
 *   loss[p] = T^2 sum_v q_v (log q_v - s[p][v] + log sum_u e^s[p][u]).
 *
 * A label outside [0, V) leaves its row out: its loss is 0, it adds nothing to
 * the gradients and its dx is 0, whatever the row holds.  So does a teacher of
 * whose entries none has a class in [0, V) and a logit above minus infinity;
 * an entry whose class is outside counts for nothing. */
enum { MOCE_LOSS_ROWS = 0, MOCE_LOSS_MEAN = 1 };

typedef struct moce_head_desc {
    int64_t P, C, V;        /* rows, features, classes */
    int32_t K;              /* entries of the teacher a row; 1 for labels */
    int32_t dtype;          /* of x, weight and their gradients: MOCE_F32 or MOCE_BF16 */
    int32_t teacher_dtype;  /* of the teacher's logits (not read for labels) */
    int32_t index_bytes;    /* of a label or class, a signed integer: 4 or 8 */
    int32_t reduction;      /* MOCE_LOSS_ROWS: loss[P]; MOCE_LOSS_MEAN: loss[1], the mean over the
                             * rows that are not left out (0 where all are) */
    float smoothing;        /* e in [0, 1] (not read by the distillation) */
    float temperature;      /* T, 2^-62 to 2^62 (not read by the cross entropy) */
    int32_t reserved;       /* set to 0 */
} moce_head_desc;

/* Elements of the float32 array `saved` that a forward leaves for the backward:
 * P (K + 1) + 2 (0 on an invalid descriptor). */
size_t moce_head_saved_floats(const moce_head_desc* desc);

/* Bytes of device workspace the two forward calls need (0 on an invalid
 * descriptor). */
size_t moce_head_workspace_bytes(const moce_head_desc* desc);

/* The losses.  x: [P][C], weight: [V][C], of the descriptor's type, 16-byte
 * aligned; shift: float32 [V] or NULL; labels [P], classes [P][K]: integers of
 * index_bytes; logits: [P][K], of teacher_dtype; loss: float32, as the reduction
 * has it; saved: float32, sized as above, or NULL where no backward follows.
 * All contiguous; no output, and not ws, may overlap an input or another output.
 * Sums are float32 (over rows float64), their order depends on the descriptor
 * alone; a row's loss that they leave below 0 is 0.  A logit of minus infinity
 * (by its shift) takes the class out, of smoothed labels and as a target's the
 * loss is infinite; one of plus infinity or NaN makes its row's loss NaN, and so
 * does a teacher's that counts.  ws: 256-byte aligned, one for each call that
 * can run at the same time, captured calls that are replayed so too.
 * Asynchronous on `stream`.  Errors: MOCE_ERR_NULL (desc, x, weight, the
 * targets, loss), MOCE_ERR_SHAPE (a size below 1, K not 1 for labels,
 * index_bytes, reduction, smoothing, temperature, memory that overlaps),
 * MOCE_ERR_DTYPE, MOCE_ERR_ALIGN, MOCE_ERR_WORKSPACE, MOCE_ERR_DEVICE;
 * MOCE_ERR_UNSUPPORTED when P exceeds 2^24, C or V 2^20, K 1024, V C 2^35, P V
 * 2^35 or P C 2^33. */
moce_status moce_head_cross_entropy(const moce_head_desc* desc, const void* x, const void* weight, const float* shift,
                                    const void* labels, float* loss, float* saved, void* ws, size_t ws_bytes,
                                    hipStream_t stream);
moce_status moce_head_distill(const moce_head_desc* desc, const void* x, const void* weight, const float* shift,
                              const void* classes, const void* logits, float* loss, float* saved, void* ws,
                              size_t ws_bytes, hipStream_t stream);

/* Gradients of the losses, each optional (NULL: not computed) and fully
 * overwritten.  With g[p] the upstream dloss[p] (MOCE_LOSS_MEAN: dloss[0] over
 * the number of rows that count), 0 for a row that is left out:
 *   cross entropy: dz[p][v] = g (softmax(z)[v] - (1 - e) [v = t] - e / V);
 *   distillation:  dz[p][v] = g T (softmax(z / T)[v] - q_v);
 *   dx[p][c] = sum_v dz[p][v] weight[v][c];   dweight[v][c] = sum_p dz[p][v] x[p][c];
 *   dshift[v] = sum_p dz[p][v]. */
typedef struct moce_head_grads {
    void* dx;             /* [P][C], type of x */
    void* dweight;        /* [V][C], type of weight */
    float* dshift;        /* [V] */
} moce_head_grads;

/* Bytes of device workspace the two backward calls need (0 on an invalid
 * descriptor). */
size_t moce_head_backward_workspace_bytes(const moce_head_desc* desc);

/* The gradients.  The inputs as in the forward, saved as it wrote them; dloss:
 * float32 [P], or [1] for MOCE_LOSS_MEAN.  For bfloat16, dz enters the products
 * rounded to its type relative to the largest |g| (for float32 as it is); sums
 * are float32, and dshift takes dz as it is (of a teacher, a row of less than
 * 2^-35 of the largest |g| may not show in it).  Rows that are left out may hold
 * anything, NaN too.  ws and errors as for the forward; MOCE_ERR_NULL for a
 * missing saved, dloss or grads.  Asynchronous on `stream`. */
moce_status moce_head_cross_entropy_backward(const moce_head_desc* desc, const void* x, const void* weight,
                                             const float* shift, const void* labels, const float* saved,
                                             const float* dloss, const moce_head_grads* grads, void* ws,
                                             size_t ws_bytes, hipStream_t stream);
moce_status moce_head_distill_backward(const moce_head_desc* desc, const void* x, const void* weight,
                                       const float* shift, const void* classes, const void* logits,
                                       const float* saved, const float* dloss, const moce_head_grads* grads, void* ws,
                                       size_t ws_bytes, hipStream_t stream);

/* ---- the global norm of a list of gradients, and clipping ------------------ */

/* One gradient: n elements of `dtype` at src (aligned to its element; n == 0
 * is allowed).  dst: where the clipped gradient goes, src itself or memory
 * that overlaps no tensor of the list (not read by moce_gradient_norm). */
typedef struct moce_gradient {
    const void* src;
    void* dst;
    int64_t n;
    int32_t dtype;        /* MOCE_F32 or MOCE_BF16 */
    int32_t reserved;     /* set to 0 */
} moce_gradient;

/* Bytes of device workspace the two calls below need for this list (0 on an
 * invalid one). */
size_t moce_gradient_workspace_bytes(const moce_gradient* grads, int32_t count);

/* *norm (device float) = sqrt(sum over all tensors and elements of g^2),
 * accumulated in float64: no square of a float32 overflows or is lost.  The
 * list is host memory, read before the call returns; count == 0 gives 0.  The
 * order of the sum depends on the sizes alone: the same gradients give the
 * same bits.  Errors: MOCE_ERR_NULL (norm, the list, a tensor's src with
 * n > 0), MOCE_ERR_SHAPE (count < 0, n < 0, norm or ws over a tensor or each
 * other), MOCE_ERR_DTYPE, MOCE_ERR_ALIGN, MOCE_ERR_WORKSPACE;
 * MOCE_ERR_UNSUPPORTED when the sizes sum to over 2^40.
 * Asynchronous on `stream`. */
moce_status moce_gradient_norm(const moce_gradient* grads, int32_t count, float* norm, void* ws, size_t ws_bytes,
                               hipStream_t stream);

/* moce_gradient_norm, then dst = src * (max_norm / norm) where norm >
 * max_norm, else dst = src (nothing is written for dst == src).  The
 * coefficient is formed on the device: no synchronisation.  A norm that is
 * not finite leaves every gradient as it is (*norm tells).  Products are
 * float32, rounded to the tensor's type.  *norm is the norm before clipping.
 * Errors: those of moce_gradient_norm; MOCE_ERR_NULL for a missing dst;
 * MOCE_ERR_SHAPE when max_norm is negative or not finite, when two tensors
 * overlap (a tensor listed twice would be scaled twice), when a dst overlaps
 * any src but its own, or its own partly, or when norm or ws overlaps a dst. */
moce_status moce_gradient_clip(const moce_gradient* grads, int32_t count, float max_norm, float* norm, void* ws,
                               size_t ws_bytes, hipStream_t stream);

/* Static string naming a status code. */
const char* moce_status_str(int status);

/* ABI version of this header: 1. */
int moce_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* MOCE_H */
