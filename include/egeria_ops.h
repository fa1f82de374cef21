/*
 * egeria_ops.h -- C ABI of the training operators of the B200 (sm_100a) library.
 *
 * Next to the plasticity evaluation of egeria.h the library has the operators that a
 * training step of the monitored network spends its time in: linear layers with what
 * surrounds the product in its epilogue and their gradients, gated feed-forward blocks
 * and their gradients, the norms of a residual stream with their gate and their
 * gradients, and two optimizer steps, AdamW over all tensors and Muon over matrices, that
 * leave the frozen modules alone by reading the freeze mask on the device.
 *
 * The conventions of egeria.h hold: device pointers are the caller's, the library
 * allocates no device memory, calls enqueue work on the stream they are given and
 * return without synchronising, errors are returned as egeria_status, nothing throws,
 * and there is no CPU path.  Besides:
 *   - Matrices are row-major with a row pitch (ld*, in elements, at least the number of
 *     columns); the elements of a row are consecutive.  Any element-aligned pointer and
 *     any pitch work; 16-byte aligned pointers and pitches that are multiples of 8 are
 *     fastest.
 *   - A handle belongs to one stream at a time: its workspace is scratch of the call in
 *     flight.  Handles are not thread-safe.
 *   - The calls of a handle may be captured into a CUDA graph and replayed in stream
 *     order.
 *   - Sums, row statistics and gradients of parameters are accumulated in 32 bits and
 *     rounded once to the output's type.  Results do not depend on timing: the same call
 *     gives the same bits.
 */
#ifndef EGERIA_OPS_H_
#define EGERIA_OPS_H_

#include "egeria.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { EGERIA_F32 = 0, EGERIA_BF16 = 1, EGERIA_F16 = 2 } egeria_type;

typedef struct egeria_ops egeria_ops;       /* opaque, library-owned host objects */
typedef struct egeria_adamw egeria_adamw;
typedef struct egeria_muon egeria_muon;

/* A handle for the calls of linear layers, gated blocks and norms.
 *   workspace  device memory, EGERIA_WORKSPACE_ALIGN-aligned, caller-owned, at least
 *              EGERIA_OPS_WORKSPACE_MIN bytes and as much as the largest call made through
 *              the handle asks for; must outlive the handle
 * Waits for the current device, whose earlier work may still use that memory, and clears the handle's part of it
 * synchronously. */
#define EGERIA_OPS_WORKSPACE_MIN 65536
egeria_status egeria_ops_create(egeria_ops **out, void *workspace, size_t workspace_bytes);
egeria_status egeria_ops_destroy(egeria_ops *ops);

/* Synchronise the stream of the last call and report the device status word: EGERIA_OK, or
 * EGERIA_ERR_TIMEOUT if a bounded wait inside a kernel ran out (the results of that call are
 * invalid; the handle can be used again), or in a checked build EGERIA_ERR_CHECK if an index check
 * inside a kernel failed. */
egeria_status egeria_ops_device_status(egeria_ops *ops);

/* Number of kernels launched through this handle so far. */
int64_t egeria_ops_launch_count(const egeria_ops *ops);

/* Test hook: in the next matrix product on the tensor cores through this handle the first thread block (or pair of them)
 * issues no loads (kind 1) or stops after its first stage (kind 2), and every wait is limited to a millisecond: the kernel
 * returns, that call's results are not valid, egeria_ops_device_status reports EGERIA_ERR_TIMEOUT once, and the handle can be
 * used again.  kind 0 takes the request back. */
egeria_status egeria_ops_debug_stall_next(egeria_ops *ops, int kind);

/* ---------------------------------------------------------------------------- linear layers */

typedef enum {
    EGERIA_ACT_NONE = 0,
    EGERIA_ACT_RELU = 1,      /* max(z, 0); slope 0 at 0 */
    EGERIA_ACT_GELU = 2,      /* z Phi(z), Phi the normal distribution */
    EGERIA_ACT_GELU_TANH = 3, /* z / (1 + exp(-2 u)), u = sqrt(2 / pi) (z + 0.044715 z^3) */
    EGERIA_ACT_SILU = 4       /* z / (1 + exp(-z)) */
} egeria_act;

/* Bytes of workspace that both linear calls of a layer with these sizes, or with smaller ones, fit into, whatever the
 * alignment of their operands.  Pure host arithmetic; 0 for invalid arguments.  (The forward call of up to 4 rows needs
 * none, up to 49152 / rows values of a row (rows = 3 counting as 4).) */
size_t egeria_linear_workspace_bytes(int64_t rows, int64_t inp, int64_t out);

/* z = x w^T + bias,  y = act(z) + residual.
 *   type      EGERIA_BF16 or EGERIA_F16, of all operands
 *   x         [rows, inp]        w  [out, inp]       bias  [out] or NULL
 *   residual  [rows, out] or NULL; may be y itself (same pointer and pitch)
 *   y         [rows, out]
 *   z         [rows, out] or NULL: the argument of the activation, for the backward call
 * Otherwise y and z share no value with an operand or each other (EGERIA_ERR_INVALID_ARG; parts of one buffer that
 * lie beside each other are fine).  rows may be 0 (nothing is done); inp and out are at least 1; none above 2^31 - 1024. */
typedef struct {
    int32_t type, act;
    int64_t rows, inp, out;
    const void *x, *w, *bias, *residual;
    int64_t ldx, ldw, ldr;
    void *y, *z;
    int64_t ldy, ldz;
} egeria_linear_forward_args;
egeria_status egeria_linear_forward(egeria_ops *ops, void *cuda_stream, const egeria_linear_forward_args *args);

/* The gradients, given dy, that of y:
 *   dz = dy * act'(z)       dx = (dz w) * act_in'(z_in)      dw = dz^T x      db = sum over rows of dz
 * The gradient of the residual is dy itself.
 *   z     [rows, out]: needed unless act is EGERIA_ACT_NONE
 *   z_in  [rows, inp]: needed unless act_in is EGERIA_ACT_NONE.  Where x came out of the
 *         activation act_in of another layer's z_in, dx is then that layer's dz, which saves
 *         a pass over it.
 *   dx, dw, db  any of them may be NULL: not computed (a frozen layer needs no dw and db)
 * The product's operand dz is rounded to `type`, as dy is; db sums it before that.  With
 * rows = 0, dw and db are set to 0. */
typedef struct {
    int32_t type, act, act_in;
    int64_t rows, inp, out;
    const void *dy, *x, *w, *z, *z_in;
    int64_t lddy, ldx, ldw, ldz, ldz_in;
    void *dx, *dw, *db;
    int64_t lddx, lddw;
} egeria_linear_backward_args;
egeria_status egeria_linear_backward(egeria_ops *ops, void *cuda_stream, const egeria_linear_backward_args *args);

/* ---------------------------------------------------------------------------- gated feed-forward blocks */

/* Bytes of workspace that both calls of a block with these sizes, or with smaller ones, fit into, whatever the alignment of
 * their operands.  Pure host arithmetic; 0 for invalid arguments. */
size_t egeria_gated_workspace_bytes(int64_t rows, int64_t inp, int64_t hidden, int64_t out);

/* g = x w_gate^T + b_gate,  u = x w_up^T + b_up,  h = act(g) u,  y = h w_down^T + b_down + residual.
 *   type      EGERIA_BF16 or EGERIA_F16, of all operands
 *   act       any egeria_act (EGERIA_ACT_NONE: the product of the two projections)
 *   x         [rows, inp]        w_gate, w_up  [hidden, inp]     w_down  [out, hidden]
 *   b_gate, b_up [hidden], b_down [out], residual [rows, out]: each may be NULL; residual may be y itself (same pointer and pitch)
 *   y         [rows, out]
 *   g, u      [rows, hidden], both or neither NULL: what the backward call needs
 * Otherwise y, g and u share no value with an operand or each other (EGERIA_ERR_INVALID_ARG; w_gate and w_up may be parts of
 * one matrix).  h is rounded to `type`, which is what the second product takes; it is made from g and u before they are rounded.
 * rows may be 0 (nothing is done); inp, hidden and out are at least 1; none above 2^31 - 1024. */
typedef struct {
    int32_t type, act;
    int64_t rows, inp, hidden, out;
    const void *x, *w_gate, *w_up, *w_down, *b_gate, *b_up, *b_down, *residual;
    int64_t ldx, ldw_gate, ldw_up, ldw_down, ldr;
    void *y, *g, *u;
    int64_t ldy, ldg, ldu;
} egeria_gated_forward_args;
egeria_status egeria_gated_forward(egeria_ops *ops, void *cuda_stream, const egeria_gated_forward_args *args);

/* The gradients, given dy, that of y, and g and u as the forward call left them:
 *   dh = dy w_down       dg = dh u act'(g)       du = dh act(g)
 *   dx = dg w_gate + du w_up     dw_gate = dg^T x     dw_up = du^T x     dw_down = dy^T (act(g) u)
 *   db_gate, db_up, db_down: the sums over rows of dg, du and dy
 * The gradient of the residual is dy itself.  Each of the seven results may be NULL: not computed (a frozen block needs dx alone).
 * x is needed for dw_gate and dw_up, w_gate and w_up for dx, w_down, g and u for all but db_down.  dh is not rounded; dg, du and
 * act(g) u are, to `type`, as operands of the products; the sums are taken before that.  The results share no value with what the
 * call reads or each other.  With rows = 0 the gradients of weights and biases are set to 0. */
typedef struct {
    int32_t type, act;
    int64_t rows, inp, hidden, out;
    const void *dy, *x, *w_gate, *w_up, *w_down, *g, *u;
    int64_t lddy, ldx, ldw_gate, ldw_up, ldw_down, ldg, ldu;
    void *dx, *dw_gate, *dw_up, *dw_down, *db_gate, *db_up, *db_down;
    int64_t lddx, lddw_gate, lddw_up, lddw_down;
} egeria_gated_backward_args;
egeria_status egeria_gated_backward(egeria_ops *ops, void *cuda_stream, const egeria_gated_backward_args *args);

/* ---------------------------------------------------------------------------- residual norms */

typedef enum { EGERIA_NORM_LAYER = 0, EGERIA_NORM_RMS = 1 } egeria_norm_kind;

#define EGERIA_NORM_MAX_COLS 8192

/* Bytes of workspace that both norm calls with these sizes, or with smaller ones, fit into.  Pure host arithmetic; 0 for
 * invalid arguments. */
size_t egeria_norm_workspace_bytes(int64_t rows, int64_t cols);

/* One boundary between two blocks of a residual network:
 *   y = alpha x + gate * N_post(f)        h = N_pre(y)
 * N(a) = (a - mean) / sqrt(var + eps) * w + b over the row (EGERIA_NORM_LAYER), or
 * N(a) = a / sqrt(mean of a^2 + eps) * w + b (EGERIA_NORM_RMS).
 *   type        of x, f, y, h: EGERIA_F32, EGERIA_BF16 or EGERIA_F16
 *   param_type  of the weights, biases and the gate: EGERIA_F32 or `type`
 *   post, pre   0 leaves that norm out (f itself is added; h is not written)
 *   gate        NULL (1 everywhere), [1, cols] with gate_rows = 0, or [ceil(rows / gate_rows),
 *               cols]: row r takes gate r / gate_rows
 *   w_*, b_*    [cols] or NULL (1, 0)
 *   stats       float [rows, 4] or NULL: mean and 1/deviation of f's row, then of y's; 0 for a norm
 *               that is left out and for the mean under EGERIA_NORM_RMS.  The backward call reads it.
 * h is normalised from y before y is rounded.  cols is 1..EGERIA_NORM_MAX_COLS, larger ones give
 * EGERIA_ERR_UNSUPPORTED_SHAPE.  y may be x, and h may be f (same pointer and pitch). */
typedef struct {
    int32_t type, param_type, kind, post, pre;
    float alpha, eps;
    int64_t rows, cols, gate_rows;
    const void *x, *f, *gate, *w_post, *b_post, *w_pre, *b_pre;
    int64_t ldx, ldf;
    void *y, *h;
    int64_t ldy, ldh;
    float *stats;
} egeria_norm_forward_args;
egeria_status egeria_norm_forward(egeria_ops *ops, void *cuda_stream, const egeria_norm_forward_args *args);

/* Its gradients, given dy (of y as the stream goes on) and dh (of h):
 *   t  = dy + (gradient of y through N_pre)      dx = alpha t
 *   df = gradient of f through N_post of gate * t
 * and the sums over rows that are the gradients of the gate, the weights and the biases, of type
 * param_type; each of those five may be NULL.  y, f, stats: as the forward call left them.  dh is
 * needed if pre, else ignored (as are y and the pre outputs).  dx may be dy, and df may be f or
 * dh (same pointer and pitch).  With rows = 0 the sums are set to 0. */
typedef struct {
    int32_t type, param_type, kind, post, pre;
    float alpha;
    int64_t rows, cols, gate_rows;
    const void *dy, *dh, *y, *f, *gate, *w_post, *b_post, *w_pre, *b_pre;
    int64_t lddy, lddh, ldy, ldf;
    const float *stats;
    void *dx, *df;
    int64_t lddx, lddf;
    void *dgate, *dw_post, *db_post, *dw_pre, *db_pre;
} egeria_norm_backward_args;
egeria_status egeria_norm_backward(egeria_ops *ops, void *cuda_stream, const egeria_norm_backward_args *args);

/* ---------------------------------------------------------------------------- AdamW */

#define EGERIA_ADAMW_BLOCK 256   /* values that share one scale of an 8-bit moment */

enum {
    /* Moments in 8 bits.  m: int8 codes c, a first moment is sign(c) (c / 127)^2 scale; v: uint8 codes,
     * the square root of a second moment is (c / 255)^2 scale.  One float scale per moment and block of
     * EGERIA_ADAMW_BLOCK consecutive values of a tensor: the largest size in the block.  A second
     * moment that is not zero has a code of at least 1.  Codes and scales are those of the
     * formula in 32 bits, every operation rounded by itself (a code is decoded as (c c) (scale * (1 / 127^2)), the roots
     * and quotients are correctly rounded, codes to the nearest, ties to even): a state can be reproduced
     * bit by bit.  A value that is not finite makes its whole
     * block NaN from the next step on (8-bit codes have no NaN of their own). */
    EGERIA_ADAMW_8BIT = 1u
};

/* One tensor of the model.  All pointers are device memory of n consecutive values, element-aligned
 * (fastest: 32-byte aligned); m and v of moments in 8 bits: 8-byte aligned is fastest. */
typedef struct {
    void *param;             /* of param_type; written */
    float *master;           /* NULL, or the 32-bit copy that the step works on; param is then its rounding */
    void *m, *v;             /* moments: float [n], or codes */
    float *m_scale, *v_scale;/* float [ceil(n / EGERIA_ADAMW_BLOCK)]; NULL unless EGERIA_ADAMW_8BIT */
    int64_t n;               /* may be 0 */
    int32_t param_type;      /* EGERIA_F32, EGERIA_BF16, EGERIA_F16 */
    int32_t grad_type;       /* EGERIA_F32 or param_type */
    float weight_decay;
    int32_t module;          /* its entry in the freeze mask, -1 = in none */
} egeria_adamw_tensor;

/* Bytes of device workspace (the table of tensors and of the pieces they are cut into).  Pure host
 * arithmetic; 0 for invalid arguments. */
size_t egeria_adamw_workspace_bytes(int count, const egeria_adamw_tensor *tensors, uint32_t flags);

/* An optimizer over `count` tensors (host array, copied).
 *   grads  host array [count] of device pointers
 *   steps  device int32 [count], the caller's: steps taken so far by each tensor
 * Waits for the current device, whose earlier work may still use the workspace, writes its tables there and synchronises. */
egeria_status egeria_adamw_create(egeria_adamw **out, int count, const egeria_adamw_tensor *tensors,
                                  const void *const *grads, int32_t *steps, void *workspace, size_t workspace_bytes,
                                  uint32_t flags);
egeria_status egeria_adamw_destroy(egeria_adamw *adamw);

/* The gradients are elsewhere from the next step on (one small copy in stream order; refused with
 * EGERIA_ERR_INVALID_ARG on a stream that is being captured). */
egeria_status egeria_adamw_set_grads(egeria_adamw *adamw, void *cuda_stream, const void *const *grads);

/* One step of every tensor that is not frozen:
 *   g = gradient * grad_scale                t = ++steps
 *   m = beta1 m + (1 - beta1) g              v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 *   grad_scale  device float [1] or NULL (1): e.g. 1 / loss scale, or the clipping factor.  If it is not
 *               finite the whole step is left out (nothing is written, no step is counted).
 *   frozen      device uint8 or NULL, indexed by `module`: the out_mask of
 *               egeria_plasticity_evaluate as it is.  A frozen tensor is neither read nor written
 *               and its step count stands still.
 * 0 <= beta1, beta2 < 1; lr and eps not negative.  The step counts live on the device, so the call can be
 * captured into a CUDA graph and replayed; lr and the betas are then those of the capture. */
egeria_status egeria_adamw_step(egeria_adamw *adamw, void *cuda_stream, double lr, double beta1, double beta2,
                                double eps, const float *grad_scale, const uint8_t *frozen);

/* Synchronise the stream of the last call and report the device status word: EGERIA_OK, or in a
 * checked build EGERIA_ERR_CHECK if an index check inside a kernel failed. */
egeria_status egeria_adamw_device_status(egeria_adamw *adamw);

/* Number of kernels launched through this handle so far. */
int64_t egeria_adamw_launch_count(const egeria_adamw *adamw);

/* ---------------------------------------------------------------------------- Muon */

#define EGERIA_MUON_MAX_STEPS 16

/* One matrix of the model, rows x cols consecutive values (a convolution's weight as its output channels by the rest), element-aligned.
 * Fastest where cols is a multiple of 8 and everything 32-byte aligned.  What a step writes (param, master, m of all matrices) shares no
 * value with itself or with a gradient (EGERIA_ERR_INVALID_ARG, also of set_grads): a weight that two layers share stands in the list
 * once.  Gradients may share values with one another. */
typedef struct {
    void *param;             /* of param_type; written */
    float *master;           /* NULL, or the 32-bit copy that the step works on; param is then its rounding */
    float *m;                /* the momentum */
    int64_t rows, cols;      /* either may be 0: nothing to do; none above 2^22 */
    int32_t param_type;      /* EGERIA_F32, EGERIA_BF16, EGERIA_F16 */
    int32_t grad_type;       /* EGERIA_F32 or param_type */
    float weight_decay;
    float scale;             /* of the update, beside lr: 0.2 sqrt(max(rows, cols)) makes its values as large as AdamW's usually are,
                                sqrt(max(1, rows / cols)) its effect on a layer's output alike for all shapes */
    int32_t module;          /* its entry in the freeze mask, -1 = in none */
} egeria_muon_tensor;

/* Bytes of device workspace: about six per value of the matrices, four per value of the squares of their shorter sides (for a matrix
 * of at most 128 by 768, instead of both, 256 for each column of its longer side rounded up to 64), and the list of the work.  Pure host arithmetic; 0 for invalid arguments. */
size_t egeria_muon_workspace_bytes(int count, const egeria_muon_tensor *tensors, int steps);

/* An optimizer over `count` matrices (host array, copied).
 *   grads  host array [count] of device pointers
 *   steps  of the orthogonalisation, 1..EGERIA_MUON_MAX_STEPS; 5 is usual
 * Waits for the current device, whose earlier work may still use the workspace, writes its tables there and synchronises. */
egeria_status egeria_muon_create(egeria_muon **out, int count, const egeria_muon_tensor *tensors, const void *const *grads, int steps,
                                 void *workspace, size_t workspace_bytes);
egeria_status egeria_muon_destroy(egeria_muon *muon);

/* The gradients are elsewhere from the next step on (one small copy in stream order; refused with
 * EGERIA_ERR_INVALID_ARG on a stream that is being captured). */
egeria_status egeria_muon_set_grads(egeria_muon *muon, void *cuda_stream, const void *const *grads);

/* One step of every matrix that is not frozen:
 *   g = gradient * grad_scale      m = beta m + (1 - beta) g      t = nesterov ? beta m + (1 - beta) g : m
 *   X = t / max(|t|, eps), |t| the root of the sum of squares; then `steps` times
 *       A = X X^T     X = 3.4445 X - 4.7750 A X + 2.0315 A^2 X
 *   p = p (1 - lr weight_decay) - lr scale X
 * The products' operands are rounded to f16 (11 digits), their sums are 32 bits: after five steps X is off by about 1.5e-3 of itself
 * (2-norm; 0.4e-3 to 2.1e-3 over the shapes and ranks tried; a matrix of two or three singular values by up to 1.6e-2, where one of them
 * meets the polynomial's steep places), after 8 by 3e-3 and after 16 by 4e-3 to 6e-3 where its rank is full.  Where it is not,
 * each step multiplies by 3.4 whatever rounding has left across the null space, in any arithmetic: 1e-2 after 8 steps, 0.1 after 10
 * and X itself after 12 (in 32 bits throughout two to three steps later).  More than seven steps are for matrices of full rank.
 * A gradient that is not finite makes its whole matrix NaN.  The sum of A's products over a long side is not split: matrices are
 * meant to be many or large, not one of a few rows by millions.
 *   grad_scale  device float [1] or NULL (1).  If it is not finite the whole step is left out.
 *   frozen      device uint8 or NULL, indexed by `module`: the out_mask of egeria_plasticity_evaluate as it is.  A frozen
 *               matrix is neither read nor written.  (Not to be written while the call runs.)
 * 0 <= beta < 1; lr not negative; eps at least 1e-30.  The call can be captured into a CUDA graph and replayed. */
egeria_status egeria_muon_step(egeria_muon *muon, void *cuda_stream, double lr, double beta, int nesterov, double eps, const float *grad_scale,
                               const uint8_t *frozen);

/* As egeria_ops_device_status, and the test hook as egeria_ops_debug_stall_next: of the next step's products. */
egeria_status egeria_muon_device_status(egeria_muon *muon);
egeria_status egeria_muon_debug_stall_next(egeria_muon *muon, int kind);

/* Number of kernels launched through this handle so far. */
int64_t egeria_muon_launch_count(const egeria_muon *muon);

#ifdef __cplusplus
}
#endif
#endif /* EGERIA_OPS_H_ */
