/*
 * pam_training.h -- C ABI of the layer-and-step side of a PAM transformer on
 * AMD Instinct MI355X (gfx950): linear layers with bias, activation and
 * residual around their PAM product (see pam.h), the gradient of what they add
 * to it, and the optimizer's step over all parameters.  Part of libpam.so.
 *
 * Kosson & Jaggi, Sec. 3.2, replace the products of the linear layers by PAM;
 * bias, activation and residual, and the optimizer, are ordinary float32
 * arithmetic here.
 *
 * The conventions of pam.h hold: device pointers, leading dimensions in
 * elements, every call asynchronous on `stream`, no allocation, arguments
 * validated before anything is launched.  A call's arguments are one structure
 * (and, for the calls over many tensors, an array of host structures), read
 * before the call returns.  The memory from a written operand's first element to
 * its last may not overlap that of another operand, unless the call says
 * otherwise: this is checked, and refused.
 */
#ifndef PAM_TRAINING_H_
#define PAM_TRAINING_H_

#include "pam.h"
#include "pam_attention.h" /* pam_type_t */

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Activations, f(z):
 *   RELU       z > 0 ? z : 0
 *   GELU       z P(N <= z), N a standard normal variable
 *   GELU_TANH  z s(2 sqrt(2/pi) (z + 0.044715 z^3)), s(u) = 1 / (1 + exp(-u))
 *   SILU       z s(z)
 * NaN gives NaN; an infinite z gives the limit or, of the smooth ones at
 * -inf, NaN where the formula does.  Results from 2^-126 on are there, however far
 * z is; of the slopes f'(z) those below 2^-118 may be zero.
 */
#ifdef __cplusplus
typedef enum : int32_t {
#else
typedef enum {
#endif
    PAM_ACT_NONE = 0,
    PAM_ACT_RELU = 1,
    PAM_ACT_GELU = 2,
    PAM_ACT_GELU_TANH = 3,
    PAM_ACT_SILU = 4
} pam_activation_t;

/*
 * A linear layer: with z = x .^ w^T + bias,  y = f(z) + residual.
 *
 *   x (m x k), w (n x k): row-major, of `type`; with float32 and mantissa_bits
 *       < 23 every element is first rounded to as many mantissa bits (bfloat16:
 *       mantissa_bits 23)
 *   bias: n float32 values, or NULL
 *   residual: m x n of out_type, or NULL; y itself (with ldr == ldy) is allowed
 *   y, z: m x n of out_type; z may be NULL (not written).  float32 arithmetic,
 *       rounded once
 *   workspace: pam_linear_workspace_size bytes, 16-byte aligned (NULL if those
 *       are 0)
 * The product's plan is pam_gemm_plan's; its tiles take long sums in parts of
 * 1024 terms (up to k = 1024 the sums are pam_gemm_batched_ws's, bit for bit).
 * k == 0 counts as a product of zeros.  m, n <= 2^31 - 1024.
 */
typedef struct {
    const void *x, *w;
    const float *bias;
    const void *residual;
    void *y, *z;
    void *workspace;
    int64_t m, n, k;
    int64_t ldx, ldw, ldr, ldy, ldz;
    int64_t workspace_bytes;
    pam_type_t type, out_type;
    pam_activation_t activation;
    int32_t mantissa_bits;
} pam_linear_t;
pam_status_t pam_linear_workspace_size(int64_t m, int64_t n, int64_t k, size_t *bytes);
pam_status_t pam_linear(const pam_linear_t *args, hipStream_t stream);

/*
 * The gradient of what a linear layer adds to its product: from dy, the
 * gradient of y, and z, as the forward pass wrote it,
 *   dz = dy f'(z)                (m x n, of dy's type, rounded once; NULL: not written)
 *   db = the sum of dz's rows    (n float32 values, from dz before its rounding; NULL: not written)
 * in an order fixed by the sizes.  RELU's slope at 0 is 0.  PAM_ACT_NONE takes
 * no z, and writes db alone (dz is dy).  dz may be dy (with lddz == lddy) or z
 * (with lddz == ldz and the same type).
 *
 *   dy, z: m x n, each float32 or bfloat16; n <= 2^31 - 1024
 *   workspace: pam_activation_grad_workspace_size bytes, 16-byte aligned (NULL if
 *       those are 0, or without db)
 */
typedef struct {
    const void *dy, *z;
    void *dz;
    float *db;
    void *workspace;
    int64_t m, n;
    int64_t lddy, ldz, lddz;
    int64_t workspace_bytes;
    pam_type_t type, z_type;
    pam_activation_t activation;
    int32_t reserved;
} pam_activation_grad_t;
pam_status_t pam_activation_grad_workspace_size(int64_t m, int64_t n, size_t *bytes);
pam_status_t pam_activation_grad(const pam_activation_grad_t *args, hipStream_t stream);

/*
 * One tensor of an optimizer's step: n parameters, contiguous, with their
 * gradients (g: of the call's gradient type) and the running averages of the
 * gradients (avg) and of their squares (sq).
 *
 * With 32-bit states avg and sq are n float32 values (the scales NULL).  With
 * 8-bit states they are n bytes, in blocks of PAM_STATE_BLOCK values, the last
 * one shorter, each with a float32 scale, the block's largest magnitude:
 *   avg: bit 7 the sign, c = the low seven bits: the scale times the float32 of
 *        encoding (c + 889) << 20 (8 steps an octave from 1 down, 16 octaves); c == 0: zero
 *   sq:  c = all eight bits: the scale times the float32 of encoding
 *        (c + 761) << 20 (32 octaves); c == 0: zero
 * A fresh state is all zeros.
 *
 * copy: n bfloat16 values, the new parameters rounded (for the products of the
 * next pass), or NULL.
 */
#define PAM_STATE_BLOCK 256
typedef struct {
    float *p;
    const void *g;
    void *avg, *sq;
    float *avg_scale, *sq_scale;
    uint16_t *copy;
    int64_t n;
} pam_step_tensor_t;

/*
 * norm = the square root of the sum of the squares of all gradients (the n
 * and g of `count` tensors; nothing else of them is looked at), one float32.
 * Summed in float64, in an order fixed by the sizes.
 *   workspace: pam_grad_norm_workspace_size bytes (at most 8 (2048 + count)),
 *       16-byte aligned; a call's own
 */
pam_status_t pam_grad_norm_workspace_size(const pam_step_tensor_t *tensors, int64_t count, size_t *bytes);
pam_status_t pam_grad_norm(const pam_step_tensor_t *tensors, int64_t count, pam_type_t grad_type, float *norm,
                                   void *workspace, int64_t workspace_bytes, hipStream_t stream);

/*
 * One AdamW step over `count` tensors:
 *   g'  = g min(1, max_norm / (norm + 1e-6))         (norm: one float32; NULL: g' = g)
 *   avg = beta1 avg + (1 - beta1) g'
 *   sq  = beta2 sq + (1 - beta2) g'^2
 *   p   = p (1 - lr weight_decay)
 *         - lr / (1 - beta1^t) avg / (sqrt(sq) / sqrt(1 - beta2^t) + eps)
 * t = step, or *step_device where that is not NULL (one int64 from 1 on, read when
 * the kernel runs, so that a captured step counts on; 1 - beta^t is then computed in
 * float32 there, and p may differ from that of the same `step` in its last bits: by
 * a dozen units of 2^-24 of what it moves by, and its rounding).  p takes the averages
 * before they are rounded to 8 bits.
 *
 * Rounding to 8 bits is stochastic: with f the float32 encoding of |value| /
 * scale, the code is (f + r) >> 20 less the offset above, at least 0, and of sq
 * at least 1 where the value is not 0; r = 16 h + 8, h the low (avg) or high
 * (sq) 16 bits of mix(i + mix(mix(seed + t 0x9E3779B9) + j)) for element i of
 * tensor j, all of 32 bits,
 *   mix(x): x = (x ^ x >> 16) 0x7FEB352D; x = (x ^ x >> 15) 0x846CA68B; x ^ x >> 16
 * (published by C. Wellons, "Prospecting for Hash Functions", 2018).
 * Each operation on the way from the old codes to the new ones is rounded to
 * float32 by itself, as
 *   avg = fl(fl(avg beta1) + fl(g' (1 - beta1))),
 *   sq  = fl(fl(sq beta2) + fl(fl(g' (1 - beta2)) g')),
 * so that the codes are the same wherever they are computed.  With states in 8
 * and in 32 bits, what is below 2^-126 counts as zero, among operands and among
 * the results of each operation: from a fresh state and beta2 = 0.999, sq (and in 8
 * bits its code) is 0 for a gradient below 3.4e-18, and p steps by avg / eps there,
 * which for eps == 0 is infinite.  A NaN or an infinity among a block's new
 * averages makes the block's averages of that kind NaN or infinite.
 *
 * A tensor of 0 values is passed over.  The tensors may not share memory.
 */
typedef struct {
    const float *norm;
    const int64_t *step_device;
    double lr, beta1, beta2, eps, weight_decay, max_norm;
    int64_t step;      /* >= 1 */
    uint32_t seed;
    int32_t state_bits; /* 8 or 32 */
    pam_type_t grad_type;
    int32_t reserved;
} pam_adamw_t;
pam_status_t pam_adamw_step(const pam_step_tensor_t *tensors, int64_t count, const pam_adamw_t *args,
                                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PAM_TRAINING_H_ */
