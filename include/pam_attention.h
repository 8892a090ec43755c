/*
 * pam_attention.h -- C ABI of the attention-side operators of a PAM
 * transformer on AMD Instinct MI355X (gfx950): norms of queries and keys
 * with the position rotation, a paged key/value cache, and attention over it
 * whose products are piecewise affine (PAM, see pam.h).  Part of libpam.so.
 *
 * Kosson & Jaggi, Sec. 3.2, replace the products of the linear layers and of
 * the attention (Q K^T and P V) by PAM; norms, the position rotation and the
 * softmax stay ordinary float32 arithmetic, and so they are here.
 *
 * The conventions of pam.h hold: device pointers, strides in elements, every
 * call asynchronous on `stream`, no allocation, arguments validated before
 * anything is launched.  What lies in device memory (positions, slots,
 * lengths, page tables) cannot be validated by the host: each call says what
 * a value out of range does, and none makes a kernel leave its buffers as
 * long as the arrays have the stated sizes.
 */
#ifndef PAM_ATTENTION_H_
#define PAM_ATTENTION_H_

#include "pam.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the heads and caches. */
#ifdef __cplusplus
typedef enum : int32_t { PAM_TYPE_F32 = 0, PAM_TYPE_BF16 = 1 } pam_type_t;
#else
typedef enum { PAM_TYPE_F32 = 0, PAM_TYPE_BF16 = 1 } pam_type_t;
#endif

/* Largest number of values per head. */
#define PAM_MAX_HEAD_DIM 256

/* Values x[t][h][i] = data[t*stride_token + h*stride_head + i] of `heads`
 * heads: views into a projection's output are such. */
typedef struct {
    void *data;
    int64_t stride_token, stride_head;
    int32_t heads;
    pam_type_t type;
} pam_heads_t;

/*
 * The position rotation: the first `rot` values of a head (even, 0..d) are
 * pairs p = 0 .. rot/2 - 1, values (p, p + rot/2), or (2p, 2p + 1) where
 * interleaved != 0.  A token at position n turns pair p by the angle whose
 * cosine and sine are cos[n*rot/2 + p] and sin[n*rot/2 + p]; the tables have
 * `rows` positions.  positions: one int32 a token.  A position outside
 * [0, rows) gives NaN in the rotated values.
 */
typedef struct {
    const int32_t *positions;
    const float *cos, *sin;
    int64_t rows;
    int32_t rot;
    int32_t interleaved;
} pam_rotation_t;

/*
 * A paged cache of one layer's keys or values: value (slot s of page p, head
 * h, index i) = data[p*stride_page + s*stride_slot + h*stride_head + i] for
 * p < pages, s < page_size, h < heads.  1 <= page_size, pages * page_size
 * < 2^31.
 */
typedef struct {
    void *data;
    int64_t stride_page, stride_slot, stride_head;
    int64_t pages;
    int32_t page_size;
    int32_t heads;
    pam_type_t type;
} pam_cache_t;

/*
 * Norm and rotation of queries and keys in one pass.  For each token t and
 * head h, with x = in[t][h] and w the weight of d values:
 *   y = x w / sqrt(mean(x^2) + eps)      (weight NULL: y = x)
 *   out[t][h] = rotation of y at the token's position
 * in float32, rounded once to out's type (nearest even).  d even, 2 .. 256.
 * q and k are each a pair of in and out with equal head counts (out may be
 * in); both or one of them given (NULL in and out: none).  q_in and k_in
 * have one type.  rotation NULL: no rotation.  tokens == 0 launches nothing.
 * eps >= 0 and finite.
 */
pam_status_t pam_norm_rope(int64_t tokens, int32_t d, const pam_heads_t *q_in, const float *q_weight,
                           const pam_heads_t *q_out, const pam_heads_t *k_in, const float *k_weight,
                           const pam_heads_t *k_out, float eps, const pam_rotation_t *rotation,
                           hipStream_t stream);

/*
 * Its gradient.  With dz = grad_out[t][h] and g = dz rotated back:
 *   dweight[i] = sum over t, h of g_i x_i r,   r = 1 / sqrt(mean(x^2) + eps)
 *   dx = r (u - x r^2 mean(u x)),   u = g w    (weight NULL: dx = g)
 * q: q_in (the forward input), q_weight, dq_out (gradient of its output),
 * dq_in (gradient of its input, written), dq_weight (d float32, written;
 * non-NULL exactly where the weight is).  The same for k; one of the two may
 * be left out.  The three heads of q and of k have one type.  The sums over
 * tokens run in a fixed order over partial sums in `workspace`
 * (pam_norm_rope_grad_workspace_size bytes, 16-byte aligned; 0 without
 * weights).  tokens == 0 writes zeros to the weights' gradients.
 */
pam_status_t pam_norm_rope_grad_workspace_size(int64_t tokens, int32_t d, int32_t q_heads, int32_t k_heads,
                                               size_t *bytes);

pam_status_t pam_norm_rope_grad(int64_t tokens, int32_t d, const pam_heads_t *q_in, const float *q_weight,
                                const pam_heads_t *dq_out, const pam_heads_t *dq_in, float *dq_weight,
                                const pam_heads_t *k_in, const float *k_weight, const pam_heads_t *dk_out,
                                const pam_heads_t *dk_in, float *dk_weight, float eps,
                                const pam_rotation_t *rotation, void *workspace, size_t workspace_bytes,
                                hipStream_t stream);

/*
 * Appends the keys and values of `tokens` tokens to a paged cache: token t
 * goes to slot slots[t] % page_size of page slots[t] / page_size; a slot
 * outside [0, pages * page_size) is not stored (padding tokens carry -1).
 * Keys are normed (k_weight non-NULL) and rotated (rotation non-NULL) on the
 * way as in pam_norm_rope, values stored as they are; both are rounded to the
 * cache's type (nearest even).  q_in / q_out (NULL: none): the same tokens'
 * queries, normed and rotated in the same launch.  k, v and q_in have one
 * type, k and v as many heads as the caches.  Two tokens with one slot race.
 */
pam_status_t pam_append_kv(int64_t tokens, int32_t d, const pam_heads_t *k, const float *k_weight,
                           const pam_heads_t *v, const pam_heads_t *q_in, const float *q_weight,
                           const pam_heads_t *q_out, float eps, const pam_rotation_t *rotation,
                           const pam_cache_t *k_cache, const pam_cache_t *v_cache, const int64_t *slots,
                           hipStream_t stream);

/*
 * PAM attention of new tokens over a paged cache.  Sequence b (0 <= b <
 * batch) has kv_lens[b] keys, key j in slot j % page_size of page
 * table[b*table_stride + j / page_size], and the new tokens q_starts[b] ..
 * q_starts[b+1] - 1 of q (q_starts NULL: token b alone), which are its last
 * positions: token i of n stands at kv_lens[b] - n + i.  Query head h reads
 * key head h / (q heads / cache heads).  With .^ the PAM product,
 *   s_j = scale * sum_i q_i .^ k_ji,  P_j = exp(s_j - max s) / sum exp(s - max s),
 *   out_i = sum_j P_j .^ v_ji
 * over the keys j the token sees: j < kv_lens[b]; j <= its position where
 * causal != 0; j > its position - window where window > 0; and those whose
 * page lies in [0, pages) and whose table entry lies below max_kv.  The
 * softmax is normalised before the second product, as a trained softmax
 * followed by a product is: PAM commutes with powers of two only.  A token
 * that sees no key gets zeros, also where all its scores are -inf; a NaN
 * score gives NaN.  Keys and values a token does not see have no influence
 * on it, whatever they hold.  PAM terms below 2^-126 may count in a sum
 * instead of as zero.
 *
 * max_q: at least every sequence's count of new tokens (tokens past it get
 * no output); max_kv: at least every kv_lens[b] (keys past it are not seen),
 * at most table_width * page_size, the table's row length.  q and out: tokens
 * x heads x d, out float32; heads a multiple of the caches'; d a multiple of
 * 8, 8 .. 256.  scale finite.  workspace: pam_paged_attention_workspace_size
 * bytes for the same sizes (0 possible), 16-byte aligned, untouched by others
 * until the call's kernels are done.
 */
typedef struct {
    const int32_t *q_starts;   /* batch + 1, or NULL */
    const int32_t *kv_lens;    /* batch */
    const int32_t *table;      /* batch rows of table_width entries */
    int64_t table_stride;
    int64_t tokens;            /* rows of q and out */
    int32_t batch;
    int32_t table_width;
    int32_t max_q;
    int32_t max_kv;
    int32_t causal;
    int32_t window;
    float scale;
} pam_sequences_t;

pam_status_t pam_paged_attention_workspace_size(int32_t d, int32_t q_heads, int32_t kv_heads, pam_type_t kv_type,
                                                int32_t batch, int32_t max_q, int32_t max_kv, size_t *bytes);

pam_status_t pam_paged_attention(int32_t d, const pam_heads_t *q, const pam_cache_t *k_cache,
                                 const pam_cache_t *v_cache, const pam_sequences_t *sequences,
                                 const pam_heads_t *out, void *workspace, size_t workspace_bytes,
                                 hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PAM_ATTENTION_H_ */
