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
 * anything is launched.  A call's arguments are one structure, read before the
 * call returns: the pointers, then the layouts and sizes.  The rows of a
 * written operand may not share memory: each of its strides is at least the
 * extent of the dimensions of smaller stride.  What lies in device memory
 * (positions, slots, lengths, page tables) cannot be validated by the host:
 * each call says what a value out of range does, and none makes a kernel leave
 * its buffers as long as the arrays have the stated sizes.
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
 * heads: views into a projection's output are such.  heads == 0: the operand
 * is not given. */
typedef struct {
    int64_t stride_token, stride_head;
    int32_t heads;
    pam_type_t type;
} pam_heads_t;

/*
 * The position rotation: the first `rot` values of a head (even, 0 .. d) are
 * pairs p = 0 .. rot/2 - 1, values (p, p + rot/2), or (2p, 2p + 1) where
 * interleaved != 0.  A token at position n turns pair p by the angle whose
 * cosine and sine are cos[n*rot/2 + p] and sin[n*rot/2 + p]; the tables have
 * `rows` positions.  positions: one int32 a token.  A position outside
 * [0, rows) gives NaN in the rotated values.  rot == 0: no rotation.
 */
typedef struct {
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
    int64_t stride_page, stride_slot, stride_head;
    int64_t pages;
    int32_t page_size;
    int32_t heads;
    pam_type_t type;
    int32_t reserved;
} pam_cache_t;

/*
 * Norm and rotation of queries and keys in one pass.  For each token t and
 * head h, with x = in[t][h] and w the weight of d values:
 *   y = x w / sqrt(mean(x^2) + eps)      (weight NULL: y = x)
 *   out[t][h] = rotation of y at the token's position
 * in float32, rounded once to out's type (nearest even).  Squares and eps below
 * 2^-126 count as zero; a mean past the float32 range gives zeros.  d even,
 * 2 .. 256.
 * q and k are each a pair of in and out with equal head counts (out may be
 * in); both or one of them given.  q_in and k_in have one type.  tokens == 0
 * launches nothing.  eps >= 0 and finite.
 */
typedef struct {
    const void *q_in;
    const float *q_weight;
    const void *k_in;
    const float *k_weight;
    const int32_t *positions;
    const float *cos, *sin;
    void *q_out;
    void *k_out;
    pam_heads_t q_in_heads, q_out_heads, k_in_heads, k_out_heads;
    pam_rotation_t rotation;
    int64_t tokens;
    int32_t d;
    float eps;
} pam_norm_rope_t;

pam_status_t pam_norm_rope(const pam_norm_rope_t *args, hipStream_t stream);

/*
 * Its gradient.  With dz = grad_out[t][h] and g = dz rotated back:
 *   dweight[i] = sum over t, h of g_i x_i r,   r = 1 / sqrt(mean(x^2) + eps)
 *   dx = r (u - x r^2 mean(u x)),   u = g w    (weight NULL: dx = g)
 * q: q_in (the forward input), q_weight, dq_out (gradient of its output),
 * dq_in (gradient of its input, written), dq_weight (d float32, written;
 * non-NULL exactly where the weight is).  The same for k; one of the two may
 * be left out.  The three heads of q and of k have one type.  The sums over
 * tokens run in a fixed order over partial sums in `workspace`
 * (pam_norm_rope_grad_workspace_size bytes, 16-byte aligned; none needed
 * without weights).  tokens == 0 writes zeros to the weights' gradients.
 */
typedef struct {
    const void *q_in;
    const float *q_weight;
    const void *dq_out;
    const void *k_in;
    const float *k_weight;
    const void *dk_out;
    const int32_t *positions;
    const float *cos, *sin;
    void *dq_in;
    float *dq_weight;
    void *dk_in;
    float *dk_weight;
    void *workspace;
    pam_heads_t q_in_heads, dq_out_heads, dq_in_heads, k_in_heads, dk_out_heads, dk_in_heads;
    pam_rotation_t rotation;
    int64_t tokens;
    int64_t workspace_bytes;
    int32_t d;
    float eps;
} pam_norm_rope_grad_t;

pam_status_t pam_norm_rope_grad_workspace_size(int64_t tokens, int32_t d, int32_t q_heads, int32_t k_heads,
                                               size_t *bytes);

pam_status_t pam_norm_rope_grad(const pam_norm_rope_grad_t *args, hipStream_t stream);

/*
 * Appends the keys and values of `tokens` tokens to a paged cache: token t
 * goes to slot slots[t] % page_size of page slots[t] / page_size; a slot
 * outside [0, pages * page_size) is not stored (padding tokens carry -1).
 * Keys are normed (k_weight non-NULL) and rotated (rot > 0) on the way as in
 * pam_norm_rope, values stored as they are; both are rounded to the cache's
 * type (nearest even).  q_in / q_out (optional): the same tokens' queries,
 * normed and rotated in the same launch.  k, v and q_in have one type, k and
 * v as many heads as the caches.  Two tokens with one slot race, and so do
 * caches that share memory.
 */
typedef struct {
    const void *k;
    const float *k_weight;
    const void *v;
    const void *q_in;
    const float *q_weight;
    const int64_t *slots;
    const int32_t *positions;
    const float *cos, *sin;
    void *k_cache;             /* written */
    void *v_cache;
    void *q_out;
    pam_heads_t k_heads, v_heads, q_in_heads, q_out_heads;
    pam_cache_t k_cache_layout, v_cache_layout;
    pam_rotation_t rotation;
    int64_t tokens;
    int32_t d;
    float eps;
} pam_append_kv_t;

pam_status_t pam_append_kv(const pam_append_kv_t *args, hipStream_t stream);

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
 * on it, whatever they hold: none on a bit of its outputs where no token of
 * its sequence and call sees them, and else, should they be inf or NaN, on
 * the order of its sums alone.  PAM terms below 2^-126 may count in a sum
 * instead of as zero.
 *
 * max_q: at least every sequence's count of new tokens (tokens past it get
 * no output, nor do tokens of no sequence); max_kv: at least every kv_lens[b]
 * (keys past it are not seen), at most table_width * page_size, the table's
 * row length.  q and out: tokens x heads x d, out float32; heads a multiple
 * of the caches'; d a multiple of 8, 8 .. 256.  window >= 0.  scale finite.
 * workspace: pam_paged_attention_workspace_size bytes for the same sizes (0
 * possible), 16-byte aligned, untouched by others until the call's kernels
 * are done.
 */
typedef struct {
    const void *q;
    const void *k_cache, *v_cache;
    const int32_t *q_starts;   /* batch + 1, or NULL */
    const int32_t *kv_lens;    /* batch */
    const int32_t *table;      /* batch rows of table_width entries */
    float *out;
    void *workspace;
    pam_heads_t q_heads, out_heads;
    pam_cache_t k_cache_layout, v_cache_layout;
    int64_t table_stride;
    int64_t tokens;            /* rows of q and out */
    int32_t d;
    int32_t batch;
    int32_t table_width;
    int32_t causal;
    int32_t window;
    float scale;
    int32_t max_q;
    int32_t max_kv;
    int64_t workspace_bytes;
} pam_paged_attention_t;

pam_status_t pam_paged_attention_workspace_size(int32_t d, int32_t q_heads, int32_t kv_heads, pam_type_t kv_type,
                                                int32_t batch, int32_t max_q, int32_t max_kv, size_t *bytes);

pam_status_t pam_paged_attention(const pam_paged_attention_t *args, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PAM_ATTENTION_H_ */
