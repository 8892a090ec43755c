// Device code shared by the PAM attention kernels (pam_attention.hip for few
// rows, pam_attention_tile.hip for many): the encodings, and which keys a
// unit's rows see.  Included by the HIP sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pam_attention_internal.h"
#include "pam_scalar.h"

namespace pamk {

constexpr float kNegInf = -__builtin_inff();

typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4a2 __attribute__((ext_vector_type(4), aligned(2)));

// 16 bytes of cache elements: T is the element's storage.
template <typename T> constexpr int kPer = 16 / sizeof(T);

template <typename T> __device__ __forceinline__ u32x4 load16(const void *base, int64_t at) {
    return *reinterpret_cast<const u32x4a2 *>(static_cast<const T *>(base) + at);
}

// Float32 encoding of element i of 16 loaded bytes.
template <typename T> __device__ __forceinline__ uint32_t element(const u32x4 &w, int i) {
    if constexpr (sizeof(T) == 4)
        return w[i];
    else
        return i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16;
}

__device__ __forceinline__ uint32_t load_bits(const void *base, int64_t at, bool bf16) {
    return bf16 ? (uint32_t) static_cast<const uint16_t *>(base)[at] << 16 : static_cast<const uint32_t *>(base)[at];
}

__device__ __forceinline__ float one_mantissa(uint32_t a) {
    return __uint_as_float((a & kMant) | kBias);
}
__device__ __forceinline__ float power(uint32_t a) { return __uint_as_float(a & kSignExp); }

// b' of an encoding: zeros and denormals as zero, NaN as inf.
__device__ __forceinline__ uint32_t biased(uint32_t b) {
    const uint32_t mag = b & kMag;
    const uint32_t flushed = mag < kMinNormal ? 0u : mag > kInf ? kInf : mag;
    return ((b & kSign) | flushed) - kBias;
}

__device__ __forceinline__ float pam_fma(float a1, float m, uint32_t b, float acc) {
    return __builtin_fmaf(__uint_as_float(__float_as_uint(a1) + b), m, acc);
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & kExpMask) != kExpMask; }

// n / divisor, the host's fast_divisor.
__device__ __forceinline__ uint32_t divided(uint32_t n, uint32_t mul, uint32_t shift) {
    return (__umulhi(n, mul) + n) >> shift;
}

// The unit a workgroup works on, and which keys its rows see.
struct Unit {
    int b, head, first_row, rows;   // rows of it that exist
    int64_t first_token;            // token of row 0 of the sequence's block of new tokens
    int64_t position;               // of the sequence's new token 0
    int kv;                         // keys of the sequence, at most max_kv
    int lo, hi;                     // keys any of the rows sees
    const int32_t *table;

    __device__ __forceinline__ Unit(const AttentionParams &p, int unit) {
        const int bh = (int)divided((uint32_t)unit, p.blocks_mul, p.blocks_shift);
        const int block = unit - bh * p.row_blocks;
        b = (int)divided((uint32_t)bh, p.heads_mul, p.heads_shift);
        head = bh - b * p.kv_heads;
        first_token = p.q_starts ? p.q_starts[b] : b;
        const int64_t count = p.q_starts ? (int64_t)p.q_starts[b + 1] - first_token : 1;
        const int64_t length = p.kv_lens[b];
        kv = (int)std::min<int64_t>(std::max<int64_t>(length, 0), p.max_kv);
        position = length - count;
        table = p.table + (int64_t)b * p.table_stride;
        first_row = block * p.rows;
        int64_t live = std::min<int64_t>(count, p.max_q);
        live = std::min<int64_t>(live, p.tokens - first_token);
        if (first_token < 0)
            live = 0;
        if (p.k.pages <= 0)
            kv = 0;
        rows = (int)std::min<int64_t>(std::max<int64_t>(live * p.group - first_row, 0), p.rows);
        lo = hi = 0;
        if (rows > 0) {
            lo = row_lo(p, 0);
            hi = row_hi(p, rows - 1);
        }
    }
    __device__ __forceinline__ int token(const AttentionParams &p, int row) const {
        return (int)divided((uint32_t)(first_row + row), p.group_mul, p.group_shift);
    }
    // Keys lo <= j < hi are those the row sees (page permitting).
    __device__ __forceinline__ int row_lo(const AttentionParams &p, int row) const {
        if (p.window <= 0)
            return 0;
        const int64_t at = position + token(p, row) - p.window + 1;
        return (int)std::min<int64_t>(std::max<int64_t>(at, 0), kv);
    }
    __device__ __forceinline__ int row_hi(const AttentionParams &p, int row) const {
        if (!p.causal)
            return kv;
        return (int)std::min<int64_t>(std::max<int64_t>(position + token(p, row) + 1, 0), kv);
    }
    __device__ __forceinline__ int64_t q_at(const AttentionParams &p, int row) const {
        const int i = token(p, row), g = first_row + row - i * p.group;
        return (first_token + i) * p.q_token + (int64_t)(head * p.group + g) * p.q_head;
    }
    __device__ __forceinline__ int64_t out_at(const AttentionParams &p, int row) const {
        const int i = token(p, row), g = first_row + row - i * p.group;
        return (first_token + i) * p.out_token + (int64_t)(head * p.group + g) * p.out_head;
    }
    // Element offset of a key's row in a cache, or -1 where its page is not one.
    __device__ __forceinline__ int64_t key_at(const AttentionParams &p, const CacheView &c, int key) const {
        const uint32_t page = divided((uint32_t)key, p.page_mul, p.page_shift);
        const int id = table[page];
        if (id < 0 || id >= c.pages)
            return -1;
        return (int64_t)id * c.page + (int64_t)(key - (int)(page * p.page_size)) * c.slot + (int64_t)head * c.head;
    }
};

// 2^(t - m); 0 for t = -inf also where the maximum is -inf.
__device__ __forceinline__ float exp2_from(float t, float m) {
    return __builtin_amdgcn_exp2f(t - (m == kNegInf ? 0.0f : m));
}

// A probability as b'; a row whose sum is NaN is set to NaN at the end.
__device__ __forceinline__ uint32_t probability(float e, float inverse) {
    const uint32_t bits = __float_as_uint(e * inverse);
    return (bits < kMinNormal || bits >= kInf ? 0u : bits) - kBias;
}

}  // namespace pamk
