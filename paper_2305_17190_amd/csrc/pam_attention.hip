// PAM attention over a paged key/value cache for gfx950 (Kosson & Jaggi, Sec.
// 3.2: the attention's products Q K^T and P V are PAM products, the softmax
// between them is ordinary).
//
//   s_j = scale sum_i q_i .^ k_ji,  P_j = exp(s_j - max s) / sum exp(s - max s),
//   out_i = sum_j P_j .^ v_ji
//
// The sum of the exponentials is known before the second product: PAM
// commutes with powers of two only, so P V cannot be rescaled afterwards, and
// each unit of work (a key head of a sequence and some of its rows) first
// scores all its keys, then reads the values.
//
// PAM on float hardware: for a = 2^E (1 + M) let a1 be the encoding of 1 + M
// and m = a with its mantissa cleared (+-2^E; +-0 for zeros and denormals),
// and b' = b's encoding less one bias.  a1 + b' as integers is the encoding of
// PAM(1 + M, b), and times m it is PAM(a, b) wherever that is a normal number:
// an integer addition and a float fma a term.  Keys and values are `a`, made
// once for all rows; queries and probabilities are `b`, where a zero's sum
// stays below the normal range and reads as zero.  A value with exponent
// field 255 has m = +-inf, and b = NaN is given inf's encoding, so that any
// NaN, inf or product past the range leaves a non-finite sum: such sums are
// computed again term by term from the complete definition, over the keys the
// row sees only.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pam_attention_device.h"

namespace pamk {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// Scores of keys begin <= j < end (within the unit's lo .. hi) into
// s[(j - begin) * R + row]; -inf where the row does not see the key.
// `lanes` L lanes hold a key, 16 bytes each.
template <typename T, int L, int R>
__device__ __forceinline__ void score_keys(const AttentionParams &p, const Unit &unit, int begin, int end, float *s,
                                           const int *lo, const int *hi) {
    constexpr int E = kPer<T>;
    constexpr int K = 64 / L;         // keys of one load of a wave
    constexpr int U = 4;              // loads in flight
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int at = (lane % L) * E;
    const bool holds = at < p.d;
    uint32_t q[R][E];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t row = r < unit.rows ? unit.q_at(p, r) : 0;
#pragma unroll
        for (int i = 0; i < E; ++i)
            q[r][i] = biased(holds && r < unit.rows ? load_bits(p.q, row + at + i, p.q_bf16) : 0u);
    }
    for (int first = begin + wave * U * K; first < end; first += waves * U * K) {
        u32x4 w[U];
        int64_t from[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = first + u * K + lane / L;
            from[u] = key < end ? unit.key_at(p, p.k, key) : -1;
            w[u] = u32x4{0, 0, 0, 0};
            if (from[u] >= 0 && holds)
                w[u] = load16<T>(p.k.data, from[u] + at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float sum[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
                sum[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t a = element<T>(w[u], i);
                const float a1 = one_mantissa(a), m = power(a);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    sum[r] = pam_fma(a1, m, q[r][i], sum[r]);
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int x = 1; x < L; x *= 2)
                    sum[r] += __shfl_xor(sum[r], x);
            const int key = first + u * K + lane / L;
            if (lane % L == 0 && key < end) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float t = kNegInf;
                    if (r < unit.rows && from[u] >= 0 && key >= lo[r] && key < hi[r]) {
                        if (!finite(sum[r])) {
                            sum[r] = 0.0f;
                            const int64_t row = unit.q_at(p, r);
                            for (int i = 0; i < p.d; ++i)
                                sum[r] += __uint_as_float(pam_full(load_bits(p.q, row + i, p.q_bf16),
                                                                   load_bits(p.k.data, from[u] + i, sizeof(T) == 2)));
                        }
                        t = sum[r] * p.scale;
                    }
                    s[(key - begin) * R + r] = t;
                }
            }
        }
    }
}

// Maximum of the rows' scores s[0 .. keys * R) over the workgroup.
template <int R> __device__ __forceinline__ void row_max(const float *s, int keys, float (&m)[R], float *scratch) {
#pragma unroll
    for (int r = 0; r < R; ++r)
        m[r] = kNegInf;
    for (int j = threadIdx.x; j < keys; j += blockDim.x)
#pragma unroll
        for (int r = 0; r < R; ++r)
            m[r] = fmaxf(m[r], s[j * R + r]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        for (int x = 1; x < 64; x *= 2)
            m[r] = fmaxf(m[r], __shfl_xor(m[r], x));
        if ((threadIdx.x & 63) == 0)
            scratch[(threadIdx.x >> 6) * R + r] = m[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
        for (int w = 0; w < (int)(blockDim.x >> 6); ++w)
            m[r] = fmaxf(m[r], scratch[w * R + r]);
}

template <int R> __device__ __forceinline__ void row_sum(float (&l)[R], float *scratch) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        for (int x = 1; x < 64; x *= 2)
            l[r] += __shfl_xor(l[r], x);
        if ((threadIdx.x & 63) == 0)
            scratch[(threadIdx.x >> 6) * R + r] = l[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        l[r] = 0.0f;
        for (int w = 0; w < (int)(blockDim.x >> 6); ++w)
            l[r] += scratch[w * R + r];
    }
}

// out[row][i] = sum over keys begin <= j < end of P .^ v, the probabilities'
// b' in pr[(j - begin) * R + row]; to out's rows (partial == nullptr) or
// partial[row * d + i].  scratch: waves * R * L * 16 / sizeof(T) floats.
template <typename T, int L, int R>
__device__ __forceinline__ void value_keys(const AttentionParams &p, const Unit &unit, int begin, int end,
                                           const uint32_t *pr, float *scratch, const int *lo, const int *hi,
                                           const float *sums, float *partial) {
    constexpr int E = kPer<T>;
    constexpr int K = 64 / L;
    constexpr int U = 4;
    constexpr int D = L * E;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int at = (lane % L) * E;
    const bool holds = at < p.d;
    float acc[R][E];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < E; ++i)
            acc[r][i] = 0.0f;
    for (int first = begin + wave * U * K; first < end; first += waves * U * K) {
        u32x4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = first + u * K + lane / L;
            const int64_t from = key < end ? unit.key_at(p, p.v, key) : -1;
            w[u] = u32x4{0, 0, 0, 0};
            if (from >= 0 && holds)
                w[u] = load16<T>(p.v.data, from + at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = min(first + u * K + lane / L, end - 1);
            uint32_t b[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
                b[r] = pr[(key - begin) * R + r];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t a = element<T>(w[u], i);
                const float a1 = one_mantissa(a), m = power(a);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    acc[r][i] = pam_fma(a1, m, b[r], acc[r][i]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < E; ++i)
#pragma unroll
            for (int x = L; x < 64; x *= 2)
                acc[r][i] += __shfl_xor(acc[r][i], x);
    if (lane < L) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < E; ++i)
                scratch[(wave * R + r) * D + at + i] = acc[r][i];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < R * D; e += blockDim.x) {
        const int r = e / D, i = e % D;
        if (r >= unit.rows || i >= p.d)
            continue;
        float sum = 0.0f;
        for (int w = 0; w < waves; ++w)
            sum += scratch[w * R * D + e];
        if (!finite(sum)) {
            // Term by term, over the keys the row sees.
            sum = 0.0f;
            for (int key = max(begin, lo[r]); key < min(end, hi[r]); ++key) {
                const int64_t from = unit.key_at(p, p.v, key);
                if (from >= 0)
                    sum += __uint_as_float(pam_full(pr[(key - begin) * R + r] + kBias,
                                                    load_bits(p.v.data, from + i, sizeof(T) == 2)));
            }
        }
        if (!(sums[r] > 0.0f))      // no weight, or a NaN score
            sum = sums[r];
        if (partial != nullptr)
            partial[r * p.d + i] = sum;
        else
            p.out[unit.out_at(p, r) + i] = sum;
    }
}

template <int R>
__device__ __forceinline__ void row_ranges(const AttentionParams &p, const Unit &unit, int *lo, int *hi) {
    if (threadIdx.x < R) {
        const int r = threadIdx.x;
        lo[r] = r < unit.rows ? unit.row_lo(p, r) : 0;
        hi[r] = r < unit.rows ? unit.row_hi(p, r) : 0;
    }
    __syncthreads();
}

// A unit in one workgroup: its scores stay in LDS.
template <typename T, int L, int R>
__global__ void __launch_bounds__(kThreads) attention_whole_kernel(const AttentionParams p) {
    extern __shared__ float s[];
    __shared__ float scratch[kWaves * R * L * kPer<T>];
    __shared__ int lo[R], hi[R];
    __shared__ float sums[R];
    const Unit unit(p, blockIdx.x);
    if (unit.rows == 0)
        return;
    row_ranges<R>(p, unit, lo, hi);
    score_keys<T, L, R>(p, unit, unit.lo, unit.hi, s, lo, hi);
    __syncthreads();
    const int keys = max(unit.hi - unit.lo, 0);
    float m[R], l[R];
    row_max<R>(s, keys, m, scratch);
#pragma unroll
    for (int r = 0; r < R; ++r)
        l[r] = 0.0f;
    for (int j = threadIdx.x; j < keys; j += blockDim.x)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float e = exp2_from(s[j * R + r], m[r]);
            l[r] += e;
            s[j * R + r] = e;
        }
    row_sum<R>(l, scratch);
    float inverse[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        inverse[r] = l[r] > 0.0f ? 1.0f / l[r] : 0.0f;
        if (threadIdx.x == 0)
            sums[r] = l[r];
    }
    for (int j = threadIdx.x; j < keys; j += blockDim.x)
#pragma unroll
        for (int r = 0; r < R; ++r)
            s[j * R + r] = __uint_as_float(probability(s[j * R + r], inverse[r]));
    __syncthreads();
    value_keys<T, L, R>(p, unit, unit.lo, unit.hi, reinterpret_cast<const uint32_t *>(s), scratch, lo, hi, sums,
                        nullptr);
}

// Long contexts, first launch: scores of one split of a unit's keys, with the
// split's maximum and sum for each row.
template <typename T, int L, int R>
__global__ void __launch_bounds__(kThreads) attention_scores_kernel(const AttentionParams p) {
    extern __shared__ float s[];
    __shared__ float scratch[kWaves * R];
    __shared__ int lo[R], hi[R];
    const int split = blockIdx.x % p.splits, index = blockIdx.x / p.splits;
    const Unit unit(p, index);
    const int begin = max(unit.lo, split * p.split_keys), end = min(unit.hi, (split + 1) * p.split_keys);
    if (unit.rows == 0 || begin >= end)
        return;
    row_ranges<R>(p, unit, lo, hi);
    score_keys<T, L, R>(p, unit, begin, end, s, lo, hi);
    __syncthreads();
    float m[R], l[R];
    row_max<R>(s, end - begin, m, scratch);
#pragma unroll
    for (int r = 0; r < R; ++r)
        l[r] = 0.0f;
    float *to = p.scores + ((int64_t)index * p.splits * p.split_keys + begin) * R;
    for (int j = threadIdx.x; j < end - begin; j += blockDim.x)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            l[r] += exp2_from(s[j * R + r], m[r]);
            to[(int64_t)j * R + r] = s[j * R + r];
        }
    row_sum<R>(l, scratch);
    if (threadIdx.x == 0) {
        float *stats = p.stats + ((int64_t)index * p.splits + split) * 2 * R;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            stats[r] = m[r];
            stats[R + r] = l[r];
        }
    }
}

// Second launch: the unit's maxima and sums from all its splits', then one
// split's part of P V.
template <typename T, int L, int R>
__global__ void __launch_bounds__(kThreads) attention_values_kernel(const AttentionParams p) {
    extern __shared__ float s[];
    __shared__ float scratch[kWaves * R * L * kPer<T>];
    __shared__ int lo[R], hi[R];
    __shared__ float sums[R];
    const int split = blockIdx.x % p.splits, index = blockIdx.x / p.splits;
    const Unit unit(p, index);
    const int begin = max(unit.lo, split * p.split_keys), end = min(unit.hi, (split + 1) * p.split_keys);
    if (unit.rows == 0 || begin >= end)
        return;
    row_ranges<R>(p, unit, lo, hi);
    const int first = unit.lo / p.split_keys, last = (unit.hi - 1) / p.split_keys;
    const float *stats = p.stats + (int64_t)index * p.splits * 2 * R;
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        m[r] = kNegInf;
    for (int j = first + threadIdx.x; j <= last; j += blockDim.x)
#pragma unroll
        for (int r = 0; r < R; ++r)
            m[r] = fmaxf(m[r], stats[j * 2 * R + r]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        for (int x = 1; x < 64; x *= 2)
            m[r] = fmaxf(m[r], __shfl_xor(m[r], x));
        if ((threadIdx.x & 63) == 0)
            scratch[(threadIdx.x >> 6) * R + r] = m[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        for (int w = 0; w < kWaves; ++w)
            m[r] = fmaxf(m[r], scratch[w * R + r]);
        l[r] = 0.0f;
    }
    for (int j = first + threadIdx.x; j <= last; j += blockDim.x)
#pragma unroll
        for (int r = 0; r < R; ++r)
            l[r] += stats[j * 2 * R + R + r] * exp2_from(stats[j * 2 * R + r], m[r]);
    row_sum<R>(l, scratch);
    float inverse[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        inverse[r] = l[r] > 0.0f ? 1.0f / l[r] : 0.0f;
        if (threadIdx.x == 0)
            sums[r] = l[r];
    }
    const float *from = p.scores + ((int64_t)index * p.splits * p.split_keys + begin) * R;
    for (int j = threadIdx.x; j < end - begin; j += blockDim.x)
#pragma unroll
        for (int r = 0; r < R; ++r)
            s[j * R + r] = __uint_as_float(probability(exp2_from(from[(int64_t)j * R + r], m[r]), inverse[r]));
    __syncthreads();
    value_keys<T, L, R>(p, unit, begin, end, reinterpret_cast<const uint32_t *>(s), scratch, lo, hi, sums,
                        p.partial + ((int64_t)index * p.splits + split) * R * p.d);
}

// Third launch: the outputs, each the sum over its unit's splits in order; four
// a thread.
__global__ void __launch_bounds__(kThreads) attention_join_kernel(const AttentionParams p, int parts) {
    const int index = blockIdx.x / parts;
    const Unit unit(p, p.first_unit + index);
    const int e = ((blockIdx.x % parts) * kThreads + threadIdx.x) * 4;
    if (e >= unit.rows * p.d)
        return;
    const int first = unit.lo / p.split_keys, last = unit.hi > unit.lo ? (unit.hi - 1) / p.split_keys : first - 1;
    const float *partial = p.partial + (int64_t)index * p.splits * p.rows * p.d + e;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j = first; j <= last; ++j)
        sum += *reinterpret_cast<const f32x4 *>(partial + (int64_t)j * p.rows * p.d);
    const int r = e / p.d;
    *reinterpret_cast<f32x4 *>(p.out + unit.out_at(p, r) + (e - r * p.d)) = sum;
}

enum Which { kWhole, kScores, kValues };

template <typename T, int L, int R>
hipError_t launch(Which which, const AttentionParams &p, hipStream_t stream) {
    const unsigned units = (unsigned)(p.batch * p.kv_heads * p.row_blocks);
    const void *kernel = which == kWhole    ? (const void *)attention_whole_kernel<T, L, R>
                         : which == kScores ? (const void *)attention_scores_kernel<T, L, R>
                                            : (const void *)attention_values_kernel<T, L, R>;
    const size_t lds = (size_t)(which == kWhole ? p.max_kv : p.split_keys) * R * sizeof(float);
    const unsigned grid = which == kWhole ? units : units * (unsigned)p.splits;
    void *args[] = {const_cast<AttentionParams *>(&p)};
    return hipLaunchKernel(kernel, dim3(grid), dim3(kThreads), args, lds, stream);
}

template <typename T, int L> hipError_t for_rows(Which which, const AttentionParams &p, hipStream_t stream) {
    switch (p.rows) {
    case 1: return launch<T, L, 1>(which, p, stream);
    case 2: return launch<T, L, 2>(which, p, stream);
    case 4: return launch<T, L, 4>(which, p, stream);
    default: return launch<T, L, 8>(which, p, stream);
    }
}

hipError_t for_type(Which which, bool bf16, int lanes, const AttentionParams &p, hipStream_t stream) {
    switch (lanes) {
    case 4: return bf16 ? for_rows<uint16_t, 4>(which, p, stream) : for_rows<float, 4>(which, p, stream);
    case 8: return bf16 ? for_rows<uint16_t, 8>(which, p, stream) : for_rows<float, 8>(which, p, stream);
    case 16: return bf16 ? for_rows<uint16_t, 16>(which, p, stream) : for_rows<float, 16>(which, p, stream);
    case 32: return bf16 ? for_rows<uint16_t, 32>(which, p, stream) : for_rows<float, 32>(which, p, stream);
    default: return for_rows<float, 64>(which, p, stream);
    }
}

}  // namespace

hipError_t launch_attention_whole(bool bf16, int lanes, const AttentionParams &p, hipStream_t stream) {
    return for_type(kWhole, bf16, lanes, p, stream);
}

hipError_t launch_attention_scores(bool bf16, int lanes, const AttentionParams &p, hipStream_t stream) {
    return for_type(kScores, bf16, lanes, p, stream);
}

hipError_t launch_attention_values(bool bf16, int lanes, const AttentionParams &p, hipStream_t stream) {
    return for_type(kValues, bf16, lanes, p, stream);
}

hipError_t launch_attention_join(const AttentionParams &p, int units, hipStream_t stream) {
    const int parts = (p.rows * p.d / 4 + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(attention_join_kernel, dim3((unsigned)(units * parts)), dim3(kThreads), 0, stream, p, parts);
    return hipGetLastError();
}

}  // namespace pamk
