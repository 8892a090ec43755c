// The layer-and-step side's streams over memory on gfx950: the activations'
// gradient with the bias's, the norm of all gradients, and the AdamW step over
// many tensors.  All are bound by reading and writing each value once; a large
// copy runs at 4.9 TB/s on these cards, reading and writing streams at up to 6.2.
// Measured (passes in a row): the gradient of 16384 x 4096 float32 values 129 us (6.2
// TB/s), bfloat16 71 us (5.7), 8192 x 2048 float32 45 us (4.5, the sums' launch 4 of
// it; on the same buffers again, which the cache holds in part, 36); the norm of 188 M
// float32 values 113 us (6.7 TB/s); the step over them 857 us (6.1 TB/s), with 8-bit
// states 535 us (5.6); the norm and the step of a decoder's 25.7 M parameters,
// gradients and copies bfloat16, 131 us (5.9).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pam_epilogue.h"
#include "pam_training_internal.h"

namespace pamk {
namespace {

// V neighbouring elements at any address.  NT: with the non-temporal hint.
template <int V, typename T> using Wide = T __attribute__((ext_vector_type(V), aligned(sizeof(T))));
template <int V, bool NT, typename T> __device__ __forceinline__ Wide<V, T> load_raw(const T *p) {
    const Wide<V, T> *at = reinterpret_cast<const Wide<V, T> *>(p);
    return NT ? __builtin_nontemporal_load(at) : *at;
}
// Elements one by one, the `have` that exist.
template <int V, typename T> __device__ __forceinline__ Wide<V, T> load_some(const T *p, int have) {
    Wide<V, T> v;
#pragma unroll
    for (int i = 0; i < V; ++i)
        v[i] = i < have ? p[i] : T(0);
    return v;
}
template <int V, typename T> __device__ __forceinline__ void widened(const Wide<V, T> &v, float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(T) == 2)
            x[i] = bf16_value(v[i]);
        else
            x[i] = v[i];
    }
}
template <int V, typename T> __device__ __forceinline__ Wide<V, T> rounded(const float (&x)[V]) {
    Wide<V, T> v;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(T) == 2)
            v[i] = bf16_bits(x[i]);
        else
            v[i] = x[i];
    }
    return v;
}
template <int V, bool NT, typename T> __device__ __forceinline__ void store_wide(T *p, const float (&x)[V]) {
    Wide<V, T> *at = reinterpret_cast<Wide<V, T> *>(p);
    if constexpr (NT)
        __builtin_nontemporal_store(rounded<V, T>(x), at);
    else
        *at = rounded<V, T>(x);
}
template <int V, typename T> __device__ __forceinline__ void store_some(T *p, int have, const float (&x)[V]) {
    const Wide<V, T> v = rounded<V, T>(x);
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < have)
            p[i] = v[i];
}

// ---------------------------------------------------------------------------
// The activations' gradient
// ---------------------------------------------------------------------------

// dz = dy f'(z) and the sums of its columns, each value read once and written once:
// the sums ride along.  A thread keeps the sums of its V columns over the rows it
// takes; the workgroup's rows are added in a tree, in LDS, and the bands' sums by
// sum_bands_kernel: an order fixed by the sizes.
template <typename T, typename Z, bool NT> __global__ void __launch_bounds__(kGradThreads) activation_grad_kernel(GradParams p) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float red[kGradThreads * V];
    const int lanes = p.lanes, at_once = kGradThreads / lanes;
    const int tx = threadIdx.x % lanes, ty = threadIdx.x / lanes;
    const int groups = (p.n + lanes * V - 1) / (lanes * V);
    const int band = blockIdx.x / groups;
    const int col = (blockIdx.x - band * groups) * lanes * V + tx * V;
    const int have = min(p.n - col, V);
    // A row's last columns, fewer than V: the V that end there, some of them the
    // neighbour's too, whose dz is then written twice with the same value.  (Single
    // elements made their whole wave wait: 197 x 771 in bfloat16 14.7 us, now 11.8.)
    // Not where dz lies on an input, which the neighbour may have overwritten.
    const int start = p.apart && p.n >= V ? min(col, p.n - V) : col;
    const int64_t end = min((int64_t)(band + 1) * p.band, p.m);
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        sum[i] = 0.0f;
    const T *dy = static_cast<const T *>(p.dy) + start;
    const Z *z = static_cast<const Z *>(p.z) + start;
    T *dz = static_cast<T *>(p.dz) + start;
    if (have > 0)
        with_activation(p.activation, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            auto slopes = [&](float (&d)[V], const Wide<V, Z> &zs) {
                if constexpr (ACT != PAM_ACT_NONE) {
                    float x[V];
                    widened<V, Z>(zs, x);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        if constexpr (ACT == PAM_ACT_RELU)
                            d[i] = x[i] <= 0.0f ? 0.0f : d[i];
                        else
                            d[i] *= activation_slope<ACT>(x[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < V; ++i)
                    sum[i] += d[i];
            };
            int64_t r = (int64_t)band * p.band + ty;
            if (have == V || start != col) {
                // U rows' loads, then their work.
                auto rows = [&](auto count) {
                    constexpr int U = decltype(count)::value;
                    Wide<V, T> d[U];
                    Wide<V, Z> x[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        d[u] = load_raw<V, NT>(dy + (r + u * at_once) * p.lddy);
                        if constexpr (ACT != PAM_ACT_NONE)
                            x[u] = load_raw<V, NT>(z + (r + u * at_once) * p.ldz);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        float g[V];
                        widened<V, T>(d[u], g);
                        slopes(g, x[u]);
                        if (ACT != PAM_ACT_NONE && p.dz != nullptr)
                            store_wide<V, false>(dz + (r + u * at_once) * p.lddz, g);
                    }
                };
                // Several rows at once where the few there are make up a thread's time
                // (64 x 512 6.5 -> 5.2 us); where memory does, one by one (8192 x 2048
                // 45.5 us, by two 45.8, by four 53.5; on the same buffers again 36.2, 37.1
                // and 40.2).
                constexpr int kRows = 4;
                if (p.bands == 1)
                    for (; r + (kRows - 1) * at_once < end; r += kRows * at_once)
                        rows(std::integral_constant<int, kRows>{});
                for (; r < end; r += at_once)
                    rows(std::integral_constant<int, 1>{});
            } else {
                for (; r < end; r += at_once) {
                    Wide<V, Z> x{};
                    if constexpr (ACT != PAM_ACT_NONE)
                        x = load_some<V>(z + r * p.ldz, have);
                    float g[V];
                    widened<V, T>(load_some<V>(dy + r * p.lddy, have), g);
                    slopes(g, x);
                    if (ACT != PAM_ACT_NONE && p.dz != nullptr)
                        store_some<V>(dz + r * p.lddz, have, g);
                }
            }
        });
    if (p.db == nullptr)
        return;
#pragma unroll
    for (int i = 0; i < V; ++i)
        red[threadIdx.x * V + i] = sum[i];
    for (int half = at_once / 2; half > 0; half /= 2) {
        __syncthreads();
        if (ty < half) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                red[threadIdx.x * V + i] += red[(threadIdx.x + half * lanes) * V + i];
        }
    }
    if (ty != 0)
        return;
    float *out = p.bands == 1 ? p.db : p.partial + (int64_t)band * p.n;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (start + i >= col && start + i < p.n)
            out[start + i] = red[threadIdx.x * V + i];
}

// db = the sum of the bands' sums: 64 columns a workgroup, a quarter of the bands
// a wave.
__global__ void __launch_bounds__(256) sum_bands_kernel(const float *__restrict__ partial, float *__restrict__ db,
                                                        int bands, int n) {
    __shared__ float red[256];
    const int col = blockIdx.x * 64 + (threadIdx.x & 63), part = threadIdx.x >> 6;
    float sum = 0.0f;
    if (col < n) {
#pragma unroll 8
        for (int b = part; b < bands; b += 4)
            sum += partial[(int64_t)b * n + col];
    }
    red[threadIdx.x] = sum;
    __syncthreads();
    if (part == 0 && col < n)
        db[col] = (sum + red[threadIdx.x + 64]) + (red[threadIdx.x + 128] + red[threadIdx.x + 192]);
}

// ---------------------------------------------------------------------------
// Many tensors at once
// ---------------------------------------------------------------------------

// The tensor that workgroup b works on: the last whose first workgroup is not
// after it.  Each lane compares one.
__device__ __forceinline__ int tensor_of(const uint32_t *first, int count, uint32_t b) {
    const int lane = threadIdx.x & 63;
    const bool before = lane < count && first[min(lane, count - 1)] <= b;
    return __builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) - 1;
}

template <typename T, bool NT> __global__ void __launch_bounds__(kStepThreads) grad_squares_kernel(NormParams p) {
    constexpr int V = 16 / sizeof(T);
    __shared__ double red[kStepThreads / 64];
    const int j = tensor_of(p.first, p.count, blockIdx.x);
    const int64_t begin = (int64_t)(blockIdx.x - p.first[j]) * p.chunk;
    const int64_t end = min(begin + p.chunk, p.n[j]);
    const T *g = static_cast<const T *>(p.g[j]);
    // In float64: a sum of 2^26 squares keeps its last bit, none overflows.
    double sum = 0.0;
    auto add = [&](const Wide<V, T> &v) {
        float x[V];
        widened<V, T>(v, x);
#pragma unroll
        for (int e = 0; e < V; ++e)
            sum = __builtin_fma((double)x[e], (double)x[e], sum);
    };
    int64_t i = begin + threadIdx.x * V;
#pragma unroll 4
    for (; i + V <= end; i += kStepThreads * V)
        add(load_raw<V, NT>(g + i));
    if (i < end)
        add(load_some<V>(g + i, (int)(end - i)));
    for (int d = 32; d > 0; d /= 2)
        sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        p.partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ void __launch_bounds__(1024) grad_norm_kernel(const double *__restrict__ partial, int64_t count, float *norm) {
    __shared__ double red[16];
    double sum = 0.0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < count; i += 1024)
        sum += partial[i];
    for (int d = 32; d > 0; d /= 2)
        sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w)
            sum += red[w];
        *norm = (float)sqrt(sum);
    }
}

// What the whole step has in common.
struct Rates {
    float step_size, sq_factor, clip;
    uint32_t key;     // of the tensor's random bits
};

// The mixer of two multiplications that C. Wellons found by search and published
// ("Prospecting for Hash Functions", 2018).
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

__device__ __forceinline__ Rates rates_of(const StepParams &p, int tensor) {
    Rates r{p.step_size, p.sq_factor, 1.0f, 0u};
    int64_t step = p.step;
    if (p.step_device != nullptr) {
        step = *p.step_device;
        // The exponents in float64, the rest in float32, for every wave does this: within a
        // dozen units of 2^-24 of the host's rates.
        r.step_size = p.step_size / -expm1f((float)((double)step * p.log_beta1));
        r.sq_factor = 1.0f / sqrtf(-expm1f((float)((double)step * p.log_beta2)));
    }
    if (p.norm != nullptr) {
        const float c = p.max_norm / (*p.norm + 1e-6f);
        r.clip = c >= 1.0f ? 1.0f : c;   // NaN stays
    }
    r.key = mix(mix(p.seed + (uint32_t)step * 0x9E3779B9u) + (uint32_t)(p.tensor0 + tensor));
    return r;
}

__device__ __forceinline__ float moved(const StepParams &p, const Rates &r, float x, float avg, float sq) {
    // Within 2 units of 2^-23 of the step; the step is small beside p.
    const float by = __builtin_fmaf(__builtin_amdgcn_sqrtf(sq), r.sq_factor, p.eps);
    return __builtin_fmaf(-r.step_size, avg * __builtin_amdgcn_rcpf(by), x * p.keep);
}

template <typename G, bool NT> __global__ void __launch_bounds__(kStepThreads) adamw_kernel(StepParams p) {
    const int j = tensor_of(p.first, p.count, blockIdx.x);
    const pam_step_tensor_t &t = p.tensor[j];
    const Rates rates = rates_of(p, j);
    const int64_t begin = (int64_t)(blockIdx.x - p.first[j]) * p.chunk;
    const int64_t end = min(begin + p.chunk, t.n);
    const G *g = static_cast<const G *>(t.g);
    float *avg = static_cast<float *>(t.avg), *sq = static_cast<float *>(t.sq);
    auto step = [&](float (&x)[4], float (&d)[4], float (&m)[4], float (&v)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            d[e] *= rates.clip;
            m[e] = __builtin_fmaf(m[e], p.beta1, d[e] * p.rest1);
            v[e] = __builtin_fmaf(v[e], p.beta2, d[e] * p.rest2 * d[e]);
            x[e] = moved(p, rates, x[e], m[e], v[e]);
        }
    };
    // A vector a thread: the chunk is kStepThreads * 4 values.
    const int64_t i = begin + threadIdx.x * 4;
    float x[4], d[4], m[4], v[4];
    if (i + 4 <= end) {
        const auto gw = load_raw<4, NT>(g + i);
        const auto xw = load_raw<4, NT>(t.p + i), mw = load_raw<4, NT>(avg + i), vw = load_raw<4, NT>(sq + i);
        widened<4, G>(gw, d);
        widened<4, float>(xw, x);
        widened<4, float>(mw, m);
        widened<4, float>(vw, v);
        step(x, d, m, v);
        store_wide<4, NT>(avg + i, m);
        store_wide<4, NT>(sq + i, v);
        store_wide<4, NT>(t.p + i, x);
        if (t.copy != nullptr)
            store_wide<4, NT>(t.copy + i, x);
    } else if (i < end) {   // a tensor's last values
        const int have = (int)(end - i);
        widened<4, G>(load_some<4>(g + i, have), d);
        widened<4, float>(load_some<4>(t.p + i, have), x);
        widened<4, float>(load_some<4>(avg + i, have), m);
        widened<4, float>(load_some<4>(sq + i, have), v);
        step(x, d, m, v);
        store_some<4>(avg + i, have, m);
        store_some<4>(sq + i, have, v);
        store_some<4>(t.p + i, have, x);
        if (t.copy != nullptr)
            store_some<4>(t.copy + i, have, x);
    }
}

// 8-bit states --------------------------------------------------------------

constexpr uint32_t kAvgLow = 889, kAvgMost = 127, kSqLow = 761, kSqMost = 255;

__device__ __forceinline__ float held(uint32_t code, uint32_t low, float scale) {
    return (code != 0u ? __uint_as_float((code + low) << 20) : 0.0f) * scale;
}

// Division by a block's scale, correctly rounded.  With s = scale / 2^e in [1, 4),
// x' = x / 2^e and r the rounded 1 / s, x' r is within two units in the last place
// of x' / s, and one correction by the residual brings it within one; from there
// q + (x' - q s) r, the residual then exact in an fma, is x' / s rounded (Markstein).
// Five operations a value in place of a division's twelve or so: the step of 188 M
// parameters 573 -> 547 us, the maxima by cross-lane moves included.  What 2^-e
// flushes is below 2^-126 of the scale, and coded as 0 anyway.
struct Divisor {
    float shift, s, r;
    __device__ __forceinline__ explicit Divisor(float scale) {
        // The shift's own field is 254 less the scale's, at least 1; without a scale
        // there is nothing to divide, and by inf every finite value gives 0.
        const int e = (int)(__float_as_uint(scale) >> 23);   // no sign
        shift = e == 255 ? 0.0f : e == 0 ? 1.0f : __uint_as_float((uint32_t)max(254 - e, 1) << 23);
        s = e == 255 || e == 0 ? 1.0f : scale * shift;
        r = 1.0f / s;
    }
    __device__ __forceinline__ float operator()(float x) const {
        const float a = x * shift, q = a * r, q1 = __builtin_fmaf(__builtin_fmaf(-q, s, a), r, q);
        return __builtin_fmaf(__builtin_fmaf(-q1, s, a), r, q1);
    }
};

// The code of a part of its block's scale (NaN: the largest).
__device__ __forceinline__ uint32_t coded(float part, uint32_t random, uint32_t low, uint32_t most) {
    const uint32_t c = (__float_as_uint(part) + random) >> 20;
    return c <= low ? 0u : min(c - low, most);
}

// The largest of the wave's magnitudes, by their encodings: NaN above all.
__device__ __forceinline__ float largest(const float (&x)[4]) {
    int m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m[i] = __float_as_int(__builtin_fabsf(x[i]));
    int u = max(max(m[0], m[1]), max(m[2], m[3]));
    // Along the rows of 16 lanes, then from row to row: lane 63 has all.
    u = max(u, __builtin_amdgcn_update_dpp(0, u, 0x111, 0xF, 0xF, true));
    u = max(u, __builtin_amdgcn_update_dpp(0, u, 0x112, 0xF, 0xF, true));
    u = max(u, __builtin_amdgcn_update_dpp(0, u, 0x114, 0xF, 0xF, true));
    u = max(u, __builtin_amdgcn_update_dpp(0, u, 0x118, 0xF, 0xF, true));
    u = max(u, __builtin_amdgcn_update_dpp(0, u, 0x142, 0xA, 0xF, true));
    u = max(u, __builtin_amdgcn_update_dpp(0, u, 0x143, 0xC, 0xF, true));
    return __int_as_float(__builtin_amdgcn_readlane(u, 63));
}

// Four codes from c, at any address; `have` of them exist.
template <bool NT> __device__ __forceinline__ uint32_t load_codes(const uint8_t *c, int have) {
    typedef uint32_t word __attribute__((aligned(1)));
    if (have >= 4)
        return NT ? __builtin_nontemporal_load(reinterpret_cast<const word *>(c)) : *reinterpret_cast<const word *>(c);
    uint32_t w = 0u;
    for (int i = 0; i < have; ++i)
        w |= (uint32_t)c[i] << (8 * i);
    return w;
}
template <bool NT> __device__ __forceinline__ void store_codes(uint8_t *c, int have, uint32_t w) {
    typedef uint32_t word __attribute__((aligned(1)));
    if (have >= 4) {
        if constexpr (NT)
            __builtin_nontemporal_store(w, reinterpret_cast<word *>(c));
        else
            *reinterpret_cast<word *>(c) = w;
    } else {
        for (int i = 0; i < have; ++i)
            c[i] = (uint8_t)(w >> (8 * i));
    }
}

// A wave holds a block of 256 values, four a lane: its scales are maxima over
// the wave, so that the states are read and written once, 16 bytes a parameter
// beside 28.  About 90 vector operations a value stay just below the memory's time.
template <typename G, bool NT> __global__ void __launch_bounds__(kStepThreads) adamw8_kernel(StepParams p) {
    const int j = tensor_of(p.first, p.count, blockIdx.x);
    const pam_step_tensor_t &t = p.tensor[j];
    const Rates rates = rates_of(p, j);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t begin = (int64_t)(blockIdx.x - p.first[j]) * p.chunk;
    const int64_t end = min(begin + p.chunk, t.n);
    const G *g = static_cast<const G *>(t.g);
    uint8_t *avg = static_cast<uint8_t *>(t.avg), *sq = static_cast<uint8_t *>(t.sq);
    auto one = [&](auto full, int64_t b) {
        constexpr bool kFull = decltype(full)::value;   // all 256 values exist
        const int64_t i = b + lane * 4, block = b / PAM_STATE_BLOCK;
        const int have = kFull ? 4 : (int)max(min(end - i, (int64_t)4), (int64_t)0);
        float x[4], d[4], m[4], v[4], size[4];
        if constexpr (kFull) {
            widened<4, G>(load_raw<4, NT>(g + i), d);
            widened<4, float>(load_raw<4, NT>(t.p + i), x);
        } else {
            widened<4, G>(load_some<4>(g + i, have), d);
            widened<4, float>(load_some<4>(t.p + i, have), x);
        }
        const uint32_t mc = load_codes<NT>(avg + i, have), vc = load_codes<NT>(sq + i, have);
        const float ms = t.avg_scale[block], vs = t.sq_scale[block];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // Each operation rounded by itself, as the codes' definition has it.
#pragma clang fp contract(off)
            const uint32_t c = (mc >> (8 * e)) & 0xFFu;
            const float old = held(c & kAvgMost, kAvgLow, ms);
            d[e] = d[e] * rates.clip;
            const float m0 = (c > kAvgMost ? -old : old) * p.beta1, m1 = d[e] * p.rest1;
            const float v0 = held((vc >> (8 * e)) & 0xFFu, kSqLow, vs) * p.beta2, v1 = d[e] * p.rest2 * d[e];
            m[e] = m0 + m1;
            v[e] = v0 + v1;
            if (e >= have)
                m[e] = v[e] = 0.0f;
            size[e] = __builtin_fabsf(m[e]);
        }
        const float ms1 = largest(size), vs1 = largest(v);
        const Divisor by_m(ms1), by_v(vs1);
        uint32_t mw = 0u, vw = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t h = mix((uint32_t)(i + e) + rates.key);
            const uint32_t cm = coded(by_m(size[e]), ((h & 0xFFFFu) << 4) + 8u, kAvgLow, kAvgMost);
            const uint32_t cv = coded(by_v(v[e]), ((h >> 16) << 4) + 8u, kSqLow, kSqMost);
            mw |= (cm | (cm != 0u && m[e] < 0.0f ? 128u : 0u)) << (8 * e);
            vw |= (v[e] != 0.0f ? max(cv, 1u) : 0u) << (8 * e);
            x[e] = moved(p, rates, x[e], m[e], v[e]);
        }
        store_codes<NT>(avg + i, have, mw);
        store_codes<NT>(sq + i, have, vw);
        if constexpr (kFull) {
            store_wide<4, NT>(t.p + i, x);
            if (t.copy != nullptr)
                store_wide<4, NT>(t.copy + i, x);
        } else {
            store_some<4>(t.p + i, have, x);
            if (t.copy != nullptr)
                store_some<4>(t.copy + i, have, x);
        }
        if (lane == 0) {
            t.avg_scale[block] = ms1;
            t.sq_scale[block] = vs1;
        }
    };
    int64_t b = begin + wave * PAM_STATE_BLOCK;
#pragma unroll 1
    for (; b + PAM_STATE_BLOCK <= end; b += kStepThreads / 64 * PAM_STATE_BLOCK)
        one(std::true_type{}, b);
    if (b < end)
        one(std::false_type{}, b);
}

}  // namespace

hipError_t launch_activation_grad(bool bf16, bool z_bf16, const GradParams &p, hipStream_t stream) {
    const int wide = p.lanes * grad_values(bf16);
    const int64_t groups = ((int64_t)p.n + wide - 1) / wide * p.bands;
    if (groups <= 0 || groups > kMostStepGroups)
        return hipErrorInvalidValue;
    const dim3 grid((unsigned)groups), block(kGradThreads);
    auto launch = [&](auto t, auto z, auto nt) {
        hipLaunchKernelGGL((activation_grad_kernel<decltype(t), decltype(z), decltype(nt)::value>), grid, block, 0, stream, p);
    };
    auto choose = [&](auto nt) {
        if (bf16 && z_bf16)
            launch(uint16_t{}, uint16_t{}, nt);
        else if (bf16)
            launch(uint16_t{}, float{}, nt);
        else if (z_bf16)
            launch(float{}, uint16_t{}, nt);
        else
            launch(float{}, float{}, nt);
    };
    if (p.streaming)
        choose(std::true_type{});
    else
        choose(std::false_type{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.db == nullptr || p.bands == 1)
        return e;
    hipLaunchKernelGGL(sum_bands_kernel, dim3((unsigned)((p.n + 63) / 64)), dim3(256), 0, stream, p.partial, p.db,
                       p.bands, p.n);
    return hipGetLastError();
}

hipError_t launch_grad_squares(uint32_t groups, const NormParams &p, hipStream_t stream) {
    const dim3 grid(groups), block(kStepThreads);
    if (p.grad_bf16 && p.streaming)
        hipLaunchKernelGGL((grad_squares_kernel<uint16_t, true>), grid, block, 0, stream, p);
    else if (p.grad_bf16)
        hipLaunchKernelGGL((grad_squares_kernel<uint16_t, false>), grid, block, 0, stream, p);
    else if (p.streaming)
        hipLaunchKernelGGL((grad_squares_kernel<float, true>), grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL((grad_squares_kernel<float, false>), grid, block, 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const double *partial, int64_t count, float *norm, hipStream_t stream) {
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, stream, partial, count, norm);
    return hipGetLastError();
}

hipError_t launch_adamw(int state_bits, uint32_t groups, const StepParams &p, hipStream_t stream) {
    const dim3 grid(groups), block(kStepThreads);
    auto launch = [&](auto g, auto nt) {
        using G = decltype(g);
        constexpr bool NT = decltype(nt)::value;
        if (state_bits == 32)
            hipLaunchKernelGGL((adamw_kernel<G, NT>), grid, block, 0, stream, p);
        else
            hipLaunchKernelGGL((adamw8_kernel<G, NT>), grid, block, 0, stream, p);
    };
    if (p.grad_bf16 && p.streaming)
        launch(uint16_t{}, std::true_type{});
    else if (p.grad_bf16)
        launch(uint16_t{}, std::false_type{});
    else if (p.streaming)
        launch(float{}, std::true_type{});
    else
        launch(float{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace pamk
