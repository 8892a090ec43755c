// Device code of the activations and of what a linear layer adds to its product
// (pam_linear of pam_training.h): z = product + bias, y = activation(z) +
// residual.  Shared by the product kernels, the reduction of split products and
// the activations' gradient.  Included by the HIP sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pam_internal.h"
#include "pam_training.h"

namespace pamk {

typedef float f32x4a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint16_t u16x8a2 __attribute__((ext_vector_type(8), aligned(2)));

constexpr float kLog2E = 1.442695041f;
constexpr float kTanh0 = 0.7978845608f;               // sqrt(2 / pi)
constexpr float kTanh1 = 0.7978845608f * 0.044715f;

// Rounded to nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ float bf16_value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// Far below zero the logistic function and the normal tail leave the float32 range
// before their products with z do (silu(-90) is -7e-38).  LIFT: they are computed
// times 2^24 there, and what they are in is to be multiplied by `down`, 1 or 2^-24.
// The activations take it, at up to 0.6% of a layer's time.  Their slopes do not:
// it made the gradient of 16384 x 4096 in bfloat16 2 to 5% slower (70.1 -> 71.6 us with
// SILU, 70.8 -> 74.8 with GELU_TANH), for slopes below 2^-118.
constexpr float kLift = 24.0f, kDown = 0x1p-24f;

// 1 / (1 + exp(-x)), over down: 0 and 1 in the limits.  Below -80 it is exp(x).
template <bool LIFT> __device__ __forceinline__ float logistic(float x, float &down) {
    const bool far = LIFT && x < -80.0f;
    const float e = __builtin_amdgcn_exp2f(far ? __builtin_fmaf(kLog2E, x, kLift) : -kLog2E * x);
    down = far ? kDown : 1.0f;
    return far ? e : __builtin_amdgcn_rcpf(1.0f + e);
}
__device__ __forceinline__ float logistic(float x) {
    float down;
    return logistic<false>(x, down);
}

// P(N <= z) of a standard normal N, and exp(-z^2 / 2), both over down.  The tail
// Q(x) = P(N > x) for x = |z| is exp(-x^2 / 2) t R(t), t = 1 / (1 + 0.3 x), where R is
// smooth on [0, 1] (the tail falls as exp(-x^2 / 2) / x): R's polynomial was fitted to
// erfc for the least relative error on 0 <= x <= 14 (Q(14) is below the float32
// range), 3.5e-9.  In float32 the result is within 3 units of 2^-24, and the tails
// keep their relative accuracy (1.5e-6 at -5), which 1 + erf(z) would not.
template <bool LIFT> __device__ __forceinline__ float normal_below(float z, float &gauss, float &down) {
    const float x = __builtin_fabsf(z);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, x, 1.0f));
    float r = -0.02061283588f;
    r = __builtin_fmaf(r, t, 0.11237581f);
    r = __builtin_fmaf(r, t, -0.2280675918f);
    r = __builtin_fmaf(r, t, 0.1915817857f);
    r = __builtin_fmaf(r, t, -0.07924741507f);
    r = __builtin_fmaf(r, t, 0.09605786949f);
    r = __builtin_fmaf(r, t, 0.07842557132f);
    r = __builtin_fmaf(r, t, 0.1102273241f);
    r = __builtin_fmaf(r, t, 0.1195728406f);
    r = __builtin_fmaf(r, t, 0.1196866333f);
    const bool far = LIFT && z < -12.0f;
    gauss = __builtin_amdgcn_exp2f(far ? __builtin_fmaf(z * z, -0.5f * kLog2E, kLift) : z * z * (-0.5f * kLog2E));
    down = far ? kDown : 1.0f;
    const float q = r * t * gauss;
    return z < 0.0f ? q : 1.0f - q;
}
__device__ __forceinline__ float normal_below(float z, float &gauss) {
    float down;
    return normal_below<false>(z, gauss, down);
}

template <int ACT> __device__ __forceinline__ float activation(float z) {
    if constexpr (ACT == PAM_ACT_RELU) {
        return z <= 0.0f ? 0.0f : z;   // NaN stays
    } else if constexpr (ACT == PAM_ACT_NONE) {
        return z;
    } else {
        float gauss, down, p;
        if constexpr (ACT == PAM_ACT_GELU)
            p = normal_below<true>(z, gauss, down);
        else if constexpr (ACT == PAM_ACT_GELU_TANH)
            p = logistic<true>(2.0f * z * __builtin_fmaf(kTanh1 * z, z, kTanh0), down);
        else
            p = logistic<true>(z, down);
        return z * p * down;
    }
}

// f'(z).  The smooth activations' slopes are 0 and 1 in float32 from |z| = 16
// (GELU, GELU_TANH) and 120 (SILU) on: taken there, no infinity meets a zero.
template <int ACT> __device__ __forceinline__ float activation_slope(float z) {
    if constexpr (ACT == PAM_ACT_RELU) {
        return z <= 0.0f ? 0.0f : 1.0f;
    } else if constexpr (ACT == PAM_ACT_NONE) {
        return 1.0f;
    } else {
        constexpr float kFar = ACT == PAM_ACT_SILU ? 120.0f : 16.0f;
        z = z > kFar ? kFar : z;      // not by min and max: NaN stays
        z = z < -kFar ? -kFar : z;
        if constexpr (ACT == PAM_ACT_GELU) {
            float gauss;
            const float p = normal_below(z, gauss);
            return __builtin_fmaf(z * 0.3989422804f, gauss, p);   // 1 / sqrt(2 pi)
        } else if constexpr (ACT == PAM_ACT_GELU_TANH) {
            const float s = logistic(2.0f * z * __builtin_fmaf(kTanh1 * z, z, kTanh0));
            return __builtin_fmaf(2.0f * z * __builtin_fmaf(3.0f * kTanh1 * z, z, kTanh0), s * (1.0f - s), s);
        } else {
            const float s = logistic(z);
            return __builtin_fmaf(z * s, 1.0f - s, s);
        }
    }
}

// f(integral_constant of the activation).
template <typename F> __device__ __forceinline__ void with_activation(int act, F f) {
    switch (act) {
    case PAM_ACT_RELU: f(std::integral_constant<int, PAM_ACT_RELU>{}); break;
    case PAM_ACT_GELU: f(std::integral_constant<int, PAM_ACT_GELU>{}); break;
    case PAM_ACT_GELU_TANH: f(std::integral_constant<int, PAM_ACT_GELU_TANH>{}); break;
    case PAM_ACT_SILU: f(std::integral_constant<int, PAM_ACT_SILU>{}); break;
    default: f(std::integral_constant<int, PAM_ACT_NONE>{}); break;
    }
}

// Element i of an array of float32 or bfloat16.
__device__ __forceinline__ float load_out(const void *base, int64_t i, bool bf16) {
    return bf16 ? bf16_value(static_cast<const uint16_t *>(base)[i]) : static_cast<const float *>(base)[i];
}
__device__ __forceinline__ void store_out(void *base, int64_t i, bool bf16, float x) {
    if (bf16)
        static_cast<uint16_t *>(base)[i] = bf16_bits(x);
    else
        static_cast<float *>(base)[i] = x;
}

// Four elements from i, at any address; `have` of them exist.
__device__ __forceinline__ void load_out4(const void *base, int64_t i, bool bf16, int have, float (&x)[4]) {
    if (have >= 4) {
        if (bf16) {
            const u16x4a2 v = *reinterpret_cast<const u16x4a2 *>(static_cast<const uint16_t *>(base) + i);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = bf16_value(v[j]);
        } else {
            const f32x4a4 v = *reinterpret_cast<const f32x4a4 *>(static_cast<const float *>(base) + i);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = v[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            x[j] = j < have ? load_out(base, i + j, bf16) : 0.0f;
    }
}
// Written once: with the non-temporal hint, as the products' outputs are.
__device__ __forceinline__ void store_out4(void *base, int64_t i, bool bf16, int have, const float (&x)[4]) {
    if (have >= 4) {
        if (bf16) {
            const u16x4a2 v = {bf16_bits(x[0]), bf16_bits(x[1]), bf16_bits(x[2]), bf16_bits(x[3])};
            __builtin_nontemporal_store(v, reinterpret_cast<u16x4a2 *>(static_cast<uint16_t *>(base) + i));
        } else {
            const f32x4a4 v = {x[0], x[1], x[2], x[3]};
            __builtin_nontemporal_store(v, reinterpret_cast<f32x4a4 *>(static_cast<float *>(base) + i));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < have)
                store_out(base, i + j, bf16, x[j]);
    }
}

__device__ __forceinline__ void load_bias4(const Epilogue &e, int col, int have, float (&bias)[4]) {
    if (e.bias != nullptr) {
        load_out4(e.bias, col, false, have, bias);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            bias[j] = 0.0f;
    }
}

__device__ __forceinline__ void load_residual4(const Epilogue &e, int64_t row, int col, int have, float (&res)[4]) {
    if (e.residual != nullptr) {
        load_out4(e.residual, row * e.ldr + col, e.out_bf16 != 0, have, res);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            res[j] = 0.0f;
    }
}

// The outputs of four neighbouring sums v of a row, from column col on; `have`
// columns are left.
template <int ACT>
__device__ __forceinline__ void finish4(const Epilogue &e, int64_t row, int col, int have, const float (&v)[4],
                                        const float (&bias)[4], const float (&res)[4]) {
    const bool bf16 = e.out_bf16 != 0;
    float z[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        z[j] = e.bias != nullptr ? v[j] + bias[j] : v[j];
        y[j] = activation<ACT>(z[j]);
        y[j] = e.residual != nullptr ? y[j] + res[j] : y[j];
    }
    if (e.z != nullptr)
        store_out4(e.z, row * e.ldz + col, bf16, have, z);
    store_out4(e.y, row * e.ldy + col, bf16, have, y);
}
__device__ __forceinline__ void finish4(const Epilogue &e, int64_t row, int col, int have, const float (&v)[4]) {
    float bias[4], res[4];
    load_bias4(e, col, have, bias);
    load_residual4(e, row, col, have, res);
    with_activation(e.activation, [&](auto act) { finish4<decltype(act)::value>(e, row, col, have, v, bias, res); });
}

// The outputs of one sum.
__device__ __forceinline__ void finish1(const Epilogue &e, int64_t row, int col, float v) {
    const bool bf16 = e.out_bf16 != 0;
    const float z = e.bias != nullptr ? v + e.bias[col] : v;
    float y = z;
    with_activation(e.activation, [&](auto act) { y = activation<decltype(act)::value>(z); });
    if (e.z != nullptr)
        store_out(e.z, row * e.ldz + col, bf16, z);
    if (e.residual != nullptr)
        y += load_out(e.residual, row * e.ldr + col, bf16);
    store_out(e.y, row * e.ldy + col, bf16, y);
}

}  // namespace pamk
