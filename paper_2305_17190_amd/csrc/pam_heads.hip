// Norms of queries and keys with the position rotation, their gradient, and
// the append to a paged key/value cache, for gfx950.  All of it is ordinary
// float32 arithmetic (Kosson & Jaggi, Sec. 3.2, replace the products of the
// linear layers and of the attention only).
//
// A head is a row of d values.  It is cut into units of 2V values, V
// neighbours from each half of V rotated pairs (or 2V values that are not
// rotated), so that a lane holds both members of its pairs and the rotation
// needs no exchange; the row's units lie on neighbouring lanes of one wave and
// only the sum of squares crosses lanes.  V is the widest of 16 bytes' worth
// of the input type, 4, 2, 1 that divides the pairs and the rest.
//
// Bound by memory: every value is read once and written once, beside a table
// row per token that its heads share through the caches.  Measured: queries and
// keys of 8192 tokens, 8 + 8 heads of 64 in float32 (68 MB) 12.3 us, 5.5 TB/s; the
// gradient (102 MB) 23.3 us, of which 4 add up the weights' gradients; that of 16384
// tokens, 32 + 8 heads of 128 in bfloat16 (505 MB) 103 us, 4.9 TB/s; their append to
// a bfloat16 cache from float32 (740 MB) 137 us, 5.4 TB/s, from bfloat16 (403 MB) 83 us,
// 4.8 TB/s; their norms and rotation alone in bfloat16 (336 MB) 68 us, 5.0 TB/s.  A 1 GiB copy runs at 5.1-5.2
// TB/s.  Eight tokens: 4 us on the GPU.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pam_attention_internal.h"

namespace pamk {
namespace {

constexpr int kThreads = 256;

// V values of one type as registers; memory at any alignment of the element.
template <typename T, int V> struct Vec;
template <int V> struct Vec<float, V> {
    typedef float type __attribute__((ext_vector_type(V), aligned(4)));
};
template <int V> struct Vec<uint16_t, V> {
    typedef uint16_t type __attribute__((ext_vector_type(V), aligned(2)));
};

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// Nearest even; NaN stays NaN.
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

template <typename T, int V> __device__ __forceinline__ void load(const void *base, uint64_t at, float (&x)[V]) {
    if constexpr (V == 1) {
        x[0] = widen(static_cast<const T *>(base)[at]);
    } else {
        const auto v = *reinterpret_cast<const typename Vec<T, V>::type *>(static_cast<const T *>(base) + at);
#pragma unroll
        for (int i = 0; i < V; ++i)
            x[i] = widen(v[i]);
    }
}

// V values as they lie in memory, to be widened when they are used.
template <typename T, int V> struct Raw {
    typename Vec<T, V>::type v;
    __device__ __forceinline__ void load(const void *base, uint64_t at) {
        v = *reinterpret_cast<const typename Vec<T, V>::type *>(static_cast<const T *>(base) + at);
    }
    __device__ __forceinline__ void get(float (&x)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i)
            x[i] = widen(v[i]);
    }
};
template <typename T> struct Raw<T, 1> {
    T v;
    __device__ __forceinline__ void load(const void *base, uint64_t at) { v = static_cast<const T *>(base)[at]; }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = widen(v); }
};

template <int V> __device__ __forceinline__ void store(void *base, uint64_t at, const float (&x)[V], bool bf16) {
    if (bf16) {
        if constexpr (V == 1) {
            static_cast<uint16_t *>(base)[at] = to_bf16(x[0]);
        } else {
            typename Vec<uint16_t, V>::type v;
#pragma unroll
            for (int i = 0; i < V; ++i)
                v[i] = to_bf16(x[i]);
            *reinterpret_cast<typename Vec<uint16_t, V>::type *>(static_cast<uint16_t *>(base) + at) = v;
        }
    } else {
        // 16 bytes a store: V == 8 are two.
        constexpr int W = V < 4 ? V : 4;
#pragma unroll
        for (int j = 0; j < V; j += W) {
            if constexpr (V == 1) {
                static_cast<float *>(base)[at] = x[0];
            } else {
                typename Vec<float, W>::type v;
#pragma unroll
                for (int i = 0; i < W; ++i)
                    v[i] = x[j + i];
                *reinterpret_cast<typename Vec<float, W>::type *>(static_cast<float *>(base) + at + j) = v;
            }
        }
    }
}

// Sum over `lanes` (a power of two) neighbouring lanes, in all of them.
template <int CTRL> __device__ __forceinline__ float plus_dpp(float x) {
    return x + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_sum(float x, int lanes) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    if (lanes > 1)
        x = plus_dpp<0xB1>(x);        // lane ^ 1
    if (lanes > 2)
        x = plus_dpp<0x4E>(x);        // lane ^ 2
    if (lanes > 4)
        x = plus_dpp<0x141>(x);       // 7 - lane: the other four
    if (lanes > 8)
        x = plus_dpp<0x140>(x);       // 15 - lane: the other eight
    if (lanes > 16) {
        const u32x2 s = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
        x = __uint_as_float(s.x) + __uint_as_float(s.y);
    }
    if (lanes > 32) {
        const u32x2 s = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
        x = __uint_as_float(s.x) + __uint_as_float(s.y);
    }
    return x;
}

// 1 / sqrt(sum / d + eps), the instruction's to 1 ulp; an infinite mean gives 0.
__device__ __forceinline__ float inverse_root(float sum, int d, float eps) {
    return __builtin_amdgcn_rsqf(sum * __builtin_amdgcn_rcpf((float)d) + eps);
}

// Where a unit's two groups of V values lie in the row, and its first pair.
template <int V> struct Unit {
    int lo, hi, pair;
    bool live, rotated;
    __device__ __forceinline__ Unit(int u, int d, int rot, bool interleaved) {
        live = u < d / (2 * V);
        pair = u * V;
        rotated = live && 2 * pair < rot;
        lo = rotated && !interleaved ? pair : 2 * pair;
        hi = rotated && !interleaved ? pair + rot / 2 : 2 * pair + V;
    }
};

// (lo, hi) turned by the pairs' angles.
template <int V>
__device__ __forceinline__ void turn(float (&lo)[V], float (&hi)[V], const float (&c)[V], const float (&s)[V],
                                     bool interleaved) {
    if (interleaved) {
        // Pair i holds values 2i, 2i + 1 of lo followed by hi.
        float z[2 * V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float a = 2 * i < V ? lo[(2 * i) % V] : hi[(2 * i) % V];
            const float b = 2 * i + 1 < V ? lo[(2 * i + 1) % V] : hi[(2 * i + 1) % V];
            z[2 * i] = a * c[i] - b * s[i];
            z[2 * i + 1] = b * c[i] + a * s[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lo[i] = z[i];
            hi[i] = z[V + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float a = lo[i], b = hi[i];
            lo[i] = a * c[i] - b * s[i];
            hi[i] = b * c[i] + a * s[i];
        }
    }
}

// The angles of V pairs of a token: NaN where its position has no table row.
template <int V>
__device__ __forceinline__ void angles(const float *cos, const float *sin, int position, int64_t rows, int rot,
                                       int pair, float (&c)[V], float (&s)[V]) {
    const bool known = position >= 0 && position < rows;
    const uint64_t at = (uint64_t)(known ? position : 0) * (uint32_t)(rot / 2) + (uint32_t)pair;
    if (rows > 0) {
        load<float, V>(cos, at, c);
        load<float, V>(sin, at, s);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        c[i] = known ? c[i] : __uint_as_float(0x7FC00000u);
        s[i] = known ? s[i] : __uint_as_float(0x7FC00000u);
    }
}

// N units a lane, `lanes` lanes a row (a power of two, at most a wave); a
// workgroup's rows are of one part, tokens times heads of it below 2^31.
template <typename T, int V, int N>
__global__ void __launch_bounds__(kThreads) head_rows_kernel(const HeadRowsParams p, int lanes) {
    const int which = p.parts > 2 && blockIdx.x >= p.part[2].first ? 2 : p.parts > 1 && blockIdx.x >= p.part[1].first ? 1 : 0;
    const HeadPart &part = p.part[which];
    const int lane = threadIdx.x & (lanes - 1);
    const uint32_t rows = (uint32_t)p.tokens * part.heads;
    const uint32_t row = (blockIdx.x - part.first) * (uint32_t)(kThreads / lanes) + threadIdx.x / (uint32_t)lanes;
    if (row >= rows)
        return;
    const uint32_t token = (__umulhi(row, part.heads_mul) + row) >> part.heads_shift;
    const uint32_t head = row - token * part.heads;
    const bool turns = p.rot > 0 && part.rotate, normed = part.weight != nullptr;
    const int position = turns ? p.positions[token] : 0;
    const int64_t slot = part.paged ? p.slots[token] : 0;
    const uint64_t in_row = (uint64_t)token * part.in_token + (uint64_t)head * part.in_head;

    float lo[N][V], hi[N][V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
        if (u.live) {
            load<T, V>(part.in, in_row + u.lo, lo[n]);
            load<T, V>(part.in, in_row + u.hi, hi[n]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                lo[n][i] = hi[n][i] = 0.0f;
        }
    }
    float wl[N][V], wh[N][V], c[N][V], s[N][V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
        if (u.live && normed) {
            load<float, V>(part.weight, u.lo, wl[n]);
            load<float, V>(part.weight, u.hi, wh[n]);
        }
        if (u.rotated && turns)
            angles<V>(p.cos, p.sin, position, p.rows, p.rot, u.pair, c[n], s[n]);
    }
    uint64_t out_row = (uint64_t)token * part.out_token + (uint64_t)head * part.out_head;
    if (part.paged) {
        if (slot < 0 || slot >= p.cache_slots)
            return;
        const uint32_t page = (__umulhi((uint32_t)slot, p.page_mul) + (uint32_t)slot) >> p.page_shift;
        out_row = (uint64_t)page * part.out_token + (uint64_t)((uint32_t)slot - page * p.page_size) * part.out_slot +
                  (uint64_t)head * part.out_head;
    }
    if (normed) {
        float sum = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < V; ++i)
                sum += lo[n][i] * lo[n][i] + hi[n][i] * hi[n][i];
        const float r = inverse_root(lane_sum(sum, lanes), p.d, p.eps);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                lo[n][i] *= r * wl[n][i];
                hi[n][i] *= r * wh[n][i];
            }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
        if (!u.live)
            continue;
        if (u.rotated && turns)
            turn<V>(lo[n], hi[n], c[n], s[n], p.interleaved);
        store<V>(part.out, out_row + u.lo, lo[n], part.out_bf16);
        store<V>(part.out, out_row + u.hi, hi[n], part.out_bf16);
    }
}

// Gradient.  A workgroup takes rows of one part in strides, a lane the same
// units of each, so the weight's gradient adds up in the lane's registers;
// the workgroup's row groups add theirs in LDS in a fixed order and leave one
// partial row, which head_weight_kernel adds up.
template <typename T, int V, int N>
__global__ void __launch_bounds__(kThreads) head_grad_kernel(const HeadGradParams p, int lanes) {
    __shared__ float sums[kThreads * 2 * V];
    const bool second = (int)blockIdx.x >= p.part[0].groups;
    const HeadGradPart &part = p.part[second];
    const int group = blockIdx.x - (second ? p.part[0].groups : 0);
    const int lane = threadIdx.x & (lanes - 1);
    const int per = kThreads / lanes;
    const uint32_t rows = (uint32_t)p.tokens * part.heads;
    const bool normed = part.weight != nullptr;

    float wl[N][V], wh[N][V], dl[N][V], dh[N][V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
#pragma unroll
        for (int i = 0; i < V; ++i)
            dl[n][i] = dh[n][i] = 0.0f;
        if (u.live && normed) {
            load<float, V>(part.weight, u.lo, wl[n]);
            load<float, V>(part.weight, u.hi, wh[n]);
        }
    }
    // A row's loads are on their way while the row before it is worked on; its
    // position, which they wait for, a row earlier still.
    const uint32_t step = (uint32_t)part.groups * per;
    auto token_of = [&](uint32_t row) { return (__umulhi(row, part.heads_mul) + row) >> part.heads_shift; };
    auto position_of = [&](uint32_t row) { return p.positions != nullptr && row < rows ? p.positions[token_of(row)] : 0; };
    struct Item {
        Raw<T, V> zl[N], zh[N], xl[N], xh[N];
        float c[N][V], s[N][V];
    };
    auto fetch = [&](uint32_t row, int position) {
        Item item;
        const uint32_t token = token_of(row), head = row - token * part.heads;
        const uint64_t x_row = (uint64_t)token * part.x_token + (uint64_t)head * part.x_head;
        const uint64_t z_row = (uint64_t)token * part.dz_token + (uint64_t)head * part.dz_head;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
            if (!u.live)
                continue;
            item.zl[n].load(part.dz, z_row + u.lo);
            item.zh[n].load(part.dz, z_row + u.hi);
            if (normed) {
                item.xl[n].load(part.x, x_row + u.lo);
                item.xh[n].load(part.x, x_row + u.hi);
            }
            if (u.rotated && p.positions != nullptr)
                angles<V>(p.cos, p.sin, position, p.rows, p.rot, u.pair, item.c[n], item.s[n]);
        }
        return item;
    };
    uint32_t row = group * per + threadIdx.x / lanes;
    Item next;
    int position = position_of(row);
    if (row < rows)
        next = fetch(row, position);
    position = position_of(row + step);
    for (; row < rows; row += step) {
        const Item item = next;
        if (row + step < rows)
            next = fetch(row + step, position);
        position = position_of(row + 2 * step);
        const uint32_t token = token_of(row), head = row - token * part.heads;
        const uint64_t d_row = (uint64_t)token * part.dx_token + (uint64_t)head * part.dx_head;
        float gl[N][V], gh[N][V], xl[N][V], xh[N][V];
        float square = 0.0f, dot = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
            if (!u.live)
                continue;
            item.zl[n].get(gl[n]);
            item.zh[n].get(gh[n]);
            if (u.rotated && p.positions != nullptr) {
                float back[V];
#pragma unroll
                for (int i = 0; i < V; ++i)
                    back[i] = -item.s[n][i];
                turn<V>(gl[n], gh[n], item.c[n], back, p.interleaved);
            }
            if (normed) {
                item.xl[n].get(xl[n]);
                item.xh[n].get(xh[n]);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    square += xl[n][i] * xl[n][i] + xh[n][i] * xh[n][i];
                    dot += gl[n][i] * wl[n][i] * xl[n][i] + gh[n][i] * wh[n][i] * xh[n][i];
                }
            }
        }
        float r = 1.0f, back = 0.0f;
        if (normed) {
            r = inverse_root(lane_sum(square, lanes), p.d, p.eps);
            back = r * r * (lane_sum(dot, lanes) * __builtin_amdgcn_rcpf((float)p.d));
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
            if (!u.live)
                continue;
            if (normed) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dl[n][i] += gl[n][i] * (xl[n][i] * r);
                    dh[n][i] += gh[n][i] * (xh[n][i] * r);
                    gl[n][i] = r * (gl[n][i] * wl[n][i] - xl[n][i] * back);
                    gh[n][i] = r * (gh[n][i] * wh[n][i] - xh[n][i] * back);
                }
            }
            store<V>(part.dx, d_row + u.lo, gl[n], sizeof(T) == 2);
            store<V>(part.dx, d_row + u.hi, gh[n], sizeof(T) == 2);
        }
    }
    if (!normed)
        return;
    // One pass of LDS per unit of a lane: [row group][lane][2V].
#pragma unroll
    for (int n = 0; n < N; ++n) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sums[i * kThreads + threadIdx.x] = dl[n][i];
            sums[(V + i) * kThreads + threadIdx.x] = dh[n][i];
        }
        __syncthreads();
        // Thread t adds value t / lanes (of the 2V, in strides) of lane t % lanes.
        for (int v = threadIdx.x / lanes; v < 2 * V; v += per) {
            const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
            if (!u.live)
                break;
            float total = 0.0f;
            for (int g = 0; g < per; ++g)
                total += sums[v * kThreads + g * lanes + lane];
            part.partial[(int64_t)group * p.d + (v < V ? u.lo + v : u.hi + v - V)] = total;
        }
    }
}

// dweight[i] = sum over the part's groups of partial[group][i]: a workgroup takes
// two columns (d is even), a lane every 256th group in order, then the lanes' sums
// are added in halves.
__global__ void __launch_bounds__(kThreads) head_weight_kernel(const HeadGradParams p) {
    typedef float f32x2 __attribute__((ext_vector_type(2), aligned(4)));
    __shared__ f32x2 sums[kThreads];
    const HeadGradPart &part = p.part[blockIdx.x / (p.d / 2)];
    const int i = (int)(blockIdx.x % (p.d / 2)) * 2;
    if (part.weight == nullptr)
        return;
    f32x2 total = {0.0f, 0.0f};
#pragma unroll 4
    for (int g = threadIdx.x; g < part.groups; g += kThreads)
        total += *reinterpret_cast<const f32x2 *>(part.partial + (int64_t)g * p.d + i);
    sums[threadIdx.x] = total;
    for (int half = kThreads / 2; half > 0; half /= 2) {
        __syncthreads();
        if (threadIdx.x < half)
            sums[threadIdx.x] += sums[threadIdx.x + half];
    }
    if (threadIdx.x == 0)
        *reinterpret_cast<f32x2 *>(part.dweight + i) = sums[0];
}

// V of a row of d values, `rot` of them rotated.
int unit_width(bool bf16, int d, int rot) {
    for (int v = bf16 ? 8 : 4; v > 1; v /= 2)
        if ((rot / 2) % v == 0 && (d - rot) % (2 * v) == 0)
            return v;
    return 1;
}

// 16 values a lane where the row has them, so that what a row costs once is
// spread over many; at most 64 lanes (V == 1, d == 256).
int units_a_lane(int v) { return v == 8 ? 1 : 2; }
// The gradient's lanes hold more of each value.
int grad_units(int v) { return v >= 4 ? 1 : 2; }

// Lanes a row with n units a lane.
int row_lanes(int units, int n) {
    int lanes = 1;
    while (lanes * n < units)
        lanes *= 2;
    return lanes;
}

template <typename T, int V, int N> hipError_t rows_launch(HeadRowsParams p, int lanes, hipStream_t stream) {
    const int64_t per = kThreads / lanes;
    int64_t groups = 0;
    for (int i = 0; i < p.parts; ++i) {
        p.part[i].first = (uint32_t)groups;
        groups += (p.tokens * p.part[i].heads + per - 1) / per;
    }
    hipLaunchKernelGGL((head_rows_kernel<T, V, N>), dim3((unsigned)groups), dim3(kThreads), 0, stream, p, lanes);
    return hipGetLastError();
}

template <typename T, int V, int N> hipError_t grad_launch(const HeadGradParams &p, int lanes, hipStream_t stream) {
    const int groups = p.part[0].groups + p.part[1].groups;
    if (groups > 0) {
        hipLaunchKernelGGL((head_grad_kernel<T, V, N>), dim3((unsigned)groups), dim3(kThreads), 0, stream, p, lanes);
        if (hipError_t e = hipGetLastError(); e != hipSuccess)
            return e;
    }
    if (p.part[0].weight == nullptr && p.part[1].weight == nullptr)
        return hipSuccess;
    hipLaunchKernelGGL(head_weight_kernel, dim3((unsigned)p.d), dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_head_rows(bool bf16, const HeadRowsParams &p, hipStream_t stream) {
    const int v = unit_width(bf16, p.d, p.rot);
    const int lanes = row_lanes(p.d / (2 * v), units_a_lane(v));
    switch (v) {
    case 8: return rows_launch<uint16_t, 8, 1>(p, lanes, stream);
    case 4: return bf16 ? rows_launch<uint16_t, 4, 2>(p, lanes, stream) : rows_launch<float, 4, 2>(p, lanes, stream);
    case 2: return bf16 ? rows_launch<uint16_t, 2, 2>(p, lanes, stream) : rows_launch<float, 2, 2>(p, lanes, stream);
    default: return bf16 ? rows_launch<uint16_t, 1, 2>(p, lanes, stream) : rows_launch<float, 1, 2>(p, lanes, stream);
    }
}

int head_grad_groups(bool bf16, int64_t rows, int d, int rot, int most) {
    const int v = unit_width(bf16, d, rot);
    const int per = kThreads / row_lanes(d / (2 * v), grad_units(v));
    // One round of workgroups: four a compute unit, three with 8 values a load.
    return (int)std::min<int64_t>((rows + per - 1) / per, v == 8 ? std::max(most * 3 / 4, 1) : most);
}

hipError_t launch_head_grad(bool bf16, const HeadGradParams &p, hipStream_t stream) {
    const int v = unit_width(bf16, p.d, p.rot);
    const int lanes = row_lanes(p.d / (2 * v), grad_units(v));
    switch (v) {
    case 8: return grad_launch<uint16_t, 8, 1>(p, lanes, stream);
    case 4: return bf16 ? grad_launch<uint16_t, 4, 1>(p, lanes, stream) : grad_launch<float, 4, 1>(p, lanes, stream);
    case 2: return bf16 ? grad_launch<uint16_t, 2, 2>(p, lanes, stream) : grad_launch<float, 2, 2>(p, lanes, stream);
    default: return bf16 ? grad_launch<uint16_t, 1, 2>(p, lanes, stream) : grad_launch<float, 1, 2>(p, lanes, stream);
    }
}

}  // namespace pamk
