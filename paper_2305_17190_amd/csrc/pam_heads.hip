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
// row per token that its heads share through the caches.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pam_attention_internal.h"

namespace pamk {
namespace {

constexpr int kThreads = 256;
// Workgroups per launch at most (the grid, in threads, stays below 2^32).
constexpr int64_t kMaxGroups = 16777215;

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
__device__ __forceinline__ uint16_t to_bf16(float x) {
    const uint32_t u = __float_as_uint(x);
    const uint32_t r = (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
    return (uint16_t)((u & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC0u : r);
}

template <typename T, int V> __device__ __forceinline__ void load(const void *base, int64_t at, float (&x)[V]) {
    if constexpr (V == 1) {
        x[0] = widen(static_cast<const T *>(base)[at]);
    } else {
        const auto v = *reinterpret_cast<const typename Vec<T, V>::type *>(static_cast<const T *>(base) + at);
#pragma unroll
        for (int i = 0; i < V; ++i)
            x[i] = widen(v[i]);
    }
}

template <int V> __device__ __forceinline__ void store(void *base, int64_t at, const float (&x)[V], bool bf16) {
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

// Sum over `lanes` (a power of two) neighbouring lanes.
__device__ __forceinline__ float lane_sum(float x, int lanes) {
    for (int s = 1; s < lanes; s *= 2)
        x += __shfl_xor(x, s);
    return x;
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
    if (position >= 0 && position < rows) {
        const int64_t at = (int64_t)position * (rot / 2) + pair;
        load<float, V>(cos, at, c);
        load<float, V>(sin, at, s);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            c[i] = s[i] = __uint_as_float(0x7FC00000u);
    }
}

// N units a lane, `lanes` lanes a row (a power of two, at most a wave); rows,
// tokens times heads, below 2^31.
template <typename T, int V, int N>
__global__ void __launch_bounds__(kThreads) head_rows_kernel(const HeadRowsParams p, int lanes) {
    const int lane = threadIdx.x & (lanes - 1);
    const int64_t rows = p.tokens * p.heads;
    for (int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / lanes; row < rows;
         row += (int64_t)gridDim.x * (kThreads / lanes)) {
        const int64_t token = (uint32_t)row / (uint32_t)p.heads;
        int head = (int)(row - token * p.heads);
        int which = 0;
        while (which + 1 < p.parts && head >= p.part[which + 1].first)
            ++which;
        const HeadPart &part = p.part[which];
        head -= part.first;

        int64_t out_row;
        if (part.paged) {
            const int64_t slot = p.slots[token];
            if (slot < 0 || slot >= p.cache_slots)
                continue;
            const uint32_t page = (uint32_t)slot / (uint32_t)p.page_size;
            out_row = (int64_t)page * part.out_token + (int64_t)((uint32_t)slot - page * p.page_size) * part.out_slot +
                      (int64_t)head * part.out_head;
        } else {
            out_row = token * part.out_token + (int64_t)head * part.out_head;
        }
        const int64_t in_row = token * part.in_token + (int64_t)head * part.in_head;

        float lo[N][V], hi[N][V];
        float sum = 0.0f;
    #pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
            if (u.live) {
                load<T, V>(part.in, in_row + u.lo, lo[n]);
                load<T, V>(part.in, in_row + u.hi, hi[n]);
    #pragma unroll
                for (int i = 0; i < V; ++i)
                    sum += lo[n][i] * lo[n][i] + hi[n][i] * hi[n][i];
            }
        }
        float r = 1.0f;
        if (part.weight != nullptr)
            r = 1.0f / sqrtf(lane_sum(sum, lanes) / (float)p.d + p.eps);
    #pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
            if (!u.live)
                continue;
            if (part.weight != nullptr) {
                float wl[V], wh[V];
                load<float, V>(part.weight, u.lo, wl);
                load<float, V>(part.weight, u.hi, wh);
    #pragma unroll
                for (int i = 0; i < V; ++i) {
                    lo[n][i] = lo[n][i] * r * wl[i];
                    hi[n][i] = hi[n][i] * r * wh[i];
                }
            }
            if (part.rotate && u.rotated) {
                float c[V], s[V];
                angles<V>(p.cos, p.sin, p.positions[token], p.rows, p.rot, u.pair, c, s);
                turn<V>(lo[n], hi[n], c, s, p.interleaved);
            }
            store<V>(part.out, out_row + u.lo, lo[n], part.out_bf16);
            store<V>(part.out, out_row + u.hi, hi[n], part.out_bf16);
        }
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
    const int64_t rows = p.tokens * part.heads;
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
    for (int64_t row = (int64_t)group * per + threadIdx.x / lanes; row < rows; row += (int64_t)part.groups * per) {
        const int64_t token = (uint32_t)row / (uint32_t)part.heads;
        const int64_t head = row - token * part.heads;
        const int64_t x_row = token * part.x_token + head * part.x_head;
        const int64_t z_row = token * part.dz_token + head * part.dz_head;
        const int64_t d_row = token * part.dx_token + head * part.dx_head;
        float gl[N][V], gh[N][V], xl[N][V], xh[N][V];
        float square = 0.0f, dot = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane + n * lanes, p.d, p.rot, p.interleaved);
            if (!u.live)
                continue;
            load<T, V>(part.dz, z_row + u.lo, gl[n]);
            load<T, V>(part.dz, z_row + u.hi, gh[n]);
            if (normed) {
                load<T, V>(part.x, x_row + u.lo, xl[n]);
                load<T, V>(part.x, x_row + u.hi, xh[n]);
            }
            if (u.rotated && p.positions != nullptr) {
                float c[V], s[V];
                angles<V>(p.cos, p.sin, p.positions[token], p.rows, p.rot, u.pair, c, s);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    s[i] = -s[i];
                turn<V>(gl[n], gh[n], c, s, p.interleaved);
            }
            if (normed) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    square += xl[n][i] * xl[n][i] + xh[n][i] * xh[n][i];
                    dot += gl[n][i] * wl[n][i] * xl[n][i] + gh[n][i] * wh[n][i] * xh[n][i];
                }
            }
        }
        float r = 1.0f, back = 0.0f;
        if (normed) {
            r = 1.0f / sqrtf(lane_sum(square, lanes) / (float)p.d + p.eps);
            back = r * r * (lane_sum(dot, lanes) / (float)p.d);
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

// dweight[i] = sum over the part's groups of partial[group][i]: 16 columns and
// 16 runs of groups a workgroup, each run in order, then the runs in order.
__global__ void __launch_bounds__(256) head_weight_kernel(const HeadGradParams p, int columns) {
    __shared__ float sums[16][17];
    const HeadGradPart &part = p.part[blockIdx.x / columns];
    const int c = threadIdx.x % 16, run = threadIdx.x / 16;
    const int i = (int)(blockIdx.x % columns) * 16 + c;
    if (part.weight == nullptr)
        return;
    float total = 0.0f;
    if (i < p.d)
        for (int g = run; g < part.groups; g += 16)
            total += part.partial[(int64_t)g * p.d + i];
    sums[run][c] = total;
    __syncthreads();
    if (run == 0 && i < p.d) {
        total = 0.0f;
        for (int r = 0; r < 16; ++r)
            total += sums[r][c];
        part.dweight[i] = total;
    }
}

// V of a row of d values, `rot` of them rotated.
int unit_width(bool bf16, int d, int rot) {
    for (int v = bf16 ? 8 : 4; v > 1; v /= 2)
        if ((rot / 2) % v == 0 && (d - rot) % (2 * v) == 0)
            return v;
    return 1;
}

// Lanes a row: its units on up to a wave's lanes.
int row_lanes(int units) {
    int lanes = 1;
    while (lanes < units && lanes < 64)
        lanes *= 2;
    return lanes;
}

template <typename T, int V, int N> hipError_t rows_launch(const HeadRowsParams &p, int lanes, hipStream_t stream) {
    const int64_t per = kThreads / lanes;
    const int64_t groups = std::min((p.tokens * p.heads + per - 1) / per, kMaxGroups);
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
    const int columns = (p.d + 15) / 16;
    hipLaunchKernelGGL(head_weight_kernel, dim3((unsigned)(2 * columns)), dim3(256), 0, stream, p, columns);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_head_rows(bool bf16, const HeadRowsParams &p, hipStream_t stream) {
    const int v = unit_width(bf16, p.d, p.rot);
    const int units = p.d / (2 * v);
    const int lanes = row_lanes(units);
    if (units > 64)   // V == 1 and d > 128
        return bf16 ? rows_launch<uint16_t, 1, 2>(p, lanes, stream) : rows_launch<float, 1, 2>(p, lanes, stream);
    switch (v) {
    case 8: return rows_launch<uint16_t, 8, 1>(p, lanes, stream);
    case 4: return bf16 ? rows_launch<uint16_t, 4, 1>(p, lanes, stream) : rows_launch<float, 4, 1>(p, lanes, stream);
    case 2: return bf16 ? rows_launch<uint16_t, 2, 1>(p, lanes, stream) : rows_launch<float, 2, 1>(p, lanes, stream);
    default: return bf16 ? rows_launch<uint16_t, 1, 1>(p, lanes, stream) : rows_launch<float, 1, 1>(p, lanes, stream);
    }
}

int head_grad_groups(bool bf16, int64_t rows, int d, int rot, int most) {
    const int per = kThreads / row_lanes(d / (2 * unit_width(bf16, d, rot)));
    return (int)std::min<int64_t>((rows + per - 1) / per, most);
}

hipError_t launch_head_grad(bool bf16, const HeadGradParams &p, hipStream_t stream) {
    const int v = unit_width(bf16, p.d, p.rot);
    const int units = p.d / (2 * v);
    const int lanes = row_lanes(units);
    if (units > 64)
        return bf16 ? grad_launch<uint16_t, 1, 2>(p, lanes, stream) : grad_launch<float, 1, 2>(p, lanes, stream);
    switch (v) {
    case 8: return grad_launch<uint16_t, 8, 1>(p, lanes, stream);
    case 4: return bf16 ? grad_launch<uint16_t, 4, 1>(p, lanes, stream) : grad_launch<float, 4, 1>(p, lanes, stream);
    case 2: return bf16 ? grad_launch<uint16_t, 2, 1>(p, lanes, stream) : grad_launch<float, 2, 1>(p, lanes, stream);
    default: return bf16 ? grad_launch<uint16_t, 1, 1>(p, lanes, stream) : grad_launch<float, 1, 1>(p, lanes, stream);
    }
}

}  // namespace pamk
