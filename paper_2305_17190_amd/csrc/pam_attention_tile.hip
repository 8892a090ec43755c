// PAM attention of many rows over a paged cache for gfx950: the two products
// as tiles on the vector ALU (PAM has no use for the matrix cores), with the
// scores between them in a workspace.
//
// A unit is 64 WM rows of one key head (its query heads times the new tokens);
// a wave owns a 64 x 64 block of outputs, a lane 8 x 8 of them, and each k step
// of a tile is 64 times one integer addition and one float fma a lane (see
// pam_attention_device.h for the encodings): keys or values as two planes (1 +
// M and the power of two), queries or probabilities as one, all staged into
// LDS a chunk of 16 k steps at a time, transposed to k-major, while the next
// chunk is on its way into registers.
//
// Scores first: a tile of 64 WM rows and 64 WN keys goes to the workspace
// key-major, with each row's maximum and sum of exponentials over the tile;
// the tile of the values then reads the row's statistics over all keys, turns
// scores into normalised probabilities as it stages them, and adds up its
// split's keys.  Storing a score costs 8 bytes of traffic, scoring again d
// PAM-MACs, which take several times as long.
//
// Bound by the vector ALU: 2 lane-ops a PAM-MAC.

#include "pam_attention_device.h"

namespace pamk {
namespace {

constexpr int kStep = 16;             // k steps of a chunk
constexpr int kPad = 4;               // words after each k step's row in LDS
// Chunks whose sums a lane adds up before they join its totals: the float32
// error of a sum grows with the length of its chain.
constexpr int kChainChunks = 16;

// A lane's 8 rows or columns of a 64-wide block: two groups of four.
__device__ __forceinline__ int place(int group, int i) { return (i / 4) * 32 + group * 4 + i % 4; }

// acc[r][c] += b[k][row r] .^ a[k][column c] over one chunk in LDS.
template <int BM, int BN>
__device__ __forceinline__ void chunk_product(const float *a1, const float *m, const uint32_t *b, int row, int col,
                                              float (&acc)[8][8]) {
#pragma unroll 2
    for (int k = 0; k < kStep; ++k) {
        float x[8], y[8];
        uint32_t z[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            *reinterpret_cast<float4 *>(x + 4 * h) = *reinterpret_cast<const float4 *>(a1 + k * (BN + kPad) + col + 32 * h);
            *reinterpret_cast<float4 *>(y + 4 * h) = *reinterpret_cast<const float4 *>(m + k * (BN + kPad) + col + 32 * h);
            *reinterpret_cast<uint4 *>(z + 4 * h) = *reinterpret_cast<const uint4 *>(b + k * (BM + kPad) + row + 32 * h);
        }
#pragma unroll
        for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int c = 0; c < 8; ++c)
                acc[r][c] = pam_fma(x[c], y[c], z[r], acc[r][c]);
    }
}

__device__ __forceinline__ bool all_finite(const float (&acc)[8][8]) {
    float probe = 0.0f;                // NaN once any element is inf or NaN
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c)
            probe = __builtin_fmaf(acc[r][c], 0.0f, probe);
    return probe == 0.0f;
}

// Replaces each inf or NaN of a lane's 8 x 8 sums by again(r, c, value).  The
// elements are picked by compares, so the array stays in registers.
template <typename F> __device__ __forceinline__ void sum_again(float (&acc)[8][8], F again) {
#pragma unroll 1
    for (int e = 0; e < 64; ++e) {
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i)
            x = i == e ? acc[i / 8][i % 8] : x;
        if (finite(x))
            continue;
        x = again(e / 8, e % 8, x);
#pragma unroll
        for (int i = 0; i < 64; ++i)
            acc[i / 8][i % 8] = i == e ? x : acc[i / 8][i % 8];
    }
}

// Eight float32 or bfloat16 values on their way into LDS.
struct Eight {
    u32x4 w[2];
    __device__ __forceinline__ void clear() { w[0] = w[1] = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void load(const void *base, int64_t at, bool bf16) {
        if (bf16) {
            w[0] = load16<uint16_t>(base, at);
        } else {
            w[0] = load16<float>(base, at);
            w[1] = load16<float>(base, at + 4);
        }
    }
    __device__ __forceinline__ uint32_t operator()(int i, bool bf16) const {
        return bf16 ? element<uint16_t>(w[0], i) : w[i / 4][i % 4];
    }
};

template <typename T, int WM, int WN, bool QB>
__global__ void __launch_bounds__(64 * WM * WN) tile_scores_kernel(const AttentionParams p) {
    constexpr int BM = 64 * WM, BN = 64 * WN, NT = 64 * WM * WN;
    constexpr int KI = 2 / WM > 0 ? 2 / WM : 1;    // key items of 8 values a lane and chunk
    constexpr int QI = 2 / WN > 0 ? 2 / WN : 1;    // query items
    constexpr bool KB = sizeof(T) == 2;
    __shared__ float a1[kStep * (BN + kPad)], am[kStep * (BN + kPad)];
    __shared__ uint32_t qb[kStep * (BM + kPad)];
    __shared__ int lo[BM], hi[BM];
    __shared__ int valid[BN];
    __shared__ float across[WN][BM];

    const int tiles = p.splits * (p.split_keys / BN);
    const int tile = blockIdx.x % tiles, index = blockIdx.x / tiles;
    const Unit unit(p, p.first_unit + index);
    const int begin = tile * BN;
    if (unit.rows == 0 || begin >= unit.hi || begin + BN <= unit.lo)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tx = lane & 7, ty = lane >> 3;
    const int row0 = (wave % WM) * 64 + ty * 4, col0 = (wave / WM) * 64 + tx * 4;

    for (int r = tid; r < BM; r += NT) {
        lo[r] = r < unit.rows ? unit.row_lo(p, r) : 0;
        hi[r] = r < unit.rows ? unit.row_hi(p, r) : 0;
    }
    // The lane's keys and queries: one row each for all chunks.
    int64_t k_from[KI], q_from[QI];
#pragma unroll
    for (int i = 0; i < KI; ++i) {
        const int item = tid + i * NT, j = item % BN, key = begin + j;
        k_from[i] = key >= unit.lo && key < unit.hi ? unit.key_at(p, p.k, key) : -1;
        if (item / BN == 0)
            valid[j] = k_from[i] >= 0;
    }
#pragma unroll
    for (int i = 0; i < QI; ++i) {
        const int r = (tid + i * NT) % BM;
        q_from[i] = r < unit.rows ? unit.q_at(p, r) : -1;
    }

    Eight kw[KI], qw[QI];
    auto fetch = [&](int d0) {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int at = d0 + (tid + i * NT) / BN * 8;
            kw[i].clear();
            if (k_from[i] >= 0 && at < p.d)
                kw[i].load(p.k.data, k_from[i] + at, KB);
        }
#pragma unroll
        for (int i = 0; i < QI; ++i) {
            const int at = d0 + (tid + i * NT) / BM * 8;
            qw[i].clear();
            if (q_from[i] >= 0 && at < p.d)
                qw[i].load(p.q, q_from[i] + at, QB);
        }
    };
    auto stage = [&]() {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int item = tid + i * NT, j = item % BN, k = item / BN * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t a = kw[i](e, KB);
                a1[(k + e) * (BN + kPad) + j] = one_mantissa(a);
                am[(k + e) * (BN + kPad) + j] = power(a);
            }
        }
#pragma unroll
        for (int i = 0; i < QI; ++i) {
            const int item = tid + i * NT, r = item % BM, k = item / BM * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                qb[(k + e) * (BM + kPad) + r] = biased(qw[i](e, QB));
        }
    };

    float acc[8][8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c)
            acc[r][c] = 0.0f;
    fetch(0);
    for (int d0 = 0; d0 < p.d; d0 += kStep) {
        __syncthreads();
        stage();
        __syncthreads();
        if (d0 + kStep < p.d)
            fetch(d0 + kStep);
        chunk_product<BM, BN>(a1, am, qb, row0, col0, acc);
    }

    if (!all_finite(acc))
        sum_again(acc, [&](int r, int c, float value) {
            const int row = row0 + place(0, r), key = begin + col0 + place(0, c);
            if (row >= unit.rows || key < lo[row] || key >= hi[row])
                return value;
            const int64_t from = unit.key_at(p, p.k, key);
            if (from < 0)
                return value;
            float sum = 0.0f;
            const int64_t q = unit.q_at(p, row);
            for (int i = 0; i < p.d; ++i)
                sum += __uint_as_float(pam_full(load_bits(p.q, q + i, QB), load_bits(p.k.data, from + i, KB)));
            return sum;
        });

    // Scaled scores, -inf where the row does not see the key; the rows' maxima.
    float *scores = p.scores + ((int64_t)index * tiles * BN + begin) * BM;
    float best[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int row = row0 + place(0, r);
        best[r] = kNegInf;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int j = col0 + place(0, c);
            const bool sees = valid[j] && begin + j >= lo[row] && begin + j < hi[row];
            acc[r][c] = sees ? acc[r][c] * p.scale : kNegInf;
            best[r] = fmaxf(best[r], acc[r][c]);
        }
#pragma unroll
        for (int x = 1; x < 8; x *= 2)
            best[r] = fmaxf(best[r], __shfl_xor(best[r], x));
        if (tx == 0)
            across[wave / WM][row] = best[r];
    }
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<float4 *>(scores + (int64_t)(col0 + place(0, c)) * BM + row0 + 32 * h) =
                make_float4(acc[4 * h][c], acc[4 * h + 1][c], acc[4 * h + 2][c], acc[4 * h + 3][c]);
    __syncthreads();
    float sum[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int row = row0 + place(0, r);
#pragma unroll
        for (int w = 0; w < WN; ++w)
            best[r] = fmaxf(best[r], across[w][row]);
        sum[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            sum[r] += exp2_from(acc[r][c], best[r]);
#pragma unroll
        for (int x = 1; x < 8; x *= 2)
            sum[r] += __shfl_xor(sum[r], x);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (tx == 0)
            across[wave / WM][row0 + place(0, r)] = sum[r];
    __syncthreads();
    float *stats = p.stats + ((int64_t)index * tiles + tile) * 2 * BM;
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (tx == 0 && wave / WM == 0) {
            const int row = row0 + place(0, r);
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < WN; ++w)
                total += across[w][row];
            stats[row] = best[r];
            stats[BM + row] = total;
        }
}

template <typename T, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) tile_values_kernel(const AttentionParams p) {
    constexpr int BM = 64 * WM, BN = 64 * WN, NT = 64 * WM * WN;
    constexpr int E = kPer<T>;
    constexpr int SI = kStep * BM / 4 / NT;        // score items of 4 rows a lane and chunk
    constexpr int VI = kStep * BN / E / NT;        // value items of 16 bytes
    constexpr int SK = NT / (BM / 4);              // keys between a lane's score items
    constexpr int VK = NT / (BN / E);              // and between its value items
    constexpr bool VB = sizeof(T) == 2;
    __shared__ float a1[kStep * (BN + kPad)], am[kStep * (BN + kPad)];
    __shared__ uint32_t pb[kStep * (BM + kPad)];
    __shared__ float row_max[BM], row_sum[BM];
    __shared__ int lo[BM], hi[BM];

    const int dtiles = (p.d + BN - 1) / BN;
    const int col_tile = blockIdx.x % dtiles;
    const int split = blockIdx.x / dtiles % p.splits, index = blockIdx.x / dtiles / p.splits;
    const Unit unit(p, p.first_unit + index);
    const int begin = max(unit.lo, split * p.split_keys), end = min(unit.hi, (split + 1) * p.split_keys);
    const bool alone = p.partial == nullptr;
    if (unit.rows == 0 || (begin >= end && !alone))
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tx = lane & 7, ty = lane >> 3;
    const int row0 = (wave % WM) * 64 + ty * 4, col0 = (wave / WM) * 64 + tx * 4;

    // The rows' maxima and sums over all key tiles.
    constexpr int kTile = 128;                     // keys of a score tile
    const int tiles = p.splits * (p.split_keys / kTile);
    const float *stats = p.stats + (int64_t)index * tiles * 2 * BM;
    const int first = unit.lo / kTile, last = unit.hi > unit.lo ? (unit.hi - 1) / kTile : first - 1;
    for (int r = tid; r < BM; r += NT) {
        float m = kNegInf, l = 0.0f;
        for (int t = first; t <= last; ++t)
            m = fmaxf(m, stats[(int64_t)t * 2 * BM + r]);
        for (int t = first; t <= last; ++t)
            l += stats[(int64_t)t * 2 * BM + BM + r] * exp2_from(stats[(int64_t)t * 2 * BM + r], m);
        row_max[r] = m;
        row_sum[r] = l;
        lo[r] = r < unit.rows ? unit.row_lo(p, r) : 0;
        hi[r] = r < unit.rows ? unit.row_hi(p, r) : 0;
    }
    __syncthreads();
    const int my_row = tid % (BM / 4) * 4;
    float m4[4], inverse4[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m4[i] = row_max[my_row + i];
        const float l = row_sum[my_row + i];
        inverse4[i] = l > 0.0f ? 1.0f / l : 0.0f;
    }

    const float *scores = p.scores + (int64_t)index * tiles * kTile * BM;
    const int col = tid % (BN / E) * E, column = col_tile * BN + col;
    float4 sw[SI];
    u32x4 vw[VI];
    int64_t v_from[VI];
    auto locate = [&](int k0) {
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int key = k0 + tid / (BN / E) + i * VK;
            v_from[i] = key >= begin && key < end && column < p.d ? unit.key_at(p, p.v, key) : -1;
        }
    };
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < SI; ++i)
            sw[i] = *reinterpret_cast<const float4 *>(scores + (int64_t)(k0 + tid / (BM / 4) + i * SK) * BM + my_row);
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            vw[i] = u32x4{0, 0, 0, 0};
            if (v_from[i] >= 0)
                vw[i] = load16<T>(p.v.data, v_from[i] + column);
        }
    };
    auto stage = [&](int k0) {
#pragma unroll
        for (int i = 0; i < SI; ++i) {
            const int k = tid / (BM / 4) + i * SK;
            const bool mine = k0 + k >= begin && k0 + k < end;
            const float t[4] = {sw[i].x, sw[i].y, sw[i].z, sw[i].w};
            uint32_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                b[e] = mine ? probability(exp2_from(t[e], m4[e]), inverse4[e]) : 0u - kBias;
            *reinterpret_cast<uint4 *>(pb + k * (BM + kPad) + my_row) = make_uint4(b[0], b[1], b[2], b[3]);
        }
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int at = (tid / (BN / E) + i * VK) * (BN + kPad) + col;
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                float x[4], y[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    const uint32_t a = element<T>(vw[i], e + f);
                    x[f] = one_mantissa(a);
                    y[f] = power(a);
                }
                *reinterpret_cast<float4 *>(a1 + at + e) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4 *>(am + at + e) = make_float4(y[0], y[1], y[2], y[3]);
            }
        }
    };

    float acc[8][8], total[8][8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c)
            acc[r][c] = total[r][c] = 0.0f;
    const int start = begin / kStep * kStep;
    if (begin < end) {
        locate(start);
        fetch(start);
        if (start + kStep < end)
            locate(start + kStep);
    }
    int chain = 0;
    for (int k0 = start; k0 < end; k0 += kStep) {
        __syncthreads();
        stage(k0);
        __syncthreads();
        if (k0 + kStep < end) {
            fetch(k0 + kStep);
            if (k0 + 2 * kStep < end)
                locate(k0 + 2 * kStep);
        }
        chunk_product<BM, BN>(a1, am, pb, row0, col0, acc);
        if (++chain == kChainChunks) {
            chain = 0;
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    total[r][c] += acc[r][c];
                    acc[r][c] = 0.0f;
                }
        }
    }
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c)
            total[r][c] += acc[r][c];

    if (!all_finite(total))
        sum_again(total, [&](int r, int c, float value) {
            const int row = row0 + place(0, r), i = col_tile * BN + col0 + place(0, c);
            if (row >= unit.rows || i >= p.d)
                return value;
            const float m = row_max[row], inverse = row_sum[row] > 0.0f ? 1.0f / row_sum[row] : 0.0f;
            float sum = 0.0f;
            for (int key = max(begin, lo[row]); key < min(end, hi[row]); ++key) {
                const int64_t from = unit.key_at(p, p.v, key);
                if (from < 0)
                    continue;
                const uint32_t b = probability(exp2_from(scores[(int64_t)key * BM + row], m), inverse);
                sum += __uint_as_float(pam_full(b + kBias, load_bits(p.v.data, from + i, VB)));
            }
            return sum;
        });
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int row = row0 + place(0, r);
        if (row >= unit.rows)
            continue;
        const float l = row_sum[row];
        float *to = alone ? p.out + unit.out_at(p, row)
                          : p.partial + (((int64_t)index * p.splits + split) * BM + row) * p.d;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = col_tile * BN + col0 + 32 * h;
            if (i >= p.d)
                continue;
            f32x4 v = {total[r][4 * h], total[r][4 * h + 1], total[r][4 * h + 2], total[r][4 * h + 3]};
            if (!(l > 0.0f))               // no weight, or a NaN score
                v = f32x4{l, l, l, l};
            *reinterpret_cast<f32x4 *>(to + i) = v;
        }
    }
}

template <typename T, bool QB> hipError_t scores_launch(const AttentionParams &p, int units, hipStream_t stream) {
    const unsigned grid = (unsigned)(units * p.splits * (p.split_keys / 128));
    if (p.rows == 128)
        hipLaunchKernelGGL((tile_scores_kernel<T, 2, 2, QB>), dim3(grid), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((tile_scores_kernel<T, 1, 2, QB>), dim3(grid), dim3(128), 0, stream, p);
    return hipGetLastError();
}

template <typename T> hipError_t values_launch(const AttentionParams &p, int units, hipStream_t stream) {
    const int wide = p.d > 64;
    const unsigned grid = (unsigned)(units * p.splits * (wide ? (p.d + 127) / 128 : 1));
    if (p.rows == 128 && wide)
        hipLaunchKernelGGL((tile_values_kernel<T, 2, 2>), dim3(grid), dim3(256), 0, stream, p);
    else if (p.rows == 128)
        hipLaunchKernelGGL((tile_values_kernel<T, 2, 1>), dim3(grid), dim3(128), 0, stream, p);
    else if (wide)
        hipLaunchKernelGGL((tile_values_kernel<T, 1, 2>), dim3(grid), dim3(128), 0, stream, p);
    else
        hipLaunchKernelGGL((tile_values_kernel<T, 1, 1>), dim3(grid), dim3(64), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_tile_scores(bool bf16, const AttentionParams &p, int units, hipStream_t stream) {
    if (bf16)
        return p.q_bf16 ? scores_launch<uint16_t, true>(p, units, stream) : scores_launch<uint16_t, false>(p, units, stream);
    return p.q_bf16 ? scores_launch<float, true>(p, units, stream) : scores_launch<float, false>(p, units, stream);
}

hipError_t launch_tile_values(bool bf16, const AttentionParams &p, int units, hipStream_t stream) {
    return bf16 ? values_launch<uint16_t>(p, units, stream) : values_launch<float>(p, units, stream);
}

}  // namespace pamk
