// PAM attention of few rows over a paged key/value cache for gfx950 (Kosson &
// Jaggi, Sec. 3.2: the attention's products Q K^T and P V are PAM products, the
// softmax between them is ordinary): single tokens, and the few tokens of a
// short chunk.
//
//   s_j = scale sum_i q_i .^ k_ji,  P_j = exp(s_j - max s) / sum exp(s - max s),
//   out_i = sum_j P_j .^ v_ji
//
// The sum of the exponentials is known before the second product: PAM
// commutes with powers of two only, so P V cannot be rescaled afterwards, and
// each unit of work (a key head of a sequence and up to 8 of its rows) first
// scores all its keys, then reads the values.
//
// A wave takes 64 keys at a time.  Lane i looks up key i's page; then every
// load of a wave fetches 64 / L whole keys, L neighbouring lanes 16 bytes each,
// so that a cache line is used by the lanes of one load, and all L loads of the
// 64 keys are on their way before the first is used.  Lanes past a head's end
// and keys that are none read something that is there instead, and count for
// nothing afterwards: a value of theirs, that of a key of the group itself, since
// its weight of zero would make NaN of an inf elsewhere.  Scores: a lane has the
// partial sums of its 16 bytes of each key; adding them up over the L lanes
// halves the number of sums a lane holds with each step (one half goes to the
// lane's partner, the other half comes), so that lane i ends with one key's
// whole sums after L - 1 additions a row instead of L log2 L.  Values: a lane
// keeps its 16 bytes' worth of outputs over all keys, the probabilities come
// from LDS, where lane i put key i's.
//
// Bound by memory for up to about 4 rows, by the vector ALU beyond: for each
// bfloat16 value read, 2 full-rate ops a row and 2.5 half-rate ones to take it
// apart.  128 sequences of up to 8192 keys, 8 heads of 128 x 4 rows, bfloat16 (2.66
// GB): 615 us, 4.3 TB/s (a 1 GiB copy: 5.1-5.2); one of 131071 keys (537 MB): 133 us,
// 4.0 TB/s.  64 sequences of 4096 keys, 8 heads of 128: with one row in float32 (2.15 GB)
// 348 us, 6.2 TB/s, in bfloat16 184 us, 5.8; with 8 rows 461 and 365 us, 4.7 and 2.9
// TB/s, 9.3 and 11.8 T PAM-MAC/s.  One of 1000 keys: 16.4 us, three launches of 7.5, 6
// and 3 us, each most of it the latency of its chain of loads.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pam_attention_device.h"

namespace pamk {
namespace {

constexpr int kThreads = 256;
constexpr int kMostWaves = 16;
// Keys a wave takes at a time: 64, or 16 in small problems, where more and
// shorter waves end sooner (F, for fine).
constexpr int kGroup = 64, kFineGroup = 16;
template <bool F> constexpr int group_keys() { return F ? kFineGroup : kGroup; }
constexpr int kLoads = 4;             // loads of a batch at most; a wave has one to two batches in flight

__device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }
__device__ __forceinline__ float real(uint32_t x) { return __uint_as_float(x); }

template <int CTRL> __device__ __forceinline__ float dpp(float x) {
    return real(__builtin_amdgcn_mov_dpp(bits(x), CTRL, 0xF, 0xF, false));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140, kRotate8 = 0x128;

// The sums of a (lanes with bit BIT of their number clear) and of b (set) over
// the two lanes of a pair.  Pairs differ in BIT, and in lower bits at will: the
// steps run from the highest bit down.
template <int BIT> __device__ __forceinline__ float merge(float a, float b, int lane) {
    if constexpr (BIT >= 4) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 s = BIT == 5 ? __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(bits(a), bits(b), false, false))
                                 : __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(bits(a), bits(b), false, false));
        return real(s.x) + real(s.y);
    } else {
        constexpr int ctrl = BIT == 3 ? kMirror : BIT == 2 ? kHalfMirror : BIT == 1 ? kXor2 : kXor1;
        const bool high = lane >> BIT & 1;
        return (high ? b : a) + dpp<ctrl>(high ? a : b);
    }
}

// Over the wave, in all lanes.
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, dpp<kXor1>(x));
    x = fmaxf(x, dpp<kXor2>(x));
    x = fmaxf(x, dpp<kHalfMirror>(x));
    x = fmaxf(x, dpp<kMirror>(x));
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp<kXor1>(x);
    x += dpp<kXor2>(x);
    x += dpp<kHalfMirror>(x);
    x += dpp<kMirror>(x);
    x = merge<4>(x, x, 0);
    return merge<5>(x, x, 0);
}

constexpr int log2_of(int x) { return x <= 1 ? 0 : 1 + log2_of(x / 2); }

// What a wave keeps in LDS of its 64 keys, and of the next 64.
template <int R> struct Area {
    int64_t from[2][kGroup];          // offsets in the cache; of something there where there is no key
    uint32_t pr[2][kGroup * R];       // probabilities, as b'
};

// A wave's loads of its keys, groups first, first + step, ... below end, in
// batches of B: while one batch is used the next is on its way, the next
// group's first at the end of a group, so that the memory always has work of
// the wave.  next(first) starts to fetch what the group from `first` on needs,
// keep(buffer) puts it where from(buffer, n) finds load n's offset; use(buffer,
// n, words) takes load n, done(buffer, first) closes a group; unless live(buffer),
// which is the same in all lanes, a group's loads go unused.
// begin() runs once the first loads are out.  Fine groups: all loads of a group
// at once, one group after the other.
template <typename T, int L, bool F, typename Next, typename Keep, typename From, typename Begin, typename Live,
          typename Use, typename Done>
__device__ __forceinline__ void stream_keys(const void *data, int first, int end, int step, Next next, Keep keep,
                                            From from, Begin begin, Live live, Use use, Done done) {
    constexpr int B = F ? L / 4 : L / 2 < kLoads ? L / 2 : kLoads;
    constexpr int N = L / B;
    if (first >= end)
        return;
    u32x4 w[2][B];
    next(first);
    keep(0);
#pragma unroll
    for (int u = 0; u < B; ++u)
        w[0][u] = load16<T>(data, from(0, u));
    begin();
    if constexpr (F) {
        for (;;) {
            if (live(0)) {
#pragma unroll
                for (int u = 0; u < B; ++u)
                    use(0, u, w[0][u]);
            }
            done(0, first);
            first += step;
            if (first >= end)
                return;
            next(first);
            keep(0);
#pragma unroll
            for (int u = 0; u < B; ++u)
                w[0][u] = load16<T>(data, from(0, u));
        }
    }
    for (int buffer = 0; first < end; first += step, buffer ^= 1) {
        next(first + step);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool last = i + 1 == N;
            if (last)
                keep(buffer ^ 1);
#pragma unroll
            for (int u = 0; u < B; ++u)
                w[(i + 1) & 1][u] = load16<T>(data, last ? from(buffer ^ 1, u) : from(buffer, (i + 1) * B + u));
            __builtin_amdgcn_sched_barrier(0);
            if (live(buffer)) {
#pragma unroll
                for (int u = 0; u < B; ++u)
                    use(buffer, i * B + u, w[i & 1][u]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        done(buffer, first);
    }
}

// A unit's rows: which keys they see, where their queries are.
template <int R> struct Rows {
    int lo[R], hi[R];
    __device__ __forceinline__ Rows(const AttentionParams &p, const Unit &unit) {
        const int lane = threadIdx.x & 63;
        const bool live = lane < unit.rows;
        const int low = live ? unit.row_lo(p, lane) : 0, high = live ? unit.row_hi(p, lane) : 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            lo[r] = __builtin_amdgcn_readlane(low, r);
            hi[r] = __builtin_amdgcn_readlane(high, r);
        }
    }
};

// Orders a wave's LDS writes before its other lanes' reads.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The b' of the rows' queries, E of them from element `at` on.
template <int E, int R>
__device__ __forceinline__ void load_queries(const AttentionParams &p, const Unit &unit, int at, uint32_t (&q)[R][E]) {
    const int lane = threadIdx.x & 63;
    const int64_t mine = lane < unit.rows ? unit.q_at(p, lane) : 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t from = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), r) << 32) |
                                       (uint32_t)__builtin_amdgcn_readlane((int)mine, r)) + at;
        u32x4 w[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
        if (r < unit.rows && at < p.d) {
            if (p.q_bf16) {
                typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
                if constexpr (E == 8) {
                    w[0] = load16<uint16_t>(p.q, from);
                } else {
                    const u32x2 h = *reinterpret_cast<const u32x2 *>(static_cast<const uint16_t *>(p.q) + from);
                    w[0].x = h.x;
                    w[0].y = h.y;
                }
            } else {
#pragma unroll
                for (int h = 0; h < E / 4; ++h)
                    w[h] = load16<float>(p.q, from + 4 * h);
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i)
            q[r][i] = biased(p.q_bf16 ? element<uint16_t>(w[0], i) : w[i / 4][i % 4]);
    }
}

// Scores, in units of log2, of the wave's keys first, first + step, ... below end, a group at a time:
// take(key, t) gets a key's scores, -inf
// where a row does not see it.
template <typename T, int L, int R, bool F, typename Take>
__device__ __forceinline__ void score_keys(const AttentionParams &p, const Unit &unit, int first, int end, int step,
                                           Area<R> &area, Take take) {
    constexpr int E = kPer<T>;
    constexpr int K = 64 / L;
    constexpr int S = log2_of(L), M = F ? S - 2 : S;   // steps, and those that merge; the others add to both sides
    constexpr int G = group_keys<F>();
    const int lane = threadIdx.x & 63;
    const int at = (lane % L) * E, reads = at < p.d ? at : 0;
    const Rows<R> rows(p, unit);
    uint32_t q[R][E];
    int64_t place = -1;
    uint64_t there[2] = {0, 0};
    float v[M + 1][R];
    stream_keys<T, L, F>(
        p.k.data, first, end, step,
        [&](int from) { place = lane < G && from + lane < end ? unit.key_at(p, p.k, from + lane) : -1; },
        [&](int buffer) {
            wave_sync();
            there[0] = there[1];
            there[1] = __ballot(place >= 0);
            area.from[buffer][lane] = place >= 0 ? place : 0;
            wave_sync();
        },
        [&](int buffer, int n) { return area.from[buffer][n * K + lane / L] + reads; },
        [&]() { load_queries<E, R>(p, unit, at, q); }, [](int) { return true; },
        [&](int, int n, const u32x4 &w) {
            float sum[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
                sum[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t a = element<T>(w, i);
                const float one = one_mantissa(a), m = power(a);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    sum[r] = pam_fma(one, m, q[r][i], sum[r]);
            }
            // Merge with the equal-sized sums before it: bit j of the load's
            // number goes with bit S - 1 - j of the lane's.
            int level = 0;
#pragma unroll
            for (int j = 0; j < M; ++j)
                level += (n & ((2 << j) - 1)) == (2 << j) - 1;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float x = sum[r];
                if constexpr (M > 0)
                    if (level > 0)
                        x = merge<S - 1>(v[0][r], x, lane);
                if constexpr (M > 1)
                    if (level > 1)
                        x = merge<S - 2>(v[1][r], x, lane);
                if constexpr (M > 2)
                    if (level > 2)
                        x = merge<S - 3>(v[2][r], x, lane);
                if constexpr (M > 3)
                    if (level > 3)
                        x = merge<S - 4>(v[3][r], x, lane);
                if constexpr (M > 4)
                    if (level > 4)
                        x = merge<S - 5>(v[4][r], x, lane);
                if constexpr (M > 5)
                    if (level > 5)
                        x = merge<0>(v[5][r], x, lane);
                v[level][r] = x;
            }
        },
        [&](int buffer, int from) {
            // The lane's own key: its number's bits from the loads' are the
            // lane's in reverse (four lanes with a key in fine groups).
            const int own = ((int)(__brev((uint32_t)(lane % L)) >> (32 - S)) & (G / K - 1)) * K + lane / L;
            const int key = from + own;
            const bool exists = there[F ? 1 : 0] >> own & 1;   // a group ahead where streamed
            float t[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float sum = v[M][r];
                if constexpr (F) {
                    sum += dpp<kXor2>(sum);
                    sum += dpp<kXor1>(sum);
                }
                const bool sees = exists && key >= rows.lo[r] && key < rows.hi[r];
                if (sees && !finite(sum)) {
                    sum = 0.0f;
                    const int64_t row = unit.q_at(p, r), k = area.from[buffer][own];
                    for (int i = 0; i < p.d; ++i)
                        sum += real(pam_full(load_bits(p.q, row + i, p.q_bf16), load_bits(p.k.data, k + i, sizeof(T) == 2)));
                }
                t[r] = sees ? sum * p.scale : kNegInf;
            }
            if (key < end && (!F || lane % 4 == 0))
                take(key, t);
        });
}

template <int R> __device__ __forceinline__ void put(float *to, const float (&t)[R]) {
    constexpr int W = R == 4 || R == 8 ? 4 : R % 2 == 0 ? 2 : 1;
    if constexpr (W == 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            to[r] = t[r];
    } else {
        typedef float vec __attribute__((ext_vector_type(W), aligned(4)));
#pragma unroll
        for (int r = 0; r < R; r += W) {
            vec v;
#pragma unroll
            for (int i = 0; i < W; ++i)
                v[i] = t[r + i];
            *reinterpret_cast<vec *>(to + r) = v;
        }
    }
}

template <int R> __device__ __forceinline__ void get(const float *from, float (&t)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r)
        t[r] = from[r];
}

// A running maximum and sum of 2^(t - maximum).
template <int R> struct Running {
    float m[R], l[R];
    __device__ __forceinline__ Running() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = kNegInf;
            l[r] = 0.0f;
        }
    }
    // Takes in `sum` with maximum `top`, row r; a NaN sum stays one.
    __device__ __forceinline__ void take(int r, float top, float sum) {
        const float to = fmaxf(m[r], top);
        l[r] = l[r] * exp2_from(m[r], to) + sum * exp2_from(top, to);
        m[r] = to;
    }
    __device__ __forceinline__ void score(const float (&t)[R]) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            take(r, t[r], 1.0f);
    }
    __device__ __forceinline__ void over_wave() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float to = wave_max(m[r]);
            l[r] = wave_sum(l[r] * exp2_from(m[r], to));
            m[r] = to;
        }
    }
    // Over the workgroup, in all lanes; scratch: two arrays of waves x R.
    __device__ __forceinline__ void over_group(float (&top)[kMostWaves][R], float (&sum)[kMostWaves][R]) {
        over_wave();
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                top[wave][r] = m[r];
                sum[wave][r] = l[r];
            }
        }
        __syncthreads();
        *this = Running();
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int r = 0; r < R; ++r)
                take(r, top[w][r], sum[w][r]);
    }
};

// out[row][i] = sum over keys begin <= j < end of P .^ v, the scores at
// scores[(j - origin) * R + row]; to out's rows (partial == nullptr) or
// partial[row * d + i].
template <typename T, int L, int R, bool F>
__device__ __forceinline__ void value_keys(const AttentionParams &p, const Unit &unit, int begin, int end,
                                           const float *scores, const Running<R> &row, Area<R> *areas, float *scratch,
                                           float *partial) {
    constexpr int E = kPer<T>;
    constexpr int K = 64 / L;
    constexpr int D = L * E;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int at = (lane % L) * E, reads = at < p.d ? at : 0;
    Area<R> &area = areas[wave];
    float inverse[R], acc[R][E];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        inverse[r] = row.l[r] > 0.0f ? 1.0f / row.l[r] : 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i)
            acc[r][i] = 0.0f;
    }
    int64_t place = -1;
    uint32_t live = 0;                 // bit `buffer`: its group has a key
    float t[R];
    constexpr int G = group_keys<F>();
    stream_keys<T, L, F>(
        p.v.data, begin + wave * G, end, waves * G,
        [&](int from) {
            const int mine = from + lane % G;
            place = mine < end ? unit.key_at(p, p.v, mine) : -1;
            get<R>(scores + (int64_t)(min(mine, end - 1) - begin) * R, t);
        },
        [&](int buffer) {
            wave_sync();
            const uint64_t there = __ballot(place >= 0);
            const int some = there != 0 ? __builtin_ctzll(there) : 0;
            const int64_t other = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(place >> 32), some) << 32 |
                                            (uint32_t)__builtin_amdgcn_readlane((int)place, some));
            live = (live & ~(1u << buffer)) | (there != 0 ? 1u << buffer : 0u);
            area.from[buffer][lane] = place >= 0 ? place : there != 0 ? other : 0;   // fine groups: four times over
#pragma unroll
            for (int r = 0; r < R; ++r)
                t[r] = real(probability(place >= 0 ? exp2_from(t[r], row.m[r]) : 0.0f, inverse[r]));
            put<R>(reinterpret_cast<float *>(area.pr[buffer]) + lane * R, t);
            wave_sync();
        },
        [&](int buffer, int n) { return area.from[buffer][n * K + lane / L] + reads; }, []() {},
        [&](int buffer) { return (live >> buffer & 1) != 0; },
        [&](int buffer, int n, const u32x4 &w) {
            float b[R];
            get<R>(reinterpret_cast<const float *>(area.pr[buffer]) + (n * K + lane / L) * R, b);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t a = element<T>(w, i);
                const float one = one_mantissa(a), m = power(a);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    acc[r][i] = pam_fma(one, m, bits(b[r]), acc[r][i]);
            }
        },
        [](int, int) {});
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (L <= 4)
                acc[r][i] += __shfl_xor(acc[r][i], 4);
            if constexpr (L <= 8)
                acc[r][i] += dpp<kRotate8>(acc[r][i]);
            if constexpr (L <= 16)
                acc[r][i] = merge<4>(acc[r][i], acc[r][i], lane);
            if constexpr (L <= 32)
                acc[r][i] = merge<5>(acc[r][i], acc[r][i], lane);
        }
    __syncthreads();                   // scratch may be where the areas are
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
        float m = 0.0f, l = 0.0f;
#pragma unroll
        for (int x = 0; x < R; ++x)
            if (x == r) {
                m = row.m[x];
                l = row.l[x];
            }
        float sum = 0.0f;
        for (int w = 0; w < waves; ++w)
            sum += scratch[w * R * D + e];
        if (!(l > 0.0f)) {                 // no weight, or a NaN score
            sum = l;
        } else if (!finite(sum)) {
            // Term by term, over the keys the row sees.
            sum = 0.0f;
            for (int key = max(begin, unit.row_lo(p, r)); key < min(end, unit.row_hi(p, r)); ++key) {
                const int64_t from = unit.key_at(p, p.v, key);
                if (from >= 0)
                    sum += real(pam_full(probability(exp2_from(scores[(int64_t)(key - begin) * R + r], m), 1.0f / l) + kBias,
                                         load_bits(p.v.data, from + i, sizeof(T) == 2)));
            }
        }
        if (partial != nullptr)
            partial[r * p.d + i] = sum;
        else
            p.out[unit.out_at(p, r) + i] = sum;
    }
}

// A unit in one workgroup: its scores stay in LDS, followed by what the waves
// keep of their keys and, in the same place, their outputs.
template <typename T, int L, int R, bool F>
__global__ void __launch_bounds__(whole_most_waves(R) * 64) attention_whole_kernel(const AttentionParams p) {
    extern __shared__ float4 lds[];
    __shared__ float top[kMostWaves][R], sum[kMostWaves][R];
    const Unit unit(p, blockIdx.x);
    if (unit.rows == 0)
        return;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    float *s = reinterpret_cast<float *>(lds), *after = reinterpret_cast<float *>(lds + (p.max_kv * R + 3) / 4);
    Area<R> *areas = reinterpret_cast<Area<R> *>(after);
    Running<R> row;
    constexpr int G = group_keys<F>();
    score_keys<T, L, R, F>(p, unit, unit.lo + wave * G, unit.hi, waves * G, areas[wave],
                        [&](int key, const float (&t)[R]) {
                            row.score(t);
                            put<R>(s + (key - unit.lo) * R, t);
                        });
    row.over_group(top, sum);
    value_keys<T, L, R, F>(p, unit, unit.lo, unit.hi, s, row, areas, after, nullptr);
}

// Consecutive workgroups, which go to the chip's eight dies in turn, take one
// split of consecutive units: with the splits of a unit in a row, sequences of
// different lengths left the dies of the last splits idle.
//
// Long contexts, first launch: scores of one split of a unit's keys, with the
// split's maximum and sum for each row.
template <typename T, int L, int R, bool F>
__global__ void __launch_bounds__(kThreads) attention_scores_kernel(const AttentionParams p) {
    __shared__ Area<R> areas[kThreads / 64];
    __shared__ float top[kMostWaves][R], sum[kMostWaves][R];
    const int units = gridDim.x / p.splits, split = blockIdx.x / units, index = blockIdx.x - split * units;
    const Unit unit(p, p.first_unit + index);
    const int begin = max(unit.lo, split * p.split_keys), end = min(unit.hi, (split + 1) * p.split_keys);
    if (unit.rows == 0 || begin >= end)
        return;
    const int wave = threadIdx.x >> 6;
    Running<R> row;
    float *scores = p.scores + (int64_t)index * p.splits * p.split_keys * R;
    constexpr int G = group_keys<F>();
    score_keys<T, L, R, F>(p, unit, begin + wave * G, end, kThreads / 64 * G, areas[wave],
                        [&](int key, const float (&t)[R]) {
                            row.score(t);
                            put<R>(scores + (int64_t)key * R, t);
                        });
    row.over_group(top, sum);
    if (threadIdx.x == 0) {
        float *stats = p.stats + ((int64_t)index * p.splits + split) * 2 * R;
        put<R>(stats, row.m);
        put<R>(stats + R, row.l);
    }
}

// Second launch: the unit's maxima and sums from all its splits', then one
// split's part of P V.
template <typename T, int L, int R, bool F>
__global__ void __launch_bounds__(kThreads) attention_values_kernel(const AttentionParams p) {
    __shared__ Area<R> areas[kThreads / 64];
    __shared__ float scratch[kThreads / 64 * R * L * kPer<T>];
    const int units = gridDim.x / p.splits, split = blockIdx.x / units, index = blockIdx.x - split * units;
    const Unit unit(p, p.first_unit + index);
    const int begin = max(unit.lo, split * p.split_keys), end = min(unit.hi, (split + 1) * p.split_keys);
    if (unit.rows == 0 || begin >= end)
        return;
    const int first = unit.lo / p.split_keys, last = (unit.hi - 1) / p.split_keys;
    const float *stats = p.stats + (int64_t)index * p.splits * 2 * R;
    Running<R> row;
    for (int j = first + (threadIdx.x & 63); j <= last; j += 64) {
        float m[R], l[R];
        get<R>(stats + j * 2 * R, m);
        get<R>(stats + j * 2 * R + R, l);
#pragma unroll
        for (int r = 0; r < R; ++r)
            row.take(r, m[r], l[r]);
    }
    row.over_wave();
    value_keys<T, L, R, F>(p, unit, begin, end, p.scores + ((int64_t)index * p.splits * p.split_keys + begin) * R, row,
                        areas, scratch, p.partial + ((int64_t)index * p.splits + split) * R * p.d);
}

// Third launch: the outputs, each the sum over its unit's splits; four a thread.
// GROUPS threads share an output's splits, each in order, then their sums in
// order.
template <int GROUPS>
__global__ void __launch_bounds__(kThreads) attention_join_kernel(const AttentionParams p, int parts) {
    constexpr int items = kThreads / GROUPS;
    __shared__ f32x4 sums[GROUPS][items];
    const int index = blockIdx.x / parts;
    const Unit unit(p, p.first_unit + index);
    const int item = threadIdx.x % items, group = threadIdx.x / items;
    const int e = ((blockIdx.x % parts) * items + item) * 4;
    const bool live = e < unit.rows * p.d;
    const int first = unit.lo / p.split_keys, last = unit.hi > unit.lo ? (unit.hi - 1) / p.split_keys : first - 1;
    const int64_t step = (int64_t)p.rows * p.d;
    const float *partial = p.partial + (int64_t)index * p.splits * step + e;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (live)
#pragma unroll 4
        for (int j = first + group; j <= last; j += GROUPS)
            sum += *reinterpret_cast<const f32x4 *>(partial + j * step);
    if constexpr (GROUPS > 1) {
        sums[group][item] = sum;
        __syncthreads();
        if (group > 0)
            return;
        for (int g = 1; g < GROUPS; ++g)
            sum += sums[g][item];
    }
    if (live) {
        const int r = e / p.d;
        *reinterpret_cast<f32x4 *>(p.out + unit.out_at(p, r) + (e - r * p.d)) = sum;
    }
}

enum Which { kWhole, kScores, kValues };

template <typename T, int L, int R, bool F>
hipError_t launch(Which which, const AttentionParams &p, int units, hipStream_t stream) {
    const void *kernel = which == kWhole    ? (const void *)attention_whole_kernel<T, L, R, F>
                         : which == kScores ? (const void *)attention_scores_kernel<T, L, R, F>
                                            : (const void *)attention_values_kernel<T, L, R, F>;
    const int threads = which == kWhole ? whole_waves(p.max_kv, R, F) * 64 : kThreads;
    const size_t lds = which == kWhole ? (size_t)whole_lds(p.max_kv, R, L, sizeof(T) == 2, F) : 0;
    const unsigned grid = (unsigned)units * (which == kWhole ? 1u : (unsigned)p.splits);
    void *args[] = {const_cast<AttentionParams *>(&p)};
    return hipLaunchKernel(kernel, dim3(grid), dim3((unsigned)threads), args, lds, stream);
}

template <typename T, int L, bool F> hipError_t for_rows(Which which, const AttentionParams &p, int units, hipStream_t stream) {
    switch (p.rows) {
    case 1: return launch<T, L, 1, F>(which, p, units, stream);
    case 2: return launch<T, L, 2, F>(which, p, units, stream);
    case 3: return launch<T, L, 3, F>(which, p, units, stream);
    case 4: return launch<T, L, 4, F>(which, p, units, stream);
    case 6: return launch<T, L, 6, F>(which, p, units, stream);
    default: return launch<T, L, 8, F>(which, p, units, stream);
    }
}

template <typename T, int L> hipError_t for_group(Which which, const AttentionParams &p, int units, hipStream_t stream) {
    return p.fine ? for_rows<T, L, true>(which, p, units, stream) : for_rows<T, L, false>(which, p, units, stream);
}

hipError_t for_type(Which which, bool bf16, int lanes, const AttentionParams &p, int units, hipStream_t stream) {
    switch (lanes) {
    case 4: return bf16 ? for_group<uint16_t, 4>(which, p, units, stream) : for_group<float, 4>(which, p, units, stream);
    case 8: return bf16 ? for_group<uint16_t, 8>(which, p, units, stream) : for_group<float, 8>(which, p, units, stream);
    case 16: return bf16 ? for_group<uint16_t, 16>(which, p, units, stream) : for_group<float, 16>(which, p, units, stream);
    case 32: return bf16 ? for_group<uint16_t, 32>(which, p, units, stream) : for_group<float, 32>(which, p, units, stream);
    default: return for_group<float, 64>(which, p, units, stream);
    }
}

}  // namespace

hipError_t launch_attention_whole(bool bf16, int lanes, const AttentionParams &p, hipStream_t stream) {
    return for_type(kWhole, bf16, lanes, p, p.batch * p.kv_heads * p.row_blocks, stream);
}

hipError_t launch_attention_scores(bool bf16, int lanes, const AttentionParams &p, int units, hipStream_t stream) {
    return for_type(kScores, bf16, lanes, p, units, stream);
}

hipError_t launch_attention_values(bool bf16, int lanes, const AttentionParams &p, int units, hipStream_t stream) {
    return for_type(kValues, bf16, lanes, p, units, stream);
}

hipError_t launch_attention_join(const AttentionParams &p, int units, hipStream_t stream) {
    // Many splits of few outputs: 16 threads an output (131071 keys, 8 units of 4 rows
    // of 128: 132 us the call, with one thread 139; 128 sequences of 8192 keys, 1024
    // such units: 934 with 16, 924 with one).
    const bool shared = p.splits > 8 && (int64_t)units * p.rows * p.d <= 1 << 17;
    const int items = shared ? kThreads / 16 : kThreads;
    const int parts = (p.rows * p.d / 4 + items - 1) / items;
    if (shared)
        hipLaunchKernelGGL(attention_join_kernel<16>, dim3((unsigned)(units * parts)), dim3(kThreads), 0, stream, p, parts);
    else
        hipLaunchKernelGGL(attention_join_kernel<1>, dim3((unsigned)(units * parts)), dim3(kThreads), 0, stream, p, parts);
    return hipGetLastError();
}

}  // namespace pamk
