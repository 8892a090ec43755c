// PAM attention of many rows over a paged cache for gfx950: the two products
// as tiles on the vector ALU (PAM has no use for the matrix cores), with the
// scores between them in a workspace.
//
// A unit is 64 WM rows of one key head (its query heads times the new tokens);
// a wave owns a 64 x 64 block of outputs, a lane 8 x 8 of them.  Both operands
// are staged into LDS a chunk of 16 k steps at a time, k-major, while the next
// chunk is on its way into registers: keys or values as they are, queries or
// probabilities less one bias.  Where no element of a chunk is zero, tiny or
// huge, a term is two additions, one of integers and one of floats; else the
// chunk's terms take the form of pam_attention_device.h, an integer addition and
// a float fma, with 1 + M and the power of two taken apart each k step.
//
// Scores first: a tile of 64 WM rows and 64 WN keys goes to the workspace
// key-major, with each row's maximum and sum of exponentials over the tile;
// the tile of the values then reads the row's statistics over all keys, turns
// scores into normalised probabilities as it stages them, and adds up its
// split's keys.  Storing a score costs 8 bytes of traffic, scoring again d
// PAM-MACs, which take several times as long.
//
// Bound by the vector ALU: 2 lane-ops a PAM-MAC, issued in pairs from four waves a
// SIMD.  512 tokens x 32 heads of 128 over 4096 keys (8 key heads, bfloat16): 660
// to 684 us by card, 24 T PAM-MAC/s, 25 T without the join's 22 us (the framework's
// matrix product on such operands: 30.8 T); the causal mask cuts 1% off what the
// tiles compute.

#include "pam_attention_device.h"

namespace pamk {
namespace {

constexpr int kStep = 16;             // k steps of a chunk
constexpr int kPad = 4;               // words after each k step's row in LDS

// A lane's 8 rows or columns of a 64-wide block: two groups of four.
__device__ __forceinline__ int place(int group, int i) { return (i / 4) * 32 + group * 4 + i % 4; }

// One row of two k steps, four columns; equal instructions stand together, so
// that neighbours are independent and pair up with another wave's.  Plain: all
// encodings' exponent fields lie in [64, 190], so a + b' is the encoding of their
// PAM itself.  The two steps' terms are added to each other first: no instruction
// more, and half as many roundings of the long sum.
__device__ __forceinline__ void plain_pair(float &c0, float &c1, float &c2, float &c3, uint32_t b, uint32_t d,
                                           const uint32_t (&a)[4], const uint32_t (&e)[4]) {
    uint32_t t0, t1, t2, t3, u0, u1, u2, u3;
    asm("v_add_u32 %[t0], %[a0], %[b]\n\tv_add_u32 %[t1], %[a1], %[b]\n\t"
        "v_add_u32 %[t2], %[a2], %[b]\n\tv_add_u32 %[t3], %[a3], %[b]\n\t"
        "v_add_u32 %[u0], %[e0], %[d]\n\tv_add_u32 %[u1], %[e1], %[d]\n\t"
        "v_add_u32 %[u2], %[e2], %[d]\n\tv_add_u32 %[u3], %[e3], %[d]\n\t"
        "v_add_f32 %[t0], %[t0], %[u0]\n\tv_add_f32 %[t1], %[t1], %[u1]\n\t"
        "v_add_f32 %[t2], %[t2], %[u2]\n\tv_add_f32 %[t3], %[t3], %[u3]\n\t"
        "v_add_f32 %[c0], %[c0], %[t0]\n\tv_add_f32 %[c1], %[c1], %[t1]\n\t"
        "v_add_f32 %[c2], %[c2], %[t2]\n\tv_add_f32 %[c3], %[c3], %[t3]"
        : [c0] "+v"(c0), [c1] "+v"(c1), [c2] "+v"(c2), [c3] "+v"(c3), [t0] "=&v"(t0), [t1] "=&v"(t1), [t2] "=&v"(t2),
          [t3] "=&v"(t3), [u0] "=&v"(u0), [u1] "=&v"(u1), [u2] "=&v"(u2), [u3] "=&v"(u3)
        : [b] "v"(b), [d] "v"(d), [a0] "v"(a[0]), [a1] "v"(a[1]), [a2] "v"(a[2]), [a3] "v"(a[3]), [e0] "v"(e[0]),
          [e1] "v"(e[1]), [e2] "v"(e[2]), [e3] "v"(e[3]));
}

// acc[r][c] += b[k][row r] .^ a[k][column c] over one chunk in LDS: `plain` or,
// for any values, with 1 + M and the power of two taken apart here.
// FIX: b' is an encoding less the bias of any value, zeros and NaN among them.
template <int BM, int BN, bool FIX>
__device__ __forceinline__ void chunk_product(const uint32_t *a, const uint32_t *b, int row, int col, bool plain,
                                              float (&acc)[8][8]) {
    auto read = [](const uint32_t *from, uint32_t (&x)[8]) {
        *reinterpret_cast<uint4 *>(x) = *reinterpret_cast<const uint4 *>(from);
        *reinterpret_cast<uint4 *>(x + 4) = *reinterpret_cast<const uint4 *>(from + 32);
    };
    // Two loops one after the other, of which one runs, by a count the compiler
    // cannot see through: as two branches the sums would be copied where they
    // meet, in 64 more registers.
    int first = __builtin_amdgcn_readfirstlane(plain ? kStep : 0);
    asm("" : "+s"(first));
    for (int k = 0; k < first; k += 2) {
        uint32_t z[2][8];
        read(b + k * (BM + kPad) + row, z[0]);
        read(b + (k + 1) * (BM + kPad) + row, z[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t x[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<uint4 *>(x[i]) = *reinterpret_cast<const uint4 *>(a + (k + i) * (BN + kPad) + col + 32 * h);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                plain_pair(acc[r][4 * h], acc[r][4 * h + 1], acc[r][4 * h + 2], acc[r][4 * h + 3], z[0][r], z[1][r], x[0], x[1]);
        }
    }
#pragma unroll 1
    for (int k = first; k < kStep; ++k) {
        uint32_t x[8], z[8];
        read(a + k * (BN + kPad) + col, x);
        read(b + k * (BM + kPad) + row, z);
        if constexpr (FIX) {
#pragma unroll
            for (int r = 0; r < 8; ++r)
                z[r] = biased(z[r] + kBias);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float one = one_mantissa(x[c]), m = power(x[c]);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                acc[r][c] = pam_fma(one, m, z[r], acc[r][c]);
        }
    }
}

// Keeps track of whether an encoding's exponent field is outside [64, 190]: the
// largest of 2 |x| - 2 * 2^(64 - 127)'s encoding, below which all are inside.
struct Odd {
    uint32_t most = 0, most16 = 0;
    __device__ __forceinline__ void take(uint32_t x, uint32_t y) {
        const uint32_t u = (x << 1) - (64u << 24), v = (y << 1) - (64u << 24);
        most = max(max(most, u), v);
    }
    // Two bfloat16 values in one word.
    __device__ __forceinline__ void take16(uint32_t w) {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        const u16x2 u = __builtin_bit_cast(u16x2, w) * (uint16_t)2 - (uint16_t)(64u << 8);
        most16 = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, most16), u));
    }
    __device__ __forceinline__ bool any() const {
        return most >= (127u << 24) || (most16 & 0xFFFFu) >= (127u << 8) || (most16 >> 16) >= (127u << 8);
    }
};

// The sum or maximum over the 8 lanes that share a lane's rows.
__device__ __forceinline__ float eight_max(float x) {
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xB1, 0xF, 0xF, false)));   // lane ^ 1
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x4E, 0xF, 0xF, false)));   // lane ^ 2
    return fmaxf(x, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x141, 0xF, 0xF, false)));   // 7 - lane
}
__device__ __forceinline__ float eight_sum(float x) {
    x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xB1, 0xF, 0xF, false));
    x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x4E, 0xF, 0xF, false));
    return x + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x141, 0xF, 0xF, false));
}

// The chunks' staging: two buffers in turn, or one with a second barrier a chunk;
// and for each chunk a word that says whether an element of it keeps it from the
// plain form, four of them, so that one is cleared two chunks before it is
// written.
template <int BM, int BN, int COUNT> struct Buffers {
    static constexpr int kCount = COUNT;
    uint32_t a[kCount][kStep * (BN + kPad)];
    uint32_t b[kCount][kStep * (BM + kPad)];
    uint32_t odd[4];
};

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
    // All eight as ones.
    __device__ __forceinline__ void ones(bool bf16) {
        const uint32_t one = bf16 ? kBias >> 16 | kBias : kBias;
        w[0] = w[1] = u32x4{one, one, one, one};
    }
    __device__ __forceinline__ void check(Odd &odd, bool bf16) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (bf16)
                odd.take16(w[0][i]);
            else
                odd.take(w[i / 2][i % 2 * 2], w[i / 2][i % 2 * 2 + 1]);
    }
};

template <typename T, int WM, int WN, bool QB>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(4, 4))) tile_scores_kernel(const AttentionParams p) {
    constexpr int BM = 64 * WM, BN = 64 * WN, NT = 64 * WM * WN;
    constexpr int KI = 2 / WM > 0 ? 2 / WM : 1;    // key items of 8 values a lane and chunk
    constexpr int QI = 2 / WN > 0 ? 2 / WN : 1;    // query items
    constexpr bool KB = sizeof(T) == 2;
    // One buffer lets a compute unit hold 16 waves of the small workgroups (many
    // 64-row tiles of 128 values a head: 447 -> 373 us with one).
    __shared__ Buffers<BM, BN, WM == 2 ? 2 : 1> buf;
    __shared__ int lo[BM], hi[BM];
    __shared__ int valid[BN];
    __shared__ float across[2][WN][BM];

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
    // Keys that every row sees, page permitting.
    const int most_lo = unit.rows == BM ? unit.row_lo(p, BM - 1) : p.max_kv, least_hi = unit.row_hi(p, 0);
    // The lane's keys and queries: one row each for all chunks.
    int64_t k_from[KI], q_from[QI];
    bool missing = false;
#pragma unroll
    for (int i = 0; i < KI; ++i) {
        const int item = tid + i * NT, j = item % BN, key = begin + j;
        k_from[i] = key >= unit.lo && key < unit.hi ? unit.key_at(p, p.k, key) : -1;
        if (item / BN == 0)
            valid[j] = k_from[i] >= 0;
        missing = missing || k_from[i] < 0;
    }
    const bool none_missing = !__syncthreads_or(missing);
#pragma unroll
    for (int i = 0; i < QI; ++i) {
        const int r = (tid + i * NT) % BM;
        q_from[i] = r < unit.rows ? unit.q_at(p, r) : -1;
    }

    // Keys and rows that do not exist hold ones: nothing of them is kept, and
    // the chunk stays plain.
    Eight kw[KI], qw[QI];
    auto fetch = [&](int d0) {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int at = d0 + (tid + i * NT) / BN * 8;
            if (k_from[i] < 0)
                kw[i].ones(KB);
            else if (at < p.d)
                kw[i].load(p.k.data, k_from[i] + at, KB);
            else
                kw[i].clear();
        }
#pragma unroll
        for (int i = 0; i < QI; ++i) {
            const int at = d0 + (tid + i * NT) / BM * 8;
            if (q_from[i] < 0)
                qw[i].ones(QB);
            else if (at < p.d)
                qw[i].load(p.q, q_from[i] + at, QB);
            else
                qw[i].clear();
        }
    };
    auto stage = [&](int chunk) {
        uint32_t *a = buf.a[chunk % buf.kCount], *b = buf.b[chunk % buf.kCount];
        Odd odd;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int item = tid + i * NT, j = item % BN, k = item / BN * 8;
            kw[i].check(odd, KB);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                a[(k + e) * (BN + kPad) + j] = kw[i](e, KB);
        }
#pragma unroll
        for (int i = 0; i < QI; ++i) {
            const int item = tid + i * NT, r = item % BM, k = item / BM * 8;
            qw[i].check(odd, QB);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                b[(k + e) * (BM + kPad) + r] = qw[i](e, QB) - kBias;
        }
        if (odd.any())
            buf.odd[chunk & 3] = 1;
    };

    float acc[8][8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c)
            acc[r][c] = 0.0f;
    if (tid < 4)
        buf.odd[tid] = 0;
    fetch(0);
    __syncthreads();
    stage(0);
    const int chunks = (p.d + kStep - 1) / kStep;
    for (int c = 0; c < chunks; ++c) {
        if (c + 1 < chunks)
            fetch((c + 1) * kStep);
        __syncthreads();
        if (tid == 0)
            buf.odd[(c + 2) & 3] = 0;
        chunk_product<BM, BN, true>(buf.a[c % buf.kCount], buf.b[c % buf.kCount], row0, col0, buf.odd[c & 3] == 0, acc);
        if (c + 1 < chunks) {
            if (buf.kCount == 1)
                __syncthreads();
            stage(c + 1);
        }
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

    // Scaled scores, -inf where the row does not see the key and 0 in rows that
    // do not exist; the rows' maxima and sums.
    float *scores = p.scores + ((int64_t)index * tiles * BN + begin) * BM;
    float best[8], sum[8];
    const bool inside = begin >= most_lo && begin + BN <= least_hi && none_missing;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        best[r] = kNegInf;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            acc[r][c] *= p.scale;
    }
    if (!inside) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const int row = row0 + place(0, r);
            const int low = lo[row] - begin, high = hi[row] - begin;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const int j = col0 + place(0, c);
                acc[r][c] = row >= unit.rows ? 0.0f : valid[j] && j >= low && j < high ? acc[r][c] : kNegInf;
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            best[r] = fmaxf(best[r], acc[r][c]);
        best[r] = eight_max(best[r]);
        if (tx == 0)
            across[0][wave / WM][row0 + place(0, r)] = best[r];
    }
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<float4 *>(scores + (int64_t)(col0 + place(0, c)) * BM + row0 + 32 * h) =
                make_float4(acc[4 * h][c], acc[4 * h + 1][c], acc[4 * h + 2][c], acc[4 * h + 3][c]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int row = row0 + place(0, r);
#pragma unroll
        for (int w = 0; w < WN; ++w)
            best[r] = fmaxf(best[r], across[0][w][row]);
        const float m = best[r] == kNegInf ? 0.0f : best[r];
        sum[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            sum[r] += __builtin_amdgcn_exp2f(acc[r][c] - m);
        sum[r] = eight_sum(sum[r]);
        if (tx == 0)
            across[1][wave / WM][row] = sum[r];
    }
    __syncthreads();
    float *stats = p.stats + ((int64_t)index * tiles + tile) * 2 * BM;
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (tx == 0 && wave / WM == 0) {
            const int row = row0 + place(0, r);
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < WN; ++w)
                total += across[1][w][row];
            stats[row] = best[r];
            stats[BM + row] = total;
        }
}

template <typename T, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(WM * WN == 1 ? 2 : 4, WM * WN == 1 ? 2 : 4))) tile_values_kernel(const AttentionParams p) {
    constexpr int BM = 64 * WM, BN = 64 * WN, NT = 64 * WM * WN;
    constexpr int E = kPer<T>;
    constexpr int SI = kStep * BM / 4 / NT;        // score items of 4 rows a lane and chunk
    constexpr int VI = kStep * BN / E / NT;        // value items of 16 bytes
    constexpr int SK = NT / (BM / 4);              // keys between a lane's score items
    constexpr int VK = NT / (BN / E);              // and between its value items
    constexpr bool VB = sizeof(T) == 2;
    __shared__ Buffers<BM, BN, 2> buf;
    __shared__ float row_max[BM], row_sum[BM], row_inverse[BM];
    extern __shared__ int64_t from[];              // the split's keys, -1: none

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
    {
        // WN lanes a row, each every WN-th tile, joined through LDS.
        const int r = tid % BM, part = tid / BM;
        float m = kNegInf, l = 0.0f;
#pragma unroll 4
        for (int t = first + part; t <= last; t += WN) {
            const float top = stats[(int64_t)t * 2 * BM + r], sum = stats[(int64_t)t * 2 * BM + BM + r];
            const float to = fmaxf(m, top);
            l = l * exp2_from(m, to) + sum * exp2_from(top, to);
            m = to;
        }
        if (part > 0) {
            row_max[r] = m;
            row_sum[r] = l;
        }
        __syncthreads();
        if (part == 0) {
            if constexpr (WN == 2) {
                const float to = fmaxf(m, row_max[r]);
                l = l * exp2_from(m, to) + row_sum[r] * exp2_from(row_max[r], to);
                m = to;
            }
            row_max[r] = m == kNegInf ? 0.0f : m;
            row_sum[r] = l;
            row_inverse[r] = r >= unit.rows ? 1.0f : l > 0.0f ? 1.0f / l : 0.0f;
        }
    }
    const int start = begin / kStep * kStep;
    for (int j = tid; j < p.split_keys; j += NT) {
        const int key = start + j;
        from[j] = key >= begin && key < end ? unit.key_at(p, p.v, key) : -1;
    }
    if (tid < 4)
        buf.odd[tid] = 0;
    __syncthreads();
    const int my_row = tid % (BM / 4) * 4;
    const float *scores = p.scores + (int64_t)index * tiles * kTile * BM;
    const int col = tid % (BN / E) * E, column = col_tile * BN + col;
    // Columns that do not exist hold ones, as rows do.
    const uint32_t none = column < p.d ? 0u : VB ? kBias >> 16 | kBias : kBias;
    float4 sw[SI];
    u32x4 vw[VI];
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < SI; ++i)
            sw[i] = *reinterpret_cast<const float4 *>(scores + (int64_t)(k0 + tid / (BM / 4) + i * SK) * BM + my_row);
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int64_t at = from[k0 - start + tid / (BN / E) + i * VK];
            if (at >= 0 && column < p.d)
                vw[i] = load16<T>(p.v.data, at + column);
            else
                vw[i] = u32x4{none, none, none, none};
        }
    };
    // Scores outside the split's keys are -inf, those of rows that do not exist
    // 0: probabilities 0 and 1.  A NaN row's probabilities are anything.
    auto stage = [&](int chunk) {
        uint32_t *a = buf.a[chunk % buf.kCount], *b = buf.b[chunk % buf.kCount];
        Odd odd;
        float least = 1.0f;
        const float4 m4 = *reinterpret_cast<const float4 *>(row_max + my_row);
        const float4 inverse4 = *reinterpret_cast<const float4 *>(row_inverse + my_row);
        const float top[4] = {m4.x, m4.y, m4.z, m4.w}, inverse[4] = {inverse4.x, inverse4.y, inverse4.z, inverse4.w};
#pragma unroll
        for (int i = 0; i < SI; ++i) {
            const int k = tid / (BM / 4) + i * SK;
            const float t[4] = {sw[i].x, sw[i].y, sw[i].z, sw[i].w};
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float pr = __builtin_amdgcn_exp2f(t[e] - top[e]) * inverse[e];
                least = fminf(least, pr);
                x[e] = __float_as_uint(pr) - kBias;
            }
            *reinterpret_cast<uint4 *>(b + k * (BM + kPad) + my_row) = make_uint4(x[0], x[1], x[2], x[3]);
        }
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int at = (tid / (BN / E) + i * VK) * (BN + kPad) + col;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (VB)
                    odd.take16(vw[i][e]);
                else if (e % 2 == 0)
                    odd.take(vw[i][e], vw[i][e + 1]);
#pragma unroll
            for (int e = 0; e < E; e += 4)
                *reinterpret_cast<uint4 *>(a + at + e) =
                    make_uint4(element<T>(vw[i], e), element<T>(vw[i], e + 1), element<T>(vw[i], e + 2),
                               element<T>(vw[i], e + 3));
        }
        if (odd.any() || least < 0x1p-63f)
            buf.odd[chunk & 3] = 1;
    };

    float acc[8][8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c)
            acc[r][c] = 0.0f;
    const int chunks = begin < end ? (end - start + kStep - 1) / kStep : 0;
    if (chunks > 0) {
        fetch(start);
        stage(0);
    }
    for (int c = 0; c < chunks; ++c) {
        if (c + 1 < chunks)
            fetch(start + (c + 1) * kStep);
        __syncthreads();
        if (tid == 0)
            buf.odd[(c + 2) & 3] = 0;
        chunk_product<BM, BN, false>(buf.a[c % buf.kCount], buf.b[c % buf.kCount], row0, col0, buf.odd[c & 3] == 0, acc);
        if (c + 1 < chunks) {
            if (buf.kCount == 1)
                __syncthreads();
            stage(c + 1);
        }
    }

    if (!all_finite(acc))
        sum_again(acc, [&](int r, int c, float value) {
            const int row = row0 + place(0, r), i = col_tile * BN + col0 + place(0, c);
            if (row >= unit.rows || i >= p.d || !(row_sum[row] > 0.0f))
                return value;
            const float m = row_max[row], inverse = 1.0f / row_sum[row];
            float sum = 0.0f;
            for (int key = max(begin, unit.row_lo(p, row)); key < min(end, unit.row_hi(p, row)); ++key) {
                const int64_t at = from[key - start];
                if (at < 0)
                    continue;
                const uint32_t b = probability(exp2_from(scores[(int64_t)key * BM + row], m), inverse);
                sum += __uint_as_float(pam_full(b + kBias, load_bits(p.v.data, at + i, VB)));
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
            f32x4 v = {acc[r][4 * h], acc[r][4 * h + 1], acc[r][4 * h + 2], acc[r][4 * h + 3]};
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
    const size_t keys = (size_t)p.split_keys * sizeof(int64_t);
    const unsigned grid = (unsigned)(units * p.splits * (wide ? (p.d + 127) / 128 : 1));
    if (p.rows == 128 && wide)
        hipLaunchKernelGGL((tile_values_kernel<T, 2, 2>), dim3(grid), dim3(256), keys, stream, p);
    else if (p.rows == 128)
        hipLaunchKernelGGL((tile_values_kernel<T, 2, 1>), dim3(grid), dim3(128), keys, stream, p);
    else if (wide)
        hipLaunchKernelGGL((tile_values_kernel<T, 1, 2>), dim3(grid), dim3(128), keys, stream, p);
    else
        hipLaunchKernelGGL((tile_values_kernel<T, 1, 1>), dim3(grid), dim3(64), keys, stream, p);
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
