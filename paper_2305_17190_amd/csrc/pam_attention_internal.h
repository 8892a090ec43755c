// Internal interface between the host layer of the attention-side operators
// (pam_attention_api.cpp) and their HIP kernels (pam_heads.hip,
// pam_attention.hip).
#pragma once

#include <stdint.h>
#include <hip/hip_runtime_api.h>

namespace pamk {

// One operand of the head kernels: rows of d values at (token, head), written
// to a tensor or, paged, to the slots of a cache.
struct HeadPart {
    const void *in;
    void *out;
    const float *weight;            // norm's weight, or nullptr: no norm
    uint32_t in_token, in_head;     // strides, elements
    uint32_t out_token, out_head;   // out_token: stride of a page where paged
    uint32_t out_slot;              // paged: stride of a slot
    uint32_t heads, heads_mul, heads_shift;   // fast_divisor(heads)
    uint32_t first;                 // first workgroup of the part
    int32_t out_bf16;
    int32_t paged;
    int32_t rotate;
};

struct HeadRowsParams {
    HeadPart part[3];
    int32_t parts;
    int64_t tokens;
    int32_t d, rot, interleaved;
    float eps;
    const int32_t *positions;
    const float *cos, *sin;
    int64_t rows;                   // positions in the tables
    const int64_t *slots;
    int64_t cache_slots;            // pages * page_size
    uint32_t page_size, page_mul, page_shift;   // fast_divisor(page_size)
};

// n / divisor for n < 2^31 by a multiplication: (mulhi(n, mul) + n) >> shift, with
// 2^shift >= divisor and mul = 2^32 (2^shift - divisor) / divisor + 1.
inline void fast_divisor(uint32_t divisor, uint32_t &mul, uint32_t &shift) {
    shift = 0;
    while (((uint64_t)1 << shift) < divisor)
        ++shift;
    mul = (uint32_t)(((((uint64_t)1 << shift) - divisor) << 32) / divisor + 1);
}

// Norm and rotation of every part's rows, into tensors or cache slots.
// bf16: the inputs are bfloat16.
hipError_t launch_head_rows(bool bf16, const HeadRowsParams &p, hipStream_t stream);

struct HeadGradPart {
    const void *x, *dz;
    void *dx;
    const float *weight;
    float *dweight;
    float *partial;                 // [groups][d]
    uint32_t x_token, x_head, dz_token, dz_head, dx_token, dx_head;
    uint32_t heads, heads_mul, heads_shift;
    int32_t groups;                 // workgroups of this part
};

struct HeadGradParams {
    HeadGradPart part[2];
    int64_t tokens;
    int32_t d, rot, interleaved;
    float eps;
    const int32_t *positions;
    const float *cos, *sin;
    int64_t rows;
};

// About the most workgroups, and so rows of partial sums, of one gradient launch.
constexpr int kHeadGradGroups = 1024;
// How many workgroups `rows` rows keep busy, at most `most`.
int head_grad_groups(bool bf16, int64_t rows, int d, int rot, int most);
hipError_t launch_head_grad(bool bf16, const HeadGradParams &p, hipStream_t stream);

// Keys or values of a paged cache.
struct CacheView {
    const void *data;
    int64_t page, slot, head;       // strides, elements
    int64_t pages;
};

// One PAM attention call.  A unit is (sequence, key head, row block): the rows
// of a key head are its query heads of the sequence's new tokens, row =
// token * group + query head in the group, `rows` of them a unit.
struct AttentionParams {
    const void *q;
    int64_t q_token, q_head;
    int32_t q_bf16;
    CacheView k, v;
    uint32_t page_size, page_mul, page_shift;   // fast_divisor(page_size)
    const int32_t *q_starts, *kv_lens, *table;
    int64_t table_stride;
    float *out;
    int64_t out_token, out_head;
    int64_t tokens;
    int32_t batch, kv_heads, group, d;
    int32_t max_q, max_kv, causal, window;
    float scale;                    // times log2(e)
    int32_t rows, row_blocks;
    uint32_t blocks_mul, blocks_shift, heads_mul, heads_shift, group_mul, group_shift;   // fast_divisor of
                                    // row_blocks, kv_heads and group
    int32_t fine;                   // few rows: waves take 16 keys at a time, not 64
    int32_t first_unit;             // of this launch; workspaces count units from it
    int32_t splits, split_keys;     // keys of a unit: splits of split_keys (a multiple of 64)
    float *scores;                  // [unit][splits * split_keys][rows], in units of log2
    float *stats;                   // [unit][split, or tile of 128 keys][2][rows]: maximum, sum of 2^(score - maximum)
    float *partial;                 // [unit][split][rows][d], or nullptr: one split, straight to the output
};

// Few rows a unit (pam_attention.hip), `lanes` lanes a key: one launch with
// the scores in LDS, or two with the keys split, of `units` units from first_unit on.
// The one launch's waves: of 16 keys each (fine) or of 64; 16 at most with up to
// 4 rows (128 registers a lane), else 8.
constexpr int whole_most_waves(int rows) { return rows <= 4 ? 16 : 8; }
inline int whole_waves(int64_t max_kv, int rows, bool fine) {
    const int64_t waves = (max_kv + 63) / (fine ? 16 : 64);
    return waves < 4 ? 4 : waves < whole_most_waves(rows) ? (int)waves : whole_most_waves(rows);
}
// Its LDS bytes: the scores, and the keys that the waves work on or, afterwards,
// their outputs.
inline int64_t whole_lds(int64_t max_kv, int rows, int lanes, bool bf16, bool fine) {
    const int64_t waves = whole_waves(max_kv, rows, fine);
    const int64_t keys = 128 * (8 + 4 * rows), out = 4 * rows * lanes * (bf16 ? 8 : 4);
    return (4 * rows * max_kv + 15) / 16 * 16 + waves * (keys > out ? keys : out);
}
constexpr int64_t kWholeLds = 131072;   // at most
hipError_t launch_attention_whole(bool bf16, int lanes, const AttentionParams &p, hipStream_t stream);
hipError_t launch_attention_scores(bool bf16, int lanes, const AttentionParams &p, int units, hipStream_t stream);
hipError_t launch_attention_values(bool bf16, int lanes, const AttentionParams &p, int units, hipStream_t stream);
// Units of 64 or 128 rows (pam_attention_tile.hip); split_keys a multiple of 128.
hipError_t launch_tile_scores(bool bf16, const AttentionParams &p, int units, hipStream_t stream);
hipError_t launch_tile_values(bool bf16, const AttentionParams &p, int units, hipStream_t stream);
// The outputs as the sums of the splits' parts, in order.
hipError_t launch_attention_join(const AttentionParams &p, int units, hipStream_t stream);

}  // namespace pamk
