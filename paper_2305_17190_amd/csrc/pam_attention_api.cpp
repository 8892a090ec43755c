// C ABI of the attention-side operators (pam_attention.h): argument
// validation, the cut of an attention call into launches, workspaces.  The
// arithmetic lives in pam_heads.hip and pam_attention.hip.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "pam_attention.h"
#include "pam_attention_internal.h"
#include "pam_internal.h"

namespace {

using pamk::api_check_device;
using pamk::api_fail;
using pamk::api_fail_hip;

pam_status_t invalid(const char *why) { return api_fail(PAM_ERROR_INVALID_VALUE, why); }

pam_status_t invalid(const char *name, const char *why) {
    char buf[160];
    snprintf(buf, sizeof buf, "%s%s", name, why);
    return invalid(buf);
}

#define PAM_TRY(call)                                       \
    do {                                                    \
        if (pam_status_t st_ = (call); st_ != PAM_SUCCESS)  \
            return st_;                                     \
    } while (0)

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kMaxRows = 0x7FFFFFFF;         // slots of a cache, positions of a table
constexpr int64_t kMaxHeadRows = (int64_t)1 << 25;  // a launch of them, 4 a workgroup, stays below 2^32 threads
constexpr int64_t kMaxStride = (int64_t)1 << 31; // times a count below 2^31: offsets stay inside int64
constexpr int64_t kMaxLaunchThreads = ((int64_t)1 << 32) - 1;
constexpr int64_t kMaxLaunchGroups = kMaxLaunchThreads / 256;

bool is_bf16(pam_type_t t) { return t == PAM_TYPE_BF16; }

pam_status_t check_heads(const void *data, const pam_heads_t &h, const char *name, int64_t tokens) {
    if (h.type != PAM_TYPE_F32 && h.type != PAM_TYPE_BF16)
        return invalid(name, ": type must be PAM_TYPE_F32 or PAM_TYPE_BF16");
    if (h.heads < 1)
        return invalid(name, ": heads must be at least 1");
    if (h.stride_token < 0 || h.stride_head < 0 || h.stride_token > kMaxStride || h.stride_head > kMaxStride)
        return invalid(name, ": strides must be in [0, 2^31]");
    if (tokens > 0 && data == nullptr)
        return invalid(name, ": data is NULL");
    return PAM_SUCCESS;
}

struct Dim {
    int64_t count, stride;
};

// Whether rows of d values share no memory: each stride at least the extent of
// all dimensions of smaller stride.  Strides lie in [0, 2^31].
template <int N> bool rows_apart(int32_t d, Dim (&dims)[N]) {
    std::sort(dims, dims + N, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    int64_t extent = d;
    for (const Dim &dim : dims) {
        if (dim.count <= 1)
            continue;
        if (dim.stride < extent)
            return false;
        extent += dim.stride * (std::min(dim.count, kMaxRows) - 1);   // past 2^31 no stride reaches it
    }
    return true;
}

// A written operand: its rows may not share memory.
pam_status_t check_written(const void *data, const pam_heads_t &h, const char *name, int64_t tokens, int32_t d) {
    PAM_TRY(check_heads(data, h, name, tokens));
    Dim dims[] = {{tokens, h.stride_token}, {h.heads, h.stride_head}};
    return rows_apart(d, dims) ? PAM_SUCCESS : invalid(name, ": rows of a written operand overlap");
}

pam_status_t check_cache(const void *data, const pam_cache_t &c, const char *name, bool must_have_data) {
    if (c.type != PAM_TYPE_F32 && c.type != PAM_TYPE_BF16)
        return invalid(name, ": type must be PAM_TYPE_F32 or PAM_TYPE_BF16");
    if (c.heads < 1 || c.page_size < 1 || c.pages < 0)
        return invalid(name, ": heads and page_size must be at least 1, pages at least 0");
    if (c.pages > kMaxRows / c.page_size)
        return invalid(name, ": pages * page_size must be below 2^31");
    if (c.stride_page < 0 || c.stride_slot < 0 || c.stride_head < 0 || c.stride_page > kMaxStride ||
        c.stride_slot > kMaxStride || c.stride_head > kMaxStride)
        return invalid(name, ": stride out of range");
    if (must_have_data && c.pages > 0 && data == nullptr)
        return invalid(name, ": data is NULL");
    return PAM_SUCCESS;
}

// A cache that is written.
pam_status_t check_written_cache(const void *data, const pam_cache_t &c, const char *name, int64_t tokens, int32_t d) {
    PAM_TRY(check_cache(data, c, name, tokens > 0));
    Dim dims[] = {{c.pages, c.stride_page}, {c.page_size, c.stride_slot}, {c.heads, c.stride_head}};
    return rows_apart(d, dims) ? PAM_SUCCESS : invalid(name, ": slots of a written cache overlap");
}

pam_status_t check_dim(int64_t tokens, int32_t d, float eps) {
    if (tokens < 0)
        return invalid("tokens must be >= 0");
    if (d < 2 || d > PAM_MAX_HEAD_DIM || d % 2 != 0)
        return invalid("d must be even and in [2, 256]");
    if (!(eps >= 0.0f) || !std::isfinite(eps))
        return invalid("eps must be finite and >= 0");
    return PAM_SUCCESS;
}

template <typename A> pam_status_t check_rotation(const A &a) {
    const pam_rotation_t &r = a.rotation;
    if (r.rot < 0 || r.rot > a.d || r.rot % 2 != 0)
        return invalid("rot must be even and in [0, d]");
    if (r.rows < 0 || r.rows > kMaxRows)
        return invalid("the rotation's rows must be in [0, 2^31)");
    if (a.tokens > 0 && r.rot > 0 && (a.positions == nullptr || (r.rows > 0 && (a.cos == nullptr || a.sin == nullptr))))
        return invalid("positions, cos and sin must be non-NULL");
    return PAM_SUCCESS;
}

template <typename P, typename A> void set_common(P &p, const A &a) {
    const bool turns = a.rotation.rot > 0;
    p.tokens = a.tokens;
    p.d = a.d;
    p.eps = a.eps;
    p.rot = a.rotation.rot;
    p.interleaved = turns && a.rotation.interleaved != 0;
    p.positions = turns ? a.positions : nullptr;
    p.cos = turns ? a.cos : nullptr;
    p.sin = turns ? a.sin : nullptr;
    p.rows = turns ? a.rotation.rows : 0;
}

pam_status_t check_rows(int64_t tokens, int64_t heads) {
    if (tokens > kMaxHeadRows / heads)
        return invalid("tokens times heads must be at most 2^25");
    return PAM_SUCCESS;
}

pamk::HeadPart &add_part(pamk::HeadRowsParams &p, const void *data, const pam_heads_t &in, const float *weight,
                         bool rotate) {
    pamk::HeadPart &part = p.part[p.parts++];
    part = pamk::HeadPart{};
    part.in = data;
    part.weight = weight;
    part.in_token = (uint32_t)in.stride_token;
    part.in_head = (uint32_t)in.stride_head;
    part.heads = (uint32_t)in.heads;
    pamk::fast_divisor(part.heads, part.heads_mul, part.heads_shift);
    part.rotate = rotate;
    return part;
}

void to_heads(pamk::HeadPart &part, void *data, const pam_heads_t &out) {
    part.out = data;
    part.out_token = (uint32_t)out.stride_token;
    part.out_head = (uint32_t)out.stride_head;
    part.out_bf16 = is_bf16(out.type);
}

void to_cache(pamk::HeadPart &part, void *data, const pam_cache_t &c) {
    part.out = data;
    part.out_token = (uint32_t)c.stride_page;
    part.out_slot = (uint32_t)c.stride_slot;
    part.out_head = (uint32_t)c.stride_head;
    part.out_bf16 = is_bf16(c.type);
    part.paged = 1;
}

// Workgroups, and partial rows, of the two parts of a gradient: the budget
// shared in proportion to the rows.
void grad_budget(int64_t q_rows, int64_t k_rows, int (&most)[2]) {
    const double all = (double)std::max<int64_t>(q_rows + k_rows, 1);
    most[0] = std::max(1, (int)(pamk::kHeadGradGroups * ((double)q_rows / all)));
    most[1] = std::max(1, (int)(pamk::kHeadGradGroups * ((double)k_rows / all)));
}

// How an attention call is cut.
enum class Form { whole, split, tiles };
struct AttentionPlan {
    Form form;
    int lanes;        // lanes a key in the kernels for few rows
    int rows, row_blocks;
    bool fine;        // few rows: waves of 16 keys
    int splits, split_keys;
    int64_t units;
    int64_t slab;     // units of one round of launches
    size_t scores, stats, partial;   // workspace bytes of a slab
    size_t bytes() const { return scores + stats + partial; }
};

// Workspace of one round of launches, about: tiles of 512 x 4 rows of 8 heads over 32768
// keys of 128 take 5.51 ms in rounds of 512 MiB, 5.75 of 128, 5.53 in one of 2 GiB.
constexpr int64_t kSlabBytes = (int64_t)512 << 20;

AttentionPlan attention_plan(int32_t d, int32_t q_heads, int32_t kv_heads, bool bf16, int32_t batch, int32_t max_q,
                             int32_t max_kv) {
    AttentionPlan a{};
    const int per = bf16 ? 8 : 4;
    a.lanes = 4;
    while (a.lanes * per < d)
        a.lanes *= 2;
    const int64_t rows = std::max<int64_t>((int64_t)max_q * (q_heads / kv_heads), 1);
    const int64_t heads = (int64_t)batch * kv_heads;

    // Few rows a unit, or tiles: by the time of each, in microseconds for MACs in
    // millions, fitted to 70 calls.  A tile's waves are few and each long (chunk of
    // 42 tokens over 291 keys of 256: 149 us as tiles, 48 with few rows), but
    // two to three times as fast where they fill the chip (512 x 4 heads over 4096
    // keys of 128: 675 us, 1384 with few rows).
    const int64_t blocks = ceil_div(rows, 8), each = ceil_div(rows, blocks);
    const int few_rows = (int)(each <= 4 ? each : each <= 6 ? 6 : 8);
    const double macs = 2e-6 * (double)d * (double)heads * (double)max_kv;
    const double few_us = 15.0 + macs * (double)(blocks * few_rows) / 12.0;
    const double tile_us = 50.0 + 0.3 * d + macs * (double)(ceil_div(rows, 64) * 64) / 22.0;
    const bool tiled = tile_us < few_us;
    if (tiled) {
        // 128 rows a unit where that leaves two rounds of score tiles, four
        // workgroups a compute unit; else 64, which waste less.  Over 4096 keys of
        // 128 x 8 heads, 512 x 4 rows a head: 653 us, in units of 64 762; 256 x 4
        // rows: 343 and 418.  Heads of 64 differ little (415 and 403 us), and the
        // limit is on the safe side: 128 x 4 rows, 1024 tiles, 195 us in units of
        // 128, 232 of 64.
        const int64_t tiles = heads * ceil_div(rows, 128) * ceil_div(max_kv, 128);
        a.rows = rows > 64 && tiles >= 2048 ? 128 : 64;
    } else {
        a.rows = few_rows;
    }
    a.row_blocks = (int)ceil_div(rows, a.rows);
    a.units = a.slab = heads * a.row_blocks;
    a.splits = 1;
    // Waves of 16 keys where waves of 64 would leave half of the 1024 SIMDs without
    // one (1000 keys x 8 heads of 128: 20.5 -> 16.4 us; 15006 keys x 4 units of 6 rows
    // of 256, 940 waves of 64: 39 us, in waves of 16 52).
    a.fine = a.units * ceil_div(max_kv, 64) <= 512;
    // One launch for short contexts (32 of 256 keys, 8 heads of 64 in float32: 7.7 us,
    // split 13.4; not of 1000: 35 in 16 waves, 21), and where the units fill the chip
    // and their scores fit in half of LDS, so that two are resident (64 sequences of
    // 1000 keys, 8 heads of 64: 41 us, split 50; 32 of 1024, 8 heads of 128 x 4 rows in
    // bfloat16: 37 and 40; 16 of them, half the units: 36 and 29).  Few units of 4
    // rows over 256 keys would be faster split (8 units of 128: 21.5 and 15.7), more
    // keys than fit in half of LDS sometimes in one launch (2048: 55.9, split 61.5).
    const int64_t lds = pamk::whole_lds(max_kv, a.rows, a.lanes, bf16, a.fine);
    const bool whole = (max_kv <= 256 && lds <= pamk::kWholeLds) || (a.units >= 256 && lds <= pamk::kWholeLds / 2);
    a.form = tiled ? Form::tiles : whole ? Form::whole : Form::split;
    if (a.form == Form::whole || a.units == 0)
        return a;
    if (a.form == Form::tiles) {
        const int64_t keys = ceil_div(std::max(max_kv, 1), 128) * 128;
        a.slab = std::min(a.units, std::max<int64_t>(kSlabBytes / (keys * a.rows * (int64_t)sizeof(float)), 1));
        // The values' workgroups fill the chip's 4096 waves; a split adds up at
        // most 256 keys one after the other, which bounds the error of its sums (of
        // 512: relative errors of 1.2e-6, three times that of short sums).
        const int64_t columns = d > 64 ? ceil_div(d, 128) : 1;
        const int64_t waves = (a.rows / 64) * (d > 64 ? 2 : 1);
        const int64_t per = ceil_div(keys * a.slab * columns * waves, 4096);
        a.split_keys = (int)std::min<int64_t>(std::max<int64_t>(ceil_div(per, 128) * 128, 128), 256);
    } else {
        // About 1024 workgroups, of 256 to 1024 keys; of 64 in waves of 16.  Short
        // splits cost a launch's start and a partial sum each (8 heads of 128 x 4 rows
        // in bfloat16, 16 sequences of 8192 keys in splits of 128, 256, 512, 1024 and
        // 2048: 195, 143, 129, 130, 125 us), long ones leave the chip empty (one sequence
        // of 32768 keys: 59, 42, 40, 44, 71).
        const int64_t keys = ceil_div((int64_t)max_kv * a.units, 1024);
        a.split_keys = (int)std::min<int64_t>(std::max<int64_t>(ceil_div(keys, 256) * 256, 256), 1024);
        if (a.fine)
            a.split_keys = 64;
    }
    a.splits = (int)ceil_div(std::max(max_kv, 1), a.split_keys);
    if (a.form == Form::split) {
        // Rounds of equal size: max_kv may be the whole reach of a table of short
        // sequences (128 of up to 1024 keys, 8 heads x 4 rows, a reach of 131072:
        // 2310 MiB and 321 us at once, 464 MiB and 338 us in five rounds; of up to
        // 8192 keys 827 us either way).
        const int64_t unit = (int64_t)a.splits * a.rows * (a.split_keys + d) * (int64_t)sizeof(float);
        const int64_t rounds = ceil_div(a.units, std::max<int64_t>(kSlabBytes / unit, 1));
        a.slab = ceil_div(a.units, rounds);
    }
    const int64_t parts = a.slab * a.splits;
    const int64_t stats = parts * (a.form == Form::tiles ? a.split_keys / 128 : 1) * 2 * a.rows;
    a.scores = (size_t)(parts * a.split_keys * a.rows) * sizeof(float);
    a.stats = (size_t)ceil_div(stats, 4) * 16;
    a.partial = a.form == Form::tiles && a.splits == 1 ? 0 : (size_t)(parts * a.rows * d) * sizeof(float);
    return a;
}

pam_status_t check_attention_sizes(int32_t d, int32_t q_heads, int32_t kv_heads, int32_t batch, int32_t max_q,
                                   int32_t max_kv) {
    if (d < 8 || d > PAM_MAX_HEAD_DIM || d % 8 != 0)
        return invalid("d must be a multiple of 8 in [8, 256]");
    if (q_heads < 1 || kv_heads < 1 || q_heads % kv_heads != 0)
        return invalid("the query heads must be a multiple of the caches' heads");
    if (batch < 0 || max_q < 0 || max_kv < 0)
        return invalid("batch, max_q and max_kv must be >= 0");
    const int64_t rows = (int64_t)max_q * q_heads;
    if (rows > kMaxRows || (batch > 0 && rows > 0 && max_kv / 256 + 1 > ((int64_t)1 << 40) / batch / rows))
        return invalid("too many rows (batch * max_q * heads * max_kv too large)");
    return PAM_SUCCESS;
}

}  // namespace

extern "C" {

pam_status_t pam_norm_rope(const pam_norm_rope_t *args, hipStream_t stream) {
    if (args == nullptr)
        return invalid("args is NULL");
    const pam_norm_rope_t &a = *args;
    PAM_TRY(check_dim(a.tokens, a.d, a.eps));
    const bool has_q = a.q_in_heads.heads != 0, has_k = a.k_in_heads.heads != 0;
    if (has_q != (a.q_out_heads.heads != 0) || has_k != (a.k_out_heads.heads != 0))
        return invalid("in and out must be given together");
    if (!has_q && !has_k)
        return invalid("neither queries nor keys given");
    if (has_q && has_k && a.q_in_heads.type != a.k_in_heads.type)
        return invalid("q_in and k_in must have one type");
    pamk::HeadRowsParams p{};
    if (has_q) {
        PAM_TRY(check_heads(a.q_in, a.q_in_heads, "q_in", a.tokens));
        PAM_TRY(check_written(a.q_out, a.q_out_heads, "q_out", a.tokens, a.d));
        if (a.q_in_heads.heads != a.q_out_heads.heads)
            return invalid("q_out: another count of heads than the input");
        to_heads(add_part(p, a.q_in, a.q_in_heads, a.q_weight, true), a.q_out, a.q_out_heads);
    }
    if (has_k) {
        PAM_TRY(check_heads(a.k_in, a.k_in_heads, "k_in", a.tokens));
        PAM_TRY(check_written(a.k_out, a.k_out_heads, "k_out", a.tokens, a.d));
        if (a.k_in_heads.heads != a.k_out_heads.heads)
            return invalid("k_out: another count of heads than the input");
        to_heads(add_part(p, a.k_in, a.k_in_heads, a.k_weight, true), a.k_out, a.k_out_heads);
    }
    PAM_TRY(check_rotation(a));
    PAM_TRY(check_rows(a.tokens, (int64_t)a.q_in_heads.heads + a.k_in_heads.heads));
    if (a.tokens == 0)
        return PAM_SUCCESS;
    PAM_TRY(api_check_device());
    set_common(p, a);
    const hipError_t e = pamk::launch_head_rows(is_bf16(has_q ? a.q_in_heads.type : a.k_in_heads.type), p, stream);
    return e == hipSuccess ? PAM_SUCCESS : api_fail_hip(e, "pam_norm_rope kernel launch");
}

pam_status_t pam_norm_rope_grad_workspace_size(int64_t tokens, int32_t d, int32_t q_heads, int32_t k_heads,
                                               size_t *bytes) {
    if (bytes == nullptr)
        return invalid("bytes is NULL");
    PAM_TRY(check_dim(tokens, d, 0.0f));
    if (q_heads < 0 || k_heads < 0 || (q_heads == 0 && k_heads == 0))
        return invalid("heads must be >= 0, and one of them positive");
    PAM_TRY(check_rows(tokens, (int64_t)q_heads + k_heads));
    int most[2];
    grad_budget(tokens * q_heads, tokens * k_heads, most);
    const int64_t rows = std::min<int64_t>(tokens * q_heads, most[0]) + std::min<int64_t>(tokens * k_heads, most[1]);
    *bytes = (size_t)ceil_div(rows * d, 4) * 16;
    return PAM_SUCCESS;
}

pam_status_t pam_norm_rope_grad(const pam_norm_rope_grad_t *args, hipStream_t stream) {
    if (args == nullptr)
        return invalid("args is NULL");
    const pam_norm_rope_grad_t &a = *args;
    PAM_TRY(check_dim(a.tokens, a.d, a.eps));
    struct Side {
        const void *x, *dz;
        void *dx;
        const pam_heads_t &x_heads, &dz_heads, &dx_heads;
        const float *weight;
        float *dweight;
        const char *names[3];
    };
    const Side sides[] = {{a.q_in, a.dq_out, a.dq_in, a.q_in_heads, a.dq_out_heads, a.dq_in_heads, a.q_weight,
                           a.dq_weight, {"q_in", "dq_out", "dq_in"}},
                          {a.k_in, a.dk_out, a.dk_in, a.k_in_heads, a.dk_out_heads, a.dk_in_heads, a.k_weight,
                           a.dk_weight, {"k_in", "dk_out", "dk_in"}}};
    if (a.q_in_heads.heads == 0 && a.k_in_heads.heads == 0)
        return invalid("neither queries nor keys given");
    pamk::HeadGradParams p{};
    const pam_type_t type = a.q_in_heads.heads != 0 ? a.q_in_heads.type : a.k_in_heads.type;
    bool weights = false;
    int64_t rows[2] = {0, 0};
    for (int i = 0; i < 2; ++i) {
        const Side &s = sides[i];
        const bool given = s.x_heads.heads != 0;
        if (given != (s.dz_heads.heads != 0) || given != (s.dx_heads.heads != 0))
            return invalid("an input and its two gradients must be given together");
        if ((s.weight == nullptr) != (s.dweight == nullptr))
            return invalid("a weight and its gradient must be given together");
        if (!given) {
            if (s.weight != nullptr)
                return invalid("a weight without its input");
            continue;
        }
        PAM_TRY(check_heads(s.x, s.x_heads, s.names[0], a.tokens));
        PAM_TRY(check_heads(s.dz, s.dz_heads, s.names[1], a.tokens));
        PAM_TRY(check_written(s.dx, s.dx_heads, s.names[2], a.tokens, a.d));
        if (s.x_heads.heads != s.dz_heads.heads || s.x_heads.heads != s.dx_heads.heads)
            return invalid(s.names[0], ": another count of heads than its gradients");
        if (s.x_heads.type != type || s.dz_heads.type != type || s.dx_heads.type != type)
            return invalid("inputs and gradients must have one type");
        pamk::HeadGradPart &part = p.part[i];
        part.x = s.x;
        part.dz = s.dz;
        part.dx = s.dx;
        part.weight = s.weight;
        part.dweight = s.dweight;
        part.x_token = (uint32_t)s.x_heads.stride_token;
        part.x_head = (uint32_t)s.x_heads.stride_head;
        part.dz_token = (uint32_t)s.dz_heads.stride_token;
        part.dz_head = (uint32_t)s.dz_heads.stride_head;
        part.dx_token = (uint32_t)s.dx_heads.stride_token;
        part.dx_head = (uint32_t)s.dx_heads.stride_head;
        part.heads = (uint32_t)s.x_heads.heads;
        pamk::fast_divisor(part.heads, part.heads_mul, part.heads_shift);
        rows[i] = a.tokens * s.x_heads.heads;
        weights = weights || s.weight != nullptr;
    }
    PAM_TRY(check_rotation(a));
    PAM_TRY(check_rows(a.tokens, (int64_t)a.q_in_heads.heads + a.k_in_heads.heads));
    if (a.tokens == 0 && !weights)
        return PAM_SUCCESS;
    set_common(p, a);
    int most[2];
    grad_budget(rows[0], rows[1], most);
    for (int i = 0; i < 2; ++i)
        p.part[i].groups = pamk::head_grad_groups(is_bf16(type), rows[i], a.d, p.rot, most[i]);
    if (weights && a.tokens > 0) {
        const int64_t need = (int64_t)(p.part[0].groups + p.part[1].groups) * a.d * (int64_t)sizeof(float);
        if (a.workspace == nullptr || a.workspace_bytes < need)
            return invalid("workspace is NULL or smaller than pam_norm_rope_grad_workspace_size says");
        if ((reinterpret_cast<uintptr_t>(a.workspace) & 15u) != 0)
            return invalid("workspace must be 16-byte aligned");
        p.part[0].partial = static_cast<float *>(a.workspace);
        p.part[1].partial = p.part[0].partial + (int64_t)p.part[0].groups * a.d;
    }
    PAM_TRY(api_check_device());
    const hipError_t e = pamk::launch_head_grad(is_bf16(type), p, stream);
    return e == hipSuccess ? PAM_SUCCESS : api_fail_hip(e, "pam_norm_rope_grad kernel launch");
}

pam_status_t pam_append_kv(const pam_append_kv_t *args, hipStream_t stream) {
    if (args == nullptr)
        return invalid("args is NULL");
    const pam_append_kv_t &a = *args;
    PAM_TRY(check_dim(a.tokens, a.d, a.eps));
    const bool has_q = a.q_in_heads.heads != 0;
    if (has_q != (a.q_out_heads.heads != 0))
        return invalid("q_in and q_out must be given together");
    const pam_cache_t &kc = a.k_cache_layout, &vc = a.v_cache_layout;
    PAM_TRY(check_heads(a.k, a.k_heads, "k", a.tokens));
    PAM_TRY(check_heads(a.v, a.v_heads, "v", a.tokens));
    PAM_TRY(check_written_cache(a.k_cache, kc, "k_cache", a.tokens, a.d));
    PAM_TRY(check_written_cache(a.v_cache, vc, "v_cache", a.tokens, a.d));
    if (a.k_heads.type != a.v_heads.type || (has_q && a.q_in_heads.type != a.k_heads.type))
        return invalid("k, v and q_in must have one type");
    if (a.k_heads.heads != kc.heads || a.v_heads.heads != vc.heads || a.k_heads.heads != a.v_heads.heads)
        return invalid("k, v and the caches must have one count of heads");
    if (kc.pages != vc.pages || kc.page_size != vc.page_size)
        return invalid("the caches must have one count and size of pages");
    PAM_TRY(check_rotation(a));
    pamk::HeadRowsParams p{};
    to_cache(add_part(p, a.k, a.k_heads, a.k_weight, true), a.k_cache, kc);
    to_cache(add_part(p, a.v, a.v_heads, nullptr, false), a.v_cache, vc);
    if (has_q) {
        PAM_TRY(check_heads(a.q_in, a.q_in_heads, "q_in", a.tokens));
        PAM_TRY(check_written(a.q_out, a.q_out_heads, "q_out", a.tokens, a.d));
        if (a.q_in_heads.heads != a.q_out_heads.heads)
            return invalid("q_out: another count of heads than the input");
        to_heads(add_part(p, a.q_in, a.q_in_heads, a.q_weight, true), a.q_out, a.q_out_heads);
    }
    PAM_TRY(check_rows(a.tokens, (int64_t)a.k_heads.heads + a.v_heads.heads + a.q_in_heads.heads));
    if (a.tokens > 0 && a.slots == nullptr)
        return invalid("slots is NULL");
    if (a.tokens == 0)
        return PAM_SUCCESS;
    PAM_TRY(api_check_device());
    set_common(p, a);
    p.slots = a.slots;
    p.page_size = (uint32_t)kc.page_size;
    pamk::fast_divisor(p.page_size, p.page_mul, p.page_shift);
    p.cache_slots = kc.pages * kc.page_size;
    const hipError_t e = pamk::launch_head_rows(is_bf16(a.k_heads.type), p, stream);
    return e == hipSuccess ? PAM_SUCCESS : api_fail_hip(e, "pam_append_kv kernel launch");
}

pam_status_t pam_paged_attention_workspace_size(int32_t d, int32_t q_heads, int32_t kv_heads, pam_type_t kv_type,
                                                int32_t batch, int32_t max_q, int32_t max_kv, size_t *bytes) {
    if (bytes == nullptr)
        return invalid("bytes is NULL");
    if (kv_type != PAM_TYPE_F32 && kv_type != PAM_TYPE_BF16)
        return invalid("kv_type must be PAM_TYPE_F32 or PAM_TYPE_BF16");
    PAM_TRY(check_attention_sizes(d, q_heads, kv_heads, batch, max_q, max_kv));
    *bytes = attention_plan(d, q_heads, kv_heads, is_bf16(kv_type), batch, max_q, max_kv).bytes();
    return PAM_SUCCESS;
}

pam_status_t pam_paged_attention(const pam_paged_attention_t *args, hipStream_t stream) {
    if (args == nullptr)
        return invalid("args is NULL");
    const pam_paged_attention_t &s = *args;
    const pam_cache_t &kc = s.k_cache_layout, &vc = s.v_cache_layout;
    if (s.tokens < 0)
        return invalid("tokens must be >= 0");
    PAM_TRY(check_attention_sizes(s.d, s.q_heads.heads, kc.heads, s.batch, s.max_q, s.max_kv));
    PAM_TRY(check_heads(s.q, s.q_heads, "q", s.tokens));
    PAM_TRY(check_written(s.out, s.out_heads, "out", s.tokens, s.d));
    if (s.out_heads.type != PAM_TYPE_F32)
        return invalid("out: must be PAM_TYPE_F32");
    if (s.out_heads.heads != s.q_heads.heads)
        return invalid("out: another count of heads than q");
    PAM_TRY(check_cache(s.k_cache, kc, "k_cache", true));
    PAM_TRY(check_cache(s.v_cache, vc, "v_cache", true));
    if (kc.type != vc.type || kc.heads != vc.heads || kc.pages != vc.pages || kc.page_size != vc.page_size)
        return invalid("the caches must agree in type, heads, pages and page_size");
    if (s.table_width < 0 || s.table_stride < s.table_width || s.table_stride > kMaxStride)
        return invalid("table_stride must be at least table_width, which must be >= 0");
    if (s.max_kv > (int64_t)s.table_width * kc.page_size)
        return invalid("max_kv must be at most table_width * page_size");
    if (s.q_starts == nullptr && s.tokens < s.batch)
        return invalid("without q_starts there must be one token a sequence");
    if (s.window < 0)
        return invalid("window must be >= 0");
    if (!std::isfinite(s.scale))
        return invalid("scale must be finite");
    if (s.batch == 0 || s.tokens == 0 || s.max_q == 0)
        return PAM_SUCCESS;
    if (s.kv_lens == nullptr || (s.max_kv > 0 && s.table == nullptr))
        return invalid("kv_lens and table must be non-NULL");
    const bool bf16 = is_bf16(kc.type);
    const AttentionPlan plan = attention_plan(s.d, s.q_heads.heads, kc.heads, bf16, s.batch, s.max_q, s.max_kv);
    const int64_t most_groups = plan.slab * plan.splits * (plan.form == Form::tiles ? std::max(plan.split_keys / 128, 2) : 1);
    // The one launch has up to 1024 threads a workgroup, all others at most 256.
    const int64_t whole_threads =
        plan.form == Form::whole ? plan.units * pamk::whole_waves(s.max_kv, plan.rows, plan.fine) * 64 : 0;
    if (plan.units > kMaxLaunchGroups || most_groups > kMaxLaunchGroups || whole_threads > kMaxLaunchThreads)
        return invalid("too many workgroups (batch * heads * rows * keys too large)");
    if (plan.bytes() > 0) {
        if (s.workspace == nullptr || s.workspace_bytes < 0 || (size_t)s.workspace_bytes < plan.bytes())
            return invalid("workspace is NULL or smaller than pam_paged_attention_workspace_size says");
        if ((reinterpret_cast<uintptr_t>(s.workspace) & 15u) != 0)
            return invalid("workspace must be 16-byte aligned");
    }
    PAM_TRY(api_check_device());

    pamk::AttentionParams p{};
    p.q = s.q;
    p.q_token = s.q_heads.stride_token;
    p.q_head = s.q_heads.stride_head;
    p.q_bf16 = is_bf16(s.q_heads.type);
    p.k = {s.k_cache, kc.stride_page, kc.stride_slot, kc.stride_head, kc.pages};
    p.v = {s.v_cache, vc.stride_page, vc.stride_slot, vc.stride_head, vc.pages};
    p.page_size = (uint32_t)kc.page_size;
    pamk::fast_divisor(p.page_size, p.page_mul, p.page_shift);
    p.q_starts = s.q_starts;
    p.kv_lens = s.kv_lens;
    p.table = s.table;
    p.table_stride = s.table_stride;
    p.out = s.out;
    p.out_token = s.out_heads.stride_token;
    p.out_head = s.out_heads.stride_head;
    p.tokens = s.tokens;
    p.batch = s.batch;
    p.kv_heads = kc.heads;
    p.group = s.q_heads.heads / kc.heads;
    p.d = s.d;
    p.max_q = s.q_starts == nullptr ? 1 : s.max_q;
    p.max_kv = s.max_kv;
    p.causal = s.causal;
    p.window = s.window;
    p.scale = (float)((double)s.scale * 1.4426950408889634);
    p.rows = plan.rows;
    p.fine = plan.fine;
    p.row_blocks = plan.row_blocks;
    pamk::fast_divisor((uint32_t)p.row_blocks, p.blocks_mul, p.blocks_shift);
    pamk::fast_divisor((uint32_t)p.kv_heads, p.heads_mul, p.heads_shift);
    pamk::fast_divisor((uint32_t)p.group, p.group_mul, p.group_shift);
    p.splits = plan.splits;
    p.split_keys = plan.split_keys;
    p.scores = static_cast<float *>(s.workspace);
    p.stats = reinterpret_cast<float *>(static_cast<char *>(s.workspace) + plan.scores);
    p.partial = reinterpret_cast<float *>(static_cast<char *>(s.workspace) + plan.scores + plan.stats);

    if (plan.partial == 0)
        p.partial = nullptr;

    hipError_t e = hipSuccess;
    if (plan.form == Form::whole) {
        e = pamk::launch_attention_whole(bf16, plan.lanes, p, stream);
    } else {
        const bool tiles = plan.form == Form::tiles;
        for (int64_t first = 0; first < plan.units && e == hipSuccess; first += plan.slab) {
            const int units = (int)std::min(plan.slab, plan.units - first);
            p.first_unit = (int32_t)first;
            e = tiles ? pamk::launch_tile_scores(bf16, p, units, stream)
                      : pamk::launch_attention_scores(bf16, plan.lanes, p, units, stream);
            if (e == hipSuccess)
                e = tiles ? pamk::launch_tile_values(bf16, p, units, stream)
                          : pamk::launch_attention_values(bf16, plan.lanes, p, units, stream);
            if (e == hipSuccess && p.partial != nullptr)
                e = pamk::launch_attention_join(p, units, stream);
        }
    }
    return e == hipSuccess ? PAM_SUCCESS : api_fail_hip(e, "pam_paged_attention kernel launch");
}

}  // extern "C"
