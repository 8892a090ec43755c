// C ABI of the layer-and-step side (pam_training.h): argument validation, the
// cut of a call into launches, workspaces.  The arithmetic lives in the product
// kernels (pam_epilogue.h) and in pam_training.hip.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <new>
#include <vector>

#include "pam_internal.h"
#include "pam_training.h"
#include "pam_training_internal.h"

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

constexpr int64_t kMaxDim = 0x7FFFFFFF;
constexpr int64_t kMaxTiled = kMaxDim - 1023;  // rows and columns, with what a last tile has beyond them
constexpr int64_t kMaxLd = (int64_t)1 << 31;   // times a count below 2^31: offsets stay inside int64

bool type_ok(pam_type_t t) { return t == PAM_TYPE_F32 || t == PAM_TYPE_BF16; }
int64_t size_of(pam_type_t t) { return t == PAM_TYPE_BF16 ? 2 : 4; }
bool activation_ok(pam_activation_t a) { return a >= PAM_ACT_NONE && a <= PAM_ACT_SILU; }

// Memory that a call reads or writes.
struct Range {
    uintptr_t begin, end;
    bool written;
};

Range range_of(const void *data, int64_t bytes, bool written) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(data);
    return {at, at + (uintptr_t)(data == nullptr ? 0 : bytes), written};
}
// rows, cols below 2^31, ld at most 2^31: the last element's place is below 2^62 + 2^31,
// its byte may not be; no memory is that large.
Range rows_of(const void *data, int64_t rows, int64_t cols, int64_t ld, int64_t size, bool written) {
    const int64_t elements = rows > 0 && cols > 0 ? (rows - 1) * ld + cols : 0;
    return range_of(data, std::min(elements, (int64_t)1 << 56) * size, written);
}

bool overlap(const Range &a, const Range &b) { return a.begin < b.end && b.begin < a.end; }

// A leading dimension: rows of a matrix that is written share no memory.
pam_status_t check_ld(const char *name, const void *data, int64_t ld, int64_t n) {
    if (data == nullptr)
        return PAM_SUCCESS;
    if (ld < std::max<int64_t>(1, n) || ld > kMaxLd)
        return invalid(name, ": the leading dimension must be in [n, 2^31]");
    return PAM_SUCCESS;
}

pam_status_t check_workspace(const void *workspace, int64_t bytes, size_t need) {
    if (need == 0)
        return PAM_SUCCESS;
    if (bytes < 0 || (size_t)bytes < need)
        return invalid("the workspace is too small");
    if (workspace == nullptr)
        return invalid("workspace is NULL");
    if ((reinterpret_cast<uintptr_t>(workspace) & 15u) != 0)
        return invalid("the workspace must be 16-byte aligned");
    return PAM_SUCCESS;
}

// ---------------------------------------------------------------------------
// The activations' gradient
// ---------------------------------------------------------------------------

// How the rows are cut.  Few rows: one band, whose sums need no second launch (2.5
// us), with as few lanes a row, down to kGradLanes, that a thread has at most
// kGradFew rows.  Otherwise 64 lanes a row (or the row's) and bands for about
// kGradGroups workgroups with at least kGradRows rows a thread.
constexpr int64_t kGradGroups = 1024;
constexpr int64_t kGradRows = 4;
constexpr int64_t kGradFew = 8;
constexpr int kGradLanes = 8;

struct GradCut {
    int lanes;
    int64_t band, bands;
};

GradCut grad_cut(int64_t m, int64_t n, int values) {
    int most = 1;
    while (most < 64 && (int64_t)most * values < n)
        most *= 2;
    for (int lanes = most; lanes >= std::min(most, kGradLanes); lanes /= 2) {
        const int64_t at_once = pamk::kGradThreads / lanes;
        if (m <= at_once * kGradFew)
            return {lanes, ceil_div(m, at_once) * at_once, 1};
    }
    const int64_t at_once = pamk::kGradThreads / most;
    const int64_t groups = ceil_div(n, (int64_t)most * values);
    const int64_t bands = std::max<int64_t>(1, std::min(ceil_div(kGradGroups, groups), m / (at_once * kGradRows)));
    const int64_t band = ceil_div(ceil_div(m, bands), at_once) * at_once;
    return {most, band, ceil_div(m, band)};
}

// ---------------------------------------------------------------------------
// Many tensors at once
// ---------------------------------------------------------------------------

// By beginning: ascending runs merged, one with the next, until one is left (lists
// of tensors in ascending order are a few runs; spare is as long as ranges).
void sort_runs(std::vector<Range> &ranges, std::vector<Range> &spare) {
    auto before = [](const Range &a, const Range &b) { return a.begin < b.begin; };
    spare.resize(ranges.size());
    for (size_t runs = 2; runs > 1;) {
        runs = 0;
        auto from = ranges.begin();
        auto to = spare.begin();
        while (from != ranges.end()) {
            const auto middle = std::is_sorted_until(from, ranges.end(), before);
            const auto end = std::is_sorted_until(middle, ranges.end(), before);
            to = std::merge(from, middle, middle, end, to, before);
            from = end;
            ++runs;
        }
        ranges.swap(spare);
    }
}

constexpr int64_t kMaxTensors = 1 << 20;
constexpr int64_t kMaxValues = (int64_t)1 << 38;   // 1 TB of float32

pam_status_t check_tensors(const pam_step_tensor_t *tensors, int64_t count, int64_t *total) {
    *total = 0;
    if (count < 0 || count > kMaxTensors)
        return invalid("count must be in [0, 2^20]");
    if (count > 0 && tensors == nullptr)
        return invalid("tensors is NULL");
    for (int64_t j = 0; j < count; ++j) {
        if (tensors[j].n < 0 || tensors[j].n > kMaxValues - *total)
            return invalid("n must be >= 0, and at most 2^38 in all");
        *total += tensors[j].n;
    }
    return PAM_SUCCESS;
}

// Values a workgroup of the norm takes: at most kNormPartials of them in all
// (but one a tensor at least), in steps of 1024.
constexpr int64_t kNormPartials = 2048;
int64_t norm_chunk(int64_t total) { return 1024 * std::max<int64_t>(1, ceil_div(total, 1024 * kNormPartials)); }

int64_t norm_groups(const pam_step_tensor_t *tensors, int64_t count, int64_t chunk) {
    int64_t groups = 0;
    for (int64_t j = 0; j < count; ++j)
        groups += ceil_div(tensors[j].n, chunk);
    return groups;
}

// Values a workgroup of the step takes.  32-bit states: one vector a thread (188 M
// parameters 857 us; with two and four 918 and 908).  8-bit ones: a block a wave
// where that makes few workgroups, else four (558 and 535 us; of 0.9 M 7.0 and 8.4).
constexpr int64_t kStepGroups = 1024;

int64_t step_chunk(int64_t total, bool bytes) {
    const int64_t least = pamk::kStepThreads * 4;
    return bytes && total >= 4 * least * kStepGroups ? 4 * least : least;
}

}  // namespace

extern "C" {

pam_status_t pam_linear_workspace_size(int64_t m, int64_t n, int64_t k, size_t *bytes) {
    if (bytes == nullptr)
        return invalid("bytes is NULL");
    return pamk::api_linear_workspace_size(m, n, k, bytes);
}

pam_status_t pam_linear(const pam_linear_t *args, hipStream_t stream) {
    if (args == nullptr)
        return invalid("args is NULL");
    const pam_linear_t &a = *args;
    if (!type_ok(a.type) || !type_ok(a.out_type))
        return invalid("type and out_type must be PAM_TYPE_F32 or PAM_TYPE_BF16");
    if (!activation_ok(a.activation))
        return invalid("unknown activation");
    if (a.mantissa_bits < 0 || a.mantissa_bits > 23)
        return invalid("mantissa_bits must be in [0, 23]");
    const bool bf16 = a.type == PAM_TYPE_BF16;
    if (bf16 && a.mantissa_bits != 23)
        return invalid("bfloat16 operands take mantissa_bits 23");
    if (a.m < 0 || a.n < 0 || a.k < 0 || a.m > kMaxTiled || a.n > kMaxTiled || a.k > kMaxDim)
        return invalid("m and n must be in [0, 2^31 - 1024], k in [0, 2^31)");
    PAM_TRY(check_ld("residual", a.residual, a.ldr, a.n));
    PAM_TRY(check_ld("z", a.z, a.ldz, a.n));
    PAM_TRY(check_ld("y", a.y, a.ldy, a.n));
    if (a.ldx < 0 || a.ldw < 0 || a.ldx > kMaxLd || a.ldw > kMaxLd)
        return invalid("leading dimensions must be in [0, 2^31]");
    const int64_t in = size_of(a.type), out = size_of(a.out_type);
    const Range y = rows_of(a.y, a.m, a.n, a.ldy, out, true), z = rows_of(a.z, a.m, a.n, a.ldz, out, true);
    const Range read[] = {rows_of(a.x, a.m, a.k, a.ldx, in, false), rows_of(a.w, a.n, a.k, a.ldw, in, false),
                          range_of(a.bias, a.n * 4, false), rows_of(a.residual, a.m, a.n, a.ldr, out, false)};
    size_t need = 0;
    PAM_TRY(pamk::api_linear_workspace_size(a.m, a.n, a.k, &need));
    const Range ws = range_of(a.workspace, (int64_t)need, true);
    if (overlap(y, z) || overlap(y, ws) || overlap(z, ws))
        return invalid("y, z and the workspace overlap");
    for (int i = 0; i < 4; ++i) {
        const bool in_place = i == 3 && a.residual == a.y && a.ldr == a.ldy;
        if ((overlap(read[i], y) && !in_place) || overlap(read[i], z) || overlap(read[i], ws))
            return invalid("an output or the workspace overlaps an input");
    }
    const pamk::Epilogue epi{a.bias, a.residual, a.y, a.z, a.ldr, a.ldy, a.ldz, a.activation,
                             a.out_type == PAM_TYPE_BF16};
    return pamk::api_linear(a.m, a.n, a.k, a.x, a.ldx, a.w, a.ldw, epi, bf16, 23 - a.mantissa_bits, a.workspace,
                            (size_t)std::max<int64_t>(a.workspace_bytes, 0), stream);
}

pam_status_t pam_activation_grad_workspace_size(int64_t m, int64_t n, size_t *bytes) {
    if (bytes == nullptr)
        return invalid("bytes is NULL");
    *bytes = 0;
    if (m < 0 || n < 0 || m > kMaxDim || n > kMaxTiled)
        return invalid("m must be in [0, 2^31), n in [0, 2^31 - 1024]");
    if (m == 0 || n == 0)
        return PAM_SUCCESS;
    for (const int values : {4, 8}) {   // either type
        const GradCut cut = grad_cut(m, n, values);
        if (cut.bands > 1)
            *bytes = std::max(*bytes, (size_t)(cut.bands * n) * sizeof(float));
    }
    return PAM_SUCCESS;
}

pam_status_t pam_activation_grad(const pam_activation_grad_t *args, hipStream_t stream) {
    if (args == nullptr)
        return invalid("args is NULL");
    const pam_activation_grad_t &a = *args;
    if (!type_ok(a.type) || !type_ok(a.z_type))
        return invalid("type and z_type must be PAM_TYPE_F32 or PAM_TYPE_BF16");
    if (!activation_ok(a.activation))
        return invalid("unknown activation");
    if (a.m < 0 || a.n < 0 || a.m > kMaxDim || a.n > kMaxTiled)
        return invalid("m must be in [0, 2^31), n in [0, 2^31 - 1024]");
    const bool none = a.activation == PAM_ACT_NONE;
    if (none && (a.z != nullptr || a.dz != nullptr))
        return invalid("without an activation there is no z, and dz is dy");
    if (a.m > 0 && a.n > 0 && (a.dy == nullptr || (!none && a.z == nullptr)))
        return invalid("dy or z is NULL");
    PAM_TRY(check_ld("dy", a.dy, a.lddy, a.n));
    PAM_TRY(check_ld("z", a.z, a.ldz, a.n));
    PAM_TRY(check_ld("dz", a.dz, a.lddz, a.n));
    size_t need = 0;
    PAM_TRY(pam_activation_grad_workspace_size(a.m, a.n, &need));
    if (a.db == nullptr)
        need = 0;
    PAM_TRY(check_workspace(a.workspace, a.workspace_bytes, need));
    const int64_t each = size_of(a.type);
    const Range dy = rows_of(a.dy, a.m, a.n, a.lddy, each, false),
                z = rows_of(a.z, a.m, a.n, a.ldz, size_of(a.z_type), false),
                dz = rows_of(a.dz, a.m, a.n, a.lddz, each, true), db = range_of(a.db, a.n * 4, true),
                ws = range_of(a.workspace, (int64_t)need, true);
    const bool on_dy = a.dz == a.dy && a.lddz == a.lddy, on_z = a.dz == a.z && a.lddz == a.ldz && a.type == a.z_type;
    if ((overlap(dz, dy) && !on_dy) || (overlap(dz, z) && !on_z))
        return invalid("dz overlaps an input");
    for (const Range &r : {dy, z, dz})
        if (overlap(r, db) || overlap(r, ws))
            return invalid("db or the workspace overlaps another operand");
    if (overlap(db, ws))
        return invalid("db and the workspace overlap");
    if (a.n == 0 || (a.db == nullptr && (a.m == 0 || none)))
        return PAM_SUCCESS;
    PAM_TRY(api_check_device());
    const bool bf16 = a.type == PAM_TYPE_BF16;
    pamk::GradParams p{};
    p.dy = a.dy;
    p.z = a.z;
    p.dz = a.dz;
    p.db = a.db;
    p.partial = static_cast<float *>(a.workspace);
    p.lddy = a.lddy;
    p.ldz = a.ldz;
    p.lddz = a.lddz;
    p.m = a.m;
    p.n = (int32_t)a.n;
    p.activation = a.activation;
    p.streaming = a.m * a.n * (each * (a.dz != nullptr ? 2 : 1) + (none ? 0 : size_of(a.z_type))) > pamk::kCacheBytes;
    p.apart = a.dz == nullptr || (a.dz != a.dy && a.dz != a.z);
    const GradCut cut = grad_cut(std::max<int64_t>(a.m, 1), a.n, pamk::grad_values(bf16));
    p.lanes = cut.lanes;
    p.band = (int32_t)std::min<int64_t>(cut.band, kMaxDim);
    p.bands = (int32_t)cut.bands;
    const hipError_t e = pamk::launch_activation_grad(bf16, a.z_type == PAM_TYPE_BF16, p, stream);
    return e == hipSuccess ? PAM_SUCCESS : api_fail_hip(e, "activation gradient launch");
}

pam_status_t pam_grad_norm_workspace_size(const pam_step_tensor_t *tensors, int64_t count, size_t *bytes) {
    if (bytes == nullptr)
        return invalid("bytes is NULL");
    *bytes = 0;
    int64_t total;
    PAM_TRY(check_tensors(tensors, count, &total));
    *bytes = (size_t)std::max<int64_t>(1, norm_groups(tensors, count, norm_chunk(total))) * sizeof(double);
    return PAM_SUCCESS;
}

pam_status_t pam_grad_norm(const pam_step_tensor_t *tensors, int64_t count, pam_type_t grad_type, float *norm,
                           void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    if (!type_ok(grad_type))
        return invalid("grad_type must be PAM_TYPE_F32 or PAM_TYPE_BF16");
    int64_t total;
    PAM_TRY(check_tensors(tensors, count, &total));
    const int64_t chunk = norm_chunk(total), groups = norm_groups(tensors, count, chunk);
    if (groups > pamk::kMostStepGroups)
        return invalid("too many values");
    if (norm == nullptr)
        return invalid("norm is NULL");
    PAM_TRY(check_workspace(workspace, workspace_bytes, (size_t)std::max<int64_t>(1, groups) * sizeof(double)));
    const Range written[] = {range_of(norm, 4, true), range_of(workspace, groups * (int64_t)sizeof(double), true)};
    if (overlap(written[0], written[1]))
        return invalid("norm and the workspace overlap");
    for (int64_t j = 0; j < count; ++j) {
        const pam_step_tensor_t &t = tensors[j];
        if (t.n > 0 && t.g == nullptr)
            return invalid("a tensor's g is NULL");
        const Range g = range_of(t.g, t.n * size_of(grad_type), false);
        if (overlap(g, written[0]) || overlap(g, written[1]))
            return invalid("norm or the workspace overlaps a gradient");
    }
    PAM_TRY(api_check_device());
    double *partial = static_cast<double *>(workspace);
    int64_t done = 0;
    for (int64_t j = 0; j < count;) {
        pamk::NormParams p{};
        p.chunk = chunk;
        p.grad_bf16 = grad_type == PAM_TYPE_BF16;
        p.streaming = total * size_of(grad_type) > pamk::kCacheBytes;
        p.partial = partial + done;
        uint32_t here = 0;
        for (; j < count && p.count < pamk::kNormTensors; ++j) {
            if (tensors[j].n == 0)
                continue;
            p.g[p.count] = tensors[j].g;
            p.n[p.count] = tensors[j].n;
            p.first[p.count++] = here;
            here += (uint32_t)ceil_div(tensors[j].n, chunk);
        }
        if (here == 0)
            break;
        const hipError_t e = pamk::launch_grad_squares(here, p, stream);
        if (e != hipSuccess)
            return api_fail_hip(e, "gradient norm launch");
        done += here;
    }
    const hipError_t e = pamk::launch_grad_norm(partial, done, norm, stream);
    return e == hipSuccess ? PAM_SUCCESS : api_fail_hip(e, "gradient norm launch");
}

pam_status_t pam_adamw_step(const pam_step_tensor_t *tensors, int64_t count, const pam_adamw_t *args,
                            hipStream_t stream) {
    if (args == nullptr)
        return invalid("args is NULL");
    const pam_adamw_t &a = *args;
    if (!type_ok(a.grad_type))
        return invalid("grad_type must be PAM_TYPE_F32 or PAM_TYPE_BF16");
    if (a.state_bits != 8 && a.state_bits != 32)
        return invalid("state_bits must be 8 or 32");
    if (a.step < 1 && a.step_device == nullptr)
        return invalid("step must be at least 1");
    if (!(a.beta1 >= 0.0 && a.beta1 < 1.0 && a.beta2 >= 0.0 && a.beta2 < 1.0))
        return invalid("the betas must be in [0, 1)");
    if (!(a.lr >= 0.0 && a.eps >= 0.0 && a.weight_decay >= 0.0))
        return invalid("lr, eps and weight_decay must be >= 0");
    if (a.norm != nullptr && !(a.max_norm > 0.0))
        return invalid("max_norm must be > 0");
    int64_t total;
    PAM_TRY(check_tensors(tensors, count, &total));
    const int64_t chunk = step_chunk(total, a.state_bits == 8);
    const bool bytes = a.state_bits == 8;
    int64_t groups = 0;
    for (int64_t j = 0; j < count; ++j) {
        const pam_step_tensor_t &t = tensors[j];
        if (t.n == 0)
            continue;
        if (t.p == nullptr || t.g == nullptr || t.avg == nullptr || t.sq == nullptr)
            return invalid("a tensor's p, g, avg or sq is NULL");
        if (bytes != (t.avg_scale != nullptr) || bytes != (t.sq_scale != nullptr))
            return invalid("8-bit states have scales, 32-bit ones none");
        groups += ceil_div(t.n, chunk);
    }
    if (groups > pamk::kMostStepGroups)
        return invalid("too many values");
    std::vector<Range> ranges, spare;
    try {
        ranges.reserve((size_t)count * 7 + 2);   // what is pushed below
        spare.resize((size_t)count * 7 + 2);
    } catch (const std::bad_alloc &) {
        return invalid("no host memory to compare the tensors' addresses");
    }
    if (a.norm != nullptr)
        ranges.push_back(range_of(a.norm, 4, false));
    if (a.step_device != nullptr)
        ranges.push_back(range_of(a.step_device, 8, false));
    // List by list: tensors made one after the other lie in ascending order.
    auto list = [&](auto data, auto size, bool written) {
        for (int64_t j = 0; j < count; ++j)
            if (tensors[j].n > 0 && data(tensors[j]) != nullptr)
                ranges.push_back(range_of(data(tensors[j]), size(tensors[j].n), written));
    };
    const int64_t grad = size_of(a.grad_type), state = bytes ? 1 : 4;
    auto scales = [](int64_t n) { return ceil_div(n, PAM_STATE_BLOCK) * 4; };
    list([](auto &t) -> const void * { return t.p; }, [](int64_t n) { return n * 4; }, true);
    list([](auto &t) -> const void * { return t.g; }, [&](int64_t n) { return n * grad; }, false);
    list([](auto &t) -> const void * { return t.avg; }, [&](int64_t n) { return n * state; }, true);
    list([](auto &t) -> const void * { return t.sq; }, [&](int64_t n) { return n * state; }, true);
    list([](auto &t) -> const void * { return t.avg_scale; }, scales, true);
    list([](auto &t) -> const void * { return t.sq_scale; }, scales, true);
    list([](auto &t) -> const void * { return t.copy; }, [](int64_t n) { return n * 2; }, true);
    sort_runs(ranges, spare);
    uintptr_t written = 0, read = 0;   // ends of the ranges so far
    for (const Range &r : ranges) {
        if (r.begin < written || (r.written && r.begin < read))
            return invalid("tensors of a step share memory");
        (r.written ? written : read) = std::max(r.written ? written : read, r.end);
    }
    if (groups == 0)
        return PAM_SUCCESS;
    PAM_TRY(api_check_device());

    pamk::StepParams p{};
    p.chunk = chunk;
    p.norm = a.norm;
    p.max_norm = (float)a.max_norm;
    p.step_device = a.step_device;
    p.step = a.step;
    p.log_beta1 = std::log(a.beta1);   // -inf for 0: 1 - beta^t is 1
    p.log_beta2 = std::log(a.beta2);
    const double t = (double)a.step;
    p.step_size = (float)(a.step_device != nullptr ? a.lr : a.lr / -std::expm1(t * p.log_beta1));
    p.sq_factor = (float)(a.step_device != nullptr ? 1.0 : 1.0 / std::sqrt(-std::expm1(t * p.log_beta2)));
    p.keep = (float)(1.0 - a.lr * a.weight_decay);
    p.beta1 = (float)a.beta1;
    p.rest1 = (float)(1.0 - a.beta1);
    p.beta2 = (float)a.beta2;
    p.rest2 = (float)(1.0 - a.beta2);
    p.eps = (float)a.eps;
    p.seed = a.seed;
    p.grad_bf16 = a.grad_type == PAM_TYPE_BF16;
    p.streaming = total * (4 + size_of(a.grad_type) + (bytes ? 2 : 8)) > pamk::kCacheBytes;
    for (int64_t j = 0; j < count;) {
        p.count = 0;
        p.tensor0 = (int32_t)j;
        uint32_t here = 0;
        // An empty tensor keeps its place, for the tensors' numbers: no workgroup is its own.
        for (; j < count && p.count < pamk::kStepTensors; ++j) {
            p.tensor[p.count] = tensors[j];
            p.first[p.count++] = here;
            here += (uint32_t)ceil_div(tensors[j].n, chunk);
        }
        if (here == 0)
            continue;
        const hipError_t e = pamk::launch_adamw(a.state_bits, here, p, stream);
        if (e != hipSuccess)
            return api_fail_hip(e, "optimizer step launch");
    }
    return PAM_SUCCESS;
}

}  // extern "C"
