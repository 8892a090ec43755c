// The host layer of the attention-side operators (pam_attention_api.cpp) with
// its kernel launches replaced by records of what would be launched, so that
// the form and cut of a call can be tested through the C ABI without a GPU.
// Built by attention_probe.py.

#include <string>

#include "pam_attention_api.cpp"

namespace {
// form: 1 one launch, 2 scores and 3 values of few rows, 4 join, 5 scores and 6
// values of tiles, 7 norm and rotation or append, 8 the gradient's.
struct Launch {
    int64_t form, bf16, lanes, rows, fine, units, first_unit, splits, split_keys, threads;
};
constexpr int kMost = 64;
Launch g_launches[kMost];
int g_count = 0;
std::string g_error;

hipError_t record(int64_t form, bool bf16, int lanes, const pamk::AttentionParams &p, int64_t units, int64_t threads) {
    if (g_count < kMost)
        g_launches[g_count] = {form, bf16, lanes, p.rows, p.fine, units, p.first_unit, p.splits, p.split_keys, threads};
    ++g_count;
    return hipSuccess;
}
int64_t all_units(const pamk::AttentionParams &p) { return (int64_t)p.batch * p.kv_heads * p.row_blocks; }
hipError_t record_heads(int64_t form) {
    if (g_count < kMost)
        g_launches[g_count] = {form};
    ++g_count;
    return hipSuccess;
}
}  // namespace

namespace pamk {
pam_status_t api_fail(pam_status_t status, const char *message) {
    g_error = message;
    return status;
}
pam_status_t api_fail_hip(hipError_t, const char *what) { return api_fail(PAM_ERROR_LAUNCH, what); }
pam_status_t api_check_device() { return PAM_SUCCESS; }
hipError_t launch_head_rows(bool, const HeadRowsParams &, hipStream_t) { return record_heads(7); }
hipError_t launch_head_grad(bool, const HeadGradParams &, hipStream_t) { return record_heads(8); }
int head_grad_groups(bool, int64_t, int, int, int most) { return most; }
hipError_t launch_attention_whole(bool bf16, int lanes, const AttentionParams &p, hipStream_t) {
    return record(1, bf16, lanes, p, all_units(p), whole_waves(p.max_kv, p.rows, p.fine) * 64);
}
hipError_t launch_attention_scores(bool bf16, int lanes, const AttentionParams &p, int units, hipStream_t) {
    return record(2, bf16, lanes, p, units, 256);
}
hipError_t launch_attention_values(bool bf16, int lanes, const AttentionParams &p, int units, hipStream_t) {
    return record(3, bf16, lanes, p, units, 256);
}
hipError_t launch_attention_join(const AttentionParams &p, int units, hipStream_t) {
    return record(4, false, 0, p, units, 256);
}
hipError_t launch_tile_scores(bool bf16, const AttentionParams &p, int units, hipStream_t) {
    return record(5, bf16, 0, p, units, 0);
}
hipError_t launch_tile_values(bool bf16, const AttentionParams &p, int units, hipStream_t) {
    return record(6, bf16, 0, p, units, 0);
}
}  // namespace pamk

extern "C" {
// The launches since the last call (at most kMost of them), and their count.
int probe_take(Launch *out) {
    const int n = g_count;
    for (int i = 0; i < kMost; ++i)
        out[i] = g_launches[i];
    g_count = 0;
    return n;
}
const char *probe_error() { return g_error.c_str(); }
}
